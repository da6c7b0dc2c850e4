// What the forward and the backward pass of the attention share: the list of work, tensor maps, tiles of rows, the products'
// wrappers and the accesses to tensor memory.
//
// A tile of queries is kt tokens of one sequence times the G heads that share a key and value head: row = token * G + head,
// kt = 128 / G. All its rows read the same keys, so that groups of heads cost nothing, and a few tokens of many heads fill a
// tile. Rows G * kt..127 do not exist where G does not divide 128.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "ones_attention.h"
#include "ones_mma.cuh"
#include "ones_train_internal.h"

namespace ones {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kRows = 128;                      // of a tile: queries (tokens x heads) or keys
constexpr int kHalfTile = kRows * 128;          // bytes of 64 columns of a tile: rows of 128 bytes, swizzled
constexpr int kKeys = 128;                      // keys of a tile

// A piece of work: tokens from `first` on of the sequence [begin, end). In the list of queries `first` starts one or two tiles of
// queries, in the list of keys a tile of keys. begin < 0: tokens [first, end) belong to no sequence and get zeros.
struct Item {
    int first, begin, end, cost;
};

// In the workspace, one for each list: how many items there are, then the items, those with the most work first.
struct PlanHead {
    int count;
    int covered[2];  // tokens [0], .., [1] - 1 belong to sequences
    int pad;
};
struct PlanArgs {
    const int64_t* offsets;
    int tokens, sequences;
    int step[2];      // tokens of an item of list 0 (queries) and 1 (keys)
    int tile[2];      // what the cost goes by
    int* start;       // [sequences + 1]
    int* prefix[2];   // [sequences + 1] items before each sequence
    Item* items[2];
    PlanHead* head;   // [2]
    unsigned* zero;   // words that are set to 0, by the first list's block
    int zeros;
};

inline int64_t items_at_most(int64_t tokens, int64_t sequences, int64_t step) {
    return tokens / step + (sequences < tokens ? sequences : tokens) + 2;
}
cudaError_t launch_plan(const PlanArgs& a, int lists, cudaStream_t stream);

// A tensor of heads as boxes of 64 values x `heads_box` heads x `tokens_box` tokens; what lies outside it reads as zeros.
cudaError_t make_heads_map(CUtensorMap* out, const ones_heads& h, int dim, int tokens, int heads_box, int tokens_box, bool f16);

// ---- device side ----

// D(tmem) (+)= A(tmem) * B(shared) for 16-bit operands: two neighbouring values along K in a 32-bit column.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}

// 32 columns of the warp's 32 lanes, without waiting: the values are there after tmem_wait on the same registers.
__device__ __forceinline__ void tmem_fetch(uint32_t addr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
}
// Waits for all fetches of the warp. The registers pass through, so that nothing that uses them moves before the wait.
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                   "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                   "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {"
        "%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two columns of each lane, for what two warps of the same lanes tell each other.
__device__ __forceinline__ void tmem_put(uint32_t addr, float a, float b) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x2.b32 [%0], {%1, %2};\n\ttcgen05.wait::st.sync.aligned;" ::"r"(addr), "f"(a), "f"(b) : "memory");
}
__device__ __forceinline__ float2 tmem_get(uint32_t addr) {
    float2 r;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x2.b32 {%0, %1}, [%2];\n\ttcgen05.wait::ld.sync.aligned;" : "=f"(r.x), "=f"(r.y) : "r"(addr) : "memory");
    return r;
}

__device__ __forceinline__ float exp2_of(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <bool F16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    uint32_t r;
    if constexpr (F16)
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ uint32_t attend_desc(bool f16, bool bmn, int width) {
    const uint32_t type = f16 ? 0u : 1u;
    return (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)bmn << 16) | ((uint32_t)(width / 8) << 17) | ((128u / 16) << 24);
}

// D = A * B^T over `steps` x 16 columns of two tiles in shared memory, both with rows of columns. Run by one thread.
__device__ __forceinline__ void product_rows(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, int steps) {
    const uint64_t da = operand_desc(a, false, 0), db = operand_desc(b, false, 0);
    for (int i = 0; i < steps; ++i) {
        const uint64_t off = (uint64_t)((i & 3) * 32 + (i >> 2) * kHalfTile) >> 4;
        mma_f16<1>(d, da + off, db + off, idesc, i != 0);
    }
}
// D (+)= A * B: A in tensor memory (16 rows of B take 8 columns of it; the second half of them starts at `a_second`), B a tile of
// 128 rows in shared memory, taken along its rows. Run by one thread.
__device__ __forceinline__ void product_tmem(uint32_t d, uint32_t a, uint32_t a_second, uint32_t b, uint32_t idesc, bool add) {
    const uint64_t db = operand_desc(b, true, kHalfTile);
#pragma unroll
    for (int i = 0; i < 8; ++i) mma_ts(d, (i < 4 ? a : a_second - 32) + 8 * i, db + (uint64_t)(i * (2048 >> 4)), idesc, add || i != 0);
}

// Zeros in rows [from, 128) of a tile, by a whole warp, before the tensor core reads it: what lies behind a sequence may hold
// anything, and 0 * NaN is NaN.
template <int HALVES>
__device__ __forceinline__ void clear_rows(uint8_t* tile, int from, int lane) {
    for (int i = from * 8 + lane; i < kRows * 8; i += 32) {
#pragma unroll
        for (int h = 0; h < HALVES; ++h) *reinterpret_cast<uint4*>(tile + h * kHalfTile + i * 16) = make_uint4(0, 0, 0, 0);
    }
    asm volatile("fence.proxy.async;" ::: "memory");
    __syncwarp();
}

// Where a row of `dim` values goes.
struct HeadsOut {
    uint16_t* p;
    int64_t token, head;
    int wide;  // rows start on 16-byte boundaries
};
__host__ inline HeadsOut heads_out(const ones_heads& h, int tokens) {
    return {static_cast<uint16_t*>(h.d_data), h.token, h.head,
            aligned(h.d_data, 16) && (h.heads <= 1 || h.head % 8 == 0) && (tokens <= 1 || h.token % 8 == 0)};
}
// 32 columns of a row, from column c on, as 16 bits.
template <bool F16>
__device__ __forceinline__ void write_columns(uint16_t* row, int c, int dim, bool wide, const float (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
        const uint4 q = make_uint4(pack16<F16>(v[i], v[i + 1]), pack16<F16>(v[i + 2], v[i + 3]), pack16<F16>(v[i + 4], v[i + 5]),
                                   pack16<F16>(v[i + 6], v[i + 7]));
        if (wide && c + i + 8 <= dim) {
            *reinterpret_cast<uint4*>(row + c + i) = q;
        } else {
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + i + j < dim) row[c + i + j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
        }
    }
}

// The items of this block: every gridDim.x-th, to and fro, so that a block that got the larger one of a turn gets the smaller
// one of the next.
__device__ __forceinline__ int64_t work_at(int turn) {
    return (int64_t)turn * gridDim.x + (turn & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
}

__device__ __forceinline__ float total_of(Pair a) { return total(a); }

// What both directions refuse. kv: of each tensor, whether its heads are those of the keys.
struct HeadsOf {
    const ones_heads* h;
    bool keys, out;
};
inline bool bad_counts(int tokens, int sequences, int heads, int kv) {
    return tokens < 0 || tokens >= 1 << 30 || sequences < 0 || sequences > 1 << 22 || heads < 1 || heads > ONES_MAX_HEADS || kv < 1 || heads % kv ||
           heads / kv > kRows;
}
inline size_t rounded(size_t n) { return (n + 255) / 256 * 256; }
int refuse_attention(const HeadsOf* all, int n, const int64_t* offsets, int tokens, int sequences, int dim, float scale, int type);

extern const WaitControl attention_waits, attention_back_waits;

}  // namespace ones
