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
// queries, in the list of keys a tile of keys. begin < 0: tokens [first, end) belong to no sequence and get zeros. slot: the sequence's
// own, below the tokens and the sequences.
struct Item {
    int first, begin, end, slot;
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
    unsigned* zero;   // words that are set to 0, by blocks of their own
    int64_t zeros;
    int lists;
};

// The first row of a tile of queries (token * group + head) that sees a key which lies `behind` tokens behind the tile's first token; far keys
// count as 256 tokens away, where a tile is seen whole or not at all: 2^30 tokens times a group of 128 do not fit 32 bits.
__host__ __device__ inline int first_row(int behind, int group) { return (behind < -256 ? -256 : behind > 256 ? 256 : behind) * group; }

inline int64_t items_at_most(int64_t tokens, int64_t sequences, int64_t step) {
    return tokens / step + (sequences < tokens ? sequences : tokens) + 2;
}
cudaError_t launch_plan(PlanArgs a, int lists, cudaStream_t stream);

// A tensor of heads as boxes of 64 values x `heads_box` heads x `tokens_box` tokens; what lies outside it reads as zeros.
cudaError_t make_heads_map(CUtensorMap* out, const ones_heads& h, int dim, int tokens, int heads_box, int tokens_box, bool f16);

// ---- device side ----

// Operand descriptors differ in their low word only: the tile's place, and what lies between chunks of 64 values (rows taken
// across). Put together where the instruction is issued, they cost one addition each.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_rows(uint32_t at) { return ((at & 0x3FFFF) >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_across(uint32_t at) { return ((at & 0x3FFFF) >> 4) | ((uint32_t)(kHalfTile >> 4) << 16); }
// D(tmem) (+)= A * B for 16-bit operands: both in shared memory, or A in tensor memory, two neighbouring values along K in a
// 32-bit column.
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.u32 p, %4, 0;\n\tmov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "r"(kDescHigh)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.u32 p, %4, 0;\n\tmov.b64 y, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "r"(kDescHigh)
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
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
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

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float log2_of(float x) {
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
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
template <int HALVES>
__device__ __forceinline__ void product_rows(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, int steps) {
    const uint32_t da = desc_rows(a), db = desc_rows(b);
#pragma unroll
    for (int i = 0; i < 4 * HALVES; ++i) {
        const uint32_t off = (uint32_t)((i & 3) * 32 + (i >> 2) * kHalfTile) >> 4;
        if (i < steps) mma_ss(d, da + off, db + off, idesc, i != 0);
    }
}
// D (+)= A * B: A in tensor memory (16 rows of B take 8 columns of it; the second half of them starts at `a_second`), B a tile of
// 128 rows in shared memory, taken along its rows. Run by one thread.
__device__ __forceinline__ void product_tmem(uint32_t d, uint32_t a, uint32_t a_second, uint32_t b, uint32_t idesc, bool add) {
    const uint32_t db = desc_across(b);
#pragma unroll
    for (int i = 0; i < 8; ++i) mma_ts(d, (i < 4 ? a : a_second - 32) + 8 * i, db + i * (2048 >> 4), idesc, add || i != 0);
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
    int wide;  // rows start on 16-byte boundaries, and are pieces of 16 bytes
};
__host__ inline HeadsOut heads_out(const ones_heads& h, int dim, int tokens) {
    return {static_cast<uint16_t*>(h.d_data), h.token, h.head,
            dim % 8 == 0 && aligned(h.d_data, 16) && (h.heads <= 1 || h.head % 8 == 0) && (tokens <= 1 || h.token % 8 == 0)};
}
// The rows that the lanes of a warp own, on their way out: 32 columns at a time as 16 bits. A store of 16 bytes by each lane to its
// own row would touch 32 lines at once, and the cache takes one a cycle: four lanes exchange pieces (through 2 KB of the warp's
// own, or by shuffles where shared memory is full) until each has the same piece of four rows, and write 64 bytes of a row
// together; predicated, since each branch around a store costs 100 cycles. Rows off 16-byte boundaries: 16 lanes exchange words,
// and write a row by 2 bytes (15 heads of 77 values, 16 thousand tokens: 260 us for the forward pass with lanes that write
// their own rows, 114 so).
constexpr int kStageBytesOfWarp = 32 * 64;
struct RowsOut {
    unsigned long long own;   // 0: not there
    unsigned long long to[4];  // of the four lanes
    __device__ __forceinline__ void set(uint16_t* row) {
        own = reinterpret_cast<unsigned long long>(row);
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = __shfl_sync(0xFFFFFFFFu, own, (threadIdx.x & 28) + i);
    }
    // WIDE: rows start on 16-byte boundaries and have a multiple of 8 columns
    template <bool F16, bool WIDE>
    __device__ __forceinline__ void write(int c, int dim, const uint32_t (&o)[32], float factor, uint8_t* stage) const {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 f = split(pair(__uint_as_float(o[2 * i]), __uint_as_float(o[2 * i + 1])) * both(factor));
            w[i] = pack16<F16>(f.x, f.y);
        }
        const int lane = threadIdx.x % 32;
        if constexpr (WIDE) {
            const int at = c + 8 * (lane % 4);
            if (stage) {
                uint4* const s = reinterpret_cast<uint4*>(stage);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * lane + (i ^ (lane >> 1 & 3))] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = (lane & 28) + i;
                    const uint4 q = s[4 * r + (lane % 4 ^ (r >> 1 & 3))];
                    w[4 * i] = q.x, w[4 * i + 1] = q.y, w[4 * i + 2] = q.z, w[4 * i + 3] = q.w;
                }
            } else {
#pragma unroll
                for (int m = 2; m; m >>= 1) {  // piece i of lane l becomes piece l of lane i, for groups of four lanes
                    const bool up = lane & m;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (i & m) continue;
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const uint32_t give = up ? w[4 * i + y] : w[4 * (i | m) + y], got = __shfl_xor_sync(0xFFFFFFFFu, give, m);
                            if (up)
                                w[4 * i + y] = got;
                            else
                                w[4 * (i | m) + y] = got;
                        }
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\t@p st.global.v4.b32 [%0], {%1, %2, %3, %4};\n\t}" ::"l"(to[i] + 2 * at),
                             "r"(w[4 * i]), "r"(w[4 * i + 1]), "r"(w[4 * i + 2]), "r"(w[4 * i + 3]), "r"((uint32_t)(to[i] != 0 && at < dim))
                             : "memory");
            return;
        }
        const int col = c + 2 * (lane % 16);
#pragma unroll
        for (int m = 8; m; m >>= 1) {  // word i of lane l becomes word l of lane i, for the 16 lanes of a half warp
            const bool up = lane & m;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (i & m) continue;
                const uint32_t give = up ? w[i] : w[i | m], got = __shfl_xor_sync(0xFFFFFFFFu, give, m);
                if (up)
                    w[i] = got;
                else
                    w[i | m] = got;
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const unsigned long long at = __shfl_sync(0xFFFFFFFFu, own, (lane & 16) + i);
            asm volatile(
                "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %3, 0;\n\tsetp.ne.u32 q, %4, 0;\n\t@p st.global.b16 [%0], %1;\n\t@q st.global.b16 [%0 + 2], %2;\n\t}" ::"l"(
                    at + 2 * col),
                "h"((uint16_t)w[i]), "h"((uint16_t)(w[i] >> 16)), "r"((uint32_t)(at != 0 && col < dim)), "r"((uint32_t)(at != 0 && col + 1 < dim))
                : "memory");
        }
    }
};

// Zeros in the own row, of tokens that belong to no sequence: rarely run, and so kept small.
__device__ __forceinline__ void write_zeros(uint16_t* row, int dim) {
#pragma unroll 1
    for (int c = 0; row && c < dim; ++c) row[c] = 0;
}

// The items of this block: every gridDim.x-th, to and fro, so that a block that got the larger one of a turn gets the smaller
// one of the next. The first of them are looked up once, by all threads, for all warps: fetched by each warp in its turn they
// cost 1000 cycles apiece, which short items wait for.
constexpr int kListed = 92;
struct Work {
    int first, begin, end, h;  // an item and its head of the keys
    uint32_t slot;
};
constexpr int kHeadBits = 10;  // ONES_MAX_HEADS; a slot has 22
struct WorkList {  // in shared memory
    int4 listed[kListed];
    int turns;
};
__device__ __forceinline__ int4 fetch_work(const Item* items, uint32_t kv, int turn) {
    const uint32_t w = turn * gridDim.x + (turn & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x), i = w / kv;
    const Item a = items[i];
    return make_int4(a.first, a.begin, a.end, (int)(w - i * kv | (uint32_t)a.slot << kHeadBits));
}
// By all threads, before a barrier of the block. Items times heads are below 2^31.
__device__ __forceinline__ void list_work(WorkList& list, const Item* items, const PlanHead* head, int kv) {
    const uint32_t total = (uint32_t)head->count * kv, two = 2 * gridDim.x, pairs = total / two, left = total - pairs * two;
    // of every two turns, the first goes to and the second fro
    const int turns = 2 * pairs + (left > blockIdx.x) + (left > two - 1 - blockIdx.x);
    for (int t = threadIdx.x; t < min(turns, kListed); t += blockDim.x) list.listed[t] = fetch_work(items, kv, t);
    if (threadIdx.x == 0) list.turns = turns;
}
struct Walk {
    const WorkList& list;
    const Item* items;
    int kv, turn = 0;
    Work it = {};
    __device__ __forceinline__ Walk(const WorkList& l, const Item* i, int heads) : list(l), items(i), kv(heads) {}
    __device__ __forceinline__ bool next() {
        if (turn >= list.turns) return false;
        const int4 a = turn < kListed ? list.listed[turn] : fetch_work(items, kv, turn);
        it = {a.x, a.y, a.z, a.w & ((1 << kHeadBits) - 1), (uint32_t)a.w >> kHeadBits};
        ++turn;
        return true;
    }
};

// Slots of a ring (or sets of buffers) by how many were taken before: where the n-th is, and the parity of its barriers' phase.
template <int SLOTS>
struct Slot {
    uint32_t at, parity;
    __device__ __forceinline__ explicit Slot(uint32_t n) : at(n % SLOTS), parity(n / SLOTS & 1) {}
};

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
