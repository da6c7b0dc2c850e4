// The matrix product of the training-step operators: C = A * B^T on 16-bit operands with 32-bit accumulators, where
// what happens to C is a policy (`Epi`), so that a softmax statistic, a gradient of the logits or a polynomial of the
// product leaves the kernel instead of the product itself.
//
// One persistent CTA per SM (CG = 1: tiles of 128 x 128) or pair of CTAs (CG = 2: tiles of 256 x 256, each CTA holds
// 128 rows of A and 128 rows of B, and both tensor cores work on one tile). A ring of kStages boxes of 64 values
// along K is filled by TMA (one thread), consumed by tcgen05.mma (one thread), and two accumulators in tensor memory
// let the epilogue warps work on one tile while the next one is multiplied. A thread of the epilogue owns one row.
//
// A operand is read as rows x K with K contiguous, or (AMN / BMN) as K x rows with the rows contiguous, straight from
// the caller's layout: nothing is transposed beforehand. Sizes need not be multiples of anything: TMA fills what lies
// outside a matrix with zeros, and epilogues skip rows and columns outside C.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "ones_mma.cuh"
#include "ones_train_internal.h"

namespace ones {

constexpr int kSms = 148;  // launch rules reckon with a B200's SMs, so that workspace sizes need no device
constexpr int kTileK = 64;       // values along K per stage: one 128-byte swizzle row
constexpr int kStages = 6;
constexpr int kHalf = 128 * kTileK * 2;  // bytes of one operand's box(es) per stage and CTA
constexpr int kStageBytes = 2 * kHalf;
// Warps of the epilogue: 16 where a tile's way out is what short products wait for (the gradients of the cross entropy:
// 32001 x 777 out of K = 1023 in 98 us with 8 and 86 us with 16, 32000 x 1024 out of K = 10 in 36 and 25 us), 8 where
// each thread needs more registers or little leaves.
template <int WARPS>
constexpr int kMatThreads = 128 + 32 * WARPS;
constexpr int kTurnBytes = 32 * 1024;  // what they have between them to turn rows round
constexpr int kMatSmem = kStages * kStageBytes + kTurnBytes + 1024;

struct MatShape {
    int M, N, K;
    int tiles_m, tiles_n, batch;
    int splits;  // > 1: K is cut into parts, at most so many, each with a C of its own in the place of a matrix of the batch
    int plan_nk; // stages of K that the number of parts goes by (K itself may be shorter); 0: K's own
    int fold;    // 2: A has two terms (a matrix of the batch each) that meet the same B: K runs over it twice
    int sym;     // only tiles on and above the diagonal are computed (C is symmetric)
    const int *live_m, *live_k;  // where M or K is known on the device only (at most the value above)
    int live_times;              // K is so many times what live_k says
    int group;  // row tiles that run through the columns together, so that both operands' tiles are met again in L2
    bool f16;
    int width;         // columns of a tile: 128 * CG, or fewer where N is to be spread evenly (multiple of 16)
    int stage_a, stage_b;  // bytes of the operands' boxes per stage and CTA
};

struct TileAt {
    int b, m, n;
};

__device__ __forceinline__ int tiles_per_matrix(const MatShape& g) {
    return g.sym ? g.tiles_m * (g.tiles_m + 1) / 2 : g.tiles_m * g.tiles_n;
}

__device__ __forceinline__ TileAt tile_at(const MatShape& g, int t, int per) {
    TileAt r;
    r.b = t / per;
    int p = t - r.b * per;
    if (g.sym) {
        int i = 0;
        while (p >= g.tiles_m - i) {
            p -= g.tiles_m - i;
            ++i;
        }
        r.m = i;
        r.n = i + p;
    } else {
        const int block = g.group * g.tiles_n, k = p / block, first = k * g.group;
        const int rows = min(g.tiles_m - first, g.group);
        p -= k * block;
        r.n = p / rows;
        r.m = first + (p - r.n * rows);
    }
    return r;
}

// ---- the parts that the warps play ----

// Ring of stages: where a warp stands in it.
struct Ring {
    uint32_t base, full, empty;  // stages; barriers
    int s = 0;
    uint32_t ph = 0;
    __device__ __forceinline__ void next() {
        if (++s == kStages) s = 0, ph ^= 1;
    }
};

// How an operand lies in memory: with K contiguous, with its rows contiguous (mn), or symmetric with only the blocks on
// and above the diagonal there (upper; blocks of BN): what lies below it is then taken from above, with the rows contiguous.
enum class Lie { k, mn, upper };
struct View {
    const CUtensorMap *k, *mn;
    Lie lie;
    int tile;  // the block of rows, for Lie::upper
    template <int BN>
    __device__ __forceinline__ bool is_mn(int kb) const {
        return lie == Lie::mn || (lie == Lie::upper && kb * kTileK / BN < tile);
    }
};

template <int CG>
__device__ __forceinline__ void fill_operand(uint32_t at, const View& v, int row, int kb, int z, uint32_t bar) {
    if (v.is_mn<128 * CG>(kb)) {
        tma_load<CG>(at, v.mn, row, kb * kTileK, z, bar);
        tma_load<CG>(at + kHalf / 2, v.mn, row + 64, kb * kTileK, z, bar);
    } else {
        tma_load<CG>(at, v.k, kb * kTileK, row, z, bar);
    }
}

// Fills the stages of one tile: K from stage k0 to k1, rows am of A and bn of B. Run by a whole warp; false: gave up.
template <int CG>
__device__ __forceinline__ bool fill_tile(Ring& r, const View& va, const View& vb, int am, int bn, int z, int k0, int k1, uint32_t rank,
                                          uint32_t full_at, uint32_t bytes = kStageBytes, int nk_one = 1 << 30) {
    for (int k = k0; k < k1; ++k) {
        const int term = k >= nk_one, kb = term ? k - nk_one : k;
        if (!warp_wait(r.empty + 8 * r.s, r.ph ^ 1)) return false;
        const uint32_t a = r.base + r.s * kStageBytes, bar = full_at + 8 * r.s;
        if (elect_one()) {
            if (rank == 0) bar_expect(r.full + 8 * r.s, CG * bytes);
            fill_operand<CG>(a, va, am, kb, z + term, bar);
            fill_operand<CG>(a + kHalf, vb, bn, kb, z, bar);
        }
        __syncwarp();
        r.next();
    }
    return true;
}

__host__ __device__ inline uint32_t instruction_desc(int cg, bool f16, bool amn, bool bmn, int width) {
    const uint32_t type = f16 ? 0u : 1u;
    return (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)amn << 15) | ((uint32_t)bmn << 16) |
           ((uint32_t)(width / 8) << 17) | ((uint32_t)(128 * cg / 16) << 24);
}

// Multiplies the nk stages of one tile into the accumulator at `acc` and lets barrier `done` know when that is through.
template <int CG>
__device__ __forceinline__ bool multiply_tile(Ring& r, uint32_t acc, int nk, const View& va, const View& vb, bool f16, uint32_t done,
                                              int width = 128 * CG) {
    const uint64_t a_k = operand_desc(r.base, false, kHalf / 2), a_mn = operand_desc(r.base, true, kHalf / 2);
    const uint64_t to_b = kHalf >> 4;
    for (int k = 0; k < nk; ++k) {
        if (!warp_wait(r.full + 8 * r.s, r.ph)) return false;
        mma_fence_after();
        const bool amn = va.is_mn<128 * CG>(k), bmn = vb.is_mn<128 * CG>(k);
        const uint64_t off = (uint64_t)(r.s * (kStageBytes >> 4));
        const uint64_t a = (amn ? a_mn : a_k) + off, b = (bmn ? a_mn : a_k) + off + to_b;
        const uint64_t step_a = (amn ? 2048 : 32) >> 4, step_b = (bmn ? 2048 : 32) >> 4;  // 16 values along K
        const uint32_t idesc = instruction_desc(CG, f16, amn, bmn, width);
        if (elect_one()) {
#pragma unroll
            for (int i = 0; i < kTileK / 16; ++i) mma_f16<CG>(acc, a + i * step_a, b + i * step_b, idesc, (k | i) != 0);
            mma_commit<CG>(r.empty + 8 * r.s);
        }
        __syncwarp();
        r.next();
    }
    if (elect_one()) mma_commit<CG>(done);
    __syncwarp();
    return true;
}

// What a block (or pair) sets up before its first tile, and gives back after its last.
struct Bench {
    uint32_t base, full, empty, done, free_, tmem;
};
struct BenchShared {
    uint64_t full[kStages], empty[kStages], done[2], free_[2];
    uint32_t tmem;
};
template <int CG, int WARPS>
__device__ __forceinline__ Bench set_up(BenchShared& s, uint8_t* smem_raw, int warp) {
    Bench w;
    w.base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    w.full = smem_u32(s.full), w.empty = smem_u32(s.empty), w.done = smem_u32(s.done), w.free_ = smem_u32(s.free_);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            bar_init(w.full + 8 * i, 1);
            bar_init(w.empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(w.done + 8 * i, 1);
            bar_init(w.free_ + 8 * i, WARPS * CG);
        }
        bar_init_done();
    }
    if (warp == 2) tmem_alloc<CG>(smem_u32(&s.tmem), 256 * CG);  // two accumulators of 128 * CG columns
    mma_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_all();
    mma_fence_after();
    w.tmem = s.tmem;
    return w;
}
template <int CG>
__device__ __forceinline__ void clear_up(const Bench& w, int warp, bool ok) {
    if (!ok) let_copies_end();
    __syncwarp();
    mma_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_all();
    mma_fence_after();
    if (warp == 2) tmem_free<CG>(w.tmem, 256 * CG);
    if constexpr (CG == 2) cluster_sync_all();  // neither CTA leaves while the other still gives its half back
}

// ---- what epilogues share ----

struct Half16 {  // two 16-bit values of the run-time type, in one word
    static __device__ __forceinline__ uint32_t pack(float lo, float hi, bool f16) {
        if (f16) {
            __half2 h = __floats2half2_rn(lo, hi);
            return *reinterpret_cast<uint32_t*>(&h);
        }
        __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<uint32_t*>(&h);
    }
};

// A thread has one row's values; stored like that, a warp's store would touch 32 rows at once. They go through shared
// memory instead, 64 (16 warps) or 128 bytes (8 warps) of a row at a time, the 16-byte chunks of a row permuted by the row
// so that neither side meets a bank twice, and leave with 4 or 8 lanes on one row.
template <int WARPS>
struct Turn {
    static constexpr int kBytes = kTurnBytes / WARPS / 32;                   // of a row
    static constexpr int kHalves = kBytes / 2, kWords = kBytes / 4;          // values of 16 and of 32 bits in them
    static constexpr int kChunks = kBytes / 16, kRowsAtOnce = 32 / kChunks;  // a warp's 16-byte accesses cover so many rows
    uint8_t* at;  // this warp's own 32 rows
    int lane;

    static __device__ __forceinline__ int place(int row, int c) { return kChunks == 8 ? c ^ (row & 7) : c ^ (row >> 1 & 3); }
    __device__ __forceinline__ uint4& chunk(int row, int c) const { return *reinterpret_cast<uint4*>(at + row * kBytes + (place(row, c) << 4)); }
    // the row and chunk of this lane's i-th access, of kChunks, to all 32 rows
    __device__ __forceinline__ int row_of(int i) const { return kRowsAtOnce * i + lane / kChunks; }
    __device__ __forceinline__ int chunk_of() const { return lane % kChunks; }

    __device__ __forceinline__ void put16(const float (&v)[kHalves], bool f16) const {
        __syncwarp();
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            chunk(lane, c) = make_uint4(Half16::pack(v[8 * c], v[8 * c + 1], f16), Half16::pack(v[8 * c + 2], v[8 * c + 3], f16),
                                        Half16::pack(v[8 * c + 4], v[8 * c + 5], f16), Half16::pack(v[8 * c + 6], v[8 * c + 7], f16));
        __syncwarp();
    }
    __device__ __forceinline__ void put32(const float (&v)[kWords]) const {
        __syncwarp();
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            chunk(lane, c) = make_uint4(__float_as_uint(v[4 * c]), __float_as_uint(v[4 * c + 1]), __float_as_uint(v[4 * c + 2]),
                                        __float_as_uint(v[4 * c + 3]));
        __syncwarp();
    }
    // A 16-bit or 32-bit value of what was put.
    __device__ __forceinline__ uint16_t half_at(int row, int c) const {
        return *reinterpret_cast<const uint16_t*>(at + row * kBytes + (place(row, c >> 3) << 4) + (c & 7) * 2);
    }
    __device__ __forceinline__ uint32_t word_at(int row, int c) const {
        return *reinterpret_cast<const uint32_t*>(at + row * kBytes + (place(row, c >> 2) << 4) + (c & 3) * 4);
    }

    // The calling thread's values as 16 bits, and with them the warp's 32 rows from row0, into columns from `col` of
    // `out` (row 0's first value), as far as they lie inside rows x cols. wide: rows start on 16-byte boundaries.
    // What is written is read first, all of it or of eight rows, since the compiler cannot tell the two memories apart.
    __device__ __forceinline__ void write16(float (&v)[kHalves], bool f16, uint16_t* out, int64_t ld, int row0, int col, int rows, int cols,
                                            bool wide) const {
        if (wide) {
            put16(v, f16);
            const int c = chunk_of(), left = cols - (col + 8 * c);
            uint16_t* p = out + (int64_t)(row0 + row_of(0)) * ld + col + 8 * c;
            uint4 q[kChunks];
#pragma unroll
            for (int i = 0; i < kChunks; ++i) q[i] = chunk(row_of(i), c);
#pragma unroll
            for (int i = 0; i < kChunks; ++i, p += kRowsAtOnce * ld) {
                if (row0 + row_of(i) >= rows || left <= 0) continue;
                if (left >= 8) {
                    *reinterpret_cast<uint4*>(p) = q[i];
                } else {
                    for (int j = 0; j < left; ++j) p[j] = half_at(row_of(i), 8 * c + j);
                }
            }
        } else {
            // Two values at a time: a row that starts on an odd 2-byte place is put one value further to the left, so that
            // its pairs lie on 4-byte boundaries on both sides; its first value goes by itself.
            constexpr int kLanes = kWords, kStep = 32 / kLanes;  // lanes on a row, rows at once
            const int n = min(32, rows - row0), width = min(kHalves, cols - col);
            uint16_t* p = out + (int64_t)row0 * ld + col;
            const bool odd = (reinterpret_cast<uintptr_t>(p + lane * ld) >> 1) & 1;
            if (odd && lane < n) p[lane * ld] = (uint16_t)Half16::pack(v[0], 0.f, f16);
#pragma unroll
            for (int i = 0; i < kHalves - 1; ++i) v[i] = odd ? v[i + 1] : v[i];
            put16(v, f16);
            p += lane / kLanes * ld;
#pragma unroll 1
            for (int r = lane / kLanes; r - lane / kLanes < n; r += 8 * kStep) {
                uint32_t q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = word_at((r + j * kStep) & 31, lane % kLanes);
#pragma unroll
                for (int j = 0; j < 8; ++j, p += kStep * ld) {
                    if (r + j * kStep >= n) continue;
                    const int c = 2 * (lane % kLanes) + ((int)(reinterpret_cast<uintptr_t>(p) >> 1) & 1);
                    if (c + 1 < width)
                        *reinterpret_cast<uint32_t*>(p + c) = q[j];
                    else if (c < width)
                        p[c] = (uint16_t)q[j];
                }
            }
        }
    }
    // The same as 32 bits.
    __device__ __forceinline__ void write32(const float (&v)[kWords], float* out, int64_t ld, int row0, int col, int rows, int cols, bool wide) const {
        put32(v);
        if (wide) {
            const int c = chunk_of(), left = cols - (col + 4 * c);
            float* p = out + (int64_t)(row0 + row_of(0)) * ld + col + 4 * c;
            uint4 q[kChunks];
#pragma unroll
            for (int i = 0; i < kChunks; ++i) q[i] = chunk(row_of(i), c);
#pragma unroll
            for (int i = 0; i < kChunks; ++i, p += kRowsAtOnce * ld) {
                if (row0 + row_of(i) >= rows || left <= 0) continue;
                if (left >= 4) {
                    *reinterpret_cast<uint4*>(p) = q[i];
                } else {
                    for (int j = 0; j < left; ++j) p[j] = __uint_as_float(word_at(row_of(i), 4 * c + j));
                }
            }
        } else {
            constexpr int kStep = 32 / kWords;
            const int n = min(32, rows - row0), c = lane % kWords;
            float* p = out + (int64_t)(row0 + lane / kWords) * ld + col + c;
#pragma unroll 1
            for (int r = lane / kWords; r - lane / kWords < n; r += 8 * kStep) {
                uint32_t q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = word_at((r + j * kStep) & 31, c);
#pragma unroll
                for (int j = 0; j < 8; ++j, p += kStep * ld)
                    if (r + j * kStep < n && col + c < cols) *p = __uint_as_float(q[j]);
            }
        }
    }
};

template <int WARPS>
__device__ __forceinline__ Turn<WARPS> turn_of(uint8_t* smem_raw, uint32_t base, int warp, int lane) {
    return {smem_raw + (base - smem_u32(smem_raw)) + kStages * kStageBytes + (warp - 4) * (kTurnBytes / WARPS), lane};
}

// The warp has read its part of an accumulator.
template <int CG>
__device__ __forceinline__ void free_accumulator(uint32_t bar, int lane) {
    mma_fence_before();
    __syncwarp();
    if (lane == 0) {
        if constexpr (CG == 2)
            bar_arrive_cluster(bar);
        else
            bar_arrive(bar);
    }
}

// Parts that K is cut into: as many as give every SM or pair (slots) a tile, none of them empty.
__host__ __device__ inline int parts_of_k(int most, int tiles, int slots, int nk) {
    int parts = tiles > 0 ? slots / tiles : 1;
    parts = parts < 1 ? 1 : parts > most ? most : parts;
    const int part = (nk + parts - 1) / parts;
    return (nk + part - 1) / part;
}

template <int CG, bool AMN, bool BMN, class Epi>
__global__ void __launch_bounds__(kMatThreads<Epi::kWarps>, 1)
    k_matmul(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const MatShape shape,
             const typename Epi::Args ea) {
    constexpr int BN = 128 * CG, kWarps = Epi::kWarps;  // columns of a tile
    constexpr int W = BN / (kWarps / 4);                // and of a warp's part of it, at most
    extern __shared__ uint8_t smem_raw[];
    __shared__ BenchShared shared;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    if (threadIdx.x == 0) {
        tma_prefetch(&map_a);
        tma_prefetch(&map_b);
    }
    const Bench w = set_up<CG, kWarps>(shared, smem_raw, warp);

    wait_for_predecessor();
    let_successor_start();

    MatShape g = shape;
    if (g.live_m) g.M = *g.live_m, g.tiles_m = (g.M + 128 * CG - 1) / (128 * CG);
    if (g.live_k) g.K = *g.live_k * g.live_times;
    const int per = tiles_per_matrix(g);
    if (g.splits > 1) g.splits = g.batch = parts_of_k(g.splits, per, kSms / CG, g.plan_nk ? g.plan_nk : max(1, (g.K + kTileK - 1) / kTileK));
    const int total = per * g.batch;
    const int first = blockIdx.x / CG, step = gridDim.x / CG;
    const int nk_one = (g.K + kTileK - 1) / kTileK, nk_all = nk_one * g.fold, nk_part = (nk_all + g.splits - 1) / g.splits;
    const View va = {&map_a, &map_a, AMN ? Lie::mn : Lie::k, 0}, vb = {&map_b, &map_b, BMN ? Lie::mn : Lie::k, 0};
    bool ok = true;

    if (warp == 0) {
        // fill the ring
        const uint32_t full_at = CG == 2 ? map_to_rank(w.full, 0) : w.full;  // the pair's bytes are counted on CTA 0's barrier
        Ring r = {w.base, w.full, w.empty};
        for (int t = first; ok && t < total; t += step) {
            const TileAt at = tile_at(g, t, per);
            const int am = at.m * 128 * CG + (int)rank * 128, bn = at.n * g.width + (int)rank * (g.width / CG);
            const int k0 = g.splits > 1 ? at.b * nk_part : 0, k1 = min(k0 + nk_part, nk_all), z = g.splits > 1 ? 0 : at.b;
            ok = fill_tile<CG>(r, va, vb, am, bn, z, k0, k1, rank, full_at, g.stage_a + g.stage_b, nk_one);
        }
    } else if (warp == 1 && rank == 0) {
        // multiply
        Ring r = {w.base, w.full, w.empty};
        int acc = 0;
        uint32_t aph = 0;
        for (int t = first; ok && t < total; t += step) {
            const int k0 = g.splits > 1 ? tile_at(g, t, per).b * nk_part : 0, nk = min(nk_part, nk_all - k0);
            if (g.splits > 1 && nk <= 0) continue;  // nothing of K is left for this part
            if (!(ok = warp_wait(w.free_ + 8 * acc, aph ^ 1))) break;
            mma_fence_after();
            ok = multiply_tile<CG>(r, w.tmem + acc * BN, nk, va, vb, g.f16, w.done + 8 * acc, g.width);
            if (++acc == 2) acc = 0, aph ^= 1;
        }
    } else if (warp >= 4) {
        // hand the accumulators on
        const int quad = warp % 4, part = (warp - 4) / 4;
        const auto turn = turn_of<kWarps>(smem_raw, w.base, warp, lane);
        const int share = kWarps == 8 ? g.width / 2 : W;  // of a tile's columns (16 bytes of 16 bits at least)
        const uint32_t free_at = CG == 2 ? map_to_rank(w.free_, 0) : w.free_;
        int acc = 0;
        uint32_t aph = 0;
        for (int t = first; t < total; t += step) {
            const TileAt at = tile_at(g, t, per);
            if (g.splits > 1 && at.b * nk_part >= nk_all) continue;
            if (!(ok = warp_wait(w.done + 8 * acc, aph))) break;
            mma_fence_after();
            const int row = at.m * 128 * CG + (int)rank * 128 + quad * 32 + lane;
            const int col = at.n * g.width + part * share, end = min(col + share, (at.n + 1) * g.width);
            Epi::template tile<W>(ea, g, w.tmem + acc * BN + part * share + ((uint32_t)quad << 21), row, col, end, at, part, turn);
            free_accumulator<CG>(free_at + 8 * acc, lane);
            if (++acc == 2) acc = 0, aph ^= 1;
        }
    }
    clear_up<CG>(w, warp, ok);
}

// ---- host side ----

struct Operand {
    const void* p;
    int64_t ld;       // values between two rows as they lie in memory
    int64_t batch_ld; // values between two matrices
    bool mn;          // memory rows run along K, and hold the operand's rows (M or N)
};

cudaError_t make_map(CUtensorMap* out, const Operand& o, int rows, int k, int batch, bool f16, int box = 128);  // box: rows (K contiguous)

int device_sms();  // of the current device; 148 where that cannot be asked


// Pairs of CTAs with tiles of 256 x 256 multiply at the tensor cores' rate (511 cycles per stage of K = 64, of 512);
// tiles of 128 x 128 are held up by what an SM gets from L2 (450 cycles of 256), but leave fewer SMs idle. A tile of the
// pair keeps it busy for two units of time, a small tile its SM for kSmallCost: the smaller number of waves times cost wins.
constexpr double kSmallCost = 1.75;

inline bool use_pairs(int M, int N, int batch, bool sym) {
    auto tiles = [&](int b) {
        const int64_t m = (M + b - 1) / b, n = (N + b - 1) / b;
        return (sym ? m * (m + 1) / 2 : m * n) * batch;
    };
    const int64_t big = (tiles(256) + kSms / 2 - 1) / (kSms / 2), small = (tiles(128) + kSms - 1) / kSms;
    return 2.0 * big <= kSmallCost * small;
}

template <int CG, bool AMN, bool BMN, class Epi>
cudaError_t launch_matmul_cg(const Operand& a, const Operand& b, MatShape g, bool f16, const typename Epi::Args& ea,
                             cudaStream_t stream, bool dependent) {
    CUtensorMap ma, mb;
    if (!g.width) {  // tiles as wide as each other: 777 columns are 4 x 208, not 3 x 256 + 9
        const int n = (g.N + 128 * CG - 1) / (128 * CG);
        g.width = ((g.N + n - 1) / n + 15) / 16 * 16;
    }
    const int matrices = g.splits > 1 ? 1 : g.batch;
    // Where the rows do not fill one tile, only their part of it is loaded; what the rest of the tile's rows hold does not matter.
    const int box_a = !AMN && CG == 1 && g.M < 128 ? (g.M + 7) / 8 * 8 : 128, box_b = BMN ? 128 : g.width / CG;
    g.stage_a = box_a * kTileK * 2, g.stage_b = box_b * kTileK * 2;
    if (!g.fold) g.fold = 1;
    cudaError_t err = make_map(&ma, a, g.M, g.K, g.fold > 1 ? g.fold : matrices, f16, box_a);
    if (err == cudaSuccess) err = make_map(&mb, b, g.N, g.K, matrices, f16, box_b);
    if (err != cudaSuccess) return err;
    g.tiles_m = (g.M + 128 * CG - 1) / (128 * CG);
    g.tiles_n = (g.N + g.width - 1) / g.width;
    g.group = 8 * (CG == 1 ? 2 : 1);
    g.f16 = f16;
    const int64_t per = g.sym ? (int64_t)g.tiles_m * (g.tiles_m + 1) / 2 : (int64_t)g.tiles_m * g.tiles_n;
    const int64_t slots = device_sms() / CG, total = per * g.batch;
    if (total > 0x7FFFFFFF) return cudaErrorInvalidValue;
    auto kernel = k_matmul<CG, AMN, BMN, Epi>;
    static std::atomic<uint64_t> ready{0};
    err = allow_smem(kernel, kMatSmem, ready);
    if (err != cudaSuccess) return err;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((total < slots ? total : slots) * CG));
    cfg.blockDim = dim3(kMatThreads<Epi::kWarps>);
    cfg.dynamicSmemBytes = kMatSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (CG == 2) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = 2;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (dependent) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kernel, ma, mb, g, ea);
}

// `dependent`: the launch before this one on the stream is one of this call's, and the kernel may be set up beside its tail.
template <bool AMN, bool BMN, class Epi>
cudaError_t launch_matmul(const Operand& a, const Operand& b, int M, int N, int K, int batch, bool sym, bool f16,
                          const typename Epi::Args& ea, cudaStream_t stream, bool dependent, const int* live_m = nullptr,
                          const int* live_k = nullptr, int width = 0, int live_times = 1) {
    MatShape g = {};
    g.width = width, g.live_times = live_times;
    g.M = M, g.N = N, g.K = K, g.batch = batch, g.splits = 1, g.sym = sym, g.live_m = live_m, g.live_k = live_k;
    return !width && use_pairs(M, N, batch, sym) ? launch_matmul_cg<2, AMN, BMN, Epi>(a, b, g, f16, ea, stream, dependent)
                                       : launch_matmul_cg<1, AMN, BMN, Epi>(a, b, g, f16, ea, stream, dependent);
}

// How a product with few tiles and a long K is cut: into at most `splits` parts of K, on pairs of CTAs or single ones. The
// time of a way is its waves times the stages of a part (and about 16 stages' time for filling the ring and storing a
// tile). Twice as many parts as M asks for are allowed, because fewer rows may take part than M.
struct Cut {
    bool pairs;
    int splits;
};
inline Cut cut_of(int M, int N, int K) {
    Cut best = {true, 1};
    double least = 0;
    const int nk = (K + kTileK - 1) / kTileK;
    for (int pairs = 1; pairs >= 0; --pairs) {
        const int64_t b = pairs ? 256 : 128, tiles = ((M + b - 1) / b) * ((N + b - 1) / b), slots = pairs ? kSms / 2 : kSms;
        for (int s = 1; s <= 16 && s <= nk; ++s) {
            const int part = (nk + s - 1) / s;
            if (s > 1 && (s - 1) * part >= nk) continue;  // no part is empty
            const double waves = (double)((tiles * s + slots - 1) / slots);
            // a unit is 0.135 us; joining the parts is a launch of about 5 us and a pass over their sums at 5 TB/s
            const double cost = waves * (part * (pairs ? 2.0 : kSmallCost) + 32) + (s > 1 ? 36 + (double)s * M * N * 8 / 675e3 : 0);
            if (least == 0 || cost < least) least = cost, best = {pairs != 0, s};
        }
    }
    if (best.splits > 1) best.splits = 2 * best.splits < nk ? 2 * best.splits : nk;
    return best;
}
// The parts that a product over `live` rows is cut into.
__host__ __device__ inline int parts_of(const Cut& cut, int live, int N, int plan_nk) {
    const int b = cut.pairs ? 256 : 128, tiles = ((live + b - 1) / b) * ((N + b - 1) / b);
    return cut.splits > 1 ? parts_of_k(cut.splits, tiles, cut.pairs ? kSms / 2 : kSms, plan_nk) : 1;
}

template <bool AMN, bool BMN, class Epi>
cudaError_t launch_matmul_cut(const Operand& a, const Operand& b, int M, int N, int K, Cut cut, bool f16,
                              const typename Epi::Args& ea, cudaStream_t stream, bool dependent, const int* live_m, int plan_nk, int fold,
                              const int* live_k = nullptr, int live_times = 1) {
    MatShape g = {};
    g.fold = fold, g.live_k = live_k, g.live_times = live_times;
    g.M = M, g.N = N, g.K = K, g.batch = g.splits = cut.splits, g.live_m = live_m, g.plan_nk = plan_nk;
    return cut.pairs ? launch_matmul_cg<2, AMN, BMN, Epi>(a, b, g, f16, ea, stream, dependent)
                     : launch_matmul_cg<1, AMN, BMN, Epi>(a, b, g, f16, ea, stream, dependent);
}

}  // namespace ones
