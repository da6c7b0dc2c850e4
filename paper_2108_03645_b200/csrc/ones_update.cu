// Orthogonalised update of matrix parameters by Newton-Schulz products.
#include <math.h>

#include "ones_matmul.cuh"
#include "ones_train.h"
#include "ones_train_internal.h"

namespace ones {

namespace {

constexpr int kNormThreads = 256, kNormBlocks = 8 * kSms;  // a warp takes a row at a time

__device__ __forceinline__ float load_as_float(const void* p, int64_t i, int type) {
    if (type == ONES_F32) return static_cast<const float*>(p)[i];
    if (type == ONES_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}

// 8 neighbouring values from a 16-byte boundary.
__device__ __forceinline__ void load8(const void* p, int64_t i, int type, float (&v)[8]) {
    if (type == ONES_F32) {
        const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
        const float4 a = q[0], b = q[1];
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        return;
    }
    const uint4 q = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float2 f;
        if (type == ONES_BF16)
            f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[j]));
        else
            f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
        v[2 * j] = f.x, v[2 * j + 1] = f.y;
    }
}

struct Source {
    const void* p;
    int64_t ld, stride;
    int m, n, type;
    bool wide;  // rows start on 16-byte boundaries and hold a multiple of 8 values
};

// Sum of squares of each matrix, in 64 bits (squares of small gradients leave the range of 32), one part per block. Also
// clears the counter that the blocks of k_ns_steps meet at. 4096 x 8192 of bfloat16: 20 us (3.3 TB/s; 64-bit sums).
__global__ void __launch_bounds__(kNormThreads) k_ns_norm(Source g, double* part, unsigned* counter) {
    __shared__ double s[kNormThreads / 32];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *counter = 0;
    double sum = 0.0;
    for (int r = blockIdx.x * (kNormThreads / 32) + warp; r < g.m; r += gridDim.x * (kNormThreads / 32)) {
        const int64_t at = blockIdx.y * g.stride + r * g.ld;
        if (g.wide) {
#pragma unroll 4
            for (int c = lane * 8; c < g.n; c += 256) {
                float v[8];
                load8(g.p, at + c, g.type, v);
                double e[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i & 3] = fma((double)v[i], (double)v[i], e[i & 3]);
                sum += (e[0] + e[1]) + (e[2] + e[3]);
            }
        } else {
#pragma unroll 8
            for (int c = lane; c < g.n; c += 32) {
                const double v = load_as_float(g.p, at + c, g.type);
                sum += v * v;
            }
        }
    }
    for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (lane == 0) s[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kNormThreads / 32; ++i) sum += s[i];
        part[blockIdx.y * gridDim.x + blockIdx.x] = sum;
    }
    let_successor_start();
}

// Between the steps X is kept as 16 bits, times a power of two. Where |G| is not small beside eps, that is `unit`, about the
// square root of the longer side: it brings X's values near 1 once its singular values have arrived there. A matrix that is
// small beside eps has |X|_F = n < 1 and is kept times up to 2^50 more, so that n * 2^j stays within (0.5, 1]; n grows in a
// step by at most |a| + |b| n^2 + |c| n^4 (X's singular values are at most n).
__device__ __forceinline__ float kept_times(float n, float unit) {
    const int j = n > 0.f && n < 1.f ? 126 - (int)(__float_as_uint(n) >> 23) : 0;  // by the exponent's bits: 0 for n in [0.5, 1)
    return __uint_as_float(__float_as_uint(unit) + ((uint32_t)(j < 50 ? j : 50) << 23));
}
__device__ __forceinline__ float inverse_of_power(float x) { return __uint_as_float((254u << 23) - __float_as_uint(x)); }
__device__ __forceinline__ float bound_after(float n, float a, float b, float c) {
    return n < 1.f ? n * (fabsf(a) + n * n * (fabsf(b) + n * n * fabsf(c))) : n;
}
// What the epilogues of a step multiply by, for each of the first kScaled steps, for those behind them (X is kept times
// `unit` there) and for the last one: .x the Gram matrix, .y the application.
constexpr int kScaled = 32;
__device__ __forceinline__ int scales_of(int k, int steps) { return k + 1 == steps ? kScaled + 1 : k < kScaled ? k : kScaled; }

// X0 = G * 2^-k in 11 significant bits, k such that the values' root mean square is about 1: exact for bfloat16 (8 bits)
// down to 2^-14 of it. What is missing to G / (|G| + eps), f = 2^k / (|G| + eps), and f^2, go into the first step's epilogues:
// scales [kScaled + 2][count] holds the factors of all steps.
struct Polynomial {
    int steps;
    float a, b, c, unit;
};
__global__ void __launch_bounds__(kNormThreads) k_ns_cast(Source g, const double* part, int parts, float eps, __half* x, int64_t ldx,
                                                          Polynomial p, float2* scales) {
    wait_for_predecessor();
    let_successor_start();
    __shared__ double s_sum[kNormThreads / 32];
    __shared__ float s_scale;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += kNormThreads) sum += part[blockIdx.y * parts + i];
    for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kNormThreads / 32; ++i) sum += s_sum[i];
        const double norm = sqrt(sum), rms = norm / sqrt((double)g.m * g.n);
        int k = rms > 0.0 && rms < 1e300 ? ilogb(rms) : 0;
        k = k < -120 ? -120 : k > 120 ? 120 : k;
        s_scale = ldexpf(1.f, -k);
        if (blockIdx.x == 0) {
            const double f = norm == 0.0 ? 0.0 : ldexp(1.0, k) / (norm + eps);  // of nothing: 1 / eps, whose square may pass 32 bits
            float2* to = scales + blockIdx.y;
            float n = (float)(norm / (norm + eps)), gram = (float)(f * f), from = (float)f;  // from: 1 / what X is kept times
            for (int i = 0; i < kScaled && i + 1 < p.steps; ++i) {
                n = bound_after(n, p.a, p.b, p.c);
                const float times = i + 1 < kScaled ? kept_times(n, p.unit) : p.unit;
                to[(int64_t)i * gridDim.y] = make_float2(gram, from * times);
                from = inverse_of_power(times), gram = from * from;
            }
            to[(int64_t)kScaled * gridDim.y] = make_float2(1.f / (p.unit * p.unit), 1.f);
            to[(int64_t)(kScaled + 1) * gridDim.y] = make_float2(gram, from);
        }
    }
    __syncthreads();
    const float scale = s_scale;
    for (int r = blockIdx.x * (kNormThreads / 32) + warp; r < g.m; r += gridDim.x * (kNormThreads / 32)) {
        const int64_t at = blockIdx.y * g.stride + r * g.ld;
        __half* out = x + ((int64_t)blockIdx.y * g.m + r) * ldx;
        if (g.wide) {
#pragma unroll 4
            for (int c = lane * 8; c < g.n; c += 256) {
                float v[8];
                load8(g.p, at + c, g.type, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= scale;
                *reinterpret_cast<uint4*>(out + c) = make_uint4(Half16::pack(v[0], v[1], true), Half16::pack(v[2], v[3], true),
                                                                Half16::pack(v[4], v[5], true), Half16::pack(v[6], v[7], true));
            }
        } else {
#pragma unroll 8
            for (int c = lane; c < g.n; c += 32) out[c] = __float2half_rn(load_as_float(g.p, at + c, g.type) * scale);
        }
    }
}

// The symmetric products have only their blocks on and above the diagonal computed and stored. The products that read
// them take what lies below from above, as an operand with its rows contiguous (Lie::upper).

// Eight warps: with 16, rounds of long products gain (2048 x 8192: 586 -> 571 us), but the many short ones lose more
// to the larger barrier and the smaller register share (8192 x 300: 179 -> 195 us).
constexpr int kStepWarps = 8;
using StepTurn = Turn<kStepWarps>;

// A = factor * X X^T, and its diagonal in 32 bits.
struct EpiGram {
    struct Args {
        __half* out;
        float* diag;  // [count][s]
        int64_t ld, batch_ld;
        int s;
        float* part;          // where K is cut: the sums of this part [count][s][ld_part], else NULL
        int64_t ld_part;
    };
    template <int W, bool CUT>
    static __device__ __forceinline__ void tile(const Args& a, uint32_t acc, int row, int col, const TileAt& at, const StepTurn& turn, float f) {
        if constexpr (CUT) {
            float* out = a.part + (int64_t)at.b * a.s * a.ld_part;
#pragma unroll 1
            for (int c = 0; c < W && col + c < a.s; c += 32) {
                float v[32];
                tmem_load(acc + c, v);
                turn.write32(v, out, a.ld_part, row - turn.lane, col + c, a.s, a.s, true);
            }
            return;
        }
        uint16_t* out = reinterpret_cast<uint16_t*>(a.out + at.b * a.batch_ld);
#pragma unroll 1
        for (int c = 0; c < W && col + c < a.s; c += 64) {
            float v[64];
            tmem_load(acc + c, v);
            const unsigned d = (unsigned)(row - (col + c));
            if (d < 64u && row < a.s) {
                float own = 0.f;
#pragma unroll
                for (int i = 0; i < 64; ++i) own = d == (unsigned)i ? v[i] : own;
                a.diag[(int64_t)at.b * a.s + row] = own * f;
            }
#pragma unroll
            for (int i = 0; i < 64; ++i) v[i] *= f;
            turn.write16(v, true, out, a.ld, row - turn.lane, col + c, a.s, a.s, true);
        }
    }
    // Joins the parts of a row's sums, in order, from the diagonal's block on. Run by a warp.
    static __device__ __forceinline__ void join(const Args& a, int parts, int64_t stride, int b, int row, int block, int lane, float f) {
        const float* from = a.part + ((int64_t)b * a.s + row) * a.ld_part;
        __half* to = a.out + b * a.batch_ld + (int64_t)row * a.ld;
        for (int c = row / block * block + 4 * lane; c < a.s; c += 128) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
            for (int k = 0; k < parts; ++k) {
                const float4 q = __ldcg(reinterpret_cast<const float4*>(from + k * stride + c));
                v.x += q.x, v.y += q.y, v.z += q.z, v.w += q.w;
            }
            v.x *= f, v.y *= f, v.z *= f, v.w *= f;
            if (row >= c && row < c + 4) a.diag[(int64_t)b * a.s + row] = row == c ? v.x : row == c + 1 ? v.y : row == c + 2 ? v.z : v.w;
            // the row is padded to whole 16 bytes; what lies behind its end is not read
            *reinterpret_cast<uint2*>(to + c) = make_uint2(Half16::pack(v.x, v.y, true), Half16::pack(v.z, v.w, true));
        }
    }
};

// An entry of the diagonal of the polynomial from the entry of A in 32 bits: a product of rounded matrices has it with
// the error of the rounded entry, which is the largest of its row and the same for the whole row of the next product.
__device__ __forceinline__ float mend_diagonal(float p, float exact, float a, float b, float c) {
    const float rounded = __half2float(__float2half_rn(exact));
    return p + a + b * (exact - rounded) + c * (exact * exact - rounded * rounded);
}
// What a row of the next product has to be multiplied by so that the rounding of the diagonal's entry does not count.
__device__ __forceinline__ float regain_row(float p) {
    const float rounded = __half2float(__float2half_rn(p)), r = __fdividef(p, rounded);
    return fabsf(r - 1.f) < 0.002f ? r : 1.f;  // not where the entry is next to nothing
}

// B = a I + b A + c A A. With a I inside B the next product needs no second operand, and B's values near the end are
// those of a I + b A + c A^2 (about 1), not of its terms (several times that), so its rounding is finer.
struct EpiPoly {
    struct Args {
        const __half* gram;
        __half* out;
        const float* diag;
        float* regain;  // [count][s]
        int64_t ld, batch_ld;
        int s;
        float a, b, c;
    };
    // A's values of 64 columns, 8 lanes to a row, as the result leaves; asked for before they are needed.
    static __device__ __forceinline__ void load(const Args& a, int row, int col, const TileAt& at, const StepTurn& turn, uint4 (&q)[8]) {
        const int c = col + 8 * turn.chunk_of();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = row - turn.lane + turn.row_of(i);  // rows of A are padded to whole 16 bytes
            q[i] = r < a.s && c < a.s ? __ldcg(reinterpret_cast<const uint4*>(a.gram + at.b * a.batch_ld + (int64_t)r * a.ld + c))
                                      : make_uint4(0, 0, 0, 0);
        }
    }
    template <int W>
    static __device__ __forceinline__ void tile(const Args& a, uint32_t acc, int row, int col, const TileAt& at, const StepTurn& turn, uint4 (&q)[8],
                                                float exact) {
        uint16_t* out = reinterpret_cast<uint16_t*>(a.out + at.b * a.batch_ld);
#pragma unroll 1
        for (int c = 0; c < W && col + c < a.s; c += 64) {
            float v[64];
            tmem_load(acc + c, v);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) turn.chunk(turn.row_of(i), turn.chunk_of()) = q[i];
            __syncwarp();
            if (c + 64 < W) load(a, row, col + c + 64, at, turn, q);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint4 p = turn.chunk(turn.lane, j);
                const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                    v[8 * j + 2 * i] = fmaf(a.c, v[8 * j + 2 * i], a.b * h.x);
                    v[8 * j + 2 * i + 1] = fmaf(a.c, v[8 * j + 2 * i + 1], a.b * h.y);
                }
            }
            const unsigned d = (unsigned)(row - (col + c));
            if (d < 64u && row < a.s) {
                float own = 0.f;
#pragma unroll
                for (int i = 0; i < 64; ++i) own = d == (unsigned)i ? v[i] : own;
                own = mend_diagonal(own, exact, a.a, a.b, a.c);
#pragma unroll
                for (int i = 0; i < 64; ++i) v[i] = d == (unsigned)i ? own : v[i];
                a.regain[(int64_t)at.b * a.s + row] = regain_row(own);
            }
            turn.write16(v, true, out, a.ld, row - turn.lane, col + c, a.s, a.s, true);
        }
    }
};

// X = factor * B X
struct EpiApply {
    struct Args {
        uint16_t* out;
        int64_t ld, batch_ld;
        int m, n;
        const float* regain;  // [count][s]: of the rows, or (tall) of the columns
        bool f16, wide;
    };
    template <int W, bool TALL>
    static __device__ __forceinline__ void tile(const Args& a, uint32_t acc, int row, int col, const TileAt& at, const StepTurn& turn, float f) {
        const float* regain = a.regain + (int64_t)at.b * a.n;
#pragma unroll 1
        for (int c = 0; c < W && col + c < a.n; c += 64) {
            float v[64], r0 = 1.f, r1 = 1.f;
            if constexpr (TALL) {
                const int k = col + c + 2 * turn.lane;
                if (k < a.n) r0 = __ldcg(regain + k);
                if (k + 1 < a.n) r1 = __ldcg(regain + k + 1);
            }
            tmem_load(acc + c, v);
#pragma unroll
            for (int i = 0; i < 64; ++i) v[i] *= f;
            if constexpr (TALL) {
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    v[2 * i] *= __shfl_sync(0xFFFFFFFFu, r0, i);
                    v[2 * i + 1] *= __shfl_sync(0xFFFFFFFFu, r1, i);
                }
            }
            turn.write16(v, a.f16, a.out + at.b * a.batch_ld, a.ld, row - turn.lane, col + c, a.m, a.n, a.wide);
        }
    }
};

// All steps in one launch. A step is three products (Gram matrix, polynomial, application), each of which needs all of
// the one before; as launches of their own the 15 of five steps cost 9 us each for small matrices and 14 for twelve of
// 768 x 768, most of it in starting, ending and first touching of code. Here the blocks stay, with their barriers and
// accumulators, and meet at a counter between products (a cooperative launch: all of them are on the GPU). Twelve of 768 x
// 768: 174 us, 15 rounds of 11.6; 4096 x 8192: 1.68 ms, 1.47 PFLOP/s, where the power cap holds it.
struct StepsArgs {
    int m, n, s, count, steps;
    int parts;  // > 1: K of the Gram matrix is cut into so many parts, joined in a round of its own
    float *diag, *regain, *part;
    int64_t ld_part, part_stride;
    bool tall;
    float a, b, c;
    __half *x[2], *gram, *poly;
    uint16_t* out;
    int64_t ldx, xs, lds, ss;
    const float2* scales;  // [kScaled + 2][count]
    unsigned* counter;
    bool wide;
};
struct StepsMaps {
    CUtensorMap rows[2], cols[2];  // X with its rows as the operand's rows, and with its columns
    CUtensorMap gram[2], poly[2];
};

// The operands of the products: X X^T or X^T X; A A; B X or X B.
__device__ __forceinline__ void operands(const StepsMaps& maps, bool tall, int which, int buf, const TileAt& at, View& a, View& b) {
    const View x = {&maps.rows[buf], &maps.cols[buf], Lie::k, 0};
    if (which == 0) {
        a = b = x;
        if (tall) a.lie = b.lie = Lie::mn;
    } else if (which == 1) {
        a = {&maps.gram[0], &maps.gram[1], Lie::upper, at.m};
        b = {&maps.gram[0], &maps.gram[1], Lie::upper, at.n};
    } else if (tall) {
        a = x;
        b = {&maps.poly[0], &maps.poly[1], Lie::upper, at.n};
    } else {
        a = {&maps.poly[0], &maps.poly[1], Lie::upper, at.m};
        b = x;
        b.lie = Lie::mn;
    }
}

// CUT: the Gram matrix's K is cut into parts; TALL: more rows than columns, the Gram matrix is X^T X and X takes the
// polynomial from the right. Both as kernels of their own: code that is not run still costs (12 of 189 us for twelve of
// 768 x 768).
template <int CG, bool CUT, bool TALL>
__global__ void __launch_bounds__(kMatThreads<kStepWarps>, 1) k_ns_steps(const __grid_constant__ StepsMaps maps, const StepsArgs p) {
    constexpr int BN = 128 * CG;
    extern __shared__ uint8_t smem_raw[];
    __shared__ BenchShared shared;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    __shared__ __align__(8) uint64_t s_round;  // tells the epilogue that the product before is complete: one poller a block
    const uint32_t round_bar = smem_u32(&s_round);
    if (threadIdx.x == 0) bar_init(round_bar, 1);
    const Bench w = set_up<CG, kStepWarps>(shared, smem_raw, warp);
    wait_for_predecessor();

    const int first = blockIdx.x / CG, step = gridDim.x / CG;
    // the three products of a step
    MatShape sym = {}, app = {};
    sym.M = sym.N = p.s, sym.batch = p.count, sym.sym = 1, sym.tiles_m = sym.tiles_n = (p.s + BN - 1) / BN;
    app.M = p.m, app.N = p.n, app.K = p.s, app.batch = p.count, app.tiles_m = (p.m + BN - 1) / BN, app.tiles_n = (p.n + BN - 1) / BN;
    app.group = 16 / CG;
    const int per_sym = tiles_per_matrix(sym), per_app = tiles_per_matrix(app);
    const int long_side = TALL ? p.m : p.n;
    const int nk_gram = (long_side + kTileK - 1) / kTileK, nk_s = (p.s + kTileK - 1) / kTileK;
    // a step's rounds: Gram matrix, (3: its parts joined,) polynomial, application
    constexpr int per_step = CUT ? 4 : 3;
    const int rounds = per_step * p.steps;
    const int gram_part = CUT ? (nk_gram + p.parts - 1) / p.parts : nk_gram;
    auto which_of = [&](int round) {
        const int i = round % per_step;
        return !CUT || i == 0 ? i : i == 1 ? 3 : i - 1;
    };
    auto tiles_in = [&](int which) { return which == 0 ? per_sym * p.count * (CUT ? p.parts : 1) : which == 1 ? per_sym * p.count : which == 2 ? per_app * p.count : 0; };
    // tile t of a round, the part of K that it takes and what that is
    auto tile_of = [&](int which, int t, int& k0, int& nk, int& cut) {
        cut = 0;
        k0 = 0, nk = which == 0 ? nk_gram : nk_s;
        if (CUT && which == 0) {
            cut = t / (per_sym * p.count);
            t -= cut * per_sym * p.count;
            k0 = cut * gram_part, nk = min(gram_part, nk_gram - k0);
        }
        return tile_at(which == 2 ? app : sym, t, which == 2 ? per_app : per_sym);
    };
    bool ok = true;

    if (warp == 0) {
        const uint32_t full_at = CG == 2 ? map_to_rank(w.full, 0) : w.full;
        Ring r = {w.base, w.full, w.empty};
        for (int round = 0; ok && round < rounds; ++round) {
            const int which = which_of(round), buf = round / per_step & 1, total = tiles_in(which);
            if (round && !(ok = wait_all(p.counter, (unsigned)round * gridDim.x))) break;
            if (round && lane == 0) bar_arrive(round_bar);
            for (int t = first; ok && t < total; t += step) {
                int k0, nk, cut;
                const TileAt at = tile_of(which, t, k0, nk, cut);
                View va, vb;
                operands(maps, TALL, which, buf, at, va, vb);
                ok = fill_tile<CG>(r, va, vb, at.m * BN + (int)rank * 128, at.n * BN + (int)rank * 128, at.b, k0, k0 + nk, rank, full_at);
            }
        }
    } else if (warp == 1 && rank == 0) {
        Ring r = {w.base, w.full, w.empty};
        int acc = 0;
        uint32_t aph = 0;
        for (int round = 0; ok && round < rounds; ++round) {
            const int which = which_of(round), total = tiles_in(which);
            for (int t = first; ok && t < total; t += step) {
                int k0, nk, cut;
                View va, vb;
                operands(maps, TALL, which, 0, tile_of(which, t, k0, nk, cut), va, vb);
                if (!(ok = warp_wait(w.free_ + 8 * acc, aph ^ 1))) break;
                mma_fence_after();
                ok = multiply_tile<CG>(r, w.tmem + acc * BN, nk, va, vb, true, w.done + 8 * acc);
                if (++acc == 2) acc = 0, aph ^= 1;
            }
        }
    } else if (warp >= 4) {
        const int quad = warp % 4, half = (warp - 4) / 4;
        const StepTurn turn = turn_of<kStepWarps>(smem_raw, w.base, warp, lane);
        const uint32_t free_at = CG == 2 ? map_to_rank(w.free_, 0) : w.free_;
        int acc = 0;
        uint32_t aph = 0;
        for (int round = 0; round < rounds; ++round) {  // a warp that gave up still comes to the barrier below
            const int which = which_of(round), k = round / per_step, buf = k & 1, total = tiles_in(which);
            if (ok && round) ok = warp_wait(round_bar, (round - 1) & 1);
            const float2* scales = p.scales + (int64_t)scales_of(k, p.steps) * p.count;
            EpiGram::Args eg = {p.gram, p.diag, p.lds, p.ss, p.s, p.part, p.ld_part};
            if (CUT && ok && which == 3)
                for (int i = blockIdx.x * kStepWarps + warp - 4; i < p.count * p.s; i += gridDim.x * kStepWarps)
                    EpiGram::join(eg, p.parts, p.part_stride, i / p.s, i % p.s, BN, lane, scales[i / p.s].x);
            for (int t = first; ok && t < total; t += step) {
                int k0, nk, cut;
                const TileAt at = tile_of(which, t, k0, nk, cut);
                const int row = at.m * BN + (int)rank * 128 + quad * 32 + lane, col = at.n * BN + half * (BN / 2);
                const uint32_t tmem = w.tmem + acc * BN + half * (BN / 2) + ((uint32_t)quad << 21);
                const EpiPoly::Args ep = {p.gram, p.poly, p.diag, p.regain, p.lds, p.ss, p.s, p.a, p.b, p.c};
                uint4 q[8];
                // what the epilogue needs of the round before, asked for while the tile is multiplied
                float own = 1.f;
                const float2 scale = scales[at.b];
                if (which == 1) EpiPoly::load(ep, row, col, at, turn, q);
                if (row < p.s && (which == 1 || (which == 2 && !TALL)))
                    own = __ldcg((which == 1 ? p.diag : p.regain) + (int64_t)at.b * p.s + row);
                if (!(ok = warp_wait(w.done + 8 * acc, aph))) break;
                mma_fence_after();
                if (which == 0) {
                    if (CUT) eg.part = p.part + cut * p.part_stride;
                    EpiGram::tile<BN / 2, CUT>(eg, tmem, row, col, at, turn, scale.x);
                } else if (which == 1) {
                    EpiPoly::tile<BN / 2>(ep, tmem, row, col, at, turn, q, own);
                } else {
                    EpiApply::Args e = {reinterpret_cast<uint16_t*>(p.x[1 - buf]), p.ldx, p.xs, p.m, p.n, p.regain, true, true};
                    if (k + 1 == p.steps) {
                        e.out = p.out, e.ld = p.n, e.batch_ld = (int64_t)p.m * p.n;
                        e.f16 = false, e.wide = p.wide;
                    }
                    EpiApply::tile<BN / 2, TALL>(e, tmem, row, col, at, turn, scale.y * own);
                }
                free_accumulator<CG>(free_at + 8 * acc, lane);
                if (++acc == 2) acc = 0, aph ^= 1;
            }
            asm volatile("bar.sync 1, %0;" ::"n"(32 * kStepWarps) : "memory");
            if (warp == 4 && lane == 0) arrive_all(p.counter);
        }
    }
    clear_up<CG>(w, warp, ok);
}

// A matrix whose shorter side is at most 128 stays in shared memory from its first reading to its result: of one CTA up
// to 512 on the longer side, of a cluster of CTAs up to 8192. X lies there as blocks of 64 columns (of the longer side)
// x 128 rows with the 128-byte swizzle, which serves both as the operand with K along the longer side (X X^T) and as the
// one with its rows along it (B X). Nothing but the input and the result touches memory. In a cluster each CTA has some
// of the columns; the CTAs' shares of the Gram matrix are added up over distributed shared memory, each CTA summing some
// of the rows for all of them, and the 128 x 128 polynomial is computed by each. 128 x 256 takes 69 us in k_ns_steps, most
// of it in the meetings of all blocks of the GPU, and 30 us here.
constexpr int kSmallSide = 128, kSmallLong = 512, kSmallThreads = 512, kBlockBytes = 128 * 128;

struct SmallArgs {
    int cluster, own;  // CTAs of a matrix, and blocks of columns that a CTA has (the last one may have fewer)
    int steps;
    float a, b, c, eps, unit;
    uint16_t* out;
    bool wide;
};

template <bool CL>
__global__ void __launch_bounds__(kSmallThreads, 1) k_ns_small(const Source g, const SmallArgs p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t s_bar;
    __shared__ uint32_t s_tmem;
    __shared__ double s_sum[kSmallThreads / 32];
    __shared__ float s_scale, s_factor, s_bound, s_regain[128], s_diag[128];
    __shared__ double s_share;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const bool tall = g.m > g.n;
    const int rank = CL ? (int)cluster_rank() : 0, matrix = CL ? blockIdx.x / p.cluster : blockIdx.x;
    const int lng = tall ? g.m : g.n, c0 = rank * p.own * 64, mine = min(p.own * 64, lng - c0);  // columns c0 .. c0 + mine - 1
    const int blocks = (mine + 63) / 64;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u, bar = smem_u32(&s_bar);
    uint8_t* x = smem_raw + (base - smem_u32(smem_raw));
    uint8_t* gram = x + p.own * kBlockBytes;
    uint8_t* poly = gram + 2 * kBlockBytes;
    const uint32_t x_at = base, gram_at = base + p.own * kBlockBytes, poly_at = gram_at + 2 * kBlockBytes;
    const uint32_t cols = p.own <= 2 ? 128 : p.own <= 4 ? 256 : 512;  // with this shared memory, what an SM's blocks take together fits
    if (threadIdx.x == 0) {
        bar_init(bar, 1);
        bar_init_done();
    }
    if (warp == 0) tmem_alloc<1>(smem_u32(&s_tmem), cols);

    // X0 as in k_ns_norm and k_ns_cast
    // (this CTA's columns of X: rows of the matrix if it is tall)
    const int64_t from = matrix * g.stride + (tall ? c0 * g.ld : c0);
    const int my_rows = tall ? mine : g.m, my_cols = tall ? g.n : mine;
    double sums[4] = {0.0, 0.0, 0.0, 0.0};  // chains of additions in 64 bits are long: four of them
#pragma unroll 4
    for (int r = warp; r < my_rows; r += kSmallThreads / 32) {
        if (g.wide) {
            for (int c = lane * 8; c < my_cols; c += 256) {
                float v[8];
                load8(g.p, from + r * g.ld + c, g.type, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sums[i & 3] = fma((double)v[i], (double)v[i], sums[i & 3]);
            }
        } else {
#pragma unroll 4
            for (int c = lane; c < my_cols; c += 32) {
                const double v = load_as_float(g.p, from + r * g.ld + c, g.type);
                sums[0] = fma(v, v, sums[0]);
            }
        }
    }
    double sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (lane == 0) s_sum[warp] = sum;
    for (int i = threadIdx.x; i < p.own * kBlockBytes / 16; i += kSmallThreads) reinterpret_cast<uint4*>(x)[i] = make_uint4(0, 0, 0, 0);
    mma_fence_before();
    __syncthreads();
    mma_fence_after();
    const uint32_t tmem = s_tmem;
    if (threadIdx.x == 0) {
        for (int i = 1; i < kSmallThreads / 32; ++i) sum += s_sum[i];
        s_share = sum;
    }
    if constexpr (CL) cluster_sync_all();
    if (threadIdx.x == 0) {
        if constexpr (CL) {
            sum = 0.0;
            for (int q = 0; q < p.cluster; ++q) {
                double share;
                asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(share) : "r"(map_to_rank(smem_u32(&s_share), q)) : "memory");
                sum += share;
            }
        }
        const double norm = sqrt(sum), rms = norm / sqrt((double)g.m * g.n);
        int k = rms > 0.0 && rms < 1e300 ? ilogb(rms) : 0;
        k = k < -120 ? -120 : k > 120 ? 120 : k;
        s_scale = ldexpf(1.f, -k);
        s_factor = norm == 0.0 ? 0.f : (float)(ldexp(1.0, k) / (norm + p.eps));  // as in k_ns_cast
        s_bound = (float)(norm / (norm + p.eps));
    }
    __syncthreads();
    const float scale = s_scale, factor = s_factor;
#pragma unroll 4
    for (int r = warp; r < my_rows; r += kSmallThreads / 32) {
        if (tall) {  // row r of the matrix is column r of X
            uint8_t* to = x + (r / 64) * kBlockBytes + (r % 8) * 2;
            for (int c = lane; c < my_cols; c += 32)
                *reinterpret_cast<__half*>(to + c * 128 + (((r % 64 / 8) ^ (c & 7)) << 4)) =
                    __float2half_rn(load_as_float(g.p, from + r * g.ld + c, g.type) * scale);
        } else if (g.wide) {
            for (int c = lane * 8; c < my_cols; c += 256) {
                float v[8];
                load8(g.p, from + r * g.ld + c, g.type, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= scale;
                *reinterpret_cast<uint4*>(x + (c / 64) * kBlockBytes + r * 128 + (((c % 64 / 8) ^ (r & 7)) << 4)) =
                    make_uint4(Half16::pack(v[0], v[1], true), Half16::pack(v[2], v[3], true), Half16::pack(v[4], v[5], true),
                               Half16::pack(v[6], v[7], true));
            }
        } else {
            for (int c = lane; c < my_cols; c += 32)
                *reinterpret_cast<__half*>(x + (c / 64) * kBlockBytes + r * 128 + (((c % 64 / 8) ^ (r & 7)) << 4) + (c % 8) * 2) =
                    __float2half_rn(load_as_float(g.p, from + r * g.ld + c, g.type) * scale);
        }
    }

    const int quad = warp % 4, part = warp / 4, row = quad * 32 + lane;  // a thread has 32 columns of a row at a time
    const uint32_t lanes = (uint32_t)quad << 21;
    const uint32_t idesc128 = instruction_desc(1, true, false, false, 128);
    uint32_t ph = 0;
    Waits arrived;
    // What the threads wrote to shared memory is there for the tensor cores; one warp issues, all wait for the end.
    auto ready = [&] {
        asm volatile("fence.proxy.async;" ::: "memory");
        mma_fence_before();
        __syncthreads();
        mma_fence_after();
    };
    auto wait = [&] {
        arrived(bar, ph);
        ph ^= 1;
        mma_fence_after();
    };
    // D[128][128] = A A^T for `n` blocks of 64 columns
    auto square = [&](uint32_t at, int n) {
        if (warp == 0) {
            const uint64_t d = operand_desc(at, false, 0);
            if (elect_one()) {
                for (int i = 0; i < n; ++i) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint64_t o = d + (uint64_t)(i * (kBlockBytes >> 4) + j * 2);
                        mma_f16<1>(tmem, o, o, idesc128, (i | j) != 0);
                    }
                }
                mma_commit<1>(bar);
            }
            __syncwarp();
        }
    };
    // 32 values of a row into the 32 columns `n` of a blocked matrix
    auto put = [&](uint8_t* to, int r, int n, const float (&e)[32], bool f16) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            *reinterpret_cast<uint4*>(to + (n / 2) * kBlockBytes + r * 128 + ((((n & 1) * 4 + c) ^ (r & 7)) << 4)) =
                make_uint4(Half16::pack(e[8 * c], e[8 * c + 1], f16), Half16::pack(e[8 * c + 2], e[8 * c + 3], f16),
                           Half16::pack(e[8 * c + 4], e[8 * c + 5], f16), Half16::pack(e[8 * c + 6], e[8 * c + 7], f16));
    };
    ready();
    float bound = s_bound, back = factor;  // of |X|; 1 / what X is kept times
    for (int k = 0; k < p.steps; ++k) {
        const float f = back * back;
        square(x_at, blocks);
        wait();
        float v[32];
        tmem_load(tmem + part * 32 + lanes, v);
        const unsigned d = (unsigned)(row - part * 32);
        float exact = 0.f;
        // the polynomial takes both its terms from the rounded A: their errors then go against each other
        if constexpr (CL) {
            // this CTA's share of the sums, in 32 bits, in the place of the polynomial and the two blocks behind it
            uint8_t* share = poly + row * 512 + part * 128;
#pragma unroll
            for (int c = 0; c < 8; ++c)
                *reinterpret_cast<float4*>(share + ((c ^ (row & 7)) << 4)) = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
            cluster_sync_all();
            const int each = (4096 + p.cluster - 1) / p.cluster, end = min(4096, (rank + 1) * each);
            for (int u = rank * each + threadIdx.x; u < end; u += kSmallThreads) {
                const int r = u / 32, c = u % 32;  // four columns from 4 * c
                const uint32_t off = poly_at + r * 512 + (c / 8) * 128 + (((c % 8) ^ (r & 7)) << 4);
                float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                for (int q = 0; q < p.cluster; ++q) {
                    float4 e;
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                 : "=f"(e.x), "=f"(e.y), "=f"(e.z), "=f"(e.w)
                                 : "r"(map_to_rank(off, q))
                                 : "memory");
                    t.x += e.x, t.y += e.y, t.z += e.z, t.w += e.w;
                }
                t.x *= f, t.y *= f, t.z *= f, t.w *= f;
                const uint32_t to = gram_at + (c / 16) * kBlockBytes + r * 128 + (((c % 16 / 2) ^ (r & 7)) << 4) + (c & 1) * 8;
                const uint32_t lo = Half16::pack(t.x, t.y, true), hi = Half16::pack(t.z, t.w, true);
                const bool diagonal = r / 4 == c;
                const float own = r % 4 == 0 ? t.x : r % 4 == 1 ? t.y : r % 4 == 2 ? t.z : t.w;
                for (int q = 0; q < p.cluster; ++q) {
                    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(map_to_rank(to, q)), "r"(lo), "r"(hi) : "memory");
                    if (diagonal) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(map_to_rank(smem_u32(&s_diag[r]), q)), "f"(own) : "memory");
                }
            }
            cluster_sync_all();
            exact = s_diag[row];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint4 e = *reinterpret_cast<const uint4*>(gram + (part / 2) * kBlockBytes + row * 128 + ((((part & 1) * 4 + c) ^ (row & 7)) << 4));
                const uint32_t w[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                    v[8 * c + 2 * i] = h.x, v[8 * c + 2 * i + 1] = h.y;
                }
            }
        } else {
            if (d < 32u) {
#pragma unroll
                for (int i = 0; i < 32; ++i) exact = d == (unsigned)i ? v[i] : exact;
                exact *= f;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __half2float(__float2half_rn(v[i] * f));
            put(gram, row, part, v, true);
        }
        ready();
        square(gram_at, 2);
        wait();
        {
            float u[32];
            tmem_load(tmem + part * 32 + lanes, u);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = fmaf(p.c, u[i], p.b * v[i]);
            if (d < 32u) {  // all of a warp or none
                float own = 0.f;
#pragma unroll
                for (int i = 0; i < 32; ++i) own = d == (unsigned)i ? v[i] : own;
                own = mend_diagonal(own, exact, p.a, p.b, p.c);
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = d == (unsigned)i ? own : v[i];
                s_regain[row] = regain_row(own);
            }
        }
        put(poly, row, part, v, true);
        ready();
        if (warp == 0) {
            const uint64_t da = operand_desc(poly_at, false, 0);
            if (elect_one()) {
                for (int n0 = 0; n0 < blocks; n0 += 4) {
                    const int n = min(4, blocks - n0);
                    const uint64_t db = operand_desc(x_at + n0 * kBlockBytes, true, kBlockBytes);
                    const uint32_t idesc = (1u << 4) | (1u << 16) | ((uint32_t)(64 * n / 8) << 17) | ((uint32_t)(128 / 16) << 24);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        mma_f16<1>(tmem + 64 * n0, da + (uint64_t)((j / 4) * (kBlockBytes >> 4) + (j % 4) * 2), db + (uint64_t)(j * (2048 >> 4)), idesc, j != 0);
                }
                mma_commit<1>(bar);
            }
            __syncwarp();
        }
        const bool last = k + 1 == p.steps;
        bound = bound_after(bound, p.a, p.b, p.c);
        const float times = last ? 1.f : kept_times(bound, p.unit), fx = back * times * s_regain[row];
        back = inverse_of_power(times);
        wait();
        for (int n = part; n < 2 * blocks; n += kSmallThreads / 128) {
            tmem_load(tmem + 32 * n + lanes, v);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= fx;
            put(x, row, n, v, !last);
        }
        ready();
    }
    // the result lies in the place of X, as bfloat16
    uint16_t* out = p.out + (int64_t)matrix * g.m * g.n + (tall ? (int64_t)c0 * g.n : c0);
    auto at = [&](int r, int c) { return x + (c / 64) * kBlockBytes + r * 128 + (((c % 64 / 8) ^ (r & 7)) << 4) + (c % 8) * 2; };
    for (int r = warp; r < my_rows; r += kSmallThreads / 32) {
        if (p.wide && !tall) {
            for (int c = lane * 8; c < my_cols; c += 256) *reinterpret_cast<uint4*>(out + (int64_t)r * g.n + c) = *reinterpret_cast<const uint4*>(at(r, c));
        } else {
            for (int c = lane; c < my_cols; c += 32) out[(int64_t)r * g.n + c] = *reinterpret_cast<const uint16_t*>(tall ? at(c, r) : at(r, c));
        }
    }
    if (!arrived.ok) let_copies_end();
    __syncthreads();
    if (warp == 0) tmem_free<1>(tmem, cols);
    if constexpr (CL) cluster_sync_all();
}

inline size_t up(size_t x, size_t a) { return (x + a - 1) / a * a; }

int64_t tiles_of(int64_t rows, int64_t cols, int64_t b) { return ((rows + b - 1) / b) * ((cols + b - 1) / b); }
int64_t half_tiles_of(int64_t s, int64_t b) { return ((s + b - 1) / b) * ((s + b - 1) / b + 1) / 2; }

// How a matrix whose shorter side is at most 128 is spread over a cluster: CTAs, and blocks of 64 columns of the longer side
// that a CTA has; {0, 0} where it does not fit, or where there are so many that k_ns_steps has work for the whole GPU.
struct Spread {
    int cluster, own;
};
Spread spread_of(int m, int n, int count) {
    const int s = m < n ? m : n, blocks = ((m < n ? n : m) + 63) / 64, most = kSmallLong / 64;
    if (s > kSmallSide) return {0, 0};
    if (blocks <= most) return {1, blocks};
    int own = 4;  // a CTA with 4 blocks has a shorter step than one with 8
    while (own < most && ((blocks + own - 1) / own > 16 || (int64_t)count * ((blocks + own - 1) / own) > kSms)) own *= 2;
    const int cluster = (blocks + own - 1) / own;
    if (cluster > 16 || (int64_t)count * cluster > kSms) return {0, 0};
    return {cluster, own};
}

// Pairs of CTAs or single ones, and the parts of the Gram matrix's K: the smallest time by the rule of use_pairs. In units
// of 256 cycles, a product takes its waves times its stages (and about 32 for the meeting of the blocks, filling the ring
// and storing the last tile); joining parts is a round of its own that reads and writes their sums.
struct Plan {
    bool pairs;
    int parts;
};
Plan plan_of(int m, int n, int count) {
    const int s = m < n ? m : n;
    Plan best = {true, 1};
    double least = 0;
    const int nl = ((m < n ? n : m) + kTileK - 1) / kTileK, ns = (s + kTileK - 1) / kTileK;
    for (int cg = 2; cg >= 1; --cg) {
        const int64_t b = 128 * cg, slots = kSms / cg, half = half_tiles_of(s, b) * count, whole = tiles_of(m, n, b) * count;
        const double unit = cg == 2 ? 2.0 : kSmallCost;
        const double rest = (double)((half + slots - 1) / slots) * (ns * unit + 32) + (double)((whole + slots - 1) / slots) * (ns * unit + 32);
        for (int parts = 1; parts <= 32 && parts <= nl; ++parts) {
            const int part = (nl + parts - 1) / parts;
            if (parts > 1 && (int64_t)(parts - 1) * part >= nl) continue;  // no part is empty
            const double bytes = parts > 1 ? 6.0 * parts * s * s * count : 0.0;  // half of the square, written and read
            if (bytes > 512e6) break;
            const double join = parts > 1 ? 32 + bytes / 0.6e6 : 0.0;
            const double cost = (double)((half * parts + slots - 1) / slots) * (part * unit + 32) + join + rest;
            if (least == 0 || cost < least) least = cost, best = {cg == 2, parts};
        }
    }
    return best;
}

struct Layout {
    size_t counter, scales, sums, x0, x1, gram, poly, diag, regain, part, total;
    int64_t ldx, lds, ld_part;
    int s;
    Plan plan;
};
Layout layout(int32_t count, int32_t m, int32_t n) {
    Layout L = {};
    if (spread_of(m, n, count).cluster) {
        L.total = 256;  // nothing, but never a size of zero
        return L;
    }
    L.s = m < n ? m : n;
    L.plan = plan_of(m, n, count);
    // Rows on 128-byte lines: on 16-byte boundaries alone, stores and loads split sectors and lines (5230 x 1832, two: 638
    // us instead of 532; 200 x 200: 80 instead of 70).
    L.ldx = (int64_t)up(n, 64);
    L.lds = (int64_t)up(L.s, 64);
    L.ld_part = (int64_t)up(L.s, 32);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = up(at + bytes, 256);
        return here;
    };
    L.counter = take(256);
    L.scales = take((size_t)(kScaled + 2) * count * sizeof(float2));
    L.sums = take((size_t)(count > kNormBlocks ? count : kNormBlocks) * 8);
    L.x0 = take((size_t)count * m * L.ldx * 2);
    L.x1 = take((size_t)count * m * L.ldx * 2);
    L.gram = take((size_t)count * L.s * L.lds * 2);
    L.poly = take((size_t)count * L.s * L.lds * 2);
    L.diag = take((size_t)count * L.s * 4);
    L.regain = take((size_t)count * L.s * 4);
    L.part = take(L.plan.parts > 1 ? (size_t)L.plan.parts * count * L.s * L.ld_part * 4 : 0);
    L.total = at;
    return L;
}

template <int CG, bool CUT, bool TALL>
cudaError_t launch_steps(const StepsMaps& maps, const StepsArgs& p, cudaStream_t stream) {
    auto kernel = k_ns_steps<CG, CUT, TALL>;
    static std::atomic<uint64_t> ready{0};
    cudaError_t err = allow_smem(kernel, kMatSmem, ready);
    if (err != cudaSuccess) return err;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kMatThreads<kStepWarps>);
    cfg.dynamicSmemBytes = kMatSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CG;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CG == 2 ? 2 : 1;
    int64_t slots = device_sms();
    if (CG == 2) {  // pairs that fit at a time: an SM without a neighbour stays out
        static std::atomic<int> fit[64];
        int dev = 0, n = 0;
        err = cudaGetDevice(&dev);
        if (err != cudaSuccess) return err;
        n = fit[dev & 63].load(std::memory_order_relaxed);
        if (!n) {
            cfg.gridDim = dim3(2);
            cfg.attrs = attr + 1;
            cfg.numAttrs = 1;
            err = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
            if (err != cudaSuccess) return err;
            if (n < 1) return cudaErrorInvalidConfiguration;
            fit[dev & 63].store(n, std::memory_order_relaxed);
            cfg.attrs = attr;
            cfg.numAttrs = 2;
        }
        slots = n;
    }
    const int64_t b = 128 * CG, half = half_tiles_of(p.s, b) * p.count * p.parts, whole = tiles_of(p.m, p.n, b) * p.count, most = half > whole ? half : whole;
    if (most > 0x7FFFFFFF) return cudaErrorInvalidValue;
    cfg.gridDim = dim3((unsigned)((most < slots ? most : slots) * CG));
    return cudaLaunchKernelEx(&cfg, kernel, maps, p);
}

template <int CG>
cudaError_t launch_steps_cg(const StepsMaps& maps, const StepsArgs& p, cudaStream_t stream) {
    if (p.parts > 1) return p.tall ? launch_steps<CG, true, true>(maps, p, stream) : launch_steps<CG, true, false>(maps, p, stream);
    return p.tall ? launch_steps<CG, false, true>(maps, p, stream) : launch_steps<CG, false, false>(maps, p, stream);
}

cudaError_t launch_small(const Source& src, const SmallArgs& sa, int count, cudaStream_t stream) {
    const bool cl = sa.cluster > 1;
    auto kernel = cl ? k_ns_small<true> : k_ns_small<false>;
    static std::atomic<uint64_t> ready[2];
    cudaError_t err = allow_smem(kernel, (kSmallLong / 64 + 6) * kBlockBytes + 1024, ready[cl]);
    if (err != cudaSuccess) return err;
    if (sa.cluster > 8) {  // more CTAs than a portable cluster has
        err = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (err != cudaSuccess) return err;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(count * sa.cluster));
    cfg.blockDim = dim3(kSmallThreads);
    cfg.dynamicSmemBytes = (sa.own + (cl ? 6 : 4)) * kBlockBytes + 1024;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = sa.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, src, sa);
}

bool bad_sizes(int32_t count, int32_t m, int32_t n) {
    return count < 1 || m < 1 || n < 1 || count > 65535 || m > (1 << 20) || n > (1 << 20);
}

}  // namespace

const WaitControl update_waits = {take_expired, limit_waits, wait_for_nothing};

}  // namespace ones

using namespace ones;

extern "C" {

size_t ones_orthogonalize_workspace_bytes(int32_t count, int32_t m, int32_t n) {
    if (bad_sizes(count, m, n)) return 0;
    return layout(count, m, n).total;
}

int ones_orthogonalize(const void* d_g, int64_t ldg, int64_t stride, int32_t count, int32_t m, int32_t n, int32_t type,
                       int32_t steps, float a, float b, float c, float eps, void* d_out, void* d_workspace,
                       size_t workspace_bytes, void* cuda_stream) {
    if (bad_sizes(count, m, n) || type < ONES_F32 || type > ONES_F16 || steps < 1 || steps > ONES_UPDATE_MAX_STEPS || !(eps > 0.f) || !isfinite(eps) ||
        !isfinite(a) || !isfinite(b) || !isfinite(c) || ldg < n || (count > 1 && stride < 0))
        return ONES_ERR_BAD_PARAM;
    if (!d_g || !d_out || !d_workspace) return ONES_ERR_NULL;
    const int size = type == ONES_F32 ? 4 : 2;
    if (!aligned(d_g, size) || !aligned(d_out, 2) || !aligned(d_workspace, 256)) return ONES_ERR_ALIGN;
    const Layout L = layout(count, m, n);
    if (workspace_bytes < L.total) return ONES_ERR_WORKSPACE;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(d_workspace);
    float2* scales = reinterpret_cast<float2*>(ws + L.scales);
    double* sums = reinterpret_cast<double*>(ws + L.sums);
    __half* x[2] = {reinterpret_cast<__half*>(ws + L.x0), reinterpret_cast<__half*>(ws + L.x1)};
    __half* gram = reinterpret_cast<__half*>(ws + L.gram);
    __half* poly = reinterpret_cast<__half*>(ws + L.poly);
    unsigned* counter = reinterpret_cast<unsigned*>(ws + L.counter);
    const bool wide = n % 8 == 0 && aligned(d_g, 16) && ldg * size % 16 == 0 && stride * size % 16 == 0;
    const Source src = {d_g, ldg, count > 1 ? stride : 0, m, n, type, wide};
    // see kept_times: after the last step X's values are about 1 / 2^q, before the first about 1 / sqrt(m n)
    int q = 0;
    while ((int64_t)1 << (2 * (q + 1)) <= (m > n ? m : n)) ++q;
    const float unit = ldexpf(1.f, q);
    const bool wide_out = n % 8 == 0 && aligned(d_out, 16);
    const Spread on = spread_of(m, n, count);
    if (on.cluster) {
        const SmallArgs sa = {on.cluster, on.own, steps, a, b, c, eps, unit, static_cast<uint16_t*>(d_out), wide_out};
        return launch_small(src, sa, count, stream) == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
    }
    int blocks = (m + kNormThreads / 32 - 1) / (kNormThreads / 32), most = kNormBlocks / count;
    if (blocks > most) blocks = most > 0 ? most : 1;
    k_ns_norm<<<dim3(blocks, count), kNormThreads, 0, stream>>>(src, sums, counter);
    cudaError_t err = cudaGetLastError();
    if (err == cudaSuccess)
        err = launch_after(k_ns_cast, dim3(blocks, count), dim3(kNormThreads), stream, src, static_cast<const double*>(sums), blocks, eps,
                           x[0], L.ldx, Polynomial{steps, a, b, c, unit}, scales);
    StepsArgs p = {};
    p.m = m, p.n = n, p.s = L.s, p.count = count, p.steps = steps, p.tall = m > n;
    p.a = a, p.b = b, p.c = c;
    p.x[0] = x[0], p.x[1] = x[1], p.gram = gram, p.poly = poly, p.out = static_cast<uint16_t*>(d_out);
    p.ldx = L.ldx, p.xs = (int64_t)m * L.ldx, p.lds = L.lds, p.ss = (int64_t)L.s * L.lds;
    p.scales = scales, p.counter = counter;
    p.parts = L.plan.parts;
    p.diag = reinterpret_cast<float*>(ws + L.diag), p.regain = reinterpret_cast<float*>(ws + L.regain);
    p.part = L.plan.parts > 1 ? reinterpret_cast<float*>(ws + L.part) : nullptr;
    p.ld_part = L.ld_part, p.part_stride = (int64_t)count * L.s * L.ld_part;
    p.wide = wide_out;
    StepsMaps maps;
    for (int i = 0; i < 2 && err == cudaSuccess; ++i) {
        err = make_map(&maps.rows[i], {x[i], L.ldx, p.xs, false}, m, n, count, true);
        if (err == cudaSuccess) err = make_map(&maps.cols[i], {x[i], L.ldx, p.xs, true}, n, m, count, true);
    }
    for (int i = 0; i < 2 && err == cudaSuccess; ++i) {
        err = make_map(&maps.gram[i], {gram, L.lds, p.ss, i == 1}, L.s, L.s, count, true);
        if (err == cudaSuccess) err = make_map(&maps.poly[i], {poly, L.lds, p.ss, i == 1}, L.s, L.s, count, true);
    }
    if (err == cudaSuccess) err = L.plan.pairs ? launch_steps_cg<2>(maps, p, stream) : launch_steps_cg<1>(maps, p, stream);
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // extern "C"
