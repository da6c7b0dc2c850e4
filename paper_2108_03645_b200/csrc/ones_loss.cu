// Cross entropy of a projection on a large vocabulary, and its gradients, without keeping the logits.
#include <math.h>

#include "ones_matmul.cuh"
#include "ones_train.h"
#include "ones_train_internal.h"

namespace ones {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The tensor cores cut off, towards zero, what a partial sum of the accumulator cannot hold after every step along K. A
// sum that grows evenly over K steps loses in the mean 2^-30 of itself per value of K (measured: 4.9e-7 at 512, 2.03e-6
// at 2048, 4.07e-6 at 4096 columns, in proportion), and all large logits lose alike, so it is given back: the relative
// error of the loss falls from 1.2e-6 to below 5e-7 at 2048 columns. It enters as part of the factor of the exponent.
// It is a mean for dense rows: a logit that comes from a few columns, the others being zero, loses nothing and is given too
// much. So nothing is given for more columns than were measured: a logit is never off by more than 2^-18 of itself for it.
__device__ __forceinline__ float regain(int k) { return 1.f + (float)min(k, 4096) * 9.3132257e-10f; }

// Softmax statistics of a tile of logits: each thread takes the maximum m and s = sum exp(l - m) of its row's columns
// here, and the logit of the row's target if it meets it. 4096 x 1024 x 50000: 254 us while the card is cool, 1.65 PFLOP/s;
// with few rows the weight's bytes bound it (51 x 3776 x 50260: 65 us, 5.8 TB/s), with few columns the exponentials.
struct EpiStats {
    static constexpr int kWarps = 8;
    struct Args {
        const int64_t* target;
        float2* part;  // [slots][rows], one slot per half tile
        float* at_target;
        int rows, vocab;
    };
    template <int W>
    static __device__ __forceinline__ void tile(const Args& a, const MatShape& g, uint32_t acc, int row, int col, int limit,
                                                const TileAt& at, int half, const Turn<kWarps>&) {
        const float up = regain(g.K), to2 = kLog2e * up;
        const int end = min(a.vocab, limit);
        const int64_t t64 = row < a.rows ? a.target[row] : -1;
        const int t = t64 >= 0 && t64 < a.vocab ? (int)t64 : -1;
        float m = -INFINITY, s = 0.f;
#pragma unroll 1
        for (int c = 0; c < W; c += 32) {
            float v[32];
            tmem_load(acc + c, v);
            const int left = end - (col + c);
            if (left <= 0) break;
            if (left < 32) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i >= left) v[i] = -INFINITY;
            }
            const unsigned at_i = (unsigned)(t - (col + c));
            if (at_i < 32u && t < end) {
                float lt = 0.f;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (at_i == (unsigned)i) lt = v[i];
                a.at_target[row] = lt * up;
            }
            float top = v[0];
#pragma unroll
            for (int i = 1; i < 32; ++i) top = fmaxf(top, v[i]);
            const float next = fmaxf(m, top);
            const float minus = next == -INFINITY ? 0.f : -next;  // nothing but -inf so far: exp gives 0
            s *= exp2_fast((m + minus) * to2);
            // the difference first, which is exact near the maximum: a row that is certain of an entry has s = 1
            Pair s2[2] = {both(0.f), both(0.f)};
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
                const float2 e = split((pair(v[i], v[i + 1]) + both(minus)) * both(to2));
                s2[i / 2 & 1] = s2[i / 2 & 1] + pair(exp2_fast(e.x), exp2_fast(e.y));
            }
            s += total(s2[0] + s2[1]);
            m = next;
        }
        if (row < a.rows) a.part[(int64_t)(at.n * 2 + half) * a.rows + row] = make_float2(m * up, s);
    }
};

// What the backward pass knows of a row that takes part, in the order in which such rows were gathered.
struct RowInfo {
    int target;   // entry of the vocabulary
    float shift;  // -lse / ln 2
    float g;      // dloss * scale
    int row;      // of the caller
};

// Gradient of a piece's logits, as 16 bits: (exp(l - lse) - [target]) * dloss * scale. 4096 x 1024 x 32000: 171 us, 1.57
// PFLOP/s at the clock that the power cap leaves.
struct EpiDlogits {
    static constexpr int kWarps = 16;
    struct Args {
        const RowInfo* info;
        uint16_t* out;
        int64_t ld;
        int rows, first, cols;  // the piece: `cols` entries from `first`
        bool f16, twice;        // twice: what the rounding left goes into a second row of ld / 2 values
    };
    template <int W>
    static __device__ __forceinline__ void tile(const Args& a, const MatShape& shape, uint32_t acc, int row, int col, int limit,
                                                const TileAt&, int, const Turn<kWarps>& turn) {
        constexpr int N = Turn<kWarps>::kHalves;
        const float to2 = kLog2e * regain(shape.K);
        const bool live = row < shape.M;
        RowInfo r = {-1, 0.f, 0.f, 0};
        if (live) r = a.info[row];
        const int t = r.target - a.first;
        // the product with the hidden rows runs over whole stages of rows: those after the last one are zero
        const int rows = min(a.rows, (shape.M + kTileK - 1) / kTileK * kTileK);
        const int end = min(a.cols, limit);
#pragma unroll 1
        for (int c = 0; c < W && col + c < end; c += N) {
            float v[N];
            tmem_load(acc + c, v);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const float2 x = split(fma2(pair(v[i], v[i + 1]), both(to2), both(r.shift)));
                const float2 y = split(pair(exp2_fast(x.x), exp2_fast(x.y)) * both(r.g));
                v[i] = y.x, v[i + 1] = y.y;
            }
            if (!live) {  // 0 * infinity, where the weight holds one, is no zero
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = 0.f;
            }
            const unsigned at_i = (unsigned)(t - (col + c));
            if (live && at_i < (unsigned)N) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (at_i == (unsigned)i) v[i] -= r.g;
            }
            turn.write16(v, a.f16, a.out, a.ld, row - turn.lane, col + c, rows, end, true);
            if (a.twice) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    v[i] -= a.f16 ? __half2float(__float2half_rn(v[i])) : __bfloat162float(__float2bfloat16_rn(v[i]));
                turn.write16(v, a.f16, a.out + a.ld / 2, a.ld, row - turn.lane, col + c, rows, end, true);
            }
        }
    }
};

__device__ __forceinline__ void store_grad4(uint16_t* out, float4 f, int left, bool f16, bool wide) {
    const uint32_t lo = Half16::pack(f.x, f.y, f16), hi = Half16::pack(f.z, f.w, f16);
    if (wide && left >= 4) {
        *reinterpret_cast<uint2*>(out) = make_uint2(lo, hi);
    } else {
        if (left > 0) out[0] = (uint16_t)lo;
        if (left > 1) out[1] = (uint16_t)(lo >> 16);
        if (left > 2) out[2] = (uint16_t)hi;
        if (left > 3) out[3] = (uint16_t)(hi >> 16);
    }
}

// Sum over the pieces: the product is added to (first piece: put into) 32-bit sums; the last piece rounds them into the
// caller's rows, unless the sums come in several parts (k_ce_rows joins those). 4096 x 1024 x 32000: 188 us, 1.43 PFLOP/s on
// 64 of 74 pairs.
struct EpiSum {
    static constexpr int kWarps = 8;
    struct Args {
        float* sum;  // [parts][rows][ld_sum]
        int64_t ld_sum;
        uint16_t* out;
        int64_t ld_out;
        const float* scale;
        const RowInfo* info;
        int rows, cols;
        bool first, last, f16, wide;
    };
    template <int W>
    static __device__ __forceinline__ void tile(const Args& a, const MatShape& shape, uint32_t acc, int row, int col, int limit,
                                                const TileAt& at, int, const Turn<kWarps>& turn) {
        const float unscale = a.last ? 1.f / *a.scale : 1.f;
        const int r0 = row - turn.lane + turn.row_of(0), k = turn.chunk_of();
        const int end = min(a.cols, limit);
#pragma unroll 1
        for (int c = 0; c < W && col + c < end; c += 32) {
            const int at_col = col + c + 4 * k, left = end - at_col;
            float* sum = a.sum + ((int64_t)at.b * a.rows + r0) * a.ld_sum + at_col;  // has whole chunks of 4 columns
            float4 old[8];
            if (!a.first) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (r0 + 4 * i < shape.M && left > 0) old[i] = *reinterpret_cast<const float4*>(sum + 4 * i * a.ld_sum);
            }
            float v[32];
            tmem_load(acc + c, v);
            turn.put32(v);
            uint4 q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = turn.chunk(turn.row_of(i), k);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float4 f = make_float4(__uint_as_float(q[i].x), __uint_as_float(q[i].y), __uint_as_float(q[i].z), __uint_as_float(q[i].w));
                if (!a.first) f.x += old[i].x, f.y += old[i].y, f.z += old[i].z, f.w += old[i].w;
                if (r0 + 4 * i >= shape.M || left <= 0) continue;
                if (!a.last) {
                    *reinterpret_cast<float4*>(sum + 4 * i * a.ld_sum) = f;
                    continue;
                }
                f.x *= unscale, f.y *= unscale, f.z *= unscale, f.w *= unscale;
                store_grad4(a.out + (int64_t)a.info[r0 + 4 * i].row * a.ld_out + at_col, f, left, a.f16, a.wide);
            }
        }
    }
};

// A piece's rows of dweight, complete: scaled back and rounded. 4096 x 1024 x 32000: 171 us, 1.57 PFLOP/s. With few rows the
// way out bounds it: 51 x 3776 x 50260 writes 380 MB in 110 us, 3.5 TB/s.
struct EpiGrad {
    static constexpr int kWarps = 16;
    struct Args {
        void* out;
        int64_t ld;
        const float* scale;
        int rows, cols;
        bool f32, f16, wide;
    };
    // 16-bit rows that start anywhere. A window of 32 columns is moved back, for each row by itself, to where the row meets
    // a 32-byte boundary; the up to 15 columns before its own are the neighbour's, and still in the accumulator. So only
    // the ends of a tile's rows are written in less than 16 bytes. first, last: the tile's columns. Writing
    // pairs of columns from each window's own start instead, the backward pass of 62 x 871 x 75300 took 259 us for 239.
    template <int W>
    static __device__ __forceinline__ void odd_rows(const Args& a, float unscale, uint32_t acc, int row, int col, int first, int last,
                                                    const Turn<kWarps>& turn) {
        static_assert(Turn<kWarps>::kHalves == 32, "");
        uint16_t* out = static_cast<uint16_t*>(a.out);
        auto phase = [&](int r) { return (int)(reinterpret_cast<uintptr_t>(out + (int64_t)r * a.ld + col) >> 1) & 15; };
        const int back = 16 - phase(row), row0 = row - turn.lane;
        const bool ends = last <= col + W;  // the tile's last column is this warp's
#pragma unroll 1
        for (int c = 0; c < W + 32; c += 32) {
            const bool extra = col + c >= last;  // what is moved back out of the last window
            if ((c == W || extra) && (!ends || col + c >= last + 32)) break;
            uint32_t w[24];
            if (col + c > first) {
                float v[16];
                tmem_load(acc + c - 16, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = Half16::pack(v[2 * i] * unscale, v[2 * i + 1] * unscale, a.f16);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = 0;
            }
            if (!extra) {
                float v[32];
                tmem_load(acc + c, v);
#pragma unroll
                for (int i = 0; i < 16; ++i) w[8 + i] = Half16::pack(v[2 * i] * unscale, v[2 * i + 1] * unscale, a.f16);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) w[8 + i] = 0;
            }
            // the 32 values from `back` (1 to 16) on
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = back & 16 ? w[i + 8] : w[i];
#pragma unroll
            for (int i = 0; i < 20; ++i) w[i] = back & 8 ? w[i + 4] : w[i];
#pragma unroll
            for (int i = 0; i < 18; ++i) w[i] = back & 4 ? w[i + 2] : w[i];
#pragma unroll
            for (int i = 0; i < 17; ++i) w[i] = back & 2 ? w[i + 1] : w[i];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], back & 1 ? 16 : 0);
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 4; ++k) turn.chunk(turn.lane, k) = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
            __syncwarp();
            uint4 q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = turn.chunk(turn.row_of(i), turn.chunk_of());
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = row0 + turn.row_of(i), at = col + c - phase(r) + 8 * turn.chunk_of();
                if (r >= a.rows) continue;
                uint16_t* p = out + (int64_t)r * a.ld + at;
                if (at >= first && at + 8 <= last) {
                    *reinterpret_cast<uint4*>(p) = q[i];
                } else {
                    const int to = min(last - at, 8);
                    int k = max(first - at, 0);
                    if (k < to && k & 1) p[k] = turn.half_at(turn.row_of(i), 8 * turn.chunk_of() + k), ++k;
                    for (; k + 1 < to; k += 2) *reinterpret_cast<uint32_t*>(p + k) = turn.word_at(turn.row_of(i), 4 * turn.chunk_of() + k / 2);
                    if (k < to) p[k] = turn.half_at(turn.row_of(i), 8 * turn.chunk_of() + k);
                }
            }
        }
    }
    template <int W>
    static __device__ __forceinline__ void tile(const Args& a, const MatShape& shape, uint32_t acc, int row, int col, int limit,
                                                const TileAt& at, int, const Turn<kWarps>& turn) {
        const float unscale = 1.f / *a.scale;
        const bool none = shape.K == 0;  // no row takes part: nothing was multiplied
        const int row0 = row - turn.lane;
        const int end = min(a.cols, limit);
        if (!a.f32 && !a.wide && !none) {
            if (col < end) odd_rows<W>(a, unscale, acc, row, col, at.n * shape.width, min(a.cols, (at.n + 1) * shape.width), turn);
            return;
        }
        constexpr int N = Turn<kWarps>::kHalves;
#pragma unroll 1
        for (int c = 0; c < W && col + c < end; c += N) {
            float v[N];
            tmem_load(acc + c, v);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = none ? 0.f : v[i] * unscale;
            if (a.f32) {
                float u[N / 2];
#pragma unroll
                for (int h = 0; h < N; h += N / 2) {
#pragma unroll
                    for (int i = 0; i < N / 2; ++i) u[i] = v[h + i];
                    turn.write32(u, static_cast<float*>(a.out), a.ld, row0, col + c + h, a.rows, end, a.wide);
                }
            } else {
                turn.write16(v, a.f16, static_cast<uint16_t*>(a.out), a.ld, row0, col + c, a.rows, end, a.wide);
            }
        }
    }
};

// Joins the slots of a row: R rows a block, 512 / R threads on a row's slots, 8 slots on their way at a time. With few
// rows R = 4 (a warp reads whole 32-byte sectors) brings more threads to a row, else R = 8.
constexpr int kJoinThreads = 512;

__device__ __forceinline__ float2 join(float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x);
    const float minus = m == -INFINITY ? 0.f : -m;
    return make_float2(m, a.y * exp2_fast((a.x + minus) * kLog2e) + b.y * exp2_fast((b.x + minus) * kLog2e));
}

template <int R>
__global__ void __launch_bounds__(kJoinThreads) k_ce_join(const float2* part, int slots, const float* at_target, const int64_t* target,
                                                          int rows, int vocab, float* loss, float* lse) {
    wait_for_predecessor();
    __shared__ float2 s[kJoinThreads];
    const int r = threadIdx.x % R, row = blockIdx.x * R + r;
    float2 v = make_float2(-INFINITY, 0.f);
    if (row < rows) {
        constexpr int kStep = kJoinThreads / R;
        for (int i = threadIdx.x / R; i < slots; i += 8 * kStep) {
            float2 q[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                q[j] = i + j * kStep < slots ? part[(int64_t)(i + j * kStep) * rows + row] : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int d = 4; d; d /= 2) {
#pragma unroll
                for (int j = 0; j < d; ++j) q[j] = join(q[j], q[j + d]);
            }
            v = join(v, q[0]);
        }
    }
    s[threadIdx.x] = v;
    __syncthreads();
    for (int n = kJoinThreads / 2; n >= R; n /= 2) {
        if ((int)threadIdx.x < n) s[threadIdx.x] = v = join(v, s[threadIdx.x + n]);
        __syncthreads();
    }
    if ((int)threadIdx.x < R && row < rows) {
        const float l = v.x + logf(v.y);
        const int64_t t = target[row];
        lse[row] = l;
        loss[row] = t >= 0 && t < vocab ? l - at_target[row] : 0.f;
    }
}

struct Header {
    int live;     // rows that take part
    float scale;  // see below
};

// Finds the rows that take part, in order, and the factor that brings their largest |dloss| to `goal`, so that the 16-bit
// gradients of the logits neither overflow nor lose their small values, whatever the scale of the loss. Where all rows have
// the same dloss, the entries at the targets, -(1 - p), then lie below a power of two and are rounded by at most 2^-9 of it
// (bfloat16); scaled by a power of two they would all lie at one place in [1, 2) and be off in one direction (error of the
// gradients against 64 bits for 1/100 each: 2.5e-3 of their norm instead of 2.0e-3). The goal is 1 for bfloat16, whose range
// is float32's, and 2^15 for float16, the most that its range holds: p * dloss of a large vocabulary reaches far down, and
// further in rows that weigh less than others. With a goal of 1, 32001 entries and rows of 1/1000 of the weight, half of all
// p * dloss would be nothing. One block, 8192 rows at a time: 3 us for so many.
constexpr int kScan = 8;
__global__ void __launch_bounds__(1024) k_ce_scan(const float* dloss, const int64_t* target, int rows, int vocab, float goal, RowInfo* info,
                                                     Header* head) {
    __shared__ int s_count[32];
    __shared__ float s_top[32];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    float top = 0.f;
    int base = 0;
    for (int r0 = 0; r0 < rows; r0 += 1024 * kScan) {
        const int first = r0 + warp * 32 * kScan + lane;
        int64_t t[kScan];
        float g[kScan];
#pragma unroll
        for (int i = 0; i < kScan; ++i) {
            t[i] = first + 32 * i < rows ? target[first + 32 * i] : -1;
            g[i] = first + 32 * i < rows ? dloss[first + 32 * i] : 0.f;
        }
        unsigned in[kScan];
        int n = 0;
#pragma unroll
        for (int i = 0; i < kScan; ++i) {
            const bool live = t[i] >= 0 && t[i] < vocab;
            if (live) top = fmaxf(top, fabsf(g[i]));
            in[i] = __ballot_sync(0xFFFFFFFFu, live);
            n += __popc(in[i]);
        }
        if (lane == 0) s_count[warp] = n;
        __syncthreads();
        int up_to = s_count[lane];  // by the warps up to the lane's
        for (int o = 1; o < 32; o *= 2) {
            const int u = __shfl_up_sync(0xFFFFFFFFu, up_to, o);
            if (lane >= o) up_to += u;
        }
        int at = base + __shfl_sync(0xFFFFFFFFu, up_to, warp) - n;
        base += __shfl_sync(0xFFFFFFFFu, up_to, 31);
#pragma unroll
        for (int i = 0; i < kScan; ++i) {
            if (in[i] >> lane & 1) info[at + __popc(in[i] & ((1u << lane) - 1))].row = first + 32 * i;
            at += __popc(in[i]);
        }
        __syncthreads();
    }
    for (int o = 16; o; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if (lane == 0) s_top[warp] = top;
    __syncthreads();
    if (threadIdx.x < 32) {
        top = s_top[threadIdx.x];
        for (int o = 16; o; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if (threadIdx.x == 0) {
            constexpr float kMost = 8.507059e37f;  // 2^126: its inverse is a normal number, too
            head->scale = top > 0.f && top < INFINITY ? fminf(goal / top, kMost) : 1.f;
            head->live = base;
        }
    }
    let_successor_start();
}

// Gathers the hidden rows that take part (and zeros up to a whole stage of rows), what the other kernels need to know of
// them, and clears the gradients of the rows that take none. A warp takes a row at a time.
__global__ void __launch_bounds__(256) k_ce_gather(const uint16_t* hidden, int64_t ldh, const int64_t* target, const float* dloss,
                                                   const float* lse, int rows, int cols, int vocab, const Header* head, RowInfo* info,
                                                   uint16_t* out, int64_t ld_out, int times, uint16_t* dhidden, int64_t lddh, bool wide_in,
                                                   bool wide_dh) {
    wait_for_predecessor();
    let_successor_start();
    const int lane = threadIdx.x % 32, live = head->live;
    const float scale = head->scale;
    const int padded = min(rows, (live + kTileK - 1) / kTileK * kTileK);
    for (int i = blockIdx.x * 8 + threadIdx.x / 32; i < rows; i += gridDim.x * 8) {
        if (i < padded) {
            const int row = i < live ? info[i].row : -1;
            const uint16_t* from = hidden + (int64_t)row * ldh;
            const int whole = wide_in || row < 0 ? cols / 8 : 0;  // ld_out is a multiple of 8
            for (int k = 0; k < times; ++k) {
                uint16_t* to = out + ((int64_t)i * times + k) * ld_out;
                for (int c = lane; c < whole; c += 32)
                    reinterpret_cast<uint4*>(to)[c] = row >= 0 ? reinterpret_cast<const uint4*>(from)[c] : make_uint4(0, 0, 0, 0);
                for (int c = whole * 8 + lane; c < cols; c += 32) to[c] = row >= 0 ? from[c] : 0;
            }
            __syncwarp();
            if (lane == 0 && row >= 0) {
                RowInfo r;
                r.target = (int)target[row];
                r.shift = -lse[row] * kLog2e;
                r.g = dloss[row] * scale;
                r.row = row;
                info[i] = r;
            }
        }
        const int64_t t = target[i];
        if (t < 0 || t >= vocab) {
            uint16_t* to = dhidden + (int64_t)i * lddh;
            const int whole = wide_dh ? cols / 8 : 0;
            for (int c = lane; c < whole; c += 32) reinterpret_cast<uint4*>(to)[c] = make_uint4(0, 0, 0, 0);
            for (int c = whole * 8 + lane; c < cols; c += 32) to[c] = 0;
        }
    }
}

// Four values of a row out of the parts of a product, in their order.
__device__ __forceinline__ float4 join_parts(const float* p, int64_t part, int parts, float scale) {
    float4 f = *reinterpret_cast<const float4*>(p);
#pragma unroll 8
    for (int k = 1; k < parts; ++k) {
        const float4 q = *reinterpret_cast<const float4*>(p + k * part);
        f.x += q.x, f.y += q.y, f.z += q.z, f.w += q.w;
    }
    f.x *= scale, f.y *= scale, f.z *= scale, f.w *= scale;
    return f;
}

// Joins the parts of the sums over the vocabulary and rounds them into the caller's rows. A warp takes 128 columns of a
// row, so that few rows fill the SMs too.
__global__ void __launch_bounds__(256) k_ce_rows(const float* sum, Cut cut, int plan_nk, int64_t ld_sum, int rows, int cols, const Header* head,
                                                 const RowInfo* info, uint16_t* out, int64_t ld_out, bool f16, bool wide) {
    wait_for_predecessor();
    const int groups = (cols + 127) / 128;
    const float unscale = 1.f / head->scale;
    const int64_t part = (int64_t)rows * ld_sum, items = (int64_t)head->live * groups;
    const int parts = parts_of(cut, head->live, cols, plan_nk);
    for (int64_t w = blockIdx.x * 8 + threadIdx.x / 32; w < items; w += gridDim.x * 8) {
        const int i = (int)(w / groups), c = (int)(w % groups) * 128 + threadIdx.x % 32 * 4;
        if (c >= cols) continue;
        store_grad4(out + (int64_t)info[i].row * ld_out + c, join_parts(sum + (int64_t)i * ld_sum + c, part, parts, unscale), cols - c, f16, wide);
    }
}

// The same for dweight's parts, over the rows that take part. With them 15006 x 72 x 899 takes 60 us backward, without 135:
// eight tiles, each with all of the rows.
__global__ void __launch_bounds__(256) k_ce_weight_rows(const float* sum, Cut cut, int fold, int64_t ld_sum, int rows, int cols, const Header* head,
                                                        void* out, int64_t ld_out, bool f32, bool f16, bool wide) {
    wait_for_predecessor();
    let_successor_start();
    const int groups = (cols + 127) / 128, nk = (head->live * fold + kTileK - 1) / kTileK;
    const float unscale = 1.f / head->scale;
    const int64_t part = (int64_t)rows * ld_sum, items = (int64_t)rows * groups;
    const int parts = nk ? parts_of(cut, rows, cols, nk) : 0;
    for (int64_t w = blockIdx.x * 8 + threadIdx.x / 32; w < items; w += gridDim.x * 8) {
        const int i = (int)(w / groups), c = (int)(w % groups) * 128 + threadIdx.x % 32 * 4, left = cols - c;
        if (left <= 0) continue;
        const float4 f = parts ? join_parts(sum + (int64_t)i * ld_sum + c, part, parts, unscale) : make_float4(0.f, 0.f, 0.f, 0.f);
        if (f32) {
            float* to = static_cast<float*>(out) + (int64_t)i * ld_out + c;
            to[0] = f.x;
            if (left > 1) to[1] = f.y;
            if (left > 2) to[2] = f.z;
            if (left > 3) to[3] = f.w;
        } else {
            store_grad4(static_cast<uint16_t*>(out) + (int64_t)i * ld_out + c, f, left, f16, wide);
        }
    }
}

// Rows that start anywhere, copied to rows on 16-byte boundaries. A thread puts together 16 bytes out of the two aligned
// blocks that hold them: four words from a distance that is the same along a row, shifted by half a word where that is
// odd. Bytes bound it: 75300 x 871 in about 50 us, 5.3 TB/s read and written.
constexpr int kAlignThreads = 256, kAlignEach = 4;
__global__ void __launch_bounds__(kAlignThreads) k_align_rows(const uint16_t* src, int64_t lds, int64_t rows, int cols, uint16_t* dst, int64_t ldd) {
    const int chunks = (cols + 7) / 8;
    const int64_t total = rows * chunks, step = (int64_t)gridDim.x * kAlignThreads * kAlignEach;
    const uintptr_t begin = reinterpret_cast<uintptr_t>(src), end = reinterpret_cast<uintptr_t>(src + (rows - 1) * lds + cols);
    for (int64_t at = (int64_t)blockIdx.x * kAlignThreads * kAlignEach + threadIdx.x; at < total; at += step) {
        int64_t row = at / chunks;
        int k = (int)(at - row * chunks);
        uint4 lo[kAlignEach], hi[kAlignEach];
        const uint16_t* from[kAlignEach];
        uint16_t* to[kAlignEach];
        int left[kAlignEach];
#pragma unroll
        for (int i = 0; i < kAlignEach; ++i) {
            from[i] = src + row * lds + 8 * k;
            to[i] = dst + row * ldd + 8 * k;
            left[i] = at + i * kAlignThreads < total ? min(8, cols - 8 * k) : 0;
            const uintptr_t a = reinterpret_cast<uintptr_t>(from[i]), block = a & ~(uintptr_t)15;
            lo[i] = hi[i] = make_uint4(0, 0, 0, 0);
            if (left[i] > 0) {
                if (block >= begin && block + 32 <= end) {
                    lo[i] = __ldg(reinterpret_cast<const uint4*>(block));
                    hi[i] = __ldg(reinterpret_cast<const uint4*>(block) + 1);
                } else {  // a block that reaches over the ends
                    uint32_t w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uintptr_t p = block + 4 * j;
                        const uint32_t x = p >= begin && p + 2 <= end ? *reinterpret_cast<const uint16_t*>(p) : 0;
                        const uint32_t y = p + 2 >= begin && p + 4 <= end ? *reinterpret_cast<const uint16_t*>(p + 2) : 0;
                        w[j] = x | y << 16;
                    }
                    lo[i] = make_uint4(w[0], w[1], w[2], w[3]), hi[i] = make_uint4(w[4], w[5], w[6], w[7]);
                }
            }
            k += kAlignThreads;
            if (k >= chunks) row += k / chunks, k %= chunks;
        }
#pragma unroll
        for (int i = 0; i < kAlignEach; ++i) {
            if (left[i] <= 0) continue;
            const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(from[i]) & 15;
            uint32_t w[8] = {lo[i].x, lo[i].y, lo[i].z, lo[i].w, hi[i].x, hi[i].y, hi[i].z, hi[i].w};
#pragma unroll
            for (int j = 0; j < 6; ++j) w[j] = off & 8 ? w[j + 2] : w[j];
#pragma unroll
            for (int j = 0; j < 5; ++j) w[j] = off & 4 ? w[j + 1] : w[j];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j] = __funnelshift_r(w[j], w[j + 1], off & 2 ? 16 : 0);
                if (left[i] < 2 * j + 2) w[j] &= left[i] <= 2 * j ? 0u : 0xFFFFu;  // zeros behind the last column
            }
            *reinterpret_cast<uint4*>(to[i]) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

inline size_t up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Columns of a tile of logits where the rows fill one tile at most (0: the usual): the weight's rows pass once and that is
// all the time, so they are spread evenly over the SMs, in as few rounds of tiles as there have to be.
inline int width_of(int32_t rows, int32_t vocab) {
    if (rows > 128) return 0;
    const int rounds = (vocab + 128 * kSms - 1) / (128 * kSms);
    return (int)up((size_t)((vocab + kSms * rounds - 1) / (kSms * rounds)), 16);
}

inline int slots_of(int32_t rows, int32_t vocab) {
    const int narrow = width_of(rows, vocab), w = narrow ? narrow : use_pairs(rows, vocab, 1, false) ? 256 : 128;
    return (vocab + w - 1) / w * 2;
}

struct ForwardLayout {
    size_t part, at_target, total;
};
ForwardLayout forward_layout(int32_t rows, int32_t vocab) {
    ForwardLayout L;
    L.part = 0;
    L.at_target = up((size_t)slots_of(rows, vocab) * rows * sizeof(float2), 256);
    L.total = up(L.at_target + (size_t)rows * 4, 256);
    return L;
}

// Entries of the vocabulary per piece. Default: as many as give 256 MiB of 16-bit gradients, spread evenly.
int32_t piece_of(int32_t rows, int32_t vocab, int32_t piece) {
    const int64_t whole = (int64_t)up(vocab, 256);
    if (piece > 0) return (int32_t)(piece < whole ? piece : whole);
    int64_t most = ((int64_t)128 << 20) / (rows > 0 ? rows : 1) / 256 * 256;
    if (most < 2048) most = 2048;
    const int64_t n = (vocab + most - 1) / most;
    return (int32_t)up((size_t)((vocab + n - 1) / n), 256);
}

// With few rows an error is not averaged over many products, and the time goes by the weight's bytes: the gradients of the
// logits are kept as two 16-bit terms then, the rounded value and what the rounding left (each row twice in the gathered
// rows, so that both terms meet it), and nothing but the roundings of the results is left of the 16 bits: 1.7e-3 of the
// norm for bfloat16 instead of up to 3.9e-3.
constexpr int32_t kFewRows = 64;
inline int fold_of(int32_t rows) { return rows <= kFewRows ? 2 : 1; }

struct BackwardLayout {
    size_t head, info, hidden, dlogits, sum, wsum, total;
    int64_t ld_sum, ld_hidden;
    int32_t piece;
    int fold;
    Cut cut;   // of the product over a piece of the vocabulary
    Cut wcut;  // of a piece's product over the rows: many rows and a small weight are few tiles with a long K
};
BackwardLayout backward_layout(int32_t rows, int32_t cols, int32_t vocab, int32_t piece) {
    BackwardLayout L;
    L.piece = piece_of(rows, vocab, piece);
    L.fold = fold_of(rows);
    L.cut = cut_of(rows, cols, (int)up(vocab < L.piece ? vocab : L.piece, kTileK) * L.fold);
    const int32_t entries = vocab < L.piece ? vocab : L.piece;
    L.wcut = cut_of(entries, cols, rows * L.fold);
    const int64_t edge = L.wcut.pairs ? 256 : 128, tiles = (entries + edge - 1) / edge * ((cols + edge - 1) / edge), most = (L.wcut.pairs ? kSms / 2 : kSms) / tiles;
    if (L.wcut.splits > most) L.wcut.splits = most > 1 ? (int)most : 1;
    L.ld_sum = (int64_t)up(cols, 32);
    L.ld_hidden = (int64_t)up(cols, 64);  // rows on 128-byte lines
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = up(at + bytes, 256);
        return here;
    };
    L.head = take(sizeof(Header));
    L.info = take((size_t)rows * sizeof(RowInfo));
    L.hidden = take((size_t)rows * L.fold * L.ld_hidden * 2);
    L.dlogits = take((size_t)rows * L.fold * L.piece * 2);
    L.sum = take(L.piece < vocab || L.cut.splits > 1 ? (size_t)L.cut.splits * rows * L.ld_sum * 4 : 0);
    L.wsum = take(L.wcut.splits > 1 ? (size_t)L.wcut.splits * entries * L.ld_sum * 4 : 0);
    L.total = at;
    return L;
}

bool bad_sizes(int32_t rows, int32_t cols, int32_t vocab) {
    return rows < 0 || cols < 1 || vocab < 1 || rows > (1 << 30) || cols > (1 << 30) || vocab > (1 << 30);
}

}  // namespace

const WaitControl loss_waits = {take_expired, limit_waits, wait_for_nothing};

}  // namespace ones

using namespace ones;

extern "C" {

int ones_align_rows(const void* d_src, int64_t lds, int32_t rows, int32_t cols, int32_t type, void* d_dst, int64_t ldd, void* cuda_stream) {
    if (rows < 0 || cols < 0 || (type != ONES_BF16 && type != ONES_F16) || lds < cols || ldd < cols) return ONES_ERR_BAD_PARAM;
    if (rows == 0 || cols == 0) return ONES_OK;
    if (!d_src || !d_dst) return ONES_ERR_NULL;
    if (!aligned(d_src, 2) || !aligned(d_dst, 16) || ldd % 8) return ONES_ERR_ALIGN;
    const int64_t need = ((int64_t)rows * ((cols + 7) / 8) + kAlignThreads * kAlignEach - 1) / (kAlignThreads * kAlignEach);
    k_align_rows<<<(unsigned)(need < 8 * kSms ? need : 8 * kSms), kAlignThreads, 0, reinterpret_cast<cudaStream_t>(cuda_stream)>>>(
        static_cast<const uint16_t*>(d_src), lds, rows, cols, static_cast<uint16_t*>(d_dst), ldd);
    return cudaGetLastError() == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

size_t ones_linear_ce_workspace_bytes(int32_t rows, int32_t vocab) {
    if (bad_sizes(rows, 1, vocab)) return 0;
    return forward_layout(rows, vocab).total;
}

int ones_linear_ce(const void* d_hidden, int64_t ldh, const void* d_weight, int64_t ldw, const int64_t* d_target,
                   int32_t rows, int32_t cols, int32_t vocab, int32_t type, float* d_loss, float* d_lse,
                   void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
    if (bad_sizes(rows, cols, vocab) || (type != ONES_BF16 && type != ONES_F16) || ldh < cols || ldw < cols)
        return ONES_ERR_BAD_PARAM;
    if (rows == 0) return ONES_OK;
    if (!d_hidden || !d_weight || !d_target || !d_loss || !d_lse || !d_workspace) return ONES_ERR_NULL;
    if (!aligned(d_hidden, 16) || !aligned(d_weight, 16) || ldh % 8 || ldw % 8 || !aligned(d_workspace, 256) || !aligned(d_target, 8) ||
        !aligned(d_loss, 4) || !aligned(d_lse, 4))
        return ONES_ERR_ALIGN;
    const ForwardLayout L = forward_layout(rows, vocab);
    if (workspace_bytes < L.total) return ONES_ERR_WORKSPACE;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(d_workspace);
    float2* part = reinterpret_cast<float2*>(ws + L.part);
    float* at_target = reinterpret_cast<float*>(ws + L.at_target);
    const Operand h = {d_hidden, ldh, 0, false}, w = {d_weight, ldw, 0, false};
    const EpiStats::Args ea = {d_target, part, at_target, rows, vocab};
    cudaError_t err = launch_matmul<false, false, EpiStats>(h, w, rows, vocab, cols, 1, false, type == ONES_F16, ea, stream, false,
                                                                  nullptr, nullptr, width_of(rows, vocab));
    const int r = rows > 4 * kSms ? 8 : 4;
    if (err == cudaSuccess)
        err = launch_after(r == 8 ? k_ce_join<8> : k_ce_join<4>, dim3((rows + r - 1) / r), dim3(kJoinThreads), stream, part,
                           slots_of(rows, vocab), at_target, d_target, rows, vocab, d_loss, d_lse);
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

size_t ones_linear_ce_backward_workspace_bytes(int32_t rows, int32_t cols, int32_t vocab, int32_t piece) {
    if (bad_sizes(rows, cols, vocab) || piece < 0 || piece % 256) return 0;
    return backward_layout(rows, cols, vocab, piece).total;
}

int ones_linear_ce_backward(const float* d_dloss, const void* d_hidden, int64_t ldh, const void* d_weight, int64_t ldw,
                            const int64_t* d_target, const float* d_lse, int32_t rows, int32_t cols, int32_t vocab,
                            int32_t type, int32_t wtype, int32_t piece, void* d_dhidden, int64_t lddh, void* d_dweight,
                            int64_t lddw, void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
    if (bad_sizes(rows, cols, vocab) || (type != ONES_BF16 && type != ONES_F16) || (wtype != type && wtype != ONES_F32) ||
        piece < 0 || piece % 256 || ldh < cols || ldw < cols || lddh < cols || lddw < cols)
        return ONES_ERR_BAD_PARAM;
    if (!d_dweight) return ONES_ERR_NULL;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    if (rows == 0) {  // no tokens: the weight's gradient is zero
        const size_t size = wtype == ONES_F32 ? 4 : 2;
        return cudaMemset2DAsync(d_dweight, lddw * size, 0, (size_t)cols * size, vocab, stream) == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
    }
    if (!d_dloss || !d_hidden || !d_weight || !d_target || !d_lse || !d_dhidden || !d_workspace) return ONES_ERR_NULL;
    const size_t wsize = wtype == ONES_F32 ? 4 : 2;
    if (!aligned(d_hidden, 2) || !aligned(d_weight, 16) || ldw % 8 || !aligned(d_dhidden, 2) ||
        !aligned(d_dweight, wsize) || !aligned(d_workspace, 256) || !aligned(d_target, 8) || !aligned(d_dloss, 4) || !aligned(d_lse, 4))
        return ONES_ERR_ALIGN;
    const BackwardLayout L = backward_layout(rows, cols, vocab, piece);
    if (workspace_bytes < L.total) return ONES_ERR_WORKSPACE;
    char* ws = static_cast<char*>(d_workspace);
    Header* head = reinterpret_cast<Header*>(ws + L.head);
    RowInfo* info = reinterpret_cast<RowInfo*>(ws + L.info);
    uint16_t* hidden = reinterpret_cast<uint16_t*>(ws + L.hidden);
    uint16_t* dl = reinterpret_cast<uint16_t*>(ws + L.dlogits);
    float* sum = reinterpret_cast<float*>(ws + L.sum);
    uint16_t* dh = static_cast<uint16_t*>(d_dhidden);
    const bool f16 = type == ONES_F16;
    const bool wide_h = aligned(d_dhidden, 16) && lddh % 8 == 0, wide_w = aligned(d_dweight, 16) && lddw % 8 == 0;
    const bool wide_in = aligned(d_hidden, 16) && ldh % 8 == 0;
    const int fold = L.fold, plan_nk = ((vocab < L.piece ? vocab : L.piece) + kTileK - 1) / kTileK * fold;  // of the first piece: later ones are no longer
    const unsigned row_blocks = (unsigned)((rows + 7) / 8 < 8 * kSms ? (rows + 7) / 8 : 8 * kSms);

    k_ce_scan<<<1, 1024, 0, stream>>>(d_dloss, d_target, rows, vocab, f16 ? 32768.f : 1.f, info, head);
    cudaError_t err = cudaGetLastError();
    if (err == cudaSuccess)
        err = launch_after(k_ce_gather, dim3(row_blocks), dim3(256), stream, static_cast<const uint16_t*>(d_hidden), ldh, d_target, d_dloss,
                           d_lse, rows, cols, vocab, static_cast<const Header*>(head), info, hidden, L.ld_hidden, fold, dh, lddh, wide_in, wide_h);
    for (int32_t v0 = 0; err == cudaSuccess && v0 < vocab; v0 += L.piece) {
        const int32_t n = vocab - v0 < L.piece ? vocab - v0 : L.piece;
        const bool last = v0 + n == vocab;
        const uint16_t* w0 = static_cast<const uint16_t*>(d_weight) + (int64_t)v0 * ldw;
        const EpiDlogits::Args e1 = {info, dl, (int64_t)L.piece * fold, rows, v0, n, f16, fold == 2};
        err = launch_matmul<false, false, EpiDlogits>({hidden, L.ld_hidden * fold, 0, false}, {w0, ldw, 0, false}, rows, n, cols, 1, false,
                                                      f16, e1, stream, true, &head->live);
        if (err != cudaSuccess) break;
        const EpiSum::Args e2 = {sum, L.ld_sum, dh, lddh, &head->scale, info, rows, cols, v0 == 0, last && L.cut.splits == 1, f16, wide_h};
        err = launch_matmul_cut<false, true, EpiSum>({dl, (int64_t)L.piece * fold, L.piece, false}, {w0, ldw, 0, true}, rows, cols, n, L.cut, f16,
                                                     e2, stream, true, &head->live, plan_nk, fold);
        if (err != cudaSuccess) break;
        if (L.wcut.splits > 1) {
            float* wsum = reinterpret_cast<float*>(ws + L.wsum);
            const EpiSum::Args e4 = {wsum, L.ld_sum, nullptr, 0, nullptr, nullptr, n, cols, true, false, f16, false};
            err = launch_matmul_cut<true, true, EpiSum>({dl, L.piece, 0, true}, {hidden, L.ld_hidden, 0, true}, n, cols, rows * fold, L.wcut, f16,
                                                        e4, stream, true, nullptr, 0, 1, &head->live, fold);
            if (err != cudaSuccess) break;
            const int64_t blocks = ((int64_t)n * ((cols + 127) / 128) + 7) / 8;
            err = launch_after(k_ce_weight_rows, dim3((unsigned)(blocks < 8 * kSms ? blocks : 8 * kSms)), dim3(256), stream,
                               static_cast<const float*>(wsum), L.wcut, fold, L.ld_sum, n, cols, static_cast<const Header*>(head),
                               static_cast<void*>(static_cast<char*>(d_dweight) + (int64_t)v0 * lddw * (int64_t)wsize), lddw, wtype == ONES_F32, f16, wide_w);
            continue;
        }
        const EpiGrad::Args e3 = {static_cast<char*>(d_dweight) + (int64_t)v0 * lddw * (int64_t)wsize, lddw, &head->scale, n, cols,
                                  wtype == ONES_F32, f16, wide_w};
        err = launch_matmul<true, true, EpiGrad>({dl, L.piece, 0, true}, {hidden, L.ld_hidden, 0, true}, n, cols, rows * fold, 1, false, f16,
                                                 e3, stream, true, nullptr, &head->live, 0, fold);
    }
    const int64_t join_blocks = ((int64_t)rows * ((cols + 127) / 128) + 7) / 8;
    if (err == cudaSuccess && L.cut.splits > 1)
        err = launch_after(k_ce_rows, dim3((unsigned)(join_blocks < 8 * kSms ? join_blocks : 8 * kSms)), dim3(256), stream, static_cast<const float*>(sum), L.cut, plan_nk, L.ld_sum, rows, cols,
                           static_cast<const Header*>(head), static_cast<const RowInfo*>(info), dh, lddh, f16, wide_h);
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // extern "C"
