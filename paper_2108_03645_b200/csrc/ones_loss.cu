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
__device__ __forceinline__ float regain(int k) { return 1.f + (float)k * 9.3132257e-10f; }

// Softmax statistics of a tile of logits: each thread takes the maximum m and s = sum exp(l - m) of its row's columns
// here, and the logit of the row's target if it meets it.
struct EpiStats {
    struct Args {
        const int64_t* target;
        float2* part;  // [slots][rows], one slot per half tile
        float* at_target;
        int rows, vocab;
    };
    template <int W>
    static __device__ __forceinline__ void tile(const Args& a, const MatShape& g, uint32_t acc, int row, int col,
                                                const TileAt& at, int half, const Turn&) {
        const float up = regain(g.K), to2 = kLog2e * up;
        const int64_t t64 = row < a.rows ? a.target[row] : -1;
        const int t = t64 >= 0 && t64 < a.vocab ? (int)t64 : -1;
        float m = -INFINITY, s = 0.f;
#pragma unroll 1
        for (int c = 0; c < W; c += 32) {
            float v[32];
            tmem_load(acc + c, v);
            const int left = a.vocab - (col + c);
            if (left <= 0) break;
            if (left < 32) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i >= left) v[i] = -INFINITY;
            }
            const unsigned at_i = (unsigned)(t - (col + c));
            if (at_i < 32u) {
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
            const float shift = next == -INFINITY ? 0.f : -next * to2;  // nothing but -inf so far: exp gives 0
            s *= exp2_fast(fmaf(m, to2, shift));
            float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 32; ++i) s4[i & 3] += exp2_fast(fmaf(v[i], to2, shift));
            s += (s4[0] + s4[1]) + (s4[2] + s4[3]);
            m = next;
        }
        if (row < a.rows) a.part[(int64_t)(at.n * 2 + half) * a.rows + row] = make_float2(m * up, s);
    }
};

// Gradient of a piece's logits, as 16 bits: (exp(l - lse) - [target]) * dloss * scale.
struct EpiDlogits {
    struct Args {
        const int64_t* target;
        const float *lse, *dloss, *scale;
        uint16_t* out;
        int64_t ld;
        int rows, vocab, first, cols;  // the piece: `cols` entries from `first`
        bool f16;
    };
    template <int W>
    static __device__ __forceinline__ void tile(const Args& a, const MatShape& shape, uint32_t acc, int row, int col,
                                                const TileAt&, int, const Turn& turn) {
        const float to2 = kLog2e * regain(shape.K);
        const int64_t t64 = row < a.rows ? a.target[row] : -1;
        const bool live = t64 >= 0 && t64 < a.vocab;
        const int t = live ? (int)(t64 - a.first) : -1;
        const float g = live ? a.dloss[row] * *a.scale : 0.f;
        const float shift = live ? -a.lse[row] * kLog2e : 0.f;
#pragma unroll 1
        for (int c = 0; c < W && col + c < a.cols; c += 64) {
            float v[64];
            tmem_load(acc + c, v);
#pragma unroll
            for (int i = 0; i < 64; ++i) {
                const float p = exp2_fast(fmaf(v[i], to2, shift));
                v[i] = live ? p * g : 0.f;
            }
            const unsigned at_i = (unsigned)(t - (col + c));
            if (at_i < 64u) {
#pragma unroll
                for (int i = 0; i < 64; ++i)
                    if (at_i == (unsigned)i) v[i] -= g;
            }
            turn.put16(v, a.f16);
            turn.store16(a.out, a.ld, row - turn.lane, col + c, a.rows, a.cols, true);
        }
    }
};

// Sum over the pieces: the product is added to (first piece: put into) 32-bit sums; the last piece rounds them.
struct EpiSum {
    struct Args {
        float* sum;
        int64_t ld_sum;
        uint16_t* out;
        int64_t ld_out;
        const float* scale;
        int rows, cols;
        bool first, last, f16, wide;
    };
    template <int W>
    static __device__ __forceinline__ void tile(const Args& a, const MatShape&, uint32_t acc, int row, int col,
                                                const TileAt&, int, const Turn& turn) {
        const float unscale = a.last ? 1.f / *a.scale : 1.f;  // a power of two
        const int r0 = row - turn.lane + turn.lane / 8, k = turn.lane & 7;
#pragma unroll 1
        for (int c = 0; c < W && col + c < a.cols; c += 32) {
            const int at_col = col + c + 4 * k, left = a.cols - at_col;
            float* sum = a.sum + (int64_t)r0 * a.ld_sum + at_col;  // has whole chunks of 32 columns
            float4 old[8];
            if (!a.first) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (r0 + 4 * i < a.rows) old[i] = *reinterpret_cast<const float4*>(sum + 4 * i * a.ld_sum);
            }
            float v[32];
            tmem_load(acc + c, v);
            turn.put32(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint4 q = turn.chunk(4 * i + turn.lane / 8, k);
                float4 f = make_float4(__uint_as_float(q.x), __uint_as_float(q.y), __uint_as_float(q.z), __uint_as_float(q.w));
                if (!a.first) f.x += old[i].x, f.y += old[i].y, f.z += old[i].z, f.w += old[i].w;
                if (r0 + 4 * i >= a.rows) continue;
                if (!a.last) {
                    *reinterpret_cast<float4*>(sum + 4 * i * a.ld_sum) = f;
                    continue;
                }
                uint16_t* out = a.out + (int64_t)(r0 + 4 * i) * a.ld_out + at_col;
                const uint32_t lo = Half16::pack(f.x * unscale, f.y * unscale, a.f16), hi = Half16::pack(f.z * unscale, f.w * unscale, a.f16);
                if (a.wide && left >= 4) {
                    *reinterpret_cast<uint2*>(out) = make_uint2(lo, hi);
                } else {
                    if (left > 0) out[0] = (uint16_t)lo;
                    if (left > 1) out[1] = (uint16_t)(lo >> 16);
                    if (left > 2) out[2] = (uint16_t)hi;
                    if (left > 3) out[3] = (uint16_t)(hi >> 16);
                }
            }
        }
    }
};

// A piece's rows of dweight, complete: scaled back and rounded.
struct EpiGrad {
    struct Args {
        void* out;
        int64_t ld;
        const float* scale;
        int rows, cols;
        bool f32, f16, wide;
    };
    template <int W>
    static __device__ __forceinline__ void tile(const Args& a, const MatShape&, uint32_t acc, int row, int col,
                                                const TileAt&, int, const Turn& turn) {
        const float unscale = 1.f / *a.scale;
        const int row0 = row - turn.lane;
#pragma unroll 1
        for (int c = 0; c < W && col + c < a.cols; c += 64) {
            float v[64];
            tmem_load(acc + c, v);
#pragma unroll
            for (int i = 0; i < 64; ++i) v[i] *= unscale;
            if (a.f32) {
                float u[32];
#pragma unroll
                for (int h = 0; h < 64; h += 32) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) u[i] = v[h + i];
                    turn.put32(u);
                    turn.store32(static_cast<float*>(a.out), a.ld, row0, col + c + h, a.rows, a.cols, a.wide);
                }
            } else {
                turn.put16(v, a.f16);
                turn.store16(static_cast<uint16_t*>(a.out), a.ld, row0, col + c, a.rows, a.cols, a.wide);
            }
        }
    }
};

// Joins the slots of a row. 4 rows x 128 threads a block: a warp reads whole 32-byte sectors.
constexpr int kJoinRows = 4, kJoinThreads = 512;

__device__ __forceinline__ float2 join(float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x);
    const float shift = m == -INFINITY ? 0.f : -m * kLog2e;
    return make_float2(m, a.y * exp2_fast(fmaf(a.x, kLog2e, shift)) + b.y * exp2_fast(fmaf(b.x, kLog2e, shift)));
}

__global__ void __launch_bounds__(kJoinThreads) k_ce_join(const float2* part, int slots, const float* at_target, const int64_t* target,
                                                          int rows, int vocab, float* loss, float* lse) {
    wait_for_predecessor();
    __shared__ float2 s[kJoinThreads];
    const int r = threadIdx.x % kJoinRows, row = blockIdx.x * kJoinRows + r;
    float2 v = make_float2(-INFINITY, 0.f);
    if (row < rows) {
        for (int i = threadIdx.x / kJoinRows; i < slots; i += kJoinThreads / kJoinRows) v = join(v, part[(int64_t)i * rows + row]);
    }
    s[threadIdx.x] = v;
    __syncthreads();
    for (int n = kJoinThreads / 2; n >= kJoinRows; n /= 2) {
        if ((int)threadIdx.x < n) s[threadIdx.x] = v = join(v, s[threadIdx.x + n]);
        __syncthreads();
    }
    if ((int)threadIdx.x < kJoinRows && row < rows) {
        const float l = v.x + logf(v.y);
        const int64_t t = target[row];
        lse[row] = l;
        loss[row] = t >= 0 && t < vocab ? l - at_target[row] : 0.f;
    }
}

// The power of two that brings the largest |dloss| of the rows that take part into [1, 2), so that the 16-bit gradients
// of the logits neither overflow nor lose their small values, whatever the scale of the loss.
__global__ void __launch_bounds__(1024) k_ce_scale(const float* dloss, const int64_t* target, int rows, int vocab, float* scale) {
    __shared__ float s[32];
    float top = 0.f;
    for (int i = threadIdx.x; i < rows; i += 1024) {
        const int64_t t = target[i];
        if (t >= 0 && t < vocab) top = fmaxf(top, fabsf(dloss[i]));
    }
    for (int o = 16; o; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if (threadIdx.x % 32 == 0) s[threadIdx.x / 32] = top;
    __syncthreads();
    if (threadIdx.x < 32) {
        top = s[threadIdx.x];
        for (int o = 16; o; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if (threadIdx.x == 0) {
            const int e = top > 0.f && top < INFINITY ? ilogbf(top) : 0;
            *scale = exp2f((float)(e < -100 ? 100 : e > 100 ? -100 : -e));
        }
    }
    let_successor_start();
}

inline size_t up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline int slots_of(int32_t rows, int32_t vocab) {
    const int w = use_pairs(rows, vocab, 1, false) ? 256 : 128;
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

struct BackwardLayout {
    size_t scale, dlogits, sum, total;
    int64_t ld_sum;
    int32_t piece;
};
BackwardLayout backward_layout(int32_t rows, int32_t cols, int32_t vocab, int32_t piece) {
    BackwardLayout L;
    L.piece = piece_of(rows, vocab, piece);
    L.ld_sum = (int64_t)up(cols, 32);
    L.scale = 0;
    L.dlogits = 256;
    L.sum = up(L.dlogits + (size_t)rows * L.piece * 2, 256);
    L.total = up(L.sum + (L.piece < vocab ? (size_t)rows * L.ld_sum * 4 : 0), 256);
    return L;
}

bool bad_sizes(int32_t rows, int32_t cols, int32_t vocab) {
    return rows < 0 || cols < 1 || vocab < 1 || rows > (1 << 30) || cols > (1 << 30) || vocab > (1 << 30);
}

}  // namespace

cudaError_t loss_wait_expired(unsigned* out) {
    cudaError_t err = cudaMemcpyFromSymbol(out, g_wait_expired, sizeof(*out));
    const unsigned zero = 0;
    if (err == cudaSuccess && *out) err = cudaMemcpyToSymbol(g_wait_expired, &zero, sizeof(zero));
    return err;
}

}  // namespace ones

using namespace ones;

extern "C" {

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
    if (!aligned(d_hidden, 16) || !aligned(d_weight, 16) || ldh % 8 || ldw % 8 || !aligned(d_workspace, 256))
        return ONES_ERR_ALIGN;
    const ForwardLayout L = forward_layout(rows, vocab);
    if (workspace_bytes < L.total) return ONES_ERR_WORKSPACE;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(d_workspace);
    float2* part = reinterpret_cast<float2*>(ws + L.part);
    float* at_target = reinterpret_cast<float*>(ws + L.at_target);
    const Operand h = {d_hidden, ldh, 0, false}, w = {d_weight, ldw, 0, false};
    const EpiStats::Args ea = {d_target, part, at_target, rows, vocab};
    cudaError_t err = launch_matmul<false, false, EpiStats>(h, w, rows, vocab, cols, 1, false, type == ONES_F16, ea, stream, false);
    if (err == cudaSuccess)
        err = launch_after(k_ce_join, dim3((rows + kJoinRows - 1) / kJoinRows), dim3(kJoinThreads), stream, part,
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
    if (!aligned(d_hidden, 16) || !aligned(d_weight, 16) || ldh % 8 || ldw % 8 || !aligned(d_dhidden, 2) ||
        !aligned(d_dweight, wsize) || !aligned(d_workspace, 256))
        return ONES_ERR_ALIGN;
    const BackwardLayout L = backward_layout(rows, cols, vocab, piece);
    if (workspace_bytes < L.total) return ONES_ERR_WORKSPACE;
    char* ws = static_cast<char*>(d_workspace);
    float* scale = reinterpret_cast<float*>(ws + L.scale);
    uint16_t* dl = reinterpret_cast<uint16_t*>(ws + L.dlogits);
    float* sum = reinterpret_cast<float*>(ws + L.sum);
    const bool f16 = type == ONES_F16;
    const bool wide_h = aligned(d_dhidden, 16) && lddh % 8 == 0, wide_w = aligned(d_dweight, 16) && lddw % 8 == 0;

    k_ce_scale<<<1, 1024, 0, stream>>>(d_dloss, d_target, rows, vocab, scale);
    cudaError_t err = cudaGetLastError();
    for (int32_t v0 = 0; err == cudaSuccess && v0 < vocab; v0 += L.piece) {
        const int32_t n = vocab - v0 < L.piece ? vocab - v0 : L.piece;
        const uint16_t* w0 = static_cast<const uint16_t*>(d_weight) + (int64_t)v0 * ldw;
        const EpiDlogits::Args e1 = {d_target, d_lse, d_dloss, scale, dl, L.piece, rows, vocab, v0, n, f16};
        err = launch_matmul<false, false, EpiDlogits>({d_hidden, ldh, 0, false}, {w0, ldw, 0, false}, rows, n, cols, 1, false,
                                                      f16, e1, stream, true);
        if (err != cudaSuccess) break;
        const EpiSum::Args e2 = {sum, L.ld_sum, static_cast<uint16_t*>(d_dhidden), lddh, scale, rows, cols, v0 == 0,
                                 v0 + n == vocab, f16, wide_h};
        err = launch_matmul<false, true, EpiSum>({dl, L.piece, 0, false}, {w0, ldw, 0, true}, rows, cols, n, 1, false, f16, e2,
                                                 stream, true);
        if (err != cudaSuccess) break;
        const EpiGrad::Args e3 = {static_cast<char*>(d_dweight) + (int64_t)v0 * lddw * (int64_t)wsize, lddw, scale, n, cols,
                                  wtype == ONES_F32, f16, wide_w};
        err = launch_matmul<true, true, EpiGrad>({dl, L.piece, 0, true}, {d_hidden, ldh, 0, true}, n, cols, rows, 1, false, f16,
                                                 e3, stream, true);
    }
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // extern "C"
