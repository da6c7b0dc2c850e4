// Layer norm and its gradients.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "ones_mma.cuh"
#include "ones_train.h"
#include "ones_train_internal.h"

namespace ones {

namespace {

// ---- elements ----
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <class T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

// V neighbouring elements, in one access.
template <class T, int V>
struct alignas(sizeof(T) * V) Pack {
    T v[V];
};

// weight or bias, whose type may be that of the rows or 32 bits; `none` where there is no such vector.
template <class T, int V>
__device__ __forceinline__ void load_param(const void* p, bool f32, int c, float none, float (&out)[V]) {
    if (!p) {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = none;
    } else if (f32) {
        const float* q = static_cast<const float*>(p) + c;
        if constexpr (V >= 4) {
#pragma unroll
            for (int i = 0; i < V / 4; ++i) {
                const float4 f = reinterpret_cast<const float4*>(q)[i];
                out[4 * i] = f.x, out[4 * i + 1] = f.y, out[4 * i + 2] = f.z, out[4 * i + 3] = f.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) out[i] = q[i];
        }
    } else {
        const Pack<T, V> r = *reinterpret_cast<const Pack<T, V>*>(static_cast<const T*>(p) + c);
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = to_f(r.v[i]);
    }
}

// Sum over the TPR threads of a row; `slot` alternates between calls that follow one another without another barrier.
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float* s, int group) {
#pragma unroll
    for (int o = 16; o; o /= 2) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
    }
    if constexpr (TPR > 32) {
        constexpr int kW = TPR / 32;
        const int w = (threadIdx.x / 32) % kW, lane = threadIdx.x % 32;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) s[(group * kW + w) * N + i] = v[i];
        }
        asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(TPR) : "memory");
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = lane < kW ? s[(group * kW + lane) * N + i] : 0.f;
#pragma unroll
            for (int o = kW / 2; o; o /= 2) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
            v[i] = __shfl_sync(0xFFFFFFFFu, v[i], 0);
        }
    }
}

struct NormIn {
    const void *x, *w, *b;
    int64_t ldx;
    int rows, cols;
    float eps;
    bool w32;
};

// A row is held in registers by TPR threads (NV packs of V neighbouring elements each): read once, the mean first and
// the squares of the differences from it second, so that no cancellation spoils the variance.
template <class T, int TPR, int NV, int V>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR)
    k_norm(const NormIn a, void* y_, int64_t ldy, float* mean_out, float* rstd_out) {
    constexpr int kThreads = TPR < 128 ? 128 : TPR, kRows = kThreads / TPR;
    __shared__ float s[2][kThreads / 32];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int row = blockIdx.x * kRows + group;
    if (row >= a.rows) return;  // whole groups, and groups of more than a warp are alone in their block
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    T* y = static_cast<T*>(y_) + row * ldy;
    float v[NV][V];
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * TPR) * V;
        if (c < a.cols) {
            const Pack<T, V> p = *reinterpret_cast<const Pack<T, V>*>(x + c);
#pragma unroll
            for (int j = 0; j < V; ++j) v[i][j] = to_f(p.v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) v[i][j] = 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < V; ++j) sum[0] += v[i][j];
    }
    row_sum<TPR>(sum, s[0], group);
    const float mean = sum[0] / a.cols;
    float sq[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if ((t + i * TPR) * V < a.cols) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v[i][j] -= mean;
                sq[0] = fmaf(v[i][j], v[i][j], sq[0]);
            }
        }
    }
    row_sum<TPR>(sq, s[1], group);
    const float rstd = 1.f / sqrtf(sq[0] / a.cols + a.eps);
    if (t == 0) {
        if (mean_out) mean_out[row] = mean;
        if (rstd_out) rstd_out[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * TPR) * V;
        if (c >= a.cols) break;
        float w[V], b[V];
        load_param<T, V>(a.w, a.w32, c, 1.f, w);
        load_param<T, V>(a.b, a.w32, c, 0.f, b);
        Pack<T, V> p;
#pragma unroll
        for (int j = 0; j < V; ++j) p.v[j] = from_f<T>(fmaf(v[i][j] * rstd, w[j], b[j]));
        *reinterpret_cast<Pack<T, V>*>(y + c) = p;
    }
}

// Rows longer than the registers of a block hold: three passes, the second and third from the caches.
constexpr int kLongThreads = 1024;
template <class T>
__global__ void __launch_bounds__(kLongThreads) k_norm_long(const NormIn a, void* y_, int64_t ldy, float* mean_out, float* rstd_out) {
    __shared__ float s[2][kLongThreads / 32];
    const int row = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    T* y = static_cast<T*>(y_) + row * ldy;
    float sum[1] = {0.f}, sq[1] = {0.f};
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) sum[0] += to_f(x[c]);
    row_sum<kLongThreads>(sum, s[0], 0);
    const float mean = sum[0] / a.cols;
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
        const float d = to_f(x[c]) - mean;
        sq[0] = fmaf(d, d, sq[0]);
    }
    row_sum<kLongThreads>(sq, s[1], 0);
    const float rstd = 1.f / sqrtf(sq[0] / a.cols + a.eps);
    if (threadIdx.x == 0) {
        if (mean_out) mean_out[row] = mean;
        if (rstd_out) rstd_out[row] = rstd;
    }
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
        float w[1], b[1];
        load_param<T, 1>(a.w, a.w32, c, 1.f, w);
        load_param<T, 1>(a.b, a.w32, c, 0.f, b);
        y[c] = from_f<T>(fmaf((to_f(x[c]) - mean) * rstd, w[0], b[0]));
    }
}

struct NormBack {
    const void *dy, *x, *w;
    const float *mean, *rstd;
    void* dx;
    float* part;  // [blocks][2][cols], or NULL: no gradient of weight and bias is wanted
    int64_t lddy, ldx, lddx;
    int rows, cols;
    bool w32;
};

constexpr int kBackParts = 2 * 148;  // blocks of the backward pass: two on every SM of a B200

// Each thread keeps the same columns for all rows of its block, and with them the block's share of dweight and dbias
// in registers; the next row's dy and x are on their way while a row is summed and written.
template <class T, int TPR, int NV, int V>
__global__ void __launch_bounds__(TPR < 512 ? 512 : TPR) k_norm_back(const NormBack a) {
    constexpr int kThreads = TPR < 512 ? 512 : TPR, kGroups = kThreads / TPR;
    __shared__ float s[2][2 * kThreads / 32];
    extern __shared__ float s_part[];  // [2][cols] when a block has several groups
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const float inv = 1.f / a.cols;
    float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * TPR) * V;
        if (c < a.cols) {
            load_param<T, V>(a.w, a.w32, c, 1.f, w[i]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) w[i][j] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) dw[i][j] = db[i][j] = 0.f;
    }
    Pack<T, V> nx[NV], ny[NV];
    float nmean = 0.f, nrstd = 0.f;
    auto fetch = [&](int row) {
        if (row >= a.rows) return;
        const T* x = static_cast<const T*>(a.x) + row * a.ldx;
        const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * V;
            if (c < a.cols) {
                nx[i] = *reinterpret_cast<const Pack<T, V>*>(x + c);
                ny[i] = *reinterpret_cast<const Pack<T, V>*>(dy + c);
            }
        }
        nmean = a.mean[row];
        nrstd = a.rstd[row];
    };
    int row = blockIdx.x * kGroups + group, turn = 0;
    const int step = gridDim.x * kGroups;
    fetch(row);
    for (; row < a.rows; row += step, turn ^= 1) {
        float xh[NV][V], g[NV][V];
        const float mean = nmean, rstd = nrstd;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool in = (t + i * TPR) * V < a.cols;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = in ? to_f(ny[i].v[j]) : 0.f;
                xh[i][j] = in ? (to_f(nx[i].v[j]) - mean) * rstd : 0.f;
                g[i][j] = d * w[i][j];
                db[i][j] += d;
                dw[i][j] = fmaf(d, xh[i][j], dw[i][j]);
                sum[0] += g[i][j];
                sum[1] = fmaf(g[i][j], xh[i][j], sum[1]);
            }
        }
        fetch(row + step);
        row_sum<TPR>(sum, s[turn], group);
        const float c1 = sum[0] * inv, c2 = sum[1] * inv;
        T* dx = static_cast<T*>(a.dx) + row * a.lddx;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * V;
            if (c >= a.cols) break;
            Pack<T, V> p;
#pragma unroll
            for (int j = 0; j < V; ++j) p.v[j] = from_f<T>(rstd * (g[i][j] - c1 - xh[i][j] * c2));
            *reinterpret_cast<Pack<T, V>*>(dx + c) = p;
        }
    }
    if (a.part) {
        float* out = a.part + (int64_t)blockIdx.x * 2 * a.cols;
        if constexpr (kGroups > 1) {
            for (int k = 0; k < kGroups; ++k) {
                if (group == k) {
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        const int c = (t + i * TPR) * V;
                        if (c >= a.cols) break;
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            s_part[c + j] = k ? s_part[c + j] + dw[i][j] : dw[i][j];
                            s_part[a.cols + c + j] = k ? s_part[a.cols + c + j] + db[i][j] : db[i][j];
                        }
                    }
                }
                __syncthreads();
            }
            for (int c = threadIdx.x; c < 2 * a.cols; c += kThreads) out[c] = s_part[c];
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * TPR) * V;
                if (c >= a.cols) break;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    out[c + j] = dw[i][j];
                    out[a.cols + c + j] = db[i][j];
                }
            }
        }
    }
    let_successor_start();
}

// Rows longer than the registers hold: dx from two passes over the row, the sums over rows by columns.
template <class T>
__global__ void __launch_bounds__(kLongThreads) k_norm_back_long(const NormBack a) {
    __shared__ float s[2 * kLongThreads / 32];
    const int row = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
    T* dx = static_cast<T*>(a.dx) + row * a.lddx;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float sum[2] = {0.f, 0.f};
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
        float w[1];
        load_param<T, 1>(a.w, a.w32, c, 1.f, w);
        const float g = to_f(dy[c]) * w[0];
        sum[0] += g;
        sum[1] = fmaf(g, (to_f(x[c]) - mean) * rstd, sum[1]);
    }
    row_sum<kLongThreads>(sum, s, 0);
    const float c1 = sum[0] / a.cols, c2 = sum[1] / a.cols;
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
        float w[1];
        load_param<T, 1>(a.w, a.w32, c, 1.f, w);
        const float xh = (to_f(x[c]) - mean) * rstd;
        dx[c] = from_f<T>(rstd * (to_f(dy[c]) * w[0] - c1 - xh * c2));
    }
}

template <class T>
__global__ void __launch_bounds__(256) k_norm_back_columns(const NormBack a) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < a.cols) {
        float dw = 0.f, db = 0.f;
        for (int row = blockIdx.y; row < a.rows; row += gridDim.y) {
            const float d = to_f(static_cast<const T*>(a.dy)[row * a.lddy + c]);
            const float xh = (to_f(static_cast<const T*>(a.x)[row * a.ldx + c]) - a.mean[row]) * a.rstd[row];
            db += d;
            dw = fmaf(d, xh, dw);
        }
        float* out = a.part + (int64_t)blockIdx.y * 2 * a.cols;
        out[c] = dw;
        out[a.cols + c] = db;
    }
    let_successor_start();
}

// dweight and dbias from the blocks' parts, in a fixed order: 32 columns x 16 threads a block.
constexpr int kJoinLanes = 16;
template <class W>
__global__ void __launch_bounds__(32 * kJoinLanes) k_norm_join(const float* part, int parts, int cols, W* dw, W* db) {
    wait_for_predecessor();
    __shared__ float s[kJoinLanes][32];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, l = threadIdx.x / 32;
    float sum = 0.f;
    if (c < 2 * cols) {
#pragma unroll 4
        for (int i = l; i < parts; i += kJoinLanes) sum += part[(int64_t)i * 2 * cols + c];
    }
    s[l][threadIdx.x % 32] = sum;
    __syncthreads();
    if (l == 0 && c < 2 * cols) {
        for (int i = 1; i < kJoinLanes; ++i) sum += s[i][threadIdx.x];
        if (c < cols) {
            if (dw) dw[c] = from_f<W>(sum);
        } else if (db) {
            db[c - cols] = from_f<W>(sum);
        }
    }
}

int parts_of(int32_t rows) { return rows < kBackParts ? rows : kBackParts; }

template <class T, int TPR, int NV, int V>
cudaError_t norm(const NormIn& a, void* y, int64_t ldy, float* mean, float* rstd, cudaStream_t stream) {
    constexpr int kThreads = TPR < 128 ? 128 : TPR, kRows = kThreads / TPR;
    k_norm<T, TPR, NV, V><<<(a.rows + kRows - 1) / kRows, kThreads, 0, stream>>>(a, y, ldy, mean, rstd);
    return cudaGetLastError();
}

template <class T>
cudaError_t norm_of(const NormIn& a, void* y, int64_t ldy, float* mean, float* rstd, bool wide, cudaStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    const int n = a.cols;
    if (wide) {
        if (n <= 32 * V) return norm<T, 32, 1, V>(a, y, ldy, mean, rstd, stream);
        if (n <= 32 * V * 4) return norm<T, 32, 4, V>(a, y, ldy, mean, rstd, stream);
        if (n <= 128 * V * 2) return norm<T, 128, 2, V>(a, y, ldy, mean, rstd, stream);
        if (n <= 128 * V * 4) return norm<T, 128, 4, V>(a, y, ldy, mean, rstd, stream);
        if (n <= 512 * V * 2) return norm<T, 512, 2, V>(a, y, ldy, mean, rstd, stream);
        if (n <= 512 * V * 4) return norm<T, 512, 4, V>(a, y, ldy, mean, rstd, stream);
    } else {
        if (n <= 32 * 32) return norm<T, 32, 32, 1>(a, y, ldy, mean, rstd, stream);
        if (n <= 128 * 32) return norm<T, 128, 32, 1>(a, y, ldy, mean, rstd, stream);
        if (n <= 512 * 32) return norm<T, 512, 32, 1>(a, y, ldy, mean, rstd, stream);
    }
    k_norm_long<T><<<a.rows, kLongThreads, 0, stream>>>(a, y, ldy, mean, rstd);
    return cudaGetLastError();
}

template <class T, int TPR, int NV, int V>
cudaError_t back(const NormBack& a, int* parts, cudaStream_t stream) {
    constexpr int kThreads = TPR < 512 ? 512 : TPR, kGroups = kThreads / TPR;
    const int need = (a.rows + kGroups - 1) / kGroups;
    *parts = need < kBackParts ? need : kBackParts;
    const size_t smem = kGroups > 1 && a.part ? (size_t)2 * a.cols * 4 : 0;  // at most 16 KiB: 2048 columns
    k_norm_back<T, TPR, NV, V><<<*parts, kThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

template <class T>
cudaError_t back_of(const NormBack& a, int* parts, bool wide, cudaStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    const int n = a.cols;
    if (wide) {
        if (n <= 32 * V) return back<T, 32, 1, V>(a, parts, stream);
        if (n <= 32 * V * 2) return back<T, 32, 2, V>(a, parts, stream);
        if (n <= 128 * V) return back<T, 128, 1, V>(a, parts, stream);
        if (n <= 128 * V * 2) return back<T, 128, 2, V>(a, parts, stream);
        if (n <= 512 * V) return back<T, 512, 1, V>(a, parts, stream);
        if (n <= 512 * V * 2) return back<T, 512, 2, V>(a, parts, stream);
    } else {
        if (n <= 32 * 16) return back<T, 32, 16, 1>(a, parts, stream);
        if (n <= 128 * 16) return back<T, 128, 16, 1>(a, parts, stream);
        if (n <= 512 * 16) return back<T, 512, 16, 1>(a, parts, stream);
    }
    k_norm_back_long<T><<<a.rows, kLongThreads, 0, stream>>>(a);
    cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess || !a.part) return err;
    *parts = parts_of(a.rows);
    k_norm_back_columns<T><<<dim3((n + 255) / 256, *parts), 256, 0, stream>>>(a);
    return cudaGetLastError();
}

template <class W>
cudaError_t join(const float* part, int parts, int cols, void* dw, void* db, cudaStream_t stream) {
    return launch_after(k_norm_join<W>, dim3((2 * cols + 31) / 32), dim3(32 * kJoinLanes), stream, part, parts, cols,
                        static_cast<W*>(dw), static_cast<W*>(db));
}

int size_of(int32_t type) { return type == ONES_F32 ? 4 : 2; }

bool bad_sizes(int32_t rows, int32_t cols, int32_t type, int32_t wtype) {
    return rows < 0 || cols < 1 || cols > ONES_NORM_MAX_COLS || type < ONES_F32 || type > ONES_F16 ||
           (wtype != ONES_F32 && wtype != type);
}

// Whether rows can be read and written 16 bytes at a time.
bool is_wide(const void* p, int64_t ld, int cols, int32_t type) {
    const int size = size_of(type);
    return aligned(p, 16) && ld * size % 16 == 0 && (int64_t)cols * size % 16 == 0;
}

}  // namespace

}  // namespace ones

using namespace ones;

extern "C" {

int ones_layer_norm(const void* d_x, int64_t ldx, const void* d_weight, const void* d_bias, int32_t rows, int32_t cols,
                    float eps, int32_t type, int32_t wtype, void* d_y, int64_t ldy, float* d_mean, float* d_rstd,
                    void* cuda_stream) {
    if (bad_sizes(rows, cols, type, wtype) || !(eps > 0.f) || !isfinite(eps) || ldx < cols || ldy < cols) return ONES_ERR_BAD_PARAM;
    if (rows == 0) return ONES_OK;
    if (!d_x || !d_y) return ONES_ERR_NULL;
    const int size = size_of(type);
    if (!aligned(d_x, size) || !aligned(d_y, size) || !aligned(d_weight, size_of(wtype)) || !aligned(d_bias, size_of(wtype)))
        return ONES_ERR_ALIGN;
    const NormIn a = {d_x, d_weight, d_bias, ldx, rows, cols, eps, wtype == ONES_F32};
    const bool wide = is_wide(d_x, ldx, cols, type) && is_wide(d_y, ldy, cols, type) && aligned(d_weight, 16) && aligned(d_bias, 16);
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    const cudaError_t err = type == ONES_F32 ? norm_of<float>(a, d_y, ldy, d_mean, d_rstd, wide, stream)
                            : type == ONES_BF16 ? norm_of<__nv_bfloat16>(a, d_y, ldy, d_mean, d_rstd, wide, stream)
                                                : norm_of<__half>(a, d_y, ldy, d_mean, d_rstd, wide, stream);
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

size_t ones_layer_norm_workspace_bytes(int32_t rows, int32_t cols) {
    if (bad_sizes(rows, cols, ONES_F32, ONES_F32)) return 0;
    const int n = parts_of(rows);
    return ((size_t)(n > 0 ? n : 1) * 2 * cols * 4 + 255) / 256 * 256;
}

int ones_layer_norm_backward(const void* d_dy, int64_t lddy, const void* d_x, int64_t ldx, const float* d_mean,
                             const float* d_rstd, const void* d_weight, int32_t rows, int32_t cols, int32_t type,
                             int32_t wtype, void* d_dx, int64_t lddx, void* d_dweight, void* d_dbias, void* d_workspace,
                             size_t workspace_bytes, void* cuda_stream) {
    if (bad_sizes(rows, cols, type, wtype) || lddy < cols || ldx < cols || lddx < cols) return ONES_ERR_BAD_PARAM;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    const int size = size_of(type), wsize = size_of(wtype);
    if (!aligned(d_dweight, wsize) || !aligned(d_dbias, wsize)) return ONES_ERR_ALIGN;
    if (rows == 0) {  // nothing to sum
        cudaError_t err = cudaSuccess;
        if (d_dweight) err = cudaMemsetAsync(d_dweight, 0, (size_t)cols * wsize, stream);
        if (d_dbias && err == cudaSuccess) err = cudaMemsetAsync(d_dbias, 0, (size_t)cols * wsize, stream);
        return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
    }
    const bool sums = d_dweight || d_dbias;
    if (!d_dy || !d_x || !d_mean || !d_rstd || !d_dx || (sums && !d_workspace)) return ONES_ERR_NULL;
    if (!aligned(d_dy, size) || !aligned(d_x, size) || !aligned(d_dx, size) || !aligned(d_weight, wsize) ||
        (sums && !aligned(d_workspace, 256)))
        return ONES_ERR_ALIGN;
    if (sums && workspace_bytes < ones_layer_norm_workspace_bytes(rows, cols)) return ONES_ERR_WORKSPACE;
    float* part = sums ? static_cast<float*>(d_workspace) : nullptr;
    const NormBack a = {d_dy, d_x, d_weight, d_mean, d_rstd, d_dx, part, lddy, ldx, lddx, rows, cols, wtype == ONES_F32};
    const bool wide = is_wide(d_dy, lddy, cols, type) && is_wide(d_x, ldx, cols, type) && is_wide(d_dx, lddx, cols, type) &&
                      aligned(d_weight, 16);
    int parts = 0;
    cudaError_t err = type == ONES_F32 ? back_of<float>(a, &parts, wide, stream)
                      : type == ONES_BF16 ? back_of<__nv_bfloat16>(a, &parts, wide, stream)
                                          : back_of<__half>(a, &parts, wide, stream);
    if (err == cudaSuccess && sums)
        err = wtype == ONES_F32 ? join<float>(part, parts, cols, d_dweight, d_dbias, stream)
              : wtype == ONES_BF16 ? join<__nv_bfloat16>(part, parts, cols, d_dweight, d_dbias, stream)
                                   : join<__half>(part, parts, cols, d_dweight, d_dbias, stream);
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // extern "C"
