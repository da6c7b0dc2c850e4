// Norms of queries and keys with the rotation of their positions, and their gradients.
//
// Bound by bytes: a vector is read once and written once (backward: x and dy read, dx written). A block takes a few tokens:
// their sines and cosines are formed once, in 64 bits up to the reduced angle, and serve all heads from shared memory; then
// groups of lanes take one vector each. A lane holds two pieces that turn into each other (value i and i + rotary / 2, or
// neighbours), so that the rotation needs no exchange between lanes, and the norm is one butterfly over the group.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "ones_attention.h"
#include "ones_mma.cuh"
#include "ones_train_internal.h"

namespace ones {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxBlocks = 148 * 4;  // partial sums of the weights' gradients: one row for each block

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

template <class T, int V>
struct alignas(sizeof(T) * V) Pack {
    T v[V];
};

struct Side {  // queries or keys
    const void *x, *dy, *weight;
    void *out, *dweight;
    int64_t x_token, x_head, dy_token, dy_head, out_token, out_head;
    int heads;
};
struct Args {
    Side side[2];
    const int64_t* positions;
    const double* frequencies;
    float* part;  // [blocks][2][dim]
    int tokens, dim, rotary, interleaved, wf32, tile;  // tile: tokens of a block at a time
    int group_log;                                     // lanes of a vector
    float eps;
};

// The two pieces of unit u: where they start, and how they turn. kind 0: not at all, 1: into each other, 2: neighbours within
// each. Either may start past the vector's end, when it is not there.
struct Unit {
    int a, b, kind, angle;  // angle: index of the first angle (kind 1), of piece a's first and, V / 2 further, of piece b's (kind 2)
};
template <int V>
__device__ __forceinline__ Unit unit_at(const Args& g, int u) {
    const int half = g.rotary / 2;
    if (V == 1 && g.interleaved) {
        const bool in = 2 * u < g.rotary;
        return {2 * u, 2 * u + 1, in ? 1 : 0, u};
    }
    if (g.interleaved) return {2 * V * u, 2 * V * u + V, 2 * V * u < g.rotary ? 2 : 0, u * V};
    if (u * V < half) return {u * V, u * V + half, 1, u * V};
    const int at = g.rotary + 2 * (u * V - half);
    return {at, at + V, 0, 0};
}

template <int V>
__device__ __forceinline__ void turn(const Unit& w, float (&x)[2 * V], const float* cs, const float* sn, float sign) {
    if (w.kind == 1) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float c = cs[w.angle + i], s = sign * sn[w.angle + i], a = x[i], b = x[V + i];
            x[i] = a * c - b * s, x[V + i] = b * c + a * s;
        }
    } else if (V > 1 && w.kind == 2) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float c = cs[w.angle + i], s = sign * sn[w.angle + i], a = x[2 * i], b = x[2 * i + 1];
            x[2 * i] = a * c - b * s, x[2 * i + 1] = b * c + a * s;
        }
    }
}

template <class T, int V>
__device__ __forceinline__ void load(const T* p, const Unit& w, int dim, float (&x)[2 * V]) {
    Pack<T, V> a = {}, b = {};
    if (w.a < dim) a = *reinterpret_cast<const Pack<T, V>*>(p + w.a);
    if (w.b < dim) b = *reinterpret_cast<const Pack<T, V>*>(p + w.b);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = w.a < dim ? to_f(a.v[i]) : 0.f, x[V + i] = w.b < dim ? to_f(b.v[i]) : 0.f;
}
template <class T, int V>
__device__ __forceinline__ void store(T* p, const Unit& w, int dim, const float (&x)[2 * V]) {
    Pack<T, V> a, b;
#pragma unroll
    for (int i = 0; i < V; ++i) a.v[i] = from_f<T>(x[i]), b.v[i] = from_f<T>(x[V + i]);
    if (w.a < dim) *reinterpret_cast<Pack<T, V>*>(p + w.a) = a;
    if (w.b < dim) *reinterpret_cast<Pack<T, V>*>(p + w.b) = b;
}
template <class T, int V>
__device__ __forceinline__ void load_weight(const void* p, bool f32, const Unit& w, int dim, float (&x)[2 * V]) {
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) {
        const int c = i < V ? w.a + i : w.b + i - V;
        x[i] = c >= dim ? 0.f : !p ? 1.f : f32 ? static_cast<const float*>(p)[c] : to_f(static_cast<const T*>(p)[c]);
    }
}

__device__ __forceinline__ float group_sum(float v, int lanes) {
    for (int m = lanes / 2; m; m >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, m);
    return v;
}

// Cosines and sines of `n` tokens from t0 on, [n][rotary / 2] each.
__device__ __forceinline__ void form_angles(const Args& g, int t0, int n, float* cs, float* sn) {
    const int half = g.rotary / 2;
    for (int i = threadIdx.x; i < n * half; i += kThreads) {
        const int t = i / half, f = i - t * half;
        double turns = (double)g.positions[t0 + t] * g.frequencies[f] * 0.15915494309189533577;  // 1 / (2 pi)
        turns -= rint(turns);
        float s, c;
        sincospif((float)(2.0 * turns), &s, &c);
        cs[i] = c, sn[i] = s;
    }
}

// U units per lane: 1 where 16-byte pieces are possible, more for single values.
template <class T, int V, int U>
__global__ void __launch_bounds__(kThreads) k_qk_norm(const __grid_constant__ Args g) {
    extern __shared__ float smem[];
    const int half = g.rotary / 2, lanes = 1 << g.group_log, groups = kThreads >> g.group_log;
    const int lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> g.group_log;
    float *cs = smem, *sn = smem + g.tile * half;
    Unit unit[U];
#pragma unroll
    for (int u = 0; u < U; ++u) unit[u] = unit_at<V>(g, lane + u * lanes);
    const int tiles = (g.tokens + g.tile - 1) / g.tile;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int t0 = tile * g.tile, n = min(g.tile, g.tokens - t0);
        __syncthreads();
        form_angles(g, t0, n, cs, sn);
        __syncthreads();
        for (int which = 0; which < 2; ++which) {
            const Side& side = g.side[which];
            if (!side.heads) continue;
            float w[U][2 * V];
#pragma unroll
            for (int u = 0; u < U; ++u) load_weight<T, V>(side.weight, g.wf32, unit[u], g.dim, w[u]);
            const int rows = n * side.heads;
            for (int first = 0; first < rows; first += groups) {
                const int row = first + group, t = min(row, rows - 1) / side.heads, h = min(row, rows - 1) - t * side.heads;
                const T* p = static_cast<const T*>(side.x) + (int64_t)(t0 + t) * side.x_token + h * side.x_head;
                float x[U][2 * V], ss = 0.f;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    load<T, V>(p, unit[u], g.dim, x[u]);
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) ss = fmaf(x[u][i], x[u][i], ss);
                }
                const float r = 1.f / sqrtf(group_sum(ss, lanes) / g.dim + g.eps);
                T* q = static_cast<T*>(side.out) + (int64_t)(t0 + t) * side.out_token + h * side.out_head;
#pragma unroll
                for (int u = 0; u < U; ++u) {
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) x[u][i] *= r * w[u][i];
                    turn<V>(unit[u], x[u], cs + t * half, sn + t * half, 1.f);
                    if (row < rows) store<T, V>(q, unit[u], g.dim, x[u]);
                }
            }
        }
    }
}

template <class T, int V, int U>
__global__ void __launch_bounds__(kThreads) k_qk_norm_back(const __grid_constant__ Args g) {
    extern __shared__ float smem[];
    const int half = g.rotary / 2, lanes = 1 << g.group_log, groups = kThreads >> g.group_log;
    const int lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> g.group_log;
    float *cs = smem, *sn = smem + g.tile * half;
    Unit unit[U];
#pragma unroll
    for (int u = 0; u < U; ++u) unit[u] = unit_at<V>(g, lane + u * lanes);
    const int tiles = (g.tokens + g.tile - 1) / g.tile;
    for (int which = 0; which < 2; ++which) {
        const Side& side = g.side[which];
        float w[U][2 * V], dw[U][2 * V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            load_weight<T, V>(side.weight, g.wf32, unit[u], g.dim, w[u]);
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) dw[u][i] = 0.f;
        }
        for (int tile = blockIdx.x; side.heads && tile < tiles; tile += gridDim.x) {
            const int t0 = tile * g.tile, n = min(g.tile, g.tokens - t0);
            __syncthreads();
            form_angles(g, t0, n, cs, sn);
            __syncthreads();
            const int rows = n * side.heads;
            for (int first = 0; first < rows; first += groups) {
                const int row = first + group, t = min(row, rows - 1) / side.heads, h = min(row, rows - 1) - t * side.heads;
                const T* p = static_cast<const T*>(side.x) + (int64_t)(t0 + t) * side.x_token + h * side.x_head;
                const T* d = static_cast<const T*>(side.dy) + (int64_t)(t0 + t) * side.dy_token + h * side.dy_head;
                float x[U][2 * V], y[U][2 * V], ss = 0.f, gx = 0.f;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    load<T, V>(p, unit[u], g.dim, x[u]);
                    load<T, V>(d, unit[u], g.dim, y[u]);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    turn<V>(unit[u], y[u], cs + t * half, sn + t * half, -1.f);
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) {
                        ss = fmaf(x[u][i], x[u][i], ss);
                        gx = fmaf(y[u][i] * w[u][i], x[u][i], gx);
                    }
                }
                const float r = 1.f / sqrtf(group_sum(ss, lanes) / g.dim + g.eps);
                const float back = r * r * (group_sum(gx, lanes) / g.dim);
                T* q = static_cast<T*>(side.out) + (int64_t)(t0 + t) * side.out_token + h * side.out_head;
#pragma unroll
                for (int u = 0; u < U; ++u) {
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) {
                        if (row < rows) dw[u][i] = fmaf(y[u][i], x[u][i] * r, dw[u][i]);
                        x[u][i] = r * (y[u][i] * w[u][i] - x[u][i] * back);
                    }
                    if (row < rows) store<T, V>(q, unit[u], g.dim, x[u]);
                }
            }
        }
        if (!g.part) continue;
        // the block's sums: group after group, in order
        __syncthreads();
        float* sums = smem;  // [groups][dim]
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) {
                const int c = i < V ? unit[u].a + i : unit[u].b + i - V;
                if (c < g.dim) sums[group * g.dim + c] = dw[u][i];
            }
        __syncthreads();
        for (int c = threadIdx.x; c < g.dim; c += kThreads) {
            float s = 0.f;
            for (int i = 0; i < groups; ++i) s += sums[i * g.dim + c];
            g.part[((int64_t)blockIdx.x * 2 + which) * g.dim + c] = s;
        }
    }
}

// Sums of the blocks' rows, in order: 32 columns a block, 8 warps with every eighth row each.
template <class W>
__global__ void __launch_bounds__(256) k_join_weights(const float* part, int blocks, int dim, W* dq, W* dk) {
    __shared__ float sums[8][32];
    wait_for_predecessor();
    const int c = blockIdx.x * 32 + threadIdx.x % 32, warp = threadIdx.x / 32;
    float s = 0.f;
    if (c < dim)
        for (int b = warp; b < blocks; b += 8) s += part[((int64_t)b * 2 + blockIdx.y) * dim + c];
    sums[warp][threadIdx.x % 32] = s;
    __syncthreads();
    W* out = blockIdx.y ? dk : dq;
    if (warp || c >= dim || !out) return;
    for (int i = 1; i < 8; ++i) s += sums[i][threadIdx.x];
    out[c] = from_f<W>(s);
}

int size_of(int type) { return type == ONES_F32 ? 4 : 2; }

bool bad_heads(const ones_heads& h, int dim, int tokens) {
    return h.heads < 0 || h.heads > ONES_MAX_HEADS || h.head < dim || (h.token < 0 && tokens > 1);
}

template <class T, int V, int U>
cudaError_t launch(Args& a, bool back, cudaStream_t stream, int* blocks) {
    const int units = V == 1 ? (a.dim + 1) / 2 : (a.dim / V + 1) / 2;
    a.group_log = 0;
    while ((1 << a.group_log) * U < units) ++a.group_log;
    const int groups = kThreads >> a.group_log, heads = max(1, a.side[0].heads + a.side[1].heads);
    // Tokens of a block: enough vectors for two turns of all groups, at most 32, and fewer where that leaves SMs idle.
    a.tile = max(1, min(32, 2 * groups / heads));
    while (a.tile > 1 && (a.tokens + a.tile - 1) / a.tile < 2 * device_sms()) a.tile = (a.tile + 1) / 2;
    const int tiles = (a.tokens + a.tile - 1) / a.tile;
    const int grid = back ? min(tiles, kMaxBlocks) : min(tiles, 148 * 8);
    const int smem = max(a.tile * a.rotary, back ? groups * a.dim : 0) * 4;
    *blocks = grid;
    auto kernel = back ? k_qk_norm_back<T, V, U> : k_qk_norm<T, V, U>;
    kernel<<<grid, kThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

template <class T>
cudaError_t launch_of(Args& a, bool back, bool wide, cudaStream_t stream, int* blocks) {
    if (wide) return launch<T, 16 / sizeof(T), 1>(a, back, stream, blocks);
    return launch<T, 1, 4>(a, back, stream, blocks);
}

int run(const ones_heads* dq, const ones_heads* dk, const ones_heads* q, const ones_heads* k, const int64_t* positions,
        const double* frequencies, const void* q_weight, const void* k_weight, int tokens, int dim, int rotary, int interleaved,
        float eps, int type, int wtype, const ones_heads* q_out, const ones_heads* k_out, void* q_dweight, void* k_dweight,
        void* workspace, size_t bytes, cudaStream_t stream, bool back) {
    if (!q || !k || !q_out || !k_out || (back && (!dq || !dk))) return ONES_ERR_NULL;
    if (tokens < 0 || dim < 1 || dim > ONES_QK_NORM_MAX_DIM || rotary < 0 || rotary > dim || rotary % 2 || !(eps >= 0.f) || !isfinite(eps) ||
        type < ONES_F32 || type > ONES_F16 || (wtype != ONES_F32 && wtype != type))
        return ONES_ERR_BAD_PARAM;
    const int size = size_of(type), wsize = size_of(wtype);
    const ones_heads* x[2] = {q, k};
    const ones_heads* y[2] = {dq, dk};
    const ones_heads* o[2] = {q_out, k_out};
    const void* w[2] = {q_weight, k_weight};
    void* dw[2] = {q_dweight, k_dweight};
    const bool sums = back && (q_dweight || k_dweight);
    Args a = {};
    const int v = 16 / size;
    // 16-byte pieces: every vector starts on such a boundary, and no piece holds both rotated values and others
    bool wide = dim % v == 0 && rotary % (2 * v) == 0;
    for (int i = 0; i < 2; ++i) {
        if (x[i]->heads != o[i]->heads || (back && x[i]->heads != y[i]->heads) || x[i]->heads < 0 || x[i]->heads > ONES_MAX_HEADS)
            return ONES_ERR_BAD_PARAM;
        for (const ones_heads* h : {x[i], o[i], back ? y[i] : x[i]}) {
            if (!h->heads) continue;
            if (bad_heads(*h, dim, tokens)) return ONES_ERR_BAD_PARAM;
            if (tokens && !h->d_data) return ONES_ERR_NULL;
            if (!aligned(h->d_data, size)) return ONES_ERR_ALIGN;
            wide = wide && aligned(h->d_data, 16) && (h->heads == 1 || h->head % v == 0) && (tokens <= 1 || h->token % v == 0);
        }
        if (!aligned(w[i], wsize) || !aligned(dw[i], wsize)) return ONES_ERR_ALIGN;
        a.side[i] = {x[i]->d_data, back ? y[i]->d_data : nullptr, w[i], o[i]->d_data, dw[i], x[i]->token, x[i]->head,
                     back ? y[i]->token : 0, back ? y[i]->head : 0, o[i]->token, o[i]->head, x[i]->heads};
    }
    if (!aligned(positions, 8) || !aligned(frequencies, 8)) return ONES_ERR_ALIGN;
    const bool none = tokens == 0 || (q->heads == 0 && k->heads == 0);
    if (!none && rotary && (!positions || !frequencies)) return ONES_ERR_NULL;
    if (sums && !none) {
        if (!workspace) return ONES_ERR_NULL;
        if (!aligned(workspace, 256)) return ONES_ERR_ALIGN;
        if (bytes < ones_qk_norm_workspace_bytes(dim)) return ONES_ERR_WORKSPACE;
    }
    cudaError_t err = cudaSuccess;
    if (none) {
        for (int i = 0; i < 2; ++i)
            if (back && dw[i] && err == cudaSuccess) err = cudaMemsetAsync(dw[i], 0, (size_t)dim * wsize, stream);
        return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
    }
    a.positions = positions, a.frequencies = frequencies, a.part = sums ? static_cast<float*>(workspace) : nullptr;
    a.tokens = tokens, a.dim = dim, a.rotary = rotary, a.interleaved = interleaved != 0, a.wf32 = wtype == ONES_F32, a.eps = eps;
    int blocks = 0;
    err = type == ONES_F32 ? launch_of<float>(a, back, wide, stream, &blocks)
          : type == ONES_BF16 ? launch_of<__nv_bfloat16>(a, back, wide, stream, &blocks)
                              : launch_of<__half>(a, back, wide, stream, &blocks);
    if (err == cudaSuccess && sums) {
        const dim3 grid((dim + 31) / 32, 2);
        err = wtype == ONES_F32 ? launch_after(k_join_weights<float>, grid, dim3(256), stream, a.part, blocks, dim, (float*)q_dweight, (float*)k_dweight)
              : wtype == ONES_BF16 ? launch_after(k_join_weights<__nv_bfloat16>, grid, dim3(256), stream, a.part, blocks, dim,
                                                  (__nv_bfloat16*)q_dweight, (__nv_bfloat16*)k_dweight)
                                   : launch_after(k_join_weights<__half>, grid, dim3(256), stream, a.part, blocks, dim, (__half*)q_dweight,
                                                  (__half*)k_dweight);
    }
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // namespace

}  // namespace ones

extern "C" {

int ones_qk_norm(const ones_heads* q, const ones_heads* k, const int64_t* d_positions, const double* d_frequencies,
                 const void* d_q_weight, const void* d_k_weight, int32_t tokens, int32_t dim, int32_t rotary,
                 int32_t interleaved, float eps, int32_t type, int32_t wtype, const ones_heads* q_out,
                 const ones_heads* k_out, void* cuda_stream) {
    return ones::run(nullptr, nullptr, q, k, d_positions, d_frequencies, d_q_weight, d_k_weight, tokens, dim, rotary, interleaved, eps, type,
                     wtype, q_out, k_out, nullptr, nullptr, nullptr, 0, reinterpret_cast<cudaStream_t>(cuda_stream), false);
}

size_t ones_qk_norm_workspace_bytes(int32_t dim) {
    if (dim < 1 || dim > ONES_QK_NORM_MAX_DIM) return 0;
    return ((size_t)ones::kMaxBlocks * 2 * dim * 4 + 255) / 256 * 256;
}

int ones_qk_norm_backward(const ones_heads* dq, const ones_heads* dk, const ones_heads* q, const ones_heads* k,
                          const int64_t* d_positions, const double* d_frequencies, const void* d_q_weight,
                          const void* d_k_weight, int32_t tokens, int32_t dim, int32_t rotary, int32_t interleaved,
                          float eps, int32_t type, int32_t wtype, const ones_heads* dq_out, const ones_heads* dk_out,
                          void* d_dq_weight, void* d_dk_weight, void* d_workspace, size_t workspace_bytes,
                          void* cuda_stream) {
    return ones::run(dq, dk, q, k, d_positions, d_frequencies, d_q_weight, d_k_weight, tokens, dim, rotary, interleaved, eps, type, wtype,
                     dq_out, dk_out, d_dq_weight, d_dk_weight, d_workspace, workspace_bytes, reinterpret_cast<cudaStream_t>(cuda_stream), true);
}

}  // extern "C"
