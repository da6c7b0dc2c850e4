// The norm of all gradients together, and their clipping.
//
// Bound by bytes: the first launch reads every value once and leaves a sum for each block, the second joins the sums (each
// block for itself, in the same order: nothing has to be counted or reset between calls) and writes the scaled values. It
// goes through the blocks' work backwards, so that it finds in the L2 cache what the first launch read last. The tensors'
// addresses travel as arguments of the launch, so that a captured call needs no copy.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "ones_attention.h"
#include "ones_mma.cuh"
#include "ones_train_internal.h"

namespace ones {

namespace {

constexpr int kThreads = 512;
constexpr int kGrid = 148 * 6;     // blocks of a launch at most (2.6 GB scaled: 1443 us with 4 x 256 threads on an SM, 1289 so)
constexpr int kUnroll = 4;         // 16-byte pieces of a thread at a time
constexpr int kChunk = kThreads * kUnroll * 16;  // bytes that a block takes at a time
constexpr int kTensors = 1000;     // of one launch: as many as 32,764 bytes of arguments hold
constexpr int kFewTensors = 32;    // arguments are copied for every launch: a small table for few tensors

template <int N>
struct Table {
    const void* in[N];
    void* out[N];
    int64_t size[N];    // values
    int first[N];       // first chunk of each; chunks are counted from the 16-byte boundary at or before the tensor
    uint8_t type[N];
    int count, chunks;
};

// The 16-byte piece as values.
template <class T>
__device__ __forceinline__ void values(const uint4& raw, float (&x)[16 / sizeof(T)]) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            x[i] = __uint_as_float(w[i]);
        } else if constexpr (std::is_same<T, __half>::value) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            x[2 * i] = f.x, x[2 * i + 1] = f.y;
        } else {
            x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}
template <class T>
__device__ __forceinline__ uint4 packed(const float (&x)[16 / sizeof(T)]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            w[i] = __float_as_uint(x[i]);
        } else if constexpr (std::is_same<T, __half>::value) {
            const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A chunk of a tensor: bytes [begin, end) of it, from the 16-byte boundary at or before the tensor on, of which the first
// `head` are not the tensor's.
struct Piece {
    const uint8_t* base;
    int64_t begin, end, head;
    int tensor;
};
template <int N>
__device__ __forceinline__ Piece piece_at(const Table<N>& t, int chunk) {
    int lo = 0, hi = t.count;  // the last tensor whose first chunk is not behind this one
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.first[mid] <= chunk)
            lo = mid;
        else
            hi = mid;
    }
    Piece p;
    p.tensor = lo;
    p.head = (int64_t)(reinterpret_cast<uintptr_t>(t.in[lo]) & 15);
    p.base = static_cast<const uint8_t*>(t.in[lo]) - p.head;
    p.begin = (int64_t)(chunk - t.first[lo]) * kChunk;
    p.end = p.head + t.size[lo] * (t.type[lo] == ONES_F32 ? 4 : 2);
    return p;
}

// Bytes [at, at + 16) of the piece's tensor, zeros where they are not its own.
template <class T>
__device__ __forceinline__ uint4 fetch(const Piece& p, int64_t at) {
    if (at >= p.head && at + 16 <= p.end) return *reinterpret_cast<const uint4*>(p.base + at);
    uint4 raw = make_uint4(0, 0, 0, 0);
    T* v = reinterpret_cast<T*>(&raw);
#pragma unroll
    for (int i = 0; i < (int)(16 / sizeof(T)); ++i) {
        const int64_t b = at + i * (int64_t)sizeof(T);
        if (b >= p.head && b < p.end) v[i] = *reinterpret_cast<const T*>(p.base + b);
    }
    return raw;
}

template <class T>
__device__ __forceinline__ double squares(const Piece& p) {
    constexpr int V = 16 / sizeof(T);
    uint4 raw[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) raw[i] = fetch<T>(p, p.begin + (int64_t)(i * kThreads + threadIdx.x) * 16);
    float s = 0.f;
    bool some = false;
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        float x[V];
        values<T>(raw[i], x);
        some = some || (raw[i].x | raw[i].y | raw[i].z | raw[i].w);
#pragma unroll
        for (int j = 0; j < V; ++j) s = fmaf(x[j], x[j], s);
    }
    // 32 bits hold the squares of values from 2^-40 to 2^60 as they are; sums outside (and NaN) are taken in 64
    if ((s > 0x1p-80f && s < 0x1p120f) || !some) return s;
    double d = 0;
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        float x[V];
        values<T>(raw[i], x);
#pragma unroll
        for (int j = 0; j < V; ++j) d = fma((double)x[j], (double)x[j], d);
    }
    return d;
}

// The sum over the block, in a fixed order; every thread has it.
__device__ __forceinline__ double block_sum(double s) {
    __shared__ double sums[kThreads / 32];
    for (int m = 16; m; m >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, m);
    __syncthreads();
    if (threadIdx.x % 32 == 0) sums[threadIdx.x / 32] = s;
    __syncthreads();
    double r = 0;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) r += sums[i];
    return r;
}

template <int N>
__global__ void __launch_bounds__(kThreads) k_squares(const __grid_constant__ Table<N> t, double* part) {
    wait_for_predecessor();
    let_successor_start();
    double s = 0;
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const Piece p = piece_at(t, c);
        const int type = t.type[p.tensor];
        s += type == ONES_F32 ? squares<float>(p) : type == ONES_BF16 ? squares<__nv_bfloat16>(p) : squares<__half>(p);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__device__ __forceinline__ double norm_of(const double* part, int parts) {
    double s = 0;
    for (int i = threadIdx.x; i < parts; i += kThreads) s += part[i];
    return sqrt(block_sum(s));
}

__global__ void __launch_bounds__(kThreads) k_norm(const double* part, int parts, float* norm) {
    wait_for_predecessor();
    const double n = norm_of(part, parts);
    if (threadIdx.x == 0) *norm = (float)n;
}

template <class T>
__device__ __forceinline__ void scale(const Piece& p, void* out, float f, float before) {
    constexpr int V = 16 / sizeof(T);
    uint8_t* o = static_cast<uint8_t*>(out) - p.head;
    const bool wide = reinterpret_cast<uintptr_t>(o) % 16 == 0;
    uint4 raw[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) raw[i] = fetch<T>(p, p.begin + (int64_t)(i * kThreads + threadIdx.x) * 16);
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        const int64_t at = p.begin + (int64_t)(i * kThreads + threadIdx.x) * 16;
        float x[V];
        values<T>(raw[i], x);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = x[j] * before * f;
        const uint4 r = packed<T>(x);
        if (wide && at >= p.head && at + 16 <= p.end) {
            *reinterpret_cast<uint4*>(o + at) = r;
        } else {
            const T* v = reinterpret_cast<const T*>(&r);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int64_t b = at + j * (int64_t)sizeof(T);
                if (b >= p.head && b < p.end) *reinterpret_cast<T*>(o + b) = v[j];
            }
        }
    }
}

template <int N>
__global__ void __launch_bounds__(kThreads) k_scale(const __grid_constant__ Table<N> t, const double* part, int parts, double max_norm,
                                                    double eps, float* norm) {
    wait_for_predecessor();
    let_successor_start();
    const double n = norm_of(part, parts);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    const double f = max_norm / (n + eps);
    // a factor that 32 bits hold no more, of gradients near the end of their range: in two steps
    const float before = f < 0x1p-100 ? 0x1p-64f : 1.f, factor = f >= 1.0 || n == 0.0 ? 1.f : (float)(f < 0x1p-100 ? f * 0x1p64 : f);
    for (int c = t.chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
        const Piece p = piece_at(t, c);
        if (factor == 1.f && t.in[p.tensor] == t.out[p.tensor]) continue;
        const int type = t.type[p.tensor];
        void* out = t.out[p.tensor];
        type == ONES_F32 ? scale<float>(p, out, factor, before)
                         : type == ONES_BF16 ? scale<__nv_bfloat16>(p, out, factor, before) : scale<__half>(p, out, factor, before);
    }
}

int64_t chunks_of(const void* p, int64_t size, int type) {
    const int64_t bytes = size * (type == ONES_F32 ? 4 : 2);
    return bytes ? ((int64_t)(reinterpret_cast<uintptr_t>(p) & 15) + bytes + kChunk - 1) / kChunk : 0;
}

// A launch beside the tail of the one before it. The table goes by reference: by value it would be copied on the way.
template <int N, class... A>
cudaError_t launch(void (*kernel)(Table<N>, A...), int grid, cudaStream_t stream, Table<N>& t, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void* p[] = {&t, &args...};
    return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(kernel), p);
}

// Fills the table from tensor `from` on; the tensor behind the last one that it holds.
template <int N>
int fill(Table<N>& t, const void* const* g, void* const* out, const int64_t* size, const int32_t* type, int count, int from) {
    t.count = 0, t.chunks = 0;
    int i = from;
    for (; i < count && t.count < N; ++i) {
        const int64_t n = chunks_of(g[i], size[i], type[i]);
        if (!n) continue;
        t.in[t.count] = g[i], t.out[t.count] = out ? out[i] : nullptr, t.size[t.count] = size[i], t.type[t.count] = (uint8_t)type[i];
        t.first[t.count] = t.chunks;
        t.chunks += (int)n;
        ++t.count;
    }
    return i;
}

template <int N>
cudaError_t run(const void* const* g, void* const* out, const int64_t* size, const int32_t* type, int count, bool clip, double max_norm,
                double eps, float* norm, double* part, cudaStream_t stream) {
    static thread_local Table<N> t;
    int parts = 0;
    for (int i = 0; i < count;) {
        i = fill(t, g, out, size, type, count, i);
        if (!t.count) break;
        const int grid = std::min(t.chunks, kGrid);
        const cudaError_t err = launch(k_squares<N>, grid, stream, t, part + parts);
        if (err != cudaSuccess) return err;
        parts += grid;
    }
    if (!clip || parts == 0) return launch_after(k_norm, dim3(1), dim3(kThreads), stream, part, parts, norm);
    for (int i = 0; i < count;) {
        const bool first = i == 0;
        i = fill(t, g, out, size, type, count, i);
        if (!t.count) break;
        const cudaError_t err = launch(k_scale<N>, std::min(t.chunks, kGrid), stream, t, static_cast<const double*>(part), parts, max_norm, eps,
                                       first ? norm : nullptr);
        if (err != cudaSuccess) return err;
    }
    return cudaSuccess;
}

int gradients(const void* const* g, void* const* out, const int64_t* size, const int32_t* type, int count, bool clip, double max_norm,
              double eps, float* norm, void* workspace, size_t bytes, cudaStream_t stream) {
    if (count < 0 || count > 1 << 20 || (clip && !(max_norm >= 0 && eps >= 0 && isfinite(max_norm) && isfinite(eps)))) return ONES_ERR_BAD_PARAM;
    if (!norm || !workspace || (count && (!g || !size || !type || (clip && !out)))) return ONES_ERR_NULL;
    if (!aligned(norm, 4) || !aligned(workspace, 256)) return ONES_ERR_ALIGN;
    int some = 0;
    int64_t total = 0;
    for (int i = 0; i < count; ++i) {
        if (size[i] < 0 || type[i] < ONES_F32 || type[i] > ONES_F16 || size[i] > (int64_t)1 << 42) return ONES_ERR_BAD_PARAM;
        if (!size[i]) continue;
        ++some;
        if (!g[i] || (clip && !out[i])) return ONES_ERR_NULL;
        const int unit = type[i] == ONES_F32 ? 4 : 2;
        if (!aligned(g[i], unit) || (clip && !aligned(out[i], unit))) return ONES_ERR_ALIGN;
        total += size[i] * unit;
        if (total > (int64_t)1 << 44) return ONES_ERR_BAD_PARAM;  // chunks are counted in 32 bits
    }
    if (bytes < ones_gradient_norm_workspace_bytes(count)) return ONES_ERR_WORKSPACE;
    double* part = static_cast<double*>(workspace);
    const cudaError_t err = some <= kFewTensors ? run<kFewTensors>(g, out, size, type, count, clip, max_norm, eps, norm, part, stream)
                                                : run<kTensors>(g, out, size, type, count, clip, max_norm, eps, norm, part, stream);
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // namespace

}  // namespace ones

extern "C" {

size_t ones_gradient_norm_workspace_bytes(int32_t count) {
    if (count < 0 || count > 1 << 20) return 0;
    return ((size_t)(count / ones::kTensors + 1) * ones::kGrid * sizeof(double) + 255) / 256 * 256;
}

int ones_gradient_norm(const void* const* d_g, const int64_t* size, const int32_t* type, int32_t count, float* d_norm,
                       void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
    return ones::gradients(d_g, nullptr, size, type, count, false, 0, 0, d_norm, d_workspace, workspace_bytes,
                           reinterpret_cast<cudaStream_t>(cuda_stream));
}

int ones_clip_gradients(const void* const* d_g, void* const* d_out, const int64_t* size, const int32_t* type, int32_t count,
                        double max_norm, double eps, float* d_norm, void* d_workspace, size_t workspace_bytes,
                        void* cuda_stream) {
    return ones::gradients(d_g, d_out, size, type, count, true, max_norm, eps, d_norm, d_workspace, workspace_bytes,
                           reinterpret_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
