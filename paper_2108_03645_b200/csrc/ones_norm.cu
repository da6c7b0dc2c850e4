// Layer norm and its gradients.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <atomic>
#include <type_traits>

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

// 16 bytes of a row: 4 values of 32 bits or 8 of 16 bits, as pairs.
template <class T>
struct Chunk {
    static constexpr int kPairs = 8 / sizeof(T);
    uint4 raw;
    __device__ __forceinline__ Pair get(int i) const {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        if constexpr (sizeof(T) == 4) {
            return pair(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
        } else if constexpr (std::is_same<T, __half>::value) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            return pair(f.x, f.y);
        } else {
            return pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
        }
    }
    __device__ __forceinline__ void set(int i, Pair p) {
        const float2 f = split(p);
        uint32_t* w = reinterpret_cast<uint32_t*>(&raw);
        if constexpr (sizeof(T) == 4) {
            w[2 * i] = __float_as_uint(f.x), w[2 * i + 1] = __float_as_uint(f.y);
        } else if constexpr (std::is_same<T, __half>::value) {
            const __half2 h = __floats2half2_rn(f.x, f.y);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
};

__device__ __forceinline__ float inv_sqrt(float x) {
    const float r = rsqrtf(x);
    return r * fmaf(-0.5f * x * r, r, 1.5f);  // a Newton step: to the last place or two
}

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

// The same for the columns of one Chunk, as pairs.
template <class T>
__device__ __forceinline__ void load_param_pairs(const void* p, bool f32, int c, float none, Pair (&out)[Chunk<T>::kPairs]) {
    constexpr int V = 2 * Chunk<T>::kPairs;
    float v[V];
    load_param<T, V>(p, f32, c, none, v);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) out[i] = pair(v[2 * i], v[2 * i + 1]);
}

// Sums of N values (1, 2 or 4) over the TPR threads of a row (or of several rows that go through together), for all of
// them. Every exchange halves the values that a lane still carries, as long as there are several: 13 shuffles for four
// values of 512 threads instead of 40. `s` alternates between calls that follow one another without another barrier.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* s, int group) {
    static_assert(N == 1 || N == 2 || N == 4, "");
    const int lane = threadIdx.x % 32;
    float x;
    int o = 16;
    if constexpr (N == 4) {
        const bool hi = lane & 16;
        const float a = (hi ? v[2] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, hi ? v[0] : v[2], 16);
        const float b = (hi ? v[3] : v[1]) + __shfl_xor_sync(0xFFFFFFFFu, hi ? v[1] : v[3], 16);
        const bool hi8 = lane & 8;
        x = (hi8 ? b : a) + __shfl_xor_sync(0xFFFFFFFFu, hi8 ? a : b, 8);
        o = 4;
    } else if constexpr (N == 2) {
        const bool hi = lane & 16;
        x = (hi ? v[1] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, hi ? v[0] : v[1], 16);
        o = 8;
    } else {
        x = v[0];
    }
#pragma unroll
    for (; o; o /= 2) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    // the lanes of each 32 / N hold one of the values
    if constexpr (TPR == 32) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = N == 1 ? x : __shfl_sync(0xFFFFFFFFu, x, i * (32 / N));
    } else {
        constexpr int kW = TPR / 32;
        const int w = (threadIdx.x / 32) % kW;
        s += group * kW * N;
        if (lane % (32 / N) == 0) s[w * N + lane / (32 / N)] = x;
        asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(TPR) : "memory");
        x = s[lane % (kW * N)];
        if constexpr (kW * N == 64) x += s[lane + 32];
#pragma unroll
        for (o = (kW * N > 32 ? 32 : kW * N) / 2; o >= N; o /= 2) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = N == 1 ? x : __shfl_sync(0xFFFFFFFFu, x, i);
    }
}

constexpr int kNormSms = 148;  // the ring kernels have one block per SM of a B200
constexpr int64_t kNoMore = (int64_t)1 << 40;  // beyond all rows: after a wait that ran out nothing is sent for any more

struct NormIn {
    const void *x, *w, *b;
    int64_t ldx;
    int rows, cols;
    float eps;
    bool w32;
};

// Short rows that do not start on 16-byte boundaries: a row is held in registers by TPR threads, read once a value at a
// time, the mean first and the squares of the differences from it second, so that no cancellation spoils the variance.
// Many independent groups hide each other's latency: 512 x 777 takes 3.5 us, 23976 x 1001 of 16 bits 36 us (2.7 TB/s).
template <class T, int TPR, int N>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR)
    k_norm(const NormIn a, void* y_, int64_t ldy, float* mean_out, float* rstd_out) {
    constexpr int kThreads = TPR < 128 ? 128 : TPR, kRows = kThreads / TPR;
    __shared__ float s[2][kThreads / 32];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int row = blockIdx.x * kRows + group;
    if (row >= a.rows) return;  // whole groups, and groups of more than a warp are alone in their block
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    T* y = static_cast<T*>(y_) + row * ldy;
    float v[N];
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = t + i * TPR < a.cols ? to_f(x[t + i * TPR]) : 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) sum[0] += v[i];
    row_sums<TPR, 1>(sum, s[0], group);
    const float mean = sum[0] / a.cols;
    float sq[1] = {0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (t + i * TPR < a.cols) {
            v[i] -= mean;
            sq[0] = fmaf(v[i], v[i], sq[0]);
        }
    }
    row_sums<TPR, 1>(sq, s[1], group);
    const float rstd = inv_sqrt(sq[0] / a.cols + a.eps);
    if (t == 0) {
        if (mean_out) mean_out[row] = mean;
        if (rstd_out) rstd_out[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = t + i * TPR;
        if (c >= a.cols) break;
        float w[1], b[1];
        load_param<T, 1>(a.w, a.w32, c, 1.f, w);
        load_param<T, 1>(a.b, a.w32, c, 0.f, b);
        y[c] = from_f<T>(fmaf(v[i] * rstd, w[0], b[0]));
    }
}

// ---- rows on 16-byte boundaries ----
// One block per SM works through the rows, TPR threads on a row, each with NV chunks of 16 bytes. The rows come by bulk
// copies into a ring of `stages` per group of TPR threads that is filled ahead: the bytes on their way depend neither on
// registers nor on how many threads wait. What is left to bound the kernels is the issue of instructions, so a thread has
// many values (the shuffles and the barrier of a sum cost as much for few) and does arithmetic on pairs.
// 32768 x 4096 of bfloat16: 82 us, 6.5 TB/s of the 6.54 that a copy reaches; 131072 x 256: 33 us, 4.1 TB/s.
constexpr int kRingThreads = 512, kRingBytes = 196 * 1024, kMaxStages = 16;
// Rows that a group takes together: short ones share the latency of their sums (their values go through one butterfly).
template <int TPR, int kValues>
constexpr int kRingRows = TPR == 32 ? (kValues <= 8 ? 4 : kValues <= 16 ? 2 : 1) : 1;
template <int TPR, int kValues>
constexpr int kRingBackRows = TPR == 32 && kValues <= 8 ? 2 : 1;

template <int TPR>
__device__ __forceinline__ void group_sync(int group) {
    if constexpr (TPR == 32)
        __syncwarp();
    else
        asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(TPR) : "memory");
}

template <class T, int TPR, int NV>
__global__ void __launch_bounds__(kRingThreads, 1)
    k_norm_ring(const NormIn a, void* y_, int64_t ldy, float* mean_out, float* rstd_out, int stages) {
    constexpr int P = Chunk<T>::kPairs, kGroups = kRingThreads / TPR, R = kRingRows<TPR, 2 * P * NV>;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ __align__(8) uint64_t s_full[kGroups * kMaxStages];
    __shared__ float s[2][2][R * kRingThreads / 32];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int cols16 = a.cols / (2 * P);  // chunks of a row
    const uint32_t bytes = a.cols * sizeof(T), full = smem_u32(s_full + group * kMaxStages);
    uint8_t* mine = ring + (size_t)group * stages * R * bytes;
    const int first = (blockIdx.x * kGroups + group) * R, step = gridDim.x * kGroups * R;
    auto fetch = [&](int64_t row, int st) {
        const int n = (int)(a.rows - row < R ? a.rows - row : R);
        bar_expect(full + 8 * st, n * bytes);
        for (int r = 0; r < n; ++r)
            bulk_load(smem_u32(mine + (st * R + r) * bytes), static_cast<const T*>(a.x) + (row + r) * a.ldx, bytes, full + 8 * st);
    };
    if (t == 0) {
        for (int i = 0; i < stages; ++i) bar_init(full + 8 * i, 1);
        bar_init_done();
        for (int i = 0; i < stages && first + (int64_t)i * step < a.rows; ++i) fetch(first + (int64_t)i * step, i);
    }
    Pair w[NV][P], b[NV][P];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = t + i * TPR;
        if (c >= cols16) break;
        load_param_pairs<T>(a.w, a.w32, c * 2 * P, 1.f, w[i]);
        load_param_pairs<T>(a.b, a.w32, c * 2 * P, 0.f, b[i]);
    }
    group_sync<TPR>(group);
    const float inv = 1.f / a.cols;
    int st = 0, turn = 0;
    uint32_t ph = 0;
    Waits wait;
    int64_t ahead = (int64_t)stages * step;  // of the row whose place is free, the next one for it
    for (int64_t row = first; row < a.rows; row += step, turn ^= 1) {
        if (!wait(full + 8 * st, ph)) ahead = kNoMore;
        Pair v[R][NV][P];
        float sum[R], sq[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint4* at = reinterpret_cast<const uint4*>(mine + (st * R + r) * bytes);
            Pair acc = both(0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (t + i * TPR < cols16 && (R == 1 || row + r < a.rows)) {
                    const Chunk<T> q = {at[t + i * TPR]};
#pragma unroll
                    for (int j = 0; j < P; ++j) acc = acc + (v[r][i][j] = q.get(j));
                }
            }
            sum[r] = total(acc);
        }
        row_sums<TPR, R>(sum, s[turn][0], group);
        // everybody has read these rows: their place is free
        if (t == 0 && row + ahead < a.rows) fetch(row + ahead, st);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sum[r] *= inv;
            const Pair minus = both(-sum[r]);
            Pair acc = both(0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (t + i * TPR < cols16) {
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        v[r][i][j] = v[r][i][j] + minus;
                        acc = fma2(v[r][i][j], v[r][i][j], acc);
                    }
                }
            }
            sq[r] = total(acc);
        }
        row_sums<TPR, R>(sq, s[turn][1], group);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (R > 1 && row + r >= a.rows) break;
            const float rstd = inv_sqrt(fmaf(sq[r], inv, a.eps));
            if (t == 0) {
                if (mean_out) mean_out[row + r] = sum[r];
                if (rstd_out) rstd_out[row + r] = rstd;
            }
            uint4* y = reinterpret_cast<uint4*>(static_cast<T*>(y_) + (row + r) * ldy);
            const Pair scale = both(rstd);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = t + i * TPR;
                if (c >= cols16) break;
                Chunk<T> q;
#pragma unroll
                for (int j = 0; j < P; ++j) q.set(j, fma2(v[r][i][j] * scale, w[i][j], b[i][j]));
                y[c] = q.raw;
            }
        }
        if (++st == stages) st = 0, ph ^= 1;
    }
    if (!wait.ok) let_copies_end();
}

// ---- rows on other boundaries ----
// The same ring, filled with whole 16-byte blocks around a row: it starts up to 14 bytes into its place. From there a
// warp reads 32-bit words, one after the other over its lanes; where a 16-bit row starts on an odd half word, a pair of
// columns is shifted together out of two. The result leaves the same way: a word is put together from the pairs of two
// lanes. A warp has 64 * NU columns in a row, so that only their ends are written as halves.
// A row whose first or last block reaches over the ends of the tensor is not copied: its values are read one by one.
// 2958 x 8111 of 32 bits: 34 us, 5.7 TB/s. 16 bits take twice the instructions for a byte (23 a value), and the block's 16
// warps issue in 47 % of the slots only: at the sums' two barriers of a row, for shared memory and for the instruction before
// they wait 1.8, 1.0 and 1.8 cycles an issue. 3889 x 6171 in 42 us, 2.3 TB/s, where one value at a time takes 100.
template <class T>
struct Unit {  // two columns of a row: neighbours for 16 bits, 32 apart for 32 bits
    static constexpr bool k16 = sizeof(T) == 2;
    static constexpr int kWords = k16 ? 1 : 2, kNext = k16 ? 1 : 32;
    uint32_t raw[kWords];
    static __device__ __forceinline__ int column(int span, int u, int lane) { return span + 64 * u + (k16 ? 2 * lane : lane); }
    __device__ __forceinline__ Pair get() const {
        if constexpr (!k16) {
            return pair(__uint_as_float(raw[0]), __uint_as_float(raw[1]));
        } else if constexpr (std::is_same<T, __half>::value) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(raw));
            return pair(f.x, f.y);
        } else {
            return pair(__uint_as_float(raw[0] << 16), __uint_as_float(raw[0] & 0xFFFF0000u));
        }
    }
};

// Rows of a tensor [rows][cols], `ld` values apart, as they go through a ring.
template <class T>
struct OddRows {
    using U = Unit<T>;
    const T* p;
    int64_t ld;
    int head, tail;  // the rows from head up to tail are copied
    __device__ __forceinline__ OddRows(const void* base, int64_t ld_, int rows, int cols) : p(static_cast<const T*>(base)), ld(ld_) {
        // rows that begin in a block before `base`'s end, or end in the block in which the tensor ends
        const uintptr_t at = reinterpret_cast<uintptr_t>(p), end = reinterpret_cast<uintptr_t>(p + (rows - 1) * ld + cols);
        const int step = (int)(ld < 16 ? ld : 16) * (int)sizeof(T);
        head = ((int)(-at & 15) + step - 1) / step;
        tail = rows - ((int)(end & 15) + step - 1) / step;
    }
    __device__ __forceinline__ bool copied(int r) const { return r >= head && r < tail; }
    // where row r starts in its first block
    __device__ __forceinline__ uint32_t offset(int r) const {
        return ((uint32_t)reinterpret_cast<uintptr_t>(p) + (uint32_t)r * (uint32_t)ld * (uint32_t)sizeof(T)) & 15;
    }
    // bytes of the blocks around row r
    __device__ __forceinline__ uint32_t bytes(int r, int cols) const {
        return copied(r) ? (offset(r) + cols * (uint32_t)sizeof(T) + 15) & ~15u : 0;
    }
    __device__ __forceinline__ const void* blocks(int r) const { return reinterpret_cast<const uint8_t*>(p + r * ld) - offset(r); }

    // The calling thread's columns of row r, out of its place in the ring; zeros behind the last column.
    template <int NU>
    __device__ __forceinline__ void read(int r, const uint8_t* place, int span, int lane, int cols, U (&q)[NU]) const {
        if (!copied(r)) {
            const T* x = p + r * ld;
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const int c = U::column(span, u, lane);
                T v[2] = {from_f<T>(0.f), from_f<T>(0.f)};
                if (c < cols) v[0] = x[c];
                if (c + U::kNext < cols) v[1] = x[c + U::kNext];
                if constexpr (U::k16)
                    q[u].raw[0] = (uint32_t)*reinterpret_cast<const uint16_t*>(v) | (uint32_t)*reinterpret_cast<const uint16_t*>(v + 1) << 16;
                else
                    q[u].raw[0] = *reinterpret_cast<const uint32_t*>(v), q[u].raw[1] = *reinterpret_cast<const uint32_t*>(v + 1);
            }
            return;
        }
        const uint32_t off = offset(r);
        const uint32_t* w = reinterpret_cast<const uint32_t*>(place + (off & ~3u)) + U::column(span, 0, lane) * sizeof(T) / 4;
        if (span + 64 * NU <= cols) {
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                q[u].raw[0] = w[(U::k16 ? 32 : 64) * u];
                if constexpr (!U::k16) q[u].raw[1] = w[64 * u + 32];
            }
            if constexpr (U::k16) {
                if (off & 2) {
#pragma unroll
                    for (int u = 0; u < NU; ++u) q[u].raw[0] = __funnelshift_r(q[u].raw[0], w[32 * u + 1], 16);
                }
            }
            return;
        }
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int c = U::column(span, u, lane);
            if constexpr (U::k16) {
                uint32_t v = c < cols ? w[32 * u] : 0;
                if (off & 2) v = __funnelshift_r(v, c + 1 < cols ? w[32 * u + 1] : 0, 16);
                q[u].raw[0] = c + 1 < cols ? v : v & 0xFFFFu;
            } else {
                q[u].raw[0] = c < cols ? w[64 * u] : 0;
                q[u].raw[1] = c + 32 < cols ? w[64 * u + 32] : 0;
            }
        }
    }
};

// Writes a warp's columns of a row: f(u) is the u-th pair. Called by whole warps.
template <class T, int NU, class F>
__device__ __forceinline__ void write_units(T* y, int span, int lane, int cols, F f) {
    using U = Unit<T>;
    const bool whole = span + 64 * NU <= cols;
    y += U::column(span, 0, lane);
    cols -= U::column(span, 0, lane);
    if constexpr (!U::k16) {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const float2 v = split(f(u));
            if (whole || 64 * u < cols) y[64 * u] = v.x;
            if (whole || 64 * u + 32 < cols) y[64 * u + 32] = v.y;
        }
    } else {
        uint16_t* half = reinterpret_cast<uint16_t*>(y);
        auto packed = [&](int u) {
            const float2 v = split(f(u));
            if constexpr (std::is_same<T, __half>::value) {
                const __half2 h = __floats2half2_rn(v.x, v.y);
                return *reinterpret_cast<const uint32_t*>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
                return *reinterpret_cast<const uint32_t*>(&h);
            }
        };
        if (!(reinterpret_cast<uintptr_t>(y) & 2)) {
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const uint32_t v = packed(u);
                if (whole || 64 * u + 1 < cols)
                    *reinterpret_cast<uint32_t*>(half + 64 * u) = v;
                else if (64 * u < cols)
                    half[64 * u] = (uint16_t)v;
            }
            return;
        }
        // an odd half word: the lane's word ends with its pair's first column and begins with the second of the lane
        // before, or of lane 31 in the unit before
        uint32_t carry = 0;
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const uint32_t v = packed(u), left = __shfl_sync(0xFFFFFFFFu, v, (lane + 31) & 31), before = lane ? left : carry;
            carry = left;
            if (u == 0 && lane == 0) {
                if (0 < cols) half[0] = (uint16_t)v;
            } else if (whole || 64 * u < cols) {
                *reinterpret_cast<uint32_t*>(half + 64 * u - 1) = __funnelshift_r(before, v, 16);
            } else if (64 * u == cols) {
                half[64 * u - 1] = (uint16_t)(before >> 16);
            }
            if (u == NU - 1 && lane == 31 && 64 * u + 1 < cols) half[64 * u + 1] = (uint16_t)(v >> 16);
        }
    }
}

// weight or bias of a thread's columns
template <class T, int NU>
__device__ __forceinline__ void load_units(const void* p, bool f32, int span, int lane, int cols, float none, Pair (&out)[NU]) {
    using U = Unit<T>;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        const int c = U::column(span, u, lane);
        float v[2][1] = {{0.f}, {0.f}};
        if (c < cols) load_param<T, 1>(p, f32, c, none, v[0]);
        if (c + U::kNext < cols) load_param<T, 1>(p, f32, c + U::kNext, none, v[1]);
        out[u] = pair(v[0][0], v[1][0]);
    }
}

// Rows that a group takes together, as above: they share the latency of their sums.
template <int NU>
constexpr int kOddRows = NU <= 8 ? 2 : 1;
constexpr int kBackOddUnits = 8, kBackOddRows = 8 * kNormSms;

// Bytes of a row's place in a ring.
inline uint32_t odd_place(int cols, int size) { return (uint32_t)((cols * size + 14 + 15) / 16 * 16); }

template <class T, int TPR, int NU>
__global__ void __launch_bounds__(kRingThreads, 1)
    k_norm_odd(const NormIn a, void* y_, int64_t ldy, float* mean_out, float* rstd_out, int stages, uint32_t place) {
    constexpr int kGroups = kRingThreads / TPR, R = kOddRows<NU>;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ __align__(8) uint64_t s_full[kGroups * kMaxStages];
    __shared__ float s[2][2][R * kRingThreads / 32];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR, lane = t % 32, span = t / 32 * (64 * NU);
    const uint32_t full = smem_u32(s_full + group * kMaxStages);
    uint8_t* mine = ring + (size_t)group * stages * R * place;
    const int first = (blockIdx.x * kGroups + group) * R, step = gridDim.x * kGroups * R;
    const OddRows<T> x(a.x, a.ldx, a.rows, a.cols);
    auto fetch = [&](int64_t row, int st) {
        uint32_t bytes[R], sum = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) sum += bytes[r] = x.bytes((int)row + r, a.cols);
        bar_expect(full + 8 * st, sum);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (bytes[r]) bulk_load(smem_u32(mine + (st * R + r) * place), x.blocks((int)row + r), bytes[r], full + 8 * st);
    };
    if (t == 0) {
        for (int i = 0; i < stages; ++i) bar_init(full + 8 * i, 1);
        bar_init_done();
        for (int i = 0; i < stages && first + (int64_t)i * step < a.rows; ++i) fetch(first + (int64_t)i * step, i);
    }
    Pair w[NU], b[NU];
    load_units<T, NU>(a.w, a.w32, span, lane, a.cols, 1.f, w);
    load_units<T, NU>(a.b, a.w32, span, lane, a.cols, 0.f, b);
    const bool whole = span + 64 * NU <= a.cols;
    group_sync<TPR>(group);
    const float inv = 1.f / a.cols;
    int st = 0, turn = 0;
    uint32_t ph = 0;
    Waits wait;
    int64_t ahead = (int64_t)stages * step;  // of the row whose place is free, the next one for it
    for (int64_t row = first; row < a.rows; row += step, turn ^= 1) {
        if (!wait(full + 8 * st, ph)) ahead = kNoMore;
        Pair v[R][NU];
        float sum[R], sq[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sum[r] = 0.f;
            if (R > 1 && row + r >= a.rows) continue;
            Unit<T> q[NU];
            x.read((int)row + r, mine + (st * R + r) * place, span, lane, a.cols, q);
            Pair acc = both(0.f);
#pragma unroll
            for (int u = 0; u < NU; ++u) acc = acc + (v[r][u] = q[u].get());
            sum[r] = total(acc);
        }
        row_sums<TPR, R>(sum, s[turn][0], group);
        // everybody has read these rows: their place is free
        if (t == 0 && row + ahead < a.rows) fetch(row + ahead, st);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sum[r] *= inv;
            Pair acc = both(0.f);
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                v[r][u] = v[r][u] + both(-sum[r]);
                if (!whole) {
                    const int c = Unit<T>::column(span, u, lane);
                    const float2 f = split(v[r][u]);
                    v[r][u] = pair(c < a.cols ? f.x : 0.f, c + Unit<T>::kNext < a.cols ? f.y : 0.f);
                }
                acc = fma2(v[r][u], v[r][u], acc);
            }
            sq[r] = total(acc);
        }
        row_sums<TPR, R>(sq, s[turn][1], group);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (R > 1 && row + r >= a.rows) break;
            const float rstd = inv_sqrt(fmaf(sq[r], inv, a.eps));
            if (t == 0) {
                if (mean_out) mean_out[row + r] = sum[r];
                if (rstd_out) rstd_out[row + r] = rstd;
            }
            write_units<T, NU>(static_cast<T*>(y_) + (row + r) * ldy, span, lane, a.cols,
                               [&](int u) { return fma2(v[r][u] * both(rstd), w[u], b[u]); });
        }
        if (++st == stages) st = 0, ph ^= 1;
    }
    if (!wait.ok) let_copies_end();
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
    row_sums<kLongThreads, 1>(sum, s[0], 0);
    const float mean = sum[0] / a.cols;
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
        const float d = to_f(x[c]) - mean;
        sq[0] = fmaf(d, d, sq[0]);
    }
    row_sums<kLongThreads, 1>(sq, s[1], 0);
    const float rstd = inv_sqrt(sq[0] / a.cols + a.eps);
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

constexpr int kBackParts = 2 * 148;  // at most so many blocks, and parts of the sums over rows: two on every SM of a B200

// The block's share of dweight and dbias out of its groups', [groups][2][cols] in shared memory, in their order.
template <int kGroups>
__device__ __forceinline__ void join_groups(const float* part, int cols, float* out) {
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * cols; c += blockDim.x) {
        float v = part[c];
#pragma unroll
        for (int k = 1; k < kGroups; ++k) v += part[(int64_t)k * 2 * cols + c];
        out[c] = v;
    }
}

// Each thread keeps the same columns for all rows of its block, and with them the block's share of dweight and dbias
// in registers; the next row's dy and x are on their way while a row is summed and written. Latency bounds it as it does
// k_norm: 512 x 777 takes 3 us, 23976 x 1001 of 16 bits 53 us (2.7 TB/s).
template <class T, int TPR, int NV, int V>
__global__ void __launch_bounds__(TPR < 512 ? 512 : TPR) k_norm_back(const NormBack a) {
    constexpr int kThreads = TPR < 512 ? 512 : TPR, kGroups = kThreads / TPR;
    __shared__ float s[2][2 * kThreads / 32];
    extern __shared__ float s_part[];  // [groups][2][cols] when a block has several groups
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
        row_sums<TPR, 2>(sum, s[turn], group);
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
        float* own = kGroups > 1 ? s_part + group * 2 * a.cols : out;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * V;
            if (c >= a.cols) break;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                own[c + j] = dw[i][j];
                own[a.cols + c + j] = db[i][j];
            }
        }
        if (kGroups > 1) join_groups<kGroups>(s_part, a.cols, out);
    }
    let_successor_start();
}

// The same for rows on 16-byte boundaries, as k_norm_ring: x and dy come by bulk copies. With 32 values a thread the
// registers do not hold the weights too: they lie in shared memory before the ring then. 32768 x 4096 of bfloat16: 139 us,
// 5.8 TB/s; the sums over a row that all threads wait for are what is missing to a copy's 6.5.
template <class T, int TPR, int NV>
__global__ void __launch_bounds__(kRingThreads, 1) k_norm_back_ring(const NormBack a, int stages) {
    constexpr int P = Chunk<T>::kPairs, kGroups = kRingThreads / TPR, R = kRingBackRows<TPR, 2 * P * NV>;
    constexpr bool kShared = 2 * P * NV > 16;
    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t* ring = smem + (kShared ? a.cols * 4 : 0);
    __shared__ __align__(8) uint64_t s_full[kGroups * kMaxStages];
    __shared__ float s[2][2 * R * kRingThreads / 32];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int cols16 = a.cols / (2 * P);
    const uint32_t bytes = a.cols * sizeof(T), full = smem_u32(s_full + group * kMaxStages);
    uint8_t* mine = ring + (size_t)group * stages * R * 2 * bytes;
    const int first = (blockIdx.x * kGroups + group) * R, step = gridDim.x * kGroups * R;
    auto fetch = [&](int64_t row, int st) {
        const int n = (int)(a.rows - row < R ? a.rows - row : R);
        bar_expect(full + 8 * st, 2 * n * bytes);
        for (int r = 0; r < n; ++r) {
            const uint32_t at = smem_u32(mine + (st * R + r) * 2 * bytes);
            bulk_load(at, static_cast<const T*>(a.x) + (row + r) * a.ldx, bytes, full + 8 * st);
            bulk_load(at + bytes, static_cast<const T*>(a.dy) + (row + r) * a.lddy, bytes, full + 8 * st);
        }
    };
    if (t == 0) {
        for (int i = 0; i < stages; ++i) bar_init(full + 8 * i, 1);
        bar_init_done();
        for (int i = 0; i < stages && first + (int64_t)i * step < a.rows; ++i) fetch(first + (int64_t)i * step, i);
    }
    Pair w[kShared ? 1 : NV][P], dw[NV][P], db[NV][P];
    // the weights of chunk i: in registers, or read from shared memory each time
    auto weights = [&](int i) -> Pair(&)[P] {
        if constexpr (kShared) {
            const float4* q = reinterpret_cast<const float4*>(smem) + (t + i * TPR) * (P / 2);
#pragma unroll
            for (int j = 0; j < P / 2; ++j) {
                const float4 f = q[j];
                w[0][2 * j] = pair(f.x, f.y), w[0][2 * j + 1] = pair(f.z, f.w);
            }
            return w[0];
        } else {
            return w[i];
        }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (t + i * TPR < cols16) {
            load_param_pairs<T>(a.w, a.w32, (t + i * TPR) * 2 * P, 1.f, w[kShared ? 0 : i]);
            if constexpr (kShared) {  // every thread reads what it wrote itself
#pragma unroll
                for (int j = 0; j < P; ++j) reinterpret_cast<float2*>(smem)[(t + i * TPR) * P + j] = split(w[0][j]);
            }
        }
#pragma unroll
        for (int j = 0; j < P; ++j) dw[i][j] = db[i][j] = both(0.f);
    }
    group_sync<TPR>(group);
    const float inv = 1.f / a.cols;
    int st = 0, turn = 0;
    uint32_t ph = 0;
    Waits wait;
    int64_t ahead = (int64_t)stages * step;  // of the row whose place is free, the next one for it
    float nmean[R], nrstd[R];
    auto statistics = [&](int64_t row) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (row + r < a.rows) nmean[r] = a.mean[row + r], nrstd[r] = a.rstd[row + r];
    };
    statistics(first);
    for (int64_t row = first; row < a.rows; row += step, turn ^= 1) {
        float mean[R], rstd[R], sum[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) mean[r] = nmean[r], rstd[r] = nrstd[r];
        statistics(row + step);
        if (!wait(full + 8 * st, ph)) ahead = kNoMore;
        Chunk<T> x[R][NV], dy[R][NV];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint4* at = reinterpret_cast<const uint4*>(mine + (st * R + r) * 2 * bytes);
            const Pair scale = both(rstd[r]), minus = both(-mean[r]);
            Pair acc1 = both(0.f), acc2 = both(0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = t + i * TPR;
                if (c >= cols16 || (R > 1 && row + r >= a.rows)) break;
                x[r][i].raw = at[c];
                dy[r][i].raw = at[cols16 + c];
                Pair(&wi)[P] = weights(i);
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const Pair d = dy[r][i].get(j), e = d * ((x[r][i].get(j) + minus) * scale);  // dy * xh
                    db[i][j] = db[i][j] + d;
                    dw[i][j] = dw[i][j] + e;
                    acc1 = fma2(d, wi[j], acc1);
                    acc2 = fma2(e, wi[j], acc2);
                }
            }
            sum[2 * r] = total(acc1), sum[2 * r + 1] = total(acc2);
        }
        row_sums<TPR, 2 * R>(sum, s[turn], group);
        // everybody has read these rows: their place is free
        if (t == 0 && row + ahead < a.rows) fetch(row + ahead, st);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (R > 1 && row + r >= a.rows) break;
            // dx = rstd * (dy * w - c1 - xh * c2)
            const Pair c1 = both(-rstd[r] * sum[2 * r] * inv), c2 = both(-rstd[r] * rstd[r] * sum[2 * r + 1] * inv);
            const Pair scale = both(rstd[r]), minus = both(-mean[r]);
            uint4* dx = reinterpret_cast<uint4*>(static_cast<T*>(a.dx) + (row + r) * a.lddx);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = t + i * TPR;
                if (c >= cols16) break;
                Chunk<T> q;
                Pair(&wi)[P] = weights(i);
#pragma unroll
                for (int j = 0; j < P; ++j)
                    q.set(j, fma2(x[r][i].get(j) + minus, c2, fma2(dy[r][i].get(j) * wi[j], scale, c1)));
                dx[c] = q.raw;
            }
        }
        if (++st == stages) st = 0, ph ^= 1;
    }
    if (!wait.ok) let_copies_end();
    if (a.part) {
        float* out = a.part + (int64_t)blockIdx.x * 2 * a.cols;
        float* own = kGroups > 1 ? reinterpret_cast<float*>(ring) + group * 2 * a.cols : out;  // the ring has done its work
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (t + i * TPR >= cols16) break;
#pragma unroll
            for (int j = 0; j < P; ++j) {
                float2* p = reinterpret_cast<float2*>(own) + (t + i * TPR) * P + j;
                p[0] = split(dw[i][j]);
                p[a.cols / 2] = split(db[i][j]);
            }
        }
        if (kGroups > 1) join_groups<kGroups>(reinterpret_cast<const float*>(ring), a.cols, out);
    }
    let_successor_start();
}

// The same for many 32-bit rows on other boundaries, as k_norm_odd. 11758 x 2041: 42 us, 6.9 TB/s with part of it in L2.
template <int TPR>
__global__ void __launch_bounds__(kRingThreads, 1) k_norm_back_odd(const NormBack a, int stages, uint32_t place) {
    constexpr int kGroups = kRingThreads / TPR, NU = kBackOddUnits;
    using T = float;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ __align__(8) uint64_t s_full[kGroups * kMaxStages];
    __shared__ float s[2][2 * kRingThreads / 32];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR, lane = t % 32, span = t / 32 * (64 * NU);
    const uint32_t full = smem_u32(s_full + group * kMaxStages);
    uint8_t* mine = ring + (size_t)group * stages * 2 * place;
    const int first = blockIdx.x * kGroups + group, step = gridDim.x * kGroups;
    const OddRows<T> x(a.x, a.ldx, a.rows, a.cols), dy(a.dy, a.lddy, a.rows, a.cols);
    auto fetch = [&](int64_t row, int st) {
        const uint32_t bx = x.bytes((int)row, a.cols), bd = dy.bytes((int)row, a.cols), at = smem_u32(mine + st * 2 * place);
        bar_expect(full + 8 * st, bx + bd);
        if (bx) bulk_load(at, x.blocks((int)row), bx, full + 8 * st);
        if (bd) bulk_load(at + place, dy.blocks((int)row), bd, full + 8 * st);
    };
    if (t == 0) {
        for (int i = 0; i < stages; ++i) bar_init(full + 8 * i, 1);
        bar_init_done();
        for (int i = 0; i < stages && first + (int64_t)i * step < a.rows; ++i) fetch(first + (int64_t)i * step, i);
    }
    Pair w[NU], dw[NU], db[NU];
    load_units<T, NU>(a.w, a.w32, span, lane, a.cols, 1.f, w);
#pragma unroll
    for (int u = 0; u < NU; ++u) dw[u] = db[u] = both(0.f);
    group_sync<TPR>(group);
    const float inv = 1.f / a.cols;
    int st = 0, turn = 0;
    uint32_t ph = 0;
    Waits wait;
    int64_t ahead = (int64_t)stages * step;  // of the row whose place is free, the next one for it
    float nmean = 0.f, nrstd = 0.f;
    auto statistics = [&](int64_t row) {
        if (row < a.rows) nmean = a.mean[row], nrstd = a.rstd[row];
    };
    statistics(first);
    for (int64_t row = first; row < a.rows; row += step, turn ^= 1) {
        const float mean = nmean, rstd = nrstd;
        statistics(row + step);
        if (!wait(full + 8 * st, ph)) ahead = kNoMore;
        Unit<T> xq[NU], dq[NU];
        x.read((int)row, mine + st * 2 * place, span, lane, a.cols, xq);
        dy.read((int)row, mine + st * 2 * place + place, span, lane, a.cols, dq);
        const Pair scale = both(rstd), minus = both(-mean);
        Pair acc1 = both(0.f), acc2 = both(0.f);
#pragma unroll
        for (int u = 0; u < NU; ++u) {  // behind the last column dy and the weight are zero
            const Pair d = dq[u].get(), e = d * ((xq[u].get() + minus) * scale);  // e: dy * xh
            db[u] = db[u] + d;
            dw[u] = dw[u] + e;
            acc1 = fma2(d, w[u], acc1);
            acc2 = fma2(e, w[u], acc2);
        }
        float sum[2] = {total(acc1), total(acc2)};
        row_sums<TPR, 2>(sum, s[turn], group);
        // everybody has read this row: its place is free
        if (t == 0 && row + ahead < a.rows) fetch(row + ahead, st);
        // dx = rstd * (dy * w - c1 - xh * c2)
        const Pair c1 = both(-rstd * sum[0] * inv), c2 = both(-rstd * rstd * sum[1] * inv);
        write_units<T, NU>(static_cast<T*>(a.dx) + row * a.lddx, span, lane, a.cols,
                           [&](int u) { return fma2(xq[u].get() + minus, c2, fma2(dq[u].get() * w[u], scale, c1)); });
        if (++st == stages) st = 0, ph ^= 1;
    }
    if (!wait.ok) let_copies_end();
    if (a.part) {
        float* out = a.part + (int64_t)blockIdx.x * 2 * a.cols;
        float* own = kGroups > 1 ? reinterpret_cast<float*>(ring) + group * 2 * a.cols : out;  // the ring has done its work
        __syncthreads();
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const float2 f = split(dw[u]), g = split(db[u]);
            const int c = Unit<T>::column(span, u, lane), d = c + Unit<T>::kNext;
            if (c < a.cols) own[c] = f.x, own[a.cols + c] = g.x;
            if (d < a.cols) own[d] = f.y, own[a.cols + d] = g.y;
        }
        if (kGroups > 1) join_groups<kGroups>(reinterpret_cast<const float*>(ring), a.cols, out);
    }
    let_successor_start();
}

// Rows longer than the registers hold: dx from two passes over the row, the sums over rows by columns, so that x and dy are
// read three times (the second time from the caches). 1499 x 16001 of 32 bits: 150 us, 80 of them here and 64 in the kernel
// below, where 288 MB once take 44: a block's registers do not hold more than 8192 such columns beside their sums.
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
    row_sums<kLongThreads, 2>(sum, s, 0);
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

// dweight and dbias from the blocks' parts, in a fixed order: 32 columns x 16 threads a block. Latency: 4 to 5 us.
constexpr int kJoinLanes = 16;
template <class W>
__global__ void __launch_bounds__(32 * kJoinLanes) k_norm_join(const float* part, int parts, int cols, W* dw, W* db) {
    wait_for_predecessor();
    __shared__ float s[kJoinLanes][32];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, l = threadIdx.x / 32;
    float sum = 0.f;
    if (c < 2 * cols) {
#pragma unroll 10
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

template <class T, int TPR, int N>
cudaError_t norm(const NormIn& a, void* y, int64_t ldy, float* mean, float* rstd, cudaStream_t stream) {
    constexpr int kThreads = TPR < 128 ? 128 : TPR, kRows = kThreads / TPR;
    k_norm<T, TPR, N><<<(a.rows + kRows - 1) / kRows, kThreads, 0, stream>>>(a, y, ldy, mean, rstd);
    return cudaGetLastError();
}

// Stages of a group's ring.
inline int ring_stages(int groups, size_t stage_bytes, size_t most) {
    const size_t n = most / (groups * stage_bytes);
    return n > kMaxStages ? kMaxStages : n < 1 ? 1 : (int)n;
}

template <class T, int TPR, int NV>
cudaError_t norm_ring(const NormIn& a, void* y, int64_t ldy, float* mean, float* rstd, cudaStream_t stream) {
    constexpr int kGroups = kRingThreads / TPR, R = kRingRows<TPR, NV * 16 / (int)sizeof(T)>;
    const int need = (a.rows + kGroups * R - 1) / (kGroups * R), blocks = need < kNormSms ? need : kNormSms;
    const size_t row = (size_t)a.cols * sizeof(T) * R;
    const int stages = ring_stages(kGroups, row, kRingBytes);
    auto kernel = k_norm_ring<T, TPR, NV>;
    static std::atomic<uint64_t> ready{0};
    cudaError_t err = allow_smem(kernel, kRingBytes, ready);
    if (err != cudaSuccess) return err;
    kernel<<<blocks, kRingThreads, kGroups * stages * row, stream>>>(a, y, ldy, mean, rstd, stages);
    return cudaGetLastError();
}

template <class T, int TPR, int NU>
cudaError_t norm_odd(const NormIn& a, void* y, int64_t ldy, float* mean, float* rstd, cudaStream_t stream) {
    constexpr int kGroups = kRingThreads / TPR, R = kOddRows<NU>;
    const int need = (a.rows + kGroups * R - 1) / (kGroups * R), blocks = need < kNormSms ? need : kNormSms;
    const uint32_t place = odd_place(a.cols, sizeof(T));
    const int stages = ring_stages(kGroups, (size_t)place * R, kRingBytes);
    auto kernel = k_norm_odd<T, TPR, NU>;
    static std::atomic<uint64_t> ready{0};
    cudaError_t err = allow_smem(kernel, kRingBytes, ready);
    if (err != cudaSuccess) return err;
    kernel<<<blocks, kRingThreads, (size_t)kGroups * stages * R * place, stream>>>(a, y, ldy, mean, rstd, stages, place);
    return cudaGetLastError();
}

template <class T>
cudaError_t norm_of(const NormIn& a, void* y, int64_t ldy, float* mean, float* rstd, bool wide, cudaStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    const int n = a.cols;
    if (wide) {
        constexpr int N = 32 / V;  // chunks that hold 32 values
        if (n <= 32 * 8) return norm_ring<T, 32, N / 4>(a, y, ldy, mean, rstd, stream);
        if (n <= 32 * 16) return norm_ring<T, 32, N / 2>(a, y, ldy, mean, rstd, stream);
        if (n <= 32 * 32) return norm_ring<T, 32, N>(a, y, ldy, mean, rstd, stream);
        if (n <= 64 * 32) return norm_ring<T, 64, N>(a, y, ldy, mean, rstd, stream);
        if (n <= 128 * 32) return norm_ring<T, 128, N>(a, y, ldy, mean, rstd, stream);
        if (n <= 256 * 32) return norm_ring<T, 256, N>(a, y, ldy, mean, rstd, stream);
        if (n <= 512 * 32) return norm_ring<T, 512, N>(a, y, ldy, mean, rstd, stream);
    } else {
        // Short rows are latency: many warps that each wait for their own row do better than the ring (777 columns, 4000
        // rows of 16 bits: 7.5 us; 512 rows of 1001: 3.8 us, ring 5.3), unless many rows of half the threads' columns go
        // by (501 columns, 47904 rows: 55 us, ring 33). With few rows the same holds for longer ones (64 x 3001: 3.4 us,
        // ring 5.0; 512 x 3001: 6.3 and 5.3; 15989 x 1501: 80 and 44).
        if (n <= 32 * 8) return norm<T, 32, 8>(a, y, ldy, mean, rstd, stream);
        if (n <= 32 * 16 && a.rows >= kOddRows<8> * (kRingThreads / 32) * kNormSms) return norm_odd<T, 32, 8>(a, y, ldy, mean, rstd, stream);
        if (n <= 128 * 8) return norm<T, 128, 8>(a, y, ldy, mean, rstd, stream);
        if (n <= 512 * 8 && a.rows <= 2 * kNormSms) return norm<T, 512, 8>(a, y, ldy, mean, rstd, stream);
        if (n <= 128 * 16) return norm_odd<T, 128, 8>(a, y, ldy, mean, rstd, stream);
        if (n <= 256 * 16) return norm_odd<T, 256, 8>(a, y, ldy, mean, rstd, stream);
        if (n <= 512 * 16) return norm_odd<T, 512, 8>(a, y, ldy, mean, rstd, stream);
        if (n <= 512 * 32) return norm_odd<T, 512, 16>(a, y, ldy, mean, rstd, stream);
    }
    k_norm_long<T><<<a.rows, kLongThreads, 0, stream>>>(a, y, ldy, mean, rstd);
    return cudaGetLastError();
}

template <class T, int TPR, int N>
cudaError_t back(const NormBack& a, int* parts, cudaStream_t stream) {
    constexpr int kThreads = TPR < 512 ? 512 : TPR, kGroups = kThreads / TPR;
    const int need = (a.rows + kGroups - 1) / kGroups;
    *parts = need < kBackParts ? need : kBackParts;
    const size_t smem = kGroups > 1 && a.part ? (size_t)kGroups * 2 * a.cols * 4 : 0;  // at most 32 KiB: 8 columns a thread
    k_norm_back<T, TPR, N, 1><<<*parts, kThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

template <class T, int TPR, int NV>
cudaError_t back_ring(const NormBack& a, int* parts, cudaStream_t stream) {
    constexpr int kGroups = kRingThreads / TPR, R = kRingBackRows<TPR, NV * 16 / (int)sizeof(T)>;
    const int need = (a.rows + kGroups * R - 1) / (kGroups * R);
    *parts = need < kNormSms ? need : kNormSms;
    const size_t stage = (size_t)a.cols * sizeof(T) * 2 * R;
    const size_t weights = NV * (16 / sizeof(T)) > 16 ? (size_t)a.cols * 4 : 0;
    const int stages = ring_stages(kGroups, stage, kRingBytes - weights);
    auto kernel = k_norm_back_ring<T, TPR, NV>;
    static std::atomic<uint64_t> ready{0};
    cudaError_t err = allow_smem(kernel, kRingBytes, ready);
    if (err != cudaSuccess) return err;
    size_t smem = kGroups * stages * stage + weights;
    const size_t join = kGroups > 1 ? (size_t)kGroups * 2 * a.cols * 4 : 0;  // its place also joins the groups' sums
    if (smem < join) smem = join;
    kernel<<<*parts, kRingThreads, smem, stream>>>(a, stages);
    return cudaGetLastError();
}

template <int TPR>
cudaError_t back_odd(const NormBack& a, int* parts, cudaStream_t stream) {
    constexpr int kGroups = kRingThreads / TPR;
    const int need = (a.rows + kGroups - 1) / kGroups;
    *parts = need < kNormSms ? need : kNormSms;
    const uint32_t place = odd_place(a.cols, 4);
    const int stages = ring_stages(kGroups, 2 * (size_t)place, kRingBytes);
    auto kernel = k_norm_back_odd<TPR>;
    static std::atomic<uint64_t> ready{0};
    cudaError_t err = allow_smem(kernel, kRingBytes, ready);
    if (err != cudaSuccess) return err;
    size_t smem = (size_t)kGroups * stages * 2 * place;
    const size_t join = kGroups > 1 ? (size_t)kGroups * 2 * a.cols * 4 : 0;  // its place also joins the groups' sums
    if (smem < join) smem = join;
    kernel<<<*parts, kRingThreads, smem, stream>>>(a, stages, place);
    return cudaGetLastError();
}

template <class T>
cudaError_t back_of(const NormBack& a, int* parts, bool wide, cudaStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    const int n = a.cols;
    if (wide) {
        constexpr int N = 16 / V;  // chunks that hold 16 values
        if (n <= 32 * 8) return back_ring<T, 32, N / 2>(a, parts, stream);
        if (n <= 32 * 16) return back_ring<T, 32, N>(a, parts, stream);
        if (n <= 64 * 16) return back_ring<T, 64, N>(a, parts, stream);
        if (n <= 128 * 16) return back_ring<T, 128, N>(a, parts, stream);
        if (n <= 256 * 16) return back_ring<T, 256, N>(a, parts, stream);
        if (n <= 512 * 16) return back_ring<T, 512, N>(a, parts, stream);
        if constexpr (sizeof(T) == 2) {
            if (n <= 512 * 32) return back_ring<T, 512, 2 * N>(a, parts, stream);
        }
    } else {
        // The ring for many 32-bit rows (11758 x 2041: 42 us, 111 without; 1184 x 3001: 11.1 and 11.7; 512 x 3001: 8.5 and
        // 7.0). 16-bit rows cost as many instructions a value for half the bytes (7997 x 3001: ring 63 us, 49 without).
        if constexpr (sizeof(T) == 4) {
            if (n > 128 * 8 && a.rows >= kBackOddRows) {
                if (n <= 128 * 16) return back_odd<128>(a, parts, stream);
                if (n <= 256 * 16) return back_odd<256>(a, parts, stream);
                if (n <= 512 * 16) return back_odd<512>(a, parts, stream);
            }
        }
        // few rows: the threads of four in a block, whatever their length (512 x 251: 2.6 us; 7.7 with sixteen)
        const bool few = a.rows <= kBackParts * (512 / 128);  // one row to a group of 128 threads
        if (n <= 32 * 8 && !few) return back<T, 32, 8>(a, parts, stream);
        if (n <= 64 * 8 && !few) return back<T, 64, 8>(a, parts, stream);
        if (n <= 128 * 8) return back<T, 128, 8>(a, parts, stream);
        if (n <= 256 * 8) return back<T, 256, 8>(a, parts, stream);
        if (n <= 512 * 8) return back<T, 512, 8>(a, parts, stream);
        if (n <= 512 * 16) return back<T, 512, 16>(a, parts, stream);
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

// Kernels count rows in 32 bits and step past the last one: by less than 8192, so that what is taken does not overflow. (Row
// numbers of 64 bits or without a sign in k_norm_back: 200000 x 5 of 16 bits backward 60 -> 88 to 96 us.)
bool bad_sizes(int32_t rows, int32_t cols, int32_t type, int32_t wtype) {
    return rows < 0 || rows > ONES_NORM_MAX_ROWS || cols < 1 || cols > ONES_NORM_MAX_COLS || type < ONES_F32 || type > ONES_F16 ||
           (wtype != ONES_F32 && wtype != type);
}

// Whether rows can be read and written 16 bytes at a time.
bool is_wide(const void* p, int64_t ld, int cols, int32_t type) {
    const int size = size_of(type);
    return aligned(p, 16) && ld * size % 16 == 0 && (int64_t)cols * size % 16 == 0;
}

}  // namespace

const WaitControl norm_waits = {take_expired, limit_waits, wait_for_nothing};

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
    if (!aligned(d_x, size) || !aligned(d_y, size) || !aligned(d_weight, size_of(wtype)) || !aligned(d_bias, size_of(wtype)) ||
        !aligned(d_mean, 4) || !aligned(d_rstd, 4))
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
        !aligned(d_mean, 4) || !aligned(d_rstd, 4) || (sums && !aligned(d_workspace, 256)))
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
