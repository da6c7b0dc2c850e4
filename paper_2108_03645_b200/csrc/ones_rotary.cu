// Norms of queries and keys with the rotation of their positions, and their gradients.
//
// Bound by bytes: a vector is read once and written once (backward: x and dy read, dx written). A block takes a few tokens at a
// time. Their sines and cosines are formed once, in 64 bits up to the reduced angle, and serve all heads from shared memory.
// Groups of lanes take one vector each, neighbours neighbouring ones: where each group kept to a token of its own, the memory was
// read in pieces of 256 bytes from ten thousand places at once (65536 x 40 x 128: 380 us for the forward pass). A lane holds two
// pieces that turn into each other (value i and i + rotary / 2, or neighbours), so that the rotation needs no exchange between
// lanes, and the norm is one butterfly over the group. Arithmetic is on pairs.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <atomic>
#include <type_traits>

#include "ones_attention.h"
#include "ones_mma.cuh"
#include "ones_train_internal.h"

namespace ones {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxBlocks = 148 * 2;  // partial sums of the weights' gradients: one row for each block

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

struct Side {  // queries or keys
    const void *x, *dy, *weight;
    void *out, *dweight;
    int64_t x_token, x_head, dy_token, dy_head, out_token, out_head;
    int heads;
    int step_t, step_h;  // from a group's vector to its next one, which lies as many vectors on as there are groups
};
struct Args {
    Side side[2];
    const int64_t* positions;
    const double* frequencies;
    float* part;  // [blocks][2][dim]
    int tokens, dim, rotary, interleaved, wf32;
    int group_log;     // lanes of a vector
    int tile, angles;  // tokens of a block at a time; room for a token's angles
    float eps, per_dim;
};

// The two pieces of unit u: where they start, and whether they turn (into each other, or with INTER and several values, as
// neighbours within each). Either may start past the vector's end, when it is not there.
struct Unit {
    int a, b, turns, angle;  // angle: the first of the V angles that turn the pieces
};
template <int V, bool INTER>
__device__ __forceinline__ Unit unit_at(const Args& g, int u) {
    const int half = g.rotary / 2;
    if (INTER) return {2 * V * u, 2 * V * u + V, 2 * V * u < g.rotary, u * V};
    if (u * V < half) return {u * V, u * V + half, 1, u * V};
    const int at = g.rotary + 2 * (u * V - half);
    return {at, at + V, 0, 0};
}

// 2 V values of a lane as V pairs: of its first piece, then of its second one (V = 1: both in one pair).
template <class T, int V>
struct Row {
    static constexpr int kWords = V * sizeof(T) / 4 > 0 ? V * sizeof(T) / 4 : 1;
    uint32_t a[kWords] = {}, b[kWords] = {};  // as they lie in memory; zeros where the vector has none
    __device__ __forceinline__ void load(const T* p, const Unit& w, int dim) {
        if constexpr (V == 1) {
            if (w.a < dim) a[0] = word(p[w.a]);
            if (w.b < dim) b[0] = word(p[w.b]);
        } else {
            if (w.a < dim) {
                const uint4 q = *reinterpret_cast<const uint4*>(p + w.a);
                a[0] = q.x, a[1] = q.y, a[2] = q.z, a[3] = q.w;
            }
            if (w.b < dim) {
                const uint4 q = *reinterpret_cast<const uint4*>(p + w.b);
                b[0] = q.x, b[1] = q.y, b[2] = q.z, b[3] = q.w;
            }
        }
    }
    __device__ __forceinline__ void take(const uint4& p, const uint4& q) {
        a[0] = p.x, a[1] = p.y, a[2] = p.z, a[3] = p.w;
        b[0] = q.x, b[1] = q.y, b[2] = q.z, b[3] = q.w;
    }
    static __device__ __forceinline__ uint32_t word(float v) { return __float_as_uint(v); }
    static __device__ __forceinline__ uint32_t word(__nv_bfloat16 v) { return __bfloat16_as_ushort(v); }
    static __device__ __forceinline__ uint32_t word(__half v) { return __half_as_ushort(v); }
    static __device__ __forceinline__ Pair pair_of(uint32_t w) {
        if constexpr (sizeof(T) == 4) return pair(0.f, 0.f);
        if constexpr (std::is_same<T, __half>::value) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
            return pair(f.x, f.y);
        }
        return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
    __device__ __forceinline__ void get(Pair (&x)[V]) const {
        if constexpr (V == 1) {
            if constexpr (sizeof(T) == 4)
                x[0] = pair(__uint_as_float(a[0]), __uint_as_float(b[0]));
            else
                x[0] = pair_of(a[0] | b[0] << 16);
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                x[i] = pair(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1])), x[2 + i] = pair(__uint_as_float(b[2 * i]), __uint_as_float(b[2 * i + 1]));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = pair_of(a[i]), x[4 + i] = pair_of(b[i]);
        }
    }
    static __device__ __forceinline__ uint32_t packed(Pair p) {
        const float2 f = split(p);
        if constexpr (std::is_same<T, __half>::value) {
            const __half2 h = __floats2half2_rn(f.x, f.y);
            return *reinterpret_cast<const uint32_t*>(&h);
        }
        const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ void store(T* p, const Unit& w, int dim, const Pair (&x)[V]) {
        if constexpr (V == 1) {
            const float2 f = split(x[0]);
            if (w.a < dim) p[w.a] = from_f<T>(f.x);
            if (w.b < dim) p[w.b] = from_f<T>(f.y);
        } else if constexpr (sizeof(T) == 4) {
            const float2 f[4] = {split(x[0]), split(x[1]), split(x[2]), split(x[3])};
            if (w.a < dim) *reinterpret_cast<float4*>(p + w.a) = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
            if (w.b < dim) *reinterpret_cast<float4*>(p + w.b) = make_float4(f[2].x, f[2].y, f[3].x, f[3].y);
        } else {
            if (w.a < dim) *reinterpret_cast<uint4*>(p + w.a) = make_uint4(packed(x[0]), packed(x[1]), packed(x[2]), packed(x[3]));
            if (w.b < dim) *reinterpret_cast<uint4*>(p + w.b) = make_uint4(packed(x[4]), packed(x[5]), packed(x[6]), packed(x[7]));
        }
    }
};

__device__ __forceinline__ Pair operator-(Pair a, Pair b) {
    Pair r;
    asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
// V / 2 pairs from shared memory
template <int V>
__device__ __forceinline__ void fetch_pairs(const float* p, Pair (&x)[V / 2]) {
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        const float4 f = reinterpret_cast<const float4*>(p)[i];
        x[2 * i] = pair(f.x, f.y), x[2 * i + 1] = pair(f.z, f.w);
    }
}
// The lane's values turned by the angles whose cosines and sines start at cs, sn (BACK: by their negatives).
template <int V, bool INTER, bool BACK>
__device__ __forceinline__ void turn(Pair (&x)[V], const float* cs, const float* sn) {
    if constexpr (V == 1) {
        const float2 f = split(x[0]);
        const float c = cs[0], s = BACK ? -sn[0] : sn[0];
        x[0] = pair(f.x * c - f.y * s, f.y * c + f.x * s);
    } else {
        Pair c[V / 2], s[V / 2];
        fetch_pairs<V>(cs, c), fetch_pairs<V>(sn, s);
        if constexpr (INTER) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float2 f = split(x[i]), cc = split(c[i / 2]), ss = split(s[i / 2]);
                const float u = i & 1 ? cc.y : cc.x, t = i & 1 ? (BACK ? -ss.y : ss.y) : (BACK ? -ss.x : ss.x);
                x[i] = pair(f.x * u - f.y * t, f.y * u + f.x * t);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const Pair a = x[i], b = x[V / 2 + i];
                x[i] = BACK ? fma2(b, s[i], a * c[i]) : a * c[i] - b * s[i];
                x[V / 2 + i] = BACK ? b * c[i] - a * s[i] : fma2(a, s[i], b * c[i]);
            }
        }
    }
}
// The weights of the lane's values, from a vector in shared memory that goes on with zeros behind dim.
template <int V>
__device__ __forceinline__ void weights(const float* w, const Unit& u, Pair (&x)[V]) {
    if constexpr (V == 1) {
        x[0] = pair(w[u.a], w[u.b]);
    } else {
        Pair a[V / 2], b[V / 2];
        fetch_pairs<V>(w + u.a, a), fetch_pairs<V>(w + u.b, b);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) x[i] = a[i], x[V / 2 + i] = b[i];
    }
}

__device__ __forceinline__ float group_sum(float v, int lanes) {
#pragma unroll
    for (int m = 16; m; m >>= 1)
        if (m < lanes) v += __shfl_xor_sync(0xFFFFFFFFu, v, m);
    return v;
}
__device__ __forceinline__ float inverse_root(float v) {
    const float r = rsqrtf(v);
    return r * fmaf(-0.5f * v * r, r, 1.5f);  // a Newton step: to the last place or two
}
constexpr int kWeightRow = ONES_QK_NORM_MAX_DIM + 16;

// Pieces of vectors on their way into shared memory. Each thread has slots of its own, so that nothing but its own copies is
// waited for.
constexpr int kStages = 4;
constexpr int kRingBytes = kStages * 4 * kThreads * 16;
__device__ __forceinline__ void copy_async(const uint4* to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}

// U units per lane: 1 where pieces of 16 bytes are possible, more for single values. Forward, the next vector of a group is on its
// way while the present one is worked on, and five blocks on an SM hide the rest (through shared memory, whose reads it is bound
// by, 240 -> 269 us for 65536 x 40 x 128). Backward, the sums for the weights leave room for two blocks, and three vectors of each
// group are on their way, through shared memory (one, in registers: 517 us, so 387 to 420).
template <class T, int V, int U, bool INTER, bool BACK>
__global__ void __launch_bounds__(kThreads, BACK ? 2 : 5) k_qk_norm(const __grid_constant__ Args g) {
    constexpr bool kRing = BACK && V > 1;
    constexpr int kPieces = 4;  // of a vector and a lane: two of x, two of dy
    extern __shared__ __align__(16) float smem[];
    __shared__ __align__(16) float s_weight[2][kWeightRow];
    const int lanes = 1 << g.group_log, groups = kThreads >> g.group_log;
    const int lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> g.group_log;
    float *cs = smem, *sn = smem + g.tile * g.angles;
    uint4* const ring = reinterpret_cast<uint4*>(sn + g.tile * g.angles) + threadIdx.x;
    Unit unit[U];
#pragma unroll
    for (int u = 0; u < U; ++u) unit[u] = unit_at<V, INTER>(g, lane + u * lanes);
    const int tiles = (g.tokens - 1) / g.tile + 1;
    for (int i = threadIdx.x; i < 2 * kWeightRow; i += kThreads) {
        const int which = i >= kWeightRow, c = i - which * kWeightRow;
        const void* p = g.side[which].weight;
        s_weight[which][c] = c >= g.dim ? 0.f : !p ? 1.f : g.wf32 ? static_cast<const float*>(p)[c] : to_f(static_cast<const T*>(p)[c]);
    }
    Pair dw[BACK ? 2 : 1][U][V];
    if (BACK) {
#pragma unroll
        for (int which = 0; which < (BACK ? 2 : 1); ++which)
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < V; ++i) dw[which][u][i] = both(0.f);
    }
    // What is copied next, three vectors ahead: through both sides of all tiles. left: rounds of this side of this tile; t, h: the
    // token in the tile and the head; slot: where to.
    struct {
        int tile, which, left, t, h, slot;
    } ahead = {(int)blockIdx.x - (int)gridDim.x, 1, 0, 0, 0, 0};
    auto copy_next = [&]() {
        while (ahead.left == 0 && ahead.tile < tiles) {
            if (ahead.which) ahead.tile += gridDim.x;
            ahead.which ^= 1;
            if (ahead.tile >= tiles) break;
            const int heads = g.side[ahead.which].heads;
            ahead.left = (min(g.tile, g.tokens - ahead.tile * g.tile) * heads + groups - 1) / groups;
            if (heads) ahead.t = group / heads, ahead.h = group - ahead.t * heads;
        }
        if (ahead.left) {
            const Side& side = g.side[ahead.which];
            const int64_t t = (int64_t)ahead.tile * g.tile + ahead.t;
            if (ahead.t < g.tile && t < g.tokens) {
                const T* const x = static_cast<const T*>(side.x) + t * side.x_token + ahead.h * side.x_head;
                const T* const y = static_cast<const T*>(side.dy) + t * side.dy_token + ahead.h * side.dy_head;
                uint4* const to = ring + ahead.slot * kPieces * kThreads;
                if (unit[0].a < g.dim) copy_async(to, x + unit[0].a);
                if (unit[0].b < g.dim) copy_async(to + kThreads, x + unit[0].b);
                if (unit[0].a < g.dim) copy_async(to + 2 * kThreads, y + unit[0].a);
                if (unit[0].b < g.dim) copy_async(to + 3 * kThreads, y + unit[0].b);
            }
            ahead.t += side.step_t, ahead.h += side.step_h;
            if (ahead.h >= side.heads) ahead.h -= side.heads, ++ahead.t;
            --ahead.left;
        }
        ahead.slot = (ahead.slot + 1) % kStages;
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int now = 0;  // the slot of the present vector
    if (kRing) {
#pragma unroll
        for (int i = 0; i < kPieces * kStages; ++i)
            if ((i & 1 ? unit[0].b : unit[0].a) >= g.dim) ring[i * kThreads] = make_uint4(0, 0, 0, 0);  // pieces that are not there
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) copy_next();
    }
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int t0 = tile * g.tile, n = min(g.tile, g.tokens - t0), half = g.rotary / 2;
        __syncthreads();
        for (int i = threadIdx.x; i < n * g.angles; i += kThreads) {
            const int t = i / g.angles, f = i - t * g.angles;
            if (f >= half) continue;
            double turns = (double)g.positions[t0 + t] * g.frequencies[f] * 0.15915494309189533577;  // 1 / (2 pi)
            turns -= rint(turns);
            sincospif((float)(2.0 * turns), &sn[i], &cs[i]);
        }
        __syncthreads();
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const Side& side = g.side[which];
            const int rows = n * side.heads;
            const T* const px = static_cast<const T*>(side.x) + (int64_t)t0 * side.x_token;
            const T* const py = static_cast<const T*>(side.dy) + (int64_t)t0 * side.dy_token;
            T* const po = static_cast<T*>(side.out) + (int64_t)t0 * side.out_token;
            Row<T, V> rx[U], ry[U], nx[U], ny[U];
            const int step_t = groups / max(side.heads, 1), step_h = groups - step_t * side.heads;
            int t = group / max(side.heads, 1), h = group - t * side.heads;
            auto fetch = [&](Row<T, V>(&x)[U], Row<T, V>(&y)[U], int t, int h) {
                if (t >= n) return;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    x[u].load(px + t * side.x_token + h * side.x_head, unit[u], g.dim);
                    if (BACK) y[u].load(py + t * side.dy_token + h * side.dy_head, unit[u], g.dim);
                }
            };
            if (!kRing && rows) fetch(rx, ry, t, h);
            for (int first = 0; first < rows; first += groups) {
                int next_t = t + step_t, next_h = h + step_h;
                if (next_h >= side.heads) next_h -= side.heads, ++next_t;
                if constexpr (kRing) {
                    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
                    const uint4* const from = ring + now * kPieces * kThreads;
                    rx[0].take(from[0], from[kThreads]);
                    ry[0].take(from[2 * kThreads], from[3 * kThreads]);
                    now = (now + 1) % kStages;
                    copy_next();
                } else {
                    fetch(nx, ny, next_t, next_h);
                }
                const bool live = t < n;
                const int at = min(t, n - 1);
                T* const q = po + at * side.out_token + h * side.out_head;
                const float *c = cs + at * g.angles, *s = sn + at * g.angles;
                Pair x[U][V], y[U][V], w[U][V], ss = both(0.f), gx = both(0.f);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    rx[u].get(x[u]);
                    if (BACK) {
                        ry[u].get(y[u]);
                        if (unit[u].turns) turn<V, INTER, true>(y[u], c + unit[u].angle, s + unit[u].angle);
                        weights<V>(s_weight[which], unit[u], w[u]);
                    }
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        ss = fma2(x[u][i], x[u][i], ss);
                        if (BACK) w[u][i] = y[u][i] * w[u][i], gx = fma2(w[u][i], x[u][i], gx);
                    }
                }
                const float v = fmaf(group_sum(total(ss), lanes), g.per_dim, g.eps);
                float f = inverse_root(v), mean = BACK ? f * group_sum(total(gx), lanes) * g.per_dim : 0.f;  // of n = x r times the gradient
                // sums that leave the range of 32 bits, or come near: again, of x times a power of two
                const bool far = !(v > 0x1p-60f && v < 0x1p100f);
                if (__any_sync(0xFFFFFFFFu, far)) {
                    const float unit = v < 1.f ? 0x1p80f : 0x1p-100f;
                    ss = gx = both(0.f);
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            const Pair z = x[u][i] * both(unit);
                            ss = fma2(z, z, ss);
                            if (BACK) gx = fma2(w[u][i], z, gx);
                        }
                    const float r = rsqrtf(fmaf(group_sum(total(ss), lanes), g.per_dim, g.eps * unit * unit)), c = BACK ? group_sum(total(gx), lanes) : 0.f;
                    if (far) f = r * unit, mean = r * c * g.per_dim;
                }
                if (!BACK) {
                    const Pair f2 = both(f);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        weights<V>(s_weight[which], unit[u], w[u]);
#pragma unroll
                        for (int i = 0; i < V; ++i) x[u][i] = x[u][i] * f2 * w[u][i];
                        if (unit[u].turns) turn<V, INTER, false>(x[u], c + unit[u].angle, s + unit[u].angle);
                        if (live) Row<T, V>::store(q, unit[u], g.dim, x[u]);
                    }
                } else {
                    const Pair m2 = both(-mean), f2 = both(f);
                    if (live) {
#pragma unroll
                        for (int u = 0; u < U; ++u) {
#pragma unroll
                            for (int i = 0; i < V; ++i) {
                                const Pair n = x[u][i] * f2;
                                dw[BACK ? which : 0][u][i] = fma2(y[u][i], n, dw[BACK ? which : 0][u][i]);
                                x[u][i] = fma2(n, m2, w[u][i]) * f2;
                            }
                            Row<T, V>::store(q, unit[u], g.dim, x[u]);
                        }
                    }
                }
                if (!kRing) {
#pragma unroll
                    for (int u = 0; u < U; ++u) rx[u] = nx[u], ry[u] = ny[u];
                }
                t = next_t, h = next_h;
            }
        }
    }
    if (!BACK || !g.part) return;
    // the block's sums: group after group, in order
#pragma unroll
    for (int which = 0; which < (BACK ? 2 : 1); ++which) {
        __syncthreads();
        float* const sums = smem;  // [groups][dim]
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float2 d = split(dw[which][u][i]);
                const int c = V == 1 ? unit[u].a : 2 * i < V ? unit[u].a + 2 * i : unit[u].b + 2 * i - V, e = V == 1 ? unit[u].b : c + 1;
                if (c < g.dim) sums[group * g.dim + c] = d.x;
                if (e < g.dim) sums[group * g.dim + e] = d.y;
            }
        __syncthreads();
        for (int c = threadIdx.x; c < g.dim; c += kThreads) {
            float s = 0.f;
            for (int i = 0; i < groups; ++i) s += sums[i * g.dim + c];
            g.part[((int64_t)blockIdx.x * 2 + which) * g.dim + c] = s;
        }
    }
}

// Sums of the blocks' rows, in a fixed order: 32 columns a block, 32 warps with every 32nd row each.
template <class W>
__global__ void __launch_bounds__(1024) k_join_weights(const float* part, int blocks, int dim, W* dq, W* dk) {
    __shared__ float sums[32][33];
    wait_for_predecessor();
    const int lane = threadIdx.x % 32, c = blockIdx.x * 32 + lane, warp = threadIdx.x / 32;
    float s = 0.f;
#pragma unroll 4
    for (int b = warp; b < blocks; b += 32)
        if (c < dim) s += part[((int64_t)b * 2 + blockIdx.y) * dim + c];
    sums[warp][lane] = s;
    __syncthreads();
    W* out = blockIdx.y ? dk : dq;
    s = sums[lane][warp];  // a warp has a column now
    for (int m = 16; m; m >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, m);
    if (lane == 0 && blockIdx.x * 32 + warp < dim && out) out[blockIdx.x * 32 + warp] = from_f<W>(s);
}

int size_of(int type) { return type == ONES_F32 ? 4 : 2; }

bool bad_heads(const ones_heads& h, int dim, int tokens) {
    return h.heads < 0 || h.heads > ONES_MAX_HEADS || (h.heads > 1 && h.head < dim) || (h.token < 0 && tokens > 1);
}

template <class T, int V, int U, bool INTER>
cudaError_t launch(Args& a, bool back, cudaStream_t stream, int* blocks) {
    const int units = V == 1 ? (a.dim + 1) / 2 : (a.dim / V + 1) / 2;
    a.group_log = 0;
    while ((1 << a.group_log) * U < units) ++a.group_log;
    const int groups = kThreads >> a.group_log, heads = max(1, a.side[0].heads + a.side[1].heads);
    // Tokens of a block at a time: enough vectors for sixteen rounds of all groups, so that the angles and the barriers around them
    // weigh little (65536 x 40 x 128 forward: four rounds 305 us, eight 274, sixteen 242), or fewer, so that all blocks together take
    // a whole number of turns. Their angles take 32 KB at most, so that five blocks are on an SM.
    a.angles = (a.rotary / 2 + 3) / 4 * 4;
    for (Side& s : a.side) s.step_t = groups / max(s.heads, 1), s.step_h = groups - s.step_t * s.heads;
    const int most = max(1, min(min(64, 16 * groups / heads), 4096 / max(a.angles, 1)));
    const int64_t slots = (back ? 2 : 5) * device_sms(), turns = (a.tokens - 1) / (most * slots) + 1;
    a.tile = (int)((a.tokens - 1) / (turns * slots)) + 1;
    const int tiles = (a.tokens - 1) / a.tile + 1;
    *blocks = back ? min(tiles, kMaxBlocks) : tiles;
    const int smem = max(2 * a.tile * a.angles * 4 + (back && V > 1 ? kRingBytes : 0), back && a.part ? groups * a.dim * 4 : 0);
    auto kernel = back ? k_qk_norm<T, V, U, INTER, true> : k_qk_norm<T, V, U, INTER, false>;
    if (smem > 46 * 1024) {  // with the weights in shared memory, what a launch gets without asking
        static std::atomic<uint64_t> ready[2];
        const cudaError_t err = allow_smem(kernel, 32 * 1024 + kRingBytes, ready[back]);
        if (err != cudaSuccess) return err;
    }
    kernel<<<*blocks, kThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

template <class T>
cudaError_t launch_of(Args& a, bool back, bool wide, cudaStream_t stream, int* blocks) {
    constexpr int V = 16 / sizeof(T);
    if (wide) return a.interleaved ? launch<T, V, 1, true>(a, back, stream, blocks) : launch<T, V, 1, false>(a, back, stream, blocks);
    return a.interleaved ? launch<T, 1, 4, true>(a, back, stream, blocks) : launch<T, 1, 4, false>(a, back, stream, blocks);
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
    // Pieces of 16 bytes: every vector starts on the boundary of one, and none holds both rotated values and others.
    bool wide = dim % v == 0 && rotary % (2 * v) == 0;
    for (int i = 0; i < 2; ++i) {
        if (x[i]->heads != o[i]->heads || (back && x[i]->heads != y[i]->heads) || x[i]->heads < 0 || x[i]->heads > ONES_MAX_HEADS)
            return ONES_ERR_BAD_PARAM;
        for (const ones_heads* h : {x[i], o[i], back ? y[i] : x[i]}) {
            if (!h->heads) continue;
            if (bad_heads(*h, dim, tokens)) return ONES_ERR_BAD_PARAM;
            if (tokens && !h->d_data) return ONES_ERR_NULL;
            if (!aligned(h->d_data, size)) return ONES_ERR_ALIGN;
            wide = wide && aligned(h->d_data, v * size) && (h->heads == 1 || h->head % v == 0) && (tokens <= 1 || h->token % v == 0);
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
    a.tokens = tokens, a.dim = dim, a.rotary = rotary, a.interleaved = interleaved != 0, a.wf32 = wtype == ONES_F32, a.eps = eps, a.per_dim = 1.f / dim;
    int blocks = 0;
    err = type == ONES_F32 ? launch_of<float>(a, back, wide, stream, &blocks)
          : type == ONES_BF16 ? launch_of<__nv_bfloat16>(a, back, wide, stream, &blocks)
                              : launch_of<__half>(a, back, wide, stream, &blocks);
    if (err == cudaSuccess && sums) {
        const dim3 grid((dim + 31) / 32, 2);
        err = wtype == ONES_F32 ? launch_after(k_join_weights<float>, grid, dim3(1024), stream, a.part, blocks, dim, (float*)q_dweight, (float*)k_dweight)
              : wtype == ONES_BF16 ? launch_after(k_join_weights<__nv_bfloat16>, grid, dim3(1024), stream, a.part, blocks, dim,
                                                  (__nv_bfloat16*)q_dweight, (__nv_bfloat16*)k_dweight)
                                   : launch_after(k_join_weights<__half>, grid, dim3(1024), stream, a.part, blocks, dim, (__half*)q_dweight,
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
