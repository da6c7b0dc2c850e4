// Orthogonalised update of matrix parameters by Newton-Schulz products.
#include <math.h>

#include "ones_matmul.cuh"
#include "ones_train.h"
#include "ones_train_internal.h"

namespace ones {

namespace {

constexpr int kNormThreads = 256, kNormBlocks = 128;  // a warp takes a row at a time

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

// Sum of squares of each matrix, in 64 bits (squares of small gradients leave the range of 32), one part per block.
__global__ void __launch_bounds__(kNormThreads) k_ns_norm(Source g, double* part) {
    __shared__ double s[kNormThreads / 32];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    double sum = 0.0;
    for (int r = blockIdx.x * (kNormThreads / 32) + warp; r < g.m; r += gridDim.x * (kNormThreads / 32)) {
        const int64_t at = blockIdx.y * g.stride + r * g.ld;
        if (g.wide) {
            for (int c = lane * 8; c < g.n; c += 256) {
                float v[8];
                load8(g.p, at + c, g.type, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += (double)v[i] * v[i];
            }
        } else {
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

// X0 = G * 2^-k in 11 significant bits, k such that the values' root mean square is about 1: exact for bfloat16 (8 bits)
// down to 2^-14 of it. What is missing to G / (|G| + eps), f = 2^k / (|G| + eps), and f^2, go into the first step's epilogues.
__global__ void __launch_bounds__(kNormThreads) k_ns_cast(Source g, const double* part, int parts, float eps, __half* x, int64_t ldx,
                                                          float2* factor) {
    wait_for_predecessor();
    let_successor_start();
    __shared__ float s_scale;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (warp == 0) {
        double sum = 0.0;
        for (int i = lane; i < parts; i += 32) sum += part[blockIdx.y * parts + i];
        for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        if (lane == 0) {
            const double norm = sqrt(sum), rms = norm / sqrt((double)g.m * g.n);
            int k = rms > 0.0 && rms < 1e300 ? ilogb(rms) : 0;
            k = k < -120 ? -120 : k > 120 ? 120 : k;
            s_scale = ldexpf(1.f, -k);
            if (blockIdx.x == 0) {
                const double f = ldexp(1.0, k) / (norm + eps);
                factor[blockIdx.y] = make_float2((float)f, (float)(f * f));
            }
        }
    }
    __syncthreads();
    const float scale = s_scale;
    for (int r = blockIdx.x * (kNormThreads / 32) + warp; r < g.m; r += gridDim.x * (kNormThreads / 32)) {
        const int64_t at = blockIdx.y * g.stride + r * g.ld;
        __half* out = x + ((int64_t)blockIdx.y * g.m + r) * ldx;
        if (g.wide) {
            for (int c = lane * 8; c < g.n; c += 256) {
                float v[8];
                load8(g.p, at + c, g.type, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= scale;
                *reinterpret_cast<uint4*>(out + c) = make_uint4(Half16::pack(v[0], v[1], true), Half16::pack(v[2], v[3], true),
                                                                Half16::pack(v[4], v[5], true), Half16::pack(v[6], v[7], true));
            }
        } else {
            for (int c = lane; c < g.n; c += 32) out[c] = __float2half_rn(load_as_float(g.p, at + c, g.type) * scale);
        }
    }
}

// The symmetric products' tiles lie on and above the diagonal; what they hold is stored on both sides of it.
__device__ __forceinline__ void store_both(__half* out, int64_t ld, int s, int row, int col, bool mirror, const float (&v)[64], const Turn& turn) {
    uint16_t* p = reinterpret_cast<uint16_t*>(out);
    turn.put16(v, true);
    turn.store16(p, ld, row - turn.lane, col, s, s, true);
    if (!mirror || row >= s) return;
    p += (int64_t)col * ld + row;
#pragma unroll
    for (int i = 0; i < 64; ++i, p += ld)
        if (col + i < s) *p = __half_as_ushort(__float2half_rn(v[i]));
}

// A = factor * X X^T
struct EpiGram {
    struct Args {
        __half* out;
        int64_t ld, batch_ld;
        int s;
        float factor;
        const float2* first;  // the first step's f^2, or NULL
    };
    template <int W>
    static __device__ __forceinline__ void tile(const Args& a, const MatShape&, uint32_t acc, int row, int col,
                                                const TileAt& at, int, const Turn& turn) {
        const float f = a.first ? a.first[at.b].y : a.factor;
#pragma unroll 1
        for (int c = 0; c < W && col + c < a.s; c += 64) {
            float v[64];
            tmem_load(acc + c, v);
#pragma unroll
            for (int i = 0; i < 64; ++i) v[i] *= f;
            store_both(a.out + at.b * a.batch_ld, a.ld, a.s, row, col + c, at.m != at.n, v, turn);
        }
    }
};

// B = a I + b A + c A A. With a I inside B the next product needs no second operand, and B's values near the end are
// those of a I + b A + c A^2 (about 1), not of its terms (several times that), so its rounding is finer.
struct EpiPoly {
    struct Args {
        const __half* gram;
        __half* out;
        int64_t ld, batch_ld;
        int s;
        float a, b, c;
    };
    template <int W>
    static __device__ __forceinline__ void tile(const Args& a, const MatShape&, uint32_t acc, int row, int col,
                                                const TileAt& at, int, const Turn& turn) {
#pragma unroll 1
        for (int c = 0; c < W && col + c < a.s; c += 64) {
            // A's values, 8 lanes to a row, by the same way that the result leaves
            const __half* gram = a.gram + at.b * a.batch_ld;
            const int k = turn.lane & 7, at_col = col + c + 8 * k;
            uint4 q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = row - turn.lane + 4 * i + turn.lane / 8;  // rows of A are padded to whole 16 bytes
                q[i] = r < a.s && at_col < a.s ? *reinterpret_cast<const uint4*>(gram + (int64_t)r * a.ld + at_col) : make_uint4(0, 0, 0, 0);
            }
            float v[64];
            tmem_load(acc + c, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) turn.chunk(4 * i + turn.lane / 8, k) = q[i];
            __syncwarp();
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
            if (d < 64u) {
#pragma unroll
                for (int i = 0; i < 64; ++i)
                    if (d == (unsigned)i) v[i] += a.a;
            }
            store_both(a.out + at.b * a.batch_ld, a.ld, a.s, row, col + c, at.m != at.n, v, turn);
            __syncwarp();
        }
    }
};

// X = factor * B X
struct EpiApply {
    struct Args {
        uint16_t* out;
        int64_t ld, batch_ld;
        int m, n;
        float factor;
        const float2* first;  // the first step's f, or NULL
        bool f16, wide;
    };
    template <int W>
    static __device__ __forceinline__ void tile(const Args& a, const MatShape&, uint32_t acc, int row, int col,
                                                const TileAt& at, int, const Turn& turn) {
        const float f = a.first ? a.factor * a.first[at.b].x : a.factor;
#pragma unroll 1
        for (int c = 0; c < W && col + c < a.n; c += 64) {
            float v[64];
            tmem_load(acc + c, v);
#pragma unroll
            for (int i = 0; i < 64; ++i) v[i] *= f;
            turn.put16(v, a.f16);
            turn.store16(a.out + at.b * a.batch_ld, a.ld, row - turn.lane, col + c, a.m, a.n, a.wide);
        }
    }
};

inline size_t up(size_t x, size_t a) { return (x + a - 1) / a * a; }

struct Layout {
    size_t factor, part, x0, x1, gram, poly, total;
    int64_t ldx, lds;
    int s;
};
Layout layout(int32_t count, int32_t m, int32_t n) {
    Layout L;
    L.s = m < n ? m : n;
    L.ldx = (int64_t)up(n, 8);
    L.lds = (int64_t)up(L.s, 8);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = up(at + bytes, 256);
        return here;
    };
    L.factor = take((size_t)count * sizeof(float2));
    L.part = take((size_t)count * kNormBlocks * 8);
    L.x0 = take((size_t)count * m * L.ldx * 2);
    L.x1 = take((size_t)count * m * L.ldx * 2);
    L.gram = take((size_t)count * L.s * L.lds * 2);
    L.poly = take((size_t)count * L.s * L.lds * 2);
    L.total = at;
    return L;
}

bool bad_sizes(int32_t count, int32_t m, int32_t n) {
    return count < 1 || m < 1 || n < 1 || count > 65535 || m > (1 << 20) || n > (1 << 20);
}

}  // namespace

cudaError_t update_wait_expired(unsigned* out) {
    cudaError_t err = cudaMemcpyFromSymbol(out, g_wait_expired, sizeof(*out));
    const unsigned zero = 0;
    if (err == cudaSuccess && *out) err = cudaMemcpyToSymbol(g_wait_expired, &zero, sizeof(zero));
    return err;
}

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
    if (bad_sizes(count, m, n) || type < ONES_F32 || type > ONES_F16 || steps < 1 || !(eps > 0.f) || !isfinite(eps) ||
        !isfinite(a) || !isfinite(b) || !isfinite(c) || ldg < n || (count > 1 && stride < 0))
        return ONES_ERR_BAD_PARAM;
    if (!d_g || !d_out || !d_workspace) return ONES_ERR_NULL;
    const int size = type == ONES_F32 ? 4 : 2;
    if (!aligned(d_g, size) || !aligned(d_out, 2) || !aligned(d_workspace, 256)) return ONES_ERR_ALIGN;
    const Layout L = layout(count, m, n);
    if (workspace_bytes < L.total) return ONES_ERR_WORKSPACE;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(d_workspace);
    float2* factor = reinterpret_cast<float2*>(ws + L.factor);
    double* part = reinterpret_cast<double*>(ws + L.part);
    __half* x[2] = {reinterpret_cast<__half*>(ws + L.x0), reinterpret_cast<__half*>(ws + L.x1)};
    __half* gram = reinterpret_cast<__half*>(ws + L.gram);
    __half* poly = reinterpret_cast<__half*>(ws + L.poly);
    const int s = L.s;
    const bool tall = m > n;  // the products run on the columns then
    const int64_t xs = (int64_t)m * L.ldx, ss = (int64_t)s * L.lds;

    const bool wide = n % 8 == 0 && aligned(d_g, 16) && ldg * size % 16 == 0 && stride * size % 16 == 0;
    const Source src = {d_g, ldg, count > 1 ? stride : 0, m, n, type, wide};
    int blocks = (m + kNormThreads / 32 - 1) / (kNormThreads / 32);
    if (blocks > kNormBlocks) blocks = kNormBlocks;
    k_ns_norm<<<dim3(blocks, count), kNormThreads, 0, stream>>>(src, part);
    cudaError_t err = cudaGetLastError();
    if (err == cudaSuccess)
        err = launch_after(k_ns_cast, dim3(blocks, count), dim3(kNormThreads), stream, src, part, blocks, eps, x[0], L.ldx, factor);
    // Between the steps X is kept times 2^p, about the square root of the longer side, which brings its values near 1:
    // after the last step they are about 1 / 2^p, before the first about 1 / sqrt(m n).
    int p = 0;
    while ((int64_t)1 << (2 * (p + 1)) <= (m > n ? m : n)) ++p;
    const float unit = ldexpf(1.f, p), one_over = ldexpf(1.f, -p);
    for (int k = 0; err == cudaSuccess && k < steps; ++k) {
        const __half* in = x[k & 1];
        const float2* first = k == 0 ? factor : nullptr;
        const EpiGram::Args eg = {gram, L.lds, ss, s, one_over * one_over, first};
        err = tall ? launch_matmul<true, true, EpiGram>({in, L.ldx, xs, true}, {in, L.ldx, xs, true}, s, s, m, count, true, true, eg, stream, true)
                   : launch_matmul<false, false, EpiGram>({in, L.ldx, xs, false}, {in, L.ldx, xs, false}, s, s, n, count, true, true, eg, stream, true);
        if (err != cudaSuccess) break;
        const EpiPoly::Args ep = {gram, poly, L.lds, ss, s, a, b, c};
        err = launch_matmul<false, false, EpiPoly>({gram, L.lds, ss, false}, {gram, L.lds, ss, false}, s, s, s, count, true, true, ep, stream, true);
        if (err != cudaSuccess) break;
        const bool last = k + 1 == steps;
        EpiApply::Args ea = {reinterpret_cast<uint16_t*>(x[1 - (k & 1)]), L.ldx, xs, m, n, 1.f, first, true, true};
        if (first) ea.factor = unit;
        if (last) {
            ea.out = static_cast<uint16_t*>(d_out), ea.ld = n, ea.batch_ld = (int64_t)m * n;
            ea.factor = first ? 1.f : one_over;
            ea.f16 = false;
            ea.wide = n % 8 == 0 && aligned(d_out, 16);
        }
        err = tall ? launch_matmul<false, false, EpiApply>({in, L.ldx, xs, false}, {poly, L.lds, ss, false}, m, n, s, count, false, true, ea, stream, true)
                   : launch_matmul<false, true, EpiApply>({poly, L.lds, ss, false}, {in, L.ldx, xs, true}, m, n, s, count, false, true, ea, stream, true);
    }
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // extern "C"
