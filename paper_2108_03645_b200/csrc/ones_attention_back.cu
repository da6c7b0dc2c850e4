// Gradients of the causal attention.
//
// Two passes over the pairs of tiles, each with sums that stay in tensor memory until they are whole: one for each tile of
// keys (dk and dv: scores, dp and two products over the queries behind it, all heads of the group one after the other), one for
// each tile of queries (dq: scores, dp and one product over the keys before it). Seven products where five would do if dq
// were added up in memory: but that takes 64 KB of atomic additions for every pair of tiles, whose order would change the
// results, or turns taken between blocks. A pair costs 2048 + 1536 cycles of products and 2 x 1024 of exponentials.
#include "ones_attention.cuh"

#include <math.h>

namespace ones {

namespace {

constexpr int kThreads = 384;  // two groups of four warps that work on scores, then load, multiply, statistics and an idle warp

struct BackArgs {
    const Item* items;
    const PlanHead* head;
    const float *lse, *delta;   // [tokens][heads]
    const unsigned* largest;    // [2][kv]: bits of the largest |dout|^2 and |v|^2 of a head (float16)
    HeadsOut dq, dk, dv;
    int tokens, heads, kv, group, kt, dim;
    float scale;
};

// float16 holds the probabilities times 2^12, and the scores' gradients times a power of two that takes their bound
// 2 max |dout| max |v| to 2^15: so that what is small beside it keeps its bits. bfloat16 has the range of 32 bits.
constexpr float kLift = 12.f;
template <bool F16>
__device__ __forceinline__ float gradient_scale(const BackArgs& g, int h) {
    if (!F16) return 1.f;
    const float bound = 2.f * sqrtf(__uint_as_float(g.largest[h])) * sqrtf(__uint_as_float(g.largest[g.kv + h]));
    if (!(bound > 0.f)) return 1.f;
    const int e = min(max(14 - ilogbf(bound), -100), 100);
    return exp2f((float)e);
}

// ---- delta = dout . out, and the largest rows ----

struct DeltaArgs {
    const uint16_t *dout, *out, *v;
    int64_t dout_token, dout_head, out_token, out_head, v_token, v_head;
    const PlanHead* head;
    float* delta;
    unsigned* largest;
    int tokens, heads, kv, dim, wide;
};

template <bool F16>
__device__ __forceinline__ float value16(uint16_t b) {
    return F16 ? __half2float(__ushort_as_half(b)) : __uint_as_float((uint32_t)b << 16);
}

// 16 lanes for a row of up to 128 values: pieces of 8 where both rows have them, single values otherwise.
template <bool F16>
__global__ void __launch_bounds__(256) k_delta(const DeltaArgs g) {
    wait_for_predecessor();
    let_successor_start();
    const int lane = threadIdx.x % 16;
    const int64_t rows = (int64_t)g.tokens * (g.heads + (F16 ? g.kv : 0));
    const int t0 = g.head->covered[0], t1 = g.head->covered[1];
    for (int64_t r0 = (int64_t)blockIdx.x * 16; r0 < rows; r0 += (int64_t)gridDim.x * 16) {
        const int64_t r = r0 + threadIdx.x / 16;
        const bool is_v = r >= (int64_t)g.tokens * g.heads;
        const int64_t q = is_v ? r - (int64_t)g.tokens * g.heads : r;
        const int n = is_v ? g.kv : g.heads;
        const int t = (int)(q / n), h = (int)(q - (int64_t)t * n);
        float dot = 0.f, square = 0.f;
        if (r < rows && t >= t0 && t < t1) {
            const uint16_t* a = is_v ? g.v + t * g.v_token + h * g.v_head : g.dout + t * g.dout_token + h * g.dout_head;
            const uint16_t* b = is_v ? a : g.out + t * g.out_token + h * g.out_head;
            if (g.wide) {
                const int c = 8 * lane;
                if (c < g.dim) {
                    const uint4 x = *reinterpret_cast<const uint4*>(a + c), y = *reinterpret_cast<const uint4*>(b + c);
                    const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float u = value16<F16>((uint16_t)(xw[i / 2] >> (16 * (i & 1)))), w = value16<F16>((uint16_t)(yw[i / 2] >> (16 * (i & 1))));
                        dot = fmaf(u, w, dot), square = fmaf(u, u, square);
                    }
                }
            } else {
                for (int c = lane; c < g.dim; c += 16) {
                    const float u = value16<F16>(a[c]), w = value16<F16>(b[c]);
                    dot = fmaf(u, w, dot), square = fmaf(u, u, square);
                }
            }
        }
#pragma unroll
        for (int m = 8; m; m >>= 1) {
            dot += __shfl_xor_sync(0xFFFFFFFFu, dot, m);
            if (F16) square += __shfl_xor_sync(0xFFFFFFFFu, square, m);
        }
        if (lane || r >= rows) continue;
        if (!is_v) g.delta[r] = dot;
        if (F16 && square > 0.f && square < INFINITY) {
            unsigned* at = g.largest + (is_v ? g.kv + h : h / (g.heads / g.kv));
            if (__float_as_uint(square) > *reinterpret_cast<volatile unsigned*>(at)) atomicMax(at, __float_as_uint(square));
        }
    }
}

template <int HALVES>
struct Back {
    static constexpr int kTile = HALVES * kHalfTile;
    // dq: queries and dout of the tile, rings of keys (needed until the last product) and values
    static constexpr int kKeySlots = HALVES == 2 ? 3 : 4, kValueSlots = HALVES == 2 ? 2 : 3;
    static constexpr int kSmemQueries = (2 + kKeySlots + kValueSlots) * kTile + 1024;
    // dk, dv: keys and values of the tile, rings of queries and dout, their statistics
    static constexpr int kSlots = HALVES == 2 ? 2 : 4;
    static constexpr int kStats = 2;
    static constexpr int kSmemKeys = (2 + 2 * kSlots) * kTile + kStats * 2 * kRows * 4 + 1024;
};

// ---- dq ----

struct QueriesShared {
    uint64_t q_full, q_free, k_full[4], k_empty[4], v_full[4], v_empty[4], s_full[2], dp_full, dp_free, ds_full[2], acc_full;
    uint32_t tmem;
};

// Tiles of keys that a tile of queries meets.
__device__ __forceinline__ int key_tiles(const Item& it, int kt) {
    return it.begin < 0 ? 0 : (min(it.first + kt, it.end) - 1 - it.begin) / kKeys + 1;
}

template <int HALVES, bool F16>
__global__ void __launch_bounds__(kThreads, 1)
    k_attention_queries(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_do,
                        const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const BackArgs g) {
    using B = Back<HALVES>;
    constexpr int kKS = B::kKeySlots, kVS = B::kValueSlots;
    extern __shared__ uint8_t smem_raw[];
    __shared__ QueriesShared sh;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t at_q = base, at_do = base + B::kTile, at_k = base + 2 * B::kTile, at_v = at_k + kKS * B::kTile;
    const uint32_t q_full = smem_u32(&sh.q_full), q_free = smem_u32(&sh.q_free), k_full = smem_u32(sh.k_full), k_empty = smem_u32(sh.k_empty),
                   v_full = smem_u32(sh.v_full), v_empty = smem_u32(sh.v_empty), s_full = smem_u32(sh.s_full), dp_full = smem_u32(&sh.dp_full),
                   dp_free = smem_u32(&sh.dp_free), ds_full = smem_u32(sh.ds_full), acc_full = smem_u32(&sh.acc_full);
    if (threadIdx.x == 0) {
        tma_prefetch(&map_q), tma_prefetch(&map_do), tma_prefetch(&map_k), tma_prefetch(&map_v);
        bar_init(q_full, 1), bar_init(q_free, 1), bar_init(dp_full, 1), bar_init(dp_free, 8), bar_init(acc_full, 1);
        for (int i = 0; i < 2; ++i) bar_init(s_full + 8 * i, 1), bar_init(ds_full + 8 * i, 8);
        for (int i = 0; i < 4; ++i) bar_init(k_full + 8 * i, 1), bar_init(k_empty + 8 * i, 1), bar_init(v_full + 8 * i, 1), bar_init(v_empty + 8 * i, 1);
        bar_init_done();
    }
    if (warp == 9) tmem_alloc<1>(smem_u32(&sh.tmem), 512);
    mma_fence_before();
    __syncthreads();
    mma_fence_after();
    const uint32_t tmem = sh.tmem, t_dp = tmem + 256, t_acc = tmem + 384;
    wait_for_predecessor();
    let_successor_start();
    const int64_t total = (int64_t)g.head->count * g.kv;
    bool ok = true;

    if (warp == 8) {
        // load
        int ks = 0, vs = 0;
        uint32_t kph = 0, vph = 0, qph = 0;
        const uint32_t qbytes = HALVES * g.group * g.kt * 128;
        for (int turn = 0; ok; ++turn) {
            const int64_t w = work_at(turn);
            if ((int64_t)turn * gridDim.x >= total) break;
            if (w >= total) continue;
            const Item it = g.items[w / g.kv];
            const int h = (int)(w % g.kv), tiles = key_tiles(it, g.kt);
            if (!tiles) continue;
            if (!(ok = warp_wait(q_free, qph ^ 1))) break;
            qph ^= 1;
            if (elect_one()) {
                bar_expect(q_full, 2 * qbytes);
                for (int x = 0; x < HALVES; ++x) {
                    tma_load<1>(at_q + x * kHalfTile, &map_q, 64 * x, h * g.group, it.first, q_full);
                    tma_load<1>(at_do + x * kHalfTile, &map_do, 64 * x, h * g.group, it.first, q_full);
                }
            }
            __syncwarp();
            for (int j = 0; j < tiles; ++j) {
                if (!(ok = warp_wait(k_empty + 8 * ks, kph ^ 1))) break;
                if (elect_one()) {
                    bar_expect(k_full + 8 * ks, B::kTile);
                    for (int x = 0; x < HALVES; ++x)
                        tma_load<1>(at_k + ks * B::kTile + x * kHalfTile, &map_k, 64 * x, h, it.begin + j * kKeys, k_full + 8 * ks);
                }
                __syncwarp();
                if (++ks == kKS) ks = 0, kph ^= 1;
                if (!(ok = warp_wait(v_empty + 8 * vs, vph ^ 1))) break;
                if (elect_one()) {
                    bar_expect(v_full + 8 * vs, B::kTile);
                    for (int x = 0; x < HALVES; ++x)
                        tma_load<1>(at_v + vs * B::kTile + x * kHalfTile, &map_v, 64 * x, h, it.begin + j * kKeys, v_full + 8 * vs);
                }
                __syncwarp();
                if (++vs == kVS) vs = 0, vph ^= 1;
            }
        }
    } else if (warp == 9) {
        // multiply
        const uint32_t id_s = attend_desc(F16, false, kKeys), id_acc = attend_desc(F16, true, 64 * HALVES);
        const int steps = (g.dim + 15) / 16;
        int ks = 0, vs = 0;
        uint32_t kph = 0, vph = 0, qph = 0, dpph = 0, t = 0;  // t: tiles so far
        for (int turn = 0; ok; ++turn) {
            const int64_t w = work_at(turn);
            if ((int64_t)turn * gridDim.x >= total) break;
            if (w >= total) continue;
            const Item it = g.items[w / g.kv];
            const int tiles = key_tiles(it, g.kt);
            if (!tiles) continue;
            if (!(ok = warp_wait(q_full, qph))) break;
            qph ^= 1;
            int before = 0;  // the slot of the keys whose dq comes next
            for (int j = 0; ok && j <= tiles; ++j) {
                const int slot = ks;
                if (j < tiles) {
                    if (!(ok = warp_wait(k_full + 8 * ks, kph))) break;
                    const int rest = it.end - it.begin - j * kKeys;
                    if (rest < kKeys) clear_rows<HALVES>(smem + (2 + ks) * B::kTile, rest, lane);
                    mma_fence_after();
                    if (elect_one()) {
                        product_rows(tmem + 128 * ((t + j) & 1), at_q, at_k + ks * B::kTile, id_s, steps);
                        mma_commit<1>(s_full + 8 * ((t + j) & 1));
                    }
                    __syncwarp();
                    if (++ks == kKS) ks = 0, kph ^= 1;
                    if (!(ok = warp_wait(v_full + 8 * vs, vph))) break;
                    if (!(ok = warp_wait(dp_free, dpph ^ 1))) break;  // what was there has been read
                    dpph ^= 1;
                    mma_fence_after();
                    if (elect_one()) {
                        product_rows(t_dp, at_do, at_v + vs * B::kTile, id_s, steps);
                        mma_commit<1>(dp_full);
                        mma_commit<1>(v_empty + 8 * vs);
                    }
                    __syncwarp();
                    if (++vs == kVS) vs = 0, vph ^= 1;
                }
                if (j > 0) {
                    const uint32_t i = t + j - 1;
                    if (!(ok = warp_wait(ds_full + 8 * (i & 1), (i >> 1) & 1))) break;
                    mma_fence_after();
                    if (elect_one()) {
                        const uint32_t a = tmem + 128 * (i & 1);
                        product_tmem(t_acc, a, a + 64, at_k + before * B::kTile, id_acc, j > 1);
                        mma_commit<1>(k_empty + 8 * before);
                    }
                    __syncwarp();
                }
                before = slot;
            }
            if (!ok) break;
            t += tiles;
            if (elect_one()) mma_commit<1>(acc_full), mma_commit<1>(q_free);
            __syncwarp();
        }
    } else if (warp < 8) {
        const int half = warp / 4, row = threadIdx.x % 128;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        const float c = g.scale * kLog2e;
        uint32_t t = 0, dpph = 0, aph = 0;
        for (int turn = 0; ok; ++turn) {
            const int64_t w = work_at(turn);
            if ((int64_t)turn * gridDim.x >= total) break;
            if (w >= total) continue;
            const Item it = g.items[w / g.kv];
            const int h = (int)(w % g.kv), tiles = key_tiles(it, g.kt);
            const int token = it.first + row / g.group, head = h * g.group + row % g.group;
            const bool live = row < g.group * g.kt && token < it.end;
            uint16_t* const out = g.dq.p + (int64_t)token * g.dq.token + head * g.dq.head;
            if (it.begin < 0) {
                if (live) {
                    float zero[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) zero[i] = 0.f;
                    for (int x = 0; x < HALVES; ++x) write_columns<F16>(out, 32 * (half * HALVES + x), g.dim, g.dq.wide, zero);
                }
                continue;
            }
            const float sigma = gradient_scale<F16>(g, h), sigma2 = F16 ? sigma * exp2f(-kLift) : 1.f;
            const int64_t at = (int64_t)token * g.heads + head;
            const Pair l2 = both(live ? (F16 ? kLift : 0.f) - g.lse[at] * kLog2e : -INFINITY), d2 = both(live ? -g.delta[at] * sigma2 : 0.f);
            const Pair c2 = both(c), s2 = both(sigma2);
            const int clean = (it.first - it.begin + 1) / kKeys;
            for (int j = 0; j < tiles; ++j, ++t) {
                if (!(ok = warp_wait(s_full + 8 * (t & 1), (t >> 1) & 1))) break;
                mma_fence_after();
                const uint32_t ts = tmem + 128 * (t & 1) + 64 * half + lanes;
                uint32_t s[2][32], dp[2][32];
                tmem_fetch(ts, s[0]), tmem_fetch(ts + 32, s[1]);
                tmem_wait(s[0]), tmem_wait(s[1]);
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const float2 e = split(fma2(pair(__uint_as_float(s[x][i]), __uint_as_float(s[x][i + 1])), c2, l2));
                        s[x][i] = __float_as_uint(exp2_of(e.x)), s[x][i + 1] = __float_as_uint(exp2_of(e.y));
                    }
                if (!(ok = warp_wait(dp_full, dpph))) break;
                dpph ^= 1;
                mma_fence_after();
                tmem_fetch(t_dp + 64 * half + lanes, dp[0]), tmem_fetch(t_dp + 64 * half + 32 + lanes, dp[1]);
                tmem_wait(dp[0]), tmem_wait(dp[1]);
                mma_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(dp_free);
                const int last = token - it.begin - j * kKeys - 64 * half;  // the last key of this half that the row sees
                uint32_t ds[32];
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const Pair p = pair(__uint_as_float(s[x][i]), __uint_as_float(s[x][i + 1]));
                        float2 v = split(p * fma2(pair(__uint_as_float(dp[x][i]), __uint_as_float(dp[x][i + 1])), s2, d2));
                        if (j >= clean) v.x = 32 * x + i > last ? 0.f : v.x, v.y = 32 * x + i + 1 > last ? 0.f : v.y;
                        ds[16 * x + i / 2] = pack16<F16>(v.x, v.y);
                    }
                tmem_store(ts, ds);
                tmem_store_wait();
                mma_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(ds_full + 8 * (t & 1));
            }
            if (!ok) break;
            if (!(ok = warp_wait(acc_full, aph))) break;
            aph ^= 1;
            mma_fence_after();
            const float f = g.scale / sigma;
            for (int x = 0; x < HALVES; ++x) {
                const int col = 32 * (half * HALVES + x);
                uint32_t o[32];
                tmem_fetch(t_acc + col + lanes, o);
                tmem_wait(o);
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(o[i]) * f;
                if (live && col < g.dim) write_columns<F16>(out, col, g.dim, g.dq.wide, v);
            }
            mma_fence_before();
        }
    }
    if (!ok) let_copies_end();
    __syncwarp();
    mma_fence_before();
    __syncthreads();
    mma_fence_after();
    if (warp == 9) tmem_free<1>(tmem, 512);
}

// ---- dk and dv ----

struct KeysShared {
    uint64_t kv_full, kv_free, q_full[4], q_empty[4], do_full[4], do_empty[4], st_full[2], st_empty[2], s_full, p_full, dp_full, ds_full, acc_full;
    uint32_t tmem;
};

// Tiles of queries that see a tile of keys: from the one that holds its first token to the sequence's last.
struct QuerySpan {
    int first, tiles;  // first token of the first tile
};
__device__ __forceinline__ QuerySpan query_span(const Item& it, int kt) {
    if (it.begin < 0) return {0, 0};
    const int f = (it.first - it.begin) / kt;
    return {it.begin + f * kt, (it.end - it.begin + kt - 1) / kt - f};
}

template <int HALVES, bool F16>
__global__ void __launch_bounds__(kThreads, 1)
    k_attention_keys(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_do,
                     const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const BackArgs g) {
    using B = Back<HALVES>;
    constexpr int kS = B::kSlots;
    extern __shared__ uint8_t smem_raw[];
    __shared__ KeysShared sh;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t at_k = base, at_v = base + B::kTile, at_q = base + 2 * B::kTile, at_do = at_q + kS * B::kTile;
    float* const stats = reinterpret_cast<float*>(smem + (2 + 2 * kS) * B::kTile);  // [stage][2][128]
    const uint32_t kv_full = smem_u32(&sh.kv_full), kv_free = smem_u32(&sh.kv_free), q_full = smem_u32(sh.q_full), q_empty = smem_u32(sh.q_empty),
                   do_full = smem_u32(sh.do_full), do_empty = smem_u32(sh.do_empty), st_full = smem_u32(sh.st_full), st_empty = smem_u32(sh.st_empty),
                   s_full = smem_u32(&sh.s_full), p_full = smem_u32(&sh.p_full), dp_full = smem_u32(&sh.dp_full), ds_full = smem_u32(&sh.ds_full),
                   acc_full = smem_u32(&sh.acc_full);
    const int qrows = g.group * g.kt;
    if (threadIdx.x == 0) {
        tma_prefetch(&map_q), tma_prefetch(&map_do), tma_prefetch(&map_k), tma_prefetch(&map_v);
        bar_init(kv_full, 1), bar_init(kv_free, 1), bar_init(s_full, 1), bar_init(p_full, 8), bar_init(dp_full, 1), bar_init(ds_full, 8), bar_init(acc_full, 1);
        for (int i = 0; i < 4; ++i) bar_init(q_full + 8 * i, 1), bar_init(q_empty + 8 * i, 1), bar_init(do_full + 8 * i, 1), bar_init(do_empty + 8 * i, 1);
        for (int i = 0; i < 2; ++i) bar_init(st_full + 8 * i, 32), bar_init(st_empty + 8 * i, 8);
        bar_init_done();
    }
    // rows that no load fills, where the heads of a group do not divide 128: zeros
    for (int s = 0; s < 2 * kS && qrows < kRows; ++s)
        for (int i = qrows * 8 + threadIdx.x; i < kRows * 8; i += kThreads)
            for (int x = 0; x < HALVES; ++x)
                *reinterpret_cast<uint4*>(smem + (2 + s) * B::kTile + x * kHalfTile + i * 16) = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async;" ::: "memory");
    if (warp == 9) tmem_alloc<1>(smem_u32(&sh.tmem), 512);
    mma_fence_before();
    __syncthreads();
    mma_fence_after();
    const uint32_t tmem = sh.tmem, t_dp = tmem + 128, t_dv = tmem + 256, t_dk = tmem + 384;
    wait_for_predecessor();
    let_successor_start();
    const int64_t total = (int64_t)g.head->count * g.kv;
    bool ok = true;

    if (warp == 8) {
        // load
        int slot = 0;
        uint32_t ph = 0, kvph = 0;
        const uint32_t qbytes = HALVES * qrows * 128;
        for (int turn = 0; ok; ++turn) {
            const int64_t w = work_at(turn);
            if ((int64_t)turn * gridDim.x >= total) break;
            if (w >= total) continue;
            const Item it = g.items[w / g.kv];
            const int h = (int)(w % g.kv);
            const QuerySpan q = query_span(it, g.kt);
            if (!q.tiles) continue;
            if (!(ok = warp_wait(kv_free, kvph ^ 1))) break;
            kvph ^= 1;
            if (elect_one()) {
                bar_expect(kv_full, 2 * B::kTile);
                for (int x = 0; x < HALVES; ++x) {
                    tma_load<1>(at_k + x * kHalfTile, &map_k, 64 * x, h, it.first, kv_full);
                    tma_load<1>(at_v + x * kHalfTile, &map_v, 64 * x, h, it.first, kv_full);
                }
            }
            __syncwarp();
            for (int i = 0; ok && i < q.tiles; ++i) {
                for (int kind = 0; ok && kind < 2; ++kind) {
                    const uint32_t full = (kind ? do_full : q_full) + 8 * slot, to = (kind ? at_do : at_q) + slot * B::kTile;
                    if (!(ok = warp_wait((kind ? do_empty : q_empty) + 8 * slot, ph ^ 1))) break;
                    if (elect_one()) {
                        bar_expect(full, qbytes);
                        for (int x = 0; x < HALVES; ++x)
                            tma_load<1>(to + x * kHalfTile, kind ? &map_do : &map_q, 64 * x, h * g.group, q.first + i * g.kt, full);
                    }
                    __syncwarp();
                }
                if (++slot == kS) slot = 0, ph ^= 1;
            }
        }
    } else if (warp == 9) {
        // multiply
        const uint32_t id_s = attend_desc(F16, false, kRows), id_acc = attend_desc(F16, true, 64 * HALVES);
        const int steps = (g.dim + 15) / 16;
        int slot = 0;
        uint32_t ph = 0, kvph = 0, pph = 0, dsph = 0;
        for (int turn = 0; ok; ++turn) {
            const int64_t w = work_at(turn);
            if ((int64_t)turn * gridDim.x >= total) break;
            if (w >= total) continue;
            const Item it = g.items[w / g.kv];
            const QuerySpan q = query_span(it, g.kt);
            if (!q.tiles) continue;
            if (!(ok = warp_wait(kv_full, kvph))) break;
            kvph ^= 1;
            // scores or dp of the tile i, in the slot s
            auto rows = [&](int i, int s, uint32_t parity, bool dp) {
                if (!warp_wait((dp ? do_full : q_full) + 8 * s, parity)) return false;
                const int rest = (it.end - q.first - i * g.kt) * g.group;
                if (rest < qrows) clear_rows<HALVES>(smem + (2 + (dp ? kS : 0) + s) * B::kTile, rest, lane);
                mma_fence_after();
                if (elect_one()) {
                    product_rows(dp ? t_dp : tmem, dp ? at_v : at_k, (dp ? at_do : at_q) + s * B::kTile, id_s, steps);
                    mma_commit<1>(dp ? dp_full : s_full);
                }
                __syncwarp();
                return true;
            };
            if (!(ok = rows(0, slot, ph, false) && rows(0, slot, ph, true))) break;
            for (int i = 0; ok && i < q.tiles; ++i) {
                const int s = slot;
                if (++slot == kS) slot = 0, ph ^= 1;
                if (!(ok = warp_wait(p_full, pph))) break;
                pph ^= 1;
                mma_fence_after();
                if (elect_one()) {
                    product_tmem(t_dv, tmem, tmem + 64, at_do + s * B::kTile, id_acc, i != 0);
                    mma_commit<1>(do_empty + 8 * s);
                }
                __syncwarp();
                if (i + 1 < q.tiles && !(ok = rows(i + 1, slot, ph, false))) break;
                if (!(ok = warp_wait(ds_full, dsph))) break;
                dsph ^= 1;
                mma_fence_after();
                if (elect_one()) {
                    product_tmem(t_dk, t_dp, t_dp + 64, at_q + s * B::kTile, id_acc, i != 0);
                    mma_commit<1>(q_empty + 8 * s);
                }
                __syncwarp();
                if (i + 1 < q.tiles && !(ok = rows(i + 1, slot, ph, true))) break;
            }
            if (!ok) break;
            if (elect_one()) mma_commit<1>(acc_full), mma_commit<1>(kv_free);
            __syncwarp();
        }
    } else if (warp == 10) {
        // statistics of the rows of queries: what the exponent subtracts, and delta
        int stage = 0;
        uint32_t ph = 0;
        for (int turn = 0; ok; ++turn) {
            const int64_t w = work_at(turn);
            if ((int64_t)turn * gridDim.x >= total) break;
            if (w >= total) continue;
            const Item it = g.items[w / g.kv];
            const int h = (int)(w % g.kv);
            const QuerySpan q = query_span(it, g.kt);
            if (!q.tiles) continue;
            const float sigma2 = F16 ? gradient_scale<F16>(g, h) * exp2f(-kLift) : 1.f;
            for (int i = 0; i < q.tiles; ++i) {
                float l[4], d[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int row = 32 * x + lane, token = q.first + i * g.kt + row / g.group, head = h * g.group + row % g.group;
                    const bool live = row < qrows && token < it.end;
                    const int64_t at = (int64_t)token * g.heads + head;
                    l[x] = live ? (F16 ? kLift : 0.f) - g.lse[at] * kLog2e : -INFINITY;
                    d[x] = live ? -g.delta[at] * sigma2 : 0.f;
                }
                if (!(ok = warp_wait(st_empty + 8 * stage, ph ^ 1))) break;
                float* const to = stats + stage * 2 * kRows;
#pragma unroll
                for (int x = 0; x < 4; ++x) to[32 * x + lane] = l[x], to[kRows + 32 * x + lane] = d[x];
                bar_arrive(st_full + 8 * stage);
                if (++stage == B::kStats) stage = 0, ph ^= 1;
            }
        }
    } else if (warp < 8) {
        const int half = warp / 4, row = threadIdx.x % 128;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        const Pair c2 = both(g.scale * kLog2e);
        int stage = 0;
        uint32_t stph = 0, ph = 0, aph = 0;
        for (int turn = 0; ok; ++turn) {
            const int64_t w = work_at(turn);
            if ((int64_t)turn * gridDim.x >= total) break;
            if (w >= total) continue;
            const Item it = g.items[w / g.kv];
            const int h = (int)(w % g.kv);
            const QuerySpan q = query_span(it, g.kt);
            const int token = it.first + row;
            const bool live = token < it.end;
            const HeadsOut& o = half ? g.dk : g.dv;
            uint16_t* const out = o.p + (int64_t)token * o.token + h * o.head;
            if (it.begin < 0) {
                if (live) {
                    float zero[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) zero[i] = 0.f;
                    for (int x = 0; x < 2 * HALVES; ++x) write_columns<F16>(out, 32 * x, g.dim, o.wide, zero);
                }
                continue;
            }
            const float sigma = gradient_scale<F16>(g, h);
            const Pair s2 = both(F16 ? sigma * exp2f(-kLift) : 1.f);
            for (int i = 0; i < q.tiles; ++i) {
                const int first = q.first + i * g.kt;  // token of the tile's first row
                const bool masked = first < it.first + kRows - 1;
                const int from = (token - first) * g.group - 64 * half;  // the first column of this half that sees this key
                const float* const st = stats + stage * 2 * kRows + 64 * half;
                if (!(ok = warp_wait(st_full + 8 * stage, stph))) break;
                if (!(ok = warp_wait(s_full, ph))) break;
                mma_fence_after();
                uint32_t s[2][32], dp[2][32], e[32];
                tmem_fetch(tmem + 64 * half + lanes, s[0]), tmem_fetch(tmem + 64 * half + 32 + lanes, s[1]);
                tmem_wait(s[0]), tmem_wait(s[1]);
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 l = *reinterpret_cast<const float4*>(st + 32 * x + j);
                        const float2 a = split(fma2(pair(__uint_as_float(s[x][j]), __uint_as_float(s[x][j + 1])), c2, pair(l.x, l.y)));
                        const float2 b = split(fma2(pair(__uint_as_float(s[x][j + 2]), __uint_as_float(s[x][j + 3])), c2, pair(l.z, l.w)));
                        float p[4] = {exp2_of(a.x), exp2_of(a.y), exp2_of(b.x), exp2_of(b.y)};
                        if (masked) {
#pragma unroll
                            for (int y = 0; y < 4; ++y) p[y] = 32 * x + j + y < from ? 0.f : p[y];
                        }
#pragma unroll
                        for (int y = 0; y < 4; ++y) s[x][j + y] = __float_as_uint(p[y]);
                        e[16 * x + j / 2] = pack16<F16>(p[0], p[1]), e[16 * x + j / 2 + 1] = pack16<F16>(p[2], p[3]);
                    }
                tmem_store(tmem + 64 * half + lanes, e);
                tmem_store_wait();
                mma_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_full);
                if (!(ok = warp_wait(dp_full, ph))) break;
                mma_fence_after();
                tmem_fetch(t_dp + 64 * half + lanes, dp[0]), tmem_fetch(t_dp + 64 * half + 32 + lanes, dp[1]);
                tmem_wait(dp[0]), tmem_wait(dp[1]);
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 d = *reinterpret_cast<const float4*>(st + kRows + 32 * x + j);
                        const float2 a = split(pair(__uint_as_float(s[x][j]), __uint_as_float(s[x][j + 1])) *
                                               fma2(pair(__uint_as_float(dp[x][j]), __uint_as_float(dp[x][j + 1])), s2, pair(d.x, d.y)));
                        const float2 b = split(pair(__uint_as_float(s[x][j + 2]), __uint_as_float(s[x][j + 3])) *
                                               fma2(pair(__uint_as_float(dp[x][j + 2]), __uint_as_float(dp[x][j + 3])), s2, pair(d.z, d.w)));
                        float v[4] = {a.x, a.y, b.x, b.y};
                        if (masked) {
#pragma unroll
                            for (int y = 0; y < 4; ++y) v[y] = 32 * x + j + y < from ? 0.f : v[y];
                        }
                        e[16 * x + j / 2] = pack16<F16>(v[0], v[1]), e[16 * x + j / 2 + 1] = pack16<F16>(v[2], v[3]);
                    }
                tmem_store(t_dp + 64 * half + lanes, e);
                tmem_store_wait();
                mma_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(ds_full), bar_arrive(st_empty + 8 * stage);
                ph ^= 1;
                if (++stage == B::kStats) stage = 0, stph ^= 1;
            }
            if (!ok) break;
            if (!(ok = warp_wait(acc_full, aph))) break;
            aph ^= 1;
            mma_fence_after();
            const float f = half ? g.scale / sigma : F16 ? exp2f(-kLift) : 1.f;
            for (int x = 0; x < 2 * HALVES; ++x) {
                uint32_t a[32];
                tmem_fetch((half ? t_dk : t_dv) + 32 * x + lanes, a);
                tmem_wait(a);
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(a[i]) * f;
                if (live && 32 * x < g.dim) write_columns<F16>(out, 32 * x, g.dim, o.wide, v);
            }
            mma_fence_before();
        }
    }
    if (!ok) let_copies_end();
    __syncwarp();
    mma_fence_before();
    __syncthreads();
    mma_fence_after();
    if (warp == 9) tmem_free<1>(tmem, 512);
}

// ---- host side ----

struct BackPlan {
    int group, kt;
    int64_t most[2];
    size_t at_start, at_prefix[2], at_items[2], at_largest, at_delta, bytes;
};
BackPlan back_plan(int tokens, int sequences, int heads, int kv) {
    BackPlan p;
    p.group = heads / kv, p.kt = kRows / p.group;
    p.most[0] = items_at_most(tokens, sequences, p.kt), p.most[1] = items_at_most(tokens, sequences, kKeys);
    size_t at = 256;
    auto take = [&at](size_t n) { const size_t was = at; at += rounded(n); return was; };
    const size_t bounds = ((size_t)sequences + 1) * 4;
    p.at_start = take(2 * bounds);
    for (int i = 0; i < 2; ++i) p.at_prefix[i] = take(bounds), p.at_items[i] = take((size_t)p.most[i] * sizeof(Item));
    p.at_largest = take((size_t)2 * kv * 4);
    p.at_delta = take((size_t)tokens * heads * 4);
    p.bytes = at;
    return p;
}

template <class K>
cudaError_t launch_pass(K kernel, int smem, std::atomic<uint64_t>& ready, int64_t work, cudaStream_t stream, const CUtensorMap (&maps)[4],
                        const BackArgs& a) {
    cudaError_t err = allow_smem(kernel, smem, ready);
    if (err != cudaSuccess) return err;
    cudaLaunchConfig_t cfg = {};
    const int64_t slots = device_sms();
    cfg.gridDim = dim3((unsigned)(work < slots ? work : slots));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, maps[0], maps[1], maps[2], maps[3], a);
}

template <int HALVES, bool F16>
cudaError_t launch_back(const ones_heads& dout, const ones_heads& q, const ones_heads& k, const ones_heads& v, const DeltaArgs& d, BackArgs a,
                        const PlanArgs& plan, const BackPlan& p, cudaStream_t stream) {
    CUtensorMap maps[4];
    cudaError_t err = make_heads_map(&maps[0], q, a.dim, a.tokens, a.group, a.kt, F16);
    if (err == cudaSuccess) err = make_heads_map(&maps[1], dout, a.dim, a.tokens, a.group, a.kt, F16);
    if (err == cudaSuccess) err = make_heads_map(&maps[2], k, a.dim, a.tokens, 1, kKeys, F16);
    if (err == cudaSuccess) err = make_heads_map(&maps[3], v, a.dim, a.tokens, 1, kKeys, F16);
    if (err == cudaSuccess) err = launch_plan(plan, 2, stream);
    if (err != cudaSuccess) return err;
    const int64_t rows = (int64_t)a.tokens * (a.heads + (F16 ? a.kv : 0)), blocks = (rows + 15) / 16, most = 8 * (int64_t)device_sms();
    err = launch_after(k_delta<F16>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), stream, d);
    if (err != cudaSuccess) return err;
    static std::atomic<uint64_t> ready[2];
    a.items = plan.items[1], a.head = plan.head + 1;
    err = launch_pass(k_attention_keys<HALVES, F16>, Back<HALVES>::kSmemKeys, ready[0], p.most[1] * a.kv, stream, maps, a);
    if (err != cudaSuccess) return err;
    a.items = plan.items[0], a.head = plan.head;
    return launch_pass(k_attention_queries<HALVES, F16>, Back<HALVES>::kSmemQueries, ready[1], p.most[0] * a.kv, stream, maps, a);
}

}  // namespace

const WaitControl attention_back_waits = {take_expired, limit_waits, wait_for_nothing};

}  // namespace ones

extern "C" {

size_t ones_attention_backward_workspace_bytes(int32_t tokens, int32_t sequences, int32_t heads, int32_t kv, int32_t dim) {
    if (ones::bad_counts(tokens, sequences, heads, kv) || dim < 1 || dim > ONES_ATTENTION_MAX_DIM) return 0;
    return ones::back_plan(tokens, sequences, heads, kv).bytes;
}

int ones_attention_backward(const ones_heads* dout, const ones_heads* q, const ones_heads* k, const ones_heads* v,
                            const ones_heads* out, const float* d_lse, const int64_t* d_offsets, int32_t tokens,
                            int32_t sequences, int32_t dim, float scale, int32_t type, const ones_heads* dq,
                            const ones_heads* dk, const ones_heads* dv, void* d_workspace, size_t workspace_bytes,
                            void* cuda_stream) {
    using namespace ones;
    const HeadsOf all[] = {{q, false, false}, {dout, false, false}, {k, true, false}, {v, true, false}, {out, false, true}, {dq, false, true},
                           {dk, true, true}, {dv, true, true}};
    const int bad = refuse_attention(all, 8, d_offsets, tokens, sequences, dim, scale, type);
    if (bad || !tokens) return bad;
    if (!d_lse || !d_workspace) return ONES_ERR_NULL;
    if (!aligned(d_lse, 4) || !aligned(d_workspace, 256)) return ONES_ERR_ALIGN;
    const BackPlan p = back_plan(tokens, sequences, q->heads, k->heads);
    if (workspace_bytes < p.bytes) return ONES_ERR_WORKSPACE;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    uint8_t* const ws = static_cast<uint8_t*>(d_workspace);
    PlanArgs plan = {};
    plan.offsets = d_offsets, plan.tokens = tokens, plan.sequences = sequences;
    plan.step[0] = p.kt, plan.tile[0] = kKeys, plan.step[1] = kKeys, plan.tile[1] = p.kt;
    plan.start = reinterpret_cast<int*>(ws + p.at_start), plan.head = reinterpret_cast<PlanHead*>(ws);
    for (int i = 0; i < 2; ++i)
        plan.prefix[i] = reinterpret_cast<int*>(ws + p.at_prefix[i]), plan.items[i] = reinterpret_cast<Item*>(ws + p.at_items[i]);
    unsigned* const largest = reinterpret_cast<unsigned*>(ws + p.at_largest);
    plan.zero = largest, plan.zeros = 2 * k->heads;
    float* const delta = reinterpret_cast<float*>(ws + p.at_delta);
    const HeadsOut o = heads_out(*out, tokens);
    const DeltaArgs d = {static_cast<const uint16_t*>(dout->d_data), o.p, static_cast<const uint16_t*>(v->d_data), dout->token, dout->head, o.token,
                         o.head, v->token, v->head, plan.head, delta, largest, tokens, q->heads, k->heads, dim, o.wide && dim % 8 == 0};
    const BackArgs a = {nullptr, nullptr, d_lse, delta, largest, heads_out(*dq, tokens), heads_out(*dk, tokens), heads_out(*dv, tokens), tokens,
                        q->heads, k->heads, p.group, p.kt, dim, scale};
    const bool f16 = type == ONES_F16;
    cudaError_t err;
    if (dim > 64)
        err = f16 ? launch_back<2, true>(*dout, *q, *k, *v, d, a, plan, p, stream) : launch_back<2, false>(*dout, *q, *k, *v, d, a, plan, p, stream);
    else
        err = f16 ? launch_back<1, true>(*dout, *q, *k, *v, d, a, plan, p, stream) : launch_back<1, false>(*dout, *q, *k, *v, d, a, plan, p, stream);
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // extern "C"
