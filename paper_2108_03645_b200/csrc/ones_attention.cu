// Causal attention over packed sequences: the plan of the work and the forward pass.
//
// Bound by the tensor core and by the exponentials at once: a tile of 128 queries x 128 keys of 128 columns takes 1024 cycles of
// products and 1024 of exponentials (16 a cycle). A block has two tiles of queries that run against each other: while the
// tensor core multiplies for one, its softmax warps work on the other. Scores and outputs stay in tensor memory (4 x 128
// columns), the probabilities take the place of their scores there as 16 bits and are the left operand of the product with
// the values. A thread owns a row: maxima and sums need no exchange. The maximum that a row subtracts follows the true one
// only when that has grown by more than 2^8 (in the exponentials): the output is then rescaled in tensor memory, else not.
#include "ones_attention.cuh"

#include <math.h>

namespace ones {

namespace {

// ---- plan ----

constexpr int kPlanThreads = 1024;
constexpr int kBins = 1024;

__device__ __forceinline__ int block_scan(int v, int* sums, bool is_max) {  // inclusive; sums[32]
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int m = 1; m < 32; m <<= 1) {
        const int o = __shfl_up_sync(0xFFFFFFFFu, v, m);
        if (lane >= m) v = is_max ? max(v, o) : v + o;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = v;
    __syncthreads();
    if (warp == 0) {
        int s = sums[lane];
        for (int m = 1; m < 32; m <<= 1) {
            const int o = __shfl_up_sync(0xFFFFFFFFu, s, m);
            if (lane >= m) s = is_max ? max(s, o) : s + o;
        }
        sums[lane] = s;
    }
    __syncthreads();
    if (warp) v = is_max ? max(v, sums[warp - 1]) : v + sums[warp - 1];
    return v;
}

// One block makes one list: the sequences' bounds, the items before each, then the items sorted by their cost (counted in
// bins; the order within a bin does not matter to any result).
__global__ void __launch_bounds__(kPlanThreads) k_plan(const PlanArgs a) {
    __shared__ int sums[32];
    __shared__ int bins[kBins];
    __shared__ int s_total;
    const int list = blockIdx.x, step = a.step[list];
    int* prefix = a.prefix[list];
    int* start = a.start + (int64_t)list * (a.sequences + 1);
    wait_for_predecessor();
    let_successor_start();
    if (list == 0)
        for (int i = threadIdx.x; i < a.zeros; i += kPlanThreads) a.zero[i] = 0;
    int carry_max = 0;
    for (int base = 0; base <= a.sequences; base += kPlanThreads) {
        const int i = base + threadIdx.x;
        int64_t v = 0;
        if (i <= a.sequences) v = a.offsets ? a.offsets[i] : (int64_t)(a.tokens / max(a.sequences, 1)) * i;
        v = v < 0 ? 0 : v > a.tokens ? a.tokens : v;
        const int m = max(block_scan((int)v, sums, true), carry_max);
        if (i <= a.sequences) start[i] = m;
        __syncthreads();
        if (threadIdx.x == kPlanThreads - 1) sums[0] = m;
        __syncthreads();
        carry_max = sums[0];
        __syncthreads();
    }
    __syncthreads();
    int carry = 0;
    for (int base = 0; base < a.sequences; base += kPlanThreads) {
        const int i = base + threadIdx.x;
        const int n = i < a.sequences ? (start[i + 1] - start[i] + step - 1) / step : 0;
        const int s = block_scan(n, sums, false) + carry;
        if (i < a.sequences) prefix[i + 1] = s;
        __syncthreads();
        if (threadIdx.x == kPlanThreads - 1) sums[0] = s;
        __syncthreads();
        carry = sums[0];
        __syncthreads();
    }
    if (threadIdx.x == 0) prefix[0] = 0, s_total = carry;
    for (int i = threadIdx.x; i < kBins; i += kPlanThreads) bins[i] = 0;
    __syncthreads();
    const int total = s_total, front = start[0], back = start[a.sequences];
    // items of tokens before the first and behind the last sequence: at the end of the list
    const int n_front = (front + step - 1) / step, n_back = (a.tokens - back + step - 1) / step;
    int shift = 0;
    while ((a.tokens / a.tile[list] + 1) >> shift >= kBins) ++shift;
    for (int pass = 0; pass < 2; ++pass) {
        for (int i = threadIdx.x; i < total; i += kPlanThreads) {
            int lo = 0, hi = a.sequences;  // the last sequence with prefix <= i
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (prefix[mid] <= i)
                    lo = mid;
                else
                    hi = mid;
            }
            Item it;
            it.begin = start[lo], it.end = start[lo + 1];
            it.first = it.begin + (i - prefix[lo]) * step;
            // queries: the keys up to their last one; keys: the queries from their first one on
            it.cost = list == 0 ? (min(it.first + step, it.end) - it.begin + a.tile[0] - 1) / a.tile[0]
                                : (it.end - it.first + a.tile[1] - 1) / a.tile[1];
            const int bin = kBins - 1 - min(it.cost >> shift, kBins - 1);
            const int at = atomicAdd(&bins[bin], 1);
            if (pass) a.items[list][at] = it;
        }
        __syncthreads();
        if (!pass) {
            const int own = bins[threadIdx.x], s = block_scan(own, sums, false);
            bins[threadIdx.x] = s - own;
            __syncthreads();
        }
    }
    for (int i = threadIdx.x; i < n_front + n_back; i += kPlanThreads) {
        Item it;
        it.begin = -1, it.cost = 0;
        it.first = i < n_front ? i * step : back + (i - n_front) * step;
        it.end = min(it.first + step, i < n_front ? front : a.tokens);
        a.items[list][total + i] = it;
    }
    if (threadIdx.x == 0) {
        PlanHead h = {};
        h.count = total + n_front + n_back;
        h.covered[0] = front, h.covered[1] = back;
        a.head[list] = h;
    }
}

// ---- forward ----

constexpr int kThreads = 384;  // two groups of softmax warps, then load, multiply and two idle warps
constexpr float kGrow = 8.f;   // a row's maximum may grow by so much (log2 of the exponentials) before it is followed

struct ForwardArgs {
    const Item* items;
    const PlanHead* head;
    HeadsOut out;
    float* lse;
    int tokens, heads, kv, group, kt, dim;
    float scale;
};

template <int HALVES>
struct Forward {
    static constexpr int kTile = HALVES * kHalfTile;
    static constexpr int kSlots = HALVES == 2 ? 5 : 8;
    static constexpr int kSmem = (2 + kSlots) * kTile + 1024;
};

struct ForwardShared {
    uint64_t q_full[2], q_free[2], full[8], empty[8], s_full[2], p_full[2], o_full[2];
    uint32_t tmem;
};

// A tile of queries of an item: its first token, how many tiles of keys it meets, where its masked ones begin.
struct QueryTile {
    int first, tiles, clean;  // tiles of keys; those before `clean` need no mask
};
__device__ __forceinline__ QueryTile query_tile(const Item& it, int which, int kt) {
    QueryTile q;
    q.first = it.first + which * kt;
    const int last = min(q.first + kt, it.end) - 1 - it.begin;  // of its tokens, from the sequence's begin
    q.tiles = it.begin < 0 || q.first >= it.end ? 0 : last / kKeys + 1;
    q.clean = q.tiles ? (q.first - it.begin + 1) / kKeys : 0;
    return q;
}

template <int HALVES, bool F16>
__global__ void __launch_bounds__(kThreads, 1)
    k_attention(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                const ForwardArgs g) {
    using F = Forward<HALVES>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ ForwardShared sh;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t ring = base + 2 * F::kTile;
    const uint32_t q_full = smem_u32(sh.q_full), q_free = smem_u32(sh.q_free), full = smem_u32(sh.full), empty = smem_u32(sh.empty),
                   s_full = smem_u32(sh.s_full), p_full = smem_u32(sh.p_full), o_full = smem_u32(sh.o_full);
    if (threadIdx.x == 0) {
        tma_prefetch(&map_q), tma_prefetch(&map_k), tma_prefetch(&map_v);
        for (int i = 0; i < 2; ++i) {
            bar_init(q_full + 8 * i, 1), bar_init(q_free + 8 * i, 1), bar_init(s_full + 8 * i, 1), bar_init(p_full + 8 * i, 4);
            bar_init(o_full + 8 * i, 1);
        }
        for (int i = 0; i < F::kSlots; ++i) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
        bar_init_done();
    }
    if (warp == 9) tmem_alloc<1>(smem_u32(&sh.tmem), 512);
    mma_fence_before();
    __syncthreads();
    mma_fence_after();
    const uint32_t tmem = sh.tmem;
    wait_for_predecessor();
    let_successor_start();
    const int64_t total = (int64_t)g.head->count * g.kv;
    bool ok = true;

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 8) {
            // load: queries of both tiles, then keys and values in turn
            int slot = 0;
            uint32_t ph = 0, qph[2] = {0, 0};
            const uint32_t qbytes = HALVES * g.group * g.kt * 128;
            for (int turn = 0; ok; ++turn) {
                const int64_t w = work_at(turn);
                if ((int64_t)turn * gridDim.x >= total) break;
                if (w >= total) continue;
                const Item it = g.items[w / g.kv];
                const int h = (int)(w % g.kv);
                const QueryTile q0 = query_tile(it, 0, g.kt), q1 = query_tile(it, 1, g.kt);
                const int tiles = max(q0.tiles, q1.tiles);
                for (int j = 0; ok && j < tiles; ++j) {
                    for (int kind = 0; ok && kind < 2; ++kind) {
                        if (kind == 0 && j == 0) {
                            for (int i = 0; ok && i < 2; ++i) {
                                if (!(i ? q1.tiles : q0.tiles)) continue;
                                if (!(ok = warp_wait(q_free + 8 * i, qph[i] ^ 1))) break;
                                qph[i] ^= 1;
                                if (elect_one()) {
                                    bar_expect(q_full + 8 * i, qbytes);
                                    for (int x = 0; x < HALVES; ++x)
                                        tma_load<1>(base + i * F::kTile + x * kHalfTile, &map_q, 64 * x, h * g.group, (i ? q1 : q0).first, q_full + 8 * i);
                                }
                                __syncwarp();
                            }
                            if (!ok) break;
                        }
                        if (!(ok = warp_wait(empty + 8 * slot, ph ^ 1))) break;
                        if (elect_one()) {
                            bar_expect(full + 8 * slot, F::kTile);
                            for (int x = 0; x < HALVES; ++x)
                                tma_load<1>(ring + slot * F::kTile + x * kHalfTile, kind ? &map_v : &map_k, 64 * x, h, it.begin + j * kKeys, full + 8 * slot);
                        }
                        __syncwarp();
                        if (++slot == F::kSlots) slot = 0, ph ^= 1;
                    }
                }
            }
        } else if (warp == 9) {
            // multiply
            const uint32_t id_s = attend_desc(F16, false, kKeys), id_o = attend_desc(F16, true, 64 * HALVES);
            const int steps = (g.dim + 15) / 16;
            int slot = 0;
            uint32_t ph = 0, qph[2] = {0, 0}, pph[2] = {0, 0};
            for (int turn = 0; ok; ++turn) {
                const int64_t w = work_at(turn);
                if ((int64_t)turn * gridDim.x >= total) break;
                if (w >= total) continue;
                const Item it = g.items[w / g.kv];
                const QueryTile q[2] = {query_tile(it, 0, g.kt), query_tile(it, 1, g.kt)};
                const int tiles = max(q[0].tiles, q[1].tiles);
                if (!tiles) continue;
                // the first scores
                if (!(ok = warp_wait(full + 8 * slot, ph))) break;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (!q[i].tiles || !ok) continue;
                    if (!(ok = warp_wait(q_full + 8 * i, qph[i]))) break;
                    qph[i] ^= 1;
                    mma_fence_after();
                    if (elect_one()) {
                        product_rows(tmem + 128 * i, base + i * F::kTile, ring + slot * F::kTile, id_s, steps);
                        mma_commit<1>(s_full + 8 * i);
                        if (q[i].tiles == 1) mma_commit<1>(q_free + 8 * i);
                    }
                    __syncwarp();
                }
                if (!ok) break;
                if (elect_one()) mma_commit<1>(empty + 8 * slot);
                __syncwarp();
                if (++slot == F::kSlots) slot = 0, ph ^= 1;
                for (int j = 0; ok && j < tiles; ++j) {
                    const int v = slot;
                    if (!(ok = warp_wait(full + 8 * v, ph))) break;
                    if (++slot == F::kSlots) slot = 0, ph ^= 1;
                    const int rest = it.end - it.begin - j * kKeys;
                    if (rest < kKeys) clear_rows<HALVES>(smem + (2 + v) * F::kTile, rest, lane);
                    const bool more = j + 1 < tiles;
                    if (more && !(ok = warp_wait(full + 8 * slot, ph))) break;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (j >= q[i].tiles || !ok) continue;
                        if (!(ok = warp_wait(p_full + 8 * i, pph[i]))) break;
                        pph[i] ^= 1;
                        mma_fence_after();
                        if (elect_one()) {
                            product_tmem(tmem + 256 + 128 * i, tmem + 128 * i, tmem + 128 * i + 32, ring + v * F::kTile, id_o, j != 0);
                            mma_commit<1>(o_full + 8 * i);
                            if (j + 1 < q[i].tiles) {
                                product_rows(tmem + 128 * i, base + i * F::kTile, ring + slot * F::kTile, id_s, steps);
                                mma_commit<1>(s_full + 8 * i);
                                if (j + 2 == q[i].tiles) mma_commit<1>(q_free + 8 * i);
                            }
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (elect_one()) {
                        mma_commit<1>(empty + 8 * v);
                        if (more) mma_commit<1>(empty + 8 * slot);
                    }
                    __syncwarp();
                    if (more && ++slot == F::kSlots) slot = 0, ph ^= 1;
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        const int which = warp / 4, row = threadIdx.x % 128;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        const uint32_t ts = tmem + 128 * which + lanes, to = tmem + 256 + 128 * which + lanes;
        const float c = g.scale * kLog2e;
        uint32_t sph = 0, oph = 0;  // oph: parity of the next product with the values that is to end
        for (int turn = 0; ok; ++turn) {
            const int64_t w = work_at(turn);
            if ((int64_t)turn * gridDim.x >= total) break;
            if (w >= total) continue;
            const Item it = g.items[w / g.kv];
            const int h = (int)(w % g.kv);
            const QueryTile q = query_tile(it, which, g.kt);
            const int token = q.first + row / g.group, head = h * g.group + row % g.group;
            const bool live = row < g.group * g.kt && token < it.end;
            uint16_t* const out = g.out.p + (int64_t)token * g.out.token + head * g.out.head;
            if (it.begin < 0) {  // tokens of no sequence
                if (live) {
                    float zero[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) zero[i] = 0.f;
                    for (int x = 0; x < 2 * HALVES; ++x) write_columns<F16>(out, 32 * x, g.dim, g.out.wide, zero);
                    g.lse[(int64_t)token * g.heads + head] = 0.f;
                }
                continue;
            }
            float top = 0.f;
            Pair sum = both(0.f);
            for (int j = 0; j < q.tiles; ++j) {
                if (!(ok = warp_wait(s_full + 8 * which, sph))) break;
                sph ^= 1;
                mma_fence_after();
                uint32_t s[4][32];
#pragma unroll
                for (int x = 0; x < 4; ++x) tmem_fetch(ts + 32 * x, s[x]);
#pragma unroll
                for (int x = 0; x < 4; ++x) tmem_wait(s[x]);
                if (j >= q.clean) {
                    const int last = token - it.begin - j * kKeys;  // the last key of the tile that the row may see
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (32 * x + i > last) s[x][i] = 0xFF800000u;  // -infinity
                }
                float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < 32; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x) m[x] = fmaxf(m[x], __uint_as_float(s[x][i]));
                float tile_top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
                if (tile_top == -INFINITY) tile_top = j ? top : 0.f;
                if (j == 0) {
                    top = tile_top;
                } else if (__any_sync(0xFFFFFFFFu, (tile_top - top) * c > kGrow)) {
                    const float next = fmaxf(top, tile_top), f = exp2_of((top - next) * c);
                    top = next;
                    sum = sum * both(f);
                    if (!(ok = warp_wait(o_full + 8 * which, oph ^ 1))) break;  // the product of the tile before
                    mma_fence_after();
                    for (int x = 0; x < 2 * HALVES; ++x) {
                        uint32_t o[32];
                        tmem_fetch(to + 32 * x, o);
                        tmem_wait(o);
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                        tmem_store(to + 32 * x, o);
                    }
                    tmem_store_wait();
                }
                const Pair c2 = both(c), t2 = both(-top * c);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t p[32];
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            const float2 e = split(fma2(pair(__uint_as_float(s[2 * half + x][i]), __uint_as_float(s[2 * half + x][i + 1])), c2, t2));
                            const float a = exp2_of(e.x), b = exp2_of(e.y);
                            sum = sum + pair(a, b);
                            p[16 * x + i / 2] = pack16<F16>(a, b);
                        }
                    tmem_store(ts + 32 * half, p);
                }
                tmem_store_wait();
                mma_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_full + 8 * which);
                oph ^= 1;
            }
            if (!ok) break;
            if (!q.tiles) continue;
            if (!(ok = warp_wait(o_full + 8 * which, oph ^ 1))) break;
            mma_fence_after();
            const float l = total_of(sum);
            const float inv = 1.f / l;
            for (int x = 0; x < 2 * HALVES; ++x) {
                uint32_t o[32];
                tmem_fetch(to + 32 * x, o);
                tmem_wait(o);
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(o[i]) * inv;
                if (live && 32 * x < g.dim) write_columns<F16>(out, 32 * x, g.dim, g.out.wide, v);
            }
            if (live) g.lse[(int64_t)token * g.heads + head] = top * g.scale + logf(l);
        }
    }
    if (!ok) let_copies_end();
    __syncwarp();
    mma_fence_before();
    __syncthreads();
    mma_fence_after();
    if (warp == 9) tmem_free<1>(tmem, 512);
}

}  // namespace

const WaitControl attention_waits = {take_expired, limit_waits, wait_for_nothing};

cudaError_t launch_plan(const PlanArgs& a, int lists, cudaStream_t stream) {
    return launch_after(k_plan, dim3(lists), dim3(kPlanThreads), stream, a);
}

cudaError_t make_heads_map(CUtensorMap* out, const ones_heads& h, int dim, int tokens, int heads_box, int tokens_box, bool f16) {
    const uint64_t row = (uint64_t)(dim + 7) / 8 * 16;  // a stride that no second head or token uses
    const uint64_t dims[3] = {(uint64_t)dim, (uint64_t)h.heads, (uint64_t)tokens};
    const uint64_t strides[2] = {h.heads > 1 ? (uint64_t)h.head * 2 : row, tokens > 1 ? (uint64_t)h.token * 2 : row};
    const uint32_t box[3] = {64, (uint32_t)heads_box, (uint32_t)tokens_box};
    return encode_box(out, h.d_data, dims, strides, box, f16);
}

int refuse_attention(const HeadsOf* all, int n, const int64_t* offsets, int tokens, int sequences, int dim, float scale, int type) {
    if (tokens < 0 || tokens >= 1 << 30 || sequences < 0 || sequences > 1 << 22 || dim < 1 || dim > ONES_ATTENTION_MAX_DIM || !(scale > 0.f) ||
        !isfinite(scale) || (type != ONES_BF16 && type != ONES_F16))
        return ONES_ERR_BAD_PARAM;
    if (!offsets && tokens && (sequences < 1 || tokens % sequences)) return ONES_ERR_BAD_PARAM;
    for (int i = 0; i < n; ++i)
        if (!all[i].h) return ONES_ERR_NULL;
    const int heads = all[0].h->heads;
    int kv = 0;
    for (int i = 0; i < n; ++i)
        if (all[i].keys) kv = all[i].h->heads;
    if (heads < 1 || heads > ONES_MAX_HEADS || kv < 1 || heads % kv || heads / kv > kRows) return ONES_ERR_BAD_PARAM;
    for (int i = 0; i < n; ++i) {
        const ones_heads& h = *all[i].h;
        if (h.heads != (all[i].keys ? kv : heads) || (h.heads > 1 && h.head < dim) || (tokens > 1 && h.token < 1)) return ONES_ERR_BAD_PARAM;
    }
    if (!tokens) return ONES_OK;
    for (int i = 0; i < n; ++i)
        if (!all[i].h->d_data) return ONES_ERR_NULL;
    if (!aligned(offsets, 8)) return ONES_ERR_ALIGN;
    for (int i = 0; i < n; ++i) {
        const ones_heads& h = *all[i].h;
        if (all[i].out ? !aligned(h.d_data, 2)
                       : !aligned(h.d_data, 16) || (h.heads > 1 && h.head % 8) || (tokens > 1 && h.token % 8))
            return ONES_ERR_ALIGN;
    }
    return ONES_OK;
}

namespace {

// Tokens of a tile of queries, and what the workspace holds.
struct ForwardPlan {
    int group, kt;
    int64_t most;
    size_t at_start, at_prefix, at_items, bytes;
};
ForwardPlan forward_plan(int tokens, int sequences, int heads, int kv) {
    ForwardPlan p;
    p.group = heads / kv, p.kt = kRows / p.group;
    p.most = items_at_most(tokens, sequences, 2 * p.kt);
    const size_t bounds = rounded(((size_t)sequences + 1) * 4);
    p.at_start = 256, p.at_prefix = p.at_start + bounds, p.at_items = p.at_prefix + bounds;
    p.bytes = p.at_items + rounded((size_t)p.most * sizeof(Item));
    return p;
}

template <int HALVES, bool F16>
cudaError_t launch_forward(const ones_heads& q, const ones_heads& k, const ones_heads& v, const ForwardArgs& a, int64_t most, cudaStream_t stream) {
    CUtensorMap mq, mk, mv;
    cudaError_t err = make_heads_map(&mq, q, a.dim, a.tokens, a.group, a.kt, F16);
    if (err == cudaSuccess) err = make_heads_map(&mk, k, a.dim, a.tokens, 1, kKeys, F16);
    if (err == cudaSuccess) err = make_heads_map(&mv, v, a.dim, a.tokens, 1, kKeys, F16);
    if (err != cudaSuccess) return err;
    auto kernel = k_attention<HALVES, F16>;
    static std::atomic<uint64_t> ready{0};
    err = allow_smem(kernel, Forward<HALVES>::kSmem, ready);
    if (err != cudaSuccess) return err;
    cudaLaunchConfig_t cfg = {};
    const int64_t work = most * a.kv, slots = device_sms();
    cfg.gridDim = dim3((unsigned)(work < slots ? work : slots));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Forward<HALVES>::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, mq, mk, mv, a);
}

}  // namespace

}  // namespace ones

extern "C" {

size_t ones_attention_workspace_bytes(int32_t tokens, int32_t sequences, int32_t heads, int32_t kv) {
    return ones::bad_counts(tokens, sequences, heads, kv) ? 0 : ones::forward_plan(tokens, sequences, heads, kv).bytes;
}

int ones_attention(const ones_heads* q, const ones_heads* k, const ones_heads* v, const int64_t* d_offsets, int32_t tokens,
                   int32_t sequences, int32_t dim, float scale, int32_t type, const ones_heads* out, float* d_lse,
                   void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
    using namespace ones;
    const HeadsOf all[] = {{q, false, false}, {k, true, false}, {v, true, false}, {out, false, true}};
    const int bad = refuse_attention(all, 4, d_offsets, tokens, sequences, dim, scale, type);
    if (bad || !tokens) return bad;
    if (!d_lse || !d_workspace) return ONES_ERR_NULL;
    if (!aligned(d_lse, 4) || !aligned(d_workspace, 256)) return ONES_ERR_ALIGN;
    const ForwardPlan p = forward_plan(tokens, sequences, q->heads, k->heads);
    if (workspace_bytes < p.bytes) return ONES_ERR_WORKSPACE;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    uint8_t* const ws = static_cast<uint8_t*>(d_workspace);
    PlanArgs plan = {};
    plan.offsets = d_offsets, plan.tokens = tokens, plan.sequences = sequences;
    plan.step[0] = 2 * p.kt, plan.tile[0] = kKeys;
    plan.start = reinterpret_cast<int*>(ws + p.at_start), plan.prefix[0] = reinterpret_cast<int*>(ws + p.at_prefix);
    plan.items[0] = reinterpret_cast<Item*>(ws + p.at_items), plan.head = reinterpret_cast<PlanHead*>(ws);
    cudaError_t err = launch_plan(plan, 1, stream);
    if (err != cudaSuccess) return ONES_ERR_CUDA;
    const ForwardArgs a = {plan.items[0], plan.head, heads_out(*out, tokens), d_lse, tokens, q->heads, k->heads, p.group, p.kt, dim, scale};
    const bool f16 = type == ONES_F16;
    if (dim > 64)
        err = f16 ? launch_forward<2, true>(*q, *k, *v, a, p.most, stream) : launch_forward<2, false>(*q, *k, *v, a, p.most, stream);
    else
        err = f16 ? launch_forward<1, true>(*q, *k, *v, a, p.most, stream) : launch_forward<1, false>(*q, *k, *v, a, p.most, stream);
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // extern "C"
