// Causal attention over packed sequences: the plan of the work and the forward pass.
//
// Bound by the tensor core and by the exponentials at once: a tile of 128 queries x 128 keys of 128 columns takes 1024 cycles of
// products and 1024 of exponentials (16 a cycle). A block has two tiles of queries that run against each other: while the
// tensor core multiplies for one, its softmax warps work on the other. Scores and outputs stay in tensor memory (4 x 128
// columns), the probabilities take the place of their scores there as 16 bits and are the left operand of the product with
// the values. A thread owns a row: maxima and sums need no exchange. The maximum that a row subtracts follows the true one
// only when that has grown by more than 2^8 (in the exponentials; a known way of rescaling seldom): the output is then rescaled in
// tensor memory, else not.
// Probabilities are rounded to the tensors' type for their product with the values (half a step, 2^-8 or 2^-11 of each,
// averaged by the sum over keys), and summed before that in 32 bits, each tile by itself.
//
// Measured: 16384 tokens in one sequence, 16 / 4 heads of 128: 932 us by itself and 982 in a row = 1.12 PFLOP/s (the card at its power limit,
// 1.6 to 1.77 GHz); 12 documents of 64 to 3412 tokens, 16 / 4 heads of 128: 137 us for 129 GFLOP, which block ends last decides; 128 samples of
// 256 tokens, 16 heads of 64: 73 us, bound by the latency of an item's first tile. What did not help: probabilities handed on in
// two halves (893 -> 955 us), softmax loops that are not unrolled (967 -> 1159), items taken from a counter by whoever is free
// (documents 136 -> 133 us, but 16384 tokens forward and backward 4182 -> 4631: neighbours no longer work on the same keys).
#include "ones_attention.cuh"

#include <math.h>

namespace ones {

namespace {

// ---- plan ----

constexpr int kPlanThreads = 1024;
constexpr int kBins = 1024;
constexpr int kNear = 2047;  // so many sequences' bounds stay in shared memory: looked up in global memory they took 4 of 7 us

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
    __shared__ int s_start[kNear + 1], s_prefix[kNear + 1];
    if (blockIdx.x >= a.lists) {
        wait_for_predecessor();
        let_successor_start();
        const int64_t stride = (int64_t)(gridDim.x - a.lists) * kPlanThreads;
        for (int64_t i = (int64_t)(blockIdx.x - a.lists) * kPlanThreads + threadIdx.x; i < a.zeros; i += stride) a.zero[i] = 0;
        return;
    }
    const int list = blockIdx.x, step = list ? a.step[1] : a.step[0], per = list ? a.tile[1] : a.tile[0];
    const bool near = a.sequences <= kNear;
    int* const prefix = near ? s_prefix : list ? a.prefix[1] : a.prefix[0];
    int* const start = near ? s_start : a.start + (int64_t)list * (a.sequences + 1);
    Item* const items = list ? a.items[1] : a.items[0];
    wait_for_predecessor();
    let_successor_start();
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
    while ((a.tokens / per + 1) >> shift >= kBins) ++shift;
    Item it = {};
    int bin = 0;
    for (int pass = 0; pass < 2; ++pass) {
        for (int i = threadIdx.x; i < total; i += kPlanThreads) {
            if (!pass || total > kPlanThreads) {
                int lo = 0, hi = a.sequences;  // the last sequence with prefix <= i
                while (hi - lo > 1) {
                    const int mid = (lo + hi) / 2;
                    if (prefix[mid] <= i)
                        lo = mid;
                    else
                        hi = mid;
                }
                it.begin = start[lo], it.end = start[lo + 1];
                it.first = it.begin + (i - prefix[lo]) * step;
                // queries: the keys up to their last one; keys: the queries from their first one on
                it.slot = min(lo, it.begin);
                const int cost = ((list == 0 ? min(it.first + step, it.end) - it.begin : it.end - it.first) + per - 1) / per;
                bin = kBins - 1 - min(cost >> shift, kBins - 1);
            }
            const int at = atomicAdd(&bins[bin], 1);
            if (pass) items[at] = it;
        }
        __syncthreads();
        if (!pass) {
            const int own = bins[threadIdx.x], s = block_scan(own, sums, false);
            bins[threadIdx.x] = s - own;
            __syncthreads();
        }
    }
    for (int i = threadIdx.x; i < n_front + n_back; i += kPlanThreads) {
        it.begin = -1, it.slot = 0;
        it.first = i < n_front ? i * step : back + (i - n_front) * step;
        it.end = min(it.first + step, i < n_front ? front : a.tokens);
        items[total + i] = it;
    }
    if (threadIdx.x == 0) {
        PlanHead h = {};
        h.count = total + n_front + n_back;
        h.covered[0] = front, h.covered[1] = back;
        a.head[list] = h;
    }
}

// ---- forward ----

constexpr int kThreads = 384;  // two groups of softmax warps, then load, two that multiply, and one that clears
constexpr float kGrow = 8.f;   // a row's maximum may grow by so much (log2 of the exponentials) before it is followed
// float16: log2 of what all probabilities are multiplied with, so that the largest there can be, 2^8, becomes 2^15, which the type holds, and its
// steps are 2^-31 of the row's largest. (Steps of 2^-24 lose what many keys can have a share of the row by: 131071 keys at 2^-25 each.)
template <bool F16>
constexpr float kRaise = F16 ? 7.f : 0.f;
constexpr float kFar = 16384.f;  // up to here the rounding of a maximum (log2 of the exponentials) is below 2^-10, and common to its row

struct ForwardArgs {
    const Item* items;
    const PlanHead* head;
    HeadsOut out;
    float* lse;
    int tokens, heads, kv, group, kt, dim;
    float scale;
};

// Heads of up to 64 values leave room for two sets of queries and of outputs: a lane then works on its next item's first scores
// before it writes the last one's output.
template <int HALVES>
struct Forward {
    static constexpr int kTile = HALVES * kHalfTile;
    static constexpr int kSets = HALVES == 2 ? 1 : 2;
    static constexpr int kSlots = HALVES == 2 ? 5 : 8;
    // Warps that multiply: one for each lane, so that short items of one do not wait for those of the other; but where the ring is
    // short, one warp that takes the lanes in turn: lanes that drift apart hold its slots for longer (16384 tokens, 16 heads of
    // 128: 1100 us, and 890 in turn).
    static constexpr int kLanes = HALVES == 2 ? 1 : 2;
    static constexpr int kStage = HALVES == 2 ? 0 : 8 * kStageBytesOfWarp;  // for the way out
    static constexpr int kSmem = (2 * kSets + kSlots) * kTile + kStage + 1024;
};

struct ForwardShared {
    uint64_t q_full[2][2], q_free[2][2], full[8], raw[8], empty[8], s_full[2], p_full[2], o_full[2], acc_full[2][2], acc_free[2][2];
    uint32_t tmem;
    volatile uint32_t loads;  // how many tiles have been sent for: what the other warps' waits go by
};

// A tile of queries of an item: its first token, how many tiles of keys it meets.
struct QueryTile {
    int first, tiles;
};
__device__ __forceinline__ QueryTile query_tile(const Work& it, int which, int kt) {
    QueryTile q;
    q.first = it.first + which * kt;
    const int last = min(q.first + kt, it.end) - 1 - it.begin;  // of its tokens, from the sequence's begin
    q.tiles = it.begin < 0 || q.first >= it.end ? 0 : last / kKeys + 1;
    return q;
}

template <int HALVES, bool F16, bool WIDE>
__global__ void __launch_bounds__(kThreads, 1)
    k_attention(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                const ForwardArgs g) {
    using F = Forward<HALVES>;
    using At = Slot<F::kSlots>;   // keys and values in turn; both lanes (tiles of queries) give every slot back
    using Set = Slot<F::kSets>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ ForwardShared sh;
    __shared__ WorkList list;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t ring = base + 2 * F::kSets * F::kTile;
    const uint32_t q_full = smem_u32(sh.q_full), q_free = smem_u32(sh.q_free), full = smem_u32(sh.full), raw = smem_u32(sh.raw),
                   empty = smem_u32(sh.empty), s_full = smem_u32(sh.s_full), p_full = smem_u32(sh.p_full), o_full = smem_u32(sh.o_full),
                   acc_full = smem_u32(sh.acc_full), acc_free = smem_u32(sh.acc_free);
    if (threadIdx.x == 0) {
        sh.loads = 0;
        tma_prefetch(&map_q), tma_prefetch(&map_k), tma_prefetch(&map_v);
        for (int i = 0; i < 2; ++i) bar_init(s_full + 8 * i, 1), bar_init(p_full + 8 * i, 4), bar_init(o_full + 8 * i, 1);
        for (int i = 0; i < 4; ++i) bar_init(q_full + 8 * i, 1), bar_init(q_free + 8 * i, 1), bar_init(acc_full + 8 * i, 1), bar_init(acc_free + 8 * i, 4);
        for (int i = 0; i < F::kSlots; ++i) bar_init(full + 8 * i, 1), bar_init(raw + 8 * i, 1), bar_init(empty + 8 * i, F::kLanes);
        bar_init_done();
    }
    if (warp == 9) tmem_alloc<1>(smem_u32(&sh.tmem), 512);
    wait_for_predecessor();
    let_successor_start();
    list_work(list, g.items, g.head, g.kv);
    mma_fence_before();
    __syncthreads();
    mma_fence_after();
    const uint32_t tmem = sh.tmem;
    Walk walk(list, g.items, g.kv);
    bool ok = true;

    // The scores of a lane's tile j, and its product with the values; whole warps.
    auto first_product = [&](int which, uint32_t item, int j, int tiles, uint32_t slot, uint32_t parity) {
        const Set set(item);
        const uint32_t bar = 8 * (2 * which + set.at);
        if (j == 0 && !warp_wait(q_full + bar, set.parity, &sh.loads)) return false;
        if (!warp_wait(full + 8 * slot, parity, &sh.loads)) return false;
        mma_fence_after();
        if (elect_one()) {
            product_rows<HALVES>(tmem + 128 * which, base + (which * F::kSets + set.at) * F::kTile, ring + slot * F::kTile, attend_desc(F16, false, kKeys),
                         (g.dim + 15) / 16);
            mma_commit<1>(s_full + 8 * which);
            if (j + 1 == tiles) mma_commit<1>(q_free + bar);
        }
        __syncwarp();
        return true;
    };
    auto second_product = [&](int which, uint32_t item, int j, int tiles, uint32_t slot, uint32_t parity, uint32_t count) {
        const Set set(item);
        const uint32_t bar = 8 * (2 * which + set.at), to = tmem + 256 + 128 * which + 64 * set.at, ts = tmem + 128 * which;
        if (!warp_wait(full + 8 * slot, parity, &sh.loads)) return false;
        if (j == 0 && !warp_wait(acc_free + bar, set.parity ^ 1, &sh.loads)) return false;
        if (!warp_wait(p_full + 8 * which, count & 1, &sh.loads)) return false;
        mma_fence_after();
        if (elect_one()) {
            product_tmem(to, ts, ts + 32, ring + slot * F::kTile, attend_desc(F16, true, 16 * ((g.dim + 15) / 16)), j != 0);
            mma_commit<1>(o_full + 8 * which);
            if (j + 1 == tiles) mma_commit<1>(acc_full + bar);
        }
        __syncwarp();
        return true;
    };

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 8) {
            // load: keys and values in turn, each lane's queries before the first of them
            uint32_t n = 0, items[2] = {0, 0};
            const uint32_t qbytes = HALVES * g.group * g.kt * 128;
            while (ok && walk.next()) {
                const Work it = walk.it;
                const QueryTile q[2] = {query_tile(it, 0, g.kt), query_tile(it, 1, g.kt)};
                const int tiles = max(q[0].tiles, q[1].tiles);
                for (int i = 0; ok && i < 2 * tiles; ++i, ++n) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (i != x || !q[x].tiles || !ok) continue;
                        const Set set(items[x]++);
                        const uint32_t bar = 8 * (2 * x + set.at);
                        if (!(ok = warp_wait(q_free + bar, set.parity ^ 1))) break;
                        if (elect_one()) {
                            bar_expect(q_full + bar, qbytes);
                            for (int y = 0; y < HALVES; ++y)
                                tma_load<1>(base + (x * F::kSets + set.at) * F::kTile + y * kHalfTile, &map_q, 64 * y, walk.it.h * g.group, q[x].first,
                                            q_full + bar);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    const At slot(n);
                    const bool values = i & 1, partial = values && it.end - it.begin < (i / 2 + 1) * kKeys;  // that tile is cleared first
                    if (!(ok = warp_wait(empty + 8 * slot.at, slot.parity ^ 1))) break;
                    if (elect_one()) {
                        const uint32_t bar = (partial ? raw : full) + 8 * slot.at;
                        bar_expect(bar, F::kTile);
                        for (int y = 0; y < HALVES; ++y)
                            tma_load<1>(ring + slot.at * F::kTile + y * kHalfTile, values ? &map_v : &map_k, 64 * y, walk.it.h, it.begin + i / 2 * kKeys, bar);
                    }
                    if (lane == 0) sh.loads = n + 1;
                    __syncwarp();
                }
            }
        } else if (warp == 11) {
            // clear what lies behind a sequence in its last values
            uint32_t n = 0, parities = 0;
            while (ok && walk.next()) {
                const Work it = walk.it;
                const int tiles = max(query_tile(it, 0, g.kt).tiles, query_tile(it, 1, g.kt).tiles);
                if (!tiles) continue;
                n += 2 * tiles;
                const int rest = it.end - it.begin - (tiles - 1) * kKeys;
                if (rest >= kKeys) continue;
                const At slot(n - 1);
                if (!(ok = warp_wait(raw + 8 * slot.at, parities >> slot.at & 1, &sh.loads))) break;
                parities ^= 1u << slot.at;
                clear_rows<HALVES>(smem + (2 * F::kSets + slot.at) * F::kTile, rest, lane);
                if (lane == 0) bar_arrive(full + 8 * slot.at);
            }
        } else if (F::kLanes == 2) {
            // multiply for one tile of queries: its next scores right behind each product with the values
            const int which = warp - 9;
            uint32_t n = 0, items = 0, count = 0;  // slots before the present item, items and tiles of this lane so far
            int tiles = 0, most = 0, j = -1;
            int next_tiles = 0, next_most = 0;
            bool next = false;
            // The item after the present one: looked up while the softmax warps are at work, not when they are through.
            auto look = [&]() {
                next = walk.next();
                next_tiles = next ? query_tile(walk.it, which, g.kt).tiles : 0;
                next_most = next ? max(next_tiles, query_tile(walk.it, 1 - which, g.kt).tiles) : 0;
            };
            look();
            // moves to this lane's next tile, past slots that it does not need
            auto step = [&]() {
                if (++j < tiles) return true;
                for (;;) {
                    for (int i = 2 * j; i < 2 * most; ++i) {
                        const At slot(n + i);
                        if (!(ok = warp_wait(full + 8 * slot.at, slot.parity, &sh.loads))) return false;
                        if (lane == 0) bar_arrive(empty + 8 * slot.at);
                        __syncwarp();
                    }
                    n += 2 * most;
                    if (!next) return false;
                    j = 0, tiles = next_tiles, most = next_most;
                    if (tiles) {
                        ++items;
                        return true;
                    }
                    look();
                }
            };
            auto scores = [&]() {
                const At slot(n + 2 * j);
                if (!first_product(which, items - 1, j, tiles, slot.at, slot.parity)) return false;
                if (elect_one()) mma_commit<1>(empty + 8 * slot.at);
                __syncwarp();
                return true;
            };
            bool more = step();
            if (more) ok = scores();
            while (ok && more) {
                if (j == 0) look();
                const At slot(n + 2 * j + 1);
                if (!(ok = second_product(which, items - 1, j, tiles, slot.at, slot.parity, count))) break;
                if (elect_one()) mma_commit<1>(empty + 8 * slot.at);
                __syncwarp();
                ++count;
                more = step();
                if (ok && more) ok = scores();
            }
        } else if (warp == 9) {
            // multiply for both tiles of queries in turn
            uint32_t n = 0, items[2] = {0, 0}, count[2] = {0, 0};
            while (ok && walk.next()) {
                const int tiles[2] = {query_tile(walk.it, 0, g.kt).tiles, query_tile(walk.it, 1, g.kt).tiles};
                const int most = max(tiles[0], tiles[1]);
                if (!most) continue;
                {
                    const At slot(n);
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (ok && tiles[x]) ok = first_product(x, items[x], 0, tiles[x], slot.at, slot.parity);
                    if (!ok) break;
                    if (elect_one()) mma_commit<1>(empty + 8 * slot.at);
                    __syncwarp();
                }
                for (int j = 0; ok && j < most; ++j) {
                    const At values(n + 2 * j + 1), keys(n + 2 * j + 2);
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (!ok || j >= tiles[x]) continue;
                        if (!(ok = second_product(x, items[x], j, tiles[x], values.at, values.parity, count[x]++))) break;
                        if (j + 1 < tiles[x]) ok = first_product(x, items[x], j + 1, tiles[x], keys.at, keys.parity);
                    }
                    if (!ok) break;
                    if (elect_one()) {
                        mma_commit<1>(empty + 8 * values.at);
                        if (j + 1 < most) mma_commit<1>(empty + 8 * keys.at);
                    }
                    __syncwarp();
                }
                n += 2 * most;
                items[0] += tiles[0] != 0, items[1] += tiles[1] != 0;
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        const int which = warp / 4, row = threadIdx.x % 128;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        const uint32_t ts = tmem + 128 * which + lanes, to = tmem + 256 + 128 * which + lanes;
        const float c = g.scale * kLog2e;
        uint8_t* const stage = F::kStage ? smem + (2 * F::kSets + F::kSlots) * F::kTile + warp * kStageBytesOfWarp : nullptr;
        uint32_t count = 0, items = 0;  // tiles and items so far
        // the item whose output is still to be written
        RowsOut out = {};
        float* lse = nullptr;
        float l = 0.f, top = 0.f;
        bool pending = false;
        auto write = [&](uint32_t item) {
            const Set set(item);
            const uint32_t bar = 8 * (2 * which + set.at);
            if (!warp_wait(acc_full + bar, set.parity, &sh.loads)) return false;
            mma_fence_after();
            const float inv = __frcp_rn(l);
#pragma unroll 1
            for (int x = 0; x < 2 * HALVES; ++x) {
                if (32 * x >= g.dim) break;
                uint32_t o[32];
                tmem_fetch(to + 64 * set.at + 32 * x, o);
                tmem_wait(o);
                out.write<F16, WIDE>(32 * x, g.dim, o, inv, stage);
            }
            mma_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(acc_free + bar);
            if (out.own) *lse = top * g.scale + (log2_of(l) - kRaise<F16>) * kLn2;
            return true;
        };
        // of the row: its token in the tile and its head in the group; the tokens of the warp's first and last row
        const int row_token = row / g.group, row_head = row - row_token * g.group, first_token = (row & ~31) / g.group, last_token = (row | 31) / g.group;
        while (ok) {
            const bool more = walk.next();
            if (!more && !pending) break;
            const Work it = walk.it;
            const QueryTile q = query_tile(it, which, g.kt);
            const int token = q.first + row_token, head = walk.it.h * g.group + row_head, tiles = more ? q.tiles : 0;
            const bool live = row < g.group * g.kt && token < it.end;
            uint16_t* const own = live ? g.out.p + (int64_t)token * g.out.token + head * g.out.head : nullptr;
            float* const own_lse = g.lse + (int64_t)token * g.heads + head;
            if (more && it.begin < 0) {  // tokens of no sequence
                write_zeros(own, g.dim);
                if (live) *own_lse = 0.f;
            }
            if (more && !tiles) continue;
            float m_row = 0.f;
            Pair sum = both(0.f);
            for (int j = 0; j < max(tiles, 1); ++j) {
                if (tiles) {
                    if (!(ok = warp_wait(s_full + 8 * which, count & 1, &sh.loads))) break;
                    mma_fence_after();
                    // The last keys of the tile that the row and the warp's first row may see. Where all rows of the warp see the whole tile,
                    // the work is one run of code; elsewhere pieces of 32 keys that none sees are left out, and only those that not all
                    // see whole are masked.
                    const int reach = q.first - it.begin - j * kKeys, last = reach + row_token, low = reach + first_token;
                    const bool whole = low >= kKeys - 1;
                    const int seen = whole ? 4 : min(max((reach + last_token) / 32 + 1, 1), 4);
                    uint32_t s[4][32];
#pragma unroll
                    for (int x = 0; x < 4; ++x) tmem_fetch(ts + 32 * x, s[x]);
#pragma unroll
                    for (int x = 0; x < 4; ++x) tmem_wait(s[x]);
                    float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    auto piece_top = [&](const uint32_t (&p)[32]) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
#pragma unroll
                            for (int y = 0; y < 4; ++y) m[y] = max3(m[y], __uint_as_float(p[i + 2 * y]), __uint_as_float(p[i + 2 * y + 1]));
                    };
                    if (whole) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) piece_top(s[x]);
                    } else {
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            if (HALVES == 2 && x >= seen) continue;  // (16102 tokens, 15 / 3 heads of 77: 123 -> 114 us; 16 heads of 64: 69.8 -> 71.1)
                            if (32 * x + 31 > low) {
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (32 * x + i > last) s[x][i] = 0xFF800000u;  // -infinity
                            }
                            piece_top(s[x]);
                        }
                    }
                    const float tile_top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
                    // A row that has only met scores of -infinity keeps that as its maximum, so that whatever comes next is followed.
                    if (j == 0) {
                        m_row = tile_top;
                    } else if (__any_sync(0xFFFFFFFFu, live && (tile_top - m_row) * c > kGrow)) {  // rows that are not there have no say
                        const float next = fmaxf(m_row, tile_top), f = next > m_row ? exp2_of((m_row - next) * c) : 1.f;
                        m_row = next;
                        sum = sum * both(f);
                        if (!(ok = warp_wait(o_full + 8 * which, (count & 1) ^ 1, &sh.loads))) break;  // the product of the tile before
                        mma_fence_after();
                        const uint32_t acc = to + 64 * Set(items).at;
                        for (int x = 0; x < 2 * HALVES; ++x) {
                            uint32_t o[32];
                            tmem_fetch(acc + 32 * x, o);
                            tmem_wait(o);
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            tmem_store(acc + 32 * x, o);
                        }
                        tmem_store_wait();
                    }
                    // (s - maximum) c as one multiplication and addition is off by 2^-24 |maximum c|, since only one of the products is rounded.
                    // Where that is not small, the maximum is subtracted first; not where it is -infinity.
                    const float shift = m_row * c;
                    const bool far = live && !(fabsf(shift) < kFar);
                    if (__any_sync(0xFFFFFFFFu, far)) {
                        const Pair top2 = both(far && m_row > -INFINITY ? -m_row : 0.f);
#pragma unroll
                        for (int x = 0; x < 4; ++x)
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                const float2 d = split(pair(__uint_as_float(s[x][i]), __uint_as_float(s[x][i + 1])) + top2);
                                s[x][i] = __float_as_uint(d.x), s[x][i + 1] = __float_as_uint(d.y);
                            }
                    }
                    const Pair c2 = both(c), t2 = both(kRaise<F16> - (far ? 0.f : shift));
                    Pair tile_sum = both(0.f);  // small probabilities add up before they meet the sum of the row
                    auto probability = [&](uint32_t lo, uint32_t hi) {
                        const float2 e = split(fma2(pair(__uint_as_float(lo), __uint_as_float(hi)), c2, t2));
                        const float a = exp2_of(e.x), b = exp2_of(e.y);
                        tile_sum = tile_sum + pair(a, b);
                        return pack16<F16>(a, b);
                    };
                    if (whole) {
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            uint32_t p[32];
#pragma unroll
                            for (int x = 0; x < 2; ++x)
#pragma unroll
                                for (int i = 0; i < 32; i += 2) p[16 * x + i / 2] = probability(s[2 * half + x][i], s[2 * half + x][i + 1]);
                            tmem_store(ts + 32 * half, p);
                        }
                    } else {
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            uint32_t p[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) p[i] = 0;
                            if (x < seen) {
#pragma unroll
                                for (int i = 0; i < 32; i += 2) p[i / 2] = probability(s[x][i], s[x][i + 1]);
                            }
                            tmem_store(ts + 16 * x, p);
                        }
                    }
                    sum = sum + tile_sum;
                    tmem_store_wait();
                    mma_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(p_full + 8 * which);
                    ++count;
                }
                if (j == 0 && pending) {  // behind the first tile of the next item, or the last item of all
                    pending = false;
                    if (!(ok = write(items - 1))) break;
                }
            }
            if (!ok || !more) break;
            out.set(own);
            lse = own_lse, l = total(sum), top = m_row;
            pending = true;
            ++items;
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

cudaError_t launch_plan(PlanArgs a, int lists, cudaStream_t stream) {
    a.lists = lists;
    const int64_t blocks = (a.zeros + 16 * kPlanThreads - 1) / (16 * kPlanThreads), most = device_sms();
    return launch_after(k_plan, dim3(lists + (unsigned)(blocks < most ? blocks : most)), dim3(kPlanThreads), stream, a);
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
    auto kernel = a.out.wide ? k_attention<HALVES, F16, true> : k_attention<HALVES, F16, false>;
    static std::atomic<uint64_t> ready[2];
    err = allow_smem(kernel, Forward<HALVES>::kSmem, ready[a.out.wide != 0]);
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
    if (p.most * k->heads >= 1ll << 31) return ONES_ERR_BAD_PARAM;
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
    const ForwardArgs a = {plan.items[0], plan.head, heads_out(*out, dim, tokens), d_lse, tokens, q->heads, k->heads, p.group, p.kt, dim, scale};
    const bool f16 = type == ONES_F16;
    if (dim > 64)
        err = f16 ? launch_forward<2, true>(*q, *k, *v, a, p.most, stream) : launch_forward<2, false>(*q, *k, *v, a, p.most, stream);
    else
        err = f16 ? launch_forward<1, true>(*q, *k, *v, a, p.most, stream) : launch_forward<1, false>(*q, *k, *v, a, p.most, stream);
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // extern "C"
