// Gradients of the causal attention.
//
// Two passes over the pairs of tiles, each with sums that stay in tensor memory until they are whole: one for each tile of
// queries (dq: scores, dp and one product over the keys before it), then one for each tile of keys (dk and dv: scores, dp and
// two products over the queries behind it, all heads of the group one after the other). Seven products where five would do
// if dq were added up in memory: but that takes 64 KB of atomic additions for every pair of tiles, whose order would change
// the results, or turns taken between blocks. A pair costs 2 x 2048 cycles of products (see below for the eighth) and 2 x 1024 of
// exponentials. Measured: 16384 tokens, 16 / 4 heads of 128: 1740 us for the queries and 1690 for the keys, 1.27 and 1.30 PFLOP/s of what they
// execute (the card at its power limit, 1.6 to 1.77 GHz). 128 samples of 256 tokens, 16 heads of 64: survey 25 us (0.14 GB in
// and out at 5.4 TB/s), queries 110, keys 101: the warps that work on scores never wait for the tensor core there, a third of their
// time goes to the way out of the sums and to what begins and ends an item.
//
// What the rounding to 16 bits costs. Probabilities and the gradients of the scores (ds) are rounded to the tensors' type for their
// products: half a step of each, averaged by the sums. Errors of bfloat16 gradients, of their norm, of which 1.66e-3 are the rounding of the
// result: dq 1.66e-3 (one tile of keys) to 2.03e-3 (4096 tokens), dk 2.35e-3, dv 2.3e-3. bfloat16 has the range for whatever ds and its operands hold; float16 takes ds times a power of two. (bfloat16 queries
// and keys laid out as float16 times a power of two for each head left 11 bits of ds, but nothing of a sequence far below its
// neighbours, or beside keys that hold the type's lowest value.) And delta = dout . out takes over the rounding of
// out: an error e that all pairs of a row share, and that adds e sum_j p_j k_j to its dq (with values that have a common mean, percents of
// its norm). The sum of a row's ds has to be 0, so the pass over the queries finds e: it adds up p k beside ds k, one product more,
// takes e times that off, and leaves the exact delta for the second pass. The last tile of a row, where e is known, needs no
// such product: its ds are formed with the exact delta at once.
#include "ones_attention.cuh"

#include <math.h>

#include <type_traits>

namespace ones {

namespace {

constexpr int kThreads = 384;  // two groups of four warps that work on scores, then load, multiply, statistics and an idle warp

struct BackArgs {
    const Item* items;
    const PlanHead* head;
    const float* lse;           // [tokens][heads]
    float* delta;               // the same; exact from the first pass on
    const uint16_t* row_top;    // float16: [tokens][heads], the largest finite |dout| of a row
    const unsigned* top;        // float16: [slots][2][kv], that and the largest finite |v| of a sequence's group of heads
    HeadsOut dq, dk, dv;
    int tokens, heads, kv, group, kt, dim;
    float scale;
};

// float16 tensors: probabilities times 2^12 for their products, so that small ones keep their bits, and ds times 2^sigma, which takes the bound
// 2 dim max |dout| max |v| of |dp - delta| to 2^15: of the row (for dq) or the sequence (for dk, where rows meet), and of the sequence's values.
template <bool F16>
constexpr int kLift = F16 ? 12 : 0;
__device__ __forceinline__ float power2(int n) { return __int_as_float((n + 127) << 23); }  // -127 < n < 128
template <bool F16>
struct Sigma {
    unsigned dout, v;  // as they lie in memory
    __device__ __forceinline__ void fetch(const BackArgs& g, const Work& it) {
        const int64_t at = (int64_t)it.slot * 2 * g.kv + it.h;
        if (F16) dout = g.top[at], v = g.top[at + g.kv];
    }
    __device__ __forceinline__ int get() const {
        auto above = [](unsigned bits) { return (int)(__float_as_uint(__half2float(__ushort_as_half((uint16_t)bits))) >> 23) - 126; };  // |x| < 2^above
        return F16 ? min(15 - 8 - above(dout) - above(v), 100) : 0;  // 2^7 >= dim
    }
};
// What the exponent of a row's probabilities subtracts. A row whose lse lies beyond 2^24, where 32 bits hold no more of its keys' shares
// than that, has only seen keys that a mask's lowest value hides: its probabilities count as 0.
__device__ __forceinline__ float row_shift(float lse, int lift) {
    const float a = fabsf(lse);
    return a >= 0x1p24f && a < INFINITY ? -INFINITY : lift - lse * kLog2e;
}

// ---- delta = dout . out, and (float16) the largest values of rows and sequences ----

struct Vectors {
    const uint16_t* p;
    int64_t token, head;
};
struct SurveyArgs {
    Vectors dout, out, v;
    const PlanHead* plan;
    float* delta;
    uint16_t *row_top, *v_top;  // float16: [tokens][heads] and [tokens][kv], the largest finite |dout| and |v|
    int tokens, heads, kv, dim, wide;  // wide: out starts on 16-byte boundaries
};

template <bool F16>
__device__ __forceinline__ float value16(uint16_t b) {
    return F16 ? __half2float(__ushort_as_half(b)) : __uint_as_float((uint32_t)b << 16);
}
template <bool F16>
__device__ __forceinline__ float2 values16(uint32_t w) {
    if constexpr (F16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}

// Values c..c + 7 of a vector of dim values that starts on a 16-byte boundary. RAGGED: dim is no multiple of 8, and what lies behind
// the vector's end is read along with it, to be masked out where the values are used (masked at once, it keeps the next loads
// waiting: 54 us instead of 35 for 16102 tokens x 15 heads x 77), but not behind the last vector of all: vectors start on 16-byte
// boundaries, so that any other one's last piece ends before the last one does.
template <bool RAGGED>
__device__ __forceinline__ uint4 eight_of(const uint16_t* p, int c, int dim, bool last) {
    if (c >= dim) return make_uint4(0, 0, 0, 0);
    if (!RAGGED || !last || c + 8 <= dim) return *reinterpret_cast<const uint4*>(p + c);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < dim) w[i / 2] |= (uint32_t)p[c + i] << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool RAGGED>
struct Own {  // which of the lane's eight values the vectors have
    uint4 mask;
    __device__ __forceinline__ Own(int c, int dim) {
        auto word = [&](int i) { return c + i + 1 < dim ? 0xFFFFFFFFu : c + i < dim ? 0xFFFFu : 0u; };
        mask = make_uint4(word(0), word(2), word(4), word(6));
    }
    __device__ __forceinline__ uint4 operator()(const uint4& v) const {
        return RAGGED ? make_uint4(v.x & mask.x, v.y & mask.y, v.z & mask.z, v.w & mask.w) : v;
    }
};
// The largest finite float16's bits.
__device__ __forceinline__ unsigned largest_of(const uint4& v) {
    constexpr unsigned kLimit = 0x7C00u;  // infinity
    const uint32_t w[4] = {v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu, v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu};
    const uint32_t m = __vmaxu2(__vmaxu2(w[0], w[1]), __vmaxu2(w[2], w[3]));
    unsigned top = max(m & 0xFFFFu, m >> 16);
    if (top >= kLimit) {
        top = 0;
        for (int i = 0; i < 8; ++i) {
            const unsigned b = w[i / 2] >> (16 * (i & 1)) & 0xFFFFu;
            if (b < kLimit) top = max(top, b);
        }
    }
    return top;
}

// LANES x 8 values are a vector, which a group of lanes takes. A block takes kTokens tokens at a time.
constexpr int kTokens = 16;
template <bool F16, int LANES, bool RAGGED>
__global__ void __launch_bounds__(256, 4) k_survey(const __grid_constant__ SurveyArgs g) {
    constexpr int kGroups = 256 / LANES, kAtOnce = 4;
    const int lane = threadIdx.x % LANES, c = 8 * lane;
    const Own<RAGGED> own_of(c, g.dim);
    wait_for_predecessor();
    let_successor_start();
    const int t0 = g.plan->covered[0], t1 = g.plan->covered[1];
    auto top_of = [](const uint4& v) {  // of the group's vector
        unsigned m = largest_of(v);
#pragma unroll
        for (int x = LANES / 2; x; x >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, x));
        return (uint16_t)m;
    };
    const int own = threadIdx.x / LANES;
    const uint32_t per_head = 0xFFFFFFFFu / g.heads + 1, per_kv = 0xFFFFFFFFu / g.kv + 1;
    auto over = [](uint32_t r, uint32_t n, uint32_t per) { return n == 1 ? r : __umulhi(r, per); };  // r / n below 2^16, with 2^32 / n rounded up
    for (int first = t0 + blockIdx.x * kTokens; first < t1; first += gridDim.x * kTokens) {
        const int n_t = min(kTokens, t1 - first);
        // Neighbouring groups have neighbouring vectors: four of each group are on their way at a time.
        const uint16_t *dout = g.dout.p + first * g.dout.token, *out = g.out.p + first * g.out.token;
        for (int r0 = 0; r0 < n_t * g.heads; r0 += kAtOnce * kGroups) {
            uint4 a[kAtOnce], b[kAtOnce];
            int at_t[kAtOnce], at_h[kAtOnce];
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) {
                const int r = r0 + x * kGroups + own;
                at_t[x] = over(r, g.heads, per_head), at_h[x] = r - at_t[x] * g.heads;
                a[x] = b[x] = make_uint4(0, 0, 0, 0);
                if (at_t[x] >= n_t) continue;
                const bool last = first + at_t[x] == g.tokens - 1 && at_h[x] == g.heads - 1;
                a[x] = eight_of<RAGGED>(dout + at_t[x] * g.dout.token + at_h[x] * g.dout.head, c, g.dim, last);
                if (g.wide) b[x] = eight_of<RAGGED>(out + at_t[x] * g.out.token + at_h[x] * g.out.head, c, g.dim, last);
            }
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) {
                const bool live = at_t[x] < n_t;
                float dot = 0.f;
                a[x] = own_of(a[x]), b[x] = own_of(b[x]);
                if (F16) {
                    const uint16_t m = top_of(a[x]);
                    if (lane == 0 && live) g.row_top[(int64_t)(first + at_t[x]) * g.heads + at_h[x]] = m;
                }
                if (g.wide) {
                    const uint32_t u[4] = {a[x].x, a[x].y, a[x].z, a[x].w}, w[4] = {b[x].x, b[x].y, b[x].z, b[x].w};
                    Pair d = both(0.f);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 y = values16<F16>(u[i]), z = values16<F16>(w[i]);
                        d = fma2(pair(y.x, y.y), pair(z.x, z.y), d);
                    }
                    dot = total(d);
                } else if (live) {  // single values, in another order: dout is read again, from the first-level cache
                    const uint16_t* const u = dout + at_t[x] * g.dout.token + at_h[x] * g.dout.head;
                    const uint16_t* const w = out + at_t[x] * g.out.token + at_h[x] * g.out.head;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (lane + i * LANES < g.dim) dot = fmaf(value16<F16>(u[lane + i * LANES]), value16<F16>(w[lane + i * LANES]), dot);
                }
#pragma unroll
                for (int m = LANES / 2; m; m >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, m);
                if (lane == 0 && live) g.delta[(int64_t)(first + at_t[x]) * g.heads + at_h[x]] = dot;
            }
        }
        for (int r0 = 0; F16 && r0 < n_t * g.kv; r0 += kAtOnce * kGroups) {
            const uint16_t* const v = g.v.p + first * g.v.token;
            uint4 a[kAtOnce];
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) {
                const int r = r0 + x * kGroups + own, t = over(r, g.kv, per_kv), h = r - t * g.kv;
                a[x] = t < n_t ? eight_of<RAGGED>(v + t * g.v.token + h * g.v.head, c, g.dim, first + t == g.tokens - 1 && h == g.kv - 1) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) {
                const int r = r0 + x * kGroups + own, t = over(r, g.kv, per_kv);
                const uint16_t m = top_of(own_of(a[x]));
                if (lane == 0 && t < n_t) g.v_top[(int64_t)first * g.kv + r] = m;
            }
        }
    }
}

// float16: the largest values of every sequence and group of heads, 128 tokens by a warp. (By themselves, since the survey knows nothing of sequences;
// 40 documents of 16102 tokens, 3 groups: 3 us.)
struct TopArgs {
    const Item* items;  // of the keys
    const PlanHead* head;
    const uint16_t *row_top, *v_top;
    unsigned* top;
    int heads, kv;
};
__global__ void __launch_bounds__(256) k_tops(const TopArgs g) {
    wait_for_predecessor();
    let_successor_start();
    const int lane = threadIdx.x % 32, group = g.heads / g.kv;
    const uint32_t total = (uint32_t)g.head->count * g.kv;
    for (uint32_t w = blockIdx.x * 8 + threadIdx.x / 32; w < total; w += gridDim.x * 8) {
        const Item it = g.items[w / g.kv];
        const int h = w % g.kv;
        if (it.begin < 0) continue;
        unsigned d = 0, v = 0;
        for (int t = it.first + lane; t < min(it.first + kKeys, it.end); t += 32) {
            v = max(v, (unsigned)g.v_top[(int64_t)t * g.kv + h]);
            const uint16_t* const rows = g.row_top + (int64_t)t * g.heads + h * group;
            for (int i = 0; i < group; ++i) d = max(d, (unsigned)rows[i]);
        }
        d = __reduce_max_sync(0xFFFFFFFFu, d), v = __reduce_max_sync(0xFFFFFFFFu, v);
        if (lane) continue;
        unsigned* const to = g.top + (int64_t)it.slot * 2 * g.kv + h;
        atomicMax(to, d), atomicMax(to + g.kv, v);
    }
}

// Heads of up to 64 values leave room for two sets of what belongs to an item (its tiles in shared memory, its sums in tensor
// memory), so that the next item's first tile is begun before the sums of the last one are written.
template <int HALVES>
struct Back {
    static constexpr int kTile = HALVES * kHalfTile;
    static constexpr int kSets = HALVES == 2 ? 1 : 2;
    // dq: queries and dout of the tile, rings of keys (needed until the last product) and values
    static constexpr int kKeySlots = HALVES == 2 ? 3 : 4, kValueSlots = HALVES == 2 ? 2 : 3;
    static constexpr int kStage = HALVES == 2 ? 0 : 8 * kStageBytesOfWarp;  // for the way out
    static constexpr int kSmemQueries = (2 * kSets + kKeySlots + kValueSlots) * kTile + kStage + 1024;
    // dk, dv: keys and values of the tile, rings of queries and dout, their statistics
    static constexpr int kSlots = HALVES == 2 ? 2 : 4;
    static constexpr int kStats = 2;
    static constexpr int kSmemKeys = (2 * kSets + 2 * kSlots) * kTile + kStats * 2 * kRows * 4 + kStage + 1024;
};

// ---- dq ----

struct QueriesShared {
    uint64_t q_full[2], q_free[2], k_full[4], k_raw[4], k_empty[4], v_full[4], v_empty[4], s_full, p_full, dp_full, ds_full, acc_full[2], acc_free[2], met[4];
    uint32_t tmem;
    volatile uint32_t loads;  // how many tiles have been sent for: what the other warps' waits go by
};

// Tiles of keys that a tile of queries meets; they are taken from the last to the first.
__device__ __forceinline__ int key_tiles(const Work& it, int kt) {
    return it.begin < 0 ? 0 : (min(it.first + kt, it.end) - 1 - it.begin) / kKeys + 1;
}

template <int HALVES, bool F16, bool WIDE>
__global__ void __launch_bounds__(kThreads, 1)
    k_attention_queries(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_do,
                        const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const BackArgs g) {
    using B = Back<HALVES>;
    using KeySlot = Slot<B::kKeySlots>;
    using ValueSlot = Slot<B::kValueSlots>;
    using Set = Slot<B::kSets>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ QueriesShared sh;
    __shared__ WorkList list;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t at_k = base + 2 * B::kSets * B::kTile, at_v = at_k + B::kKeySlots * B::kTile;  // before: queries and dout of each set
    const uint32_t q_full = smem_u32(sh.q_full), q_free = smem_u32(sh.q_free), k_full = smem_u32(sh.k_full), k_raw = smem_u32(sh.k_raw),
                   k_empty = smem_u32(sh.k_empty), v_full = smem_u32(sh.v_full), v_empty = smem_u32(sh.v_empty), s_full = smem_u32(&sh.s_full),
                   p_full = smem_u32(&sh.p_full), dp_full = smem_u32(&sh.dp_full), ds_full = smem_u32(&sh.ds_full),
                   acc_full = smem_u32(sh.acc_full), acc_free = smem_u32(sh.acc_free), met = smem_u32(sh.met) + 8 * (warp % 4);  // of the two warps that have the same rows
    if (threadIdx.x == 0) {
        sh.loads = 0;
        tma_prefetch(&map_q), tma_prefetch(&map_do), tma_prefetch(&map_k), tma_prefetch(&map_v);
        bar_init(s_full, 1), bar_init(p_full, 8), bar_init(dp_full, 1), bar_init(ds_full, 8);
        for (int i = 0; i < 4; ++i) bar_init(smem_u32(&sh.met[i]), 2);
        for (int i = 0; i < 2; ++i) {
            bar_init(q_full + 8 * i, 1), bar_init(q_free + 8 * i, 1);
            bar_init(acc_full + 8 * i, 1), bar_init(acc_free + 8 * i, 8);
        }
        for (int i = 0; i < 4; ++i) {
            bar_init(k_full + 8 * i, 1), bar_init(k_raw + 8 * i, 1), bar_init(k_empty + 8 * i, 1);
            bar_init(v_full + 8 * i, 1), bar_init(v_empty + 8 * i, 1);
        }
        bar_init_done();
    }
    if (warp == 9) tmem_alloc<1>(smem_u32(&sh.tmem), 512);
    wait_for_predecessor();
    let_successor_start();
    list_work(list, g.items, g.head, g.kv);
    mma_fence_before();
    __syncthreads();
    mma_fence_after();
    const uint32_t tmem = sh.tmem, t_dp = tmem + 128, t_acc = tmem + 256, t_pk = tmem + 384;
    Walk walk(list, g.items, g.kv);
    bool ok = true;

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 8) {
            // load
            uint32_t n = 0, items = 0;
            const uint32_t qbytes = HALVES * g.group * g.kt * 128;
            while (ok && walk.next()) {
                const Work it = walk.it;
                const int tiles = key_tiles(it, g.kt);
                if (!tiles) continue;
                const Set set(items++);
                if (!(ok = warp_wait(q_free + 8 * set.at, set.parity ^ 1))) break;
                if (elect_one()) {
                    const uint32_t to = base + 2 * set.at * B::kTile, bar = q_full + 8 * set.at;
                    bar_expect(bar, 2 * qbytes);
                    for (int x = 0; x < HALVES; ++x) {
                        tma_load<1>(to + x * kHalfTile, &map_q, 64 * x, walk.it.h * g.group, it.first, bar);
                        tma_load<1>(to + B::kTile + x * kHalfTile, &map_do, 64 * x, walk.it.h * g.group, it.first, bar);
                    }
                }
                __syncwarp();
                for (int j = tiles - 1; j >= 0; --j, ++n) {
                    const KeySlot ks(n);
                    const bool partial = it.end - it.begin < (j + 1) * kKeys;  // that tile is cleared first
                    if (!(ok = warp_wait(k_empty + 8 * ks.at, ks.parity ^ 1))) break;
                    if (elect_one()) {
                        const uint32_t bar = (partial ? k_raw : k_full) + 8 * ks.at;
                        bar_expect(bar, B::kTile);
                        for (int x = 0; x < HALVES; ++x)
                            tma_load<1>(at_k + ks.at * B::kTile + x * kHalfTile, &map_k, 64 * x, walk.it.h, it.begin + j * kKeys, bar);
                    }
                    __syncwarp();
                    const ValueSlot vs(n);
                    if (!(ok = warp_wait(v_empty + 8 * vs.at, vs.parity ^ 1))) break;
                    if (elect_one()) {
                        const uint32_t bar = v_full + 8 * vs.at;
                        bar_expect(bar, B::kTile);
                        for (int x = 0; x < HALVES; ++x)
                            tma_load<1>(at_v + vs.at * B::kTile + x * kHalfTile, &map_v, 64 * x, walk.it.h, it.begin + j * kKeys, bar);
                    }
                    if (lane == 0) sh.loads = n + 1;
                    __syncwarp();
                }
            }
        } else if (warp == 10) {
            // clear what lies behind a sequence in its last keys
            uint32_t n = 0, parities = 0;
            while (ok && walk.next()) {
                const Work it = walk.it;
                const int tiles = key_tiles(it, g.kt), rest = it.end - it.begin - (tiles - 1) * kKeys;
                if (tiles && rest < kKeys) {
                    const KeySlot ks(n);
                    if (!(ok = warp_wait(k_raw + 8 * ks.at, parities >> ks.at & 1, &sh.loads))) break;
                    parities ^= 1u << ks.at;
                    clear_rows<HALVES>(smem + (2 * B::kSets + ks.at) * B::kTile, rest, lane);
                    if (lane == 0) bar_arrive(k_full + 8 * ks.at);
                }
                n += tiles;
            }
        } else if (warp == 9) {
            // multiply: p or ds with the keys, and behind each product the next tile's scores or dp in the place of what it used
            const uint32_t id_rows = attend_desc(F16, false, kKeys), id_acc = attend_desc(F16, true, 16 * ((g.dim + 15) / 16));
            const int steps = (g.dim + 15) / 16;
            uint32_t t = 0, items = 0;  // the present tile, counted through all items; items begun
            int tiles = 0, j = 0;       // of the present item, tile j from the last on
            auto step = [&]() {
                if (--j >= 0) return true;
                do {
                    if (!walk.next()) return false;
                    tiles = key_tiles(walk.it, g.kt);
                } while (!tiles);
                j = tiles - 1;
                ++items;
                return true;
            };
            auto scores = [&](uint32_t n) {
                const Set set(items - 1);
                const KeySlot ks(n);
                if (j == tiles - 1 && !warp_wait(q_full + 8 * set.at, set.parity, &sh.loads)) return false;
                if (!warp_wait(k_full + 8 * ks.at, ks.parity, &sh.loads)) return false;
                mma_fence_after();
                if (elect_one()) {
                    product_rows<HALVES>(tmem, base + 2 * set.at * B::kTile, at_k + ks.at * B::kTile, id_rows, steps);
                    mma_commit<1>(s_full);
                }
                __syncwarp();
                return true;
            };
            auto products_of_dout = [&](uint32_t n) {
                const Set set(items - 1);
                const ValueSlot vs(n);
                if (!warp_wait(v_full + 8 * vs.at, vs.parity, &sh.loads)) return false;
                mma_fence_after();
                if (elect_one()) {
                    product_rows<HALVES>(t_dp, base + (2 * set.at + 1) * B::kTile, at_v + vs.at * B::kTile, id_rows, steps);
                    mma_commit<1>(dp_full);
                    mma_commit<1>(v_empty + 8 * vs.at);
                    if (j == 0) mma_commit<1>(q_free + 8 * set.at);
                }
                __syncwarp();
                return true;
            };
            bool any = step();
            if (any) ok = scores(0) && products_of_dout(0);
            while (ok && any) {
                const Set set(items - 1);
                const KeySlot ks(t);
                const bool first = j == tiles - 1, last = j == 0;
                const uint32_t k = at_k + ks.at * B::kTile;
                if (!(ok = warp_wait(p_full, t & 1, &sh.loads))) break;
                if (first && !(ok = warp_wait(acc_free + 8 * set.at, set.parity ^ 1, &sh.loads))) break;
                mma_fence_after();
                if (!last) {
                    if (elect_one()) product_tmem(t_pk + 64 * set.at, tmem, tmem + 64, k, id_acc, !first);
                    __syncwarp();
                }
                any = step();
                if (any && !(ok = scores(t + 1))) break;
                if (!(ok = warp_wait(ds_full, t & 1, &sh.loads))) break;
                mma_fence_after();
                if (elect_one()) {
                    product_tmem(t_acc + 64 * set.at, t_dp, t_dp + 64, k, id_acc, !first);
                    if (last) product_tmem(t_acc + 64 * set.at, t_dp + 32, t_dp + 96, k, id_acc, true);
                    mma_commit<1>(k_empty + 8 * ks.at);
                    if (last) mma_commit<1>(acc_full + 8 * set.at);
                }
                __syncwarp();
                if (any && !(ok = products_of_dout(t + 1))) break;
                ++t;
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int half = warp / 4, row = threadIdx.x % 128;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        uint32_t t = 0, items = 0, mph = 0;
        uint8_t* const stage = B::kStage ? smem + (2 * B::kSets + B::kKeySlots + B::kValueSlots) * B::kTile + warp * kStageBytesOfWarp : nullptr;
        // of the row: its token in the tile and its head in the group; the tokens of the warp's first and last row
        const int row_token = row / g.group, row_head = row - row_token * g.group, first_token = (row & ~31) / g.group, last_token = (row | 31) / g.group;
        // the item whose dq is still to be written
        RowsOut out = {};
        float factor = 0.f, excess = 0.f;  // excess: of its ds (but those of the last tile), for each p
        bool pending = false, several = false;
        auto write = [&](uint32_t item) {
            const Set set(item);
            if (!warp_wait(acc_full + 8 * set.at, set.parity, &sh.loads)) return false;
            mma_fence_after();
#pragma unroll 1
            for (int x = 0; x < HALVES; ++x) {
                const int col = 32 * (half * HALVES + x);
                if (col >= g.dim) break;
                uint32_t o[32];
                tmem_fetch(t_acc + 64 * set.at + col + lanes, o);
                tmem_wait(o);
                if (several) {
                    uint32_t pk[32];
                    tmem_fetch(t_pk + 64 * set.at + col + lanes, pk);
                    tmem_wait(pk);
                    const Pair e2 = both(-excess);
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const float2 d = split(fma2(pair(__uint_as_float(pk[i]), __uint_as_float(pk[i + 1])), e2, pair(__uint_as_float(o[i]), __uint_as_float(o[i + 1]))));
                        o[i] = __float_as_uint(d.x), o[i + 1] = __float_as_uint(d.y);
                    }
                }
                out.write<F16, WIDE>(col, g.dim, o, factor, stage);
            }
            mma_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(acc_free + 8 * set.at);
            return true;
        };
        // what the next item needs of memory is fetched before the present one is worked on (128 samples of 256 tokens: 118 -> 113 us;
        // the same in the pass over the keys, which needs the powers only: 120 -> 126)
        struct {
            float lse, delta;
            Sigma<F16> sigma;
        } ahead = {};
        bool more;
        auto look = [&]() {
            more = walk.next();
            if (!more || walk.it.begin < 0) return;
            const int token = walk.it.first + row_token;
            const int64_t at = (int64_t)token * g.heads + walk.it.h * g.group + row_head;
            ahead.sigma.fetch(g, walk.it);
            if (row < g.group * g.kt && token < walk.it.end) {
                ahead.lse = g.lse[at], ahead.delta = g.delta[at];
                if (F16) ahead.sigma.dout = g.row_top[at];
            }
        };
        look();
        while (ok && more) {
            const Work it = walk.it;
            const int h = it.h, tiles = key_tiles(it, g.kt);
            const int token = it.first + row_token, head = h * g.group + row_head;
            const bool live = row < g.group * g.kt && token < it.end;
            uint16_t* const own = live ? g.dq.p + (int64_t)token * g.dq.token + head * g.dq.head : nullptr;
            const int sigma = ahead.sigma.get();
            const float lse = ahead.lse, delta = live ? ahead.delta : 0.f;
            look();
            if (it.begin < 0) {
                if (half == 0) write_zeros(own, g.dim);
                continue;
            }
            const float unit = power2(sigma - kLift<F16>);  // of ds by that of p
            float fix = 0.f;
            const int64_t at = (int64_t)token * g.heads + head;
            const Pair c2 = both(g.scale * kLog2e), l2 = both(live ? row_shift(lse, kLift<F16>) : -INFINITY), s2 = both(unit);
            Pair d2 = both(-delta * unit), sum = both(0.f), lost = both(0.f);  // lost: what the rounding of ds adds to its sum
            for (int j = tiles - 1; j >= 0; --j, ++t) {
                if (!(ok = warp_wait(s_full, t & 1, &sh.loads))) break;
                mma_fence_after();
                const uint32_t ts = tmem + 64 * half + lanes, td = t_dp + 64 * half + lanes;
                uint32_t s[2][32], dp[2][32];
                tmem_fetch(ts, s[0]), tmem_fetch(ts + 32, s[1]);
                tmem_wait(s[0]), tmem_wait(s[1]);
                auto probabilities = [&](uint32_t (&p)[32]) {
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const float2 e = split(fma2(pair(__uint_as_float(p[i]), __uint_as_float(p[i + 1])), c2, l2));
                        p[i] = __float_as_uint(exp2_of(e.x)), p[i + 1] = __float_as_uint(exp2_of(e.y));
                    }
                };
                // of this half: the last key that the row sees, that the warp's first and that its last row does
                const int last = token - it.begin - j * kKeys - 64 * half, low = last - (row_token - first_token), high = low + (last_token - first_token);
                if (low >= 63) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) probabilities(s[x]);
                } else {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (high < 32 * x) {  // none of the warp's rows sees any of these keys
#pragma unroll
                            for (int i = 0; i < 32; ++i) s[x][i] = 0;
                            continue;
                        }
                        probabilities(s[x]);
                        if (low >= 32 * x + 31) continue;
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (32 * x + i > last) s[x][i] = 0;
                    }
                }
                if (j) {
                    uint32_t p[32];
#pragma unroll
                    for (int i = 0; i < 64; i += 2) p[i / 2] = pack16<F16>(__uint_as_float(s[i / 32][i % 32]), __uint_as_float(s[i / 32][i % 32 + 1]));
                    tmem_store(ts, p);
                    tmem_store_wait();
                }
                mma_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_full);
                if (!(ok = warp_wait(dp_full, t & 1, &sh.loads))) break;
                mma_fence_after();
                tmem_fetch(td, dp[0]), tmem_fetch(td + 32, dp[1]);
                tmem_wait(dp[0]), tmem_wait(dp[1]);
                if (it.end - it.begin < (j + 1) * kKeys) {  // values behind the sequence's end
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (32 * x + i > last) dp[x][i] = 0;
                }
                auto p_at = [&](int x, int i) { return pair(__uint_as_float(s[x][i]), __uint_as_float(s[x][i + 1])); };
                auto ds_at = [&](int x, int i) {
                    const Pair y = pair(__uint_as_float(dp[x][i]), __uint_as_float(dp[x][i + 1]));
                    return p_at(x, i) * (F16 ? fma2(y, s2, d2) : y + d2);
                };
                if (j == 0) {
                    // the last tile: what the row's ds add up to is what its delta is off by
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 32; i += 2) sum = sum + ds_at(x, i);
                    // the other half of the columns is with the warp of the same lanes: they meet in columns that dp has left
                    const float own_sum = total(sum), own_lost = total(lost);
                    tmem_put(td + 32, own_sum, own_lost);
                    mma_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(met);
                    if (!(ok = warp_wait(met, mph, &sh.loads))) break;
                    mph ^= 1;
                    mma_fence_after();
                    const float2 other = tmem_get(t_dp + 64 * (1 - half) + 32 + lanes);
                    const float r = own_sum + other.x;
                    if (half == 0 && live) g.delta[at] = delta + r * power2(-sigma);
                    fix = (r + (own_lost + other.y)) * power2(-kLift<F16>);
                    d2 = d2 + both(-fix);
                    // both have read before either writes there again
                    mma_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(met);
                    if (!(ok = warp_wait(met, mph, &sh.loads))) break;
                    mph ^= 1;
                    mma_fence_after();
                    // The last tile, which is the only one of short rows, has ds in two terms (128 x 256 tokens: error of dq 2.5e-3 -> 1.72e-3 of its
                    // norm, of which 1.66e-3 are the rounding of the result; 4096 tokens 2.4e-3 -> 2.03e-3).
                    uint32_t ds[32], rest[32];
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            const float2 f = split(ds_at(x, i));
                            const uint32_t d = pack16<F16>(f.x, f.y);
                            const float2 e = values16<F16>(d);
                            ds[16 * x + i / 2] = d, rest[16 * x + i / 2] = pack16<F16>(f.x - e.x, f.y - e.y);
                        }
                    tmem_store(td + 32, rest);
                    tmem_store(td, ds);
                } else {
                    uint32_t ds[32];
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            const Pair v = ds_at(x, i);
                            const float2 f = split(v);
                            const uint32_t d = pack16<F16>(f.x, f.y);
                            const float2 e = values16<F16>(d);
                            ds[16 * x + i / 2] = d;
                            sum = sum + v, lost = lost + fma2(both(-1.f), v, pair(e.x, e.y));
                        }
                    tmem_store(td, ds);
                }
                tmem_store_wait();
                mma_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(ds_full);
                if (j == tiles - 1 && pending) {
                    pending = false;
                    if (!(ok = write(items - 1))) break;
                }
            }
            if (!ok) break;
            out.set(own);
            factor = g.scale * power2(-sigma);
            excess = fix, several = tiles > 1;
            pending = true;
            ++items;
        }
        if (ok && pending) ok = write(items - 1);
    }
    if (!ok) let_copies_end();
    __syncwarp();
    mma_fence_before();
    __syncthreads();
    mma_fence_after();
    if (warp == 9) tmem_free<1>(tmem, 512);
}

// ---- dk and dv ----

// float16 tensors: where few tiles add up to dk, the rounding of ds would show beside that of the result (error of dk 1.52 times that of
// one rounding at 195 queries of 5 heads): ds has two terms there, one product more. With more tiles it averages out (1.38 to 1.45).
constexpr int kFineTiles = 16;

struct KeysShared {
    uint64_t kv_full[2], kv_free[2], q_full[4], q_raw[4], q_empty[4], do_full[4], do_raw[4], do_empty[4], st_full[2], st_empty[2], s_full, p_full, dp_full,
        ds_full, acc_full[2], acc_free[2];
    uint32_t tmem;
    volatile uint32_t loads;  // how many tiles have been sent for: what the other warps' waits go by
};

// Tiles of queries that see a tile of keys: from the one that holds its first token to the sequence's last.
struct QuerySpan {
    int first, tiles;  // first token of the first tile
};
__device__ __forceinline__ QuerySpan query_span(const Work& it, int kt) {
    if (it.begin < 0) return {0, 0};
    const int f = (it.first - it.begin) / kt;
    return {it.begin + f * kt, (it.end - it.begin + kt - 1) / kt - f};
}

template <int HALVES, bool F16, bool WIDE>
__global__ void __launch_bounds__(kThreads, 1)
    k_attention_keys(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_do,
                     const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const BackArgs g) {
    using B = Back<HALVES>;
    using At = Slot<B::kSlots>;
    using Set = Slot<B::kSets>;
    using Stat = Slot<B::kStats>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ KeysShared sh;
    __shared__ WorkList list;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - smem_u32(smem_raw));
    constexpr int kRing = 2 * B::kSets;  // tiles before the rings: keys and values of each set
    const uint32_t at_q = base + kRing * B::kTile, at_do = at_q + B::kSlots * B::kTile;
    float* const stats = reinterpret_cast<float*>(smem + (kRing + 2 * B::kSlots) * B::kTile);  // [stage][2][128]
    const uint32_t kv_full = smem_u32(sh.kv_full), kv_free = smem_u32(sh.kv_free), q_full = smem_u32(sh.q_full), q_raw = smem_u32(sh.q_raw),
                   q_empty = smem_u32(sh.q_empty), do_full = smem_u32(sh.do_full), do_raw = smem_u32(sh.do_raw), do_empty = smem_u32(sh.do_empty),
                   st_full = smem_u32(sh.st_full), st_empty = smem_u32(sh.st_empty), s_full = smem_u32(&sh.s_full), p_full = smem_u32(&sh.p_full),
                   dp_full = smem_u32(&sh.dp_full), ds_full = smem_u32(&sh.ds_full), acc_full = smem_u32(sh.acc_full), acc_free = smem_u32(sh.acc_free);
    const int qrows = g.group * g.kt;
    if (threadIdx.x == 0) {
        sh.loads = 0;
        tma_prefetch(&map_q), tma_prefetch(&map_do), tma_prefetch(&map_k), tma_prefetch(&map_v);
        bar_init(s_full, 1), bar_init(p_full, 8), bar_init(dp_full, 1), bar_init(ds_full, 8);
        for (int i = 0; i < 4; ++i) {
            bar_init(q_full + 8 * i, 1), bar_init(q_raw + 8 * i, 1), bar_init(q_empty + 8 * i, 1);
            bar_init(do_full + 8 * i, 1), bar_init(do_raw + 8 * i, 1), bar_init(do_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(kv_full + 8 * i, 1), bar_init(kv_free + 8 * i, 1), bar_init(st_full + 8 * i, 32), bar_init(st_empty + 8 * i, 8);
            bar_init(acc_full + 8 * i, 1), bar_init(acc_free + 8 * i, 8);
        }
        bar_init_done();
    }
    // rows that no load fills, where the heads of a group do not divide 128: zeros
    for (int s = 0; s < 2 * B::kSlots && qrows < kRows; ++s)
        for (int i = qrows * 8 + threadIdx.x; i < kRows * 8; i += kThreads)
            for (int x = 0; x < HALVES; ++x)
                *reinterpret_cast<uint4*>(smem + (kRing + s) * B::kTile + x * kHalfTile + i * 16) = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async;" ::: "memory");
    if (warp == 9) tmem_alloc<1>(smem_u32(&sh.tmem), 512);
    wait_for_predecessor();
    let_successor_start();
    list_work(list, g.items, g.head, g.kv);
    mma_fence_before();
    __syncthreads();
    mma_fence_after();
    const uint32_t tmem = sh.tmem, t_dp = tmem + 128, t_dv = tmem + 256, t_dk = tmem + 384;
    Walk walk(list, g.items, g.kv);
    bool ok = true;

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 8) {
            // load
            uint32_t n = 0, items = 0;
            const uint32_t qbytes = HALVES * qrows * 128;
            while (ok && walk.next()) {
                const Work it = walk.it;
                const QuerySpan q = query_span(it, g.kt);
                if (!q.tiles) continue;
                const Set set(items++);
                if (!(ok = warp_wait(kv_free + 8 * set.at, set.parity ^ 1))) break;
                if (elect_one()) {
                    const uint32_t to = base + 2 * set.at * B::kTile, bar = kv_full + 8 * set.at;
                    bar_expect(bar, 2 * B::kTile);
                    for (int x = 0; x < HALVES; ++x) {
                        tma_load<1>(to + x * kHalfTile, &map_k, 64 * x, walk.it.h, it.first, bar);
                        tma_load<1>(to + B::kTile + x * kHalfTile, &map_v, 64 * x, walk.it.h, it.first, bar);
                    }
                }
                __syncwarp();
                for (int i = 0; ok && i < q.tiles; ++i, ++n) {
                    const At slot(n);
                    const int first = q.first + i * g.kt;
                    const bool partial = it.end - first < g.kt;  // that tile is cleared first
                    for (int kind = 0; kind < 2; ++kind) {
                        const uint32_t full = (kind ? partial ? do_raw : do_full : partial ? q_raw : q_full) + 8 * slot.at;
                        const uint32_t to = (kind ? at_do : at_q) + slot.at * B::kTile;
                        if (!(ok = warp_wait((kind ? do_empty : q_empty) + 8 * slot.at, slot.parity ^ 1))) break;
                        if (elect_one()) {
                            bar_expect(full, qbytes);
                            for (int x = 0; x < HALVES; ++x)
                                tma_load<1>(to + x * kHalfTile, kind ? &map_do : &map_q, 64 * x, walk.it.h * g.group, first, full);
                        }
                        __syncwarp();
                    }
                    if (lane == 0) sh.loads = n + 1;
                }
            }
        } else if (warp == 11) {
            // clear what lies behind a sequence in its last queries
            uint32_t n = 0, parities = 0;
            while (ok && walk.next()) {
                const Work it = walk.it;
                const QuerySpan q = query_span(it, g.kt);
                n += q.tiles;
                const int rest = it.end - q.first - (q.tiles - 1) * g.kt;
                if (!q.tiles || rest >= g.kt) continue;
                const At slot(n - 1);
                for (int kind = 0; kind < 2; ++kind) {
                    if (!(ok = warp_wait((kind ? do_raw : q_raw) + 8 * slot.at, parities >> slot.at & 1, &sh.loads))) break;
                    clear_rows<HALVES>(smem + (kRing + (kind ? B::kSlots : 0) + slot.at) * B::kTile, rest * g.group, lane);
                    if (lane == 0) bar_arrive((kind ? do_full : q_full) + 8 * slot.at);
                }
                parities ^= 1u << slot.at;
            }
        } else if (warp == 9) {
            // multiply: each product with the queries or dout, and behind it the next tile's scores or dp in the place of what it used
            const uint32_t id_rows = attend_desc(F16, false, kRows), id_acc = attend_desc(F16, true, 16 * ((g.dim + 15) / 16));
            const int steps = (g.dim + 15) / 16;
            uint32_t t = 0, items = 0;  // the present tile, counted through all items; items begun
            int i = 0, tiles = 0;
            auto step = [&]() {
                if (++i < tiles) return true;
                while (walk.next()) {
                    tiles = query_span(walk.it, g.kt).tiles;
                    if (!tiles) continue;
                    i = 0;
                    ++items;
                    return true;
                }
                return false;
            };
            // scores or dp of tile n, the i-th of its item
            auto rows = [&](uint32_t n, bool dp) {
                const At slot(n);
                const Set set(items - 1);
                if (!dp && i == 0 && !warp_wait(kv_full + 8 * set.at, set.parity, &sh.loads)) return false;
                if (!warp_wait((dp ? do_full : q_full) + 8 * slot.at, slot.parity, &sh.loads)) return false;
                mma_fence_after();
                if (elect_one()) {
                    product_rows<HALVES>(dp ? t_dp : tmem, base + (2 * set.at + dp) * B::kTile, (dp ? at_do : at_q) + slot.at * B::kTile, id_rows, steps);
                    mma_commit<1>(dp ? dp_full : s_full);
                    if (dp && i + 1 == tiles) mma_commit<1>(kv_free + 8 * set.at);
                }
                __syncwarp();
                return true;
            };
            bool any = step();
            if (any) ok = rows(0, false) && rows(0, true);
            while (ok && any) {
                const At slot(t);
                const Set set(items - 1);
                const bool first = i == 0, last = i + 1 == tiles, fine = F16 && tiles <= kFineTiles;
                if (!(ok = warp_wait(p_full, t & 1, &sh.loads))) break;
                if (first && !(ok = warp_wait(acc_free + 8 * set.at, set.parity ^ 1, &sh.loads))) break;
                mma_fence_after();
                if (elect_one()) {
                    product_tmem(t_dv + 64 * set.at, tmem, tmem + 64, at_do + slot.at * B::kTile, id_acc, !first);
                    mma_commit<1>(do_empty + 8 * slot.at);
                }
                __syncwarp();
                any = step();
                if (any && !(ok = rows(t + 1, false))) break;
                if (!(ok = warp_wait(ds_full, t & 1, &sh.loads))) break;
                mma_fence_after();
                if (elect_one()) {
                    const uint32_t acc = t_dk + 64 * set.at, b = at_q + slot.at * B::kTile;
                    product_tmem(acc, t_dp, t_dp + 64, b, id_acc, !first);
                    if (fine) product_tmem(acc, t_dp + 32, t_dp + 96, b, id_acc, true);
                    mma_commit<1>(q_empty + 8 * slot.at);
                    if (last) mma_commit<1>(acc_full + 8 * set.at);
                }
                __syncwarp();
                if (any && !(ok = rows(t + 1, true))) break;
                ++t;
            }
        } else if (warp == 10) {
            // statistics of the rows of queries: what the exponent subtracts, and delta
            uint32_t n = 0;
            while (ok && walk.next()) {
                const Work it = walk.it;
                const QuerySpan q = query_span(it, g.kt);
                if (!q.tiles) continue;
                Sigma<F16> sigma;
                sigma.fetch(g, it);
                const float unit = power2(sigma.get() - kLift<F16>);
                for (int i = 0; i < q.tiles; ++i, ++n) {
                    const Stat stage(n);
                    float l[4], d[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int row = 32 * x + lane, token = q.first + i * g.kt + row / g.group, head = walk.it.h * g.group + row % g.group;
                        const bool live = row < qrows && token < it.end;
                        const int64_t at = (int64_t)token * g.heads + head;
                        l[x] = live ? row_shift(g.lse[at], kLift<F16>) : -INFINITY;
                        d[x] = live ? -g.delta[at] * unit : 0.f;
                    }
                    if (!(ok = warp_wait(st_empty + 8 * stage.at, stage.parity ^ 1, &sh.loads))) break;
                    float* const to = stats + stage.at * 2 * kRows;
#pragma unroll
                    for (int x = 0; x < 4; ++x) to[32 * x + lane] = l[x], to[kRows + 32 * x + lane] = d[x];
                    bar_arrive(st_full + 8 * stage.at);
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int half = warp / 4, row = threadIdx.x % 128;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        uint32_t t = 0, items = 0;
        uint8_t* const stage = B::kStage ? smem + (kRing + 2 * B::kSlots) * B::kTile + B::kStats * 2 * kRows * 4 + warp * kStageBytesOfWarp : nullptr;
        // the item whose sums are still to be written: one half of the warps has dv, the other dk
        RowsOut out = {};
        float factor = 0.f;
        bool pending = false;
        auto write = [&](uint32_t item) {
            const Set set(item);
            if (!warp_wait(acc_full + 8 * set.at, set.parity, &sh.loads)) return false;
            mma_fence_after();
#pragma unroll 1
            for (int x = 0; x < 2 * HALVES; ++x) {
                if (32 * x >= g.dim) break;
                uint32_t a[32];
                tmem_fetch((half ? t_dk : t_dv) + 64 * set.at + 32 * x + lanes, a);
                tmem_wait(a);
                out.write<F16, WIDE>(32 * x, g.dim, a, factor, stage);
            }
            mma_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(acc_free + 8 * set.at);
            return true;
        };
        while (ok && walk.next()) {
            const Work it = walk.it;
            const int h = walk.it.h;
            const QuerySpan q = query_span(it, g.kt);
            const int token = it.first + row;
            const HeadsOut& o = half ? g.dk : g.dv;
            uint16_t* const own = token < it.end ? o.p + (int64_t)token * o.token + h * o.head : nullptr;
            if (it.begin < 0) {
                write_zeros(own, g.dim);
                continue;
            }
            Sigma<F16> raw;
            raw.fetch(g, it);
            const int sigma = raw.get();
            const Pair c2 = both(g.scale * kLog2e), s2 = both(power2(sigma - kLift<F16>));
            const bool fine = F16 && q.tiles <= kFineTiles;
            for (int i = 0; i < q.tiles; ++i, ++t) {
                const Stat step(t);
                const int first = q.first + i * g.kt;  // token of the tile's first row
                // the first column of this half that sees this key, the warp's first and its last key
                const int low = first_row(token - lane - first, g.group) - 64 * half, from = low + lane * g.group, high = low + 31 * g.group;
                const float* const st = stats + step.at * 2 * kRows + 64 * half;
                if (!(ok = warp_wait(st_full + 8 * step.at, step.parity, &sh.loads))) break;
                if (!(ok = warp_wait(s_full, t & 1, &sh.loads))) break;
                mma_fence_after();
                uint32_t s[2][32], dp[2][32], e[32], rest[32];
                tmem_fetch(tmem + 64 * half + lanes, s[0]), tmem_fetch(tmem + 64 * half + 32 + lanes, s[1]);
                tmem_wait(s[0]), tmem_wait(s[1]);
                auto probabilities = [&](int x) {
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 l = *reinterpret_cast<const float4*>(st + 32 * x + j);
                        const float2 a = split(fma2(pair(__uint_as_float(s[x][j]), __uint_as_float(s[x][j + 1])), c2, pair(l.x, l.y)));
                        const float2 b = split(fma2(pair(__uint_as_float(s[x][j + 2]), __uint_as_float(s[x][j + 3])), c2, pair(l.z, l.w)));
                        s[x][j] = __float_as_uint(exp2_of(a.x)), s[x][j + 1] = __float_as_uint(exp2_of(a.y));
                        s[x][j + 2] = __float_as_uint(exp2_of(b.x)), s[x][j + 3] = __float_as_uint(exp2_of(b.y));
                    }
                };
                if (high <= 0) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) probabilities(x);
                } else {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (low >= 32 * x + 32) {  // none of these queries sees any of the warp's keys
#pragma unroll
                            for (int j = 0; j < 32; ++j) s[x][j] = 0;
                            continue;
                        }
                        probabilities(x);
                        if (high <= 32 * x) continue;
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (32 * x + j < from) s[x][j] = 0;
                    }
                }
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int j = 0; j < 32; j += 2) e[16 * x + j / 2] = pack16<F16>(__uint_as_float(s[x][j]), __uint_as_float(s[x][j + 1]));
                tmem_store(tmem + 64 * half + lanes, e);
                tmem_store_wait();
                mma_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_full);
                if (!(ok = warp_wait(dp_full, t & 1, &sh.loads))) break;
                mma_fence_after();
                tmem_fetch(t_dp + 64 * half + lanes, dp[0]), tmem_fetch(t_dp + 64 * half + 32 + lanes, dp[1]);
                tmem_wait(dp[0]), tmem_wait(dp[1]);
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 d = *reinterpret_cast<const float4*>(st + kRows + 32 * x + j);
                        auto ds_at = [&](int i, float d0, float d1) {
                            const Pair y = pair(__uint_as_float(dp[x][i]), __uint_as_float(dp[x][i + 1])), d2 = pair(d0, d1);
                            return split(pair(__uint_as_float(s[x][i]), __uint_as_float(s[x][i + 1])) * (F16 ? fma2(y, s2, d2) : y + d2));
                        };
                        const float2 a = ds_at(j, d.x, d.y), b = ds_at(j + 2, d.z, d.w);
                        const float v[4] = {a.x, a.y, b.x, b.y};  // 0 where the probability is
                        e[16 * x + j / 2] = pack16<F16>(v[0], v[1]), e[16 * x + j / 2 + 1] = pack16<F16>(v[2], v[3]);
                        if (fine) {
                            const float2 a16 = __half22float2(*reinterpret_cast<const __half2*>(&e[16 * x + j / 2]));
                            const float2 b16 = __half22float2(*reinterpret_cast<const __half2*>(&e[16 * x + j / 2 + 1]));
                            rest[16 * x + j / 2] = pack16<true>(v[0] - a16.x, v[1] - a16.y);
                            rest[16 * x + j / 2 + 1] = pack16<true>(v[2] - b16.x, v[3] - b16.y);
                        }
                    }
                tmem_store(t_dp + 64 * half + lanes, e);
                if (fine) tmem_store(t_dp + 64 * half + 32 + lanes, rest);
                tmem_store_wait();
                mma_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(ds_full), bar_arrive(st_empty + 8 * step.at);
                if (i == 0 && pending) {
                    pending = false;
                    if (!(ok = write(items - 1))) break;
                }
            }
            if (!ok) break;
            out.set(own);
            factor = half ? g.scale * power2(-sigma) : power2(-kLift<F16>);
            pending = true;
            ++items;
        }
        if (ok && pending) ok = write(items - 1);
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
    int64_t most[2], slots;
    size_t at_start, at_prefix[2], at_items[2], at_delta, at_row_top, at_v_top, at_top, bytes;
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
    p.at_delta = take((size_t)tokens * heads * 4);
    p.slots = tokens < sequences ? tokens : sequences;
    p.at_row_top = take((size_t)tokens * heads * 2), p.at_v_top = take((size_t)tokens * kv * 2), p.at_top = take((size_t)p.slots * 2 * kv * 4);
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

template <int HALVES, bool F16, bool WIDE>
cudaError_t launch_back(const ones_heads& dout, const ones_heads& q, const ones_heads& k, const ones_heads& v, const SurveyArgs& d, BackArgs a,
                        const PlanArgs& plan, const BackPlan& p, cudaStream_t stream) {
    constexpr int kLanes = 8 * HALVES;
    CUtensorMap maps[4];
    cudaError_t err = make_heads_map(&maps[0], q, a.dim, a.tokens, a.group, a.kt, F16);
    if (err == cudaSuccess) err = make_heads_map(&maps[1], dout, a.dim, a.tokens, a.group, a.kt, F16);
    if (err == cudaSuccess) err = make_heads_map(&maps[2], k, a.dim, a.tokens, 1, kKeys, F16);
    if (err == cudaSuccess) err = make_heads_map(&maps[3], v, a.dim, a.tokens, 1, kKeys, F16);
    if (err == cudaSuccess) err = launch_plan(plan, 2, stream);
    if (err != cudaSuccess) return err;
    const int blocks = (a.tokens + kTokens - 1) / kTokens, most = 8 * device_sms(), grid = blocks < most ? blocks : most;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid), cfg.blockDim = dim3(256), cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr, cfg.numAttrs = 1;
    err = cudaLaunchKernelEx(&cfg, a.dim % 8 ? k_survey<F16, kLanes, true> : k_survey<F16, kLanes, false>, d);
    if (F16 && err == cudaSuccess) {
        const TopArgs t = {plan.items[1], plan.head + 1, d.row_top, d.v_top, const_cast<unsigned*>(a.top), a.heads, a.kv};
        const int64_t warps = (p.most[1] * a.kv + 7) / 8, slots = 8 * device_sms();
        err = launch_after(k_tops, dim3((unsigned)(warps < slots ? warps : slots)), dim3(256), stream, t);
    }
    if (err != cudaSuccess) return err;
    static std::atomic<uint64_t> ready[2];
    a.items = plan.items[0], a.head = plan.head;
    err = launch_pass(k_attention_queries<HALVES, F16, WIDE>, Back<HALVES>::kSmemQueries, ready[0], p.most[0] * a.kv, stream, maps, a);
    if (err != cudaSuccess) return err;
    a.items = plan.items[1], a.head = plan.head + 1;
    return launch_pass(k_attention_keys<HALVES, F16, WIDE>, Back<HALVES>::kSmemKeys, ready[1], p.most[1] * a.kv, stream, maps, a);
}

}  // namespace

const WaitControl attention_back_waits = {take_expired, limit_waits, wait_for_nothing};

}  // namespace ones

extern "C" {

int ones_attention_first_row(int behind, int group) { return ones::first_row(behind, group); }

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
    if (p.most[0] * k->heads >= 1ll << 31) return ONES_ERR_BAD_PARAM;
    if (workspace_bytes < p.bytes) return ONES_ERR_WORKSPACE;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    uint8_t* const ws = static_cast<uint8_t*>(d_workspace);
    PlanArgs plan = {};
    plan.offsets = d_offsets, plan.tokens = tokens, plan.sequences = sequences;
    plan.step[0] = p.kt, plan.tile[0] = kKeys, plan.step[1] = kKeys, plan.tile[1] = p.kt;
    plan.start = reinterpret_cast<int*>(ws + p.at_start), plan.head = reinterpret_cast<PlanHead*>(ws);
    for (int i = 0; i < 2; ++i)
        plan.prefix[i] = reinterpret_cast<int*>(ws + p.at_prefix[i]), plan.items[i] = reinterpret_cast<Item*>(ws + p.at_items[i]);
    unsigned* const top = reinterpret_cast<unsigned*>(ws + p.at_top);
    plan.zero = top, plan.zeros = type == ONES_F16 ? p.slots * 2 * k->heads : 0;
    uint16_t *const row_top = reinterpret_cast<uint16_t*>(ws + p.at_row_top), *const v_top = reinterpret_cast<uint16_t*>(ws + p.at_v_top);
    float* const delta = reinterpret_cast<float*>(ws + p.at_delta);
    auto vectors = [](const ones_heads& h) { return Vectors{static_cast<const uint16_t*>(h.d_data), h.token, h.head}; };
    SurveyArgs d = {vectors(*dout), vectors(*out), vectors(*v)};
    d.plan = plan.head, d.delta = delta, d.row_top = row_top, d.v_top = v_top, d.tokens = tokens, d.heads = q->heads, d.kv = k->heads, d.dim = dim;
    d.wide = aligned(out->d_data, 16) && (out->heads <= 1 || out->head % 8 == 0) && (tokens <= 1 || out->token % 8 == 0);
    const BackArgs a = {nullptr, nullptr, d_lse, delta, row_top, top, heads_out(*dq, dim, tokens), heads_out(*dk, dim, tokens), heads_out(*dv, dim, tokens), tokens,
                        q->heads, k->heads, p.group, p.kt, dim, scale};
    const bool f16 = type == ONES_F16;
    cudaError_t err;
    auto launch = [&](auto narrow) {
        constexpr int H = decltype(narrow)::value;
        if (a.dq.wide && a.dk.wide && a.dv.wide)
            return f16 ? launch_back<H, true, true>(*dout, *q, *k, *v, d, a, plan, p, stream) : launch_back<H, false, true>(*dout, *q, *k, *v, d, a, plan, p, stream);
        return f16 ? launch_back<H, true, false>(*dout, *q, *k, *v, d, a, plan, p, stream) : launch_back<H, false, false>(*dout, *q, *k, *v, d, a, plan, p, stream);
    };
    err = dim > 64 ? launch(std::integral_constant<int, 2>{}) : launch(std::integral_constant<int, 1>{});
    return err == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // extern "C"
