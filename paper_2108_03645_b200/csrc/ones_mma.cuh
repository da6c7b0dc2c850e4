// Thin wrappers of the sm_100a instructions that the training-step kernels use: mbarriers, tiled TMA loads and
// stores, the fifth-generation tensor core (tcgen05) and programmatic dependent launch.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace ones {

// Every wait ends: after this many nanoseconds without what it waits for, the waiter gives up, and does not wait again in
// its kernel. A translation unit has its own limit and its own flag, which kernels set when a wait has run out.
constexpr unsigned long long kWaitLimitNs = 4000000000ull;
static __device__ unsigned long long g_wait_limit = kWaitLimitNs;
static __device__ unsigned g_wait_expired;
constexpr uint64_t kShortWaitNs = 20000;  // the limit is not looked at before: that is an access to memory

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// One lane of the (converged) warp, always the same. TMA, tcgen05.mma and their barriers take their operands from uniform
// registers: when a whole warp runs a loop and only the instruction itself is given to one lane, the operands are
// computed there; a loop that one lane runs alone moves them over for every instruction (measured: 650 instead of 512
// cycles for the four products of a stage).
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void cluster_sync_all() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Address of the same shared-memory variable in the CTA `rank` of this cluster.
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

// ---- arithmetic on pairs ----
// Two 32-bit values that go through one instruction.
struct Pair {
    unsigned long long v;
};
__device__ __forceinline__ Pair pair(float lo, float hi) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ Pair both(float x) { return pair(x, x); }
__device__ __forceinline__ float2 split(Pair a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ float total(Pair a) {
    const float2 f = split(a);
    return f.x + f.y;
}

// ---- programmatic dependent launch ----
__device__ __forceinline__ void wait_for_predecessor() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_successor_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- mbarriers ----
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_init_done() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }

__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// `bar` is a shared::cluster address: the barrier may lie in another CTA of the cluster. Orders no memory accesses (those
// of tensor memory are ordered by the tcgen05 fences): a release would wait for every store on its way.
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// Waits for the phase of the given parity; false (and the flag set) when it has not come within the limit.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
    if (bar_try(bar, parity)) return true;
    const uint64_t begin = now_ns();
    while (!bar_try(bar, parity)) {
        const uint64_t waited = now_ns() - begin;
        if (waited > kShortWaitNs && waited > g_wait_limit) {
            atomicExch(&g_wait_expired, 1u);
            return false;
        }
    }
    return true;
}
// The same by a whole warp, with one answer for all of it: lanes may see the limit pass at different looks, and those that
// give up alone would be missing where the warp meets next.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, bar_wait(bar, parity)); }
// Waits that may span many steps of another warp of the block, which counts them in `steps` (shared memory): the limit is one for the
// time without a step, so that they end when that warp's own waits do.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, const volatile uint32_t* steps) {
    if (bar_try(bar, parity)) return true;
    uint64_t begin = now_ns();
    uint32_t seen = *steps;
    while (!bar_try(bar, parity)) {
        const uint64_t waited = now_ns() - begin;
        if (waited > kShortWaitNs && waited > g_wait_limit) {
            const uint32_t n = *steps;
            if (n == seen) {
                atomicExch(&g_wait_expired, 1u);
                return false;
            }
            seen = n, begin += waited;
        }
    }
    return true;
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const volatile uint32_t* steps) {
    return __all_sync(0xFFFFFFFFu, bar_wait(bar, parity, steps));
}
// The waits of a thread that comes by again and again: after one that ran out, a look is all. That is asked only where the
// first look has found nothing: asked before it, a pass over 8192 rows of 2048 takes 22.4 us instead of 22.1.
struct Waits {
    bool ok = true;
    __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) {
        if (bar_try(bar, parity)) return true;
        return ok = ok && bar_wait(bar, parity);
    }
};

// After a wait that ran out, copies and products may still be on their way: gives them time before their memory goes.
__device__ __forceinline__ void let_copies_end() {
    const uint64_t begin = now_ns();
    while (now_ns() - begin < 10000000ull) __nanosleep(1000);
}

// ---- between the blocks of a cooperative launch ----
// One thread counts its block in, after a barrier of all threads whose writes the others are to see.
__device__ __forceinline__ void arrive_all(unsigned* counter) {
    __threadfence();
    asm volatile("fence.proxy.async;" ::: "memory");  // the others read by TMA
    asm volatile("red.relaxed.gpu.global.add.u32 [%0], 1;" ::"l"(counter) : "memory");
}
// Waits (a whole warp) until the counter has reached `target`; false when that has not come within the limit.
__device__ __forceinline__ bool wait_all(const unsigned* counter, unsigned target) {
    bool ok = true;
    if (threadIdx.x % 32 == 0) {
        uint64_t begin = 0;
        for (;;) {
            unsigned v;
            asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(counter) : "memory");
            if ((int)(v - target) >= 0) break;
            const uint64_t now = now_ns();
            if (!begin) begin = now;
            if (now - begin > kShortWaitNs && now - begin > g_wait_limit) {
                atomicExch(&g_wait_expired, 1u);
                ok = false;
                break;
            }
        }
        __threadfence();  // once, not with every look at the counter
    }
    __syncwarp();
    ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
    asm volatile("fence.proxy.async;" ::: "memory");
    return ok;
}

// One warp that waits as a warp and then `times` times as threads for what nobody sends: shows that waits end, once for all,
// and that the flag is set.
static __global__ void k_wait_for_nothing(int times) {
    __shared__ __align__(8) uint64_t s_bar;
    if (threadIdx.x == 0) {
        bar_init(smem_u32(&s_bar), 1);
        bar_init_done();
    }
    __syncwarp();
    if (warp_wait(smem_u32(&s_bar), 0)) return;
    Waits wait;
    for (int i = 0; i < times; ++i) wait(smem_u32(&s_bar), 0);
}

// A translation unit's waits, seen from the host.
static inline cudaError_t take_expired(unsigned* out) {  // reads and clears the flag
    cudaError_t err = cudaMemcpyFromSymbol(out, g_wait_expired, sizeof(*out));
    const unsigned zero = 0;
    if (err == cudaSuccess && *out) err = cudaMemcpyToSymbol(g_wait_expired, &zero, sizeof(zero));
    return err;
}
static inline cudaError_t limit_waits(unsigned long long ns) {  // 0: the default
    if (!ns) ns = kWaitLimitNs;
    return cudaMemcpyToSymbol(g_wait_limit, &ns, sizeof(ns));
}
static inline cudaError_t wait_for_nothing(int times, cudaStream_t stream) {
    k_wait_for_nothing<<<1, 32, 0, stream>>>(times);
    return cudaGetLastError();
}
struct WaitControl {
    cudaError_t (*expired)(unsigned*);
    cudaError_t (*limit)(unsigned long long);
    cudaError_t (*nothing)(int, cudaStream_t);
};
extern const WaitControl norm_waits, loss_waits, update_waits;

// ---- TMA ----
// The map of a three-dimensional tensor of 16-bit values (strides in bytes) in boxes with the 128-byte swizzle.
cudaError_t encode_box(CUtensorMap* out, const void* p, const uint64_t (&dims)[3], const uint64_t (&strides)[2], const uint32_t (&box)[3], bool f16);

__device__ __forceinline__ void tma_prefetch(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// One box of a three-dimensional tensor into this CTA's shared memory; CG = 2: the bytes are counted on a barrier
// that may lie in the other CTA of the pair.
template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    if constexpr (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], "
            "[%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], "
            "[%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
}

// `bytes` (a multiple of 16, from and to 16-byte boundaries) into shared memory, counted on the barrier.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}

// ---- tcgen05 ----
template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t dst_smem, uint32_t cols) {
    if constexpr (CG == 2)
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(cols) : "memory");
    else
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(cols) : "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t cols) {
    if constexpr (CG == 2) {
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}

__device__ __forceinline__ void mma_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mma_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// D(tmem) (+)= A * B for 16-bit operands in shared memory and 32-bit accumulators; issued by one thread.
template <int CG>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    if constexpr (CG == 2)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
            : "memory");
}

// Arrives on the barrier (CG = 2: on the one at the same place in both CTAs of the pair) when all products that this
// thread issued before are done.
template <int CG>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (CG == 2)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
            "h"((uint16_t)3)
            : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// 16, 32 or 64 consecutive columns of the calling warp's 32 lanes (one row of the accumulator per thread).
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[16]) {
    uint32_t r[16];
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
          "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]),
          "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]),
          "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[64]) {
    uint32_t r[64];
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
        "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
        "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
          "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]),
          "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]),
          "=r"(r[29]), "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]),
          "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]), "=r"(r[41]), "=r"(r[42]),
          "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]),
          "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]), "=r"(r[56]),
          "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 64; ++i) v[i] = __uint_as_float(r[i]);
}

// Shared-memory descriptor of a 16-bit operand tile with the 128-byte swizzle.
//  K contiguous: rows of 64 values (128 bytes), groups of 8 rows 1024 bytes apart (the leading offset is not used).
//  MN contiguous: chunks of 64 values along MN, each with its K rows of 128 bytes one below the other: groups of
//  8 K rows 1024 bytes apart (stride), chunks `chunk_bytes` apart (leading).
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool mn, uint32_t chunk_bytes) {
    uint64_t d = (uint64_t)((addr & 0x3FFFF) >> 4);
    d |= (uint64_t)(mn ? (chunk_bytes >> 4) : 1u) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

}  // namespace ones
