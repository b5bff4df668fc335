// tcgen05.cuh — inline PTX of the 5th-generation tensor cores: tensor memory,
// shared-memory operand descriptors, MMA issue and completion.
#pragma once

#include "common.cuh"

namespace kvg {

// CTAS: 1, or 2 for the pair of CTAs of a cluster that work on one tile (all of
// a kernel's tensor-core instructions name the same).

// ------------------------------------------------------------ tensor memory --
// Whole warps (of both CTAs): columns (a power of two >= 32) of the SM's tensor
// memory; the address is written to shared memory.
template <int COLS, int CTAS>
__device__ __forceinline__ void tmem_alloc(uint32_t *dst) {
    if constexpr (CTAS == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(dst)), "n"(COLS)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(dst)), "n"(COLS)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
}
template <int COLS, int CTAS>
__device__ __forceinline__ void tmem_free(uint32_t addr) {
    if constexpr (CTAS == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "n"(COLS));
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "n"(COLS));
}

__device__ __forceinline__ void tc_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 consecutive columns of the thread's lane (a warp reads the 32 lanes of
// its quarter), to or from registers r[0, 32).
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
// 16 lanes x 32 columns from addr on: r[4 i + 2 e + c] is row lane / 4 + 8 e, column 8 i + 2 (lane % 4) + c.
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}

// --------------------------------------------------------------------- MMA --
// True in one thread of the (converged) warp.  What it guards stays uniform for
// the compiler: behind `lane == 0` the same 32 MMAs took 72 to 74 cycles each to
// issue beside busy warps, behind this 64, the tensor cores' own time.
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// Shared-memory operand in the 128-byte swizzle (atoms of 8 rows x 128 bytes,
// base 1024-byte aligned, 1024 bytes from one atom to the next along the rows:
// along m or n for a K-major operand, along k for an MN-major one).  `lead`:
// bytes between groups of 64 16-bit elements along m or n (MN-major).  Of the
// descriptor only the low word varies; a step of x bytes adds x / 16 to it, so
// that the issuing thread spends one addition per operand.
__device__ __forceinline__ uint32_t smem_desc(uint32_t addr, uint32_t lead) {
    return (addr & 0x3ffff) >> 4 | (lead >> 4) << 16;
}
constexpr uint32_t kDescHigh = (1024 >> 4) | 1u << 14 | 2u << 29;  // stride, version, swizzle

// Instruction descriptor of kind::f16: bf16 (or f16) operands, fp32 accumulator,
// A K-major; `negate` takes -A.
constexpr uint32_t mma_desc(int m, int n, bool f16, bool b_mn_major) {
    return 1u << 4 | (f16 ? 0u : 1u) << 7 | (f16 ? 0u : 1u) << 10 | (b_mn_major ? 1u : 0u) << 16 |
           (uint32_t)(n / 8) << 17 | (uint32_t)(m / 16) << 24;
}
constexpr uint32_t kMmaNegateA = 1u << 13;

// One thread (of a pair's first CTA): D[tmem] (+)= A . B, k = 16; a, b: low
// words of the descriptors.  A pair's A and D rows are split over the CTAs (half
// of m each), its B over them along n; the addresses are the same in both.
#define KVG_MMA_SS(GROUP)                                                                                          \
    asm volatile(                                                                                                  \
        "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 x, {%1, %5};\n\t"                \
        "mov.b64 y, {%2, %5};\n\ttcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d),     \
        "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "n"(kDescHigh)                                      \
        : "memory")
#define KVG_MMA_TS(GROUP)                                                                                          \
    asm volatile(                                                                                                  \
        "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 y, {%2, %5};\n\t"                   \
        "tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d),                          \
        "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "n"(kDescHigh)                                      \
        : "memory")
template <int CTAS>
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate) {
    if constexpr (CTAS == 1)
        KVG_MMA_SS("1");
    else
        KVG_MMA_SS("2");
}
// A in tensor memory (two 16-bit elements a column).
template <int CTAS>
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate) {
    if constexpr (CTAS == 1)
        KVG_MMA_TS("1");
    else
        KVG_MMA_TS("2");
}
#undef KVG_MMA_SS
#undef KVG_MMA_TS
// One thread: `bar` (of both CTAs of a pair) gets an arrival once its MMAs so
// far have completed.
template <int CTAS>
__device__ __forceinline__ void mma_commit(uint64_t *bar) {
    if constexpr (CTAS == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar))
                     : "memory");
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                smem_addr(bar)),
            "h"((uint16_t)3)
            : "memory");
}

// ----------------------------------------------------------------- cluster --
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
// What CTA `cta` of the cluster has at the place of p in its shared memory.
__device__ __forceinline__ int load_of_cta(const int *p, int cta) {
    int v;
    asm volatile(
        "{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.b32 %0, [a];\n\t}"
        : "=r"(v)
        : "r"(smem_addr(p)), "r"(cta)
        : "memory");
    return v;
}
// All threads of the cluster's CTAs; orders their shared-memory accesses.
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// An arrival on the barrier at the same place in the cluster's first CTA.  What
// it hands over lies in this SM's own memories, where the pair's products read
// it: tensor-memory stores that have been waited for, shared-memory writes behind
// fence.proxy.async, copies that have landed.  So it needs no fence of the
// cluster's scope (with .release.cluster each arrival took 1,200 cycles, which
// made it what a tile waited for).
__device__ __forceinline__ void mbar_arrive_first(uint64_t *bar) {
    asm volatile(
        "{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, 0;\n\t"
        "mbarrier.arrive.shared::cluster.b64 _, [a];\n\t}" ::"r"(smem_addr(bar))
        : "memory");
}

// ------------------------------------------------------- work of other CTAs --
// One thread: asks for a CTA (a cluster) of the grid that has not started, to do
// its work instead; the answer, 16 bytes, lands at `answer` and completes 16
// bytes on `bar` (of every CTA of a cluster).  Not to be asked again after a no.
template <int CTAS>
__device__ __forceinline__ void ask_for_cta(uint4 *answer, uint64_t *bar) {
    if constexpr (CTAS == 1)
        asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                         smem_addr(answer)),
                     "r"(smem_addr(bar))
                     : "memory");
    else
        asm volatile(
            "clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.multicast::cluster::all.b128 "
            "[%0], [%1];" ::"r"(smem_addr(answer)),
            "r"(smem_addr(bar))
            : "memory");
}
// The x index of that CTA (the cluster's first), or -1.
__device__ __forceinline__ int answered_cta(const uint4 *answer) {
    uint32_t x = 0, yes;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b128 a;\n\tld.shared.b128 a, [%2];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n\tselp.u32 %1, 1, 0, p;\n\tmov.u32 %0, 0;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, a;\n\t}"
        : "=r"(x), "=r"(yes)
        : "r"(smem_addr(answer))
        : "memory");
    return yes ? (int)x : -1;
}

// ---------------------------------------------------- packed fp32 and exp2 --
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "mul.rn.f32x2 w, x, y;\n\tmov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "add.rn.f32x2 w, x, y;\n\tmov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

}  // namespace kvg
