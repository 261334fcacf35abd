// Tensor-memory, asynchronous-copy and barrier instructions of sm_103a as inline PTX, and the
// host side of tensor maps.  Used by the attention kernels (cr_attn.cu).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

__device__ __forceinline__ uint32_t cr_smem(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- mbarriers -----------------------------------------------------------------------------
__device__ __forceinline__ void cr_bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void cr_bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cr_bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool cr_bar_try(uint32_t bar, uint32_t parity)
{
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

// Wait for a phase with a limit: after two seconds (or once another warp of the CTA has given
// up) the wait returns false and the caller leaves its role.
__device__ __forceinline__ bool cr_bar_wait(uint32_t bar, uint32_t parity, volatile int *gave_up)
{
    if (cr_bar_try(bar, parity)) return true;
    unsigned long long t0 = 0, t;
    for (uint32_t i = 1;; ++i) {
        if (cr_bar_try(bar, parity)) return true;
        if ((i & 63u) == 0) {
            if (*gave_up) return false;
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            if (t0 == 0) t0 = t;
            if (t - t0 > 2000000000ull) {
                *gave_up = 1;
                return false;
            }
        }
    }
}

// Writes of this thread to shared memory become visible to the asynchronous proxy (copies, tcgen05).
__device__ __forceinline__ void cr_fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor copies -------------------------------------------------------------------------
__device__ __forceinline__ void cr_tma_load(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z, int w)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}
__device__ __forceinline__ void cr_tma_prefetch_map(const CUtensorMap *map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// ---- tensor memory and the fifth-generation tensor core ---------------------------------------
__device__ __forceinline__ void cr_tmem_alloc(uint32_t smem_dst, uint32_t cols)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void cr_tmem_free(uint32_t tmem, uint32_t cols)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));
}
__device__ __forceinline__ void cr_tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void cr_tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Products and commits are issued by one thread of a warp that runs the surrounding code as a whole: so the
// operands' descriptors stay in uniform registers (issued from a branch of one lane, every product waits for
// its descriptors to be moved there, and the tensor cores for the products).
__device__ __forceinline__ uint32_t cr_elect()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r;
}
// The barrier gets one arrival when every tcgen05 operation the elected thread issued before has finished.
__device__ __forceinline__ void cr_tc_commit(uint32_t bar, uint32_t elected)
{
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
        ::"r"(bar), "r"(elected)
        : "memory");
}
// D += A B (acc = 0: D = A B), A and B through shared-memory descriptors
__device__ __forceinline__ void cr_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t elected)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(elected)
        : "memory");
}
// the same with A in tensor memory
__device__ __forceinline__ void cr_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t elected)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc), "r"(elected)
        : "memory");
}

// Instruction descriptor of kind::f16: fp32 accumulators, both operands of one 16-bit type,
// A with its contraction index contiguous; b_mn: B with its other index contiguous.
__host__ __device__ constexpr uint32_t cr_idesc(bool bf16, int m, int n, bool b_mn)
{
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// Shared-memory descriptor of an operand in 128-byte swizzled rows: `stride` between groups of
// eight rows, `lead` between 64-element column blocks (read only where the contiguous index is
// not the contraction's).
__device__ __forceinline__ uint64_t cr_sdesc(uint32_t addr, uint32_t lead, uint32_t stride)
{
    return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(stride >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}

#define CR_LD32(a, o)                                                                                              \
    "=r"((a)[(o) + 0]), "=r"((a)[(o) + 1]), "=r"((a)[(o) + 2]), "=r"((a)[(o) + 3]), "=r"((a)[(o) + 4]),            \
        "=r"((a)[(o) + 5]), "=r"((a)[(o) + 6]), "=r"((a)[(o) + 7]), "=r"((a)[(o) + 8]), "=r"((a)[(o) + 9]),        \
        "=r"((a)[(o) + 10]), "=r"((a)[(o) + 11]), "=r"((a)[(o) + 12]), "=r"((a)[(o) + 13]), "=r"((a)[(o) + 14]),   \
        "=r"((a)[(o) + 15]), "=r"((a)[(o) + 16]), "=r"((a)[(o) + 17]), "=r"((a)[(o) + 18]), "=r"((a)[(o) + 19]),   \
        "=r"((a)[(o) + 20]), "=r"((a)[(o) + 21]), "=r"((a)[(o) + 22]), "=r"((a)[(o) + 23]), "=r"((a)[(o) + 24]),   \
        "=r"((a)[(o) + 25]), "=r"((a)[(o) + 26]), "=r"((a)[(o) + 27]), "=r"((a)[(o) + 28]), "=r"((a)[(o) + 29]),   \
        "=r"((a)[(o) + 30]), "=r"((a)[(o) + 31])
// 32 consecutive columns of the calling thread's lane of tensor memory (warp-collective)
__device__ __forceinline__ void cr_tmem_ld(uint32_t addr, uint32_t *v)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : CR_LD32(v, 0)
        : "r"(addr));
}
#define CR_LD16(a)                                                                                                 \
    "=r"((a)[0]), "=r"((a)[1]), "=r"((a)[2]), "=r"((a)[3]), "=r"((a)[4]), "=r"((a)[5]), "=r"((a)[6]),              \
        "=r"((a)[7]), "=r"((a)[8]), "=r"((a)[9]), "=r"((a)[10]), "=r"((a)[11]), "=r"((a)[12]), "=r"((a)[13]),      \
        "=r"((a)[14]), "=r"((a)[15])
#define CR_ST16(a)                                                                                                 \
    "r"((a)[0]), "r"((a)[1]), "r"((a)[2]), "r"((a)[3]), "r"((a)[4]), "r"((a)[5]), "r"((a)[6]), "r"((a)[7]),        \
        "r"((a)[8]), "r"((a)[9]), "r"((a)[10]), "r"((a)[11]), "r"((a)[12]), "r"((a)[13]), "r"((a)[14]), "r"((a)[15])
__device__ __forceinline__ void cr_tmem_ld16(uint32_t addr, uint32_t *v)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : CR_LD16(v)
        : "r"(addr));
}
__device__ __forceinline__ void cr_tmem_st16(uint32_t addr, const uint32_t *v)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::CR_ST16(v), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void cr_tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void cr_tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 bytes, aligned so
__device__ __forceinline__ void cr_store32(void *p, const uint32_t *v)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]),
                 "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}

// ---- arithmetic ----------------------------------------------------------------------------
__device__ __forceinline__ float cr_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float cr_max3(float a, float b, float c)
{
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ unsigned long long cr_pair(float x, float y)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void cr_unpair(unsigned long long v, float &x, float &y)
{
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v));
}
__device__ __forceinline__ unsigned long long cr_fma2(unsigned long long a, unsigned long long b, unsigned long long c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ unsigned long long cr_add2(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// two floats rounded to the 16-bit type, the first in the low half
template <bool BF16>
__device__ __forceinline__ uint32_t cr_pack16(float lo, float hi)
{
    uint32_t r;
    if (BF16)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
