// bsm_tc.h -- PTX wrappers shared by the kernels on the 5th-generation tensor
// cores: mbarriers with bounded waits, descriptors, tensor memory, programmatic
// launch.  Device code.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace bsm {

constexpr uint64_t kGemmWaitNs = 2000000000ull;     // bound of every wait below

__device__ __forceinline__ uint32_t saddr(const void *p)
{
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

__device__ __forceinline__ uint64_t gtimer()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// True in one lane of the (converged) warp, the same one every time.  The
// tensor-core and TMA instructions take their operands from uniform
// registers: issued under this election in a loop that the whole warp runs,
// they cost a few cycles each; issued by a lane that left the warp (lane == 0
// around the loop) about 250 (measured: 64 K blocks of a 256 x 256 tile,
// operands not even loaded, 36 us against 17 us of tensor time).
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xFFFFFFFF;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(p));
    return p != 0;
}

__device__ __forceinline__ void bar_init(uint64_t *b, uint32_t n)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(saddr(b)), "r"(n) : "memory");
}

__device__ __forceinline__ void bar_arrive(uint64_t *b)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(saddr(b)) : "memory");
}

__device__ __forceinline__ void bar_expect(uint64_t *b, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(saddr(b)), "r"(bytes)
                 : "memory");
}

__device__ __forceinline__ bool bar_try(uint64_t *b, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(saddr(b)), "r"(parity), "r"(50000u)
        : "memory");
    return ok != 0;
}

// Bounded wait for the phase of `parity`; false on abort or time out.
static __device__ __noinline__ bool bar_wait(uint64_t *b, uint32_t parity, const volatile int32_t *abort)
{
    if (bar_try(b, parity))
        return true;
    const uint64_t t0 = gtimer();
    for (uint32_t it = 0; it < (1u << 28); ++it) {
        if (bar_try(b, parity))
            return true;
        if (abort && *abort)
            return false;
        if (gtimer() - t0 > kGemmWaitNs)
            return false;
    }
    return false;
}

// The same wait inline and without the suspend hint, the clock read once in
// 256 tries: for the waits on a stage, of which there is one per K block.
__device__ __forceinline__ bool bar_spin(uint64_t *b, uint32_t parity, const volatile int32_t *abort)
{
    const uint32_t addr = saddr(b);
    uint64_t t0 = 0;
    for (uint32_t it = 0; it < (1u << 28); ++it) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(addr), "r"(parity)
            : "memory");
        if (ok)
            return true;
        if ((it & 255u) == 255u) {
            const uint64_t t = gtimer();
            t0 = t0 ? t0 : t;
            if (*abort || t - t0 > kGemmWaitNs)
                return false;
        }
    }
    return false;
}

// A place in the stage ring and the phase it is in, stepped instead of divided
// out of a running count (a division per K block is a chain of about 150
// cycles in the one warp that feeds the tensor cores).
struct RingPos {
    int s = 0;
    uint32_t ph = 0;
    __device__ __forceinline__ void step(int S)
    {
        if (++s == S) {
            s = 0;
            ph ^= 1u;
        }
    }
};

// Shared-memory matrix descriptor of a K-major operand tile whose rows are
// 128 bytes (64 bf16) laid out with the 128-byte swizzle by TMA: start
// address (16-byte units), leading-dimension offset (unused for this
// layout: 1), stride between 8-row groups = 1024 bytes, descriptor version 1,
// base offset 0 (tiles are 1024-byte aligned), swizzle mode 2 = 128 bytes.
__device__ __forceinline__ uint64_t smem_desc(const void *tile)
{
    const uint64_t a = (saddr(tile) & 0x3FFFFu) >> 4;
    return a | (1ull << 16) | (uint64_t(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// Arrive once on `bar` when every tcgen05.mma issued so far by this thread is done.
__device__ __forceinline__ void mma_commit(uint64_t *bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(saddr(bar))
                 : "memory");
}

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 consecutive fp32 columns of this thread's TMEM lane (no wait).
__device__ __forceinline__ void tmem_ld32_nowait(uint32_t taddr, uint32_t *r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
        "%14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}

__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Programmatic dependent launch: the kernel may start while the previous
// kernel of the stream is finishing; this waits until that kernel has
// completed and its writes are visible (a no-op without such a predecessor).
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Let the next kernel of the stream start its launch (it still waits on its own
// grid_dependency_wait before touching memory).
__device__ __forceinline__ void grid_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace bsm
