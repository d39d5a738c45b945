// What the tensor-core kernels of the replica operators share: barriers in shared memory with bounded waits, the order
// between threads and tensor memory, operand descriptors.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace grawa {
namespace replica {

__device__ __forceinline__ unsigned smem_address(const void* p) { return static_cast<unsigned>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ unsigned long long nanoseconds()
{
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ void barrier_init(unsigned bar, unsigned count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_expect(unsigned bar, unsigned bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// PAIR: arrivals may come from the other CTA of a pair (a wider acquire, which takes longer).
template <bool PAIR>
__device__ __forceinline__ bool barrier_try(unsigned bar, unsigned parity)
{
    unsigned ok;
    if constexpr (PAIR)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
    return ok != 0;
}
// False when the limit passed, or another wait of the CTA gave up (`gave_up`, which may be NULL).  Lanes of a warp may get
// different answers.  `timeouts`: the device's count of waits that ran out.
template <unsigned long long LIMIT, bool PAIR>
__device__ __forceinline__ bool bounded_wait(unsigned bar, unsigned parity, volatile int* gave_up, unsigned* timeouts)
{
    if (barrier_try<PAIR>(bar, parity)) return true;
    const unsigned long long t0 = nanoseconds();
    for (;;) {
        if (barrier_try<PAIR>(bar, parity)) return true;
        if (gave_up && *gave_up) return false;
        if (nanoseconds() - t0 > LIMIT) {
            if (gave_up) *gave_up = 1;
            atomicAdd(timeouts, 1u);
            return false;
        }
    }
}
__device__ __forceinline__ void order_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void order_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Shared-memory matrix descriptor, 128-byte swizzle.  K-major: groups of 8 rows 1024 bytes apart.
// MN-major: blocks of 64 elements `lead` bytes apart, groups of 8 k 1024 bytes apart.
__device__ __forceinline__ unsigned long long matrix_descriptor(unsigned address, unsigned lead)
{
    return static_cast<unsigned long long>((address & 0x3ffff) >> 4) | static_cast<unsigned long long>(lead >> 4) << 16 |
           static_cast<unsigned long long>(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
template <typename T> struct TypeCode;      // of both operands, in the instruction descriptor
template <> struct TypeCode<__half> { static constexpr unsigned value = 0; };
template <> struct TypeCode<__nv_bfloat16> { static constexpr unsigned value = 1; };

}  // namespace replica
}  // namespace grawa
