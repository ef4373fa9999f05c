// The matrix unit of sm_100a by hand: operands in shared memory without a swizzle, sums in tensor memory, copies in bulk, barriers
// whose waits end.
#pragma once

#include <stdint.h>

namespace kvp {

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- barriers in shared memory ----
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t arrivals) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(arrivals) : "memory"); }
__device__ __forceinline__ void barrier_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void barrier_arrive_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// has the phase of `parity` ended?
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Waits for the end of the phase of `parity`, two seconds at most; false if it did not come, or if another waiter of the CTA gave up before. Of the time between two
// looks a millisecond counts at most: a GPU that was given to another process meanwhile has not kept anyone waiting.
static __device__ __noinline__ bool barrier_wait_long(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up)
{
    uint64_t last, now, waited = 0;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(last));
    while (true) {
        for (int i = 0; i < 256; ++i) {
            if (barrier_try(bar, parity)) return true;
            __nanosleep(20);                                           // others have work for the issue slots
        }
        if (*gave_up) return false;
        asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
        waited += now - last < 1000000ull ? now - last : 1000000ull;
        last = now;
        if (waited > 2000000000ull) {
            *gave_up = 1;
            return false;
        }
    }
}
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up)
{
    return barrier_try(bar, parity) || barrier_wait_long(bar, parity, gave_up);
}

// `bytes` (a multiple of 16) from global to shared memory, both 16-byte aligned; counted at the barrier
__device__ __forceinline__ void copy_bulk(uint32_t to, const void* from, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}
// what threads wrote to shared memory is seen by the matrix unit and by copies
__device__ __forceinline__ void show_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor memory: 128 lanes x 512 columns of 32 bits ----
template <uint32_t COLUMNS>
__device__ __forceinline__ void tensor_alloc(uint32_t to)          // a whole warp
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "n"(COLUMNS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
template <uint32_t COLUMNS>
__device__ __forceinline__ void tensor_free(uint32_t at)           // the same warp
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "n"(COLUMNS));
}
__device__ __forceinline__ void tensor_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tensor_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// the numbers of a load are not used before here (the compiler knows no other order between a load's registers and the wait)
template <int N>
__device__ __forceinline__ void tensor_hold(float (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+f"(x[i]));
}
// four or eight columns of this thread's lane (warp w of a team of four has lanes 32 w .. 32 w + 31)
__device__ __forceinline__ void tensor_load(uint32_t at, float (&x)[4])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]) : "r"(at));
}
__device__ __forceinline__ void tensor_load(uint32_t at, float (&x)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "r"(at));
}
__device__ __forceinline__ void tensor_store(uint32_t at, const float (&x)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]),
                 "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
}

// ---- products ----
// An operand in shared memory whose k lies contiguous, in cores of 8 rows x 16 bytes (128 bytes, rows one behind the other):
// `along_k` bytes from a core to the next one in k, `along_rows` to the next eight rows; all multiples of 16.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t along_k, uint32_t along_rows)
{
    return (uint64_t)(at >> 4) | (uint64_t)(along_k >> 4) << 16 | (uint64_t)(along_rows >> 4) << 32 | 1ull << 46;
}
// The right operand may have its columns contiguous instead: cores of 16 columns x 8 in k, `along_k` to the next eight in k, `along_rows` to the next 16 columns.
constexpr uint32_t kColumnsContiguous = 1u << 16;
// sums in fp32 of e4m3 times e4m3, 128 rows x `columns` (a multiple of 16, at most 256)
__host__ __device__ constexpr uint32_t shape_e4m3(uint32_t columns) { return 1u << 4 | (columns / 8) << 17 | (128u / 16) << 24; }
// sums [128 lanes][columns] (+)= a [128][32 in k] b [columns][32 in k]^T; one thread
__device__ __forceinline__ void multiply_e4m3(uint32_t sums, uint64_t a, uint64_t b, uint32_t shape, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(sums), "l"(a), "l"(b),
                 "r"(shape), "r"((uint32_t)add) : "memory");
}
// the barrier gets an arrival when all products issued by this thread so far are done
__device__ __forceinline__ void products_arrive(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

}  // namespace kvp
