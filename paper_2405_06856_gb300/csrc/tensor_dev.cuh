// Tensor memory and the fifth-generation tensor cores: what the kernels of many rows share.
#pragma once

#include "worker_dev.cuh"

namespace aladdin {
namespace wk {

__device__ __forceinline__ void tmem_alloc(uint32_t where, int cols)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t at, int cols)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(cols));
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// The barrier counts one arrival when all products issued so far are done.
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar)
                 : "memory");
}
// A descriptor by its two halves: the lower holds the address.
__device__ __forceinline__ uint64_t whole(uint32_t lo, uint32_t hi) { return (uint64_t)hi << 32 | lo; }
__device__ __forceinline__ bool elected()
{
    uint32_t is;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(is));
    return is;
}
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t inst, bool add)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
                 "l"(a), "l"(b), "r"(inst), "r"((uint32_t)add)
                 : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t inst, bool add)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
                 "r"(a), "l"(b), "r"(inst), "r"((uint32_t)add)
                 : "memory");
}
#define ALADDIN_R8(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7])
#define ALADDIN_I8(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
// 32 columns of this thread's lane: starts the load; tmem_loaded makes its registers valid.
__device__ __forceinline__ void tmem_start(uint32_t (&v)[32], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, "
                 "%13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, "
                 "[%32];"
                 : ALADDIN_R8(v, 0), ALADDIN_R8(v, 8), ALADDIN_R8(v, 16), ALADDIN_R8(v, 24)
                 : "r"(at)
                 : "memory");
}
#define ALADDIN_U8(v, i) "+r"(v[i]), "+r"(v[i + 1]), "+r"(v[i + 2]), "+r"(v[i + 3]), "+r"(v[i + 4]), "+r"(v[i + 5]), "+r"(v[i + 6]), "+r"(v[i + 7])
__device__ __forceinline__ void tmem_loaded(uint32_t (&v)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : ALADDIN_U8(v, 0), ALADDIN_U8(v, 8), ALADDIN_U8(v, 16), ALADDIN_U8(v, 24)::"memory");
}
__device__ __forceinline__ void tmem_load(uint32_t (&v)[32], uint32_t at)
{
    tmem_start(v, at);
    tmem_loaded(v);
}
// 16 columns, at once.
__device__ __forceinline__ void tmem_load16(uint32_t (&v)[16], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, "
                 "%13, %14, %15}, [%16];\n tcgen05.wait::ld.sync.aligned;"
                 : ALADDIN_R8(v, 0), ALADDIN_R8(v, 8)
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tmem_store32(uint32_t at, const uint32_t (&v)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, "
                 "%13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
                 "%32};" ::"r"(at),
                 ALADDIN_I8(v, 0), ALADDIN_I8(v, 8), ALADDIN_I8(v, 16), ALADDIN_I8(v, 24)
                 : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&v)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, "
                 "%13, %14, %15, %16};" ::"r"(at),
                 ALADDIN_I8(v, 0), ALADDIN_I8(v, 8)
                 : "memory");
}
__device__ __forceinline__ void tmem_store8(uint32_t at, const uint32_t (&v)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at),
                 ALADDIN_I8(v, 0)
                 : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Descriptor of an operand in shared memory: rows of 128 bytes (64 values), the
// 16-byte pieces of a row exchanged by the row's place among eight; blocks of eight
// rows follow one another. `next` is the distance of the next 64 values: of the
// columns of an operand whose rows are its other index (values), unused else.
__device__ __forceinline__ uint32_t operand_lo(uint32_t addr, uint32_t next)
{
    return (addr & 0x3ffff) >> 4 | (next >> 4) << 16;
}
constexpr uint32_t OPERAND_HI = (1024 >> 4) | 1u << 14 | 2u << 29;

// Shape and types of a product: 128 rows, n columns, 32-bit sums; turned: the second
// operand's rows are the index that is summed over.
template <typename T>
__device__ __forceinline__ constexpr uint32_t product(int n, bool turned)
{
    const uint32_t type = std::is_same<T, __half>::value ? 0 : 1;
    return 1u << 4 | type << 7 | type << 10 | (turned ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (128u >> 4) << 24;
}

}  // namespace wk
}  // namespace aladdin
