// Device helpers of the worker step's kernels: asynchronous copies, barriers, matrix
// fragments, prefix sums over the requests.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "worker.h"

namespace aladdin {
namespace wk {

__device__ __forceinline__ uint32_t smem_addr(const void* p)
{
    return (uint32_t)__cvta_generic_to_shared(p);
}

// 16 bytes from global to shared memory; zeros where !ok (src is not read).
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool ok)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0)
                 : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool ok)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(ok ? 4 : 0)
                 : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Barriers in shared memory that count arrivals and bytes, by address.
__device__ __forceinline__ void mbar_init(uint32_t bar, int count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
// Makes this thread's barriers visible to copies.
__device__ __forceinline__ void mbar_init_fence()
{
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Whether the phase of that parity has come.
__device__ __forceinline__ bool mbar_test(uint32_t bar, unsigned parity)
{
    unsigned done;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done;
}
// Waits for the phase of that parity; false where it did not come within a second.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, unsigned parity)
{
    unsigned long long end = 0;
    for (unsigned it = 0;; ++it) {
        unsigned done;
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}"
            : "=r"(done)
            : "r"(bar), "r"(parity), "r"(20000)  // nanoseconds that the thread may sleep
            : "memory");
        if (done) return true;
        if ((it & 63) == 63) {
            unsigned long long now;
            asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
            if (!end) end = now + 1000000000ull;
            else if (now > end) return mbar_test(bar, parity);  // (the thread may have been off for longer)
        }
    }
}
// Orders this thread's plain accesses to shared memory before later copies by the
// asynchronous proxy.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}

// The 8 x 8 matrix of 16-bit values whose row g, columns 2t and 2t + 1 lane
// 4 g + t holds, transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// 2^x; -inf gives 0.
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

template <typename T>
struct Num;
template <>
struct Num<__nv_bfloat16> {
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<uint32_t*>(&v);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t u)
    {
        return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
    }
    // whether one of the two values is infinite or NaN
    static __device__ __forceinline__ bool wild(uint32_t u)
    {
        return (u & 0x7f80u) == 0x7f80u || (u & 0x7f800000u) == 0x7f800000u;
    }
    // 0 in the place of those
    static __device__ __forceinline__ uint32_t tame(uint32_t u)
    {
        if ((u & 0x7f80u) == 0x7f80u) u &= 0xffff0000u;
        return (u & 0x7f800000u) == 0x7f800000u ? u & 0xffffu : u;
    }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                               uint32_t b1)
    {
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
            "{%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
template <>
struct Num<__half> {
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<uint32_t*>(&v);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t u)
    {
        return __half22float2(*reinterpret_cast<__half2*>(&u));
    }
    static __device__ __forceinline__ bool wild(uint32_t u)
    {
        return (u & 0x7c00u) == 0x7c00u || (u & 0x7c000000u) == 0x7c000000u;
    }
    static __device__ __forceinline__ uint32_t tame(uint32_t u)
    {
        if ((u & 0x7c00u) == 0x7c00u) u &= 0xffff0000u;
        return (u & 0x7c000000u) == 0x7c000000u ? u & 0xffffu : u;
    }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                               uint32_t b1)
    {
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
            "{%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};

// pre[r] = tiles of the requests before r, pre[n] = all; the block's threads
// together. tiles(r) is called once a request. Returns pre[n], or -1 (pre
// undefined) where it does not fit an int. scratch: 32 long longs.
template <int NT, typename F>
__device__ __forceinline__ int plan_prefix(int n, int* pre, long long* scratch, F tiles)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long base = 0;
    for (int r0 = 0; r0 < n; r0 += NT) {
        const int r = r0 + tid;
        const long long mine = r < n ? tiles(r) : 0;
        long long v = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        if (lane == 31) scratch[warp] = v;
        __syncthreads();
        long long before = base, all = base;
#pragma unroll
        for (int w = 0; w < NT / 32; ++w) {
            if (w < warp) before += scratch[w];
            all += scratch[w];
        }
        if (r < n) pre[r] = (int)(before + v - mine);
        base = all;
        __syncthreads();
    }
    if (base > 0x7fffffffll) return -1;
    if (tid == 0) pre[n] = (int)base;
    __syncthreads();
    return (int)base;
}

// The request that tile x (< pre[n]) belongs to.
__device__ __forceinline__ int plan_find(const int* pre, int n, int x)
{
    int lo = 0, hi = n;  // pre[lo] <= x < pre[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pre[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

}  // namespace wk
}  // namespace aladdin
