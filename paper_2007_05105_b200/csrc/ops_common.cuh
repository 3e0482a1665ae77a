#pragma once
// Shared by the language-model operators (ops_embed.cu, ops_distill.cu, ops_norm.cu): element types,
// 16-byte accesses, launches and argument checks.  The operators' C ABI is include/adascale_ops.h.
#include "../../include/adascale_ops.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>

namespace {

typedef __nv_bfloat16 bf16;

constexpr long long kMaxRows = ADASCALE_OPS_MAX_ROWS;

// ---- element types -------------------------------------------------------------------------

template <int DT> struct ElemOf;
template <> struct ElemOf<ADASCALE_F32> { typedef float type; };
template <> struct ElemOf<ADASCALE_BF16> { typedef bf16 type; };

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float *p, float x) { *p = x; }
__device__ __forceinline__ void put(bf16 *p, float x) { *p = __float2bfloat16_rn(x); }

// The two bf16 values of a 32-bit word, widened (exact).
__device__ __forceinline__ float bf_lo(unsigned w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(unsigned w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ unsigned bf_pack(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned *>(&v);
}

// V adjacent elements as 32-bit floats; V > 1 wants the address aligned to the smaller of V
// elements and 16 bytes.
template <int V> __device__ __forceinline__ void load_vec(const float *p, float (&x)[V])
{
    if constexpr (V == 1) {
        x[0] = *p;
    } else {
        static_assert(V % 4 == 0, "whole 16-byte accesses");
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const float4 q = reinterpret_cast<const float4 *>(p)[i];
            x[4 * i] = q.x;
            x[4 * i + 1] = q.y;
            x[4 * i + 2] = q.z;
            x[4 * i + 3] = q.w;
        }
    }
}
template <int V> __device__ __forceinline__ void load_vec(const bf16 *p, float (&x)[V])
{
    if constexpr (V == 1) {
        x[0] = to_f32(*p);
    } else if constexpr (V == 4) {
        const uint2 q = *reinterpret_cast<const uint2 *>(p);
        x[0] = bf_lo(q.x);
        x[1] = bf_hi(q.x);
        x[2] = bf_lo(q.y);
        x[3] = bf_hi(q.y);
    } else {
        static_assert(V % 8 == 0, "whole 16-byte accesses");
#pragma unroll
        for (int i = 0; i < V / 8; ++i) {
            const uint4 q = reinterpret_cast<const uint4 *>(p)[i];
            x[8 * i] = bf_lo(q.x);
            x[8 * i + 1] = bf_hi(q.x);
            x[8 * i + 2] = bf_lo(q.y);
            x[8 * i + 3] = bf_hi(q.y);
            x[8 * i + 4] = bf_lo(q.z);
            x[8 * i + 5] = bf_hi(q.z);
            x[8 * i + 6] = bf_lo(q.w);
            x[8 * i + 7] = bf_hi(q.w);
        }
    }
}
template <int V> __device__ __forceinline__ void store_vec(float *p, const float (&x)[V])
{
    if constexpr (V == 1) {
        *p = x[0];
    } else {
#pragma unroll
        for (int i = 0; i < V / 4; ++i)
            reinterpret_cast<float4 *>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    }
}
template <int V> __device__ __forceinline__ void store_vec(bf16 *p, const float (&x)[V])
{
    if constexpr (V == 1) {
        put(p, x[0]);
    } else if constexpr (V == 4) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(bf_pack(x[0], x[1]), bf_pack(x[2], x[3]));
    } else {
#pragma unroll
        for (int i = 0; i < V / 8; ++i)
            reinterpret_cast<uint4 *>(p)[i] = make_uint4(bf_pack(x[8 * i], x[8 * i + 1]), bf_pack(x[8 * i + 2], x[8 * i + 3]),
                                                         bf_pack(x[8 * i + 4], x[8 * i + 5]), bf_pack(x[8 * i + 6], x[8 * i + 7]));
    }
}

// Two 32-bit floats in a register pair: sm_100 adds, multiplies and multiply-adds both with one
// instruction, each rounded as it would be alone.
typedef unsigned long long f2;

__device__ __forceinline__ f2 pack2(float lo, float hi)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(f2 v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b)
{
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b)
{
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c)
{
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// Stores of what this kernel does not read again: they leave the L2 cache first.
template <int V> __device__ __forceinline__ void store_vec_streaming(float *p, const float (&x)[V])
{
    if constexpr (V == 1) {
        __stcs(p, x[0]);
    } else {
#pragma unroll
        for (int i = 0; i < V / 4; ++i)
            __stcs(reinterpret_cast<float4 *>(p) + i, make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]));
    }
}
template <int V> __device__ __forceinline__ void store_vec_streaming(bf16 *p, const float (&x)[V])
{
    if constexpr (V == 8)
        __stcs(reinterpret_cast<uint4 *>(p), make_uint4(bf_pack(x[0], x[1]), bf_pack(x[2], x[3]), bf_pack(x[4], x[5]), bf_pack(x[6], x[7])));
    else if constexpr (V == 4)
        __stcs(reinterpret_cast<uint2 *>(p), make_uint2(bf_pack(x[0], x[1]), bf_pack(x[2], x[3])));
    else
        store_vec<V>(p, x);
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// A token id or label of either width.
__device__ __forceinline__ long long load_id(const void *p, int wide, long long i)
{
    return wide ? static_cast<const long long *>(p)[i] : (long long)static_cast<const int *>(p)[i];
}

// ---- programmatic dependent launch ---------------------------------------------------------
// The rule of adascale_kernels.cuh: a kernel lets its successor start early only after its own
// wait has returned, and touches nothing in global memory before that wait.  A kernel that writes gradients lets only another
// kernel of its call start early: a step that reads its rows ahead of the kernel before it (ADASCALE_FLAG_GRADS_READY) may come next.
__device__ __forceinline__ void griddep_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void griddep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ---- asynchronous 16-byte copies into shared memory ----------------------------------------
__device__ __forceinline__ void copy_async(void *dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((unsigned)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ---- bulk copies into shared memory, completed on mbarriers ----------------------------------
typedef unsigned long long u64;
constexpr u64 kWaitNs = 2000000000ull;   // no wait lasts longer than two seconds
constexpr unsigned kWaitHintNs = 20000;  // how long one poll may sleep (it wakes on completion)

__device__ __forceinline__ unsigned smem_u32(const void *p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(u64 *bar, unsigned count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(u64 *bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(u64 *bar, unsigned bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// Makes initialised barriers known to the copy engine.
__device__ __forceinline__ void mbar_publish() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
// One poll.  CLUSTER: what other blocks of the cluster wrote before they arrived is seen.
template <bool CLUSTER> __device__ __forceinline__ bool mbar_poll(unsigned addr, unsigned parity)
{
    unsigned done;
    if constexpr (CLUSTER)
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done)
                     : "r"(addr), "r"(parity), "r"(kWaitHintNs)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done)
                     : "r"(addr), "r"(parity), "r"(kWaitHintNs)
                     : "memory");
    return done;
}
template <bool CLUSTER> __device__ __noinline__ bool mbar_wait_long(unsigned addr, unsigned parity)
{
    u64 t0 = 0;
    for (unsigned spin = 0; spin < 1u << 22; ++spin) {
        if (mbar_poll<CLUSTER>(addr, parity)) return true;
        if ((spin & 63u) == 63u) {
            u64 now;
            asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
            if (t0 == 0) t0 = now;
            else if (now - t0 > kWaitNs) return false;
        }
    }
    return false;
}
// False if the phase did not complete within kWaitNs.
template <bool CLUSTER = false> __device__ __forceinline__ bool mbar_wait(u64 *bar, unsigned parity)
{
    const unsigned addr = smem_u32(bar);
    return mbar_poll<CLUSTER>(addr, parity) || mbar_wait_long<CLUSTER>(addr, parity);
}
// Orders this thread's writes to shared memory before copies out of it that start after a barrier.
__device__ __forceinline__ void copy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// shared -> global, by the thread's bulk groups
__device__ __forceinline__ void bulk_store(void *dst, const void *src, unsigned bytes)
{
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_u32(src)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// until at most N groups have not read their shared memory yet; until all writes are done
template <int N> __device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// global -> shared; both addresses and the size are multiples of 16
__device__ __forceinline__ void bulk_load(void *dst, const void *src, unsigned bytes, u64 *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(src), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// ---- host side -----------------------------------------------------------------------------

// cluster > 1: blocks per cluster (n_blocks is a multiple of it).
template <typename Args>
cudaError_t launch(void (*kernel)(Args), long long n_blocks, int threads, size_t smem, cudaStream_t s, const Args &a,
                   int cluster = 1)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)n_blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

#define OPS_CU(...)                                    \
    do {                                               \
        if ((__VA_ARGS__) != cudaSuccess) {            \
            (void)cudaGetLastError(); /* not sticky */ \
            return ADASCALE_ERR_CUDA;                  \
        }                                              \
    } while (0)

// Streaming multiprocessors of the current device (asked once per device).
inline int sm_count()
{
    static std::atomic<int> known[64];  // every thread writes the same number
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < 64) n = known[dev].load(std::memory_order_relaxed);
    if (n) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < 64) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

// Per device: whether a kernel's attributes have been set there.  Threads that race set them twice, to the same values.
struct OncePerDevice {
    std::atomic<bool> done[64];
    // False where there is something to do for device `dev`; devices beyond the table are done every time.
    bool has(int dev) const { return dev >= 0 && dev < 64 && done[dev].load(std::memory_order_acquire); }
    void set(int dev)
    {
        if (dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_release);
    }
};

// Lets a kernel have as much dynamic shared memory on the current device as there is beside its static one.  The attribute
// replaces what was set before, and calls from other threads may want other sizes of the same kernel: one value for all.
inline cudaError_t allow_smem(const void *kernel, OncePerDevice &known)
{
    int dev = 0, most = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || known.has(dev)) return e;
    cudaFuncAttributes f;
    e = cudaFuncGetAttributes(&f, kernel);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most - (int)f.sharedSizeBytes);
    if (e == cudaSuccess) known.set(dev);
    return e;
}

inline bool is_dtype(int d) { return d == ADASCALE_F32 || d == ADASCALE_BF16; }
inline bool is_itype(int d) { return d == ADASCALE_I32 || d == ADASCALE_I64; }
inline int elem_bytes(int dtype) { return dtype == ADASCALE_F32 ? 4 : 2; }
inline int id_bytes(int itype) { return itype == ADASCALE_I32 ? 4 : 8; }
inline bool on(const void *p, int bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }
// Every row of the matrix starts on a boundary of `bytes`; an absent matrix does not object.
inline bool rows_on(const void *p, long long ld, long long n_rows, int elem, int bytes)
{
    return !p || (on(p, bytes) && (n_rows <= 1 || ld * elem % bytes == 0));
}
__host__ __device__ inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

}  // namespace
