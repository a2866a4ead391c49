// Shared by the operators that need no context: element types, vectors of 16 bytes, reductions over the threads of a row,
// and the guard that leaves the caller's current device as it was.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/moe_ovl.h"

namespace moe_ovl {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// VEC neighbouring elements; one load or store of 16 bytes where VEC * sizeof(T) is 16, in general of their size.
template <typename T, int VEC> struct alignas(sizeof(T) * VEC) Pack { T v[VEC]; };

template <typename T, int VEC> __device__ __forceinline__ Pack<T, VEC> load_pack(const T *p)
{
    Pack<T, VEC> r;
    if constexpr (sizeof(r) == 16) *reinterpret_cast<uint4 *>(&r) = *reinterpret_cast<const uint4 *>(p);
    else r = *reinterpret_cast<const Pack<T, VEC> *>(p);
    return r;
}
template <typename T, int VEC> __device__ __forceinline__ void store_pack(T *p, const Pack<T, VEC> &r)
{
    if constexpr (sizeof(r) == 16) *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(&r);
    else *reinterpret_cast<Pack<T, VEC> *>(p) = r;
}

// Two neighbouring values as floats, and back with one rounding each.
__device__ __forceinline__ float2 to_f32x2(const float *p) { return make_float2(p[0], p[1]); }
__device__ __forceinline__ float2 to_f32x2(const __nv_bfloat16 *p)
{
    const uint32_t u = *reinterpret_cast<const uint32_t *>(p);
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
__device__ __forceinline__ float2 to_f32x2(const __half *p) { return __half22float2(*reinterpret_cast<const __half2 *>(p)); }
__device__ __forceinline__ void from_f32x2(float *p, float2 v) { p[0] = v.x, p[1] = v.y; }
__device__ __forceinline__ void from_f32x2(__nv_bfloat16 *p, float2 v) { *reinterpret_cast<__nv_bfloat162 *>(p) = __float22bfloat162_rn(v); }
__device__ __forceinline__ void from_f32x2(__half *p, float2 v) { *reinterpret_cast<__half2 *>(p) = __float22half2_rn(v); }
// a + b, rounded once to the type
__device__ __forceinline__ void add_round2(float *a, const float *b) { a[0] += b[0], a[1] += b[1]; }
__device__ __forceinline__ void add_round2(__nv_bfloat16 *a, const __nv_bfloat16 *b)
{
    __nv_bfloat162 *p = reinterpret_cast<__nv_bfloat162 *>(a);
    *p = __hadd2(*p, *reinterpret_cast<const __nv_bfloat162 *>(b));
}
__device__ __forceinline__ void add_round2(__half *a, const __half *b)
{
    __half2 *p = reinterpret_cast<__half2 *>(a);
    *p = __hadd2(*p, *reinterpret_cast<const __half2 *>(b));
}

// Two 32-bit operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(*reinterpret_cast<unsigned long long *>(&d))
        : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)),
          "l"(*reinterpret_cast<unsigned long long *>(&c)));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;"
        : "=l"(*reinterpret_cast<unsigned long long *>(&d))
        : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(*reinterpret_cast<unsigned long long *>(&d))
        : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)));
    return d;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// The largest magnitude; NaN where any is.
__device__ __forceinline__ float max_abs(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}
__device__ __forceinline__ float max_abs(float a, float2 b)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b.x), "f"(b.y));
    return r;
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Largest value over the warp; NaN where any is.
__device__ __forceinline__ float warp_max(float v)
{
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// Makes `device` current for one call and puts the caller's device back.
struct DeviceGuard {
    int before = -1;
    bool ok = false;
    explicit DeviceGuard(int device)
    {
        if (cudaGetDevice(&before) != cudaSuccess) return;
        ok = before == device || cudaSetDevice(device) == cudaSuccess;
        if (before == device) before = -1;
    }
    ~DeviceGuard()
    {
        if (before >= 0) cudaSetDevice(before);
    }
};

// Kernels of a stream may be brought onto the device before the one in front has ended (launch_behind): their first blocks are then
// in place when it ends.  Every thread calls after_previous() before it reads or writes global memory or starts a wait with a
// time limit; it returns when everything before the kernel in the stream has ended and its writes are visible.  may_follow()
// lets the next kernel in, once every block has called it.  A kernel that allocates tensor memory calls it after
// the allocation: a block that came in early and holds tensor memory must not keep one it waits for from getting its own.
// Norm, choice, 8-bit product, gate and product for one token (2048 x 1408, 64 experts, 6 of them), one behind the other: 27.3 us
// without, 24.4 us with it.
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void may_follow() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// cluster: CTAs per cluster, 1 for none.
template <typename... P, typename... A>
int launch_behind(void (*kernel)(P...), unsigned blocks, dim3 threads, int smem, unsigned cluster, cudaStream_t stream, const A &...args)
{
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = threads;
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? MOE_OVL_OK : MOE_OVL_ERR_CUDA;
}

inline int launched() { return cudaGetLastError() == cudaSuccess ? MOE_OVL_OK : MOE_OVL_ERR_CUDA; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool known_dtype(int t) { return t == MOE_OVL_BF16 || t == MOE_OVL_F16 || t == MOE_OVL_F32; }
inline int dtype_bytes(int t) { return t == MOE_OVL_F32 ? 4 : 2; }

// Calls f with a value of the element type.
template <typename F> int with_dtype(int t, F f)
{
    if (t == MOE_OVL_BF16) return f(__nv_bfloat16());
    if (t == MOE_OVL_F16) return f(__half());
    return f(0.0f);
}

}  // namespace moe_ovl
