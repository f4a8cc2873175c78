// Values of the training operators: conversions, eights of them in memory, and the start of a kernel behind its predecessor.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace hapop {

__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(float x) { return x; }
// A kernel that was launched with its predecessor's end still ahead (see launch_next) starts by letting its successor do the same,
// and touches no memory that others write before the predecessor's work is whole.
__device__ __forceinline__ void launch_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_last() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ float from_float(float x) { return x; }
__device__ __forceinline__ uint32_t pack2(float x, float y, __nv_bfloat16) { __nv_bfloat162 v = __floats2bfloat162_rn(x, y); return *(uint32_t *)&v; }
__device__ __forceinline__ uint32_t pack2(float x, float y, __half) { __half2 v = __floats2half2_rn(x, y); return *(uint32_t *)&v; }
__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16) { return __bfloat1622float2(*(__nv_bfloat162 *)&w); }
__device__ __forceinline__ float2 unpack2(uint32_t w, __half) { return __half22float2(*(__half2 *)&w); }

// eight values side by side, at an address that is a multiple of 16 bytes
template <typename T> __device__ __forceinline__ void load8(const T *p, float (&x)[8])
{
    if constexpr (sizeof(T) == 4) {
        const float4 a = ((const float4 *)p)[0], b = ((const float4 *)p)[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        const uint4 a = *(const uint4 *)p;
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 f = unpack2(w[i], T());
            x[2 * i] = f.x, x[2 * i + 1] = f.y;
        }
    }
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&x)[8])
{
    if constexpr (sizeof(T) == 4) {
        ((float4 *)p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        ((float4 *)p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        *(uint4 *)p = make_uint4(pack2(x[0], x[1], T()), pack2(x[2], x[3], T()), pack2(x[4], x[5], T()), pack2(x[6], x[7], T()));
    }
}
// values in front of the first one whose address, and those of the following eights, is a multiple of 16 bytes
template <typename T> __device__ __forceinline__ int in_front(const T *p) { return (int)(((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T)); }

// 16 bytes to shared memory, on their way while the thread goes on, or 16 zeros where `bytes` is 0; it sees them itself behind
// copies_arrived<0>(), and no other thread is meant to.  copies_arrived<N>: all but the last N groups are there.
__device__ __forceinline__ void copy16(void *to, const void *from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void end_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

} // namespace hapop
