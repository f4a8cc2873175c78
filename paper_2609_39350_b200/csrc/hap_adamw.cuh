// One AdamW step over many tensors in one launch: m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2,
// p = p (1 - lr wd) - lr (m / c1) / (sqrt(v / c2) + eps) with c = 1 - b^step.  The tensors' descriptors travel as the kernel's
// arguments, so a call keeps nothing and a captured one replays with the same addresses.
// Moments in 8 bits: 256 values of a tensor share a scale s, the largest magnitude among them.  A first moment is c in
// -127 .. 127 and stands for s t |t|, t = c / 127; a second moment c in 0 .. 255, s t^4 with t = c / 255 (its square root,
// which the update divides by, is then s' t^2: both are finer near 0, where most of a block lies).  A second moment above 0
// keeps a code of at least 1.  Everything up to the codes is one IEEE operation per operator, rounded to nearest, so codes
// are the same wherever they are computed.
#pragma once
#include "hap_products.cuh"
#include "../../include/hap.h"

namespace hapop {

constexpr int ADAMW_BLOCK = 256;        // values that share a scale
constexpr int ADAMW_CHUNK = 4096;       // values that a block of threads takes

struct AdamwTensor { void *p; const void *g; void *m, *v; float *ms, *vs; void *copy; uint64_t n; };
struct AdamwFactors { float b1, b2, a1, a2, decay, step, root, eps; int copy16; };      // a = 1 - b; step = lr / c1; root = 1 / sqrt(c2)
// descriptors of one launch; the larger form fills most of a launch's 32 KB of arguments
template <int N> struct AdamwList { AdamwTensor t[N]; unsigned first[N + 1]; int n; };      // first: first chunk of each tensor

template <int N> __device__ __forceinline__ int adamw_tensor(const AdamwList<N> &list, unsigned chunk)
{
    int lo = 0, hi = list.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (list.first[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ float adamw_value(float p, float m, float v, const AdamwFactors &f)
{
    return p * f.decay - f.step * m / (sqrtf(v) * f.root + f.eps);
}
__device__ __forceinline__ float adamw_read_m(int c, float s)
{
    const float t = __fmul_rn((float)c, 1.0f / 127.0f);
    return __fmul_rn(__fmul_rn(t, fabsf(t)), s);
}
__device__ __forceinline__ float adamw_read_v(int c, float s)
{
    const float t = __fmul_rn((float)c, 1.0f / 255.0f), q = __fmul_rn(t, t);
    return __fmul_rn(__fmul_rn(q, q), s);
}
__device__ __forceinline__ float adamw_first(float m, float g, const AdamwFactors &f) { return __fadd_rn(__fmul_rn(m, f.b1), __fmul_rn(g, f.a1)); }
__device__ __forceinline__ float adamw_second(float v, float g, const AdamwFactors &f) { return __fadd_rn(__fmul_rn(v, f.b2), __fmul_rn(__fmul_rn(g, g), f.a2)); }
// largest of two magnitudes; a NaN stays
__device__ __forceinline__ float larger(float a, float b) { return a != a ? a : b > a || b != b ? b : a; }
// the copy in 16 bits of a parameter that is held in 32
__device__ __forceinline__ void adamw_copy(void *copy, int fp16, uint64_t i, float x)
{
    if (fp16) ((__half *)copy)[i] = __float2half_rn(x);
    else ((__nv_bfloat16 *)copy)[i] = __float2bfloat16_rn(x);
}

template <typename P, typename G, int N> __global__ void __launch_bounds__(256) adamw_kernel(const __grid_constant__ AdamwList<N> list, AdamwFactors f, const float *grad_scale)
{
    const int k = adamw_tensor(list, blockIdx.x);
    const AdamwTensor &t = list.t[k];
    const uint64_t from = (uint64_t)(blockIdx.x - list.first[k]) * ADAMW_CHUNK;
    const int n = (int)min((uint64_t)ADAMW_CHUNK, t.n - from);
    P *p = (P *)t.p + from;
    const G *g = (const G *)t.g + from;
    float *m = (float *)t.m + from, *v = (float *)t.v + from;
    const float scale = grad_scale ? *grad_scale : 1.0f;
    for (int i = threadIdx.x; i < n; i += 256) {
        const float x = to_float(g[i]) * scale;
        const float mi = adamw_first(m[i], x, f), vi = adamw_second(v[i], x, f);
        m[i] = mi, v[i] = vi;
        const float y = adamw_value(to_float(p[i]), mi, vi, f);
        p[i] = from_float<P>(y);
        if (t.copy) adamw_copy(t.copy, f.copy16, from + i, y);
    }
}

template <typename P, typename G, int N> __global__ void __launch_bounds__(256) adamw8_kernel(const __grid_constant__ AdamwList<N> list, AdamwFactors f, const float *grad_scale)
{
    const int k = adamw_tensor(list, blockIdx.x);
    const AdamwTensor &t = list.t[k];
    const float scale = grad_scale ? *grad_scale : 1.0f;
    const int lane = threadIdx.x & 31;
    const uint64_t first = (uint64_t)(blockIdx.x - list.first[k]) * ADAMW_CHUNK;
    for (int w = threadIdx.x >> 5; w < ADAMW_CHUNK / ADAMW_BLOCK; w += 8) {
        const uint64_t from = first + w * ADAMW_BLOCK, block = from / ADAMW_BLOCK;
        if (from >= t.n) break;
        const int n = (int)min((uint64_t)ADAMW_BLOCK, t.n - from);
        P *p = (P *)t.p + from;
        const G *g = (const G *)t.g + from;
        int8_t *m = (int8_t *)t.m + from;
        uint8_t *v = (uint8_t *)t.v + from;
        const float ms = t.ms[block], vs = t.vs[block];
        float mi[8], vi[8], mt = 0.0f, vt = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int i = lane + 32 * j;
            mi[j] = vi[j] = 0.0f;
            if (i >= n) continue;
            const float x = __fmul_rn(to_float(g[i]), scale);
            mi[j] = adamw_first(adamw_read_m(m[i], ms), x, f);
            vi[j] = adamw_second(adamw_read_v(v[i], vs), x, f);
            const float y = adamw_value(to_float(p[i]), mi[j], vi[j], f);
            p[i] = from_float<P>(y);
            if (t.copy) adamw_copy(t.copy, f.copy16, from + i, y);
            mt = larger(mt, fabsf(mi[j])), vt = larger(vt, vi[j]);
        }
#pragma unroll
        for (int d = 16; d; d /= 2) {
            mt = larger(mt, __shfl_xor_sync(~0u, mt, d));
            vt = larger(vt, __shfl_xor_sync(~0u, vt, d));
        }
        if (lane == 0) t.ms[block] = mt, t.vs[block] = vt;
        // (codes of a block whose scale is not finite are read as values that are not finite, whatever they are)
        const float md = mt > 0.0f ? mt : 1.0f, vd = vt > 0.0f ? vt : 1.0f;
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int i = lane + 32 * j;
            if (i >= n) continue;
            const float q = rintf(__fmul_rn(__fsqrt_rn(__fdiv_rn(fabsf(mi[j]), md)), 127.0f));
            const float u = rintf(__fmul_rn(__fsqrt_rn(__fsqrt_rn(__fdiv_rn(vi[j], vd))), 255.0f));
            m[i] = (int8_t)(int)copysignf(fminf(q, 127.0f), mi[j]);
            v[i] = (uint8_t)(vi[j] > 0.0f ? min(255, max(1, (int)u)) : 0);
        }
    }
}

// the values that 8-bit moments stand for
template <int N> __global__ void __launch_bounds__(256) adamw_values_kernel(const __grid_constant__ AdamwList<N> list)
{
    const int k = adamw_tensor(list, blockIdx.x);
    const AdamwTensor &t = list.t[k];                           // (p: m's values, copy: v's values)
    const uint64_t from = (uint64_t)(blockIdx.x - list.first[k]) * ADAMW_CHUNK;
    const int n = (int)min((uint64_t)ADAMW_CHUNK, t.n - from);
    for (int i = threadIdx.x; i < n; i += 256) {
        const uint64_t at = from + i, block = at / ADAMW_BLOCK;
        if (t.p) ((float *)t.p)[at] = adamw_read_m(((const int8_t *)t.m)[at], t.ms[block]);
        if (t.copy) ((float *)t.copy)[at] = adamw_read_v(((const uint8_t *)t.v)[at], t.vs[block]);
    }
}

} // namespace hapop
