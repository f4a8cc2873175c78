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
// Values that a block of threads takes: the larger number where there are blocks enough for every multiprocessor to have several
constexpr int ADAMW_CHUNK = 4096, ADAMW_SHORT = 1024;

struct AdamwTensor { void *p; const void *g; void *m, *v; float *ms, *vs; void *copy; uint64_t n; };
struct AdamwFactors { float b1, b2, a1, a2, decay, step, root, eps; int copy16; };      // a = 1 - b; step = lr / c1; root = 1 / sqrt(c2)
// descriptors of one launch; the larger form fills most of a launch's 32 KB of arguments
template <int N> struct AdamwList { AdamwTensor t[N]; unsigned first[N + 1]; int n, chunk; };      // first: first chunk of each tensor

template <int N> __device__ __forceinline__ int adamw_tensor(const AdamwList<N> &list, unsigned chunk)
{
    int lo = 0, hi = list.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (list.first[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ float root_of(float x) { float y; asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// The new parameter.  Held in 16 bits it is rounded by more than a root and a quotient that are off by a unit or two in the last
// place; held in 32 it may be the update and little else (weights that begin at 0), and both are rounded to nearest.  (100 M
// parameters in 32 bits: 412 us either way with states in 32 bits, 346 against 318 in 8.)
template <typename P> __device__ __forceinline__ float adamw_value(float p, float m, float v, const AdamwFactors &f)
{
    if constexpr (sizeof(P) == 4) return p * f.decay - __fdiv_rn(f.step * m, __fsqrt_rn(v) * f.root + f.eps);
    else return p * f.decay - __fdividef(f.step * m, root_of(v) * f.root + f.eps);
}
__device__ __forceinline__ float adamw_read_m(float c, float s)
{
    const float t = __fmul_rn(c, 1.0f / 127.0f);
    return __fmul_rn(__fmul_rn(t, fabsf(t)), s);
}
__device__ __forceinline__ float adamw_read_v(float c, float s)
{
    const float t = __fmul_rn(c, 1.0f / 255.0f), q = __fmul_rn(t, t);
    return __fmul_rn(__fmul_rn(q, q), s);
}
__device__ __forceinline__ float adamw_first(float m, float g, const AdamwFactors &f) { return __fadd_rn(__fmul_rn(m, f.b1), __fmul_rn(g, f.a1)); }
__device__ __forceinline__ float adamw_second(float v, float g, const AdamwFactors &f) { return __fadd_rn(__fmul_rn(v, f.b2), __fmul_rn(__fmul_rn(g, g), f.a2)); }
// A magnitude's bits, which order as the values do, infinity and then NaN above all.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
// 0 .. 255 as a float: in the low bits of 2^23
__device__ __forceinline__ float byte_value(uint32_t c) { return __uint_as_float(0x4b000000u | c) - 8388608.0f; }
__device__ __forceinline__ float signed_byte_value(uint32_t c) { return __uint_as_float(0x4b000000u | (c ^ 0x80u)) - 8388736.0f; }

// the copy in 16 bits of a parameter that is held in 32
__device__ __forceinline__ void adamw_copy(void *copy, int fp16, uint64_t i, float x)
{
    if (fp16) ((__half *)copy)[i] = __float2half_rn(x);
    else ((__nv_bfloat16 *)copy)[i] = __float2bfloat16_rn(x);
}

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
__device__ __forceinline__ void copy8(void *copy, int fp16, uint64_t i, const float (&x)[8])
{
    if (fp16) store8((__half *)copy + i, x);
    else store8((__nv_bfloat16 *)copy + i, x);
}
// values in front of the first one whose address, and those of the following eights, is a multiple of 16 bytes
template <typename T> __device__ __forceinline__ int in_front(const T *p) { return (int)(((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T)); }

// States in 32 bits: 12 to 30 bytes a value and nothing else to do; bound by memory.  Tensors that begin at the same odd place in
// all of their buffers (views of flat buffers) move in eights from the first aligned value on; others value by value.
template <typename P, typename G, int N> __global__ void __launch_bounds__(256) adamw_kernel(const __grid_constant__ AdamwList<N> list, AdamwFactors f, const float *grad_scale)
{
    const int k = adamw_tensor(list, blockIdx.x);
    const AdamwTensor &t = list.t[k];
    const uint64_t from = (uint64_t)(blockIdx.x - list.first[k]) * list.chunk;
    const int n = (int)min((uint64_t)list.chunk, t.n - from);
    P *p = (P *)t.p + from;
    const G *g = (const G *)t.g + from;
    float *m = (float *)t.m + from, *v = (float *)t.v + from;
    char *copy = t.copy ? (char *)t.copy + 2 * from : nullptr;
    const float scale = grad_scale ? *grad_scale : 1.0f;
    auto one = [&](int i) {
        const float x = to_float(g[i]) * scale;
        const float mi = adamw_first(m[i], x, f), vi = adamw_second(v[i], x, f);
        m[i] = mi, v[i] = vi;
        const float y = adamw_value<P>(to_float(p[i]), mi, vi, f);
        p[i] = from_float<P>(y);
        if (copy) adamw_copy(copy, f.copy16, i, y);
    };
    const int h = max(in_front(p), max(in_front(g), copy ? in_front((const __half *)copy) : 0));
    const bool eights = !(((uintptr_t)(p + h) | (uintptr_t)(g + h) | (uintptr_t)(m + h) | (uintptr_t)(v + h) | (copy ? (uintptr_t)(copy + 2 * h) : 0)) & 15);
    if (!eights) {
        for (int i = threadIdx.x; i < n; i += 256) one(i);
        return;
    }
    const int groups = n > h ? (n - h) / 8 : 0, rest = h + groups * 8;
#pragma unroll 2
    for (int i = threadIdx.x; i < groups; i += 256) {
        const int at = h + i * 8;
        float x[8], a[8], b[8], y[8];
        load8(g + at, x), load8(m + at, a), load8(v + at, b), load8(p + at, y);
#pragma unroll
        for (int j = 0; j < 8; j++) {
            x[j] *= scale;
            a[j] = adamw_first(a[j], x[j], f), b[j] = adamw_second(b[j], x[j], f);
            y[j] = adamw_value<P>(y[j], a[j], b[j], f);
        }
        store8(m + at, a), store8(v + at, b), store8(p + at, y);
        if (copy) copy8(copy, f.copy16, at, y);
    }
    if (threadIdx.x < min(h, n)) one(threadIdx.x);
    if (rest + (int)threadIdx.x < n) one(rest + threadIdx.x);          // (fewer than eight)
}

// c of a magnitude x under the scale s, as the definition's operations round it.  The quick way's result q is off by less than 1e-4
// (some units in the last place of at most 255), so only where it lies that near to a border are the operations themselves made;
// made everywhere they took most of the kernel's time.  (A quotient below 2^-126 counts as 0: its code is 0 either way.)
__device__ __forceinline__ float quick_root(float x) { float y; asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
template <bool FOURTH> __device__ __forceinline__ uint32_t adamw_code(float x, float s, float inverse)
{
    const float most = FOURTH ? 255.0f : 127.0f;
    float q = quick_root(x * inverse);
    if (FOURTH) q = quick_root(q);
    q *= most;
    float c = q + 12582912.0f;                              // 1.5 * 2^23: rounds to a whole number, which is in the low bits
    if (!(fabsf(q - (c - 12582912.0f)) < 0.4998f)) {
        q = __fsqrt_rn(__fdiv_rn(x, s));
        if (FOURTH) q = __fsqrt_rn(q);
        c = fminf(__fmul_rn(q, most), most) + 12582912.0f;  // (fminf: a number also from NaN)
    }
    return __float_as_uint(c) & 0xffu;
}

// States in 8 bits: a warp takes the 256 values of a block (WHOLE: it has so many), eight for each lane, side by side where every
// address allows it (EIGHTS).
template <typename P, typename G, bool EIGHTS, bool WHOLE> __device__ __forceinline__ void adamw8_block(const AdamwTensor &t, uint64_t from, const AdamwFactors &f, float scale, int lane)
{
    const uint64_t block = from / ADAMW_BLOCK;
    const int n = (int)min((uint64_t)ADAMW_BLOCK, t.n - from);
    P *p = (P *)t.p + from;
    const G *g = (const G *)t.g + from;
    int8_t *m = (int8_t *)t.m + from;
    uint8_t *v = (uint8_t *)t.v + from;
    char *copy = t.copy ? (char *)t.copy + 2 * from : nullptr;
    const float ms = t.ms[block], vs = t.vs[block];
    float x[8], y[8], a[8], b[8];
    auto at = [&](int j) { return EIGHTS ? lane * 8 + j : lane + 32 * j; };
    if (EIGHTS) {
        const uint2 cm = *(const uint2 *)(m + lane * 8), cv = *(const uint2 *)(v + lane * 8);
        load8(g + lane * 8, x), load8(p + lane * 8, y);
#pragma unroll
        for (int j = 0; j < 8; j++) {
            a[j] = signed_byte_value(__byte_perm(j < 4 ? cm.x : cm.y, 0, 0x4440 + (j & 3)));
            b[j] = byte_value(__byte_perm(j < 4 ? cv.x : cv.y, 0, 0x4440 + (j & 3)));
        }
    } else {
        uint32_t cm[8], cv[8];
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int i = at(j);
            const bool in = WHOLE || i < n;
            cm[j] = in ? ((const uint8_t *)m)[i] : 0, cv[j] = in ? v[i] : 0, x[j] = in ? to_float(g[i]) : 0.0f, y[j] = in ? to_float(p[i]) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; j++) a[j] = signed_byte_value(cm[j]), b[j] = byte_value(cv[j]);
    }
    uint32_t mt = 0, vt = 0;                                // (behind the tensor's end everything is 0)
#pragma unroll
    for (int j = 0; j < 8; j++) {
        x[j] = __fmul_rn(x[j], scale);
        if (!WHOLE && at(j) >= n) x[j] = 0.0f;
        a[j] = adamw_first(adamw_read_m(a[j], ms), x[j], f);
        b[j] = adamw_second(adamw_read_v(b[j], vs), x[j], f);
        y[j] = adamw_value<P>(y[j], a[j], b[j], f);
        if (WHOLE || at(j) < n) mt = max(mt, magnitude(a[j])), vt = max(vt, magnitude(b[j]));
    }
    if (EIGHTS) {
        store8(p + lane * 8, y);
        if (copy) copy8(copy, f.copy16, lane * 8, y);
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int i = at(j);
            if (WHOLE || i < n) p[i] = from_float<P>(y[j]);
            if ((WHOLE || i < n) && copy) adamw_copy(copy, f.copy16, i, y[j]);
        }
    }
    const float mtop = __uint_as_float(__reduce_max_sync(~0u, mt)), vtop = __uint_as_float(__reduce_max_sync(~0u, vt));
    if (lane == 0) t.ms[block] = mtop, t.vs[block] = vtop;
    // (codes of a block whose scale is not finite are read as values that are not finite, whatever they are; where a scale's
    // inverse would overflow or be 0 the quick way gets no number, and the operations are made)
    const float md = mtop > 0.0f ? mtop : 1.0f, vd = vtop > 0.0f ? vtop : 1.0f;
    const float mr = md < 1e37f ? __fdividef(1.0f, md) : NAN, vr = vd < 1e37f ? __fdividef(1.0f, vd) : NAN;
    uint32_t cm[2] = {0, 0}, cv[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; j++) {
        uint32_t c = adamw_code<false>(fabsf(a[j]), md, mr), w = adamw_code<true>(b[j], vd, vr);
        c = a[j] < 0.0f ? (0u - c) & 0xffu : c;
        w = b[j] > 0.0f ? max(w, 1u) : 0;
        if (EIGHTS) {
            cm[j / 4] |= c << 8 * (j & 3), cv[j / 4] |= w << 8 * (j & 3);
        } else if (WHOLE || at(j) < n) {
            ((uint8_t *)m)[at(j)] = (uint8_t)c, v[at(j)] = (uint8_t)w;
        }
    }
    if (EIGHTS) {
        *(uint2 *)(m + lane * 8) = make_uint2(cm[0], cm[1]);
        *(uint2 *)(v + lane * 8) = make_uint2(cv[0], cv[1]);
    }
}

template <typename P, typename G, int N> __global__ void __launch_bounds__(256, 4) adamw8_kernel(const __grid_constant__ AdamwList<N> list, AdamwFactors f, const float *grad_scale)
{
    const int k = adamw_tensor(list, blockIdx.x);
    const AdamwTensor &t = list.t[k];
    const float scale = grad_scale ? *grad_scale : 1.0f;
    const uint64_t first = (uint64_t)(blockIdx.x - list.first[k]) * list.chunk;
    const bool eights = !(((uintptr_t)t.p | (uintptr_t)t.g | (uintptr_t)t.copy) & 15) && !(((uintptr_t)t.m | (uintptr_t)t.v) & 7);
    for (int w = threadIdx.x >> 5; w < list.chunk / ADAMW_BLOCK; w += 8) {
        const uint64_t from = first + w * ADAMW_BLOCK;
        if (from >= t.n) break;
        if (from + ADAMW_BLOCK > t.n) adamw8_block<P, G, false, false>(t, from, f, scale, threadIdx.x & 31);
        else if (eights) adamw8_block<P, G, true, true>(t, from, f, scale, threadIdx.x & 31);
        else adamw8_block<P, G, false, true>(t, from, f, scale, threadIdx.x & 31);
    }
}

// the values that 8-bit moments stand for
template <int N> __global__ void __launch_bounds__(256) adamw_values_kernel(const __grid_constant__ AdamwList<N> list)
{
    const int k = adamw_tensor(list, blockIdx.x);
    const AdamwTensor &t = list.t[k];                           // (p: m's values, copy: v's values)
    const uint64_t from = (uint64_t)(blockIdx.x - list.first[k]) * list.chunk;
    const int n = (int)min((uint64_t)list.chunk, t.n - from);
    // four at a time from the first place on where codes and values are aligned, if there is one (views of flat buffers)
    auto read = [&](const uint8_t *codes, const float *scales, float *to, auto value) {
        codes += from, to += from, scales += from / ADAMW_BLOCK;
        const int h = (int)((16 - ((uintptr_t)to & 15)) & 15) / 4;
        const bool fours = ((uintptr_t)(codes + h) & 3) == 0;
        const int groups = fours && n > h ? (n - h) / 4 : 0, head = fours ? min(h, n) : n, rest = head + groups * 4;
#pragma unroll 4
        for (int g = threadIdx.x; g < groups; g += 256) {
            const int i = h + g * 4;
            const uint32_t c = *(const uint32_t *)(codes + i);
            const float a = scales[i / ADAMW_BLOCK], b = scales[(i + 3) / ADAMW_BLOCK];     // (four values can be of two blocks)
            const int turn = ADAMW_BLOCK - i % ADAMW_BLOCK;                                 // values of the first
            *(float4 *)(to + i) = make_float4(value(c & 255, a), value(c >> 8 & 255, turn > 1 ? a : b), value(c >> 16 & 255, turn > 2 ? a : b), value(c >> 24, turn > 3 ? a : b));
        }
        for (int i = threadIdx.x; i < head; i += 256) to[i] = value(codes[i], scales[i / ADAMW_BLOCK]);
        for (int i = rest + threadIdx.x; i < n; i += 256) to[i] = value(codes[i], scales[i / ADAMW_BLOCK]);
    };
    if (t.p) read((const uint8_t *)t.m, t.ms, (float *)t.p, [](uint32_t c, float s) { return adamw_read_m(signed_byte_value(c), s); });
    if (t.copy) read((const uint8_t *)t.v, t.vs, (float *)t.copy, [](uint32_t c, float s) { return adamw_read_v(byte_value(c), s); });
}

} // namespace hapop
