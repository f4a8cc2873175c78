// Products of a handful of experts' rows (a token or a few at a time): out[i] = a[i] w_e^T, plain or gated.  The weights of the
// experts that have rows are read once and nothing else costs, so every warp of the device takes columns of its own: 16 bytes of
// two weight rows (of g and u) in each lane at a time, eight steps in flight, sums in fp32 in the lanes and over them at the end.
// With tiles instead, one token's two experts of 1024 columns are 16 blocks' work: 19 us where this takes 8.6.
#pragma once
#include "hap_products.cuh"

namespace hapop {

// Rows of a call up to which this is the faster way.  Measured against tiles, 8 experts, 1024 x 4096: two rows of two experts 8.7
// and 19.4 us, of 14336 x 4096 47 and 48 us; but four rows of one expert 54 and 26 us, since a row costs instructions here.
constexpr int FEW_ROWS = 2;

template <typename T> __device__ __forceinline__ void unpack8(const uint4 w, float (&x)[8])
{
    const uint32_t y[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float2 f = unpack2(y[i], T());
        x[2 * i] = f.x, x[2 * i + 1] = f.y;
    }
}

// Eight values from p on of which n are there, zeros behind them: the last ones one by one, since a row may end where its buffer does.
__device__ __forceinline__ uint4 eight(const void *p, int n)
{
    if (n >= 8) return *(const uint4 *)p;
    uint32_t w[4] = {};
#pragma unroll
    for (int i = 0; i < 7; i++)
        if (i < n) w[i / 2] |= (uint32_t)((const uint16_t *)p)[i] << 16 * (i & 1);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T, int EPI> __global__ void __launch_bounds__(256) few_rows_kernel(const __grid_constant__ Args p)
{
    __shared__ int expert[FEW_ROWS], low[FEW_ROWS], high[FEW_ROWS], experts;
    __shared__ int bound[MAX_GROUPS + 1];
    launch_next();
    wait_for_last();
    for (int i = threadIdx.x; i <= p.groups; i += 256) {
        const int64_t o = p.offsets[i];
        bound[i] = o < 0 ? 0 : o > p.rows ? p.rows : (int)o;
    }
    __syncthreads();
    if (threadIdx.x < 32) {             // the experts that have rows, at most as many as there are rows
        const int lane = threadIdx.x;
        int below = 0, at = 0;
        for (int i0 = 0; i0 < p.groups; i0 += 32) {
            const int i = i0 + lane;
            int lo = i < p.groups ? bound[i] : 0, hi = i < p.groups ? bound[i + 1] : 0;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {           // offsets made ascending: the largest so far
                const int x = __shfl_up_sync(~0u, lo, d);
                if (lane >= d) lo = max(lo, x);
            }
            lo = max(lo, below), hi = max(hi, lo);
            const unsigned some = __ballot_sync(~0u, hi > lo);
            const int k = at + __popc(some & ((1u << lane) - 1));
            if (hi > lo && k < FEW_ROWS) expert[k] = i, low[k] = lo, high[k] = hi;
            at += __popc(some);
            below = __shfl_sync(~0u, hi, 31);
        }
        if (lane == 0) experts = min(at, FEW_ROWS);
    }
    __syncthreads();
    const int lane = threadIdx.x & 31, pairs = EPI == GATED ? p.ncols : (p.ncols + 1) / 2;
    const int units = experts * pairs;
    for (int u = blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += gridDim.x * 8) {
        const int k = u / pairs, c = u - k * pairs, e = expert[k], lo = low[k], hi = high[k];
        // two rows of w: columns 2c and 2c + 1, or g's and u's of column c
        const int n0 = EPI == GATED ? c : 2 * c, n1 = EPI == GATED ? p.ncols + c : min(2 * c + 1, p.ncols - 1);
        const T *w0 = (const T *)p.b + e * p.bgroup + n0 * p.ldb, *w1 = (const T *)p.b + e * p.bgroup + n1 * p.ldb;
        const int r0 = lo, nr = min(FEW_ROWS, hi - lo);
        float s0[FEW_ROWS] = {}, s1[FEW_ROWS] = {};
        const T *a = (const T *)p.a + r0 * p.lda;
        auto step = [&](const uint4 q0, const uint4 q1, int at, int valid) {
            float x0[8], x1[8];
            unpack8<T>(q0, x0), unpack8<T>(q1, x1);
#pragma unroll
            for (int r = 0; r < FEW_ROWS; r++) {
                if (r >= nr) break;
                float y[8];
                unpack8<T>(eight(a + r * p.lda + at, valid), y);
#pragma unroll
                for (int i = 0; i < 8; i++) s0[r] = fmaf(x0[i], y[i], s0[r]), s1[r] = fmaf(x1[i], y[i], s1[r]);
            }
        };
        int at = lane * 8;
        for (; at + 3 * 256 + 8 <= p.kdim; at += 4 * 256) {
            uint4 q0[4], q1[4];
#pragma unroll
            for (int i = 0; i < 4; i++) q0[i] = __ldcs((const uint4 *)(w0 + at + i * 256)), q1[i] = __ldcs((const uint4 *)(w1 + at + i * 256));
#pragma unroll
            for (int i = 0; i < 4; i++) step(q0[i], q1[i], at + i * 256, 8);
        }
#pragma unroll 1
        for (; at < p.kdim; at += 256) step(eight(w0 + at, p.kdim - at), eight(w1 + at, p.kdim - at), at, p.kdim - at);
#pragma unroll
        for (int r = 0; r < FEW_ROWS; r++) {
            if (r >= nr) break;
#pragma unroll
            for (int d = 16; d; d /= 2) s0[r] += __shfl_xor_sync(~0u, s0[r], d), s1[r] += __shfl_xor_sync(~0u, s1[r], d);
            if (lane) continue;
            const int64_t row = r0 + r;
            T *o = (T *)p.out + row * p.ldo;
            if (EPI == GATED) {
                if (p.out) o[n0] = from_float<T>(s0[r]), o[n1] = from_float<T>(s1[r]);
                ((T *)p.h)[row * p.ldh + c] = from_float<T>(gate(s0[r], s1[r]));
            } else {
                o[n0] = from_float<T>(p.accumulate ? s0[r] + to_float(o[n0]) : s0[r]);
                if (n1 > n0) o[n1] = from_float<T>(p.accumulate ? s1[r] + to_float(o[n1]) : s1[r]);
            }
        }
    }
}

} // namespace hapop
