// Layer norm over rows of H: y = (x - mean) r w + b with r = 1 / sqrt(variance + eps), or without mean and b (CENTRED false); and its
// gradients dx = base + r (g - mean(g) - xh mean(g xh)), g = dy w, xh = (x - mean) r; dw = sum over rows of dy xh, db = sum of dy.
// All of it is bound by memory: a row is read once and stays in registers.  The variance is that of the differences to the mean,
// not a difference of squares.
#pragma once
#include "hap_rows.cuh"

namespace hapop {

constexpr int MOST_NORM = 16384;        // columns

struct NormArgs {
    int64_t rows;
    int H, blocks, add;             // blocks: of the backward pass, each with partial sums of its own; add: to what dw and db hold
    float eps;
    const void *x, *w, *b, *dy, *base;
    int64_t ldx, ldy, lddy, ldbase, lddx;
    void *y, *dx, *dw, *db;
    float *mean, *rstd;             // forwards written, backwards read
    float *parts;                   // [blocks][1 or 2][H]
};

// the sum over a row's threads, LANES of them: a warp, or a block's warps through shared memory
template <int N> __device__ __forceinline__ void row_sums(float (&s)[N], int threads, float (*space)[32])
{
#pragma unroll
    for (int i = 0; i < N; i++)
#pragma unroll
        for (int d = 16; d; d /= 2) s[i] += __shfl_xor_sync(~0u, s[i], d);
    if (threads <= 32) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; i++) space[i][warp] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++) {
        s[i] = lane < threads / 32 ? space[i][lane] : 0.0f;
#pragma unroll
        for (int d = 16; d; d /= 2) s[i] += __shfl_xor_sync(~0u, s[i], d);
    }
}

// A row for each blockDim.x threads, EIGHTS eights of columns for each; blockDim.y rows of one warp each where a row is that short
template <typename T, typename P, int EIGHTS, bool WIDE, bool CENTRED> __global__ void __launch_bounds__(EIGHTS == 4 ? 256 : 1024) norm_kernel(const NormArgs p)
{
    __shared__ float space[2][1][32];
    launch_next();
    wait_for_last();
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const int threads = blockDim.x;
    if (row >= p.rows) return;                              // (whole warps: with one row for a block all are here)
    const T *x = (const T *)p.x + row * p.ldx;
    float v[EIGHTS][8], s[1] = {0};
#pragma unroll
    for (int r = 0; r < EIGHTS; r++) {
        load_columns<WIDE>(x, 8 * r * threads, threadIdx.x, threads, p.H, v[r]);
        if (CENTRED)
#pragma unroll
            for (int i = 0; i < 8; i++) s[0] += v[r][i];
    }
    float mean = 0;
    if (CENTRED) {
        row_sums(s, threads, space[0]);
        mean = s[0] / (float)p.H;
        s[0] = 0;
    }
#pragma unroll
    for (int r = 0; r < EIGHTS; r++)
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (CENTRED) v[r][i] = column<WIDE>(8 * r * threads, threadIdx.x, threads, i) < p.H ? v[r][i] - mean : 0.0f;
            s[0] = fmaf(v[r][i], v[r][i], s[0]);
        }
    row_sums(s, threads, space[1]);
    const float rstd = 1.0f / sqrtf(s[0] / (float)p.H + p.eps);
    if (threadIdx.x == 0) {
        if (CENTRED && p.mean) p.mean[row] = mean;
        if (p.rstd) p.rstd[row] = rstd;
    }
#pragma unroll
    for (int r = 0; r < EIGHTS; r++) {
        float w[8], b[8];
        if (p.w) load_columns<WIDE>((const P *)p.w, 8 * r * threads, threadIdx.x, threads, p.H, w);
        if (p.b) load_columns<WIDE>((const P *)p.b, 8 * r * threads, threadIdx.x, threads, p.H, b);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float xh = v[r][i] * rstd;
            v[r][i] = p.w ? p.b ? fmaf(xh, w[i], b[i]) : xh * w[i] : p.b ? xh + b[i] : xh;
        }
        store_columns<WIDE>((T *)p.y + row * p.ldy, 8 * r * threads, threadIdx.x, threads, p.H, v[r]);
    }
}

// Backwards: a block of up to MOST threads takes rows one after the other and holds its threads' columns of dw and db in registers, in 32 bits.
template <typename T, typename P, int EIGHTS, int MOST, bool WIDE, bool CENTRED> __global__ void __launch_bounds__(MOST) norm_backward_kernel(const NormArgs p)
{
    __shared__ float space[2][2][32];
    launch_next();
    wait_for_last();
    const int threads = blockDim.x, t = threadIdx.x;
    float dw[EIGHTS][8] = {}, db[EIGHTS][8] = {};
    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
        float x[EIGHTS][8], g[EIGHTS][8], s[2] = {0, 0};
        const float mean = CENTRED ? p.mean[row] : 0.0f, rstd = p.rstd[row];
#pragma unroll
        for (int r = 0; r < EIGHTS; r++) {
            load_columns<WIDE>((const T *)p.x + row * p.ldx, 8 * r * threads, t, threads, p.H, x[r]);
            load_columns<WIDE>((const T *)p.dy + row * p.lddy, 8 * r * threads, t, threads, p.H, g[r]);
        }
#pragma unroll
        for (int r = 0; r < EIGHTS; r++) {
            float w[8];
            if (p.w) load_columns<WIDE>((const P *)p.w, 8 * r * threads, t, threads, p.H, w);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                x[r][i] = (x[r][i] - mean) * rstd;          // (behind the row's end dy is 0)
                dw[r][i] = fmaf(g[r][i], x[r][i], dw[r][i]);
                if (CENTRED) db[r][i] += g[r][i];
                if (p.w) g[r][i] *= w[i];
                s[0] = fmaf(g[r][i], x[r][i], s[0]);
                if (CENTRED) s[1] += g[r][i];
            }
        }
        if (!p.dx) continue;
        row_sums(s, threads, space[turn]);
        const float a = s[0] / (float)p.H, m = s[1] / (float)p.H;
#pragma unroll
        for (int r = 0; r < EIGHTS; r++) {
            float d[8] = {};
            if (p.base) load_columns<WIDE>((const T *)p.base + row * p.ldbase, 8 * r * threads, t, threads, p.H, d);
#pragma unroll
            for (int i = 0; i < 8; i++) d[i] = fmaf(rstd, fmaf(-x[r][i], a, CENTRED ? g[r][i] - m : g[r][i]), d[i]);
            store_columns<WIDE>((T *)p.dx + row * p.lddx, 8 * r * threads, t, threads, p.H, d);
        }
    }
    if (!p.parts) return;
    float *part = p.parts + (int64_t)blockIdx.x * (CENTRED ? 2 : 1) * p.H;
#pragma unroll
    for (int r = 0; r < EIGHTS; r++)
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int c = column<WIDE>(8 * r * threads, t, threads, i);
            if (c < p.H) {
                part[c] = dw[r][i];
                if (CENTRED) part[p.H + c] = db[r][i];
            }
        }
}

// The blocks' sums, joined in a fixed order: 32 columns for a block, eight parts of the list side by side
template <typename O> __global__ void __launch_bounds__(256) norm_join_kernel(const NormArgs p, int both)
{
    __shared__ float space[8][33];
    launch_next();
    wait_for_last();
    const int64_t c = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31), width = (int64_t)p.H * (both ? 2 : 1);
    float sum = 0;
    if (c < width)
#pragma unroll 8
        for (int b = threadIdx.x >> 5; b < p.blocks; b += 8) sum += p.parts[b * width + c];
    space[threadIdx.x >> 5][threadIdx.x & 31] = sum;
    __syncthreads();
    if (threadIdx.x >= 32 || c >= width) return;
    sum = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) sum += space[i][threadIdx.x];
    O *out = c < p.H ? (O *)p.dw : (O *)p.db;
    if (!out) return;
    O &at = out[c < p.H ? c : c - p.H];
    at = from_float<O>(p.add ? to_float(at) + sum : sum);
}

} // namespace hapop
