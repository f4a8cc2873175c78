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
    int ahead;                      // backwards: 1 where the next row is brought while one is worked on
    float eps, inverse;             // inverse: 1 / H, rounded: a product is off by a unit more than a quotient and takes one instruction
    const void *x, *w, *b, *dy, *base;
    int64_t ldx, ldy, lddy, ldbase, lddx;
    void *y, *dx, *dw, *db;
    float *mean, *rstd;             // forwards written, backwards read
    float *parts;                   // [blocks][1 or 2][H]
};

// Sums over a row's threads: of a warp, or of a block's warps through shared memory, where every thread reads all of them.
template <int N> __device__ __forceinline__ void row_sums(float (&s)[N], int threads, float (*space)[32])
{
#pragma unroll
    for (int i = 0; i < N; i++)
#pragma unroll
        for (int d = 16; d; d /= 2) s[i] += __shfl_xor_sync(~0u, s[i], d);
    if (threads <= 32) return;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; i++) space[i][threadIdx.x >> 5] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++) s[i] = 0;
    for (int w = 0; w < threads / 32; w += 4)               // (a row's warps are a multiple of four here, or the rest is 0)
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float4 x = *(const float4 *)&space[i][w];
            s[i] += (x.x + x.y) + (x.z + x.w);
        }
}

// A thread's columns of rows that are `step` values apart, brought to shared memory one row after the other, where it alone reads them:
// 0 behind the row's end.
template <typename T, int EIGHTS, bool WIDE> struct Rows {
    const T *row;
    int64_t step;
    __device__ __forceinline__ Rows(const void *x, int64_t ld, int64_t first, int64_t by, int t) : row((const T *)x + first * ld + (WIDE ? 8 * t : t)), step(by * ld) {}
    __device__ __forceinline__ void bring(T *to, int t, int n, int H)
    {
        if constexpr (WIDE) {
#pragma unroll
            for (int r = 0; r < EIGHTS; r++) {
                const int c = 8 * r * n, there = c + 8 * t < H ? 16 : 0;
                const T *from = row + (there ? c : -8 * t);
                copy16(to + c + 8 * t, from, there);
                if (sizeof(T) == 4) copy16(to + c + 8 * t + 4, from + 4, there);
            }
        } else {
#pragma unroll
            for (int r = 0; r < 8 * EIGHTS; r++) to[t + n * r] = t + n * r < H ? row[n * r] : from_float<T>(0.0f);
        }
        row += step;
    }
};
// and what has come: whole eights, whatever H is
template <bool WIDE, typename T> __device__ __forceinline__ Eight brought(const T *from, int first, int t, int n)
{
    if constexpr (WIDE) return load_eight(from + first + 8 * t);
    else {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; j++) x[j] = to_float(from[first + t + n * j]);
        return {{pair(x[0], x[1]), pair(x[2], x[3]), pair(x[4], x[5]), pair(x[6], x[7])}};
    }
}
// A thread's columns of w in shared memory, or `none` of each: read by itself alone, without a condition
template <bool WIDE, typename P> __device__ __forceinline__ void keep_columns(P *to, const void *w, int all, int t, int n, int H, float none)
{
    const P fill = from_float<P>(none);
    for (int r = 0; r < all; r += 8 * n) {
        if (WIDE && w && r + 8 * t < H) {
#pragma unroll
            for (int i = 0; i < sizeof(P) / 2; i++) ((uint4 *)(to + r + 8 * t))[i] = ((const uint4 *)((const P *)w + r + 8 * t))[i];
            continue;
        }
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int c = column<WIDE>(r, t, n, j);
            to[c] = w && c < H ? ((const P *)w)[c] : fill;
        }
    }
}
// 1 / sqrt(x) to a unit in the last place: the approximation and a step of Newton's (a root and a quotient to nearest are six times as
// many instructions, which every thread of a row has to make)
__device__ __forceinline__ float inverse_root(float x)
{
    const float y = rsqrtf(x), z = y * fmaf(-0.5f * x * y, y, 1.5f);
    return x > 0.0f && x < INFINITY ? z : y;
}
// A thread's columns of w, or `none` of each.  Behind the row's end they are those of column 0, where they meet what is 0 or is not written.
template <bool WIDE, typename P> __device__ __forceinline__ Eight weights_of(const void *w, int from, int t, int n, int H, float none)
{
    if (!w) return eight_of(none);
    if constexpr (WIDE) return load_eight((const P *)w + (from + 8 * t < H ? from + 8 * t : 0));
    else {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; j++) x[j] = to_float(((const P *)w)[from + t + n * j < H ? from + t + n * j : 0]);
        return {{pair(x[0], x[1]), pair(x[2], x[3]), pair(x[4], x[5]), pair(x[6], x[7])}};
    }
}

// Forwards: blockDim.x threads take a row, EIGHTS eights of columns each (blockDim.y rows of one warp each in a block, where a row is
// that short), and then the rows that are gridDim.x blocks further.  RING: the next row is brought while one is worked on, so that
// memory is never idle between the two sums and the write; without it for few rows, whose latency counts.  32760 rows of 5120 in 16 bits:
// 137 us, 4.9 TB/s; 326 instructions for a warp's 512 columns, where ones for absent weights and zeros behind a row's end are
// values in shared memory like others (as conditions they were 406, and 235 us).  Six warps of four eights instead of ten of two:
// fewer instructions, but 53 us against 45 for 8192 rows.
template <typename T, typename P, int EIGHTS, bool RING, bool WIDE, bool CENTRED> __global__ void __launch_bounds__(1024) norm_kernel(const NormArgs p)
{
    extern __shared__ __align__(16) char ring[];            // w, b; [blockDim.y][2][8 EIGHTS threads]
    __shared__ __align__(16) float space[2][2][32];
    const int threads = blockDim.x, t = threadIdx.x, all = 8 * EIGHTS * threads;
    launch_next();
    if (threadIdx.y == 0)
        for (int i = t; i < 128; i += threads) (&space[0][0][0])[i] = 0;
    __syncthreads();
    wait_for_last();
    int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const int64_t step = (int64_t)gridDim.x * blockDim.y;
    P *w_kept = (P *)ring, *b_kept = w_kept + blockDim.y * all;
    T *stage = (T *)(RING ? (void *)(b_kept + blockDim.y * all) : ring) + threadIdx.y * 2 * all;
    w_kept += threadIdx.y * all, b_kept += threadIdx.y * all;
    if (RING) keep_columns<WIDE>(w_kept, p.w, all, t, threads, p.H, 1.0f), keep_columns<WIDE>(b_kept, p.b, all, t, threads, p.H, 0.0f);
    Rows<T, EIGHTS, WIDE> x(p.x, p.ldx, row, step, t);
    auto inside = [&](int r, int i) { return column<WIDE>(8 * r * threads, t, threads, WIDE ? 0 : i) < p.H; };
    if (RING && row < p.rows) x.bring(stage, t, threads, p.H);
    end_copies();
    for (int turn = 0; row < p.rows; row += step, turn ^= 1) {              // (whole warps; whole blocks, where a row has several)
        Eight v[EIGHTS];
        if (RING) {
            if (row + step < p.rows) x.bring(stage + (turn ^ 1) * all, t, threads, p.H);
            end_copies();
            copies_arrived<1>();
        }
#pragma unroll
        for (int r = 0; r < EIGHTS; r++)
            v[r] = RING ? brought<WIDE>(stage + turn * all, 8 * r * threads, t, threads) : load_columns<WIDE>((const T *)p.x + row * p.ldx, 8 * r * threads, t, threads, p.H);
        float mean = 0, s[1];
        if (CENTRED) {
            Pair sum = pair(0.0f);
#pragma unroll
            for (int r = 0; r < EIGHTS; r++)
#pragma unroll
                for (int i = 0; i < 4; i++) sum = sum + v[r].v[i];
            s[0] = sum_of(sum);
            row_sums(s, threads, &space[0][turn]);
            mean = s[0] * p.inverse;
        }
        Pair squares = pair(0.0f);
#pragma unroll
        for (int r = 0; r < EIGHTS; r++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if (CENTRED) {
                    v[r].v[i] = v[r].v[i] + pair(-mean);
                    if (p.H != all && (WIDE ? !inside(r, 0) : !inside(r, 2 * i + 1))) {    // behind the row's end the differences are 0 too
                        const float2 f = both(v[r].v[i]);
                        v[r].v[i] = pair(!WIDE && inside(r, 2 * i) ? f.x : 0.0f, 0.0f);
                    }
                }
                squares = fma2(v[r].v[i], v[r].v[i], squares);
            }
        s[0] = sum_of(squares);
        row_sums(s, threads, &space[1][turn]);
        const float rstd = inverse_root(fmaf(s[0], p.inverse, p.eps));
        if (t == 0) {
            if (CENTRED && p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
#pragma unroll
        for (int r = 0; r < EIGHTS; r++) {
            const Eight w = RING ? brought<WIDE>(w_kept, 8 * r * threads, t, threads) : weights_of<WIDE, P>(p.w, 8 * r * threads, t, threads, p.H, 1.0f);
            const Eight b = RING ? brought<WIDE>(b_kept, 8 * r * threads, t, threads) : weights_of<WIDE, P>(p.b, 8 * r * threads, t, threads, p.H, 0.0f);
#pragma unroll
            for (int i = 0; i < 4; i++) v[r].v[i] = fma2(v[r].v[i] * pair(rstd), w.v[i], b.v[i]);
            store_columns<WIDE>((T *)p.y + row * p.ldy, 8 * r * threads, t, threads, p.H, v[r]);
        }
    }
}

// Backwards: a row's threads take rows one after the other, the next one on its way meanwhile, and hold their columns' sums of dw and
// db in registers, in 32 bits.  What has arrived is read twice, for the sums and for dx.  32760 rows of 5120 in 16 bits with base: 240 us,
// 5.6 TB/s (rows read into registers when their turn comes: 640).  Up to 5120 columns two blocks or more share a multiprocessor and
// hide each other's barriers; above one is alone there, and above 7680 in 32 bits the next row is not brought ahead.  Without base, with
// a mean, 8192 rows in 16 bits: of 5120 72 us, 6144 88, 7168 and 8192 107; 4096 of 12288 152, of 16384 186 (1024 threads with 64
// registers, which spill); in 32 bits 8192 of 5120 166, 4096 of 8192 139, of 16384 297.
template <typename T, typename P, int EIGHTS, int MOST, bool WIDE, bool CENTRED> __global__ void __launch_bounds__(MOST) norm_backward_kernel(const NormArgs p)
{
    extern __shared__ __align__(16) char ring[];            // w; [blockDim.y][1 + ahead][x, dy, base where it fits][8 EIGHTS threads]
    __shared__ __align__(16) float space[2][2][32];
    const int threads = blockDim.x, t = threadIdx.x, all = 8 * EIGHTS * threads;
    constexpr int three = MOST < 1024 ? 3 : 2;              // (long rows leave no shared memory for base)
    launch_next();
    if (threadIdx.y == 0)
        for (int i = t; i < 128; i += threads) (&space[0][0][0])[i] = 0;
    __syncthreads();
    wait_for_last();
    const int64_t first = (int64_t)blockIdx.x * blockDim.y + threadIdx.y, step = (int64_t)gridDim.x * blockDim.y;
    P *w_kept = (P *)ring + threadIdx.y * all;
    T *stage = (T *)((P *)ring + blockDim.y * all) + threadIdx.y * (1 + p.ahead) * three * all;
    keep_columns<WIDE>(w_kept, p.w, all, t, threads, p.H, 1.0f);
    if (three == 3 && !p.base)
        for (int s = 0; s <= p.ahead; s++) keep_columns<WIDE>(stage + (s * three + 2) * all, nullptr, all, t, threads, 0, 0.0f);
    Rows<T, EIGHTS, WIDE> rx(p.x, p.ldx, first, step, t), rdy(p.dy, p.lddy, first, step, t), rbase(p.base, p.ldbase, first, step, t);
    auto bring = [&](int turn) {
        T *to = stage + (turn & p.ahead) * three * all;
        rx.bring(to, t, threads, p.H), rdy.bring(to + all, t, threads, p.H);
        if (three == 3 && p.base) rbase.bring(to + 2 * all, t, threads, p.H);
    };
    Eight dw[EIGHTS], db[EIGHTS];
#pragma unroll
    for (int r = 0; r < EIGHTS; r++) dw[r] = db[r] = eight_of(0.0f);
    float mean = 0, rstd = 0;
    if (first < p.rows) {
        bring(0);
        if (CENTRED) mean = p.mean[first];
        rstd = p.rstd[first];
    }
    end_copies();
    int turn = 0;
    for (int64_t row = first; row < p.rows; row += step, turn ^= 1) {
        float next_mean = 0, next_rstd = 0;
        if (row + step < p.rows) {
            if (p.ahead) bring(turn ^ 1);
            if (CENTRED) next_mean = p.mean[row + step];
            next_rstd = p.rstd[row + step];
        }
        end_copies();
        if (p.ahead) copies_arrived<1>();
        else copies_arrived<0>();
        const T *here = stage + (turn & p.ahead) * three * all;
        const Pair scale = pair(rstd), shift = pair(-mean);                 // (x - mean first: differences of near values are exact)
        Pair by_xh = pair(0.0f), plain = pair(0.0f);
#pragma unroll
        for (int r = 0; r < EIGHTS; r++) {
            const Eight x = brought<WIDE>(here, 8 * r * threads, t, threads), g = brought<WIDE>(here + all, 8 * r * threads, t, threads);
            const Eight w = brought<WIDE>(w_kept, 8 * r * threads, t, threads);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const Pair xh = (CENTRED ? x.v[i] + shift : x.v[i]) * scale, gw = g.v[i] * w.v[i];       // (behind the row's end dy is 0)
                dw[r].v[i] = fma2(g.v[i], xh, dw[r].v[i]);
                by_xh = fma2(gw, xh, by_xh);
                if (CENTRED) db[r].v[i] = db[r].v[i] + g.v[i], plain = plain + gw;
            }
        }
        if (p.dx) {
            float s[CENTRED ? 2 : 1];
            s[0] = sum_of(by_xh);
            if (CENTRED) s[CENTRED] = sum_of(plain);
            row_sums(s, threads, space[turn]);
            // g w - mean(g w) - xh mean(g w xh)
            const Pair by_x = pair(-s[0] * p.inverse * rstd), rest = pair(CENTRED ? -s[CENTRED] * p.inverse : 0.0f);
#pragma unroll
            for (int r = 0; r < EIGHTS; r++) {
                const Eight x = brought<WIDE>(here, 8 * r * threads, t, threads), g = brought<WIDE>(here + all, 8 * r * threads, t, threads);
                const Eight w = brought<WIDE>(w_kept, 8 * r * threads, t, threads);
                Eight d = three == 3 ? brought<WIDE>(here + 2 * all, 8 * r * threads, t, threads)
                        : p.base ? load_columns<WIDE>((const T *)p.base + row * p.ldbase, 8 * r * threads, t, threads, p.H) : eight_of(0.0f);
#pragma unroll
                for (int i = 0; i < 4; i++) d.v[i] = fma2(fma2(g.v[i], w.v[i], CENTRED ? fma2(x.v[i] + shift, by_x, rest) : x.v[i] * by_x), scale, d.v[i]);
                store_columns<WIDE>((T *)p.dx + row * p.lddx, 8 * r * threads, t, threads, p.H, d);
            }
        }
        mean = next_mean, rstd = next_rstd;
        if (!p.ahead && row + step < p.rows) bring(0);
    }
    if (!p.parts) return;
    float *part = p.parts + first * (CENTRED ? 2 : 1) * p.H;
#pragma unroll
    for (int r = 0; r < EIGHTS; r++) {
        store_columns<WIDE>(part, 8 * r * threads, t, threads, p.H, dw[r]);
        if (CENTRED) store_columns<WIDE>(part + p.H, 8 * r * threads, t, threads, p.H, db[r]);
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
