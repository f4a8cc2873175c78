// Products of the training operators: tiles of grouped matrix products, their scheduling over the groups and what happens to
// a finished tile.  Three forms share everything here:
//   NT  out[i][n] = sum_k a[i][k] w_e[n][k]      rows i of group e (forward; logits)
//   NN  out[i][n] = sum_k a[i][k] w_e[k][n]      (gradient of the input)
//   TN  out_e[m][n] = sum over rows i of group e of a[i][m] b[i][n]   (gradient of the weight)
// Group e holds rows offsets[e] .. offsets[e+1]; without offsets there is one group of all rows.
#pragma once
#include "hap_values.cuh"

namespace hapop {

enum Form { NT = 0, NN = 1, TN = 2 };
enum Epilogue {
    STORE = 0,      // out = scale * acc (+ out)
    GATED = 1,      // tile columns are 128 of g and the same 128 of u: keep them, h = silu(g) u
    GATED_BACK = 2, // acc is dh: dg, du and h from it and the kept g, u
    LSE = 3,        // logits: the row's maximum and sum of exponentials over the tile's columns, the target's logit
    DLOGIT = 4,     // logits again: (softmax - one-hot) * 2^15 in 16 bits
    SUM32 = 5,      // gradient of the loss's input over several pieces of the vocabulary: kept in 32 bits between them
    STORE32 = 6     // STORE to fp32
};

constexpr int MAX_GROUPS = 1024;
constexpr int TILE_N = 256;         // columns of a tile
constexpr int PART_N = 128;         // columns that one partial result of the loss's statistics covers, in every variant
constexpr int BAND = 16;            // row tiles of a group that are worked on side by side, for reuse in L2
// softmax gradients are held in 16 bits times this: fp16's normal range ends at 6e-5, a probability of a large vocabulary
// is smaller; 2^15 keeps 1 below 65504 and 2e-9 normal.  The factor is a power of two and leaves with the gradient's scale.
constexpr float DLOGIT_SCALE = 32768.0f;

struct Args {
    const int64_t *offsets;         // [groups + 1] or null
    int groups, rows;               // rows: of a (and of b in TN)
    int mdim;                       // TN: rows of out_e
    int ncols;                      // columns of out (GATED: columns of h)
    int kdim;                       // contraction in NT, NN
    const void *a, *b;              // operands as the plain variant reads them
    int64_t lda, ldb, bgroup;       // bgroup: distance of two groups' w
    // epilogue
    void *out;
    int64_t ldo, ogroup;            // ogroup: distance of two groups' out (TN)
    int accumulate, out_mapped;     // out_mapped: a tensor map describes out (TN, STORE32)
    const float *scale;             // device scalar, or null: 1
    float scale_by;                 // times this
    const void *gu;                 // GATED_BACK: kept g | u
    int kept_mapped;                // a tensor map describes it
    int64_t ldgu;
    void *h;
    int64_t ldh;
    const int64_t *target;          // LSE, DLOGIT
    int64_t ignore;
    int64_t vocab;
    int col0;                       // first column's place in the vocabulary
    float2 *part;                   // [pieces of PART_N columns][rows]
    float *at_target;               // [rows]
    const float *lse;
    float *residual;                // DLOGIT, SUM32: [rows] what rounding took from the target's element
    int64_t low;                    // DLOGIT: distance of what rounding took from all elements, or 0
    const void *w;                  // SUM32: the whole weight
    int64_t ldw;
    float *acc32;                   // SUM32: [rows][ncols]
    int first, last;
    int splits, split_k;            // SUM32: the contraction in this many parts of split_k, each with sums of its own in acc32
};

// 32 consecutive values of a row, as many as the row has: in 16-byte pieces where the address allows
template <typename T> __device__ __forceinline__ void store32(T *p, const float (&v)[32], int n)
{
    if (n >= 32 && ((uintptr_t)p & 15) == 0) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; i++) ((float4 *)p)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++)
                ((uint4 *)p)[i] = make_uint4(pack2(v[8 * i], v[8 * i + 1], T()), pack2(v[8 * i + 2], v[8 * i + 3], T()),
                                             pack2(v[8 * i + 4], v[8 * i + 5], T()), pack2(v[8 * i + 6], v[8 * i + 7], T()));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 32; i++)
        if (i < n) p[i] = from_float<T>(v[i]);
}
template <typename T> __device__ __forceinline__ void load32(const T *p, float (&v)[32], int n)
{
    if (n >= 32 && ((uintptr_t)p & 15) == 0) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float4 x = ((const float4 *)p)[i];
                v[4 * i] = x.x, v[4 * i + 1] = x.y, v[4 * i + 2] = x.z, v[4 * i + 3] = x.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint4 x = ((const uint4 *)p)[i];
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float2 f = unpack2(w[j], T());
                    v[8 * i + 2 * j] = f.x, v[8 * i + 2 * j + 1] = f.y;
                }
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 32; i++) v[i] = i < n ? to_float(p[i]) : 0.0f;
}

// 2^x and 1 / x in one instruction each, off by two units in the last place; below 2^-126 they are 0
__device__ __forceinline__ float quick_exp2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float quick_inverse(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// 1 / (1 + exp(-g)): 0 where the exponential is infinite.  (With __expf and __fdividef, which also take care of what lies below
// 2^-126: 198 us instead of 193 for the backward pass of 64 experts with 32760 rows, 2048 x 1024.)
__device__ __forceinline__ float sigma(float g) { return quick_inverse(1.0f + quick_exp2(g * -1.4426950408889634f)); }
// h = silu(g) u
__device__ __forceinline__ float gate(float g, float u) { return g * sigma(g) * u; }
// from g, u and dh: g becomes h, u becomes du, dh becomes dg.  With s = sigma(g): dg = dh u (s + g s (1 - s)), du = dh g s, h = g s u
__device__ __forceinline__ void gate_back(float &g, float &u, float &dh)
{
    const float s = sigma(g), gs = g * s, du = dh * gs;
    dh = dh * u * fmaf(gs, 1.0f - s, s);
    g = gs * u;
    u = du;
}

// How a warp's 32 rows of 32 16-bit values (row = lane) go to and come from memory: through 2 KB of shared memory, so that four
// lanes take a row's 64 bytes and whole sectors are moved.  From the rows directly a 16-byte piece of every row went at a time,
// half sectors: 854 us instead of 678 for 8 weight gradients of 4096 x 14336 from 8192 rows.  Pieces of 16 bytes are swizzled over the banks.
struct WarpRows {
    char *staged;                   // null: each lane moves its own row
    int lane, live;                 // rows 0 .. live-1 exist
    __device__ __forceinline__ uint4 *piece(int row, int c) const { return (uint4 *)(staged + row * 64 + ((c ^ (row >> 1 & 3)) << 4)); }
    template <typename T> __device__ __forceinline__ bool whole(const T *first, int64_t ld, int n) const { return staged && n >= 32 && ((uintptr_t)first & 15) == 0 && ld % 8 == 0; }
    // first: column col of row 0
    template <typename T> __device__ __forceinline__ void store(T *first, int64_t ld, const float (&v)[32], int n) const
    {
        if (!whole(first, ld, n)) {
            if (lane < live) store32(first + lane * ld, v, n);
            return;
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; i++)
            *piece(lane, i) = make_uint4(pack2(v[8 * i], v[8 * i + 1], T()), pack2(v[8 * i + 2], v[8 * i + 3], T()), pack2(v[8 * i + 4], v[8 * i + 5], T()), pack2(v[8 * i + 6], v[8 * i + 7], T()));
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int r = i * 8 + (lane >> 2);
            if (r < live) *(uint4 *)(first + r * ld + (lane & 3) * 8) = *piece(r, lane & 3);
        }
    }
};

// What happens to the 32 columns col .. of 32 output rows, one for each lane of a warp, from `row0` on (in TN rows of out_e, and
// then e is its group; in SUM32 the part of the contraction).  v: the sums; v2: those of u in GATED.  The softmax statistics of a row over a tile are held in m
// (maximum) and s.  All lanes call, those of rows that do not exist too.
template <typename T, int EPI> struct RowEpilogue {
    const Args &p;
    const WarpRows w;
    const int64_t row0;
    const int e;
    const bool live;
    float m = -INFINITY, s = 0.0f;
    int64_t target = -1;            // LSE, DLOGIT: column of the row's target in this launch's columns, or outside of them
    bool kept = true;
    float lse = 0.0f, scale = 1.0f;
    __device__ __forceinline__ RowEpilogue(const Args &args, const WarpRows &w, int64_t row0, int e) : p(args), w(w), row0(row0), e(e), live(w.lane < w.live)
    {
        if constexpr (EPI == STORE || EPI == SUM32)
            if (p.scale) scale = *p.scale * p.scale_by;
        if constexpr (EPI == LSE || EPI == DLOGIT) {
            if (live) {
                const int64_t t = p.target[row0 + w.lane];
                kept = t != p.ignore && t >= 0 && t < p.vocab;
                target = t - p.col0;
                if constexpr (EPI == DLOGIT) lse = p.lse[row0 + w.lane];
            }
        }
    }
    __device__ __forceinline__ void columns(int col, float (&v)[32], float (&v2)[32])
    {
        const int n = p.ncols - col;
        if (n <= 0) return;
        if constexpr (EPI == STORE) {
#pragma unroll
            for (int i = 0; i < 32; i++) v[i] *= scale;
            T *o = (T *)p.out + e * p.ogroup + row0 * p.ldo + col;
            if (p.accumulate) {
                load32(o + w.lane * p.ldo, v2, live ? n : 0);
#pragma unroll
                for (int i = 0; i < 32; i++) v[i] += v2[i];
            }
            w.store(o, p.ldo, v, n);
        }
        if constexpr (EPI == STORE32) {         // four at a time: a whole tile's half row is in registers here
            float *o = (float *)p.out + e * p.ogroup + (row0 + w.lane) * p.ldo + col;
            if (!live) return;
            if (n >= 32 && ((uintptr_t)o & 15) == 0) {
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    float4 x = p.accumulate ? *(const float4 *)(o + i) : make_float4(0, 0, 0, 0);
                    x.x += v[i], x.y += v[i + 1], x.z += v[i + 2], x.w += v[i + 3];
                    *(float4 *)(o + i) = x;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 32; i++)
                    if (i < n) o[i] = p.accumulate ? o[i] + v[i] : v[i];
            }
        }
        if constexpr (EPI == GATED) {
            if (p.out) {
                T *o = (T *)p.out + row0 * p.ldo + col;
                w.store(o, p.ldo, v, n);
                w.store(o + p.ncols, p.ldo, v2, n);
            }
#pragma unroll
            for (int i = 0; i < 32; i++) v[i] = gate(v[i], v2[i]);
            w.store((T *)p.h + row0 * p.ldh + col, p.ldh, v, n);
        }
        if constexpr (EPI == GATED_BACK) {
            float g[32];
            const T *gu = (const T *)p.gu + (row0 + w.lane) * p.ldgu + col;
            load32(gu, g, live ? n : 0);
            load32(gu + p.ncols, v2, live ? n : 0);
#pragma unroll
            for (int i = 0; i < 32; i++) gate_back(g[i], v2[i], v[i]);
            T *o = (T *)p.out + row0 * p.ldo + col;
            w.store(o, p.ldo, v, n);
            w.store(o + p.ncols, p.ldo, v2, n);
            if (p.h) w.store((T *)p.h + row0 * p.ldh + col, p.ldh, g, n);
        }
        if constexpr (EPI == LSE) {
            float top = m;
#pragma unroll
            for (int i = 0; i < 32; i++) {
                if (i >= n) v[i] = -INFINITY;
                top = fmaxf(top, v[i]);
            }
            const float from = top == -INFINITY ? 0.0f : top * 1.4426950408889634f;
            // (the sum so far by the difference: 1 exactly while the maximum stays.  By m and `from` it would be off by from's rounding
            // each time, 1e-5 of the sum over 128 columns under a maximum of 100.)
            float sum = m == -INFINITY ? 0.0f : s * quick_exp2((m - top) * 1.4426950408889634f);
#pragma unroll
            for (int i = 0; i < 32; i++) sum += quick_exp2(fmaf(v[i], 1.4426950408889634f, -from));
            m = top, s = sum;
            if (live && target >= col && target < col + 32 && target < p.ncols) {
                float z = 0.0f;
#pragma unroll
                for (int i = 0; i < 32; i++) z = col + i == target ? v[i] : z;
                p.at_target[row0 + w.lane] = z;
            }
        }
        if constexpr (EPI == DLOGIT) {
            const float from = lse * 1.4426950408889634f;
#pragma unroll
            for (int i = 0; i < 32; i++) {
                float d = quick_exp2(fmaf(v[i], 1.4426950408889634f, -from));
                d = col + i == target ? d - 1.0f : d;
                v[i] = kept ? d * DLOGIT_SCALE : 0.0f;
            }
            T *o = (T *)p.out + row0 * p.ldo + col;
            w.store(o, p.ldo, v, n);
            const bool here = live && kept && target >= col && target < col + 32 && target < p.ncols;
            if (p.low || __any_sync(~0u, here)) {
                float r = 0.0f;
#pragma unroll
                for (int i = 0; i < 32; i++) {
                    v[i] -= to_float(from_float<T>(v[i]));
                    r = col + i == target ? v[i] : r;
                }
                if (here) p.residual[row0 + w.lane] = r;
                if (p.low) w.store(o + p.low, p.ldo, v, n);
            }
        }
        if constexpr (EPI == SUM32) {
            float *a = p.acc32 + (e * (int64_t)p.rows + row0 + w.lane) * p.ncols + col;         // e: the part
            if (!p.first) {
                load32(a, v2, live ? n : 0);
#pragma unroll
                for (int i = 0; i < 32; i++) v[i] += v2[i];
            }
            if (p.last) {
                // the target's element is most of a row, and its rounding would be most of the error: what it took comes back
                const int64_t t = live ? p.target[row0 + w.lane] : p.ignore;
                if (t != p.ignore && t >= 0 && t < p.vocab) {
                    const float r = p.residual[row0 + w.lane];
                    load32((const T *)p.w + t * p.ldw + col, v2, n);
#pragma unroll
                    for (int i = 0; i < 32; i++) v[i] = fmaf(r, v2[i], v[i]);
                }
#pragma unroll
                for (int i = 0; i < 32; i++) v[i] *= scale;
                w.store((T *)p.out + row0 * p.ldo + col, p.ldo, v, n);
            } else if (live) {
                store32(a, v, n);
            }
        }
    }
    __device__ __forceinline__ void end(int col)        // behind PART_N columns from col on
    {
        if constexpr (EPI == LSE)
            if (live && col < p.ncols) p.part[(int64_t)(col / PART_N) * p.rows + row0 + w.lane] = make_float2(m, s);
    }
};

// Tiles of all groups in one order, in which workers (blocks or pairs of blocks) take every n-th: those at work at one time share
// operands in L2.  (Groups with few rows, whose weights cost more to read than to multiply, in turns with the others instead of
// where they come: no difference, 129 us either way at 64 experts with 32768 rows by Zipf's law, 1024 -> 2048.)
// Offsets come from device memory: they are clamped to the rows and made ascending here, so that no offset can lead outside of
// the operands.
template <int BM> struct Schedule {
    int bound[MAX_GROUPS + 1];
    int first[MAX_GROUPS + 1];      // first tile of each group (NT, NN)
    struct Tile { int e, m, n, lo, hi; };

    __device__ static int row_tiles(int n) { return (n + BM - 1) / BM; }
    // the offsets, by all threads of the block; a barrier of the block follows
    __device__ void fetch(const Args &p)
    {
        for (int i = threadIdx.x; i <= p.groups; i += blockDim.x) {
            const int64_t o = p.offsets ? p.offsets[i] : i ? p.rows : 0;
            bound[i] = o < 0 ? 0 : o > p.rows ? p.rows : (int)o;
        }
    }
    // by all threads of a warp
    __device__ void build(const Args &p, int col_tiles, int lane)
    {
        int below = 0, tiles = 0;   // carried over the blocks of 32
        for (int i0 = 0; i0 <= p.groups; i0 += 32) {
            const int i = i0 + lane;
            int b = max(i <= p.groups ? bound[i] : 0, below);
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int x = __shfl_up_sync(~0u, b, d);
                if (lane >= d) b = max(b, x);
            }
            int last = __shfl_up_sync(~0u, b, 1);
            if (lane == 0) last = below;
            int t = i > 0 && i <= p.groups ? row_tiles(b - last) * col_tiles : 0;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int x = __shfl_up_sync(~0u, t, d);
                if (lane >= d) t += x;
            }
            if (i <= p.groups) bound[i] = b, first[i] = tiles + t;
            below = __shfl_sync(~0u, b, 31);
            tiles += __shfl_sync(~0u, t, 31);
        }
        __syncwarp();
    }
    __device__ int total(const Args &p, int form, int col_tiles) const { return form == TN ? p.groups * row_tiles(p.mdim) * col_tiles : first[p.groups]; }
    __device__ Tile tile(const Args &p, int form, int col_tiles, int t) const
    {
        Tile r;
        int rows;
        if (form == TN) {
            rows = p.mdim;
            const int per = row_tiles(rows) * col_tiles;
            r.e = t / per;
            t -= r.e * per;
        } else {
            int lo = 0, hi = p.groups - 1;                  // last group whose first tile is not behind t
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (first[mid] <= t) lo = mid; else hi = mid - 1;
            }
            r.e = lo;
            t -= first[lo];
            rows = bound[lo + 1] - bound[lo];
        }
        r.lo = bound[r.e], r.hi = bound[r.e + 1];
        const int mt = row_tiles(rows), band = min(mt, BAND);
        const int which = t / (band * col_tiles);
        t -= which * band * col_tiles;
        const int high = min(band, mt - which * band);
        r.n = t / high;
        r.m = which * band + t - r.n * high;
        return r;
    }
};

// ---- plain variant ----------------------------------------------------------------------------------------------------
// For operands that a tensor map cannot describe (addresses or row distances that are not multiples of 16 bytes).  Tiles of
// 32 rows and 256 columns, a thread sums 4 x 8 of them in fp32 from shared memory.
constexpr int PM = 32, PK = 16;

template <typename T, int FORM, int EPI> __global__ void __launch_bounds__(256) plain_product_kernel(const __grid_constant__ Args p)
{
    __shared__ Schedule<PM> sched;
    __shared__ float shared[PM * (TILE_N + 1)];     // the tile's sums; before that the operands' slices, which are smaller
    float (*sc)[TILE_N + 1] = (float (*)[TILE_N + 1])shared;
    float (*sa)[PM + 1] = (float (*)[PM + 1])shared, (*sb)[TILE_N + 1] = (float (*)[TILE_N + 1])(shared + PK * (PM + 1));
    const int tid = threadIdx.x;
    constexpr int BN = EPI == GATED ? TILE_N / 2 : TILE_N;
    const int col_tiles = (p.ncols + BN - 1) / BN;
    sched.fetch(p);
    __syncthreads();
    if (tid < 32) sched.build(p, col_tiles, tid);
    __syncthreads();
    const int total = sched.total(p, FORM, col_tiles);
    for (int t = blockIdx.x; t < total; t += gridDim.x) {
        const auto tile = sched.tile(p, FORM, col_tiles, t);
        const int m0 = tile.m * PM, n0 = tile.n * BN;
        const int mrows = FORM == TN ? p.mdim - m0 : tile.hi - tile.lo - m0;        // rows of out from m0 on
        const int K = FORM == TN ? tile.hi - tile.lo : p.kdim;
        const T *a = (const T *)p.a, *b = (const T *)p.b + (FORM == TN ? 0 : tile.e * p.bgroup);
        float acc[4][8] = {};
        const int tm = (tid & 7) * 4, tn = (tid >> 3);                              // columns tn + 32 j
        for (int k0 = 0; k0 < K; k0 += PK) {
            for (int i = tid; i < PM * PK; i += 256) {
                const int m = FORM == TN ? i % PM : i / PK, k = FORM == TN ? i / PM : i % PK;
                const bool in = m < mrows && k0 + k < K;
                sa[k][m] = !in ? 0.0f : to_float(FORM == TN ? a[(int64_t)(tile.lo + k0 + k) * p.lda + m0 + m] : a[(int64_t)(tile.lo + m0 + m) * p.lda + k0 + k]);
            }
            for (int i = tid; i < TILE_N * PK; i += 256) {
                const int n = FORM == NT ? i / PK : i % TILE_N, k = FORM == NT ? i % PK : i / TILE_N;
                const int col = n0 + (EPI == GATED ? n % BN : n);
                const bool in = col < p.ncols && k0 + k < K;
                const int64_t from = EPI == GATED && n >= BN ? col + p.ncols : col;
                sb[k][n] = !in ? 0.0f : to_float(FORM == NT ? b[from * p.ldb + k0 + k] : b[(int64_t)((FORM == TN ? tile.lo : 0) + k0 + k) * p.ldb + col]);
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < PK; k++) {
                float x[4];
#pragma unroll
                for (int i = 0; i < 4; i++) x[i] = sa[k][tm + i];
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const float y = sb[k][tn + 32 * j];
#pragma unroll
                    for (int i = 0; i < 4; i++) acc[i][j] = fmaf(x[i], y, acc[i][j]);
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int j = 0; j < 8; j++) sc[tm + i][tn + 32 * j] = acc[i][j];
        __syncthreads();
        // 8 threads share a row; two where its statistics run over the columns
        constexpr int SHARE = EPI == LSE ? TILE_N / PART_N : 8, EACH = BN / 32 / SHARE > 0 ? BN / 32 / SHARE : 1;
        const int r = tid & 31, c = tid >> 5;
        if (c * EACH < BN / 32 && c < SHARE) {
            RowEpilogue<T, EPI> row(p, WarpRows{nullptr, r, min(max(mrows, 0), 32)}, (FORM == TN ? 0 : (int64_t)tile.lo) + m0, FORM == TN ? tile.e : 0);
            float v[32], v2[32];
            for (int q = c * EACH; q < (c + 1) * EACH; q++) {
#pragma unroll
                for (int i = 0; i < 32; i++) v[i] = sc[r][q * 32 + i], v2[i] = EPI == GATED ? sc[r][BN + q * 32 + i] : 0.0f;
                row.columns(n0 + q * 32, v, v2);
            }
            row.end(n0 + c * PART_N);
        }
        __syncthreads();
    }
}

// ---- the loss from the pieces' statistics -----------------------------------------------------------------------------
// lse = M + log(sum_t s_t exp(m_t - M)).  A block takes 8 rows, whose statistics lie side by side, and 32 slices of the pieces.
__global__ void __launch_bounds__(256) loss_rows_kernel(const float2 *part, int pieces, int rows, const float *at_target, const int64_t *target,
                                                        int64_t ignore, int V, float *loss, float *lse)
{
    launch_next();
    wait_for_last();
    __shared__ float2 sh[32][8];
    const int r = threadIdx.x & 7, slice = threadIdx.x >> 3, row = blockIdx.x * 8 + r;
    float m = -INFINITY, s = 0.0f;
    if (row < rows) {
#pragma unroll 4
        for (int t = slice; t < pieces; t += 32) {
            const float2 x = part[(int64_t)t * rows + row];
            const float top = fmaxf(m, x.x);
            const float from = top == -INFINITY ? 0.0f : top;
            s = s * __expf(m - from) + x.y * __expf(x.x - from);
            m = top;
        }
    }
    sh[slice][r] = make_float2(m, s);
    __syncthreads();
    if (slice || row >= rows) return;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 32; i++) top = fmaxf(top, sh[i][r].x);
    const float from = top == -INFINITY ? 0.0f : top;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; i++) s += sh[i][r].y * __expf(sh[i][r].x - from);
    const float l = top + logf(s);
    lse[row] = l;
    const int64_t t = target[row];
    loss[row] = t == ignore ? 0.0f : t < 0 || t >= V ? NAN : l - at_target[row];
}

// dx of few rows from the parts of the contraction: their sum in order, what rounding took from the target's element, the scale.
template <typename T> __global__ void __launch_bounds__(256) join_parts_kernel(const __grid_constant__ Args p)
{
    launch_next();
    wait_for_last();
    const int64_t n = (int64_t)p.rows * p.ncols;
    const float f = *p.scale * p.scale_by;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
        const int64_t row = i / p.ncols, col = i - row * p.ncols, t = p.target[row];
        float x = 0.0f;
#pragma unroll 8
        for (int s = 0; s < p.splits; s++) x += p.acc32[s * n + i];
        if (t != p.ignore && t >= 0 && t < p.vocab) x = fmaf(p.residual[row], to_float(((const T *)p.w)[t * p.ldw + col]), x);
        ((T *)p.out)[row * p.ldo + col] = from_float<T>(x * f);
    }
}

} // namespace hapop
