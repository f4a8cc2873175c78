// Rows on their way to the experts and back, and rows of an embedding: orders by a small key, copies, and sums over what belongs
// together.  All of it moves memory; the kernels are laid out so that every thread has several 16-byte reads on their way.
#pragma once
#include "hap_values.cuh"

namespace hapop {

constexpr int MOST_CHOSEN = 32;         // experts of a row

// ---- eights of a row's columns ------------------------------------------------------------------------------------------
// Thread t of n takes eight of the 8 n columns that begin at `from`: side by side where rows begin at multiples of 16 bytes
// (WIDE), n apart where they do not, so that a warp's accesses still lie side by side.
template <bool WIDE> __device__ __forceinline__ int column(int from, int t, int n, int j) { return WIDE ? from + 8 * t + j : from + t + n * j; }
template <bool WIDE, typename T> __device__ __forceinline__ void load_columns(const T *row, int from, int t, int n, int H, float (&x)[8])
{
    if (WIDE && from + 8 * t + 8 <= H) {
        load8(row + from + 8 * t, x);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const int c = column<WIDE>(from, t, n, j);
        x[j] = c < H ? to_float(row[c]) : 0.0f;
    }
}
template <bool WIDE, typename T> __device__ __forceinline__ void store_columns(T *row, int from, int t, int n, int H, const float (&x)[8])
{
    if (WIDE && from + 8 * t + 8 <= H) {
        store8(row + from + 8 * t, x);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const int c = column<WIDE>(from, t, n, j);
        if (c < H) row[c] = from_float<T>(x[j]);
    }
}

// ---- order by a key -------------------------------------------------------------------------------------------------------
// A stable pass of a counting sort: blocks take chunks of the list, warps parts of a chunk.  A block's numbers of each key are
// counted first (order_count_kernel); then every block adds up what lies in front of its own, and its warps place their entries in
// order.  A list that one block takes needs no counting kernel.
constexpr int ORDER_WARPS = 8, MOST_KEYS = 1024;

struct OrderArgs {
    int64_t n;
    int keys, chunk;                // keys 0 .. keys - 1; entries of a block, a multiple of 32 * ORDER_WARPS
    int *counts;                    // [blocks][keys]
    // what the entries are: expert numbers, or (value, number) pairs by the digit at `shift`, made of tokens in the first pass
    const int *experts;
    int first;
    const int64_t *tokens;
    int64_t first_token;
    int V, shift, mask;
    const uint2 *from;
    uint2 *to;
    int *places;
    int64_t *offsets;
    unsigned *present;              // a bit for every value < V that the tokens have, or null
};
enum { BY_EXPERT = 0, BY_TOKEN = 1, BY_PAIR = 2 };

template <int WHAT> __device__ __forceinline__ int order_key(const OrderArgs &p, int64_t i, uint2 &entry)
{
    if (i >= p.n) return -1;
    if (WHAT == BY_EXPERT) {
        const int64_t e = (int64_t)p.experts[i] - p.first;
        return e >= 0 && e < p.keys ? (int)e : -1;
    }
    if (WHAT == BY_TOKEN) {
        const int64_t t = p.tokens[i];
        const int64_t v = (int64_t)((uint64_t)t - (uint64_t)p.first_token);
        entry = make_uint2(t >= p.first_token && v >= 0 && v < p.V ? (unsigned)v : (unsigned)p.V, (unsigned)i);
    } else entry = p.from[i];
    return entry.x >> p.shift & p.mask;
}

template <int WHAT> __global__ void __launch_bounds__(32 * ORDER_WARPS) order_count_kernel(const OrderArgs p)
{
    __shared__ int count[MOST_KEYS];
    launch_next();
    for (int d = threadIdx.x; d < p.keys; d += blockDim.x) count[d] = 0;
    __syncthreads();
    wait_for_last();
    if (WHAT == BY_TOKEN && p.present)
        for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < (p.V + 31) / 32; i += gridDim.x * blockDim.x) p.present[i] = 0;
    const int64_t from = (int64_t)blockIdx.x * p.chunk;
    for (int i = threadIdx.x; i < p.chunk; i += blockDim.x) {
        uint2 entry;
        const int key = order_key<WHAT>(p, from + i, entry);
        if (key >= 0) atomicAdd(&count[key], 1);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < p.keys; d += blockDim.x) p.counts[(int64_t)blockIdx.x * p.keys + d] = count[d];
}

template <int WHAT> __global__ void __launch_bounds__(32 * ORDER_WARPS) order_place_kernel(const OrderArgs p)
{
    extern __shared__ int at[];                             // [ORDER_WARPS][keys]: where a warp's next entry of a key goes
    __shared__ int sums[ORDER_WARPS];
    constexpr int THREADS = 32 * ORDER_WARPS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, each = p.chunk / ORDER_WARPS;
    const int64_t from = (int64_t)blockIdx.x * p.chunk + warp * each;
    launch_next();
    for (int d = threadIdx.x; d < ORDER_WARPS * p.keys; d += THREADS) at[d] = 0;
    __syncthreads();
    wait_for_last();
    if (WHAT == BY_TOKEN && p.present && gridDim.x == 1)
        for (int i = threadIdx.x; i < (p.V + 31) / 32; i += THREADS) p.present[i] = 0;
    for (int i = lane; i < each; i += 32) {
        uint2 entry;
        const int key = order_key<WHAT>(p, from + i, entry);
        if (key >= 0) atomicAdd(&at[warp * p.keys + key], 1);
    }
    __syncthreads();
    // a thread's keys follow one another: their numbers in all blocks, in the blocks ahead, and so where they begin
    const int per = (p.keys + THREADS - 1) / THREADS, key0 = threadIdx.x * per;
    int total[MOST_KEYS / THREADS], ahead[MOST_KEYS / THREADS], mine = 0;
#pragma unroll
    for (int i = 0; i < MOST_KEYS / THREADS; i++) {
        total[i] = ahead[i] = 0;
        if (i < per && key0 + i < p.keys) {
            if (gridDim.x == 1) {
                for (int w = 0; w < ORDER_WARPS; w++) total[i] += at[w * p.keys + key0 + i];
            } else {
                for (int b = 0; b < gridDim.x; b++) {
                    const int c = p.counts[(int64_t)b * p.keys + key0 + i];
                    total[i] += c, ahead[i] += b < blockIdx.x ? c : 0;
                }
            }
            mine += total[i];
        }
    }
    int before = mine;
    for (int d = 1; d < 32; d *= 2) {
        const int x = __shfl_up_sync(~0u, before, d);
        if (lane >= d) before += x;
    }
    if (lane == 31) sums[warp] = before;
    __syncthreads();
    before -= mine;
    for (int w = 0; w < warp; w++) before += sums[w];
#pragma unroll
    for (int i = 0; i < MOST_KEYS / THREADS; i++)
        if (i < per && key0 + i < p.keys) {
            if (WHAT == BY_EXPERT && blockIdx.x == 0) {
                p.offsets[key0 + i] = before;
                if (key0 + i == p.keys - 1) p.offsets[p.keys] = before + total[i];
            }
            int next = before + ahead[i];
            for (int w = 0; w < ORDER_WARPS; w++) {
                const int c = at[w * p.keys + key0 + i];
                at[w * p.keys + key0 + i] = next;
                next += c;
            }
            before += total[i];
        }
    __syncthreads();
    for (int i = 0; i < each; i += 32) {
        if (from + i >= p.n) break;
        uint2 entry;
        const int key = order_key<WHAT>(p, from + i + lane, entry);
        const unsigned same = __match_any_sync(~0u, key);
        const int ahead_of = __popc(same & ((1u << lane) - 1));
        const int place = key >= 0 ? at[warp * p.keys + key] + ahead_of : -1;
        __syncwarp();
        if (key >= 0 && ahead_of == 0) at[warp * p.keys + key] = place + __popc(same);
        __syncwarp();
        if (from + i + lane >= p.n) continue;
        if (WHAT == BY_EXPERT) p.places[from + i + lane] = place;
        else p.to[place] = entry;
        if (WHAT == BY_TOKEN && p.present && entry.x < p.V) atomicOr(&p.present[entry.x >> 5], 1u << (entry.x & 31));
    }
}

// ---- rows to the experts and back -----------------------------------------------------------------------------------------
struct RowsArgs {
    int64_t rows, placed;           // placed: rows of the experts' matrix; a place that is not among them is none
    int k, H, piece;                // piece: columns of a warp, a multiple of 256
    const int *places;              // [rows][k]
    const float *weights;           // [rows][k], null: 1
    const void *x, *y, *base;       // x: [rows][H]; y: by place
    int64_t ldx, ldy, ldbase;
    void *out;
    int64_t ldo;
    float *dweights;
};
// the column piece and the row of a warp
struct Piece { int64_t row; int from, to; };
__device__ __forceinline__ Piece piece_of(const RowsArgs &p)
{
    const int pieces = (p.H + p.piece - 1) / p.piece;
    const int64_t w = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    Piece r;
    r.row = w / pieces, r.from = (int)(w % pieces) * p.piece, r.to = min(r.from + p.piece, p.H);
    return r;
}

// out[place] = x[row]: a row is read once and written to its places.  U: values of the size, copied as they are.
template <typename U, bool WIDE> __global__ void __launch_bounds__(256) dispatch_kernel(const RowsArgs p)
{
    launch_next();
    wait_for_last();
    const Piece r = piece_of(p);
    const int lane = threadIdx.x & 31;
    if (r.row >= p.rows) return;
    const int *places = p.places + r.row * p.k;
    int place = -1;
    if (lane < p.k) place = places[lane];
    unsigned there = __ballot_sync(~0u, place >= 0 && place < p.placed);
    if (!there) return;
    const U *x = (const U *)p.x + r.row * p.ldx;
    if (WIDE) {
        constexpr int N = 16 / sizeof(U);
        for (int c = r.from + lane * N; c < r.to; c += 32 * N) {
            if (c + N <= r.to) {
                const uint4 v = *(const uint4 *)(x + c);
                for (unsigned left = there; left; left &= left - 1) *(uint4 *)((U *)p.out + (int64_t)places[__ffs(left) - 1] * p.ldo + c) = v;
            } else {
                for (unsigned left = there; left; left &= left - 1)
                    for (int i = c; i < r.to; i++) ((U *)p.out + (int64_t)places[__ffs(left) - 1] * p.ldo)[i] = x[i];
            }
        }
    } else {
        for (int c = r.from + lane; c < r.to; c += 32) {
            const U v = x[c];
            for (unsigned left = there; left; left &= left - 1) ((U *)p.out + (int64_t)places[__ffs(left) - 1] * p.ldo)[c] = v;
        }
    }
}

// out[row] = base[row] + sum_j weight_j y[place_j]
template <typename T, bool WIDE> __global__ void __launch_bounds__(256) combine_kernel(const RowsArgs p)
{
    launch_next();
    wait_for_last();
    const Piece r = piece_of(p);
    const int lane = threadIdx.x & 31;
    if (r.row >= p.rows) return;
    int place = -1;
    float weight = 1.0f;
    if (lane < p.k) {
        place = p.places[r.row * p.k + lane];
        if (p.weights) weight = p.weights[r.row * p.k + lane];
    }
    const unsigned there = __ballot_sync(~0u, place >= 0 && place < p.placed);
    for (int c = r.from; c < r.to; c += 256) {
        float sum[8] = {};
        if (p.base) load_columns<WIDE>((const T *)p.base + r.row * p.ldbase, c, lane, 32, r.to, sum);
        for (unsigned left = there; left; ) {
            float x[4][8], w[4];
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const int j = left ? __ffs(left) - 1 : -1;
                left &= left - 1;
                const int at = __shfl_sync(~0u, place, j & 31);
                w[u] = __shfl_sync(~0u, weight, j & 31);
                if (j >= 0) load_columns<WIDE>((const T *)p.y + (int64_t)at * p.ldy, c, lane, 32, r.to, x[u]);
                else {
                    w[u] = 0;
#pragma unroll
                    for (int i = 0; i < 8; i++) x[u][i] = 0;
                }
            }
#pragma unroll
            for (int u = 0; u < 4; u++)
#pragma unroll
                for (int i = 0; i < 8; i++) sum[i] = fmaf(w[u], x[u][i], sum[i]);
        }
        store_columns<WIDE>((T *)p.out + r.row * p.ldo, c, lane, 32, r.to, sum);
    }
}

// dy[place_j] = weight_j dout[row] and dweight_j = <dout[row], y[place_j]>, a block for each row: dout is read once, y once.
template <typename T, bool WIDE> __global__ void __launch_bounds__(256) combine_backward_kernel(const RowsArgs p)
{
    __shared__ float parts[8][MOST_CHOSEN];
    launch_next();
    wait_for_last();
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int *places = p.places + row * p.k;
    for (int j0 = 0; j0 < p.k; j0 += 8) {                   // (dout again, from L1, where there are more than eight)
        float dot[8] = {};
        for (int c = 0; c < p.H; c += 8 * blockDim.x) {
            float d[8];
            load_columns<WIDE>((const T *)p.x + row * p.ldx, c, threadIdx.x, blockDim.x, p.H, d);
#pragma unroll
            for (int u = 0; u < 8; u++) {
                if (j0 + u >= p.k) break;
                const int at = places[j0 + u];
                if (at < 0 || at >= p.placed) continue;
                if (p.dweights) {
                    float y[8];
                    load_columns<WIDE>((const T *)p.y + (int64_t)at * p.ldy, c, threadIdx.x, blockDim.x, p.H, y);
#pragma unroll
                    for (int i = 0; i < 8; i++) dot[u] = fmaf(y[i], d[i], dot[u]);
                }
                if (p.out) {
                    const float w = p.weights ? p.weights[row * p.k + j0 + u] : 1.0f;
                    float x[8];
#pragma unroll
                    for (int i = 0; i < 8; i++) x[i] = w * d[i];
                    store_columns<WIDE>((T *)p.out + (int64_t)at * p.ldo, c, threadIdx.x, blockDim.x, p.H, x);
                }
            }
        }
        if (!p.dweights) continue;
#pragma unroll
        for (int u = 0; u < 8; u++) {
#pragma unroll
            for (int s = 16; s; s /= 2) dot[u] += __shfl_xor_sync(~0u, dot[u], s);
            if (lane == 0 && j0 + u < p.k) parts[warp][j0 + u] = dot[u];
        }
    }
    if (!p.dweights) return;
    __syncthreads();
    if (threadIdx.x < p.k) {
        float sum = 0;
        for (int w = 0; w < warps; w++) sum += parts[w][threadIdx.x];
        p.dweights[row * p.k + threadIdx.x] = sum;
    }
}

// ---- embedding --------------------------------------------------------------------------------------------------------------
struct EmbeddingArgs {
    int64_t n, first;
    int64_t ldw, ldx, ldo;
    int H, piece, V, chunk, accumulate;
    float scale;
    const int64_t *tokens;
    const void *w, *x;              // x: the gradient dy
    void *out;
    const uint2 *sorted;            // (row of w, number of the token) by row; those of no row behind them
    float *parts;                   // [chunks][2][H]: sums of a chunk's first and last row, where they are of more than one chunk
    const unsigned *present;
};

template <typename T, bool WIDE> __global__ void __launch_bounds__(256) embedding_kernel(const EmbeddingArgs p)
{
    launch_next();
    wait_for_last();
    const int pieces = (p.H + p.piece - 1) / p.piece, lane = threadIdx.x & 31;
    const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), row = w / pieces;
    if (row >= p.n) return;
    const int from = (int)(w % pieces) * p.piece, to = min(from + p.piece, p.H);
    const int64_t t = p.tokens[row], v = (int64_t)((uint64_t)t - (uint64_t)p.first);
    const bool there = t >= p.first && v >= 0 && v < p.V;
    T *out = (T *)p.out + row * p.ldo;
    const T *in = (const T *)p.w + (there ? v : 0) * p.ldw;
    for (int c = from; c < to; c += 256) {
        float x[8] = {};
        if (there) load_columns<WIDE>(in, c, lane, 32, to, x);
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] *= p.scale;
        store_columns<WIDE>(out, c, lane, 32, to, x);
    }
}

// Rows of the gradient that no token has
template <typename O, bool WIDE> __global__ void __launch_bounds__(256) embedding_clear_kernel(const EmbeddingArgs p)
{
    launch_next();
    wait_for_last();
    const int lane = threadIdx.x & 31;
    const float zero[8] = {};
    for (int64_t v = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); v < p.V; v += (int64_t)gridDim.x * 8) {
        if (p.present[v >> 5] >> (v & 31) & 1) continue;
        for (int c = 0; c < p.H; c += 256) store_columns<WIDE>((O *)p.out + v * p.ldo, c, lane, 32, p.H, zero);
    }
}

template <typename O, bool WIDE> __device__ __forceinline__ void embedding_put(const EmbeddingArgs &p, unsigned v, int c, const float (&sum)[8])
{
    O *out = (O *)p.out + (int64_t)v * p.ldo;
    float x[8] = {};
    if (p.accumulate) load_columns<WIDE>(out, c, threadIdx.x, blockDim.x, p.H, x);
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = fmaf(sum[i], p.scale, x[i]);
    store_columns<WIDE>(out, c, threadIdx.x, blockDim.x, p.H, x);
}

// Sums of dy over the tokens of a row of w: blocks take chunks of the sorted list and eights of columns.  A row whose tokens are of
// one chunk is finished here; sums of a part of a row go to `parts` and are joined in order.
template <typename T, typename O, bool WIDE> __global__ void __launch_bounds__(256) embedding_sum_kernel(const EmbeddingArgs p)
{
    launch_next();
    wait_for_last();
    const int64_t from = (int64_t)blockIdx.x * p.chunk, to = min(from + p.chunk, p.n);
    const int c = blockIdx.y * blockDim.x * 8;
    const uint2 *s = p.sorted;
    unsigned v = s[from].x;
    if (v >= p.V) return;
    bool first = from > 0 && s[from - 1].x == v;            // the row began in front of this chunk
    const unsigned behind = to < p.n ? s[to].x : p.V;
    float sum[8] = {};
    auto put = [&](bool last) {
        if (first || last) {
            float *part = p.parts + ((int64_t)blockIdx.x * 2 + (first ? 0 : 1)) * p.H;
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const int at = column<WIDE>(c, threadIdx.x, blockDim.x, j);
                if (at < p.H) part[at] = sum[j];
            }
        } else embedding_put<O, WIDE>(p, v, c, sum);
    };
    for (int64_t i = from; i < to; i += 4) {
        float x[4][8];
        unsigned of[4];
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const uint2 e = i + u < to ? s[i + u] : make_uint2(p.V, 0);
            of[u] = e.x;
            if (e.x < p.V) load_columns<WIDE>((const T *)p.x + (int64_t)e.y * p.ldx, c, threadIdx.x, blockDim.x, p.H, x[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; u++) {
            if (of[u] != v) {
                if (v < p.V) put(false);
                v = of[u], first = false;
#pragma unroll
                for (int j = 0; j < 8; j++) sum[j] = 0;
            }
            if (v < p.V)
#pragma unroll
                for (int j = 0; j < 8; j++) sum[j] += x[u][j];
        }
    }
    if (v < p.V) put(v == behind);
}

template <typename O, bool WIDE> __global__ void __launch_bounds__(256) embedding_join_kernel(const EmbeddingArgs p)
{
    launch_next();
    wait_for_last();
    // rows that begin in this chunk and go on in the next
    const int64_t chunks = (p.n + p.chunk - 1) / p.chunk, from = (int64_t)blockIdx.x * p.chunk, to = from + p.chunk;
    if (to >= p.n) return;
    const unsigned v = p.sorted[to].x;
    if (v >= p.V || p.sorted[to - 1].x != v) return;
    if (p.sorted[from].x == v && from > 0 && p.sorted[from - 1].x == v) return;
    int64_t lo = blockIdx.x + 1, hi = chunks;               // the last chunk that begins with the row
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) / 2;
        if (p.sorted[mid * p.chunk].x == v) lo = mid; else hi = mid;
    }
    const int c = blockIdx.y * blockDim.x * 8;
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const int at = column<WIDE>(c, threadIdx.x, blockDim.x, j);
        sum[j] = at < p.H ? p.parts[((int64_t)blockIdx.x * 2 + 1) * p.H + at] : 0.0f;
    }
#pragma unroll 4
    for (int64_t b = blockIdx.x + 1; b <= lo; b++)
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int at = column<WIDE>(c, threadIdx.x, blockDim.x, j);
            if (at < p.H) sum[j] += p.parts[b * 2 * p.H + at];
        }
    embedding_put<O, WIDE>(p, v, c, sum);
}

} // namespace hapop
