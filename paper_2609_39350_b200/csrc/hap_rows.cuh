// Rows on their way to the experts and back, and rows of an embedding: orders by a small key, copies, and sums over what belongs
// together.  All of it moves memory; the kernels are laid out so that every thread has several 16-byte reads on their way.
#pragma once
#include "hap_values.cuh"

namespace hapop {

constexpr int MOST_CHOSEN = 32;         // experts of a row

// ---- two values at a time -------------------------------------------------------------------------------------------------
// Two values in 32 bits side by side in a register pair: one instruction adds or multiplies both, each rounded as by itself.
struct Pair { uint64_t v; };
__device__ __forceinline__ Pair pair(float x, float y) { Pair p; asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(x), "f"(y)); return p; }
__device__ __forceinline__ Pair pair(float x) { return pair(x, x); }
__device__ __forceinline__ float2 both(Pair p) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p.v)); return r; }
__device__ __forceinline__ Pair operator+(Pair a, Pair b) { Pair r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ Pair operator*(Pair a, Pair b) { Pair r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) { Pair r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }
__device__ __forceinline__ float sum_of(Pair p) { const float2 f = both(p); return f.x + f.y; }
__device__ __forceinline__ Pair pair_of(uint32_t w, __nv_bfloat16) { return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ Pair pair_of(uint32_t w, __half) { const float2 f = __half22float2(*(__half2 *)&w); return pair(f.x, f.y); }

// ---- eights of a row's columns ------------------------------------------------------------------------------------------
// Thread t of n takes eight of the 8 n columns that begin at `from`: side by side where rows begin at multiples of 16 bytes and are
// whole eights long (WIDE), n apart where they are not, so that a warp's accesses still lie side by side.
struct Eight { Pair v[4]; };
template <bool WIDE> __device__ __forceinline__ int column(int from, int t, int n, int j) { return WIDE ? from + 8 * t + j : from + t + n * j; }
__device__ __forceinline__ Eight eight_of(float x) { return {{pair(x), pair(x), pair(x), pair(x)}}; }
// eight values side by side at a multiple of 16 bytes
template <typename T> __device__ __forceinline__ Eight load_eight(const T *p)
{
    if constexpr (sizeof(T) == 4) {
        const float4 a = ((const float4 *)p)[0], b = ((const float4 *)p)[1];
        return {{pair(a.x, a.y), pair(a.z, a.w), pair(b.x, b.y), pair(b.z, b.w)}};
    } else {
        const uint4 a = *(const uint4 *)p;
        return {{pair_of(a.x, T()), pair_of(a.y, T()), pair_of(a.z, T()), pair_of(a.w, T())}};
    }
}
template <typename T> __device__ __forceinline__ void store_eight(T *p, const Eight &x)
{
    const float2 a = both(x.v[0]), b = both(x.v[1]), c = both(x.v[2]), d = both(x.v[3]);
    if constexpr (sizeof(T) == 4) {
        ((float4 *)p)[0] = make_float4(a.x, a.y, b.x, b.y);
        ((float4 *)p)[1] = make_float4(c.x, c.y, d.x, d.y);
    } else *(uint4 *)p = make_uint4(pack2(a.x, a.y, T()), pack2(b.x, b.y, T()), pack2(c.x, c.y, T()), pack2(d.x, d.y, T()));
}
// A thread's columns of a row; those behind its H are 0, or not written.
template <bool WIDE, typename T> __device__ __forceinline__ Eight load_columns(const T *row, int from, int t, int n, int H)
{
    if constexpr (WIDE) {
        if (from + 8 * t < H) return load_eight(row + from + 8 * t);
        return eight_of(0.0f);
    } else {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; j++) x[j] = from + t + n * j < H ? to_float(row[from + t + n * j]) : 0.0f;
        return {{pair(x[0], x[1]), pair(x[2], x[3]), pair(x[4], x[5]), pair(x[6], x[7])}};
    }
}
template <bool WIDE, typename T> __device__ __forceinline__ void store_columns(T *row, int from, int t, int n, int H, const Eight &x)
{
    if constexpr (WIDE) {
        if (from + 8 * t < H) store_eight(row + from + 8 * t, x);
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const float2 f = both(x.v[j / 2]);
            if (from + t + n * j < H) row[from + t + n * j] = from_float<T>(j & 1 ? f.y : f.x);
        }
    }
}

// ---- order by a key -------------------------------------------------------------------------------------------------------
// A stable pass of a counting sort.  A block takes a chunk of the list, tile by tile; a warp's entries of a tile are in its lanes'
// registers, their ranks among the warp's equal ones come from matching lanes, and one number for every warp and key says how many
// lie in the warps ahead.  Several blocks count their chunks first (order_count_kernel; a pass that places also counts for the next
// one), and each adds up what lies in front of its own.  A list of one tile needs the placing kernel alone.  Bound by latency: three
// rounds of reads and barriers (196602 entries: 4 and 5 us; with a warp's entries read one after the other 6 and 9).
constexpr int ORDER_WARPS = 16, ORDER_ITEMS = 4, ORDER_TILE = 32 * ORDER_WARPS * ORDER_ITEMS, MOST_KEYS = 1024;

struct OrderArgs {
    int64_t n;
    int keys, chunk;                // keys 0 .. keys - 1; entries of a block, a multiple of ORDER_TILE
    int *counts;                    // [passes][blocks][keys], of which this pass is number `pass`
    int pass, passes;
    // what the entries are: expert numbers, or (value, number) pairs by the digit at `shift`, made of tokens in the first pass
    const int *experts;
    int first;
    const int64_t *tokens;
    int64_t first_token;
    int V, shift, bits;
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
    return entry.x >> p.shift & (1 << p.bits) - 1;
}

template <int WHAT> __global__ void __launch_bounds__(32 * ORDER_WARPS) order_count_kernel(const OrderArgs p)
{
    __shared__ int count[MOST_KEYS];
    constexpr int THREADS = 32 * ORDER_WARPS;
    launch_next();
    for (int d = threadIdx.x; d < p.keys; d += THREADS) count[d] = 0;
    __syncthreads();
    wait_for_last();
    const int all = gridDim.x * THREADS, me = blockIdx.x * THREADS + threadIdx.x;
    if (WHAT == BY_TOKEN && p.present)
        for (int i = me; i < (p.V + 31) / 32; i += all) p.present[i] = 0;
    for (int i = me; i < (p.passes - 1) * (int)gridDim.x * p.keys; i += all) p.counts[gridDim.x * p.keys + i] = 0;      // the later passes'
    const int64_t from = (int64_t)blockIdx.x * p.chunk;
    for (int i = threadIdx.x; i < p.chunk; i += THREADS * ORDER_ITEMS) {
        int key[ORDER_ITEMS];
#pragma unroll
        for (int u = 0; u < ORDER_ITEMS; u++) {
            uint2 entry;
            key[u] = order_key<WHAT>(p, from + i + u * THREADS, entry);
        }
#pragma unroll
        for (int u = 0; u < ORDER_ITEMS; u++)
            if (key[u] >= 0) atomicAdd(&count[key[u]], 1);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < p.keys; d += THREADS) p.counts[blockIdx.x * p.keys + d] = count[d];
}

template <int WHAT> __global__ void __launch_bounds__(32 * ORDER_WARPS) order_place_kernel(const OrderArgs p)
{
    extern __shared__ uint16_t at[];                        // [ORDER_WARPS][keys, even]: entries of a key in a warp, then in those ahead
    __shared__ int base[MOST_KEYS], total[MOST_KEYS], sums[ORDER_WARPS];     // where a key's next entry goes; its number
    constexpr int THREADS = 32 * ORDER_WARPS, PER = MOST_KEYS / THREADS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, width = (p.keys + 1) & ~1, blocks = gridDim.x;
    launch_next();
    for (int d = threadIdx.x; d < p.keys; d += THREADS) base[d] = total[d] = 0;
    __syncthreads();
    wait_for_last();
    if (WHAT == BY_TOKEN && p.present && blocks == 1)
        for (int i = threadIdx.x; i < (p.V + 31) / 32; i += THREADS) p.present[i] = 0;
    if (blocks > 1) {                                       // numbers of all blocks, and of the blocks ahead
        const int *counts = p.counts + (int64_t)p.pass * blocks * p.keys;
        const int ahead = blockIdx.x * p.keys, all = blocks * p.keys;
#pragma unroll 4
        for (int i = threadIdx.x; i < all; i += THREADS) {
            const int c = counts[i], d = i % p.keys;
            if (c) {
                atomicAdd(&total[d], c);
                if (i < ahead) atomicAdd(&base[d], c);
            }
        }
    }
    int *next = p.pass + 1 < p.passes && blocks > 1 ? p.counts + (int64_t)(p.pass + 1) * blocks * p.keys : nullptr;
    for (int tile = 0; tile < p.chunk; tile += ORDER_TILE) {
        const int64_t from = (int64_t)blockIdx.x * p.chunk + tile + warp * 32 * ORDER_ITEMS + lane;
        if (tile > 0 && (int64_t)blockIdx.x * p.chunk + tile >= p.n) break;
        uint2 entry[ORDER_ITEMS];
        int key[ORDER_ITEMS], rank[ORDER_ITEMS];
#pragma unroll
        for (int u = 0; u < ORDER_ITEMS; u++) key[u] = order_key<WHAT>(p, from + 32 * u, entry[u]);
        uint16_t *mine = at + warp * width;
        for (int d = lane; d < width / 2; d += 32) ((uint32_t *)mine)[d] = 0;
        __syncwarp();
#pragma unroll
        for (int u = 0; u < ORDER_ITEMS; u++) {
            const unsigned same = __match_any_sync(~0u, key[u]);
            const int lower = __popc(same & ((1u << lane) - 1)), before = key[u] >= 0 ? mine[key[u]] : 0;
            rank[u] = before + lower;
            __syncwarp();
            if (key[u] >= 0 && lower == 0) mine[key[u]] = (uint16_t)(before + __popc(same));
            __syncwarp();
        }
        __syncthreads();
        int number[PER], sum = 0;                           // of this tile, for PER keys that follow one another
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int d = threadIdx.x * PER + i;
            number[i] = 0;
            if (d < p.keys)
                for (int w = 0; w < ORDER_WARPS; w++) {
                    const int c = at[w * width + d];
                    at[w * width + d] = (uint16_t)number[i];
                    number[i] += c;
                }
            if (d < p.keys && tile == 0) {
                if (blocks == 1) total[d] = number[i];
                sum += total[d];
            }
        }
        if (tile == 0) {                                    // a key's entries lie behind those of all smaller keys
            int before = sum;
            for (int d = 1; d < 32; d *= 2) {
                const int x = __shfl_up_sync(~0u, before, d);
                if (lane >= d) before += x;
            }
            if (lane == 31) sums[warp] = before;
            __syncthreads();
            before -= sum;
            for (int w = 0; w < warp; w++) before += sums[w];
#pragma unroll
            for (int i = 0; i < PER; i++) {
                const int d = threadIdx.x * PER + i;
                if (d >= p.keys) break;
                if (WHAT == BY_EXPERT && blockIdx.x == 0) {
                    p.offsets[d] = before;
                    if (d == p.keys - 1) p.offsets[p.keys] = before + total[d];
                }
                base[d] += before;
                before += total[d];
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < ORDER_ITEMS; u++) {
            const int64_t i = from + 32 * u;
            if (i >= p.n) continue;
            const int place = key[u] >= 0 ? base[key[u]] + mine[key[u]] + rank[u] : -1;
            if (WHAT == BY_EXPERT) p.places[i] = place;
            else {
                p.to[place] = entry[u];
                if (next) atomicAdd(&next[place / p.chunk * p.keys + (int)(entry[u].x >> p.shift + p.bits & (1 << p.bits) - 1)], 1);
            }
            if (WHAT == BY_TOKEN && p.present && entry[u].x < p.V) atomicOr(&p.present[entry[u].x >> 5], 1u << (entry[u].x & 31));
        }
        if (tile + ORDER_TILE >= p.chunk) break;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; i++)
            if (threadIdx.x * PER + i < p.keys) base[threadIdx.x * PER + i] += number[i];
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

// out[place] = x[row]: a row is read once and written to its places, four pieces at a time.  U: values of the size, copied as they are.
// Bound by memory: 8192 rows of 5120 to six places each, 105 us, 5.6 TB/s.
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
        for (int c = r.from + lane * N; c < r.to; c += 4 * 32 * N) {
            uint4 v[4];
#pragma unroll
            for (int u = 0; u < 4; u++)
                if (c + u * 32 * N < r.to) v[u] = *(const uint4 *)(x + c + u * 32 * N);
            for (unsigned left = there; left; left &= left - 1) {
                U *out = (U *)p.out + (int64_t)places[__ffs(left) - 1] * p.ldo + c;
#pragma unroll
                for (int u = 0; u < 4; u++)
                    if (c + u * 32 * N < r.to) *(uint4 *)(out + u * 32 * N) = v[u];
            }
        }
    } else {
        for (int c = r.from + lane; c < r.to; c += 32) {
            const U v = x[c];
            for (unsigned left = there; left; left &= left - 1) ((U *)p.out + (int64_t)places[__ffs(left) - 1] * p.ldo)[c] = v;
        }
    }
}

template <int N> struct Count { static constexpr int value = N; };

// Eight values as they are read: unpacked where they are used, so that many reads are on their way in few registers
template <typename T, bool WIDE> struct Raw {
    uint4 v[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *row, int from, int t, int n, int H)
    {
#pragma unroll
        for (int i = 0; i < sizeof(T) / 2; i++) v[i] = ((const uint4 *)(row + from + 8 * t))[i];
    }
    __device__ __forceinline__ Eight eight() const
    {
        if constexpr (sizeof(T) == 2) return {{pair_of(v[0].x, T()), pair_of(v[0].y, T()), pair_of(v[0].z, T()), pair_of(v[0].w, T())}};
        else {
            const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
            Eight x;
#pragma unroll
            for (int i = 0; i < 4; i++) x.v[i] = pair(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
            return x;
        }
    }
};
template <typename T> struct Raw<T, false> {
    T v[8];
    __device__ __forceinline__ void load(const T *row, int from, int t, int n, int H)
    {
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = row[from + t + n * j < H ? from + t + n * j : 0];
    }
    __device__ __forceinline__ Eight eight() const
    {
        Eight x;
#pragma unroll
        for (int j = 0; j < 4; j++) x.v[j] = pair(to_float(v[2 * j]), to_float(v[2 * j + 1]));
        return x;
    }
};

// out[row] = base[row] + sum_j weight_j y[place_j].  The rows that are there, with their weights, are listed in shared memory, so that
// reads are not behind conditions: eight rows are on their way at once.  Bound by memory: 65536 rows of 8192 in 16 bits, weighted, 229 us,
// 5.9 TB/s (read under conditions, four at a time, 366; a warp's columns 256, 1024, 2048 and 8192 of a row 247, 232, 230 and 267).
template <typename T, bool WIDE> __global__ void __launch_bounds__(256) combine_kernel(const RowsArgs p)
{
    __shared__ int2 list[8][MOST_CHOSEN];
    launch_next();
    wait_for_last();
    const Piece r = piece_of(p);
    const int lane = threadIdx.x & 31;
    if (r.row >= p.rows) return;
    int2 *mine = list[threadIdx.x >> 5];
    int place = -1;
    float weight = 1.0f;
    if (lane < p.k) {
        place = p.places[r.row * p.k + lane];
        if (p.weights) weight = p.weights[r.row * p.k + lane];
    }
    const bool is = place >= 0 && place < p.placed;
    const unsigned there = __ballot_sync(~0u, is);
    if (is) mine[__popc(there & ((1u << lane) - 1))] = make_int2(place, __float_as_int(weight));
    __syncwarp();
    const int n = __popc(there);
    for (int c = r.from; c < r.to; c += 256) {
        if (WIDE && c + 8 * lane >= r.to) break;
        Eight sum = eight_of(0.0f);
        if (p.base) {
            Raw<T, WIDE> x;
            x.load((const T *)p.base + r.row * p.ldbase, c, lane, 32, r.to);
            sum = x.eight();
        }
        auto add = [&](int j, auto count) {
            constexpr int N = decltype(count)::value;
            Raw<T, WIDE> x[N];
#pragma unroll
            for (int u = 0; u < N; u++) x[u].load((const T *)p.y + (int64_t)mine[j + u].x * p.ldy, c, lane, 32, r.to);
#pragma unroll
            for (int u = 0; u < N; u++) {
                const Eight e = x[u].eight();
                const Pair w = pair(__int_as_float(mine[j + u].y));
#pragma unroll
                for (int i = 0; i < 4; i++) sum.v[i] = fma2(w, e.v[i], sum.v[i]);
            }
        };
        int j = 0;
        if (sizeof(T) == 2)
            for (; j + 8 <= n; j += 8) add(j, Count<8>());
        for (; j + 4 <= n; j += 4) add(j, Count<4>());
        if (n - j >= 2) add(j, Count<2>()), j += 2;
        if (n - j) add(j, Count<1>());
        store_columns<WIDE>((T *)p.out + r.row * p.ldo, c, lane, 32, r.to, sum);
    }
}

// dy[place_j] = weight_j dout[row] and dweight_j = <dout[row], y[place_j]>, a block for each row: dout is read once, y once.  Up to
// eight rows of y are on their way at once; with more than eight dout is read again, from L1.  Six at once, since four and two are two
// passes over the row: 16384 rows of 5120 with six places 373 us, without 424 (with seven 479 and 530; in 32 bits four
// rows are as many bytes as eight).  Bound by memory: 4001 rows of 5120 with six places each 96 us, 5.6 TB/s.
template <typename T, bool WIDE> __global__ void __launch_bounds__(256) combine_backward_kernel(const RowsArgs p)
{
    __shared__ float parts[8][MOST_CHOSEN];
    __shared__ int2 list[MOST_CHOSEN];                      // of the rows that are there: place, weight
    __shared__ int order[MOST_CHOSEN];
    launch_next();
    wait_for_last();
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int place = lane < p.k ? p.places[row * p.k + lane] : -1;
    const bool is = place >= 0 && place < p.placed;
    const unsigned there = __ballot_sync(~0u, is);
    const int n = __popc(there);
    if (warp == 0 && is) {
        const int at = __popc(there & ((1u << lane) - 1));
        list[at] = make_int2(place, __float_as_int(p.weights ? p.weights[row * p.k + lane] : 1.0f)), order[at] = lane;
    }
    __syncthreads();
    if (p.dweights && warp == 0 && lane < p.k && !is) p.dweights[row * p.k + lane] = 0;
    auto some = [&](int j0, auto count) {
        constexpr int N = decltype(count)::value;
        Pair dot[N];
#pragma unroll
        for (int u = 0; u < N; u++) dot[u] = pair(0.0f);
        for (int c = 0; c < p.H; c += 8 * blockDim.x) {
            if (WIDE && c + 8 * threadIdx.x >= p.H) break;
            Raw<T, WIDE> rd, ry[N];
            rd.load((const T *)p.x + row * p.ldx, c, threadIdx.x, blockDim.x, p.H);
            if (p.dweights)
#pragma unroll
                for (int u = 0; u < N; u++) ry[u].load((const T *)p.y + (int64_t)list[j0 + u].x * p.ldy, c, threadIdx.x, blockDim.x, p.H);
            Eight d = rd.eight();
            if (!WIDE) {                                    // (behind the row's end the first column was read)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float2 f = both(d.v[i]);
                    d.v[i] = pair(column<WIDE>(c, threadIdx.x, blockDim.x, 2 * i) < p.H ? f.x : 0.0f, column<WIDE>(c, threadIdx.x, blockDim.x, 2 * i + 1) < p.H ? f.y : 0.0f);
                }
            }
#pragma unroll
            for (int u = 0; u < N; u++) {
                if (p.dweights) {
                    Eight y = ry[u].eight();
                    if (!WIDE) {
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            const float2 f = both(y.v[i]);
                            y.v[i] = pair(column<WIDE>(c, threadIdx.x, blockDim.x, 2 * i) < p.H ? f.x : 0.0f, column<WIDE>(c, threadIdx.x, blockDim.x, 2 * i + 1) < p.H ? f.y : 0.0f);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; i++) dot[u] = fma2(y.v[i], d.v[i], dot[u]);
                }
                if (p.out) {
                    const Pair w = pair(__int_as_float(list[j0 + u].y));
                    Eight x;
#pragma unroll
                    for (int i = 0; i < 4; i++) x.v[i] = w * d.v[i];
                    store_columns<WIDE>((T *)p.out + (int64_t)list[j0 + u].x * p.ldo, c, threadIdx.x, blockDim.x, p.H, x);
                }
            }
        }
        if (!p.dweights) return;
#pragma unroll
        for (int u = 0; u < N; u++) {
            float sum = sum_of(dot[u]);
#pragma unroll
            for (int s = 16; s; s /= 2) sum += __shfl_xor_sync(~0u, sum, s);
            if (lane == 0) parts[warp][j0 + u] = sum;
        }
    };
    int j = 0;
    if (sizeof(T) == 2)
        for (; j + 8 <= n; j += 8) some(j, Count<8>());
    if (sizeof(T) == 2 && n - j >= 6) some(j, Count<6>()), j += 6;
    for (; j + 4 <= n; j += 4) some(j, Count<4>());
    if (n - j >= 2) some(j, Count<2>()), j += 2;
    if (n - j) some(j, Count<1>());
    if (!p.dweights) return;
    __syncthreads();
    if (threadIdx.x < n) {
        float sum = 0;
        for (int w = 0; w < warps; w++) sum += parts[w][threadIdx.x];
        p.dweights[row * p.k + order[threadIdx.x]] = sum;
    }
}

// ---- embedding --------------------------------------------------------------------------------------------------------------
struct EmbeddingArgs {
    int64_t n, first;
    int64_t ldw, ldx, ldo;
    int H, piece, V, accumulate, sums, columns;             // sums: blocks that sum, others clear; columns: eights of threads in a row
    float scale;
    const int64_t *tokens;
    const void *w, *x;              // x: the gradient dy
    void *out;
    const uint2 *sorted;            // (row of w, number of the token) by row; those of no row behind them
    float *parts;                   // [chunks][2][H]: sums of a chunk's first and last row, where they are of more than one chunk
    const unsigned *present;
};

// out[i] = scale w[token_i - first]: a warp for a row or a piece of one, four reads on their way (8192 rows of 5120: 35 us; one 45)
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
    if (!there) {
        for (int c = from; c < to; c += 256) store_columns<WIDE>(out, c, lane, 32, to, eight_of(0.0f));
        return;
    }
    auto some = [&](int c, auto count) {
        constexpr int N = decltype(count)::value;
        Raw<T, WIDE> x[N];
#pragma unroll
        for (int u = 0; u < N; u++) x[u].load(in, c + 256 * u, lane, 32, to);
#pragma unroll
        for (int u = 0; u < N; u++) {
            Eight y = x[u].eight();
#pragma unroll
            for (int i = 0; i < 4; i++) y.v[i] = y.v[i] * pair(p.scale);
            store_columns<WIDE>(out, c + 256 * u, lane, 32, to, y);
        }
    };
    int c = from;
    for (; c + 1024 <= to; c += 1024) some(c, Count<4>());
    for (; c < to; c += 256)
        if (!WIDE || c + 8 * lane < to) some(c, Count<1>());
}

// The gradient.  The first blocks sum dy over the tokens of a row of w: they take chunks of the sorted list and an eight of columns
// for every thread, four rows of dy (and of what they are added to) on their way at once.  A row whose tokens are of one chunk is
// finished here; sums of a part of a row go to `parts` and are joined in order.  The blocks behind them write the rows that no
// token has, which is most of the bytes where nothing is added to; where something is, there are none.  Bound by memory: 16384 tokens
// into 102400 rows of 5120, 198 us for 168 MB read and 1.05 GB written, which a plain fill takes 270 for (sums and clearing side by
// side: 250; chunks of 16 and 8 tokens: 5 and 17 us more).
constexpr int EMBEDDING_CHUNK = 32;
template <typename T, typename O, bool WIDE> __global__ void __launch_bounds__(256) embedding_gradient_kernel(const EmbeddingArgs p)
{
    __shared__ uint2 list[EMBEDDING_CHUNK + 2];             // the token in front of the chunk's, the chunk's, the one behind
    launch_next();
    wait_for_last();
    const int t = threadIdx.x, n = blockDim.x;
    if (blockIdx.x >= p.sums) {
        const Eight zero = eight_of(0.0f);
        const int lane = t & 31, warps = n >> 5;
        for (int64_t v = (int64_t)(blockIdx.x - p.sums) * warps + (t >> 5); v < p.V; v += (int64_t)(gridDim.x - p.sums) * warps) {
            if (p.present[v >> 5] >> (v & 31) & 1) continue;
            for (int c = 0; c < p.H; c += 256) store_columns<WIDE>((O *)p.out + v * p.ldo, c, lane, 32, p.H, zero);
        }
        return;
    }
    const int64_t tasks = (p.n + EMBEDDING_CHUNK - 1) / EMBEDDING_CHUNK * p.columns;
    for (int64_t task = blockIdx.x; task < tasks; task += p.sums) {
        const int chunk = (int)(task / p.columns), c = (int)(task % p.columns) * n * 8;
        const int64_t from = (int64_t)chunk * EMBEDDING_CHUNK;
        __syncthreads();
        if (t < EMBEDDING_CHUNK) {
            const uint2 none = make_uint2(p.V, 0);
            list[t + 1] = from + t < p.n ? p.sorted[from + t] : none;
            if (t == 0) list[0] = from > 0 ? p.sorted[from - 1] : none;
            if (t == 1) list[EMBEDDING_CHUNK + 1] = from + EMBEDDING_CHUNK < p.n ? p.sorted[from + EMBEDDING_CHUNK] : none;
        }
        __syncthreads();
        const uint2 *s = list + 1;
        const unsigned V = p.V;
        if (s[0].x >= V) return;                                // (tokens of no row are behind all others)
        if (WIDE && c + 8 * t >= p.H) continue;
        float *part = p.parts + (int64_t)chunk * 2 * p.H;
        Eight sum = eight_of(0.0f);
        bool first = list[0].x == s[0].x;                       // the row began in front of this chunk
        for (int i = 0; i < EMBEDDING_CHUNK; i += 4) {
            if (s[i].x >= V) break;
            Raw<T, WIDE> x[4];
            Raw<O, WIDE> before[4];
#pragma unroll
            for (int u = 0; u < 4; u++) x[u].load((const T *)p.x + (int64_t)s[i + u].y * p.ldx, c, t, n, p.H);
            if (p.accumulate)                                   // (of a row's last token; others read row 0, which stays in L1)
#pragma unroll
                for (int u = 0; u < 4; u++) before[u].load((const O *)p.out + (s[i + u].x < V && s[i + u + 1].x != s[i + u].x ? (int64_t)s[i + u].x * p.ldo : 0), c, t, n, p.H);
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const unsigned v = s[i + u].x;
                if (v >= V) break;
                const Eight e = x[u].eight();
#pragma unroll
                for (int j = 0; j < 4; j++) sum.v[j] = sum.v[j] + e.v[j];
                const bool last = s[i + u + 1].x != v, whole = last && !first;
                if (whole) {
                    Eight y = p.accumulate ? before[u].eight() : eight_of(0.0f);
#pragma unroll
                    for (int j = 0; j < 4; j++) y.v[j] = fma2(sum.v[j], pair(p.scale), y.v[j]);
                    store_columns<WIDE>((O *)p.out + (int64_t)v * p.ldo, c, t, n, p.H, y);
                } else if (last || i + u == EMBEDDING_CHUNK - 1) store_columns<WIDE>(part + (first ? 0 : p.H), c, t, n, p.H, sum);
                if (last) first = false, sum = eight_of(0.0f);
            }
        }
    }
}

// Rows that begin in one chunk and end in another: their parts, in order.  (As many chunks are asked at once for the row's end as there are
// threads.)
template <typename O, bool WIDE> __global__ void __launch_bounds__(256) embedding_join_kernel(const EmbeddingArgs p)
{
    launch_next();
    wait_for_last();
    const int chunks = (int)((p.n + EMBEDDING_CHUNK - 1) / EMBEDDING_CHUNK), chunk = blockIdx.x / p.columns, t = threadIdx.x, n = blockDim.x, c = blockIdx.x % p.columns * n * 8;
    const int64_t from = (int64_t)chunk * EMBEDDING_CHUNK, to = from + EMBEDDING_CHUNK;
    const unsigned v = p.sorted[to].x, inside = p.sorted[to - 1].x, begin = p.sorted[from].x, before = from > 0 ? p.sorted[from - 1].x : p.V;
    if (v >= p.V || inside != v || (begin == v && before == v)) return;
    int lo = chunk;                                         // the last chunk that begins with the row: as many are asked as there are threads
    for (int some = n; some == n; lo += some) some = __syncthreads_count(lo + 1 + t < chunks && p.sorted[(int64_t)(lo + 1 + t) * EMBEDDING_CHUNK].x == v);
    if (WIDE && c + 8 * t >= p.H) return;
    O *out = (O *)p.out + (int64_t)v * p.ldo;
    const Eight was = p.accumulate ? load_columns<WIDE>((const O *)out, c, t, n, p.H) : eight_of(0.0f);
    Raw<float, WIDE> x;
    x.load(p.parts + ((int64_t)chunk * 2 + 1) * p.H, c, t, n, p.H);
    Eight sum = x.eight();
    for (int b = chunk + 1; b <= lo; b += 4) {
        Raw<float, WIDE> y[4];
#pragma unroll
        for (int u = 0; u < 4; u++) y[u].load(p.parts + (int64_t)min(b + u, lo) * 2 * p.H, c, t, n, p.H);
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const Eight e = y[u].eight();
            if (b + u <= lo)
#pragma unroll
                for (int j = 0; j < 4; j++) sum.v[j] = sum.v[j] + e.v[j];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; j++) sum.v[j] = fma2(sum.v[j], pair(p.scale), was.v[j]);
    store_columns<WIDE>(out, c, t, n, p.H, sum);
}

} // namespace hapop
