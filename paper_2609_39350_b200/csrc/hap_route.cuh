// The router's choice: k of E experts for every row from its logits z, and the logits' gradient from the weights'.
// Scores s = softmax(z) or 1 / (1 + e^-z), values v = s + bias; of groups of experts that follow one another the `kept` with the
// largest sums of their `best` largest v; in them the k largest v, descending, ties to the lowest index; weights scale s, or scale
// s over the sum of the chosen s.
#pragma once
#include "hap_rows.cuh"

#include <float.h>

namespace hapop {

constexpr int MOST_EXPERT_GROUPS = 32;
constexpr int ROUTE_WARPS = 4, ROUTE_BLOCKS = 5;       // of a block; blocks of a multiprocessor
constexpr float NONE = -INFINITY;

struct RouteArgs {
    const void *z;
    int64_t ld, rows;
    const float *bias;              // null: none
    int E, k, sigmoid, groups, kept, best, renormalise;
    float scale;
    int size, per, lanes_log;       // experts of a group; of a row's lanes, 2^lanes_log hold a group, `per` experts each
    int room;                       // doubles of a warp's own: a row's values, or its lanes' keys in order
    int slow, eights;               // all rows the slow way; logits (and their gradients) are read (written) in eights
    int *experts;                   // [rows][k]
    float *weights;
    const int *chosen;              // backwards
    const float *dweights;
    void *dz;
    int64_t ldd;
};

template <int L> __device__ __forceinline__ float most_of(float x)
{
#pragma unroll
    for (int d = L / 2; d; d /= 2) x = fmaxf(x, __shfl_xor_sync(~0u, x, d));
    return x;
}
template <int L> __device__ __forceinline__ float sum_of(float x)
{
#pragma unroll
    for (int d = L / 2; d; d /= 2) x += __shfl_xor_sync(~0u, x, d);
    return x;
}
template <int L> __device__ __forceinline__ uint32_t most_of(uint32_t x)
{
    if constexpr (L == 32) return __reduce_max_sync(~0u, x);
    else {
#pragma unroll
        for (int d = L / 2; d; d /= 2) x = max(x, __shfl_xor_sync(~0u, x, d));
        return x;
    }
}
// A number's bits so that they order as numbers do (-0 as 0), above 0; and back
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u); }
template <int L> __device__ __forceinline__ unsigned lanes_of(int lane) { return L == 32 ? ~0u : ((1u << (L & 31)) - 1) << (lane & ~(L - 1)); }

// A chosen expert's sigmoid score times e^-m, m = min(0, the largest chosen logit): the quotients of scores are right however small
// the scores are.
__device__ __forceinline__ float sigmoid_score(float z, float m) { return z <= 0.0f ? expf(z - m) / (1.0f + expf(z)) : 1.0f / (1.0f + expf(-z)); }

// One row by a whole warp with values in 64 bits: for rows whose values 32 bits cannot tell apart, for layouts of groups that do not fit
// the lanes, and for groups that are judged by more than two values.  Such layouts are four to seven times slower: 32768 rows of 256 in
// eight groups by their best three 220 to 244 us (by their best two 51), of 1020 in 17 groups 952 us (rows of 1024 alone 145).  space: E doubles of this warp's own.
struct RowStart { float m, sum; bool bad; };
template <typename T> __device__ __noinline__ RowStart route_slowly(const RouteArgs &p, int64_t row, double *space, int *ce)
{
    const int lane = threadIdx.x & 31, size = p.size;
    const T *z = (const T *)p.z + row * p.ld;
    float top = NONE;
    bool bad = false;
    for (int e = lane; e < p.E; e += 32) {
        const float x = to_float(z[e]), b = p.bias ? p.bias[e] : 0.0f;
        bad |= isnan(x) || isnan(b) || b == INFINITY || (!p.sigmoid && x == INFINITY);
        top = fmaxf(top, x);
    }
    top = most_of<32>(top);
    bad = __any_sync(~0u, bad);
    const double m = top > NONE ? top : 0.0;
    double sum = 0;
    if (!p.sigmoid) {
        for (int e = lane; e < p.E; e += 32) sum += exp((double)to_float(z[e]) - m);
        for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
    }
    if (bad) {                                                      // (the experts of a row without an order: the weights' logits are read by them)
        if (lane < p.k) ce[lane] = lane;
        __syncwarp();
        return {(float)m, (float)sum, true};
    }
    for (int e = lane; e < p.E; e += 32) {
        const double x = to_float(z[e]), b = p.bias ? p.bias[e] : 0.0;
        const double s = p.sigmoid ? 1.0 / (1.0 + exp(-x)) : exp(x - m) / sum;
        // (without a bias and sums of several the logits order as the scores do, and exactly)
        space[e] = x == -INFINITY || b == -INFINITY ? -INFINITY : p.bias ? s + b : p.groups > 1 && p.best > 1 ? s : x;
    }
    __syncwarp();
    if (p.groups > 1) {
        double total = -INFINITY;
        if (lane < p.groups) {
            double last = INFINITY, sums = 0;
            int at = -1;
            for (int n = 0; n < p.best; n++) {                      // the next in (value, index)
                double most = -INFINITY;
                int who = -1;
                for (int i = 0; i < size; i++) {
                    const double v = space[lane * size + i];
                    if (v > most && (v < last || (v == last && i > at))) most = v, who = i;
                }
                if (who < 0) break;
                sums += most, total = sums, last = most, at = who;
            }
        }
        int ahead = 0;
        for (int g = 0; g < p.groups; g++) {
            const double other = __shfl_sync(~0u, total, g);
            ahead += other > total || (other == total && g < lane);
        }
        const unsigned kept = __ballot_sync(~0u, lane < p.groups && ahead < p.kept);
        for (int e = lane; e < p.E; e += 32)
            if (!(kept >> (e / size) & 1)) space[e] = -INFINITY;
            else if (!p.bias && space[e] > -INFINITY) space[e] = to_float(z[e]);
        __syncwarp();
    }
    for (int j = 0; j < p.k; j++) {
        double most = -INFINITY;
        int who = 1 << 30;
        for (int e = lane; e < p.E; e += 32)
            if (space[e] > most) most = space[e], who = e;
        for (int d = 16; d; d /= 2) {
            const double other = __shfl_xor_sync(~0u, most, d);
            const int at = __shfl_xor_sync(~0u, who, d);
            if (other > most || (other == most && at < who)) most = other, who = at;
        }
        const bool any = most > -INFINITY;
        if (lane == 0) {
            ce[j] = any ? who : -1;
            if (any) space[who] = -INFINITY;
        }
        __syncwarp();
    }
    return {(float)m, (float)sum, false};
}

// Values that 32 bits cannot tell apart among the chosen of a row and the one behind them (entries of ce, k + 1 at most 32): they are put
// in order by their values in 64 bits, a lane for each.
template <typename T> __device__ __noinline__ void route_settle(const RouteArgs &p, int64_t row, int *ce)
{
    const int lane = threadIdx.x & 31;
    const T *z = (const T *)p.z + row * p.ld;
    double m = 0, sum = 1;
    if (!p.sigmoid && p.bias) {
        float top = NONE;
        for (int e = lane; e < p.E; e += 32) top = fmaxf(top, to_float(z[e]));
        m = most_of<32>(top), sum = 0;
        for (int e = lane; e < p.E; e += 32) sum += exp((double)to_float(z[e]) - m);
        for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
    }
    const int e = lane <= p.k ? ce[lane] : -1;
    const double x = e >= 0 ? to_float(z[e]) : 0.0;
    const double v = e < 0 ? -INFINITY : !p.bias ? x : (p.sigmoid ? 1.0 / (1.0 + exp(-x)) : exp(x - m) / sum) + p.bias[e];
    int ahead = 0;
    for (int j = 0; j <= p.k; j++) {
        const double other = __shfl_sync(~0u, v, j);
        const int its = __shfl_sync(~0u, e, j);
        ahead += other > v || (other == v && its < e);
    }
    __syncwarp();
    if (e >= 0) ce[ahead] = e;
    __syncwarp();
}

// Whether this lane's group is kept, by sums of up to two values in 64 bits: for rows whose groups 32 bits cannot tell apart.  The lanes of
// a row hold its groups as in route_kernel, n experts from `first` on for each.
template <typename T, int L> __device__ __noinline__ bool route_groups(const RouteArgs &p, int64_t row, int first, int n, int group)
{
    const T *z = (const T *)p.z + row * p.ld;
    double m = 0, sum = 1;
    if (!p.sigmoid) {
        float top = NONE;
        for (int i = 0; i < n; i++) top = fmaxf(top, to_float(z[first + i]));
        top = most_of<L>(top);
        m = top > NONE ? top : 0.0f, sum = 0;
#pragma unroll 4
        for (int i = 0; i < n; i++) sum += exp((double)to_float(z[first + i]) - m);
        for (int d = L / 2; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
    }
    double a = -INFINITY, b = -INFINITY;
#pragma unroll 4
    for (int i = 0; i < n; i++) {
        const double x = to_float(z[first + i]), add = p.bias ? p.bias[first + i] : 0.0;
        const double v = x == -INFINITY || add == -INFINITY ? -INFINITY : (p.sigmoid ? 1.0 / (1.0 + exp(-x)) : exp(x - m) / sum) + add;
        b = fmax(b, fmin(a, v)), a = fmax(a, v);
    }
    for (int d = (1 << p.lanes_log) / 2; d; d /= 2) {
        const double c = __shfl_xor_sync(~0u, a, d), e = __shfl_xor_sync(~0u, b, d);
        b = fmax(fmin(a, c), fmax(b, e)), a = fmax(a, c);
    }
    const double total = p.best > 1 && b > -INFINITY ? a + b : a;
    int ahead = 0;
    for (int g = 0; g < p.groups; g++) {
        const double other = __shfl_sync(~0u, total, g << p.lanes_log, L);
        ahead += other > total || (other == total && g < group);
    }
    return ahead < p.kept && total > -INFINITY;
}

// The larger of two, a NaN where one is
__device__ __forceinline__ float most_or_nan(float x, float y) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y)); return r; }

// Descending order of the N numbers from LO on: halves put in order and merged, Batcher's way.  All of it is laid out at compile time
// (left as loops the numbers were in local memory, and a row took three times the instructions).
template <int LO, int N, int R, int ALL> __device__ __forceinline__ void merged(uint32_t (&x)[ALL])
{
    auto exchange = [&](int i) { const uint32_t a = x[i], b = x[i + R]; x[i] = max(a, b), x[i + R] = min(a, b); };
    if constexpr (2 * R < N) {
        merged<LO, N, 2 * R>(x), merged<LO + R, N, 2 * R>(x);
#pragma unroll
        for (int i = LO + R; i + R < LO + N; i += 2 * R) exchange(i);
    } else exchange(LO);
}
template <int LO, int N, int ALL> __device__ __forceinline__ void in_order(uint32_t (&x)[ALL])
{
    if constexpr (N > 1) in_order<LO, N / 2>(x), in_order<LO + N / 2, N / 2>(x), merged<LO, N, 1>(x);
}

// L lanes for a row, up to PER experts each.  Values are in 32 bits, without the last few, where an expert's place in its lane stands;
// the choice is the same as in exact arithmetic where neighbours in the order are further apart than both are off; where they are not,
// groups and chosen are settled by their values in 64 bits, and hardly ever the row is done once more (settled by whole rows, one row
// in 300 made the kernel a third longer: those that wait for it are few, but they are the last).  A lane's values are put in order
// once, so that taking the largest k of a row is one maximum over the lanes and one read in one of them each.  Bound by latency with
// few warps: 32768 rows of 256 with a bias and groups, 782 instructions a row, 53 us (every lane's maximum found anew for each: 1730,
// 91 us); logits alone in 16 bits 29 us; 5 and 3 us would be the bytes.  A scheduler has 4.8 warps (96 registers a thread) and issues
// in 55 % of its cycles, the ALU pipe is busy in half of them; of the 8.7 cycles between two instructions of a warp 2.3 are the first's
// own, 1.6 wait for shuffles and shared memory (the k + 2 rounds, one behind the other), 1.3 for memory.  Rows of 1024: 145 us, 21
// would be the bytes; 3.1 warps a scheduler (128 registers).
template <typename T, int L, int PER> __global__ void __launch_bounds__(32 * ROUTE_WARPS, PER == 32 ? 4 : ROUTE_BLOCKS) route_kernel(const RouteArgs p)
{
    extern __shared__ double space[];                       // `room` for each warp, then for each row the chosen and their keys, two more
    constexpr int ROWS = 32 / L;
    constexpr uint32_t PLACES = PER - 1, LEAST = 0x007fffff;     // (-inf's)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane & (L - 1);
    int *ce = (int *)(space + ROUTE_WARPS * p.room) + (warp * ROWS + lane / L) * 2 * (p.k + 2);
    uint32_t *keys = (uint32_t *)(ce + p.k + 2);
    const unsigned mine = lanes_of<L>(lane);
    const int lanes = 1 << p.lanes_log, group = sub >> p.lanes_log, from = (sub & (lanes - 1)) * p.per, first = group * p.size + from;
    const int own = group < p.groups ? max(0, min(p.per, p.size - from)) : 0;          // experts of this lane
    launch_next();
    wait_for_last();
    // a row's eights are read while the one before it is worked on
    constexpr int EIGHTS = PER / 8;
    Raw<T, true> next[EIGHTS];
    auto bring = [&](int64_t row) {
        const T *zr = (const T *)p.z + (row < p.rows ? row : 0) * p.ld;
#pragma unroll
        for (int i = 0; i < EIGHTS; i++) next[i].load(zr, own > 8 * i ? first + 8 * i : 0, 0, 0, 0);
    };
    const int64_t step = (int64_t)gridDim.x * ROUTE_WARPS * ROWS;
    int64_t row = ((int64_t)blockIdx.x * ROUTE_WARPS + warp) * ROWS + lane / L;
    if (p.eights && !p.slow) bring(row);
    for (; row - lane / L < p.rows; row += step) {            // (a warp's rows together)
        const bool here = row < p.rows;
        float m = 0, sum = 1;
        bool bad = false, again = p.slow;
        if (!p.slow) {
            const int n = here ? own : 0;
            float z[PER], v[PER];
            if (p.eights) {
#pragma unroll
                for (int i = 0; i < EIGHTS; i++) {
                    const Eight x = next[i].eight();
#pragma unroll
                    for (int j = 0; j < 8; j++) z[8 * i + j] = n > 8 * i ? (j & 1 ? both(x.v[j / 2]).y : both(x.v[j / 2]).x) : NONE;
                }
                bring(row + step);
            } else {
                const T *zr = (const T *)p.z + row * p.ld + first;
#pragma unroll
                for (int i = 0; i < PER; i++) z[i] = i < n ? to_float(zr[i]) : NONE;
            }
            const bool sums = p.groups > 1 && p.best > 1;       // scores are added up
            float most = z[0];
#pragma unroll
            for (int i = 1; i < PER; i++) most = most_or_nan(most, z[i]);
            bad = isnan(most) || (!p.sigmoid && most == INFINITY);
            if (!p.sigmoid && (p.bias || sums || !p.renormalise)) {
                m = most_of<L>(most);
                if (m == NONE) m = 0;
                sum = 0;
#pragma unroll
                for (int i = 0; i < PER; i++) sum += p.renormalise ? __expf(z[i] - m) : expf(z[i] - m);        // (a weight's, or the choice's alone)
                sum = sum_of<L>(sum);
            }
            // What a score is off by.  Sigmoid: e^-z by 2^-22 + 1.5 |z| 2^-23 of itself, which s (1 - s) takes to 1e-7, two roundings and
            // the quotient 3e-7.  Softmax: of the largest score, 2^-22 for the term and the sum's up to 37 roundings, 2.5e-6 in all.
            // `off` is at least what two values differ by wrongly; a sum with the bias has a rounding of its own.
            const float inverse = sum > 0.0f ? __fdividef(1.0f, sum) : 0.0f, off = p.sigmoid ? 8e-7f : 6e-6f * inverse;
            auto score = [&](float x) { return p.sigmoid ? __fdividef(1.0f, 1.0f + __expf(-x)) : __expf(x - m) * inverse; };
            if (p.bias) {
                float b[PER];
                if (p.eights) {
#pragma unroll
                    for (int i = 0; i < EIGHTS; i++) {
                        float x[8];
                        load8(p.bias + (n > 8 * i ? first + 8 * i : 0), x);
#pragma unroll
                        for (int j = 0; j < 8; j++) b[8 * i + j] = x[j];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < PER; i++) b[i] = i < n ? p.bias[first + i] : 0.0f;
                }
                float top = 0;
#pragma unroll
                for (int i = 0; i < PER; i++) v[i] = score(z[i]) + b[i], top = most_or_nan(top, v[i]), v[i] = z[i] == NONE ? NONE : v[i];
                bad |= !(top < INFINITY);                       // (of a bias that is no number, or +inf)
            } else {
#pragma unroll
                for (int i = 0; i < PER; i++) v[i] = z[i];
            }
            bad = (__ballot_sync(~0u, bad && here) & mine) != 0;
            if (p.groups > 1) {
                float a = NONE, b = NONE;                       // a group's largest and the next
#pragma unroll
                for (int i = 0; i < PER; i++) b = fmaxf(b, fminf(a, v[i])), a = fmaxf(a, v[i]);
                for (int d = lanes / 2; d; d /= 2) {
                    const float c = __shfl_xor_sync(~0u, a, d), e = __shfl_xor_sync(~0u, b, d);
                    b = fmaxf(fminf(a, c), fmaxf(b, e)), a = fmaxf(a, c);
                }
                const bool any = a > NONE, two = b > NONE;
                if (sums && !p.bias) a = score(a), b = score(b);
                const float total = !any ? NONE : sums && two ? a + b : a;
                int ahead = 0;
                for (int g = 0; g < p.groups; g++) {
                    const float other = __shfl_sync(~0u, total, g << p.lanes_log, L);
                    ahead += other > total || (other == total && g < group);
                }
                bool kept = ahead < p.kept && any;
                if (p.bias || sums) {
                    // What a group's value is off by: `off` for its scores; a rounding of each of its values and of their sum, which go with
                    // the values' sizes where these cancel, and of what stands here.  (Sums beyond the largest number are anything.)
                    const float error = off + 4e-7f * (sums && two ? fabsf(a) + fabsf(b) : fabsf(a));
                    const uint32_t low = ~most_of<L>(kept ? ~ordered(fmaxf(total - error, -FLT_MAX)) : 0u), high = most_of<L>(!kept && any ? ordered(fminf(total + error, FLT_MAX)) : 0u);
                    const bool near = !bad && low <= high;
                    if (__any_sync(~0u, near)) kept = route_groups<T, L>(p, here ? row : 0, first, n, group);
                }
                if (!kept)
#pragma unroll
                    for (int i = 0; i < PER; i++) v[i] = NONE;
            }
            // A value as a whole number that orders as it does, up to LEAST for none, with its place among the lane's in the last bits
            uint32_t key[PER];
#pragma unroll
            for (int i = 0; i < PER; i++) key[i] = (ordered(v[i]) & ~PLACES) | (PLACES - i);
            in_order<0, PER>(key);
            const bool check = p.bias || sizeof(T) == 4;        // (logits in 16 bits lose nothing with their last bits)
            const int rounds = check ? p.k + 2 : p.k;
            uint32_t *rest = (uint32_t *)(space + warp * p.room) + lane, head = key[0];           // (the others wait in shared memory)
#pragma unroll
            for (int i = 1; i < PER; i++) rest[32 * i] = key[i];
            rest[32 * PER] = 0;
            int taken = 0;
            for (int j = 0; j < rounds; j++) {
                const uint32_t value = head & ~PLACES, top = most_of<L>(value);
                const unsigned who = __ballot_sync(~0u, value == top) & mine;          // (the first lane of several)
                if (lane == __ffs(who) - 1) {
                    ce[j] = top > LEAST ? first + (int)(PLACES - (head & PLACES)) : -1, keys[j] = top;
                    taken += taken < PER, head = rest[32 * taken];
                }
            }
            __syncwarp();
            // Neighbours that may be the other way round: the chosen and the one behind them are settled by themselves; where the one behind
            // these may be among them too, the whole row is done again.
            bool near = false, at_end = false, behind = false;
            for (int j = sub + 1; check && j < rounds; j += L) {
                if (keys[j] <= LEAST) continue;
                const float x = from_ordered(keys[j - 1]), y = from_ordered(keys[j]);          // (logits in 32: where what is left is equal)
                const bool is = p.bias ? x - y <= off + PER * 1.2e-7f * fmaxf(fabsf(x), fabsf(y)) : keys[j - 1] == keys[j];
                near |= is && j <= p.k, at_end |= is && j == p.k, behind |= is && j == p.k + 1;
            }
            near = (__ballot_sync(~0u, near) & mine) != 0, at_end = (__ballot_sync(~0u, at_end) & mine) != 0, behind = (__ballot_sync(~0u, behind) & mine) != 0;
            again |= (at_end && behind) || (near && p.k == 32);
            again = (__ballot_sync(~0u, again) & mine) != 0;
            for (unsigned left = __ballot_sync(~0u, sub == 0 && here && near && !again && !bad); left; left &= left - 1) {
                const int who = __ffs(left) - 1;
                route_settle<T>(p, __shfl_sync(~0u, row, who), (int *)(space + ROUTE_WARPS * p.room) + (warp * ROWS + who / L) * 2 * (p.k + 2));
            }
        }
        unsigned slow = __ballot_sync(~0u, sub == 0 && here && again && !bad);
        while (slow) {
            const int who = __ffs(slow) - 1;
            slow &= slow - 1;
            __syncwarp();
            const RowStart r = route_slowly<T>(p, __shfl_sync(~0u, row, who), space + warp * p.room, (int *)(space + ROUTE_WARPS * p.room) + (warp * ROWS + who / L) * 2 * (p.k + 2));
            if (lane / L == who / L) m = r.m, sum = r.sum, bad = r.bad;
        }
        __syncwarp();
        // the chosen's weights: a lane has number sub, sub + L, ...
        constexpr int SLOTS = L >= 8 ? 32 / L : 8;              // (k is at most 32 and the lanes' experts, eight each where there are few lanes)
        const T *z = (const T *)p.z + (here ? row : 0) * p.ld;
        int e[SLOTS];
        float x[SLOTS], top = NONE, total = 0;
#pragma unroll
        for (int q = 0; q < SLOTS; q++) {
            e[q] = sub + q * L < p.k ? ce[sub + q * L] : -1;
            x[q] = e[q] >= 0 && here ? to_float(z[e[q]]) : NONE;
            top = fmaxf(top, x[q]);
        }
        if (p.renormalise) {
            top = most_of<L>(top);
            if (top == NONE) top = 0;
            if (p.sigmoid) top = fminf(top, 0.0f);
        } else top = p.sigmoid ? 0.0f : m;
#pragma unroll
        for (int q = 0; q < SLOTS; q++) {
            x[q] = e[q] < 0 ? 0.0f : p.sigmoid ? sigmoid_score(x[q], top) : expf(x[q] - top);
            total += x[q];
        }
        if (p.renormalise) total = sum_of<L>(total);
        else total = p.sigmoid ? 1.0f : sum;
        const float by = p.scale / total;
        __syncwarp();                                           // (the next row's chosen go where these were)
#pragma unroll
        for (int q = 0; q < SLOTS; q++) {
            const int j = sub + q * L;
            if (j >= p.k || !here) break;
            p.experts[row * p.k + j] = bad ? j : e[q];
            p.weights[row * p.k + j] = bad ? NAN : e[q] < 0 ? 0.0f : x[q] * by;
        }
    }
}

// The gradient of the logits.  With p_j = s_j over the sum of the chosen s and G = sum_j g_j p_j:
//   softmax, renormalised   dz_j = scale p_j (g_j - G)
//   sigmoid, renormalised   dz_j = scale p_j (1 - s_j) (g_j - G)
//   sigmoid                 dz_j = scale g_j s_j (1 - s_j)
//   softmax                 dz_e = scale s_e (g_e - sum_j g_j s_j) over all e, g_e = 0 where e is not chosen
// All but the last are 0 beside the chosen: their logits alone are read.  32768 rows of 256 in 32 bits:
// 17 us, 34 MB written (8 would be the bytes), and 20 us over all e (11): a warp has one chain of reads and ends.
template <typename T, int L, int PER> __global__ void __launch_bounds__(32 * ROUTE_WARPS) route_backward_kernel(const RouteArgs p)
{
    constexpr int ROWS = 32 / L;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane & (L - 1);
    launch_next();
    wait_for_last();
    const int64_t row = ((int64_t)blockIdx.x * ROUTE_WARPS + warp) * ROWS + lane / L;
    const bool here = row < p.rows, all = !p.sigmoid && !p.renormalise;
    const T *z = (const T *)p.z + (here ? row : 0) * p.ld;
    T *dz = (T *)p.dz + (here ? row : 0) * p.ldd;
    const int *chosen = p.chosen + (here ? row : 0) * p.k;
    const float *dweights = p.dweights + (here ? row : 0) * p.k;
    const int first = sub * p.per, n = here ? max(0, min(p.per, p.E - first)) : 0;
    // a lane's chosen: number sub, sub + L, ...  (k is at most 32 and the lanes' experts, eight each where there are few lanes)
    constexpr int SLOTS = L >= 8 ? 32 / L : 8;
    int e[SLOTS];
    float g[SLOTS], x[SLOTS];
#pragma unroll
    for (int q = 0; q < SLOTS; q++) {
        const int j = sub + q * L;
        e[q] = here && j < p.k ? chosen[j] : -1;
        g[q] = e[q] >= 0 && e[q] < p.E ? dweights[j] : 0.0f;
        e[q] = e[q] < p.E ? e[q] : -1;
        x[q] = e[q] >= 0 ? to_float(z[e[q]]) : NONE;
    }
    float m = 0, inverse = 0, top = NONE, total = 0, mean = 0;
    float s[PER];
#pragma unroll
    for (int i = 0; i < PER; i++) s[i] = 0;
    if (all) {
        if (p.eights) {
#pragma unroll
            for (int i = 0; i < PER; i += 8) {
                float y[8];
                if (n > i) load8(z + first + i, y);
#pragma unroll
                for (int j = 0; j < 8; j++) s[i + j] = n > i ? y[j] : NONE;
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER; i++) s[i] = i < n ? to_float(z[first + i]) : NONE;
        }
#pragma unroll
        for (int i = 0; i < PER; i++) m = i ? fmaxf(m, s[i]) : s[0];
        m = most_of<L>(m);
        if (m == NONE) m = 0;
        float sum = 0;
#pragma unroll
        for (int i = 0; i < PER; i++) sum += s[i] = expf(s[i] - m);
        sum = sum_of<L>(sum);
        inverse = sum > 0.0f || isnan(sum) ? 1.0f / sum : 0.0f;
    }
    if (p.renormalise) {
#pragma unroll
        for (int q = 0; q < SLOTS; q++) top = fmaxf(top, x[q]);
        top = most_of<L>(top);
        if (top == NONE) top = 0;
        if (p.sigmoid) top = fminf(top, 0.0f);
    }
    // an expert's score: over the sum of all, times e^-top, or as it is
    auto score = [&](float x) { return all ? expf(x - m) * inverse : p.sigmoid ? sigmoid_score(x, p.renormalise ? top : 0.0f) : expf(x - top); };
    float s_of[SLOTS];
#pragma unroll
    for (int q = 0; q < SLOTS; q++) {
        s_of[q] = e[q] >= 0 ? score(x[q]) : 0.0f;
        total += s_of[q], mean = fmaf(g[q], s_of[q], mean);
    }
    total = sum_of<L>(total), mean = sum_of<L>(mean);
    if (p.renormalise) mean = total > 0.0f || isnan(total) ? mean / total : 0.0f;
    const float rest = all ? -mean * inverse * p.scale : 0.0f;          // what an expert that is not chosen gets, over e^(z - m)
    if (p.eights) {
#pragma unroll
        for (int i = 0; i < PER; i += 8) {
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; j++) y[j] = s[i + j] * rest;
            if (n > i) store8(dz + first + i, y);
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; i++)
            if (i < n) dz[first + i] = from_float<T>(s[i] * rest);
    }
    // (an expert that is there twice has the gradients of both, and both write the same)
    float sums[SLOTS];
    int times[SLOTS];
#pragma unroll
    for (int q = 0; q < SLOTS; q++) sums[q] = 0, times[q] = 0;
#pragma unroll
    for (int r = 0; r < SLOTS; r++)
        for (int i = 0; i < L && r * L + i < p.k; i++) {
            const int other = __shfl_sync(~0u, e[r], i, L);
            const float its = __shfl_sync(~0u, g[r], i, L);
#pragma unroll
            for (int q = 0; q < SLOTS; q++)
                if (other == e[q]) sums[q] += its, times[q]++;
        }
    __syncwarp();
#pragma unroll
    for (int q = 0; q < SLOTS; q++) {
        if (e[q] < 0) continue;
        float d;
        if (all) d = s_of[q] * (sums[q] - mean);
        else if (p.renormalise) d = s_of[q] / total * (sums[q] - times[q] * mean) * (p.sigmoid ? 1.0f / (1.0f + expf(x[q])) : 1.0f);
        else d = sums[q] * s_of[q] / (1.0f + expf(x[q]));
        dz[e[q]] = from_float<T>(d * p.scale);
    }
}

} // namespace hapop
