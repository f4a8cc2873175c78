// The router's choice: k of E experts for every row from its logits z, and the logits' gradient from the weights'.
// Scores s = softmax(z) or 1 / (1 + e^-z), values v = s + bias; of groups of experts that follow one another the `kept` with the
// largest sums of their `best` largest v; in them the k largest v, descending, ties to the lowest index; weights scale s, or scale
// s over the sum of the chosen s.
#pragma once
#include "hap_rows.cuh"

namespace hapop {

constexpr int MOST_EXPERT_GROUPS = 32;
constexpr int ROUTE_WARPS = 4;
constexpr float NONE = -INFINITY;

struct RouteArgs {
    const void *z;
    int64_t ld, rows;
    const float *bias;              // null: none
    int E, k, sigmoid, groups, kept, best, renormalise;
    float scale;
    int per, lanes;                 // of a row's lanes, `lanes` hold a group, `per` experts each
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
    if (L == 32) return __reduce_max_sync(~0u, x);
#pragma unroll
    for (int d = L / 2; d; d /= 2) x = max(x, __shfl_xor_sync(~0u, x, d));
    return x;
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

// One row by a whole warp with values in 64 bits: for rows whose values 32 bits cannot tell apart, and for layouts of groups that do
// not fit the lanes.  space: E doubles of this warp's own.
struct RowStart { float m, sum; bool bad; };
template <typename T> __device__ __noinline__ RowStart route_slowly(const RouteArgs &p, int64_t row, double *space, int *ce, float *cz)
{
    const int lane = threadIdx.x & 31, size = p.E / p.groups;
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
    if (bad) return {(float)m, (float)sum, true};
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
            ce[j] = any ? who : -1, cz[j] = any ? to_float(z[who]) : NONE;
            if (any) space[who] = -INFINITY;
        }
        __syncwarp();
    }
    return {(float)m, (float)sum, false};
}

// L lanes for a row, up to PER experts each.  Values are in 32 bits; the choice is the same as in exact arithmetic where
// neighbours in the order are further apart than both are off, and the row is done once more in 64 bits where they are not.
template <typename T, int L, int PER> __global__ void __launch_bounds__(32 * ROUTE_WARPS) route_kernel(const RouteArgs p)
{
    extern __shared__ double space[];                       // E for each warp, then the chosen of each row
    constexpr int ROWS = 32 / L;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane & (L - 1);
    launch_next();
    wait_for_last();
    const int64_t row = ((int64_t)blockIdx.x * ROUTE_WARPS + warp) * ROWS + lane / L;
    const bool here = row < p.rows;
    int *ce = (int *)(space + ROUTE_WARPS * p.E) + (warp * ROWS + lane / L) * 2 * p.k;
    float *cz = (float *)(ce + p.k);
    const unsigned mine = lanes_of<L>(lane);
    float m = 0, sum = 1;
    bool bad = false, again = p.slow;
    if (!p.slow) {
        const int size = p.E / p.groups, group = sub / p.lanes, from = (sub & (p.lanes - 1)) * p.per, first = group * size + from;
        const int n = here && group < p.groups ? max(0, min(p.per, size - from)) : 0;
        const T *zr = (const T *)p.z + row * p.ld + first;
        float z[PER], v[PER];
        if (PER == 8 && p.eights) {
            float x[8];
            if (n > 0) load8(zr, x);
#pragma unroll
            for (int i = 0; i < PER; i++) z[i] = n > 0 ? x[i & 7] : NONE;
        } else {
#pragma unroll
            for (int i = 0; i < PER; i++) z[i] = i < n ? to_float(zr[i]) : NONE;
        }
        const bool values = p.bias || (p.groups > 1 && p.best > 1);         // whether scores decide, or logits do
#pragma unroll
        for (int i = 0; i < PER; i++) bad |= isnan(z[i]) || (!p.sigmoid && z[i] == INFINITY);
        float off = 0;                                                      // two values that are further apart are in order
        if (!p.sigmoid && (values || !p.renormalise)) {
#pragma unroll
            for (int i = 0; i < PER; i++) m = i ? fmaxf(m, z[i]) : z[0];
            m = most_of<L>(m);
            if (m == NONE) m = 0;
            sum = 0;
#pragma unroll
            for (int i = 0; i < PER; i++) sum += p.renormalise ? __expf(z[i] - m) : expf(z[i] - m);        // (a weight's, or the choice's alone)
            sum = sum_of<L>(sum);
        }
#pragma unroll
        for (int i = 0; i < PER; i++) v[i] = z[i];
        if (values) {
            // What a score is off by.  Sigmoid: e^-z by 2^-22 + 1.5 |z| 2^-23 of itself, which s (1 - s) takes to 1e-7, two
            // roundings and the quotient 3e-7.  Softmax: of the largest score, 2^-22 for the term and the sum's up to 37 roundings,
            // 2.5e-6 in all.  `off` is at least what two values differ by wrongly; a sum with the bias has a rounding of its own.
            const float inverse = __fdividef(1.0f, sum);
            off = p.sigmoid ? 1.5e-6f : 6e-6f * inverse;
            float b[PER];
            if (!p.bias) {
#pragma unroll
                for (int i = 0; i < PER; i++) b[i] = 0;
            } else if (PER == 8 && p.eights) {
                float x[8];
                load8(p.bias + (n > 0 ? first : 0), x);
#pragma unroll
                for (int i = 0; i < PER; i++) b[i] = x[i & 7];
            } else {
#pragma unroll
                for (int i = 0; i < PER; i++) b[i] = i < n ? p.bias[first + i] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < PER; i++) {
                bad |= isnan(b[i]) || b[i] == INFINITY;
                const float s = p.sigmoid ? __fdividef(1.0f, 1.0f + __expf(-z[i])) : __expf(z[i] - m) * inverse;
                v[i] = z[i] == NONE || b[i] == NONE ? NONE : s + b[i];
            }
        }
        bad = (__ballot_sync(~0u, bad) & mine) != 0;
        if (p.groups > 1) {
            float a = NONE, b = NONE;                       // a group's largest and the next
#pragma unroll
            for (int i = 0; i < PER; i++) b = fmaxf(b, fminf(a, v[i])), a = fmaxf(a, v[i]);
            for (int d = p.lanes / 2; d; d /= 2) {
                const float c = __shfl_xor_sync(~0u, a, d), e = __shfl_xor_sync(~0u, b, d);
                b = fmaxf(fminf(a, c), fmaxf(b, e)), a = fmaxf(a, c);
            }
            const float total = p.best > 1 && b > NONE ? a + b : a;
            int ahead = 0;
            for (int g = 0; g < L / p.lanes; g++) {
                const float other = __shfl_sync(~0u, total, (lane & ~(L - 1)) + g * p.lanes);
                ahead += other > total || (other == total && g < group);
            }
            const bool kept = ahead < p.kept;
            if (values) {
                const float low = -most_of<L>(kept && total > NONE ? -total : NONE), high = most_of<L>(kept ? NONE : total);
                again |= low < INFINITY && high > NONE && low - high <= 2 * off + 4e-7f * (fabsf(low) + fabsf(high));
            }
#pragma unroll
            for (int i = 0; i < PER; i++) v[i] = !kept || v[i] == NONE ? NONE : p.bias ? v[i] : z[i];
        }
        // The largest k as whole numbers, which order as the values do, 0 for none: the row's largest of the lanes' largest, taken
        // from the first lane that has it and there from the first place.
        uint32_t key[PER], best = 0;
#pragma unroll
        for (int i = 0; i < PER; i++) key[i] = v[i] == NONE ? 0 : ordered(v[i]), best = max(best, key[i]);
        const bool check = p.bias;                          // (without one the logits decide in the groups)
        uint32_t last = ~0u;
        for (int j = 0; j < p.k + check; j++) {
            const uint32_t top = most_of<L>(best);
            const unsigned who = __ballot_sync(~0u, best == top) & mine;
            if (check && top && j > 0) {
                const float x = from_ordered(last), y = from_ordered(top);
                again |= x - y <= off + 2e-7f * (fabsf(x) + fabsf(y));
            }
            last = top;
            if (lane == __ffs(who) - 1) {
                int at = PER - 1;
                float x = z[PER - 1];
#pragma unroll
                for (int i = PER - 2; i >= 0; i--)
                    if (key[i] == top) at = i, x = z[i];
                best = 0;
#pragma unroll
                for (int i = 0; i < PER; i++) key[i] = i == at ? 0 : key[i], best = max(best, key[i]);
                if (j < p.k) ce[j] = top ? first + at : -1, cz[j] = top ? x : NONE;
            }
        }
    }
    unsigned slow = __ballot_sync(~0u, sub == 0 && here && again && !bad);
    while (slow) {
        const int who = __ffs(slow) - 1;
        slow &= slow - 1;
        int *to = (int *)(space + ROUTE_WARPS * p.E) + (warp * ROWS + who / L) * 2 * p.k;
        __syncwarp();
        const RowStart r = route_slowly<T>(p, __shfl_sync(~0u, row, who), space + warp * p.E, to, (float *)(to + p.k));
        if (lane / L == who / L) m = r.m, sum = r.sum, bad = r.bad;
    }
    __syncwarp();
    float top = NONE, total = 0;
    if (p.renormalise) {
        for (int j = sub; j < p.k; j += L) top = fmaxf(top, cz[j]);
        top = most_of<L>(top);
        if (top == NONE) top = 0;
        if (p.sigmoid) top = fminf(top, 0.0f);
        for (int j = sub; j < p.k; j += L) total += ce[j] < 0 ? 0.0f : p.sigmoid ? sigmoid_score(cz[j], top) : expf(cz[j] - top);
        total = sum_of<L>(total);
    }
    if (!here) return;
    for (int j = sub; j < p.k; j += L) {
        float w = 0;
        if (ce[j] >= 0) {
            if (p.renormalise) w = (p.sigmoid ? sigmoid_score(cz[j], top) : expf(cz[j] - top)) / total;
            else w = p.sigmoid ? sigmoid_score(cz[j], 0.0f) : expf(cz[j] - m) / sum;
        }
        p.experts[row * p.k + j] = bad ? j : ce[j];
        p.weights[row * p.k + j] = bad ? NAN : w * p.scale;
    }
}

// The gradient of the logits.  With p_j = s_j over the sum of the chosen s and G = sum_j g_j p_j:
//   softmax, renormalised   dz_j = scale p_j (g_j - G)
//   sigmoid, renormalised   dz_j = scale p_j (1 - s_j) (g_j - G)
//   sigmoid                 dz_j = scale g_j s_j (1 - s_j)
//   softmax                 dz_e = scale s_e (g_e - sum_j g_j s_j) over all e, g_e = 0 where e is not chosen
// All but the last are 0 beside the chosen: their logits alone are read.
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
        if (PER == 8 && p.eights) {
            float x[8];
            if (n > 0) load8(z + first, x);
#pragma unroll
            for (int i = 0; i < PER; i++) s[i] = n > 0 ? x[i & 7] : NONE;
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
    if (PER == 8 && p.eights) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; i++) y[i] = s[i & (PER - 1)] * rest;
        if (n > 0) store8(dz + first, y);
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
