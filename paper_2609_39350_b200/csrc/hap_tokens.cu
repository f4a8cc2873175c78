// Host side of the operators on a token's way: routing, experts' rows, embedding, layer norm.
#include "hap_norm.cuh"
#include "hap_route.cuh"
#include "hap_rows.cuh"
#include "hap_launch.h"

#include <type_traits>

using namespace hapop;

static bool dtype_fits(int32_t t) { return t == HAP_BF16 || t == HAP_FP16 || t == HAP_FP32; }
// a matrix whose rows all begin at multiples of 16 bytes
static bool wide(const void *p, int64_t ld, int32_t dtype) { return aligned(p, 16) && ld * size_of(dtype) % 16 == 0; }       // (beside H % 8 == 0)
// an output in the place of an input whose rows are another distance apart: rows would be written before they are read
static bool astray(const void *out, int64_t ldo, const void *in, int64_t ldi, int64_t rows) { return out && out == in && ldo != ldi && rows > 1; }
static bool grid_fits(int64_t blocks) { return blocks <= INT32_MAX; }

// f(T()) of an element type
template <typename F> static hap_status by_type(int32_t dtype, F &&f)
{
    return dtype == HAP_BF16 ? f(__nv_bfloat16()) : dtype == HAP_FP16 ? f(__half()) : f(float());
}

// ---- routing -------------------------------------------------------------------------------------------------------------
static bool routing_fits(const hap_routing *r)
{
    return r && r->E >= 1 && r->E <= 1024 && r->k >= 1 && r->k <= r->E && r->k <= MOST_CHOSEN && (r->scores == HAP_SOFTMAX || r->scores == HAP_SIGMOID) && r->groups >= 1 &&
           r->groups <= MOST_EXPERT_GROUPS && r->E % r->groups == 0 && r->kept_groups >= 1 && r->kept_groups <= r->groups && r->group_best >= 1;
}

// A row's lanes: as few as hold it with eight experts each, so that short rows share a warp; 16 each from 16 lanes on.
struct RouteLayout { int L, PER; bool fits; };
static RouteLayout route_layout(int size, int groups, int &per, int &lanes_log)
{
    int slots = 1;
    while (slots < groups) slots *= 2;
    lanes_log = 0;
    for (int L = slots; L <= 16; L *= 2, lanes_log++) {
        per = (size + (1 << lanes_log) - 1) >> lanes_log;
        if (per <= 8) return {L, 8, true};
        if (L == 16 && per <= 16) return {L, 16, true};
    }
    if (slots == 32) lanes_log = 0;
    per = (size + (1 << lanes_log) - 1) >> lanes_log;
    return {32, per <= 16 ? 16 : 32, per <= 32};
}

template <typename T, int L, int PER> static hap_status launch_route(const RouteArgs &p, bool backward, cudaStream_t s)
{
    int64_t blocks = ceil_div(p.rows, ROUTE_WARPS * (32 / L));
    if (!grid_fits(blocks)) return HAP_E_RANGE;
    if (backward) return launch_next(route_backward_kernel<T, L, PER>, blocks, 32 * ROUTE_WARPS, 0, 1, s, p);
    RouteArgs a = p;
    a.room = p.E > 16 * (PER + 1) ? p.E : 16 * (PER + 1);   // (a lane's keys and a 0 behind them)
    // warps go from row to row: as many blocks as run at once on 148 multiprocessors (of 32 experts a lane, whose threads have 128
    // registers, four fifths do; the rest follow)
    if (blocks > 148 * ROUTE_BLOCKS) blocks = 148 * ROUTE_BLOCKS;
    return launch_next(route_kernel<T, L, PER>, blocks, 32 * ROUTE_WARPS, ROUTE_WARPS * (a.room + 32 / L * (p.k + 2)) * 8, 1, s, a);
}

static hap_status run_route(RouteArgs p, int32_t dtype, bool backward, cudaStream_t s)
{
    const int groups = backward ? 1 : p.groups;
    p.size = p.E / groups;
    const RouteLayout at = route_layout(p.size, groups, p.per, p.lanes_log);
    p.slow = !backward && (!at.fits || (p.groups > 1 && p.best > 2));
    const bool dense = !p.sigmoid && !p.renormalise;        // (else the backward pass does not read whole rows)
    if (p.size % 8 == 0 && (backward && !dense ? true : wide(p.z, p.ld, dtype)) && (!backward || wide(p.dz, p.ldd, dtype)) && aligned(p.bias, 16)) p.per = (p.per + 7) / 8 * 8, p.eights = 1;
    return by_type(dtype, [&](auto t) {
        using T = decltype(t);
        switch (at.L + at.PER) {
        case 1 + 8: return launch_route<T, 1, 8>(p, backward, s);
        case 2 + 8: return launch_route<T, 2, 8>(p, backward, s);
        case 4 + 8: return launch_route<T, 4, 8>(p, backward, s);
        case 8 + 8: return launch_route<T, 8, 8>(p, backward, s);
        case 16 + 8: return launch_route<T, 16, 8>(p, backward, s);
        case 16 + 16: return launch_route<T, 16, 16>(p, backward, s);
        case 32 + 16: return launch_route<T, 32, 16>(p, backward, s);
        default: return launch_route<T, 32, 32>(p, backward, s);
        }
    });
}

extern "C" hap_status hap_route(const hap_routing *r, int32_t dtype, int64_t rows, const void *logits, int64_t ld, const float *bias, int32_t *experts, float *weights, void *stream)
{
    if (!routing_fits(r) || !dtype_fits(dtype) || rows < 0 || ld < r->E || !aligned(logits, size_of(dtype)) || !aligned(bias, 4) || !aligned(experts, 4) || !aligned(weights, 4)) return HAP_E_INVALID;
    if (rows == 0) return HAP_OK;
    if (!logits || !experts || !weights) return HAP_E_INVALID;
    RouteArgs p{};
    p.z = logits, p.ld = ld, p.rows = rows, p.bias = bias;
    p.E = r->E, p.k = r->k, p.sigmoid = r->scores == HAP_SIGMOID, p.groups = r->groups, p.kept = r->kept_groups, p.best = r->group_best, p.renormalise = r->renormalise != 0, p.scale = r->scale;
    p.experts = experts, p.weights = weights;
    return run_route(p, dtype, false, (cudaStream_t)stream);
}

extern "C" hap_status hap_route_backward(const hap_routing *r, int32_t dtype, int64_t rows, const void *logits, int64_t ld, const int32_t *experts, const float *dweights, void *dlogits,
                                         int64_t ldd, void *stream)
{
    if (!routing_fits(r) || !dtype_fits(dtype) || rows < 0 || ld < r->E || ldd < r->E || !aligned(logits, size_of(dtype)) || !aligned(dlogits, size_of(dtype)) || !aligned(experts, 4) ||
        !aligned(dweights, 4))
        return HAP_E_INVALID;
    if (rows == 0) return HAP_OK;
    if (!logits || !experts || !dweights || !dlogits || dlogits == logits) return HAP_E_INVALID;
    RouteArgs p{};
    p.z = logits, p.ld = ld, p.rows = rows;
    p.E = r->E, p.k = r->k, p.sigmoid = r->scores == HAP_SIGMOID, p.groups = 1, p.renormalise = r->renormalise != 0, p.scale = r->scale;
    p.chosen = experts, p.dweights = dweights, p.dz = dlogits, p.ldd = ldd;
    return run_route(p, dtype, true, (cudaStream_t)stream);
}

// ---- order by a key ------------------------------------------------------------------------------------------------------
// Entries of a block and the blocks of a pass: a tile each, several where there would be more than 128 blocks
struct OrderShape { int chunk, blocks; };
static OrderShape order_shape(int64_t n)
{
    const int64_t chunk = ceil_div(ceil_div(n < 1 ? 1 : n, 128), ORDER_TILE) * ORDER_TILE;
    return {(int)chunk, (int)ceil_div(n < 1 ? 1 : n, chunk)};
}
static uint64_t order_bytes(int64_t n, int keys, int passes)
{
    const OrderShape o = order_shape(n);
    return o.blocks > 1 ? up256((uint64_t)o.blocks * keys * passes * 4) : 0;
}
template <int WHAT> static hap_status run_order(OrderArgs &p, cudaStream_t s)
{
    const OrderShape o = order_shape(p.n);
    p.chunk = o.chunk;
    if (o.blocks > 1 && p.pass == 0) {
        const hap_status st = launch_next(order_count_kernel<WHAT>, o.blocks, 32 * ORDER_WARPS, 0, 1, s, p);
        if (st != HAP_OK) return st;
    }
    return launch_next(order_place_kernel<WHAT>, o.blocks, 32 * ORDER_WARPS, ORDER_WARPS * ((p.keys + 1) & ~1) * 2, 1, s, p);
}

static bool order_sizes(int64_t rows, int32_t k, int32_t E) { return rows >= 0 && rows <= INT32_MAX && k >= 1 && k <= MOST_CHOSEN && rows * k <= INT32_MAX && E >= 1 && E <= MOST_KEYS; }

extern "C" hap_status hap_expert_order_workspace(int64_t rows, int32_t k, int32_t E, uint64_t *host_bytes)
{
    if (!host_bytes || !order_sizes(rows, k, E)) return HAP_E_INVALID;
    *host_bytes = order_bytes(rows * k, E, 1);
    return HAP_OK;
}

extern "C" hap_status hap_expert_order(int64_t rows, int32_t k, int32_t first, int32_t E, const int32_t *experts, int64_t *offsets, int32_t *places, void *workspace, uint64_t bytes,
                                       void *stream)
{
    uint64_t need = 0;
    if (hap_expert_order_workspace(rows, k, E, &need) != HAP_OK || !offsets || !aligned(offsets, 8) || !aligned(experts, 4) || !aligned(places, 4)) return HAP_E_INVALID;
    if (rows > 0 && (!experts || !places)) return HAP_E_INVALID;
    if (need && (!workspace || bytes < need || !aligned(workspace, 256))) return HAP_E_INVALID;
    OrderArgs p{};
    p.n = rows * k, p.keys = E, p.passes = 1, p.counts = (int *)workspace, p.experts = experts, p.first = first, p.places = places, p.offsets = offsets;
    return run_order<BY_EXPERT>(p, (cudaStream_t)stream);
}

// ---- rows ----------------------------------------------------------------------------------------------------------------
// Columns of a warp: whole rows, unless there are too few of them for the device's warps (16 of each multiprocessor)
static int piece_of(int64_t rows, int64_t H)
{
    const int64_t most = ceil_div(H, 256), want = ceil_div(148 * 16, rows < 1 ? 1 : rows), pieces = want < most ? want : most;
    return (int)(ceil_div(ceil_div(H, pieces), 256) * 256);
}
static bool rows_sizes(int64_t rows, int32_t k, int32_t H, int64_t placed) { return rows >= 0 && rows <= INT32_MAX && k >= 1 && k <= MOST_CHOSEN && H >= 1 && H < (1 << 28) && placed >= 0; }

extern "C" hap_status hap_expert_dispatch(int32_t dtype, int64_t rows, int32_t k, int32_t H, int64_t placed, const void *x, int64_t ldx, const int32_t *places, void *out, int64_t ldo,
                                          void *stream)
{
    if (!dtype_fits(dtype) || !rows_sizes(rows, k, H, placed) || ldx < H || ldo < H || !aligned(x, size_of(dtype)) || !aligned(out, size_of(dtype)) || !aligned(places, 4)) return HAP_E_INVALID;
    if (rows == 0 || placed == 0) return HAP_OK;
    if (!x || !places || !out) return HAP_E_INVALID;
    // values are copied as they are, so several may be one: rows of an even length, at even distances and addresses, are of half as many
    // twice as long (49152 rows of 5124 in 16 bits: 287 -> 169 us, of 5122 317 -> 241; of 5120, in whole sixteen bytes, 115)
    int64_t unit = size_of(dtype);
    const bool w = H % 8 == 0 && wide(x, ldx, dtype) && wide(out, ldo, dtype);
    while (!w && unit < 8 && H % 2 == 0 && ldx % 2 == 0 && ldo % 2 == 0 && aligned(x, 2 * unit) && aligned(out, 2 * unit)) unit *= 2, H /= 2, ldx /= 2, ldo /= 2;
    RowsArgs p{};
    p.rows = rows, p.placed = placed, p.k = k, p.H = H, p.piece = piece_of(rows, H), p.places = places, p.x = x, p.ldx = ldx, p.out = out, p.ldo = ldo;
    const int64_t blocks = ceil_div(rows * ceil_div(H, p.piece), 8);
    if (!grid_fits(blocks)) return HAP_E_RANGE;
    auto *kernel = w ? (unit == 2 ? dispatch_kernel<uint16_t, true> : dispatch_kernel<uint32_t, true>)
                     : unit == 2 ? dispatch_kernel<uint16_t, false> : unit == 4 ? dispatch_kernel<uint32_t, false> : dispatch_kernel<uint64_t, false>;
    return launch_next(kernel, blocks, 256, 0, 1, (cudaStream_t)stream, p);
}

extern "C" hap_status hap_expert_combine(int32_t dtype, int64_t rows, int32_t k, int32_t H, int64_t placed, const void *y, int64_t ldy, const int32_t *places, const float *weights,
                                         const void *base, int64_t ldbase, void *out, int64_t ldo, void *stream)
{
    const int64_t size = size_of(dtype);
    if (!dtype_fits(dtype) || !rows_sizes(rows, k, H, placed) || ldy < H || ldo < H || (base && ldbase < H) || !aligned(y, size) || !aligned(base, size) || !aligned(out, size) ||
        !aligned(places, 4) || !aligned(weights, 4) || astray(out, ldo, base, ldbase, rows))
        return HAP_E_INVALID;
    if (rows == 0) return HAP_OK;
    if ((!y && placed > 0) || !places || !out) return HAP_E_INVALID;
    RowsArgs p{};
    p.rows = rows, p.placed = placed, p.k = k, p.H = H, p.piece = (int)(piece_of(rows, H) < 1024 ? piece_of(rows, H) : 1024), p.places = places, p.weights = weights, p.y = y, p.ldy = ldy, p.base = base, p.ldbase = ldbase;
    p.out = out, p.ldo = ldo;
    const int64_t blocks = ceil_div(rows * ceil_div(H, p.piece), 8);
    if (!grid_fits(blocks)) return HAP_E_RANGE;
    const bool w = H % 8 == 0 && wide(y, ldy, dtype) && wide(out, ldo, dtype) && (!base || wide(base, ldbase, dtype));
    return by_type(dtype, [&](auto t) {
        using T = decltype(t);
        return launch_next(w ? combine_kernel<T, true> : combine_kernel<T, false>, blocks, 256, 0, 1, (cudaStream_t)stream, p);
    });
}

extern "C" hap_status hap_expert_combine_backward(int32_t dtype, int64_t rows, int32_t k, int32_t H, int64_t placed, const void *dout, int64_t lddout, const void *y, int64_t ldy,
                                                  const int32_t *places, const float *weights, void *dy, int64_t lddy, float *dweights, void *stream)
{
    const int64_t size = size_of(dtype);
    if (!dtype_fits(dtype) || !rows_sizes(rows, k, H, placed) || lddout < H || (dweights && ldy < H) || (dy && lddy < H) || !aligned(dout, size) || !aligned(y, size) || !aligned(dy, size) ||
        !aligned(places, 4) || !aligned(weights, 4) || !aligned(dweights, 4) || (dy && dy == y && lddy != ldy))
        return HAP_E_INVALID;
    if (rows == 0 || (!dy && !dweights)) return HAP_OK;
    if (!dout || !places || (dweights && placed > 0 && !y)) return HAP_E_INVALID;
    RowsArgs p{};
    p.rows = rows, p.placed = placed, p.k = k, p.H = H, p.places = places, p.weights = weights, p.x = dout, p.ldx = lddout, p.y = y, p.ldy = ldy, p.out = dy, p.ldo = lddy, p.dweights = dweights;
    const bool w = H % 8 == 0 && wide(dout, lddout, dtype) && (!dweights || wide(y, ldy, dtype)) && (!dy || wide(dy, lddy, dtype));
    // four warps for a row; eight where there are too few rows for the device
    const int64_t most = ceil_div(H, 256), want = rows < 148 * 8 ? 8 : 4;
    const int threads = (int)(32 * (most < want ? most : want));
    return by_type(dtype, [&](auto t) {
        using T = decltype(t);
        return launch_next(w ? combine_backward_kernel<T, true> : combine_backward_kernel<T, false>, rows, threads, 0, 1, (cudaStream_t)stream, p);
    });
}

// ---- embedding -----------------------------------------------------------------------------------------------------------
static bool embedding_sizes(int64_t n, int32_t H, int64_t V) { return n >= 0 && n <= INT32_MAX && H >= 1 && H < (1 << 28) && V >= 1 && V < (1 << 28); }

extern "C" hap_status hap_embedding(int32_t dtype, int64_t n, int32_t H, int64_t V, int64_t first, const int64_t *tokens, const void *w, int64_t ldw, float scale, void *out, int64_t ldo,
                                    void *stream)
{
    if (!dtype_fits(dtype) || !embedding_sizes(n, H, V) || ldw < H || ldo < H || !aligned(w, size_of(dtype)) || !aligned(out, size_of(dtype)) || !aligned(tokens, 8)) return HAP_E_INVALID;
    if (n == 0) return HAP_OK;
    if (!tokens || !w || !out) return HAP_E_INVALID;
    EmbeddingArgs p{};
    p.n = n, p.first = first, p.H = H, p.V = (int)V, p.tokens = tokens, p.w = w, p.ldw = ldw, p.out = out, p.ldo = ldo, p.scale = scale, p.piece = piece_of(n, H);
    const int64_t blocks = ceil_div(n * ceil_div(H, p.piece), 8);
    if (!grid_fits(blocks)) return HAP_E_RANGE;
    const bool wd = H % 8 == 0 && wide(w, ldw, dtype) && wide(out, ldo, dtype);
    return by_type(dtype, [&](auto t) {
        using T = decltype(t);
        return launch_next(wd ? embedding_kernel<T, true> : embedding_kernel<T, false>, blocks, 256, 0, 1, (cudaStream_t)stream, p);
    });
}

// Digits of the sort: as few passes of up to ten bits as the values 0 .. V need
struct Digits { int passes, bits; };
static Digits digits_of(int64_t V)
{
    int bits = 1;
    while (V >> bits) bits++;
    const int passes = (bits + 9) / 10;
    return {passes, (bits + passes - 1) / passes};
}
struct EmbeddingSpace { uint64_t other, counts, present, parts, bytes; };
static EmbeddingSpace embedding_space(int64_t n, int64_t H, int64_t V)
{
    const Digits d = digits_of(V);
    EmbeddingSpace s;
    s.other = up256((uint64_t)n * 8);
    s.counts = s.other + (d.passes > 1 ? up256((uint64_t)n * 8) : 0);
    s.present = s.counts + order_bytes(n, 1 << d.bits, d.passes);
    s.parts = s.present + up256((uint64_t)(V + 31) / 32 * 4);
    s.bytes = s.parts + (n > EMBEDDING_CHUNK ? up256((uint64_t)ceil_div(n, EMBEDDING_CHUNK) * 2 * H * 4) : 0);
    return s;
}

extern "C" hap_status hap_embedding_backward_workspace(int64_t n, int32_t H, int64_t V, uint64_t *host_bytes)
{
    if (!host_bytes || !embedding_sizes(n, H, V)) return HAP_E_INVALID;
    *host_bytes = embedding_space(n, H, V).bytes;
    return HAP_OK;
}

extern "C" hap_status hap_embedding_backward(int32_t dtype, int32_t out_dtype, int32_t accumulate, int64_t n, int32_t H, int64_t V, int64_t first, const int64_t *tokens, const void *dy,
                                             int64_t lddy, float scale, void *dw, int64_t lddw, void *workspace, uint64_t bytes, void *stream)
{
    if (!dtype_fits(dtype) || (out_dtype != dtype && out_dtype != HAP_FP32) || !embedding_sizes(n, H, V) || lddy < H || lddw < H || !aligned(dy, size_of(dtype)) ||
        !aligned(dw, size_of(out_dtype)) || !aligned(tokens, 8) || !dw)
        return HAP_E_INVALID;
    if (n > 0 && (!tokens || !dy)) return HAP_E_INVALID;
    const EmbeddingSpace at = embedding_space(n, H, V);
    if (!workspace || bytes < at.bytes || !aligned(workspace, 256)) return HAP_E_INVALID;
    if (n == 0 && accumulate) return HAP_OK;
    cudaStream_t s = (cudaStream_t)stream;
    char *space = (char *)workspace;
    uint2 *a = (uint2 *)space, *b = (uint2 *)(space + at.other);
    const Digits d = digits_of(V);
    OrderArgs o{};
    o.n = n, o.keys = 1 << d.bits, o.bits = d.bits, o.passes = d.passes, o.counts = (int *)(space + at.counts), o.tokens = tokens, o.first_token = first, o.V = (int)V;
    o.present = accumulate ? nullptr : (unsigned *)(space + at.present);
    o.to = a;
    hap_status st = run_order<BY_TOKEN>(o, s);
    for (int i = 1; i < d.passes && st == HAP_OK; i++) {
        o.from = i & 1 ? a : b, o.to = i & 1 ? b : a, o.shift = i * d.bits, o.pass = i;
        st = run_order<BY_PAIR>(o, s);
    }
    if (st != HAP_OK) return st;
    EmbeddingArgs p{};
    p.n = n, p.H = H, p.V = (int)V, p.accumulate = accumulate != 0, p.scale = scale, p.x = dy, p.ldx = lddy, p.out = dw, p.ldo = lddw;
    p.sorted = o.to, p.parts = (float *)(space + at.parts), p.present = o.present;
    const bool w = H % 8 == 0 && wide(dy, lddy, dtype) && wide(dw, lddw, out_dtype);
    const int threads = (int)(ceil_div(H, 8) < 256 ? ceil_div(ceil_div(H, 8), 32) * 32 : 256);
    const int64_t chunks = ceil_div(n, EMBEDDING_CHUNK), columns = ceil_div(H, 8 * threads), tasks = chunks * columns;
    if (!grid_fits(tasks)) return HAP_E_RANGE;
    // blocks that sum: three a multiprocessor, which run at once (but two do, by their registers, where dy is in 32 bits or rows are not
    // whole sixteen bytes, and the third follows); behind them those that clear
    const int64_t most = 148 * 3, rows = ceil_div(V, threads / 32), clear = accumulate ? 0 : rows < 148 * 8 ? rows : 148 * 8;
    p.columns = (int)columns, p.sums = (int)(tasks < most ? tasks : most);
    const int64_t grid = p.sums + clear;
    auto all = [&](auto t, auto u) {
        using T = decltype(t);
        using O = decltype(u);
        const hap_status st = launch_next(w ? embedding_gradient_kernel<T, O, true> : embedding_gradient_kernel<T, O, false>, grid, threads, 0, 1, s, p);
        if (st != HAP_OK || chunks < 2) return st;
        return launch_next(w ? embedding_join_kernel<O, true> : embedding_join_kernel<O, false>, (chunks - 1) * columns, threads, 0, 1, s, p);
    };
    return by_type(dtype, [&](auto t) { return out_dtype == dtype ? all(t, t) : all(t, float()); });
}

// ---- layer norm ----------------------------------------------------------------------------------------------------------
static bool norm_sizes(int64_t rows, int32_t H) { return rows >= 0 && rows <= INT32_MAX && H >= 1 && H <= MOST_NORM; }

// A row's threads, two eights of columns each (four in half as many threads took 53 and 93 us against 46 and 77 for 8192 rows of 5120,
// forwards and backwards), and how many rows a device of 148 multiprocessors works on at once: as many as each has registers for, `most`
// threads, and shared memory, whose `row_bytes` hold the row that is worked on and the next.
constexpr int NORM_EIGHTS = 2;
static int norm_threads(int32_t H, int eights) { return (int)(ceil_div(ceil_div(H, 8 * eights), 32) * 32); }
static int norm_high(int threads) { return threads == 32 ? 4 : 1; }             // rows of a block
static int64_t norm_bytes(int32_t H, int arrays, int32_t dtype) { return (int64_t)arrays * 8 * NORM_EIGHTS * norm_threads(H, NORM_EIGHTS) * size_of(dtype); }
static int64_t norm_rows_at_once(int32_t H, int64_t row_bytes, int most)
{
    const int64_t threads = norm_threads(H, NORM_EIGHTS), by_threads = most / threads, by_bytes = (220 << 10) / (row_bytes + 1024);
    const int64_t n = by_threads < by_bytes ? by_threads : by_bytes;
    return 148 * (n < 1 ? 1 : n);
}
// Rows of partial sums: not more than a quarter of the rows, so that there is something to sum, but one for each multiprocessor
static int64_t norm_parts(int64_t rows, int32_t H, int64_t row_bytes)
{
    const int64_t at_once = norm_rows_at_once(H, row_bytes, 682), few = rows < 148 ? rows : rows / 4 < 148 ? 148 : rows / 4;
    const int64_t n = few < at_once ? few : at_once, high = norm_high(norm_threads(H, NORM_EIGHTS));
    return ceil_div(n, high) * high;
}

// the kernel may have this much shared memory, on this device
template <auto KERNEL> static hap_status allow_shared(Device d, int64_t bytes)
{
    static std::atomic<uint64_t> allowed;
    const uint64_t bit = d.id < DEVICES ? 1ull << d.id : 0;
    if (bytes <= 40 << 10 || (allowed.load(std::memory_order_relaxed) & bit)) return HAP_OK;
    if (status_of(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 << 10)) != HAP_OK) return HAP_E_CUDA;
    allowed.fetch_or(bit, std::memory_order_relaxed);
    return HAP_OK;
}
template <auto KERNEL> static hap_status launch_norm(const NormArgs &p, int64_t blocks, int threads, int high, int64_t bytes, cudaStream_t s)
{
    const Device d = device();
    if (!d.sms) return HAP_E_CUDA;
    const hap_status st = allow_shared<KERNEL>(d, bytes);
    if (st != HAP_OK) return st;
    cudaLaunchConfig_t c = shape_of(blocks, threads, (int)bytes, s);
    c.blockDim.y = high;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization, attr.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &attr, c.numAttrs = 1;
    return start(KERNEL, c, p);
}

extern "C" hap_status hap_layer_norm(int32_t dtype, int32_t param_dtype, int32_t centred, int64_t rows, int32_t H, const void *x, int64_t ldx, const void *w, const void *b, float eps, void *y,
                                     int64_t ldy, float *mean, float *rstd, void *stream)
{
    if (!dtype_fits(dtype) || (param_dtype != dtype && param_dtype != HAP_FP32) || !norm_sizes(rows, H) || ldx < H || ldy < H || !(eps >= 0) || !aligned(x, size_of(dtype)) ||
        !aligned(y, size_of(dtype)) || !aligned(w, size_of(param_dtype)) || !aligned(b, size_of(param_dtype)) || !aligned(mean, 4) || !aligned(rstd, 4) ||
        astray(y, ldy, x, ldx, rows))
        return HAP_E_INVALID;
    if (rows == 0) return HAP_OK;
    if (!x || !y) return HAP_E_INVALID;
    NormArgs p{};
    p.rows = rows, p.H = H, p.inverse = 1.0f / (float)H, p.eps = eps, p.x = x, p.ldx = ldx, p.w = w, p.b = b, p.y = y, p.ldy = ldy, p.mean = mean, p.rstd = rstd;
    const bool wd = H % 8 == 0 && wide(x, ldx, dtype) && wide(y, ldy, dtype) && aligned(w, 16) && aligned(b, 16);
    cudaStream_t s = (cudaStream_t)stream;
    // few rows: one eight for each thread (up to 8192 columns), and every row a block of its own
    const bool few = rows < 148 * 4;
    auto run = [&](auto t, auto u) {
        using T = decltype(t);
        using P = decltype(u);
        auto pick = [&](auto centre) {
            constexpr bool C = decltype(centre)::value;
            const int threads = norm_threads(H, few && H <= 8192 ? 1 : NORM_EIGHTS), high = norm_high(threads);
            const int64_t blocks = ceil_div(rows, high);
            if (few && H <= 8192) return wd ? launch_norm<norm_kernel<T, P, 1, false, true, C>>(p, blocks, threads, high, 0, s) : launch_norm<norm_kernel<T, P, 1, false, false, C>>(p, blocks, threads, high, 0, s);
            const int64_t row_bytes = 2 * norm_bytes(H, 1, dtype) + norm_bytes(H, 2, param_dtype);
            if (high * row_bytes > 220 << 10) {             // (long rows in 32 bits: each a block of its own)
                if constexpr (sizeof(T) == 4) return wd ? launch_norm<norm_kernel<T, P, NORM_EIGHTS, false, true, C>>(p, blocks, threads, high, 0, s) : launch_norm<norm_kernel<T, P, NORM_EIGHTS, false, false, C>>(p, blocks, threads, high, 0, s);
                return HAP_E_INVALID;
            }
            const int64_t most = ceil_div(norm_rows_at_once(H, row_bytes, 1024), high), grid = blocks < most ? blocks : most;
            return wd ? launch_norm<norm_kernel<T, P, NORM_EIGHTS, true, true, C>>(p, grid, threads, high, high * row_bytes, s)
                      : launch_norm<norm_kernel<T, P, NORM_EIGHTS, true, false, C>>(p, grid, threads, high, high * row_bytes, s);
        };
        return centred ? pick(std::true_type()) : pick(std::false_type());
    };
    return by_type(dtype, [&](auto t) { return param_dtype == dtype ? run(t, t) : run(t, float()); });
}

extern "C" hap_status hap_layer_norm_backward_workspace(int64_t rows, int32_t H, uint64_t *host_bytes)
{
    if (!host_bytes || !norm_sizes(rows, H)) return HAP_E_INVALID;
    *host_bytes = up256((uint64_t)norm_parts(rows, H, 0) * 2 * H * 4);      // (as for rows that need no shared memory)
    return HAP_OK;
}

extern "C" hap_status hap_layer_norm_backward(int32_t dtype, int32_t param_dtype, int32_t grad_dtype, int32_t accumulate, int32_t centred, int64_t rows, int32_t H, const void *dy, int64_t lddy,
                                              const void *x, int64_t ldx, const void *w, const float *mean, const float *rstd, const void *base, int64_t ldbase, void *dx, int64_t lddx, void *dw,
                                              void *db, void *workspace, uint64_t bytes, void *stream)
{
    const int64_t size = size_of(dtype), gsize = size_of(grad_dtype);
    if (!dtype_fits(dtype) || (param_dtype != dtype && param_dtype != HAP_FP32) || (grad_dtype != param_dtype && grad_dtype != HAP_FP32) || !norm_sizes(rows, H) || lddy < H || ldx < H ||
        (base && ldbase < H) || (dx && lddx < H) || !aligned(dy, size) || !aligned(x, size) || !aligned(base, size) || !aligned(dx, size) || !aligned(w, size_of(param_dtype)) ||
        !aligned(dw, gsize) || !aligned(db, gsize) || !aligned(mean, 4) || !aligned(rstd, 4) || (db && !centred) || astray(dx, lddx, dy, lddy, rows) ||
        astray(dx, lddx, x, ldx, rows) || astray(dx, lddx, base, ldbase, rows))
        return HAP_E_INVALID;
    if (rows > 0 && (!dy || !x || !rstd || (centred && !mean))) return HAP_E_INVALID;
    uint64_t need = 0;
    hap_layer_norm_backward_workspace(rows, H, &need);
    const bool sums = dw || db;
    if (sums && need && (!workspace || bytes < need || !aligned(workspace, 256))) return HAP_E_INVALID;
    if ((!dx && !sums) || (rows == 0 && (!sums || accumulate))) return HAP_OK;
    NormArgs p{};
    p.rows = rows, p.H = H, p.inverse = 1.0f / (float)H, p.add = accumulate != 0, p.x = x, p.ldx = ldx, p.w = w, p.dy = dy, p.lddy = lddy, p.base = base, p.ldbase = ldbase;
    p.dx = dx, p.lddx = lddx, p.dw = dw, p.db = db, p.mean = (float *)mean, p.rstd = (float *)rstd, p.parts = sums ? (float *)workspace : nullptr;
    cudaStream_t s = (cudaStream_t)stream;
    const bool wd = H % 8 == 0 && wide(x, ldx, dtype) && wide(dy, lddy, dtype) && (!base || wide(base, ldbase, dtype)) && (!dx || wide(dx, lddx, dtype)) && aligned(w, 16);
    const int threads = norm_threads(H, NORM_EIGHTS), high = norm_high(threads);
    const int64_t one = norm_bytes(H, threads <= 640 ? 3 : 2, dtype), kept = norm_bytes(H, 1, param_dtype);
    p.ahead = 2 * one + kept <= 220 << 10;                  // (long rows in 32 bits fill the shared memory alone)
    const int64_t row_bytes = (1 + p.ahead) * one + kept;
    p.blocks = (int)norm_parts(rows, H, row_bytes);
    auto run = [&](auto t, auto u) {
        using T = decltype(t);
        using P = decltype(u);
        auto pick = [&](auto centre, auto most) {
            constexpr bool C = decltype(centre)::value;
            constexpr int M = decltype(most)::value;
            return wd ? launch_norm<norm_backward_kernel<T, P, NORM_EIGHTS, M, true, C>>(p, p.blocks / high, threads, high, high * row_bytes, s)
                      : launch_norm<norm_backward_kernel<T, P, NORM_EIGHTS, M, false, C>>(p, p.blocks / high, threads, high, high * row_bytes, s);
        };
        using Few = std::integral_constant<int, 640>;
        using Many = std::integral_constant<int, 1024>;
        if (centred) return threads <= 640 ? pick(std::true_type(), Few()) : pick(std::true_type(), Many());
        return threads <= 640 ? pick(std::false_type(), Few()) : pick(std::false_type(), Many());
    };
    hap_status st = rows > 0 ? by_type(dtype, [&](auto t) { return param_dtype == dtype ? run(t, t) : run(t, float()); }) : HAP_OK;
    if (st != HAP_OK || !sums) return st;
    const int64_t blocks = ceil_div((int64_t)H * (centred ? 2 : 1), 32);
    return by_type(grad_dtype, [&](auto t) { return launch_next(norm_join_kernel<decltype(t)>, blocks, 256, 0, 1, s, p, centred ? 1 : 0); });
}
