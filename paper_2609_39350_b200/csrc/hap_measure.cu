// Times of the training operators on the current device, as entries of a planning problem's profile: the first step of the
// paper's pipeline (profile, model, search) for the one kind of device that the library runs on.  Runs the operators through
// their entry points on made-up values; nothing here knows how they work.
#include "../../include/hap.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdlib.h>

namespace {

constexpr int RANK_EXPERTS = 8;             // experts of the rank whose share is measured (all, where a layer has fewer)
constexpr int64_t PARAMETERS = 1 << 24;     // of the optimizer's step: their 12 bytes each are more than L2 holds
constexpr int TIMES = 5;                    // runs behind one that is not counted; the median counts

// values like a layer's: a sum of four uniform ones, scaled
__global__ void fill_kernel(__nv_bfloat16 *p, uint64_t n, float scale, uint32_t seed)
{
    for (uint64_t i = blockIdx.x * (uint64_t)blockDim.x + threadIdx.x; i < n; i += (uint64_t)gridDim.x * blockDim.x) {
        uint32_t x = (uint32_t)i * 2654435761u ^ (uint32_t)(i >> 32) ^ seed * 0x9e3779b9u;
        x ^= x >> 16, x *= 0x7feb352du, x ^= x >> 15, x *= 0x846ca68bu, x ^= x >> 16;
        const float s = (float)(x & 255) + (float)(x >> 8 & 255) + (float)(x >> 16 & 255) + (float)(x >> 24);
        p[i] = __float2bfloat16_rn((s - 510.0f) * (scale / 148.0f));
    }
}
__global__ void fill_targets_kernel(int64_t *p, int64_t n, int64_t V)
{
    for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) p[i] = (i * 7919) % V;
}
// offsets of E groups of equal sizes
__global__ void fill_offsets_kernel(int64_t *p, int E, int64_t rows)
{
    for (int i = threadIdx.x; i <= E; i += blockDim.x) p[i] = rows * i / E;
}
__global__ void fill_one_kernel(float *p, float x) { *p = x; }

// Memory of a workspace in the order it is asked for; without one it only counts.  Nothing may be launched on what was taken
// unless all of it fits.
struct Space {
    char *base;
    uint64_t bytes = 0, at = 0;
    template <typename T> T *take(uint64_t n)
    {
        const uint64_t from = at;
        at = (at + n * sizeof(T) + 255) / 256 * 256;
        return base && at <= bytes ? (T *)(base + from) : nullptr;
    }
    bool fits() const { return at <= bytes; }
};

int64_t shard(int64_t n, int64_t by) { const int64_t s = (n + by - 1) / by; return (s + 7) / 8 * 8; }       // a rank's share, as kernels like it

// The status of a CUDA call; a failed one's error is not left behind for the next launch to be blamed for.
hap_status status_of(cudaError_t e) { return e == cudaSuccess ? HAP_OK : (cudaGetLastError(), HAP_E_CUDA); }

struct Timer {
    cudaStream_t stream;
    cudaEvent_t from = nullptr, to = nullptr;
    bool good;
    explicit Timer(cudaStream_t s) : stream(s) { good = status_of(cudaEventCreate(&from)) == HAP_OK && status_of(cudaEventCreate(&to)) == HAP_OK; }
    ~Timer() { if (from) cudaEventDestroy(from); if (to) cudaEventDestroy(to); }
    // median time of `run` in ns, < 0 on an error, whose status is kept
    hap_status status = HAP_OK;
    template <typename F> double time(F &&run)
    {
        double t[TIMES];
        for (int i = -1; i < TIMES; i++) {
            float ms = 0;
            status = status_of(cudaEventRecord(from, stream));
            if (status == HAP_OK) status = run();
            if (status == HAP_OK) status = status_of(cudaEventRecord(to, stream));
            if (status == HAP_OK) status = status_of(cudaEventSynchronize(to));
            if (status == HAP_OK) status = status_of(cudaEventElapsedTime(&ms, from, to));
            if (status != HAP_OK) return -1;
            if (i >= 0) t[i] = (double)ms * 1e6;
        }
        for (int i = 1; i < TIMES; i++)
            for (int j = i; j > 0 && t[j] < t[j - 1]; j--) { const double x = t[j]; t[j] = t[j - 1], t[j - 1] = x; }
        return t[TIMES / 2];
    }
};

// The feed-forward block of E experts of width F on `rows` rows in equal shares: buffers and passes.
struct Block {
    int64_t rows;
    int H, F, E;
    int64_t *offsets;
    __nv_bfloat16 *x, *w13, *w2, *gu, *h, *y, *dy, *dgu, *dx, *dw13, *dw2;
    Block(Space &s, int64_t rows, int H, int F, int E) : rows(rows), H(H), F(F), E(E)
    {
        const uint64_t r = (uint64_t)rows, w = (uint64_t)E * F * H;
        offsets = s.take<int64_t>(E + 1);
        x = s.take<__nv_bfloat16>(r * H), w13 = s.take<__nv_bfloat16>(2 * w), w2 = s.take<__nv_bfloat16>(w), gu = s.take<__nv_bfloat16>(2 * r * F), h = s.take<__nv_bfloat16>(r * F);
        y = s.take<__nv_bfloat16>(r * H), dy = s.take<__nv_bfloat16>(r * H), dgu = s.take<__nv_bfloat16>(2 * r * F), dx = s.take<__nv_bfloat16>(r * H);
        dw13 = s.take<__nv_bfloat16>(2 * w), dw2 = s.take<__nv_bfloat16>(w);
    }
    void fill(cudaStream_t st)
    {
        const uint64_t r = (uint64_t)rows, w = (uint64_t)E * F * H;
        fill_offsets_kernel<<<1, 256, 0, st>>>(offsets, E, rows);
        fill_kernel<<<1024, 256, 0, st>>>(x, r * H, 1.0f, 1);
        fill_kernel<<<1024, 256, 0, st>>>(dy, r * H, 1.0f, 2);
        fill_kernel<<<1024, 256, 0, st>>>(w13, 2 * w, 1.0f / sqrtf((float)H), 3);
        fill_kernel<<<1024, 256, 0, st>>>(w2, w, 1.0f / sqrtf((float)F), 4);
    }
    hap_status forward(void *st)
    {
        hap_status s = hap_expert_gated(HAP_BF16, E, rows, H, F, offsets, x, H, w13, H, gu, 2 * F, h, F, st);
        return s != HAP_OK ? s : hap_expert_matmul(HAP_EXPERT_FORWARD, HAP_BF16, HAP_BF16, 0, E, rows, H, F, offsets, h, F, w2, F, y, H, st);
    }
    hap_status backward(void *st)
    {
        hap_status s = hap_expert_gated_backward(HAP_BF16, E, rows, H, F, offsets, dy, H, w2, F, gu, 2 * F, dgu, 2 * F, h, F, st);
        if (s == HAP_OK) s = hap_expert_matmul(HAP_EXPERT_GRAD_INPUT, HAP_BF16, HAP_BF16, 0, E, rows, 2 * F, H, offsets, dgu, 2 * F, w13, H, dx, H, st);
        if (s == HAP_OK) s = hap_expert_matmul(HAP_EXPERT_GRAD_WEIGHT, HAP_BF16, HAP_BF16, 0, E, rows, H, F, offsets, dy, H, h, F, dw2, F, st);
        if (s == HAP_OK) s = hap_expert_matmul(HAP_EXPERT_GRAD_WEIGHT, HAP_BF16, HAP_BF16, 0, E, rows, 2 * F, H, offsets, dgu, 2 * F, x, H, dw13, H, st);
        return s;
    }
};

struct Head {
    int64_t rows, V;
    int H;
    uint64_t bytes = 0;
    __nv_bfloat16 *x, *w, *dx, *dw;
    int64_t *target;
    float *loss, *lse, *grad;
    void *space;
    Head(Space &s, int64_t rows, int H, int64_t V) : rows(rows), V(V), H(H)
    {
        hap_linear_cross_entropy_workspace(rows, H, V, &bytes);
        x = s.take<__nv_bfloat16>((uint64_t)rows * H), w = s.take<__nv_bfloat16>((uint64_t)V * H), dx = s.take<__nv_bfloat16>((uint64_t)rows * H), dw = s.take<__nv_bfloat16>((uint64_t)V * H);
        target = s.take<int64_t>(rows), loss = s.take<float>(rows), lse = s.take<float>(rows), grad = s.take<float>(1), space = s.take<char>(bytes);
    }
    void fill(cudaStream_t st)
    {
        fill_kernel<<<1024, 256, 0, st>>>(x, (uint64_t)rows * H, 1.0f, 5);
        fill_kernel<<<1024, 256, 0, st>>>(w, (uint64_t)V * H, 2.0f / sqrtf((float)H), 6);
        fill_targets_kernel<<<64, 256, 0, st>>>(target, rows, V);
        fill_one_kernel<<<1, 1, 0, st>>>(grad, 1.0f / (float)rows);
    }
    hap_status run(void *st)
    {
        hap_status s = hap_linear_cross_entropy(HAP_BF16, rows, H, V, x, H, w, H, target, -100, loss, lse, space, bytes, st);
        return s != HAP_OK ? s : hap_linear_cross_entropy_backward(HAP_BF16, rows, H, V, x, H, w, H, target, -100, lse, grad, dx, H, dw, H, space, bytes, st);
    }
};

struct Update {
    hap_adamw_tensor t{};
    explicit Update(Space &s)
    {
        t.param = s.take<__nv_bfloat16>(PARAMETERS), t.grad = s.take<__nv_bfloat16>(PARAMETERS), t.m = s.take<float>(PARAMETERS), t.v = s.take<float>(PARAMETERS);
        t.count = PARAMETERS;
    }
    hap_status fill(cudaStream_t st)
    {
        fill_kernel<<<1024, 256, 0, st>>>((__nv_bfloat16 *)t.param, PARAMETERS, 0.02f, 7);
        fill_kernel<<<1024, 256, 0, st>>>((__nv_bfloat16 *)t.grad, PARAMETERS, 1e-3f, 8);
        return status_of(cudaMemsetAsync(t.m, 0, PARAMETERS * 4, st)) == HAP_OK ? status_of(cudaMemsetAsync(t.v, 0, PARAMETERS * 4, st)) : HAP_E_CUDA;
    }
    hap_status run(void *st)
    {
        const hap_adamw_options o = {1e-4, 0.9, 0.95, 1e-8, 0.1, 100};
        return hap_adamw_step(&t, 1, HAP_BF16, HAP_BF16, HAP_BF16, 32, &o, nullptr, st);
    }
};

struct Embedding {
    int64_t rows, V, words;
    int H;
    uint64_t bytes = 0;
    int64_t *tokens;
    __nv_bfloat16 *w, *out, *dy, *dw;
    void *space;
    Embedding(Space &s, int64_t rows, int H, int64_t V, int64_t words) : rows(rows), V(V), words(words), H(H)
    {
        hap_embedding_backward_workspace(rows, H, V, &bytes);
        tokens = s.take<int64_t>(rows), w = s.take<__nv_bfloat16>((uint64_t)V * H), out = s.take<__nv_bfloat16>((uint64_t)rows * H);
        dy = s.take<__nv_bfloat16>((uint64_t)rows * H), dw = s.take<__nv_bfloat16>((uint64_t)V * H), space = s.take<char>(bytes);
    }
    void fill(cudaStream_t st)
    {
        fill_targets_kernel<<<64, 256, 0, st>>>(tokens, rows, words);
        fill_kernel<<<1024, 256, 0, st>>>(w, (uint64_t)V * H, 0.02f, 9);
        fill_kernel<<<1024, 256, 0, st>>>(dy, (uint64_t)rows * H, 1.0f, 10);
    }
    hap_status run(void *st)
    {
        const hap_status s = hap_embedding(HAP_BF16, rows, H, V, 0, tokens, w, H, 1.0f, out, H, st);
        return s != HAP_OK ? s : hap_embedding_backward(HAP_BF16, HAP_BF16, 0, rows, H, V, 0, tokens, dy, H, 1.0f, dw, H, space, bytes, st);
    }
};

struct Norm {
    int64_t rows;
    int H;
    uint64_t bytes = 0;
    __nv_bfloat16 *x, *w, *b, *y, *dy, *dx, *dw, *db;
    float *mean, *rstd;
    void *space;
    Norm(Space &s, int64_t rows, int H) : rows(rows), H(H)
    {
        hap_layer_norm_backward_workspace(rows, H, &bytes);
        const uint64_t n = (uint64_t)rows * H;
        x = s.take<__nv_bfloat16>(n), y = s.take<__nv_bfloat16>(n), dy = s.take<__nv_bfloat16>(n), dx = s.take<__nv_bfloat16>(n);
        w = s.take<__nv_bfloat16>(H), b = s.take<__nv_bfloat16>(H), dw = s.take<__nv_bfloat16>(H), db = s.take<__nv_bfloat16>(H);
        mean = s.take<float>(rows), rstd = s.take<float>(rows), space = s.take<char>(bytes);
    }
    void fill(cudaStream_t st)
    {
        fill_kernel<<<1024, 256, 0, st>>>(x, (uint64_t)rows * H, 1.0f, 11);
        fill_kernel<<<1024, 256, 0, st>>>(dy, (uint64_t)rows * H, 1.0f, 12);
        fill_kernel<<<16, 256, 0, st>>>(w, H, 1.0f, 13);
        fill_kernel<<<16, 256, 0, st>>>(b, H, 0.1f, 14);
    }
    hap_status forward(void *st) { return hap_layer_norm(HAP_BF16, HAP_BF16, 1, rows, H, x, H, w, b, 1e-5f, y, H, mean, rstd, st); }
    hap_status backward(void *st)
    {
        return hap_layer_norm_backward(HAP_BF16, HAP_BF16, HAP_BF16, 0, 1, rows, H, dy, H, x, H, w, mean, rstd, nullptr, 0, dx, H, dw, db, space, bytes, st);
    }
};

// What a layer of experts does beside their products, on a device that has all of them: the router's logits and choice, the rows' way
// to the experts and back, and all of it backwards.
struct Router {
    int64_t rows;
    int H, E, k, ld;
    uint64_t bytes = 0;
    hap_routing how;
    __nv_bfloat16 *x, *w, *z, *dz, *there, *back, *y, *dx, *dw;
    int32_t *experts, *places;
    int64_t *offsets, *all;
    float *weights, *dweights;
    void *space;
    Router(Space &s, int64_t rows, int H, int E, int k) : rows(rows), H(H), E(E), k(k), ld((E + 7) / 8 * 8), how{E, k, HAP_SOFTMAX, 1, 1, 1, 1, 1.0f}
    {
        hap_expert_order_workspace(rows, k, E, &bytes);
        const uint64_t n = (uint64_t)rows * H, c = (uint64_t)rows * k;
        x = s.take<__nv_bfloat16>(n), w = s.take<__nv_bfloat16>((uint64_t)E * H), z = s.take<__nv_bfloat16>((uint64_t)rows * ld), dz = s.take<__nv_bfloat16>((uint64_t)rows * ld);
        there = s.take<__nv_bfloat16>(c * H), back = s.take<__nv_bfloat16>(c * H), y = s.take<__nv_bfloat16>(n), dx = s.take<__nv_bfloat16>(n), dw = s.take<__nv_bfloat16>((uint64_t)E * H);
        experts = s.take<int32_t>(c), places = s.take<int32_t>(c), offsets = s.take<int64_t>(E + 1), all = s.take<int64_t>(2);
        weights = s.take<float>(c), dweights = s.take<float>(c), space = s.take<char>(bytes);
    }
    void fill(cudaStream_t st)
    {
        fill_offsets_kernel<<<1, 32, 0, st>>>(all, 1, rows);
        fill_kernel<<<1024, 256, 0, st>>>(x, (uint64_t)rows * H, 1.0f, 15);
        fill_kernel<<<1024, 256, 0, st>>>(w, (uint64_t)E * H, 1.0f / sqrtf((float)H), 16);
        fill_kernel<<<1024, 256, 0, st>>>(y, (uint64_t)rows * H, 1.0f, 17);
    }
    hap_status forward(void *st)
    {
        hap_status s = hap_expert_matmul(HAP_EXPERT_FORWARD, HAP_BF16, HAP_BF16, 0, 1, rows, E, H, all, x, H, w, H, z, ld, st);
        if (s == HAP_OK) s = hap_route(&how, HAP_BF16, rows, z, ld, nullptr, experts, weights, st);
        if (s == HAP_OK) s = hap_expert_order(rows, k, 0, E, experts, offsets, places, space, bytes, st);
        if (s == HAP_OK) s = hap_expert_dispatch(HAP_BF16, rows, k, H, rows * k, x, H, places, there, H, st);
        if (s == HAP_OK) s = hap_expert_combine(HAP_BF16, rows, k, H, rows * k, there, H, places, weights, x, H, y, H, st);
        return s;
    }
    hap_status backward(void *st)
    {
        hap_status s = hap_expert_combine_backward(HAP_BF16, rows, k, H, rows * k, y, H, there, H, places, weights, back, H, dweights, st);
        if (s == HAP_OK) s = hap_expert_combine(HAP_BF16, rows, k, H, rows * k, back, H, places, nullptr, y, H, dx, H, st);
        if (s == HAP_OK) s = hap_route_backward(&how, HAP_BF16, rows, z, ld, experts, dweights, dz, ld, st);
        if (s == HAP_OK) s = hap_expert_matmul(HAP_EXPERT_GRAD_INPUT, HAP_BF16, HAP_BF16, 1, 1, rows, E, H, all, dz, ld, w, H, dx, H, st);
        if (s == HAP_OK) s = hap_expert_matmul(HAP_EXPERT_GRAD_WEIGHT, HAP_BF16, HAP_BF16, 0, 1, rows, E, H, all, dz, ld, x, H, dw, H, st);
        return s;
    }
};

bool list_fits(const int32_t *l, int n)
{
    if (n < 1 || n > HAP_MAX_LIST || !l) return false;
    for (int i = 0; i < n; i++)
        if (l[i] < 1) return false;
    return true;
}

bool fits(const hap_model *m, const hap_profile *p)
{
    return m && p && m->S >= 1 && m->S <= (1 << 24) && m->H >= 8 && m->H % 8 == 0 && m->H <= (1 << 20) && m->E >= 0 && m->E <= (1 << 16) && m->k >= 0 && m->k <= m->E && m->F_dense >= 0 &&
           m->F_exp >= 0 && m->F_dense <= (1 << 20) && m->F_exp <= (1 << 20) && m->F_dense + m->F_exp > 0 && m->V >= 1 && m->beta == 2.0 && list_fits(p->tp_list, p->ntp) &&
           list_fits(p->cp_list, p->ncp) && list_fits(p->mb_list, p->nmb);
}

int64_t tokens(const hap_model &m, int64_t b, int64_t cp) { const int64_t t = b * m.S / cp; return t < 1 ? 1 : t; }
// f(index, tokens, TP) for every entry of the profile's tables
template <typename F> void each_entry(const hap_model &m, const hap_profile &p, F &&f)
{
    for (int itp = 0; itp < p.ntp; itp++)
        for (int icp = 0; icp < p.ncp; icp++)
            for (int ib = 0; ib < p.nmb; ib++) f((itp * p.ncp + icp) * p.nmb + ib, tokens(m, p.mb_list[ib], p.cp_list[icp]), (int64_t)p.tp_list[itp]);
}
int64_t most_tokens(const hap_model &m, const hap_profile &p)
{
    int64_t most = 0;
    each_entry(m, p, [&](int, int64_t t, int64_t) { most = t > most ? t : most; });
    return most;
}
bool has_experts(const hap_model &m) { return m.E > 0 && m.k > 0 && m.F_exp > 0; }

struct Share { int E; int64_t rows; };
// of E experts' rows on one micro-batch, those of the measured rank
Share rank_share(const hap_model &m, int64_t toks)
{
    const int e = m.E < RANK_EXPERTS ? m.E : RANK_EXPERTS;
    const int64_t rows = toks * m.k * e / m.E;
    return {e, rows < e ? e : rows};
}

constexpr int64_t ROUTED_TOKENS = 8192;     // of the router's measurement, at most: its time is proportional to them
bool has_router(const hap_model &m) { return m.E > 0 && m.E <= 1024 && m.k > 0 && m.k <= 32; }
bool has_norm(const hap_model &m) { return m.H <= 16384; }
int64_t routed_tokens(const hap_model &m, const hap_profile &p) { const int64_t t = most_tokens(m, p); return t < ROUTED_TOKENS ? t : ROUTED_TOKENS; }

// A stream that may be measured on
hap_status not_captured(cudaStream_t s)
{
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    if (status_of(cudaStreamIsCapturing(s, &capture)) != HAP_OK) return HAP_E_CUDA;
    return capture == cudaStreamCaptureStatusNone ? HAP_OK : HAP_E_STATE;
}

} // namespace

extern "C" hap_status hap_measure_workspace(const hap_model *m, const hap_profile *p, uint64_t *host_bytes)
{
    if (!host_bytes || !fits(m, p)) return HAP_E_INVALID;
    const int64_t most = most_tokens(*m, *p);
    if (most >= (1ll << 29)) return HAP_E_RANGE;
    uint64_t need = 0;
    auto count = [&](auto &&make) {
        Space s{nullptr};
        make(s);
        need = s.at > need ? s.at : need;
    };
    // Everything that hap_measure_profile lays out.  The most tokens alone do not tell: the head's workspace is not monotone in
    // its rows, and eta takes a block of the whole width, whatever the degrees are.
    each_entry(*m, *p, [&](int, int64_t t, int64_t tp) {
        for (int F : {m->F_dense, m->F_exp})
            if (F > 0) count([&](Space &s) { Block(s, t, m->H, (int)shard(F, tp), 1); });
        count([&](Space &s) { Head(s, t, m->H, shard(m->V, tp)); });
    });
    if (has_experts(*m)) {
        const Share r = rank_share(*m, most);
        const int F = (int)shard(m->F_exp, 1);
        count([&](Space &s) { Block(s, most, m->H, F, 1); });
        count([&](Space &s) { Block(s, r.rows, m->H, F, r.E); });
        count([&](Space &s) { Block(s, 2 * r.rows, m->H, F, r.E); });
    }
    count([&](Space &s) { Update u(s); });
    *host_bytes = need;
    return HAP_OK;
}

extern "C" hap_status hap_measure_profile(const hap_model *m, const hap_profile *p, hap_measured *out, void *workspace, uint64_t bytes, void *stream)
{
    uint64_t need = 0;
    const hap_status st = hap_measure_workspace(m, p, &need);
    if (st != HAP_OK) return st;
    if (!out || !out->tff || !out->tfb || !out->tpost || !workspace || bytes < need || ((uintptr_t)workspace & 255)) return HAP_E_INVALID;
    cudaStream_t s = (cudaStream_t)stream;
    const hap_status free_stream = not_captured(s);
    if (free_stream != HAP_OK) return free_stream;
    Timer timer(s);
    if (!timer.good) return HAP_E_CUDA;
    // the same sizes come up under several degrees (tokens b S / CP): each is measured once
    struct Known { int64_t t; int64_t width; double f, b; };
    const int most_known = 2 * HAP_MAX_LIST * HAP_MAX_LIST * HAP_MAX_LIST;
    Known *heads = (Known *)malloc(sizeof(Known) * most_known), *blocks = (Known *)malloc(sizeof(Known) * most_known);
    if (!heads || !blocks) {
        free(heads), free(blocks);
        return HAP_E_NOMEM;
    }
    int n_heads = 0, n_blocks = 0;
    auto block = [&](int64_t t, int F, int E, double &f, double &b) {
        for (int i = 0; E == 1 && i < n_blocks; i++)
            if (blocks[i].t == t && blocks[i].width == F) { f = blocks[i].f, b = blocks[i].b; return timer.status; }
        Space sp{(char *)workspace, bytes};
        Block x(sp, t, m->H, F, E);
        if (!sp.fits()) return HAP_E_INVALID;
        x.fill(s);
        f = timer.time([&] { return x.forward(stream); });
        b = timer.status == HAP_OK ? timer.time([&] { return x.backward(stream); }) : 0;
        if (E == 1 && timer.status == HAP_OK && n_blocks < most_known) blocks[n_blocks++] = {t, F, f, b};
        return timer.status;
    };
    hap_status bad = HAP_OK;
    each_entry(*m, *p, [&](int at, int64_t t, int64_t tp) {
        for (int kind = 0; kind < 2 && bad == HAP_OK; kind++) {
            const int F = kind == HAP_DENSE ? m->F_dense : m->F_exp;
            double f = 0, b = 0;
            if (F > 0) bad = block(t, (int)shard(F, tp), 1, f, b);
            out->tff[2 * at + kind] = f, out->tfb[2 * at + kind] = b;
        }
        if (bad != HAP_OK) return;
        const int64_t V = shard(m->V, tp);
        double f = -1;
        for (int i = 0; i < n_heads; i++)
            if (heads[i].t == t && heads[i].width == V) f = heads[i].f;
        if (f < 0) {
            Space sp{(char *)workspace, bytes};
            Head h(sp, t, m->H, V);
            if (!sp.fits()) {
                bad = HAP_E_INVALID;
                return;
            }
            h.fill(s);
            f = timer.time([&] { return h.run(stream); });
            if ((bad = timer.status) == HAP_OK && n_heads < most_known) heads[n_heads++] = {t, V, f, 0};
        }
        out->tpost[at] = f;
    });
    out->eta = 1, out->gamma = 0;
    if (bad == HAP_OK && has_experts(*m)) {
        const int64_t t = most_tokens(*m, *p);
        const int F = (int)shard(m->F_exp, 1);
        const Share r = rank_share(*m, t);
        double f1 = 0, b1 = 0, f2 = 0, b2 = 0, f = 0, b = 0;
        bad = block(t, F, 1, f, b);                         // one block on the micro-batch's tokens
        if (bad == HAP_OK) bad = block(r.rows, F, r.E, f1, b1);
        if (bad == HAP_OK) bad = block(2 * r.rows, F, r.E, f2, b2);
        if (bad == HAP_OK) {
            const double ideal = (f + b) * (double)r.rows / (double)t, even = f1 + b1, twice = f2 + b2;
            out->eta = ideal < even ? ideal / even : 1;
            const double g = twice / even - 1;
            out->gamma = g < 0 ? 0 : g > 1 ? 1 : g;
        }
    }
    if (bad == HAP_OK) {
        Space sp{(char *)workspace, bytes};
        Update u(sp);
        bad = sp.fits() ? u.fill(s) : HAP_E_INVALID;
        if (bad == HAP_OK) {
            out->copt = timer.time([&] { return u.run(stream); }) / (double)PARAMETERS;
            bad = timer.status;
        }
    }
    free(heads), free(blocks);
    return bad;
}

extern "C" hap_status hap_measure_tokens_workspace(const hap_model *m, const hap_profile *p, uint64_t *host_bytes)
{
    if (!host_bytes || !fits(m, p)) return HAP_E_INVALID;
    if (most_tokens(*m, *p) >= (1ll << 29)) return HAP_E_RANGE;
    uint64_t need = 0;
    auto count = [&](auto &&make) {
        Space s{nullptr};
        make(s);
        need = s.at > need ? s.at : need;
    };
    each_entry(*m, *p, [&](int, int64_t t, int64_t tp) {
        count([&](Space &s) { Embedding(s, t, m->H, shard(m->V, tp), m->V); });
        if (has_norm(*m)) count([&](Space &s) { Norm(s, t, m->H); });
    });
    if (has_router(*m)) count([&](Space &s) { Router(s, routed_tokens(*m, *p), m->H, m->E, m->k); });
    *host_bytes = need;
    return HAP_OK;
}

extern "C" hap_status hap_measure_tokens(const hap_model *m, const hap_profile *p, hap_measured_tokens *out, void *workspace, uint64_t bytes, void *stream)
{
    uint64_t need = 0;
    hap_status bad = hap_measure_tokens_workspace(m, p, &need);
    if (bad != HAP_OK) return bad;
    if (!out || !out->tpre || !out->tnorm || !workspace || bytes < need || ((uintptr_t)workspace & 255)) return HAP_E_INVALID;
    cudaStream_t s = (cudaStream_t)stream;
    if ((bad = not_captured(s)) != HAP_OK) return bad;
    Timer timer(s);
    if (!timer.good) return HAP_E_CUDA;
    // entry 0 of a table is made whatever was before it: sizes that came up are looked for among the entries that are done
    auto before = [&](int at, int64_t t, int64_t V) {
        int found = -1;
        each_entry(*m, *p, [&](int i, int64_t t2, int64_t tp2) {
            if (i < at && found < 0 && t2 == t && (V < 0 || shard(m->V, tp2) == V)) found = i;
        });
        return found;
    };
    each_entry(*m, *p, [&](int at, int64_t t, int64_t tp) {
        if (bad != HAP_OK) return;
        const int64_t V = shard(m->V, tp);
        int was = before(at, t, V);
        if (was >= 0) out->tpre[at] = out->tpre[was];
        else {
            Space sp{(char *)workspace, bytes};
            Embedding e(sp, t, m->H, V, m->V);
            if (!sp.fits()) { bad = HAP_E_INVALID; return; }
            e.fill(s);
            out->tpre[at] = timer.time([&] { return e.run(stream); });
            if ((bad = timer.status) != HAP_OK) return;
        }
        was = before(at, t, -1);
        double *norm = out->tnorm + 2 * at;
        if (!has_norm(*m)) norm[0] = norm[1] = 0;
        else if (was >= 0) norm[0] = out->tnorm[2 * was], norm[1] = out->tnorm[2 * was + 1];
        else {
            Space sp{(char *)workspace, bytes};
            Norm n(sp, t, m->H);
            if (!sp.fits()) { bad = HAP_E_INVALID; return; }
            n.fill(s);
            norm[0] = timer.time([&] { return n.forward(stream); });
            if ((bad = timer.status) == HAP_OK) norm[1] = timer.time([&] { return n.backward(stream); });
            if (bad == HAP_OK) bad = timer.status;
        }
    });
    out->croute = 0;
    if (bad == HAP_OK && has_router(*m)) {
        const int64_t t = routed_tokens(*m, *p);
        Space sp{(char *)workspace, bytes};
        Router r(sp, t, m->H, m->E, m->k);
        if (!sp.fits()) return HAP_E_INVALID;
        r.fill(s);
        const double f = timer.time([&] { return r.forward(stream); });
        if ((bad = timer.status) != HAP_OK) return bad;
        const double b = timer.time([&] { return r.backward(stream); });
        if ((bad = timer.status) != HAP_OK) return bad;
        out->croute = (f + b) / (3.0 * (double)t * (double)m->H);
    }
    return bad;
}
