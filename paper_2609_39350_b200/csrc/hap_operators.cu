// Host side of the training operators: checks of arguments, choice of variant, launches.
#include "hap_adamw.cuh"
#include "hap_products_experts.cuh"
#include "hap_products_few.cuh"
#include "hap_products_tc.cuh"

#include <atomic>
#include <math.h>

using namespace hapop;


// The status of a CUDA call.  A failed one also leaves its error behind, for whoever asks for the last error next: it is taken back.
static hap_status status_of(cudaError_t e) { return e == cudaSuccess ? HAP_OK : (cudaGetLastError(), HAP_E_CUDA); }
// Launches, and says whether this launch was made, not whether any call so far left an error behind.  Arguments of the kernel's own
// types are passed where they are, without a copy.
template <typename T> struct Same { using type = T; };
template <typename... P> static hap_status start(void (*kernel)(P...), const cudaLaunchConfig_t &c, const typename Same<P>::type &...args)
{
    void *at[] = {(void *)&args...};
    return status_of(cudaLaunchKernelExC(&c, (const void *)kernel, at));
}
static cudaLaunchConfig_t shape_of(int64_t grid, int threads, int smem, cudaStream_t stream)
{
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)grid), c.blockDim = dim3((unsigned)threads), c.dynamicSmemBytes = (size_t)smem, c.stream = stream;
    return c;
}

// The current device and its multiprocessors; 0 of them: no device.  What does not change is asked once for each device.
struct Device { int id = 0, sms = 0; };
constexpr int DEVICES = 64;

static Device device()
{
    static std::atomic<int> known[DEVICES];
    Device d;
    if (status_of(cudaGetDevice(&d.id)) != HAP_OK || d.id < 0) return d;
    if (d.id < DEVICES) d.sms = known[d.id].load(std::memory_order_relaxed);
    if (d.sms) return d;
    if (status_of(cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, d.id)) != HAP_OK) d.sms = 0;
    if (d.id < DEVICES) known[d.id].store(d.sms, std::memory_order_relaxed);
    return d;
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---- tensor maps ------------------------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiled encode_tiled()
{
    static const EncodeTiled f = [] {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (status_of(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &r)) != HAP_OK || r != cudaDriverEntryPointSuccess) fn = nullptr;
        return (EncodeTiled)fn;
    }();
    return f;
}

// `count` matrices [rows][cols] of 16-bit values, read in boxes of 64 columns and box_rows rows; what lies outside arrives as 0
static bool make_map(CUtensorMap *map, bool fp16, const void *base, int64_t cols, int64_t rows, int64_t count, int64_t ld, int64_t distance, int box_rows)
{
    if (count < 2) distance = ld * rows;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)count}, strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)distance * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, each[3] = {1, 1, 1};
    return encode_tiled()(map, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, (void *)base, dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// whether TMA can address an operand
static bool mappable(const void *base, int64_t ld) { return ((uintptr_t)base & 15) == 0 && ld % 8 == 0 && ld < (1ll << 36); }

// Launches a kernel that may start while its predecessor in the stream still ends: its setup (barriers, tensor memory, maps) and the
// launch itself then cost nothing (loss of 129 rows: 28.7 -> 25.3 us).  The kernel waits for the predecessor before it reads.
template <typename... P> static hap_status launch_next(void (*kernel)(P...), int64_t grid, int threads, int smem, int cluster, cudaStream_t stream, const typename Same<P>::type &...args)
{
    cudaLaunchConfig_t c = shape_of(grid, threads, smem, stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization, attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension, attr[1].val.clusterDim = {(unsigned)cluster, 1, 1};
    c.attrs = attr, c.numAttrs = cluster > 1 ? 2 : 1;
    return start(kernel, c, args...);
}

// a persistent kernel of blocks or pairs of blocks, as many as fit and `most` tiles need
template <auto KERNEL, int CG = 2, int THREADS = 320, typename... A> static hap_status launch_pairs(int smem, int64_t most, Device d, cudaStream_t stream, const A &...args)
{
    static std::atomic<uint64_t> allowed;                   // devices on which the kernel may have this much shared memory
    const uint64_t bit = d.id < DEVICES ? 1ull << d.id : 0;
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
        if (status_of(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != HAP_OK) return HAP_E_CUDA;
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    const int64_t at_once = d.sms / CG;
    return launch_next(KERNEL, (most < at_once ? most : at_once) * CG, THREADS, smem, CG, stream, args...);
}

template <typename T, int FORM, int EPI, int CG> static hap_status launch_tensor(Args p, Device d, cudaStream_t stream)
{
    using S = Shape<EPI, CG>;
    const int64_t cols = ceil_div(p.ncols, TILE_N) * (EPI == SUM32 ? p.splits : 1);
    const int64_t most = cols * (FORM == TN ? p.groups * ceil_div(p.mdim, S::BM) : ceil_div(p.rows, S::BM) + (p.offsets ? p.groups : 0));
    if (most > INT32_MAX) return HAP_E_RANGE;
    constexpr bool fp16 = TypeBits<T>::value == 0;
    CUtensorMap ma, mb, mo{};
    const int64_t wrows = FORM == NT ? p.ncols : p.kdim;
    const bool good = FORM == TN ? make_map(&ma, fp16, p.a, p.mdim, p.rows, 1, p.lda, 0, BK) && make_map(&mb, fp16, p.b, p.ncols, p.rows, 1, p.ldb, 0, BK)
                                 : make_map(&ma, fp16, p.a, p.kdim, p.rows, 1, p.lda, 0, 128) &&
                                       make_map(&mb, fp16, p.b, FORM == NT ? p.kdim : p.ncols, wrows, p.groups, p.ldb, p.bgroup, FORM == NT ? 128 : BK);
    if (!good) return HAP_E_CUDA;
    if (EPI == STORE32 && FORM == TN && ((uintptr_t)p.out & 15) == 0 && p.ldo % 4 == 0 && p.ldo < (1ll << 35) && p.ogroup < (1ll << 35)) {
        const cuuint64_t dims[3] = {(cuuint64_t)p.ncols, (cuuint64_t)p.mdim, (cuuint64_t)p.groups};
        const cuuint64_t strides[2] = {(cuuint64_t)p.ldo * 4, (cuuint64_t)(p.groups > 1 ? p.ogroup : p.ldo * p.mdim) * 4};
        const cuuint32_t box[3] = {32, 32, 1}, each[3] = {1, 1, 1};
        p.out_mapped = encode_tiled()(&mo, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, p.out, dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                      CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    }
    constexpr int smem = 1024 + S::STAGES * S::STAGE + 8 * S::OUT + sizeof(Shared<EPI, CG>);
    return launch_pairs<product_kernel<T, FORM, EPI, CG>, CG, FORM == TN ? 352 : 320>(smem, most, d, stream, p, ma, mb, mo);
}

// experts' rows as columns of the products (NT, NN; out in 16 bits)
template <typename T, int FORM, int EPI> static hap_status launch_experts(Args p, Device d, cudaStream_t stream)
{
    using S = Turned<EPI>;
    const int64_t most = ceil_div(p.ncols, 256) * (ceil_div(p.rows, S::ROWS) + p.groups);
    if (most > INT32_MAX) return HAP_E_RANGE;
    constexpr bool fp16 = TypeBits<T>::value == 0;
    CUtensorMap mw, mr, mf, mk{};
    const int64_t wrows = FORM == NT ? (EPI == GATED ? 2ll * p.ncols : p.ncols) : p.kdim;
    if (!make_map(&mw, fp16, p.b, FORM == NT ? p.kdim : p.ncols, wrows, p.groups, p.ldb, p.bgroup, FORM == NT ? 128 : BK) ||
        !make_map(&mr, fp16, p.a, p.kdim, p.rows, 1, p.lda, 0, S::ROWS / 2) || !make_map(&mf, fp16, p.a, p.kdim, p.rows, 1, p.lda, 0, 16))
        return HAP_E_CUDA;
    if (EPI == GATED_BACK && mappable(p.gu, p.ldgu) && p.ncols % 8 == 0) {      // (u begins ncols values behind g, at a multiple of 16 bytes)
        const cuuint64_t dims[3] = {2 * (cuuint64_t)p.ncols, (cuuint64_t)p.rows, 1}, strides[2] = {(cuuint64_t)p.ldgu * 2, (cuuint64_t)p.ldgu * 2 * (cuuint64_t)p.rows};
        const cuuint32_t box[3] = {32, 16, 1}, each[3] = {1, 1, 1};
        p.kept_mapped = encode_tiled()(&mk, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, (void *)p.gu, dims, strides, box, each,
                                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    }
    return launch_pairs<expert_kernel<T, FORM, EPI>>(1024 + S::STAGES * S::STAGE + 8 * (S::OUT + S::KEPT) + sizeof(TurnedShared<EPI>), most, d, stream, p, mw, mr, mf, mk);
}

template <typename T, int FORM, int EPI> static hap_status launch_plain(const Args &p, int sms, cudaStream_t stream)
{
    if (EPI == SUM32 && p.splits > 1) return HAP_E_INVALID;                     // (it makes one sum)
    const int64_t cols = ceil_div(p.ncols, EPI == GATED ? TILE_N / 2 : TILE_N);
    const int64_t most = cols * (FORM == TN ? p.groups * ceil_div(p.mdim, PM) : ceil_div(p.rows, PM) + p.groups);
    if (most > INT32_MAX) return HAP_E_RANGE;
    return start(plain_product_kernel<T, FORM, EPI>, shape_of(most < 4 * sms ? most : 4 * sms, 256, 0, stream), p);
}

// whether a product runs on the tensor cores, or in the plain kernel
static bool on_tensor_cores(const Args &p) { return p.rows > 0 && mappable(p.a, p.lda) && mappable(p.b, p.ldb) && p.bgroup < (1ll << 36) && encode_tiled(); }

template <typename T, int FORM, int EPI> static hap_status launch_product(const Args &p, cudaStream_t stream)
{
    const Device d = device();
    if (!d.sms) return HAP_E_CUDA;
    if (!on_tensor_cores(p)) return launch_plain<T, FORM, EPI>(p, d.sms, stream);
    if constexpr (FORM != TN && (EPI == STORE || EPI == GATED || EPI == GATED_BACK)) {
        if constexpr (FORM == NT) {
            if (p.rows <= FEW_ROWS) {
                const int64_t warps = p.groups * (EPI == GATED ? (int64_t)p.ncols : ceil_div(p.ncols, 2)), blocks = ceil_div(warps, 8);
                return launch_next(few_rows_kernel<T, EPI>, blocks < 4 * d.sms ? blocks : 4 * d.sms, 256, 0, 1, stream, p);
            }
        }
        return launch_experts<T, FORM, EPI>(p, d, stream);
    } else {
        // rows of the output: up to 128 fill one block's tile, and pairs cost more to start (loss of 128 rows, 1024 x 32003: 17.5 us
        // alone, 23.4 in pairs; 8192 x 16000: 67 and 58); above, a pair reads each operand half as often (8192 x 8192 x 8192: 1483
        // and 1662 TFLOP/s)
        const int64_t high = FORM == TN ? p.mdim : p.rows;
        return high > 128 ? launch_tensor<T, FORM, EPI, 2>(p, d, stream) : launch_tensor<T, FORM, EPI, 1>(p, d, stream);
    }
}

static bool dtype16(int32_t t) { return t == HAP_BF16 || t == HAP_FP16; }
static int64_t size_of(int32_t t) { return t == HAP_FP32 ? 4 : 2; }
static bool aligned(const void *p, int64_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
// sizes that the kernels' 32-bit indexes hold
static bool sizes_fit(int64_t rows, int64_t n, int64_t k) { return rows >= 0 && rows < (1ll << 30) && n >= 1 && n < (1 << 28) && k >= 1 && k < (1 << 28); }

extern "C" hap_status hap_expert_matmul(int32_t form, int32_t dtype, int32_t out_dtype, int32_t accumulate, int32_t E, int64_t rows, int32_t N, int32_t K,
                                        const int64_t *offsets, const void *a, int64_t lda, const void *b, int64_t ldb, void *out, int64_t ldo, void *stream)
{
    if (form < HAP_EXPERT_FORWARD || form > HAP_EXPERT_GRAD_WEIGHT || !dtype16(dtype) || (out_dtype != dtype && out_dtype != HAP_FP32)) return HAP_E_INVALID;
    if (E < 1 || E > MAX_GROUPS || !sizes_fit(rows, N, K)) return HAP_E_INVALID;
    const bool grad_w = form == HAP_EXPERT_GRAD_WEIGHT;
    if (!offsets || (!out && (rows > 0 || grad_w)) || (rows > 0 && (!a || !b))) return HAP_E_INVALID;
    if (lda < (form == HAP_EXPERT_FORWARD ? K : N) || ldb < K || ldo < (form == HAP_EXPERT_FORWARD ? N : K)) return HAP_E_INVALID;
    if (!aligned(a, 2) || !aligned(b, 2) || !aligned(out, size_of(out_dtype)) || !aligned(offsets, 8)) return HAP_E_INVALID;
    if (rows == 0 && (!grad_w || accumulate)) return HAP_OK;
    Args p{};
    p.offsets = offsets, p.groups = E, p.rows = (int)rows;
    p.mdim = N, p.ncols = form == HAP_EXPERT_FORWARD ? N : K, p.kdim = form == HAP_EXPERT_FORWARD ? K : N;
    p.a = a, p.b = b, p.lda = lda, p.ldb = ldb, p.bgroup = (int64_t)N * ldb;
    p.out = out, p.ldo = ldo, p.ogroup = grad_w ? (int64_t)N * ldo : 0;
    p.accumulate = accumulate != 0;
    cudaStream_t s = (cudaStream_t)stream;
#define HAP_BY_TYPE(FORM, EPI) (dtype == HAP_BF16 ? launch_product<__nv_bfloat16, FORM, EPI>(p, s) : launch_product<__half, FORM, EPI>(p, s))
    if (out_dtype == HAP_FP32) return form == HAP_EXPERT_FORWARD ? HAP_BY_TYPE(NT, STORE32) : grad_w ? HAP_BY_TYPE(TN, STORE32) : HAP_BY_TYPE(NN, STORE32);
    return form == HAP_EXPERT_FORWARD ? HAP_BY_TYPE(NT, STORE) : grad_w ? HAP_BY_TYPE(TN, STORE) : HAP_BY_TYPE(NN, STORE);
}

extern "C" hap_status hap_expert_gated(int32_t dtype, int32_t E, int64_t rows, int32_t H, int32_t F, const int64_t *offsets, const void *x, int64_t ldx,
                                       const void *w, int64_t ldw, void *gu, int64_t ldgu, void *h, int64_t ldh, void *stream)
{
    if (!dtype16(dtype) || E < 1 || E > MAX_GROUPS || !sizes_fit(rows, 2ll * F, H)) return HAP_E_INVALID;
    if (!offsets || (rows > 0 && (!x || !w || !h))) return HAP_E_INVALID;
    if (ldx < H || ldw < H || ldh < F || (gu && ldgu < 2ll * F)) return HAP_E_INVALID;
    if (!aligned(x, 2) || !aligned(w, 2) || !aligned(gu, 2) || !aligned(h, 2) || !aligned(offsets, 8)) return HAP_E_INVALID;
    if (rows == 0) return HAP_OK;
    Args p{};
    p.offsets = offsets, p.groups = E, p.rows = (int)rows, p.ncols = F, p.kdim = H;
    p.a = x, p.b = w, p.lda = ldx, p.ldb = ldw, p.bgroup = 2ll * F * ldw;
    p.out = gu, p.ldo = ldgu, p.h = h, p.ldh = ldh;
    cudaStream_t s = (cudaStream_t)stream;
    return HAP_BY_TYPE(NT, GATED);
}

extern "C" hap_status hap_expert_gated_backward(int32_t dtype, int32_t E, int64_t rows, int32_t H, int32_t F, const int64_t *offsets, const void *dy,
                                                int64_t ldy, const void *w2, int64_t ldw, const void *gu, int64_t ldgu, void *dgu, int64_t lddgu,
                                                void *h, int64_t ldh, void *stream)
{
    if (!dtype16(dtype) || E < 1 || E > MAX_GROUPS || !sizes_fit(rows, 2ll * F, H)) return HAP_E_INVALID;
    if (!offsets || (rows > 0 && (!dy || !w2 || !gu || !dgu))) return HAP_E_INVALID;
    if (ldy < H || ldw < F || ldgu < 2ll * F || lddgu < 2ll * F || (h && ldh < F)) return HAP_E_INVALID;
    if (!aligned(dy, 2) || !aligned(w2, 2) || !aligned(gu, 2) || !aligned(dgu, 2) || !aligned(h, 2) || !aligned(offsets, 8)) return HAP_E_INVALID;
    if (gu == dgu && ldgu != lddgu) return HAP_E_INVALID;
    if (rows == 0) return HAP_OK;
    Args p{};
    p.offsets = offsets, p.groups = E, p.rows = (int)rows, p.ncols = F, p.kdim = H;
    p.a = dy, p.b = w2, p.lda = ldy, p.ldb = ldw, p.bgroup = (int64_t)H * ldw;
    p.out = dgu, p.ldo = lddgu, p.gu = gu, p.ldgu = ldgu, p.h = h, p.ldh = ldh;
    cudaStream_t s = (cudaStream_t)stream;
    return HAP_BY_TYPE(NN, GATED_BACK);
}

// ---- cross entropy of the output head ----------------------------------------------------------------------------------
// Columns of the vocabulary per piece of the backward pass: the piece's softmax gradients (rows x columns x 2 bytes) take up to
// 192 MiB.  Fewer pieces read and write dx's sums less often, but hold more of what is not to be kept (4096 rows, 5120 x 102400:
// 9.1 ms with 48 MiB, 8.7 with 96, 8.6 with 192, 8.5 with 384).
static int64_t piece_columns(int64_t rows, int64_t V)
{
    int64_t c = (192ll << 20) / (2 * (rows < 1 ? 1 : rows)) / TILE_N * TILE_N;
    if (c < 8 * TILE_N) c = 8 * TILE_N;
    const int64_t whole = ceil_div(V, TILE_N) * TILE_N;
    return c < whole ? c : whole;
}
static uint64_t up256(uint64_t n) { return (n + 255) / 256 * 256; }

// With few rows a gradient of the weight is one row's or a few rows' and the roundings of the softmax gradients are not averaged:
// up to this many rows they are kept as two 16-bit numbers each, and the product runs over both halves.  (With more, the error
// is 1.0 to 1.4 times that of rounding the result alone.)
constexpr int64_t TWICE_ROWS = 128;

// dx of few rows is few tiles with the longest contraction there is, the vocabulary: it is split so that each of the device's 74
// pairs of blocks has a tile, into parts of at least 1024 (8 rows, 1024 x 100000: 618 -> 128 us)
static int parts_of_dx(int64_t rows, int64_t H, int64_t piece)
{
    const int64_t tiles = ceil_div(rows < 1 ? 1 : rows, 2 * 128) * ceil_div(H, TILE_N), fit = 74 / tiles, most = ceil_div(piece, 1024);
    return (int)(fit < 2 ? 1 : fit < most ? fit : most);
}

// where the parts of the backward pass's workspace begin
struct LossSpace { uint64_t residual, acc, x2, bytes; };
static LossSpace loss_space(int64_t rows, int64_t H, int64_t V)
{
    const uint64_t n = (uint64_t)rows, piece = (uint64_t)piece_columns(rows, V), halves = rows <= TWICE_ROWS ? 2 : 1;
    LossSpace s;
    s.residual = up256(halves * n * piece * 2);
    s.acc = s.residual + up256(n * 4);
    const uint64_t parts = (uint64_t)parts_of_dx(rows, H, (int64_t)piece);
    s.x2 = s.acc + ((int64_t)piece < V || parts > 1 ? up256(parts * n * H * 4) : 0);
    s.bytes = s.x2 + (halves > 1 ? up256(2 * n * ((H + 7) / 8 * 8) * 2) : 0);
    return s;
}

static bool loss_sizes(int64_t rows, int64_t H, int64_t V) { return sizes_fit(rows, V, H); }

extern "C" hap_status hap_linear_cross_entropy_workspace(int64_t rows, int32_t H, int64_t V, uint64_t *host_bytes)
{
    if (!host_bytes || !loss_sizes(rows, H, V)) return HAP_E_INVALID;
    const uint64_t n = (uint64_t)rows;
    const uint64_t forward = up256(ceil_div(V, PART_N) * n * 8) + up256(n * 4), backward = loss_space(rows, H, V).bytes;
    *host_bytes = forward > backward ? forward : backward;
    return HAP_OK;
}

static hap_status loss_args(int32_t dtype, int64_t rows, int32_t H, int64_t V, const void *x, int64_t ldx, const void *w, int64_t ldw, const int64_t *target,
                            const void *workspace, uint64_t bytes)
{
    if (!dtype16(dtype) || !loss_sizes(rows, H, V) || ldx < H || ldw < H || !aligned(x, 2) || !aligned(w, 2) || !aligned(target, 8)) return HAP_E_INVALID;
    if (rows > 0 && (!x || !w || !target)) return HAP_E_INVALID;
    uint64_t need = 0;
    hap_linear_cross_entropy_workspace(rows, H, V, &need);
    return need && (!workspace || bytes < need || !aligned(workspace, 256)) ? HAP_E_INVALID : HAP_OK;
}

extern "C" hap_status hap_linear_cross_entropy(int32_t dtype, int64_t rows, int32_t H, int64_t V, const void *x, int64_t ldx, const void *w, int64_t ldw,
                                               const int64_t *target, int64_t ignore, float *loss, float *lse, void *workspace, uint64_t bytes, void *stream)
{
    const hap_status bad = loss_args(dtype, rows, H, V, x, ldx, w, ldw, target, workspace, bytes);
    if (bad != HAP_OK) return bad;
    if (rows == 0) return HAP_OK;
    if (!loss || !lse || !aligned(loss, 4) || !aligned(lse, 4)) return HAP_E_INVALID;
    const int pieces = (int)ceil_div(V, PART_N);
    Args p{};
    p.groups = 1, p.rows = (int)rows, p.ncols = (int)V, p.kdim = H;
    p.a = x, p.b = w, p.lda = ldx, p.ldb = ldw;
    p.target = target, p.ignore = ignore, p.vocab = V;
    p.part = (float2 *)workspace, p.at_target = (float *)((char *)workspace + up256((uint64_t)pieces * rows * 8));
    cudaStream_t s = (cudaStream_t)stream;
    const hap_status st = HAP_BY_TYPE(NT, LSE);
    if (st != HAP_OK) return st;
    return launch_next(loss_rows_kernel, ceil_div(rows, 8), 256, 0, 1, s, (const float2 *)p.part, pieces, (int)rows, (const float *)p.at_target, target, ignore, (int)V, loss, lse);
}

extern "C" hap_status hap_linear_cross_entropy_backward(int32_t dtype, int64_t rows, int32_t H, int64_t V, const void *x, int64_t ldx, const void *w,
                                                        int64_t ldw, const int64_t *target, int64_t ignore, const float *lse, const float *grad, void *dx,
                                                        int64_t lddx, void *dw, int64_t lddw, void *workspace, uint64_t bytes, void *stream)
{
    const hap_status bad = loss_args(dtype, rows, H, V, x, ldx, w, ldw, target, workspace, bytes);
    if (bad != HAP_OK) return bad;
    if (!grad || !aligned(grad, 4) || !aligned(dx, 2) || !aligned(dw, 2) || (dx && lddx < H) || (dw && lddw < H)) return HAP_E_INVALID;
    if (rows > 0 && (!lse || !aligned(lse, 4))) return HAP_E_INVALID;
    cudaStream_t s = (cudaStream_t)stream;
    const int64_t piece = piece_columns(rows, V), H8 = (H + 7) / 8 * 8;
    const LossSpace at = loss_space(rows, H, V);
    char *d = (char *)workspace, *x2 = d + at.x2;
    float *acc = (float *)(d + at.acc), *residual = (float *)(d + at.residual);
    const bool twice = rows <= TWICE_ROWS && rows > 0 && dw;
    Args of_dx{};                                           // dx's product, but for the piece
    of_dx.groups = 1, of_dx.rows = (int)rows, of_dx.ncols = H, of_dx.a = d, of_dx.lda = piece, of_dx.b = w, of_dx.ldb = ldw;
    // parts of its contraction, of the same length in every piece, so that none is empty and those of a later, shorter piece are
    // among the first one's (the plain kernel makes one sum; a piece begins at a multiple of 512 bytes of w, so all run as the first)
    const int64_t whole = V < piece ? V : piece, split_k = ceil_div(ceil_div(whole, on_tensor_cores(of_dx) ? parts_of_dx(rows, H, piece) : 1), BK) * BK;
    const int parts = (int)ceil_div(whole, split_k);
    if (twice)
        for (int i = 0; i < 2; i++)
            if (status_of(cudaMemcpy2DAsync(x2 + i * rows * H8 * 2, H8 * 2, x, ldx * 2, (size_t)H * 2, (size_t)rows, cudaMemcpyDeviceToDevice, s)) != HAP_OK) return HAP_E_CUDA;
    for (int64_t c0 = 0; c0 < V; c0 += piece) {
        const int64_t cols = V - c0 < piece ? V - c0 : piece;
        const char *wc = (const char *)w + c0 * ldw * 2;
        hap_status st = HAP_OK;
        if (rows > 0) {
            Args p{};
            p.groups = 1, p.rows = (int)rows, p.ncols = (int)cols, p.kdim = H;
            p.a = x, p.b = wc, p.lda = ldx, p.ldb = ldw;
            p.target = target, p.ignore = ignore, p.vocab = V, p.col0 = (int)c0, p.lse = lse;
            p.out = d, p.ldo = piece, p.residual = residual, p.low = twice ? rows * piece : 0;
            st = HAP_BY_TYPE(NT, DLOGIT);
        }
        if (st == HAP_OK && dx && rows > 0) {
            Args p = of_dx;
            p.kdim = (int)cols, p.b = wc;
            const bool last = c0 + cols == V;
            p.splits = (int)ceil_div(cols, split_k), p.split_k = (int)split_k;
            p.out = dx, p.ldo = lddx, p.acc32 = acc, p.first = c0 == 0, p.last = last && parts == 1;
            p.scale = grad, p.scale_by = 1.0f / DLOGIT_SCALE;
            p.target = target, p.ignore = ignore, p.vocab = V, p.residual = residual, p.w = w, p.ldw = ldw;
            st = HAP_BY_TYPE(NN, SUM32);
            if (st == HAP_OK && last && parts > 1) {
                p.splits = parts;
                const int64_t blocks = ceil_div(rows * H, 256);
                const int64_t grid = blocks < 8 * 148 ? blocks : 8 * 148;
                st = dtype == HAP_BF16 ? launch_next(join_parts_kernel<__nv_bfloat16>, grid, 256, 0, 1, s, p) : launch_next(join_parts_kernel<__half>, grid, 256, 0, 1, s, p);
            }
        }
        if (st == HAP_OK && dw) {
            Args p{};
            p.groups = 1, p.rows = (int)(twice ? 2 * rows : rows), p.mdim = (int)cols, p.ncols = H;
            p.a = d, p.b = twice ? x2 : x, p.lda = piece, p.ldb = twice ? H8 : ldx;
            p.out = (char *)dw + c0 * lddw * 2, p.ldo = lddw;
            p.scale = grad, p.scale_by = 1.0f / DLOGIT_SCALE;
            st = HAP_BY_TYPE(TN, STORE);
        }
        if (st != HAP_OK) return st;
    }
    return HAP_OK;
}

// ---- AdamW ------------------------------------------------------------------------------------------------------------
// Descriptors of one launch: a short list for the usual call on few tensors, whose arguments are copied faster, and one that
// fills most of the 32 KB that a launch may carry.
constexpr int FEW = 56, MANY = 440;

template <int N, typename F> static hap_status adamw_launches(const hap_adamw_tensor *tensors, int32_t n, float *const *m_out, float *const *v_out, F &&launch)
{
    AdamwList<N> list;
    uint64_t all = 0;
    for (int i = 0; i < n; i++) all += tensors[i].count;
    list.chunk = all < 4ull * 148 * ADAMW_CHUNK ? ADAMW_SHORT : ADAMW_CHUNK;
    for (int i = 0; i < n;) {
        list.n = 0;
        uint64_t chunks = 0;
        for (; i < n && list.n < N; i++) {
            const hap_adamw_tensor &t = tensors[i];
            if (!t.count) continue;
            const uint64_t c = (t.count + list.chunk - 1) / list.chunk;
            if (chunks + c > INT32_MAX) {
                if (!list.n) return HAP_E_RANGE;
                break;
            }
            list.t[list.n] = {m_out ? m_out[i] : t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, m_out || v_out ? (void *)(v_out ? v_out[i] : nullptr) : t.copy, t.count};
            if (!m_out && v_out) list.t[list.n].p = nullptr;
            list.first[list.n++] = (unsigned)chunks;
            chunks += c;
        }
        if (!list.n) break;
        const hap_status st = launch(list, (int64_t)chunks);
        if (st != HAP_OK) return st;
    }
    return HAP_OK;
}

template <typename P, typename G> static hap_status adamw_run(const hap_adamw_tensor *tensors, int32_t n, int bits, const AdamwFactors &f, const float *grad_scale, cudaStream_t s)
{
    auto launch = [&](auto &list, int64_t chunks) {
        constexpr int N = sizeof(list.t) / sizeof(AdamwTensor);
        return start(bits == 8 ? adamw8_kernel<P, G, N> : adamw_kernel<P, G, N>, shape_of(chunks, 256, 0, s), list, f, grad_scale);
    };
    return n <= FEW ? adamw_launches<FEW>(tensors, n, nullptr, nullptr, launch) : adamw_launches<MANY>(tensors, n, nullptr, nullptr, launch);
}

extern "C" hap_status hap_adamw_step(const hap_adamw_tensor *tensors, int32_t n, int32_t pt, int32_t gt, int32_t ct, int32_t bits,
                                     const hap_adamw_options *o, const float *grad_scale, void *stream)
{
    if (n < 0 || (n > 0 && !tensors) || !o || pt < HAP_BF16 || pt > HAP_FP32 || gt < HAP_BF16 || gt > HAP_FP32 || (bits != 32 && bits != 8)) return HAP_E_INVALID;
    if (gt != pt && gt != HAP_FP32 && pt != HAP_FP32) return HAP_E_INVALID;
    if (!(o->beta1 >= 0 && o->beta1 < 1 && o->beta2 >= 0 && o->beta2 < 1 && o->eps >= 0 && o->step >= 1) || !isfinite(o->lr) || !isfinite(o->weight_decay) || !isfinite(o->eps) || !aligned(grad_scale, 4)) return HAP_E_INVALID;
    for (int i = 0; i < n; i++) {
        const hap_adamw_tensor &t = tensors[i];
        if (!t.count) continue;
        if (t.count > (1ull << 42)) return HAP_E_RANGE;
        if (!t.param || !t.grad || !t.m || !t.v || !aligned(t.param, size_of(pt)) || !aligned(t.grad, size_of(gt))) return HAP_E_INVALID;
        if (bits == 32 ? !aligned(t.m, 4) || !aligned(t.v, 4) : !t.m_scale || !t.v_scale || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4)) return HAP_E_INVALID;
        if (t.copy && (!dtype16(ct) || pt != HAP_FP32 || !aligned(t.copy, 2))) return HAP_E_INVALID;
    }
    const double c1 = 1 - pow(o->beta1, (double)o->step), c2 = 1 - pow(o->beta2, (double)o->step);
    const AdamwFactors f = {(float)o->beta1, (float)o->beta2, (float)(1 - o->beta1), (float)(1 - o->beta2), (float)(1 - o->lr * o->weight_decay),
                            (float)(o->lr / c1), (float)(1 / sqrt(c2)), (float)o->eps, ct == HAP_FP16};
    cudaStream_t s = (cudaStream_t)stream;
    if (pt == HAP_BF16) return gt == HAP_FP32 ? adamw_run<__nv_bfloat16, float>(tensors, n, bits, f, grad_scale, s) : adamw_run<__nv_bfloat16, __nv_bfloat16>(tensors, n, bits, f, grad_scale, s);
    if (pt == HAP_FP16) return gt == HAP_FP32 ? adamw_run<__half, float>(tensors, n, bits, f, grad_scale, s) : adamw_run<__half, __half>(tensors, n, bits, f, grad_scale, s);
    return gt == HAP_FP32 ? adamw_run<float, float>(tensors, n, bits, f, grad_scale, s)
         : gt == HAP_BF16 ? adamw_run<float, __nv_bfloat16>(tensors, n, bits, f, grad_scale, s) : adamw_run<float, __half>(tensors, n, bits, f, grad_scale, s);
}

extern "C" hap_status hap_adamw_state(const hap_adamw_tensor *tensors, int32_t n, float *const *host_m, float *const *host_v, void *stream)
{
    if (n < 0 || (n > 0 && !tensors)) return HAP_E_INVALID;
    if (!host_m && !host_v) return HAP_OK;
    for (int i = 0; i < n; i++) {
        const hap_adamw_tensor &t = tensors[i];
        if (!t.count) continue;
        if (t.count > (1ull << 42)) return HAP_E_RANGE;
        if (!t.m || !t.v || !t.m_scale || !t.v_scale || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4)) return HAP_E_INVALID;
        if ((host_m && !aligned(host_m[i], 4)) || (host_v && !aligned(host_v[i], 4))) return HAP_E_INVALID;
    }
    cudaStream_t s = (cudaStream_t)stream;
    auto launch = [&](auto &list, int64_t chunks) {
        constexpr int N = sizeof(list.t) / sizeof(AdamwTensor);
        return start(adamw_values_kernel<N>, shape_of(chunks, 256, 0, s), list);
    };
    return n <= FEW ? adamw_launches<FEW>(tensors, n, host_m, host_v, launch) : adamw_launches<MANY>(tensors, n, host_m, host_v, launch);
}

extern "C" hap_status hap_operator_status(uint32_t *host_bits)
{
    if (!host_bits) return HAP_E_INVALID;
    *host_bits = 0;
    const unsigned zero = 0;
    if (status_of(cudaDeviceSynchronize()) != HAP_OK || status_of(cudaMemcpyFromSymbol(host_bits, operator_error, sizeof zero)) != HAP_OK) return HAP_E_CUDA;
    return status_of(cudaMemcpyToSymbol(operator_error, &zero, sizeof zero));
}

#ifdef HAP_CHECKED
// Self-checking build: the operators' bounded wait on a barrier that nothing arrives at, for `limit` ns (a second at most), by one warp.
__global__ void wait_check_kernel(uint64_t limit)
{
    __shared__ uint64_t bar;
    __shared__ int stop;
    if (threadIdx.x == 0) {
        bar_init(&bar, 1);
        stop = 0;
    }
    __syncthreads();
    bar_wait_long(smem_u32(&bar), 0, &stop, limit);
}
extern "C" hap_status hap_operator_wait_check(uint64_t limit, void *stream)
{
    if (limit > 1000000000ull) return HAP_E_INVALID;
    return start(wait_check_kernel, shape_of(1, 32, 0, (cudaStream_t)stream), limit);
}
#endif
