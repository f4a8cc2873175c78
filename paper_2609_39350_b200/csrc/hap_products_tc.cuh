// Grouped products on the tensor cores: tcgen05.mma with operands that TMA brings into shared memory and sums in tensor
// memory.  A persistent kernel: a block (or a pair of blocks, which then share one product of 256 x 256) takes tile after tile.
//   warp 0   brings stages of 64 along the contraction, as far ahead as there are stages
//   warp 1   issues the products (in a pair the first block's does for both)
//   others   take finished sums out of tensor memory (lane = row) through the epilogue, while the next are made: two sets of
//            256 columns
// Operands along the contraction (K-major) lie as rows of 128 bytes, those across it (MN-major) as strips of 64 columns with
// a row per step of the contraction; both under the 128-byte swizzle that the descriptors name.
// Ragged ends: rows of other groups in a tile of NT, NN give rows of sums that are not stored; columns and steps outside of a
// matrix arrive as zeros.  In TN the steps are rows, and those behind a group's last are another group's: a warp of its own
// overwrites them with zeros (in both operands: 0 times what lies there could be NaN) before the stage is handed on.  (8 weight
// gradients of 4096 x 14336, 8192 rows: 2403 us with such stages loaded by the producer's threads, 1373 where the producer
// cleared them, 1266 with the warp.)
#pragma once
#include <cuda.h>
#include "hap_products.cuh"

namespace hapop {

constexpr int BK = 64;

template <int EPI, int CG> struct Shape {
    static constexpr int BM = 128 * CG;                 // rows of a tile
    static constexpr int BROWS = TILE_N / CG;           // columns of a tile that a block holds
    static constexpr int A_BYTES = 128 * BK * 2, B_BYTES = BROWS * BK * 2, STAGE = A_BYTES + B_BYTES;
    // outputs leave through shared memory, for each warp 32 rows of 64 bytes, or of 128 where they are fp32
    static constexpr int OUT = EPI == STORE32 ? 4096 : 2048;
    static constexpr int STAGES = CG == 1 ? (EPI == STORE32 ? 3 : 4) : (EPI == STORE32 ? 5 : 6);
    // Tensor cores add to a sum by truncating: after n products of 16 steps it is short by about n 2^-25 of its magnitude (at
    // 3500 rows 2.4e-6, six times the error of sums rounded to nearest; 7.7e-7 this way).  Results that are kept in fp32 are summed over
    // 1024 steps there, and these sums in registers, under the next products.  The logits of the loss's two passes have to be the
    // same sums: what they are off by leaves in z - lse, and p - 1 of a row whose target leads is small (logits of 25 over 8192
    // steps, one long sum in the backward pass: 9e-4 times the target's row in dx where 1e-8 is right).
    static constexpr bool SUMS = EPI == STORE32 || EPI == LSE || EPI == DLOGIT;
    static constexpr int SUM_STEPS = 1024;
};

template <int EPI, int CG> struct Shared {
    Schedule<Shape<EPI, CG>::BM> sched;
    uint64_t full[8], empty[8], acc_full[2], acc_empty[2], end[8];
    uint32_t tmem;
    int stop;
};

__device__ unsigned operator_error;

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
// One lane of a converged warp.  Unlike a test of the lane number it tells the compiler that a single thread follows, so that
// the operands of TMA and tcgen05 go to uniform registers directly (8192 x 8192 x 8192: 1451 -> 1593 TFLOP/s).
__device__ __forceinline__ bool elected()
{
    uint32_t p;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(p));
    return p;
}
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// address of the same place in the first block of the pair
__device__ __forceinline__ uint32_t of_leader(uint32_t a) { uint32_t r; asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(a)); return r; }
__device__ __forceinline__ void bar_init(uint64_t *b, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(n) : "memory"); }
// Arrivals and waits carry the block's scope only, but where data written by threads goes with them: a fence for the cluster on
// every stage made the producer the slowest of all (8192 x 8192 x 8192: 731 TFLOP/s with it, 1451 without).
template <int CG> __device__ __forceinline__ void bar_expect_at(uint32_t addr, uint32_t bytes)
{
    if constexpr (CG == 1) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(addr), "r"(bytes) : "memory");
    else asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(addr), "r"(bytes) : "memory");
}
template <int CG> __device__ __forceinline__ void bar_arrive_at(uint32_t addr)
{
    if constexpr (CG == 1) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(addr) : "memory");
    else asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
__device__ __forceinline__ void bar_arrive_with_data_at(uint32_t addr) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory"); }
__device__ __forceinline__ bool bar_try(uint32_t a, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(a), "r"(parity), "r"(1000000) : "memory");
    return ok;
}
__device__ __forceinline__ void acquire_cluster() { asm volatile("fence.acq_rel.cluster;" ::: "memory"); }
__device__ __forceinline__ uint64_t nanoseconds() { uint64_t t; asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t)); return t; }

// A try suspends the warp for up to a millisecond: ten warps that ask all the time take issue slots and power (1530 -> 1642 TFLOP/s).
// Waits for a phase, ten seconds at most (the longest tile, 2^30 rows of contraction, takes about five).  False: it ran out,
// here or in another warp of the block; the kernel then ends early and the device word says so.
__device__ __noinline__ bool bar_wait_long(uint32_t a, uint32_t parity, volatile int *stop, uint64_t limit)
{
    const uint64_t from = nanoseconds();
    for (unsigned i = 0;; i++) {
        if (bar_try(a, parity)) return true;
        if (*stop) return false;
        if (nanoseconds() - from > limit) break;
    }
    *stop = 1;
    atomicOr(&operator_error, 1u);
    return false;
}
__device__ __forceinline__ bool bar_wait(uint64_t *b, uint32_t parity, volatile int *stop)
{
    const uint32_t a = smem_u32(b);
    for (int i = 0; i < 4; i++)
        if (bar_try(a, parity)) return true;
    return bar_wait_long(a, parity, stop, 10000000000ull);
}

template <int CG> __device__ __forceinline__ void tma_load(const CUtensorMap *map, uint32_t dst, uint32_t bar, int x, int y, int z)
{
    if constexpr (CG == 1)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
template <int CG> __device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    if constexpr (CG == 1)
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((int)add) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((int)add) : "memory");
}
// the products issued so far arrive at the barrier, in a pair at that of both blocks
template <int CG> __device__ __forceinline__ void mma_commit(uint64_t *bar)
{
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32])
{
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, "
                 "%23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
                   "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
#pragma unroll
    for (int i = 0; i < 32; i++) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_load8(uint32_t addr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr));
}
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[32]) { tmem_load32(addr, v); }
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[16])
{
    uint32_t r[16];
    tmem_load16(addr, r);
#pragma unroll
    for (int i = 0; i < 16; i++) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// all 512 columns of tensor memory, by a whole warp (in a pair by one of each block)
template <int CG> __device__ __forceinline__ void tmem_alloc(uint32_t *at)
{
    if constexpr (CG == 1)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\ntcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::"r"(smem_u32(at)) : "memory");
    else
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;\ntcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::"r"(smem_u32(at)) : "memory");
}
template <int CG> __device__ __forceinline__ void tmem_free(uint32_t tmem)
{
    if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}
// cut short: waits, a tenth of a second each at most, for the stages that are still on their way
__device__ __noinline__ void drain(uint64_t *full, uint32_t at, uint32_t stages)
{
    for (uint32_t i = at > stages ? at - stages : 0; i < at; i++) {
        const uint64_t from = nanoseconds();
        while (!bar_try(smem_u32(&full[i % stages]), (i / stages) & 1) && nanoseconds() - from < 100000000ull) {}
    }
}

// The products of a pair arrive at the barriers of both blocks: one whose last stages' arrivals are still on their way must not
// leave its memory.  (What the epilogue waits for comes behind them, but by another barrier.)
template <int STAGES> __device__ __forceinline__ void wait_for_empty(uint64_t *empty, uint32_t at, volatile int *stop)
{
    for (uint32_t i = at; i < at + STAGES; i++)
        if (!bar_wait(&empty[i % STAGES], (i / STAGES + 1) & 1, stop)) break;
}

// Shared-memory descriptor under the 128-byte swizzle; lead, stride: bytes between the 1024-byte pieces of 8 rows (K-major: stride
// along the rows, lead unused; MN-major: stride along the contraction, lead between strips of 64 columns).
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead, uint32_t stride)
{
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
template <typename T> struct TypeBits { static constexpr uint32_t value = 0; };
template <> struct TypeBits<__nv_bfloat16> { static constexpr uint32_t value = 1; };
// instruction descriptor: sums in fp32, operand types, which operands are MN-major, sizes
template <typename T, int FORM, int CG> struct Instruction {
    static constexpr uint32_t bits = 1u << 4 | TypeBits<T>::value << 7 | TypeBits<T>::value << 10 | (FORM == TN ? 1u << 15 : 0) | (FORM != NT ? 1u << 16 : 0) |
                                     (uint32_t)(TILE_N / 8) << 17 | (uint32_t)(128 * CG / 16) << 24;
};

// Rows valid .. 63 of a stage's strips become zeros, by a warp.
__device__ __forceinline__ void clear_rows(char *strips, int n, int valid, int lane)
{
    for (int s = 0; s < n; s++)
        for (int r = valid + (lane >> 3); r < BK; r += 4) *(uint4 *)(strips + s * BK * 128 + r * 128 + (lane & 7) * 16) = make_uint4(0, 0, 0, 0);
}

template <typename T, int FORM, int EPI, int CG>
__global__ void __launch_bounds__(FORM == TN ? 352 : 320, 1) product_kernel(const __grid_constant__ Args p, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                         const __grid_constant__ CUtensorMap map_out)
{
    using S = Shape<EPI, CG>;
    extern __shared__ char raw[];
    char *stages = (char *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    char *outs = stages + S::STAGES * S::STAGE;
    Shared<EPI, CG> &sh = *(Shared<EPI, CG> *)(outs + 8 * S::OUT);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 1 ? 0 : cluster_rank();
    constexpr int BN = TILE_N;
    // the parts of a split contraction are so many more columns of tiles
    const int part_tiles = (p.ncols + BN - 1) / BN, col_tiles = EPI == SUM32 ? part_tiles * p.splits : part_tiles;

    launch_next();
    if (threadIdx.x == 0) prefetch_map(&map_a), prefetch_map(&map_b);
    if (warp == 1) {
        if (lane == 0) {
            for (int i = 0; i < S::STAGES; i++) bar_init(&sh.full[i], CG), bar_init(&sh.empty[i], 1);
            for (int i = 0; i < 2; i++) bar_init(&sh.acc_full[i], 1), bar_init(&sh.acc_empty[i], 8 * CG);
            for (int i = 0; i < S::STAGES; i++) bar_init(&sh.end[i], 1);
            sh.stop = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async;" ::: "memory");
        }
        __syncwarp();
        tmem_alloc<CG>(&sh.tmem);
    }
    wait_for_last();
    sh.sched.fetch(p);
    __syncthreads();
    if (warp == 0) sh.sched.build(p, col_tiles, lane);
    fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();
    fence_after();
    const uint32_t tmem = *(volatile uint32_t *)&sh.tmem;
    volatile int *stop = &sh.stop;
    const int total = sh.sched.total(p, FORM, col_tiles), step = gridDim.x / CG, begin = blockIdx.x / CG;

    if (warp == 0) {
        uint32_t at = 0;                                    // stages brought so far
        bool good = true;
        for (int t = begin; t < total && good; t += step) {
            const auto tile = sh.sched.tile(p, FORM, col_tiles, t);
            const int part = EPI == SUM32 ? tile.n / part_tiles : 0;
            const int m0 = tile.m * S::BM + rank * 128, n0 = (tile.n - part * part_tiles) * BN;
            const int K = FORM == TN ? tile.hi - tile.lo : EPI == SUM32 ? min(p.kdim, (part + 1) * p.split_k) : p.kdim;
            for (int k = EPI == SUM32 ? part * p.split_k : 0; k < K && good; k += BK, at++) {
                const int s = at % S::STAGES;
                if (!(good = bar_wait(&sh.empty[s], (at / S::STAGES + 1) & 1, stop))) break;
                const bool ends_here = FORM == TN && K - k < BK && tile.hi < p.rows;     // (behind the last row of all zeros arrive)
                char *a = stages + s * S::STAGE, *b = a + S::A_BYTES;
                const uint32_t full = ends_here ? smem_u32(&sh.end[s]) : CG == 1 ? smem_u32(&sh.full[s]) : of_leader(smem_u32(&sh.full[s]));
                if (elected()) {
                    bar_expect_at<CG>(full, S::STAGE);
                    const uint32_t da = smem_u32(a), db = smem_u32(b);
                    if (FORM == TN) {
#pragma unroll
                        for (int i = 0; i < 2; i++) tma_load<CG>(&map_a, da + i * BK * 128, full, m0 + 64 * i, tile.lo + k, 0);
                    } else {
                        tma_load<CG>(&map_a, da, full, k, tile.lo + m0, 0);
                    }
                    if (FORM == NT) {                       // boxes of 128 rows of w
#pragma unroll
                        for (int i = 0; i < S::BROWS / 128; i++) tma_load<CG>(&map_b, db + i * 128 * 128, full, k, n0 + ((int)rank * (S::BROWS / 128) + i) * 128, tile.e);
                    } else {
#pragma unroll
                        for (int i = 0; i < S::BROWS / 64; i++)
                            tma_load<CG>(&map_b, db + i * BK * 128, full, n0 + (int)rank * S::BROWS + 64 * i, FORM == TN ? tile.lo + k : k, FORM == TN ? 0 : tile.e);
                    }
                }
                __syncwarp();
            }
        }
        if (CG == 2 && good) wait_for_empty<S::STAGES>(sh.empty, at, stop);
        if (*stop && rank == 0) drain(sh.full, at, S::STAGES);
    } else if (warp == 1) {
        if (rank == 0) {
            constexpr uint32_t idesc = Instruction<T, FORM, CG>::bits;
            uint32_t at = 0, sums = 0;
            bool good = true;
            for (int t = begin; t < total && good; t += step) {
                int K = p.kdim;
                if (EPI == SUM32) {
                    const int part = sh.sched.tile(p, FORM, col_tiles, t).n / part_tiles;
                    K = min(p.kdim - part * p.split_k, p.split_k);
                }
                if (FORM == TN) {
                    const auto tile = sh.sched.tile(p, FORM, col_tiles, t);
                    K = tile.hi - tile.lo;
                    if (!K) continue;                       // nothing to sum: the epilogue writes zeros by itself
                }
                for (int k0 = 0; k0 < K && good; k0 += S::SUMS ? S::SUM_STEPS : K) {
                    const int end = S::SUMS ? min(K, k0 + S::SUM_STEPS) : K, set = sums & 1;
                    if (!(good = bar_wait(&sh.acc_empty[set], (sums / 2 + 1) & 1, stop))) break;
                    sums++;
                    fence_after();
                    for (int k = k0; k < end; k += BK, at++) {
                        const int s = at % S::STAGES;
                        if (!(good = bar_wait(&sh.full[s], (at / S::STAGES) & 1, stop))) break;
                        if (CG == 2 && FORM == TN && K - k < BK) acquire_cluster();      // (rows cleared by threads)
                        fence_after();
                        if (elected()) {
                            const uint32_t a = smem_u32(stages + s * S::STAGE), b = a + S::A_BYTES;
                            const uint64_t da = FORM == TN ? smem_desc(a, BK * 128, 1024) : smem_desc(a, 16, 1024);
                            const uint64_t db = FORM != NT ? smem_desc(b, BK * 128, 1024) : smem_desc(b, 16, 1024);
#pragma unroll
                            for (int i = 0; i < BK / 16; i++)   // 16 steps of the contraction: 32 bytes along K-major rows, 16 rows of MN-major strips
                                mma<CG>(tmem + set * TILE_N, da + i * (FORM == TN ? 128 : 2), db + i * (FORM != NT ? 128 : 2), idesc, k > k0 || i > 0);
                            mma_commit<CG>(&sh.empty[s]);
                            if (k + BK >= end) mma_commit<CG>(&sh.acc_full[set]);
                        }
                        __syncwarp();
                    }
                }
            }
        }
    } else if (FORM == TN && warp == 10) {
        uint32_t at = 0, phases = 0;
        for (int t = begin; t < total; t += step) {
            const auto tile = sh.sched.tile(p, FORM, col_tiles, t);
            const int K = tile.hi - tile.lo, rest = K % BK;
            at += (K + BK - 1) / BK;
            if (!rest || tile.hi >= p.rows) continue;
            const int s = (at - 1) % S::STAGES;
            if (!bar_wait(&sh.end[s], phases >> s & 1, stop)) break;
            phases ^= 1u << s;
            clear_rows(stages + s * S::STAGE, 2 + S::BROWS / 64, rest, lane);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            const uint32_t full = smem_u32(&sh.full[s]);
            if (lane == 0) bar_arrive_with_data_at(CG == 1 ? full : of_leader(full));
        }
    } else {
        uint32_t sums = 0;
        // two warps for each quarter of tensor memory's rows (those that a warp may read), with half of the tile's columns each
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        constexpr int CHUNKS = BN / 64;                     // pieces of 32 columns that a warp has
        char *staged = outs + (warp - 2) * S::OUT;
        const uint32_t from = tmem + ((uint32_t)quarter << 21) + half * CHUNKS * 32;
        for (int t = begin; t < total; t += step) {
            const auto tile = sh.sched.tile(p, FORM, col_tiles, t);
            const int part = EPI == SUM32 ? tile.n / part_tiles : 0;
            const int m = tile.m * S::BM + rank * 128 + quarter * 32, n0 = (tile.n - part * part_tiles) * BN + half * CHUNKS * 32;
            const int K = FORM == TN ? tile.hi - tile.lo : p.kdim;
            if (FORM == TN && !K && p.accumulate) continue;
            const int live = (FORM == TN ? p.mdim : tile.hi - tile.lo) - m;
            RowEpilogue<T, EPI> row(p, WarpRows{staged, lane, min(max(live, 0), 32)}, (FORM == TN ? 0 : (int64_t)tile.lo) + m, FORM == TN ? tile.e : part);
            // the set's sums are out of tensor memory: the next may be summed there
            auto taken = [&](int set) {
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_at<CG>(CG == 1 ? smem_u32(&sh.acc_empty[set]) : of_leader(smem_u32(&sh.acc_empty[set])));
            };
            if constexpr (S::SUMS) {
                float acc[CHUNKS][32];
#pragma unroll
                for (int q = 0; q < CHUNKS; q++)
#pragma unroll
                    for (int i = 0; i < 32; i++) acc[q][i] = 0.0f;
                bool good = true;
                for (int k = 0; k < K; k += S::SUM_STEPS) {
                    const int set = sums & 1;
                    if (!(good = bar_wait(&sh.acc_full[set], (sums / 2) & 1, stop))) break;
                    sums++;
                    fence_after();
#pragma unroll
                    for (int q = 0; q < 4 * CHUNKS; q++) {  // eight at a time: the sums fill the registers
                        uint32_t v[8];
                        __syncwarp();
                        tmem_load8(from + set * TILE_N + q * 8, v);
                        tmem_load_wait();
#pragma unroll
                        for (int i = 0; i < 8; i++) acc[q / 4][q % 4 * 8 + i] += __uint_as_float(v[i]);
                    }
                    taken(set);
                }
                if (!good) break;
                if (EPI == STORE32 && FORM == TN && p.out_mapped) {
                    // through shared memory (rows of 128 bytes, swizzled as the map says), so that whole lines are written; an
                    // addition is made in L2, without reading: 1584 -> 1209 us at 8 x 4096 x 14336 with 8192 rows.  (Boxes
                    // that are loaded, added to and stored took 983 against 1078 of this at even loads and 1446 against 1373 at uneven ones.)
#pragma unroll
                    for (int q = 0; q < CHUNKS; q++) {
                        const int col = n0 + q * 32;
                        if (m >= p.mdim || col >= p.ncols) continue;
                        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");      // (by the lane that stored; others have nothing to wait for)
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 8; i++)
                            *(float4 *)(staged + lane * 128 + ((i ^ (lane & 7)) << 4)) = make_float4(acc[q][4 * i], acc[q][4 * i + 1], acc[q][4 * i + 2], acc[q][4 * i + 3]);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) {
                            if (p.accumulate)
                                asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(&map_out), "r"(smem_u32(staged)), "r"(col), "r"(m), "r"(tile.e) : "memory");
                            else
                                asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(&map_out), "r"(smem_u32(staged)), "r"(col), "r"(m), "r"(tile.e) : "memory");
                            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                        }
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < CHUNKS; q++) {
                        float v2[32];
                        row.columns(n0 + q * 32, acc[q], v2);
                    }
                    row.end(n0);
                }
            } else {
                const int set = sums & 1, chunks = min(CHUNKS, (p.ncols - n0 + 31) / 32);
                if (K) {
                    if (!bar_wait(&sh.acc_full[set], (sums / 2) & 1, stop)) break;
                    sums++;
                    fence_after();
                    if (chunks <= 0) taken(set);
                }
                for (int q = 0; q < chunks; q++) {
                    float v[32], v2[32];
                    if (K) {
                        __syncwarp();
                        tmem_load32(from + set * TILE_N + q * 32, v);
                        tmem_load_wait();
                        if (q == chunks - 1) taken(set);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; i++) v[i] = 0.0f;
                    }
                    row.columns(n0 + q * 32, v, v2);
                }
            }
        }
        if (EPI == STORE32) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();                  // the other block's copies and arrivals come to this one's memory
    fence_after();
    if (warp == 1) tmem_free<CG>(tmem);
}

} // namespace hapop
