// Grouped products on the tensor cores: tcgen05.mma with operands that TMA brings into shared memory and sums in tensor
// memory.  A persistent kernel: a block (or a pair of blocks, which then share one product of 256 x 256) takes tile after tile.
//   warp 0   brings stages of 64 along the contraction, as far ahead as there are stages
//   warp 1   issues the products (in a pair the first block's does for both)
//   others   take finished sums out of tensor memory (lane = row) through the epilogue, while the next tile is summed: two
//            sets of 256 columns
// Operands along the contraction (K-major) lie as rows of 128 bytes, those across it (MN-major) as strips of 64 columns with
// a row per step of the contraction; both under the 128-byte swizzle that the descriptors name.
// Ragged ends: rows of other groups in a tile of NT, NN give rows of sums that are not stored; columns and steps outside of a
// matrix arrive as zeros.  In TN the steps are rows, and those behind a group's last are another group's: such a stage is
// written by the producer warp itself, zeros behind the last row (both operands: 0 times what lies there could be NaN).
#pragma once
#include <cuda.h>
#include "hap_products.cuh"

namespace hapop {

constexpr int BK = 64;

template <int CG> struct Shape {
    static constexpr int BM = 128 * CG;                 // rows of a tile
    static constexpr int BROWS = TILE_N / CG;           // columns of a tile that a block holds
    static constexpr int A_BYTES = 128 * BK * 2, B_BYTES = BROWS * BK * 2, STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = CG == 1 ? 4 : 6;
};

template <int CG> struct Shared {
    Schedule<Shape<CG>::BM> sched;
    uint64_t full[8], empty[8], acc_full[2], acc_empty[2];
    uint32_t tmem;
    int stop;
};

__device__ unsigned operator_error;

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// address of the same place in the first block of the pair
__device__ __forceinline__ uint32_t of_leader(uint32_t a) { uint32_t r; asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(a)); return r; }
__device__ __forceinline__ void bar_init(uint64_t *b, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_arrive_at(uint32_t cluster_addr) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory"); }
__device__ __forceinline__ void bar_expect_at(uint32_t cluster_addr, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.release.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(cluster_addr), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t a, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(a), "r"(parity) : "memory");
    return ok;
}
__device__ __forceinline__ uint64_t nanoseconds() { uint64_t t; asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t)); return t; }

// Waits for a phase, ten seconds at most (the longest tile, 2^30 rows of contraction, takes about five).  False: it ran out,
// here or in another warp of the block; the kernel then ends early and the device word says so.
__device__ __noinline__ bool bar_wait_long(uint32_t a, uint32_t parity, volatile int *stop, uint64_t limit)
{
    const uint64_t from = nanoseconds();
    for (unsigned i = 0;; i++) {
        if (bar_try(a, parity)) return true;
        if ((i & 63) == 63) {
            if (*stop) return false;
            if (nanoseconds() - from > limit) break;
        }
    }
    *stop = 1;
    atomicOr(&operator_error, 1u);
    return false;
}
__device__ __forceinline__ bool bar_wait(uint64_t *b, uint32_t parity, volatile int *stop)
{
    const uint32_t a = smem_u32(b);
    for (int i = 0; i < 16; i++)
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
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

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
                                     (uint32_t)(TILE_N / 8) << 17 | (uint32_t)(Shape<CG>::BM / 16) << 24;
};

// One stage of an operand whose contraction runs over rows, written by the warp: rows first .. of `src` (row distance ld) as far
// as `valid`, zeros behind, columns col0 .. as far as `cols`, in strips of 64 columns under the swizzle.
template <typename T> __device__ void write_strips(char *dst, int strips, const T *src, int64_t ld, int64_t first, int valid, int col0, int cols, int lane)
{
    for (int s = 0; s < strips; s++) {
        const int c = col0 + s * 64 + (lane & 7) * 8;
#pragma unroll 4
        for (int r0 = 0; r0 < BK; r0 += 4) {
            const int r = r0 + (lane >> 3);
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < valid && c < cols) {
                const T *q = src + (first + r) * ld + c;
                v = *(const uint4 *)q;                  // (row distances are multiples of 8: the 16 bytes are within the row's distance)
                if (c + 8 > cols) {
                    uint32_t *w = (uint32_t *)&v;
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        if (c + i >= cols) w[i / 2] &= i % 2 ? 0x0000ffffu : 0xffff0000u;
                }
            }
            *(uint4 *)(dst + s * BK * 128 + r * 128 + (((lane & 7) ^ (r & 7)) << 4)) = v;
        }
    }
}

template <typename T, int FORM, int EPI, int CG>
__global__ void __launch_bounds__(192, 1) product_kernel(const __grid_constant__ Args p, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b)
{
    using S = Shape<CG>;
    extern __shared__ char raw[];
    char *stages = (char *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    Shared<CG> &sh = *(Shared<CG> *)(stages + S::STAGES * S::STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 1 ? 0 : cluster_rank();
    constexpr int BN = EPI == GATED ? TILE_N / 2 : TILE_N;
    const int col_tiles = (p.ncols + BN - 1) / BN;

    if (warp == 0) sh.sched.build(p, FORM, col_tiles, lane);
    if (warp == 1) {
        if (lane == 0) {
            for (int i = 0; i < S::STAGES; i++) bar_init(&sh.full[i], CG), bar_init(&sh.empty[i], 1);
            for (int i = 0; i < 2; i++) bar_init(&sh.acc_full[i], 1), bar_init(&sh.acc_empty[i], 4 * CG);
            sh.stop = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async;" ::: "memory");
        }
        __syncwarp();
        if constexpr (CG == 1)
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\ntcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::"r"(smem_u32(&sh.tmem)) : "memory");
        else
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;\ntcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::"r"(smem_u32(&sh.tmem)) : "memory");
    }
    fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();
    fence_after();
    const uint32_t tmem = *(volatile uint32_t *)&sh.tmem;
    volatile int *stop = &sh.stop;
    const int total = sh.sched.total(p, FORM, col_tiles);
    const int step = gridDim.x / CG, begin = blockIdx.x / CG;

    if (warp == 0) {
        uint32_t at = 0;                                    // stages brought so far
        bool good = true;
        for (int t = begin; t < total && good; t += step) {
            const auto tile = sh.sched.tile(p, FORM, col_tiles, t);
            const int m0 = tile.m * S::BM + rank * 128, n0 = tile.n * BN;
            const int K = FORM == TN ? tile.hi - tile.lo : p.kdim;
            for (int k = 0; k < K; k += BK, at++) {
                const int s = at % S::STAGES;
                if (!(good = bar_wait(&sh.empty[s], (at / S::STAGES + 1) & 1, stop))) break;
                char *a = stages + s * S::STAGE, *b = a + S::A_BYTES;
                const uint32_t full = CG == 1 ? smem_u32(&sh.full[s]) : of_leader(smem_u32(&sh.full[s]));
                if (FORM == TN && K - k < BK) {             // the group ends in this stage
                    write_strips((char *)a, 2, (const T *)p.a, p.lda, (int64_t)tile.lo + k, K - k, m0, p.mdim, lane);
                    write_strips((char *)b, S::BROWS / 64, (const T *)p.b, p.ldb, (int64_t)tile.lo + k, K - k, n0 + (int)rank * S::BROWS, p.ncols, lane);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) bar_arrive_at(full);
                } else if (lane == 0) {
                    bar_expect_at(full, S::STAGE);
                    const uint32_t da = smem_u32(a), db = smem_u32(b);
                    if (FORM == TN) {
#pragma unroll
                        for (int i = 0; i < 2; i++) tma_load<CG>(&map_a, da + i * BK * 128, full, m0 + 64 * i, tile.lo + k, 0);
                    } else {
                        tma_load<CG>(&map_a, da, full, k, tile.lo + m0, 0);
                    }
                    if (FORM == NT) {                       // boxes of 128 rows of w
#pragma unroll
                        for (int i = 0; i < S::BROWS / 128; i++) {
                            const int half = rank * (S::BROWS / 128) + i;
                            tma_load<CG>(&map_b, db + i * 128 * 128, full, k, EPI == GATED ? n0 + half * p.ncols : n0 + half * 128, tile.e);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < S::BROWS / 64; i++)
                            tma_load<CG>(&map_b, db + i * BK * 128, full, n0 + (int)rank * S::BROWS + 64 * i, FORM == TN ? tile.lo + k : k, FORM == TN ? 0 : tile.e);
                    }
                }
                __syncwarp();
            }
        }
        if (*stop && rank == 0)                             // cut short: nothing of ours may still be on its way
            for (uint32_t i = at > S::STAGES ? at - S::STAGES : 0; i < at; i++) {
                const uint64_t from = nanoseconds();
                while (!bar_try(smem_u32(&sh.full[i % S::STAGES]), (i / S::STAGES) & 1) && nanoseconds() - from < 100000000ull) {}
            }
    } else if (warp == 1) {
        if (rank == 0) {
            constexpr uint32_t idesc = Instruction<T, FORM, CG>::bits;
            uint32_t at = 0, tiles = 0;
            bool good = true;
            for (int t = begin; t < total && good; t += step) {
                int K = p.kdim;
                if (FORM == TN) {
                    const auto tile = sh.sched.tile(p, FORM, col_tiles, t);
                    K = tile.hi - tile.lo;
                    if (!K) continue;                       // nothing to sum: the epilogue writes zeros by itself
                }
                const int set = tiles & 1;
                if (!(good = bar_wait(&sh.acc_empty[set], (tiles / 2 + 1) & 1, stop))) break;
                tiles++;
                fence_after();
                for (int k = 0; k < K; k += BK, at++) {
                    const int s = at % S::STAGES;
                    if (!(good = bar_wait(&sh.full[s], (at / S::STAGES) & 1, stop))) break;
                    fence_after();
                    if (lane == 0) {
                        const uint32_t a = smem_u32(stages + s * S::STAGE), b = a + S::A_BYTES;
#pragma unroll
                        for (int i = 0; i < BK / 16; i++) {
                            // 16 steps of the contraction: 32 bytes along K-major rows, 16 rows of MN-major strips
                            const uint64_t da = FORM == TN ? smem_desc(a + i * 2048, BK * 128, 1024) : smem_desc(a + i * 32, 16, 1024);
                            const uint64_t db = FORM != NT ? smem_desc(b + i * 2048, BK * 128, 1024) : smem_desc(b + i * 32, 16, 1024);
                            mma<CG>(tmem + set * TILE_N, da, db, idesc, k > 0 || i > 0);
                        }
                        mma_commit<CG>(&sh.empty[s]);
                        if (k + BK >= K) mma_commit<CG>(&sh.acc_full[set]);
                    }
                    __syncwarp();
                }
            }
        }
    } else {
        uint32_t tiles = 0;
        const int quarter = warp & 3;                       // the rows of tensor memory that this warp may read
        for (int t = begin; t < total; t += step) {
            const auto tile = sh.sched.tile(p, FORM, col_tiles, t);
            const int r = tile.m * S::BM + rank * 128 + quarter * 32 + lane, n0 = tile.n * BN;
            const bool live = r < (FORM == TN ? p.mdim : tile.hi - tile.lo), some = FORM != TN || tile.hi > tile.lo;
            const int set = tiles & 1;
            if (some) {
                if (!bar_wait(&sh.acc_full[set], (tiles / 2) & 1, stop)) break;
                tiles++;
                fence_after();
            } else if (p.accumulate) {
                continue;
            }
            RowEpilogue<T, EPI> row(p, (FORM == TN ? 0 : (int64_t)tile.lo) + r, FORM == TN ? tile.e : 0, live);
            const uint32_t from = tmem + set * TILE_N + ((uint32_t)quarter << 21);
            for (int q = 0; q < BN / 32 && n0 + q * 32 < p.ncols; q++) {
                float v[32], v2[32];
                if (some) {
                    __syncwarp();
                    tmem_load32(from + q * 32, v);
                    if (EPI == GATED) tmem_load32(from + BN + q * 32, v2);
                    tmem_load_wait();
                } else {
#pragma unroll
                    for (int i = 0; i < 32; i++) v[i] = v2[i] = 0.0f;
                }
                if (live) row.columns(n0 + q * 32, v, v2);
            }
            if (live) row.end(tile.n);
            if (some) {
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_at(CG == 1 ? smem_u32(&sh.acc_empty[set]) : of_leader(smem_u32(&sh.acc_empty[set])));
            }
        }
    }
    fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();                  // the other block's copies and arrivals come to this one's memory
    fence_after();
    if (warp == 1) {
        if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

} // namespace hapop
