// Products of the experts' rows on the tensor cores, turned around: the weight's columns are the 256 rows of a product (128 for
// each block of a pair) and the expert's rows its columns, 32 to 256 of them in steps of 32.  So an expert with 40 rows costs 64
// columns, not 128 or 256 rows, and experts have few rows each: of 32 experts with 8190 rows by Zipf's law, tiles of 256 rows
// would be 63 % filled, of 128 rows 82 %, these are 95 %: 145 -> 128 us for the input's gradient of 20 experts, 835 -> 704 gated.  Sums come out of tensor memory with a weight's column in each lane;
// they are turned back in shared memory.
//   NT  out[i][n] = sum_k a[i][k] w_e[n][k]          NN  out[i][k] = sum_n a[i][n] w_e[n][k]
// GATED makes two products of 256 x 128 in a tile, g and u of the same columns in the same lanes.
// The rest is as in hap_products_tc.cuh, whose pieces this uses.
#pragma once
#include "hap_products_tc.cuh"

namespace hapop {

template <int EPI> struct Turned {
    static constexpr int ROWS = EPI == GATED ? 128 : 256;           // most rows of a tile
    static constexpr int A_BYTES = (EPI == GATED ? 2 : 1) * 128 * BK * 2, B_BYTES = ROWS / 2 * BK * 2, STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = EPI == STORE ? 6 : 5;
    // GATED_BACK: two buffers of each warp for 16 rows of 32 values of the kept g and u
    static constexpr int KEPT = EPI == GATED_BACK ? 2 * 2 * 1024 : 0;
    static constexpr int PIECE = EPI == STORE ? 32 : 16;            // rows that a warp takes at a time: what fits its registers
    static constexpr int OUT = PIECE * 64;                          // shared memory of a warp for them
};

template <int EPI> struct TurnedShared {
    Schedule<Turned<EPI>::ROWS> sched;
    uint64_t full[8], empty[8], acc_full[2], acc_empty[2], kept[8][2];
    uint32_t tmem;
    int stop;
};

// A warp's 32 columns (one for each lane) of R rows of 16-bit values, to and from memory through shared memory: words of two
// rows of a column, R / 2 rows of 32 words.  Four lanes take two rows' 64 bytes; of pairs side by side one reads the words the
// other way around, so that the banks differ.
struct WarpColumns {
    uint32_t *staged;
    int lane;
    template <typename T> __device__ __forceinline__ bool whole(const T *first, int64_t ld, int cols) const { return cols >= 32 && ((uintptr_t)first & 15) == 0 && ld % 8 == 0; }
    __device__ __forceinline__ uint4 *words(int pair, int c, int h) const { return (uint4 *)(staged + pair * 32 + c * 8 + h * 4); }
    // first: row 0 of the first lane's column; rows, cols: how many there are
    template <typename T, int R> __device__ __forceinline__ void store(T *first, int64_t ld, const float (&v)[R], int rows, int cols) const
    {
        if (!whole(first, ld, cols)) {
#pragma unroll
            for (int i = 0; i < R; i++)
                if (i < rows && lane < cols) first[i * ld + lane] = from_float<T>(v[i]);
            return;
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < R / 2; i++) staged[i * 32 + lane] = pack2(v[2 * i], v[2 * i + 1], T());
        __syncwarp();
#pragma unroll
        for (int i = 0; i < R / 16; i++) {
            const int pair = i * 8 + (lane >> 2), c = lane & 3, odd = pair & 1;
            const uint4 x = *words(pair, c, odd), y = *words(pair, c, odd ^ 1);
            const uint4 lo = odd ? y : x, hi = odd ? x : y;
            T *o = first + 2 * pair * ld + c * 8;
            if (2 * pair < rows) *(uint4 *)o = make_uint4(__byte_perm(lo.x, lo.y, 0x5410), __byte_perm(lo.z, lo.w, 0x5410), __byte_perm(hi.x, hi.y, 0x5410), __byte_perm(hi.z, hi.w, 0x5410));
            if (2 * pair + 1 < rows)
                *(uint4 *)(o + ld) = make_uint4(__byte_perm(lo.x, lo.y, 0x7632), __byte_perm(lo.z, lo.w, 0x7632), __byte_perm(hi.x, hi.y, 0x7632), __byte_perm(hi.z, hi.w, 0x7632));
        }
    }
    template <typename T, int R> __device__ __forceinline__ void read(const T *first, int64_t ld, float (&v)[R], int rows, int cols) const
    {
#pragma unroll
        for (int i = 0; i < R; i++) v[i] = i < rows && lane < cols ? to_float(first[i * ld + lane]) : 0.0f;
    }
};

template <typename T, int FORM, int EPI>
__global__ void __launch_bounds__(320, 1) expert_kernel(const __grid_constant__ Args p, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_rows,
                                                        const __grid_constant__ CUtensorMap map_few, const __grid_constant__ CUtensorMap map_kept)
{
    using S = Turned<EPI>;
    extern __shared__ char raw[];
    char *stages = (char *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    char *outs = stages + S::STAGES * S::STAGE;
    TurnedShared<EPI> &sh = *(TurnedShared<EPI> *)(outs + 8 * (S::OUT + S::KEPT));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    constexpr int BN = 256;                                 // columns of out that a tile covers
    const int col_tiles = (p.ncols + BN - 1) / BN;

    launch_next();
    if (threadIdx.x == 0) prefetch_map(&map_w), prefetch_map(&map_rows);
    if (warp == 1) {
        if (lane == 0) {
            for (int i = 0; i < S::STAGES; i++) bar_init(&sh.full[i], 2), bar_init(&sh.empty[i], 1);
            for (int i = 0; i < 2; i++) bar_init(&sh.acc_full[i], 1), bar_init(&sh.acc_empty[i], 16);
            for (int i = 0; i < 16; i++) bar_init(&sh.kept[i / 2][i % 2], 1);
            sh.stop = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async;" ::: "memory");
        }
        __syncwarp();
        tmem_alloc<2>(&sh.tmem);
    }
    wait_for_last();
    sh.sched.fetch(p);
    __syncthreads();
    if (warp == 0) sh.sched.build(p, col_tiles, lane);
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    const uint32_t tmem = *(volatile uint32_t *)&sh.tmem;
    volatile int *stop = &sh.stop;
    const int total = sh.sched.total(p, FORM, col_tiles), step = gridDim.x / 2, begin = blockIdx.x / 2;
    // rows of a tile, as the products count them
    auto rows_of = [](const auto &tile) { return min(S::ROWS, (tile.hi - tile.lo - tile.m * S::ROWS + 31) & ~31); };

    if (warp == 0) {
        uint32_t at = 0;
        bool good = true;
        for (int t = begin; t < total && good; t += step) {
            const auto tile = sh.sched.tile(p, FORM, col_tiles, t);
            const int n0 = tile.n * BN + (int)rank * 128, half = rows_of(tile) / 2, row = tile.lo + tile.m * S::ROWS + (int)rank * half;
            for (int k = 0; k < p.kdim; k += BK, at++) {
                const int s = at % S::STAGES;
                if (!(good = bar_wait(&sh.empty[s], (at / S::STAGES + 1) & 1, stop))) break;
                const uint32_t a = smem_u32(stages + s * S::STAGE), b = a + S::A_BYTES, full = of_leader(smem_u32(&sh.full[s]));
                if (elected()) {
                    bar_expect_at<2>(full, S::A_BYTES + half * 128);
                    if (FORM == NT) {
                        tma_load<2>(&map_w, a, full, k, n0, tile.e);
                        if (EPI == GATED) tma_load<2>(&map_w, a + 128 * 128, full, k, p.ncols + n0, tile.e);
                    } else {
                        tma_load<2>(&map_w, a, full, n0, k, tile.e);
                        tma_load<2>(&map_w, a + BK * 128, full, n0 + 64, k, tile.e);
                    }
                    if (half == S::ROWS / 2) tma_load<2>(&map_rows, b, full, k, row, 0);
                    else
                        for (int i = 0; i < half; i += 16) tma_load<2>(&map_few, b + i * 128, full, k, row + i, 0);
                }
                __syncwarp();
            }
        }
        if (good) wait_for_empty<S::STAGES>(sh.empty, at, stop);
        if (*stop && rank == 0) drain(sh.full, at, S::STAGES);
    } else if (warp == 1) {
        if (rank == 0) {
            constexpr uint32_t idesc = 1u << 4 | TypeBits<T>::value << 7 | TypeBits<T>::value << 10 | (FORM == NN ? 1u << 15 : 0) | (256u / 16) << 24;
            uint32_t at = 0, sums = 0;
            bool good = true;
            for (int t = begin; t < total && good; t += step) {
                const auto tile = sh.sched.tile(p, FORM, col_tiles, t);
                const uint32_t of = idesc | (uint32_t)(rows_of(tile) / 8) << 17;
                const int set = sums & 1;
                if (!(good = bar_wait(&sh.acc_empty[set], (sums / 2 + 1) & 1, stop))) break;
                sums++;
                fence_after();
                for (int k = 0; k < p.kdim; k += BK, at++) {
                    const int s = at % S::STAGES;
                    if (!(good = bar_wait(&sh.full[s], (at / S::STAGES) & 1, stop))) break;
                    fence_after();
                    if (elected()) {
                        const uint32_t a = smem_u32(stages + s * S::STAGE), b = a + S::A_BYTES;
                        const uint64_t da = FORM == NN ? smem_desc(a, BK * 128, 1024) : smem_desc(a, 16, 1024), db = smem_desc(b, 16, 1024);
#pragma unroll
                        for (int i = 0; i < BK / 16; i++) {
                            mma<2>(tmem + set * 256, da + i * (FORM == NN ? 128 : 2), db + i * 2, of, k > 0 || i > 0);
                            if (EPI == GATED) mma<2>(tmem + set * 256 + 128, da + 1024 + i * 2, db + i * 2, of, k > 0 || i > 0);
                        }
                        mma_commit<2>(&sh.empty[s]);
                        if (k + BK >= p.kdim) mma_commit<2>(&sh.acc_full[set]);
                    }
                    __syncwarp();
                }
            }
        }
    } else {
        uint32_t sums = 0, asked = 0, used = 0;             // asked, used: pieces of the kept g and u
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        char *kept = outs + 8 * S::OUT + (warp - 2) * S::KEPT;
        const WarpColumns w{(uint32_t *)(outs + (warp - 2) * S::OUT), lane};
        const uint32_t from = tmem + ((uint32_t)quarter << 21);
        for (int t = begin; t < total; t += step) {
            const auto tile = sh.sched.tile(p, FORM, col_tiles, t);
            const int set = sums & 1, col = tile.n * BN + (int)rank * 128 + quarter * 32, cols = p.ncols - col;
            constexpr int R = S::PIECE;
            const int pieces = rows_of(tile) / R, live = tile.hi - tile.lo - tile.m * S::ROWS;
            const int64_t row0 = (int64_t)tile.lo + tile.m * S::ROWS;
            // the kept g and u of a piece come by TMA, two pieces ahead (loads of the lanes, turned in shared memory, one piece ahead:
            // 193 us at 64 experts with 32760 rows, 2048 x 1024, where this takes 151)
            const bool mapped = EPI == GATED_BACK && p.kept_mapped;
            auto bring = [&](int q) {
                if (mapped && lane == 0) {
                    const uint32_t bar = smem_u32(&sh.kept[warp - 2][asked & 1]), to = smem_u32(kept + (asked & 1) * 2048);
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], 2048;" ::"r"(bar) : "memory");
                    tma_load<1>(&map_kept, to, bar, col, (int)row0 + q * R, 0);
                    tma_load<1>(&map_kept, to + 1024, bar, p.ncols + col, (int)row0 + q * R, 0);
                }
                if (mapped) asked++;
            };
            if (cols > 0)
                for (int q = half; q < min(pieces, half + 4); q += 2) bring(q);
            if (!bar_wait(&sh.acc_full[set], (sums / 2) & 1, stop)) break;
            sums++;
            fence_after();
            auto taken = [&] {
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_at<2>(of_leader(smem_u32(&sh.acc_empty[set])));
            };
            if (cols <= 0 || half >= pieces) {
                taken();
                continue;
            }
            for (int q = half; q < pieces; q += 2) {
                const int n = live - q * R;                 // rows of this piece
                const int64_t row = row0 + q * R;
                float v[R];
                __syncwarp();
                tmem_load(from + set * 256 + q * R, v);
                if constexpr (EPI == STORE) {
                    tmem_load_wait();
                    if (q + 2 >= pieces) taken();
                    T *o = (T *)p.out + row * p.ldo + col;
                    if (p.accumulate) {
#pragma unroll
                        for (int i = 0; i < R; i++)
                            if (i < n && lane < cols) v[i] += to_float(o[i * p.ldo + lane]);
                    }
                    w.store(o, p.ldo, v, n, cols);
                }
                if constexpr (EPI == GATED) {
                    float v2[R];
                    tmem_load(from + set * 256 + 128 + q * R, v2);
                    tmem_load_wait();
                    if (q + 2 >= pieces) taken();
                    if (p.out) {
                        T *o = (T *)p.out + row * p.ldo + col;
                        w.store(o, p.ldo, v, n, cols);
                        w.store(o + p.ncols, p.ldo, v2, n, cols);
                    }
#pragma unroll
                    for (int i = 0; i < R; i++) v[i] = gate(v[i], v2[i]);
                    w.store((T *)p.h + row * p.ldh + col, p.ldh, v, n, cols);
                }
                if constexpr (EPI == GATED_BACK) {
                    float g[R], u[R];
                    if (mapped) {
                        const T *at = (const T *)(kept + (used & 1) * 2048) + lane;
                        if (!bar_wait(&sh.kept[warp - 2][used & 1], used >> 1 & 1, stop)) break;
                        used++;
#pragma unroll
                        for (int i = 0; i < R; i++) g[i] = to_float(at[i * 32]), u[i] = to_float(at[512 + i * 32]);
                        __syncwarp();
                        if (q + 4 < pieces) bring(q + 4);
                    } else {
                        const T *gu = (const T *)p.gu + row * p.ldgu + col;
                        w.read(gu, p.ldgu, g, n, cols);
                        w.read(gu + p.ncols, p.ldgu, u, n, cols);
                    }
                    tmem_load_wait();
                    if (q + 2 >= pieces) taken();
#pragma unroll
                    for (int i = 0; i < R; i++) gate_back(g[i], u[i], v[i]);
                    T *o = (T *)p.out + row * p.ldo + col;
                    w.store(o, p.ldo, v, n, cols);
                    w.store(o + p.ncols, p.ldo, u, n, cols);
                    if (p.h) w.store((T *)p.h + row * p.ldh + col, p.ldh, g, n, cols);
                }
            }
        }
        if (EPI == GATED_BACK && lane == 0)                 // cut short: what is still on its way
            for (; used < asked; used++) {
                const uint64_t since = nanoseconds();
                while (!bar_try(smem_u32(&sh.kept[warp - 2][used & 1]), used >> 1 & 1) && nanoseconds() - since < 100000000ull) {}
            }
    }
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    if (warp == 1) tmem_free<2>(tmem);
}

} // namespace hapop
