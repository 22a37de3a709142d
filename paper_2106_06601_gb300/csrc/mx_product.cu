// C = alpha A B^T + beta C with A (m x k) and B (n x k) in E2M1, on the tensor
// cores' block-scaled 4-bit products.
//
// One thread block takes a tile of 128 rows of B (the lanes of tensor memory)
// and NT rows of A (its columns), so that a warp's lanes hold neighbouring
// elements of a row of C and few rows of A need few columns.  The first four or
// eight warps write the tile out, one or two to a quarter of the lanes; the next
// brings operands and scales into a ring of stages of 256 columns of k, and one
// thread of the last issues the products.  Tiles of 256
// rows of A are taken by pairs of blocks, with 256 rows of B: each block then
// brings half of A's rows, a third less for the L2 cache to deliver.  Calls with
// few tiles split k over a cluster and join the parts in their order.  A long k
// takes several sums of a tile, one after another.
//
// GB300: 8192 x 16384 x 8192 302 us, 7.3 PFLOP/s, where four times the measured
// rate of library bf16 products is 7.8: the tensor pipe is 75% busy; of 784 cycles
// a stage its queue takes 621, among them some 150 for copies of scales, and
// operands come late in 105.  1023 x 4096 x 4096 10.7 us: one round of tiles, its
// fill and its way out.  1 x 16384 x 4096 8.8 us for 35.6 MB of weights (4.0
// TB/s): fill, and the join of two halves of k.
#include <algorithm>

#include "costa_internal.h"
#include "mx_tc.cuh"

namespace costa {
namespace mx {
namespace {

constexpr int kRows = 128;  // rows of B in a block's tile
constexpr int kPrefetch = 4;  // stages of B on their way to the L2 early (0, 4, 8, 16: 1 x 16384 x 4096 10.5, 9.8, 10.1, 10.1 us)
constexpr int kMaxSplit = 8;
// A stage holds 256 elements of k: 128 bytes of a row, 2 tiles of scales.
// The tensor cores' sums truncate: for values of one sign some 1.4e-8 of the sum for each product over 64 elements
// (1.4e-5 after 65536 elements). So a sum in tensor memory takes 32 stages at most (8e-7 of it), and sums of a longer k
// are joined in registers, rounded to nearest (LONG): 8192 x 8192 x 8448 163 -> 171 us, 4096 x 8192 x 32768 296 -> 307.
// (16 stages: 3e-7, but 8192 x 16384 x 8192 302 -> 317 us, and 178, 320.)
constexpr int kSumStages = 32;

__device__ unsigned g_failed;

struct Params {
    const uint8_t *a_scales, *b_scales;  // not for pairs
    int steps;           // products of 64 elements over k
    int scale_tiles;     // tiles of scales over k
    int n_tiles, m_tiles;
};

// The columns of tensor memory and the stages of a tile of NT rows of A.
template <int NT> struct Shape {
    static constexpr bool pair = NT == 256;
    static constexpr int blocks = pair ? 2 : 1, rows = blocks * kRows;  // of a tile
    static constexpr int bands = NT > 128 ? 2 : 1;                      // of 128 rows of A's scales
    // Two sums of NT columns, so that one is written out while the next
    // builds.  Two of 256 would leave no room for the scales: they share
    // columns 208 .. 255, which the epilogue reads first (or, of the second
    // sum, also first) and then hands over.
    static constexpr int second = NT == 256 ? 208 : NT;
    static constexpr int scales = NT == 256 ? 464 : 2 * NT;
    static constexpr int scale_cols = 8 + 8 * bands;  // of a stage: 2 tiles of B, 2 of each band of A
    static constexpr int used = scales + 2 * scale_cols;
    static constexpr int cols = used <= 64 ? 64 : used <= 128 ? 128 : used <= 256 ? 256 : 512;
    static constexpr int a_rows = NT / blocks;  // in a block
    // Warps that write a tile out.  Eight would leave registers for one block of an SM, where small tiles have two
    // (1 x 16384 x 4096 9.7, 14.9 us; 1023 x 4096 x 4096 15.2, 14.2).
    static constexpr int writers = NT >= 128 ? 8 : 4, threads = (writers + 2) * 32;
    static constexpr int b_bytes = kRows * 128, a_bytes = a_rows * 128, sf_bytes = 1024 * (1 + bands);
    static constexpr int stage = (b_bytes + a_bytes + sf_bytes + 1023) / 1024 * 1024;
    static constexpr int stages = NT == 256 ? 6 : NT == 128 ? 5 : 4;
    static constexpr int smem = stages * stage + 1024;
    static_assert(smem <= 226 * 1024 && kRows * NT * 4 <= stages * stage, "a tile's partial sums fit the stages");
};

// LONG: a block's k takes more than one sum.
template <int NT, bool LONG, typename T>
__global__ void __launch_bounds__(Shape<NT>::threads, LONG && NT <= 64 ? 2 : 1)
    product_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                   const __grid_constant__ CUtensorMap a_scale_map, const __grid_constant__ CUtensorMap b_scale_map,
                   const Params p, const Output<T> out, const int split) {
    using S = Shape<NT>;
    constexpr bool kPair = S::pair;
    constexpr int kLag = NT == 256 ? 1 : 2;  // the tile whose epilogue a tile waits for
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::stages + 4];
    __shared__ uint32_t tmem_slot;
    __shared__ uint32_t failed_word;
    volatile uint32_t *failed = &failed_word;
    const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u;
    float *const part_sums = reinterpret_cast<float *>(raw + (ring - smem_addr(raw)));
    const uint32_t bar0 = smem_addr(bars);
    auto full = [&](int s) { return bar0 + 8 * s; };  // (a pair's first block's) operands have landed
    auto empty = [&](int s) { return bar0 + 8 * (S::stages + s); };
    auto sum_full = [&](int i) { return bar0 + 8 * (2 * S::stages + i); };
    auto sum_empty = [&](int i) { return bar0 + 8 * (2 * S::stages + 2 + i); };  // (first block's)
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rank = static_cast<int>(cluster_rank()), half = kPair ? rank & 1 : 0;

    if (threadIdx.x == 0) {
        failed_word = 0;
        for (int s = 0; s < S::stages; ++s) {
            bar_init(full(s), 1);
            bar_init(empty(s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(sum_full(i), 1);
            bar_init(sum_empty(i), S::writers * S::blocks);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == S::writers + 1) {
        if constexpr (kPair)
            tmem_alloc_pair(&tmem_slot, S::cols);
        else
            tmem_alloc(&tmem_slot, S::cols);
    }
    fence_before();
    __syncthreads();
    if constexpr (kPair) cluster_sync();
    fence_after();
    const uint32_t tmem = tmem_slot;
    let_next_start();

    // This block's share of k, in stages; and its tiles.  (Pairs do not split k.)
    const int stages_k = (p.steps + 3) / 4;
    const int part = kPair ? 0 : rank, per_tile = kPair ? 2 : split;
    const int k_first = static_cast<int>(int64_t(stages_k) * part / split);
    const int k_last = static_cast<int>(int64_t(stages_k) * (part + 1) / split);
    const int sums = (k_last - k_first + kSumStages - 1) / kSumStages, sum_k = (k_last - k_first + sums - 1) / sums;  // LONG: stages of each
    const int tiles = p.n_tiles * p.m_tiles, first = blockIdx.x / per_tile, stride = gridDim.x / per_tile;
    // Few rows of A: the time is that of reading B, which starts while the kernel before this one ends.
    if (NT <= 64 && warp == S::writers && first < tiles && elect_one())
        for (int k = k_first; k < min(k_last, k_first + kPrefetch); ++k)
            tma_prefetch_2d(&b_map, k * 128, first / p.m_tiles * kRows);
    __syncwarp();
    after_previous();

    if (warp == S::writers) {
        if (elect_one()) {
            Ring<S::stages> at;
            for (int t = first; t < tiles && !*failed; t += stride) {
                const int nt = t / p.m_tiles, mt = t % p.m_tiles;
                for (int k = k_first; k < k_last; ++k, at.next()) {
                    if (!bar_wait(empty(at.s), at.parity ^ 1, failed)) break;
                    const uint32_t to = ring + at.s * S::stage, sf = to + S::b_bytes + S::a_bytes, bar = full(at.s);
                    if constexpr (kPair) {
                        // tiles past the last over k, and bands past the last, bring what no product reads
                        if (half == 0) bar_expect(bar, 2 * (S::b_bytes + S::a_bytes + S::sf_bytes));
                        const int band = mt * 2, row = nt * 2 + half;
                        tma_load_2d_at(to, &b_map, k * 128, row * kRows, bar, 0);
                        tma_load_2d_at(to + S::b_bytes, &a_map, k * 128, mt * NT + half * S::a_rows, bar, 0);
                        tma_load_2d_at(sf, &b_scale_map, 0, row * p.scale_tiles + 2 * k, bar, 0);
                        for (int b = 0; b < 2; ++b)
                            tma_load_2d_at(sf + 1024 * (1 + b), &a_scale_map, 0, (band + b) * p.scale_tiles + 2 * k, bar, 0);
                    } else {
                        const int sft = min(2, p.scale_tiles - 2 * k);  // tiles of scales of this stage
                        bar_expect(bar, S::b_bytes + S::a_bytes + 2 * sft * 512);
                        tma_load_2d(to, &b_map, k * 128, nt * kRows, bar);
                        tma_load_2d(to + S::b_bytes, &a_map, k * 128, mt * NT, bar);
                        bulk_load(sf, p.b_scales + (int64_t(nt) * p.scale_tiles + 2 * k) * 512, sft * 512, bar);
                        bulk_load(sf + 1024, p.a_scales + (int64_t(mt) * p.scale_tiles + 2 * k) * 512, sft * 512, bar);
                    }
                }
            }
        }
    } else if (warp == S::writers + 1) {
        if (half == 0 && elect_one()) {
            auto commit = [&](uint32_t bar) {
                if constexpr (kPair)
                    mma_commit_pair(bar, 3);
                else
                    mma_commit(bar);
            };
            auto copy_scales = [&](uint32_t to, uint32_t from) {
                if constexpr (kPair)
                    scales_to_tmem_pair(to, scales_desc(from));
                else
                    scales_to_tmem(to, scales_desc(from));
            };
            Ring<S::stages> at;
            int done = 0;
            uint32_t turn = 0;
            for (int t = first, from_k = k_first; t < tiles && !*failed; ++done) {  // all sums of this block's tiles
                const uint32_t d = tmem + (done & 1 ? S::second : 0);
                const int before = done - kLag, to_k = LONG ? min(k_last, from_k + sum_k) : k_last;
                if (before >= 0 && !bar_wait(sum_empty(before & 1), (before >> 1) & 1, failed)) break;
                fence_after();
                for (int k = from_k; k < to_k; ++k, at.next()) {
                    if (!bar_wait(full(at.s), at.parity, failed)) break;
                    fence_after();
                    const uint32_t from = ring + at.s * S::stage, sf = from + S::b_bytes + S::a_bytes;
                    const uint32_t sfd = tmem + S::scales + turn * S::scale_cols;
                    turn ^= 1;
                    const int steps = min(4, p.steps - 4 * k);
                    // columns of the scales: B's two tiles, then A's as (k tile, band)
                    for (int c = 0; 2 * c < steps; ++c) {
                        copy_scales(sfd + 4 * c, sf + 512 * c);
                        for (int b = 0; b < S::bands; ++b)
                            copy_scales(sfd + 8 + 4 * (S::bands * c + b), sf + 1024 * (1 + b) + 512 * c);
                    }
                    const uint64_t da = operand_desc(from, 16, 1024), db = operand_desc(from + S::b_bytes, 16, 1024);
                    for (int q = 0; q < steps; ++q) {
                        const uint32_t idesc = idesc_e2m1(S::rows, NT, (q & 1) * 2), sfa = sfd + 4 * (q >> 1),
                                       sfb = sfd + 8 + 4 * S::bands * (q >> 1);
                        if constexpr (kPair)
                            mma_e2m1_pair(d, da + 2 * q, db + 2 * q, idesc, sfa, sfb, k > from_k || q > 0);
                        else
                            mma_e2m1(d, da + 2 * q, db + 2 * q, idesc, sfa, sfb, k > from_k || q > 0);
                    }
                    commit(empty(at.s));
                }
                if (*failed) break;
                commit(sum_full(done & 1));
                from_k = LONG && to_k < k_last ? to_k : k_first;
                if (from_k == k_first) t += stride;
            }
        }
    } else if constexpr (LONG) {  // the sums of a tile are joined in registers, rounded to nearest
        constexpr int kStep = S::writers / 4, kOwn = NT / 16 / kStep;  // this warp's chunks of 16 columns: pick, pick + kStep, ..
        const int pick = warp / 4, quarter = warp % 4 * 32;
        int done = 0;
        for (int t = first; t < tiles; t += stride) {
            float acc[kOwn * 16];
#pragma unroll
            for (int i = 0; i < kOwn * 16; ++i) acc[i] = 0.0f;
            bool ok = true;
            for (int c = 0; c < sums && ok; ++c, ++done) {
                ok = __all_sync(~0u, bar_wait(sum_full(done & 1), (done >> 1) & 1, failed));
                if (!ok) break;
                fence_after();
                const uint32_t from = tmem + (done & 1 ? S::second : 0) + (uint32_t(quarter) << 16) + pick * 16;
#pragma unroll
                for (int j = 0; j < kOwn; ++j) {
                    // The columns that either sum shares first: one order for both, as two ways through here would hold
                    // the sums twice.
                    static_assert(kLag != 1 || (kOwn >= 4 && 2 * kStep >= 3), "they are among each warp's outer four chunks");
                    const int own = kLag != 1 ? j : j < 2 ? j : j < 4 ? kOwn - 4 + j : j - 2;
                    uint32_t r[16];
                    tmem_ld16(from + kStep * own * 16, r);
                    tmem_wait_ld(r);
                    if (j == (kLag == 1 ? 3 : kOwn - 1)) {
                        fence_before();
                        __syncwarp();
                        if (lane == 0) {
                            if constexpr (kPair)
                                bar_arrive_at(sum_empty(done & 1), 0);
                            else
                                bar_arrive(sum_empty(done & 1));
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[own * 16 + i] += __uint_as_float(r[i]);
                }
            }
            if (!ok) break;
            const int64_t row0 = int64_t(t % p.m_tiles) * NT + pick * 16;
            const int64_t col = int64_t(t / p.m_tiles) * S::rows + half * kRows + quarter + lane;
#pragma unroll
            for (int own = 0; own < kOwn; ++own) {
                if (split > 1) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        part_sums[((pick + kStep * own) * 16 + i) * kRows + quarter + lane] = acc[own * 16 + i];
                } else {
                    out.put_each(row0 + kStep * own * 16, col, [&](int i) { return acc[own * 16 + i]; });
                }
            }
        }
    } else {
        int done = 0;
        for (int t = first; t < tiles; t += stride, ++done) {
            if (!__all_sync(~0u, bar_wait(sum_full(done & 1), (done >> 1) & 1, failed))) break;
            fence_after();
            const int nt = t / p.m_tiles, mt = t % p.m_tiles;
            const uint32_t d = tmem + (done & 1 ? S::second : 0);
            // Chunks of 16 columns, the warps of a quarter in turn; the shared columns first: chunks 13 .. 15 of the first
            // sum, 0 .. 2 of the second.
            constexpr int kChunks = NT / 16, kStep = S::writers / 4;
            const int shift = kLag == 1 && !(done & 1) ? kChunks - 3 : 0, pick = warp / 4, quarter = warp % 4 * 32;
            const uint32_t lanes = d + (uint32_t(quarter) << 16);
            const int64_t row0 = int64_t(mt) * NT;
            const int64_t col = int64_t(nt) * S::rows + half * kRows + quarter + lane;
            auto load = [&](int j, uint32_t(&r)[16]) { tmem_ld16(lanes + (j + shift) % kChunks * 16, r); };
            auto write = [&](int j, const uint32_t(&r)[16]) {
                const int ch = (j + shift) % kChunks;
                if (split > 1) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) part_sums[(ch * 16 + i) * kRows + quarter + lane] = __uint_as_float(r[i]);
                } else {
                    out.put16(row0 + ch * 16, col, [&](int i) { return __uint_as_float(r[i]); });
                }
            };
            auto drained = [&] {
                fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (kPair)
                        bar_arrive_at(sum_empty(done & 1), 0);
                    else
                        bar_arrive(sum_empty(done & 1));
                }
            };
            static_assert(kLag != 1 || 2 * kStep >= 3, "the shared columns are among the first two of each warp");
            constexpr int kFirst = kLag == 1 ? 2 : 0;  // of a warp, among them the shared columns: read before any is written
            if constexpr (kFirst > 0) {
                uint32_t r[2][16];
                load(pick, r[0]);
                load(pick + kStep, r[1]);
                tmem_wait_ld(r[0]);
                tmem_wait_ld(r[1]);
                drained();
                write(pick, r[0]);
                write(pick + kStep, r[1]);
            }
            // a chunk is loaded while the one before it is written
            uint32_t r[2][16];
            load(pick + kStep * kFirst, r[0]);
#pragma unroll 1
            for (int j = pick + kStep * kFirst; j < kChunks; j += 2 * kStep) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (j + kStep * h >= kChunks) break;
                    tmem_wait_ld(r[h]);
                    if (j + kStep * (h + 1) < kChunks) load(j + kStep * (h + 1), r[1 - h]);
                    write(j + kStep * h, r[h]);
                }
            }
            if constexpr (kFirst == 0) drained();
        }
    }
    __syncwarp();

    if (*failed) let_copies_land();
    if (split > 1) {  // one tile to a cluster
        cluster_sync();
        join_split<kMaxSplit>(out, ring, 0, 1, part, split, threadIdx.x, S::threads, int64_t(first % p.m_tiles) * NT,
                              int64_t(first / p.m_tiles) * kRows, NT);
        cluster_sync();
    }
    fence_before();
    __syncthreads();
    if constexpr (kPair) cluster_sync();  // neither block leaves while the other's products run
    if (warp == S::writers + 1) {
        fence_after();
        if constexpr (kPair)
            tmem_free_pair(tmem, S::cols);
        else
            tmem_free(tmem, S::cols);
    }
    if (threadIdx.x == 0 && *failed) atomicAdd(&g_failed, 1u);
}

template <int NT, typename T>
cudaError_t launch(const costa_mx_matrix &A, const costa_mx_matrix &B, float alpha, float beta, const costa_mx_dense &C,
                   int sms, cudaStream_t s) {
    using S = Shape<NT>;
    const int64_t nb = mx_blocks(A.cols);
    CUtensorMap a_map, b_map, a_scale_map, b_scale_map;
    cudaError_t e = mx_byte_map(&a_map, A.codes, 16 * nb, A.rows, A.ld, S::a_rows);
    if (e == cudaSuccess) e = mx_byte_map(&b_map, B.codes, 16 * nb, B.rows, B.ld, kRows);
    if constexpr (S::pair) {
        const int64_t tiles_k = mx_scale_tiles(A.cols), a_tiles = mx_ceil(A.rows, 128) * tiles_k,
                      b_tiles = mx_ceil(B.rows, 128) * tiles_k;
        if (a_tiles > INT32_MAX / 2 || b_tiles > INT32_MAX / 2) return cudaErrorInvalidValue;
        if (e == cudaSuccess) e = mx_scale_map(&a_scale_map, A.scales, a_tiles, 2);
        if (e == cudaSuccess) e = mx_scale_map(&b_scale_map, B.scales, b_tiles, 2);
    } else {
        a_scale_map = a_map;
        b_scale_map = b_map;
    }
    if (e != cudaSuccess) return e;
    Params p;
    p.a_scales = static_cast<const uint8_t *>(A.scales);
    p.b_scales = static_cast<const uint8_t *>(B.scales);
    p.steps = static_cast<int>(mx_ceil(nb, 2));
    p.scale_tiles = static_cast<int>(mx_scale_tiles(A.cols));
    p.n_tiles = static_cast<int>(mx_ceil(C.cols, S::rows));
    p.m_tiles = static_cast<int>(mx_ceil(C.rows, NT));
    const Output<T> out{static_cast<T *>(C.ptr), C.ld, C.rows, C.cols, alpha, beta};
    const int64_t tiles = int64_t(p.n_tiles) * p.m_tiles;
    if (tiles > INT32_MAX / 2) return cudaErrorInvalidValue;
    const int stages_k = (p.steps + 3) / 4;
    // As many parts of k as run at a time, of two stages at least.
    int split = 1;
    while (!S::pair && split < kMaxSplit && tiles <= mx_clusters(2 * split, NT <= 64 ? 2 : 1) && stages_k >= 4 * split)
        split *= 2;
    const int64_t blocks = S::blocks * (split > 1 ? tiles * split : std::min<int64_t>(tiles, sms / S::blocks));
    const bool one_sum = mx_ceil(stages_k, split) <= kSumStages;
    return mx_launch(one_sum ? product_kernel<NT, false, T> : product_kernel<NT, true, T>, blocks, S::threads, S::smem, S::blocks * split, s, a_map, b_map, a_scale_map,
                     b_scale_map, p, out, split);
}

template <typename T>
cudaError_t by_rows(const costa_mx_matrix &A, const costa_mx_matrix &B, float alpha, float beta, const costa_mx_dense &C,
                    int sms, cudaStream_t s) {
    if (C.rows <= 16) return launch<16, T>(A, B, alpha, beta, C, sms, s);
    if (C.rows <= 32) return launch<32, T>(A, B, alpha, beta, C, sms, s);
    if (C.rows <= 64) return launch<64, T>(A, B, alpha, beta, C, sms, s);
    // A round of tiles of 256 x 256 on all pairs takes 1.26 times as long as one of 128 x 128 on all SMs (1100 x 4096 x
    // 4096, two rounds of either: 20.7 and 17.5 us with the quantisation; 768 rows, one round and two: 13.7, 16.5;
    // 512 rows, one of either: 12.9, 10.9; 2048 rows, two and four: 23.1, 29.3).
    const int64_t small = mx_ceil(mx_ceil(C.rows, 128) * mx_ceil(C.cols, 128), sms),
                  large = mx_ceil(mx_ceil(C.rows, 256) * mx_ceil(C.cols, 256), sms / 2);
    if (C.rows <= 128 || 4 * small <= 5 * large) return launch<128, T>(A, B, alpha, beta, C, sms, s);
    return launch<256, T>(A, B, alpha, beta, C, sms, s);
}

}  // namespace
}  // namespace mx

cudaError_t launch_mx_product(const costa_mx_matrix &A, const costa_mx_matrix &B, float alpha, float beta,
                              const costa_mx_dense &C, cudaStream_t s) {
    if (A.cols == 0) return launch_mx_scale(beta, C, s);
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    return C.type == COSTA_MX_F32 ? mx::by_rows<float>(A, B, alpha, beta, C, sms, s)
                                  : mx::by_rows<__nv_bfloat16>(A, B, alpha, beta, C, sms, s);
}

cudaError_t mx_product_failures(unsigned *count) {
    return cudaMemcpyFromSymbol(count, mx::g_failed, sizeof *count);
}

}  // namespace costa
