// dW = alpha dY^T X + beta dW with X (m x k) from its 8-bit checkpoint and dY
// (m x n) in bf16 or f32, on the tensor cores' bf16 products.
//
// A checkpoint's value is an integer below 2^7 times a power of two: exact in
// bf16.  An f32 gradient is cut into three bf16 parts of 8 bits each (by
// truncation, so no part overflows), and their products are summed in the same
// accumulator.  So every product is that of the values, and only the sums round.
//
// A pair of thread blocks takes a tile of 256 columns of X (the lanes of tensor
// memory, 128 in each block: neighbouring elements of a row of dW) and NT
// columns of dY, half of which each block holds, and runs over the tokens in
// stages of 64.  The checkpoint's codes and scales are brought in by bulk copies
// and cp.async; converter warps turn them into bf16 in the tensor cores' layout.
// dY comes by bulk copies as it is where it is bf16 with 16-byte aligned rows
// (kDirect); else the converter warps load, cut and store it.
//
// The tensor cores' sums truncate, about 1.3e-8 of the sum's magnitude for each
// product over 16 tokens (measured: 1.3e-5 after 1024).  So a sum takes
// kProducts of them at most, in one of two places in tensor memory; eight warps
// add each to sums in registers, rounded to nearest, while the next one builds.
#include <algorithm>
#include <type_traits>

#include "costa_internal.h"
#include "mx_tc.cuh"

namespace costa {
namespace mx {
namespace {

constexpr int kCols = 128;     // columns of X in a block's half of a tile
constexpr int kTokens = 64;    // of a stage
constexpr int kProducts = 32;  // to a sum in tensor memory

__device__ unsigned g_failed;

struct Params {
    const uint8_t *scales;
    int64_t pitch;       // bytes of a row of scales
    const void *dy;      // not kDirect
    int64_t ldy;
    bool vec;            // its rows are 16-byte aligned
    int64_t m, n;
    int n_tiles, k_tiles;
};

enum Source { kDirect = 0, kBf16 = 1, kF32 = 3 };  // of dY; the number of parts if not direct

template <int NT, int SRC> struct Shape {
    static constexpr int parts = SRC == kF32 ? 3 : 1;
    static constexpr int half = NT / 2;  // columns of dY in a block
    static constexpr int x_bytes = kCols * kTokens * 2, y_part = half * kTokens * 2, y_bytes = parts * y_part;
    static constexpr int operands = x_bytes + y_bytes;         // of a stage, in the tensor cores' layout
    static constexpr int raw = kCols * kTokens + kTokens * 4;  // codes and scales
    static constexpr int stages = SRC == kF32 ? 4 : 5, raw_stages = 6;
    static constexpr int smem = stages * operands + raw_stages * raw + 1024;
    static constexpr int converters = 4, sets = SRC == kDirect ? 3 : 2;  // warps of a stage; sets that take turns
    static constexpr int warps = 8 + 4 + sets * converters;    // 8 for the sums; copies of dY and of X, products
    static constexpr int cols = 2 * NT;
    // registers of a thread: at launch, and then of the sums', the copies' and the converters' warpgroups
    static constexpr int at_launch = SRC == kDirect ? 80 : 96;
    static constexpr int for_sums = SRC == kDirect ? 168 : 112, for_copies = SRC == kDirect ? 24 : 64,
                         for_converters = SRC == kDirect ? 40 : 96;
    static_assert(2 * for_sums + for_copies + sets * for_converters <= warps / 4 * at_launch, "registers");
    static constexpr int chunk = kProducts / (parts * (kTokens / 16));  // stages to a sum
    static_assert(smem <= 226 * 1024 && kCols * NT * 4 <= stages * operands, "shared memory");
};

// Four codes of one word as bf16 pairs, times 2^e given as a bf16 pair.  With 7
// low bits r and sign bit s a code is r - 128 s; as bf16, 0x4300 | r is 128 + r,
// and 0x4300 | 128 s is 128 or 256.  The pairs are elements 0, 2 and 1, 3, which
// saves two permutations: positions 1 and 2 of each four columns of a tile are
// exchanged until the sums are written out.
__device__ __forceinline__ void codes_to_bf16(uint32_t w, __nv_bfloat162 unit, uint32_t &lo, uint32_t &hi) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t two = h ? w >> 8 : w;
        const uint32_t a = (two & 0x007f007fu) | 0x43004300u, b = (two & 0x00800080u) | 0x43004300u;
        __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
        v = __hmul2(v, unit);
        (h ? hi : lo) = *reinterpret_cast<const uint32_t *>(&v);
    }
}
// The column in a tile whose sum a lane has.
__device__ __forceinline__ int column_of(int lane) { return (lane & ~3) | (lane & 1) << 1 | (lane >> 1 & 1); }

// 2^(s - 133), the unit of codes with scale byte s, as a bf16 pair: subnormal below 2^-126; NaN for 255.
__device__ __forceinline__ __nv_bfloat162 bf16_unit(uint32_t s) {
    const uint32_t one = s == 255 ? 0x7fffu : s <= 6 ? 1u << s : (s - 6) << 7;
    const uint32_t two = one | one << 16;
    return *reinterpret_cast<const __nv_bfloat162 *>(&two);
}

__device__ __forceinline__ uint2 load8b(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}
__device__ __forceinline__ uint32_t load_byte(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ void store16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// The next 8 bits of each of two numbers as a bf16 pair, taken off them.
__device__ __forceinline__ uint32_t take_part(float &a, float &b) {
    const uint32_t x = __float_as_uint(a) & 0xffff0000u, y = __float_as_uint(b) & 0xffff0000u;
    a -= __uint_as_float(x);
    b -= __uint_as_float(y);
    return x >> 16 | y;
}

template <int NT, int SRC, typename T>
__global__ void __launch_bounds__(Shape<NT, SRC>::warps * 32, 1)
    grad_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap y_map, const Params p,
                const Output<T> out, const int split) {
    using S = Shape<NT, SRC>;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[2 * (S::stages + S::raw_stages) + 4];
    __shared__ uint32_t tmem_slot;
    __shared__ uint32_t failed_word;
    volatile uint32_t *failed = &failed_word;
    const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u, raws = ring + S::stages * S::operands;
    float *const part_sums = reinterpret_cast<float *>(raw + (ring - smem_addr(raw)));
    const uint32_t bar0 = smem_addr(bars), bar1 = bar0 + 16 * S::stages, bar2 = bar1 + 16 * S::raw_stages;
    auto full = [&](int s) { return bar0 + 16 * s; };        // (first block's) both blocks' operands
    auto empty = [&](int s) { return bar0 + 16 * s + 8; };   // products have read the stage
    auto landed = [&](int r) { return bar1 + 16 * r; };      // codes and scales
    auto taken = [&](int r) { return bar1 + 16 * r + 8; };   // converters have read them
    auto sum_full = [&](int i) { return bar2 + 8 * i; };
    auto sum_empty = [&](int i) { return bar2 + 16 + 8 * i; };  // (first block's)
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rank = static_cast<int>(cluster_rank()), half = rank & 1, lead = rank & ~1, part = rank >> 1;

    let_next_start();
    if (threadIdx.x == 0) {
        failed_word = 0;
        for (int s = 0; s < S::stages; ++s) {
            bar_init(full(s), (SRC == kDirect) + 2 * S::converters);
            bar_init(empty(s), 1);
        }
        for (int r = 0; r < S::raw_stages; ++r) {
            bar_init(landed(r), 1 + 32);
            bar_init(taken(r), S::converters);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(sum_full(i), 1);
            bar_init(sum_empty(i), 16);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) tmem_alloc_pair(&tmem_slot, S::cols);
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    const uint32_t tmem = tmem_slot;
    after_previous();

    const int64_t stages_m = (p.m + kTokens - 1) / kTokens;
    const int64_t s_first = stages_m * part / split, s_last = stages_m * (part + 1) / split;
    const int tiles = p.n_tiles * p.k_tiles, first = blockIdx.x / (2 * split), stride = gridDim.x / (2 * split);

    // Each role takes its registers first, so that its code is laid out for them.
    if (warp < 8) {  // sums; warp w: lanes of quarter w % 4, half of the columns
        more_registers<S::for_sums>();
        const int64_t chunks = (s_last - s_first + S::chunk - 1) / S::chunk;
        const uint32_t at = tmem + (uint32_t(warp % 4 * 32) << 16) + warp / 4 * S::half;
        int64_t sum = 0;
        for (int t = first; t < tiles; t += stride) {
            float acc[S::half];
#pragma unroll
            for (int i = 0; i < S::half; ++i) acc[i] = 0.0f;
            bool ok = true;
            for (int64_t c = 0; c < chunks && ok; ++c, ++sum) {
                ok = __all_sync(~0u, bar_wait(sum_full(sum & 1), (sum >> 1) & 1, failed));
                fence_after();
#pragma unroll
                for (int g = 0; g < S::half / 16; ++g) {
                    uint32_t r[16];
                    tmem_ld16(at + (sum & 1) * NT + g * 16, r);
                    tmem_wait_ld(r);
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[g * 16 + i] += __uint_as_float(r[i]);
                }
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_at(sum_empty(sum & 1), lead);
            }
            if (!ok) break;
            const int64_t row0 = int64_t(t / p.k_tiles) * NT + warp / 4 * S::half;
            const int64_t col = int64_t(t % p.k_tiles) * (2 * kCols) + half * kCols + warp % 4 * 32 + column_of(lane);
#pragma unroll
            for (int i = 0; i < S::half; i += 16) {
                if (split > 1) {
#pragma unroll
                    for (int j = i; j < i + 16; ++j)
                        part_sums[(warp / 4 * S::half + j) * kCols + warp % 4 * 32 + column_of(lane)] = acc[j];
                } else {
                    out.put16(row0 + i, col, [&](int j) { return acc[i + j]; });
                }
            }
        }
    } else if (warp < 12) {
        fewer_registers<S::for_copies>();
        if (warp == 8) {  // dY as it is
            if (SRC == kDirect && elect_one()) {
                Ring<S::stages> at;
                for (int t = first; t < tiles && !*failed; t += stride) {
                    const int n0 = t / p.k_tiles * NT + half * S::half;
                    for (int64_t st = s_first; st < s_last; ++st, at.next()) {
                        if (!bar_wait(empty(at.s), at.parity ^ 1, failed)) break;
                        if (half == 0) bar_expect(full(at.s), 2 * S::y_bytes);
                        const uint32_t to = ring + at.s * S::operands + S::x_bytes;
                        for (int g = 0; g < S::half / 64; ++g)
                            tma_load_2d_at(to + g * (kTokens * 128), &y_map, n0 + g * 64, static_cast<int>(st) * kTokens,
                                           full(at.s), lead);
                    }
                }
            }
            __syncwarp();
        } else if (warp == 10) {  // X's codes and scales
            Ring<S::raw_stages> at;
            for (int t = first; t < tiles; t += stride) {
                const int k0 = t % p.k_tiles * (2 * kCols) + half * kCols;
                // 4 scales of a token; zeros past the last token, and past X's columns
                const uint8_t *src = p.scales + k0 / 32 + (s_first * kTokens + lane) * p.pitch;
                const bool cols = k0 / 32 < p.pitch;
                for (int64_t st = s_first; st < s_last; ++st, at.next()) {
                    if (!__all_sync(~0u, bar_wait(taken(at.s), at.parity ^ 1, failed))) break;
                    const uint32_t codes = raws + at.s * S::raw, sc = codes + kCols * kTokens;
                    if (lane == 0) {
                        bar_expect(landed(at.s), kCols * kTokens);
                        tma_load_2d(codes, &x_map, k0, static_cast<int>(st) * kTokens, landed(at.s));
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const bool in = cols && st * kTokens + lane + 32 * h < p.m;
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(sc + 4 * (lane + 32 * h)),
                                     "l"(in ? src + 32 * h * p.pitch : p.scales), "r"(in ? 4 : 0)
                                     : "memory");
                    }
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(landed(at.s)) : "memory");
                    src += kTokens * p.pitch;
                }
                if (*failed) break;
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
        } else if (warp == 9) {  // products, of both blocks
            if (half == 0 && elect_one()) {
                const uint32_t both = 3u << rank;
                Ring<S::stages> at;
                Ring<2> sum;
                for (int t = first; t < tiles && !*failed; t += stride) {
                    int in_sum = 0;  // stages
                    for (int64_t st = s_first; st < s_last; ++st, at.next()) {
                        if (in_sum == 0 && !bar_wait(sum_empty(sum.s), sum.parity ^ 1, failed)) break;
                        if (!bar_wait(full(at.s), at.parity, failed)) break;
                        fence_after();
                        const uint32_t d = tmem + sum.s * NT, from = ring + at.s * S::operands;
                        // 64 columns to a group of kTokens rows of 128 bytes
                        const uint64_t dx = operand_desc(from, kTokens * 128, 1024);
#pragma unroll
                        for (int h = 0; h < S::parts; ++h) {
                            const uint64_t dy = operand_desc(from + S::x_bytes + h * S::y_part, kTokens * 128, 1024);
#pragma unroll
                            for (int q = 0; q < kTokens / 16; ++q)
                                mma_bf16_pair(d, dx + 128 * q, dy + 128 * q, idesc_bf16_pair(NT),
                                              in_sum > 0 || h > 0 || q > 0);
                        }
                        mma_commit_pair(empty(at.s), both);
                        if (++in_sum == S::chunk || st == s_last - 1) {
                            mma_commit_pair(sum_full(sum.s), both);
                            sum.next();
                            in_sum = 0;
                        }
                    }
                }
            }
            __syncwarp();
        }
    } else {  // to bf16
        if constexpr (S::for_converters < S::at_launch) fewer_registers<S::for_converters>();
        using Y = std::conditional_t<SRC == kF32, float, __nv_bfloat16>;
        constexpr int kConv = S::converters * 32;
        constexpr int kPieces = S::half / 8, kTasks = SRC == kDirect ? 1 : kTokens * kPieces / kConv;
        const Y *const dy = static_cast<const Y *>(p.dy);
        const int id = threadIdx.x % kConv, set = threadIdx.x / kConv - 3;
        // 16 codes of a token to a thread, four times: two pieces of 8 codes, 16 bytes of bf16.  Which piece comes
        // first goes by the columns' group and the token, so that the loads of 16 lanes and the stores of 8 fill
        // all banks.
        const int c = id % 8, row = id / 8;
        const int x = (c / 4) ^ (row & 1);
        const uint32_t load_1 = id * 16 + 8 * x, load_2 = load_1 ^ 8;
        const uint32_t store_1 = (c / 4) * (kTokens * 128) + row * 128 + (((2 * (c % 4) + x) ^ (row & 7)) << 4),
                       store_2 = store_1 ^ 16;
        Ring<S::stages> at;
        Ring<S::raw_stages> from;
        int turn = set;  // stages until this set's next one
        for (int t = first; t < tiles; t += stride) {
            const int64_t n0 = int64_t(t / p.k_tiles) * NT + half * S::half;
            for (int64_t st = s_first; st < s_last; ++st, at.next(), from.next()) {
                if (turn-- != 0) continue;
                turn = S::sets - 1;
                const uint32_t to = ring + at.s * S::operands;
                [[maybe_unused]] float y[kTasks][8];
                if constexpr (SRC != kDirect) {  // 8 columns of a token to a thread; under way before the waits
#pragma unroll
                    for (int j = 0; j < kTasks; ++j) {
                        const int64_t tok = st * kTokens + id / kPieces + j * (kConv / kPieces);
                        load8(dy + (tok < p.m ? tok : 0) * p.ldy, n0 + id % kPieces * 8, tok < p.m ? p.n : 0, p.vec, y[j]);
                    }
                }
                if (!__all_sync(~0u, bar_wait(landed(from.s), from.parity, failed))) goto out;
                const uint32_t codes = raws + from.s * S::raw, sc = codes + kCols * kTokens;
                uint2 w[4][2];
                uint32_t s4[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    w[j][0] = load8b(codes + load_1 + j * (16 * kCols));
                    w[j][1] = load8b(codes + load_2 + j * (16 * kCols));
                    s4[j] = load_byte(sc + row * 4 + c / 2 + j * 64);
                }
                if (!__all_sync(~0u, bar_wait(empty(at.s), at.parity ^ 1, failed))) goto out;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const __nv_bfloat162 unit = bf16_unit(s4[j]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t v[4];
                        codes_to_bf16(w[j][h].x, unit, v[0], v[1]);
                        codes_to_bf16(w[j][h].y, unit, v[2], v[3]);
                        store16(to + (h ? store_2 : store_1) + j * (16 * 128), v[0], v[1], v[2], v[3]);
                    }
                }
                if constexpr (SRC != kDirect) {
#pragma unroll
                    for (int j = 0; j < kTasks; ++j) {
                        const int p8 = id % kPieces, tok = id / kPieces + j * (kConv / kPieces);
                        const uint32_t line = to + S::x_bytes + (p8 / 8) * (kTokens * 128) + tok * 128 +
                                              (((p8 % 8) ^ (tok & 7)) << 4);
#pragma unroll
                        for (int h = 0; h < S::parts; ++h) {
                            const uint32_t a = take_part(y[j][0], y[j][1]), b = take_part(y[j][2], y[j][3]),
                                           d = take_part(y[j][4], y[j][5]), e = take_part(y[j][6], y[j][7]);
                            store16(line + h * S::y_part, a, b, d, e);
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    bar_arrive_at(full(at.s), lead);
                    bar_arrive(taken(from.s));
                }
            }
        }
    out:;
    }

    if (*failed) let_copies_land();
    if (split > 1)  // one tile to a cluster
        join_split(out, ring, half, 2, part, split, int64_t(first / p.k_tiles) * NT,
                   int64_t(first % p.k_tiles) * (2 * kCols) + half * kCols, NT);
    fence_before();
    __syncthreads();
    cluster_sync();  // neither block leaves, or frees tensor memory, while the other's products run
    if (warp == 9) {
        fence_after();
        tmem_free_pair(tmem, S::cols);
    }
    if (threadIdx.x == 0 && *failed) atomicAdd(&g_failed, 1u);
}

template <int NT, int SRC, typename T>
cudaError_t launch(const costa_mx_dense &dY, const costa_mx_matrix &Q, float alpha, float beta, const costa_mx_dense &dW,
                   int sms, cudaStream_t s) {
    using S = Shape<NT, SRC>;
    CUtensorMap x_map, y_map;
    cudaError_t e = mx_byte_map(&x_map, Q.codes, 32 * mx_blocks(Q.cols), Q.rows, Q.ld, kTokens, false);
    y_map = x_map;
    if (e == cudaSuccess && SRC == kDirect) e = mx_bf16_map(&y_map, dY.ptr, dY.cols, dY.rows, dY.ld, kTokens);
    if (e != cudaSuccess) return e;
    Params p;
    p.scales = static_cast<const uint8_t *>(Q.scales);
    p.pitch = mx_scale_pitch(Q.cols);
    p.dy = dY.ptr;
    p.ldy = dY.ld;
    const int64_t es = SRC == kF32 ? 4 : 2;
    p.vec = reinterpret_cast<uint64_t>(dY.ptr) % 16 == 0 && dY.ld * es % 16 == 0;
    p.m = dY.rows;
    p.n = dY.cols;
    p.n_tiles = static_cast<int>(mx_ceil(dY.cols, NT));
    p.k_tiles = static_cast<int>(mx_ceil(Q.cols, 2 * kCols));
    const Output<T> out{static_cast<T *>(dW.ptr), dW.ld, dW.rows, dW.cols, alpha, beta};
    const int64_t tiles = int64_t(p.n_tiles) * p.k_tiles, stages = mx_ceil(p.m, kTokens);
    if (tiles > INT32_MAX / 2) return cudaErrorInvalidValue;
    const int64_t pairs = sms / 2;
    int split = 1;
    while (split < 4 && tiles * split * 2 <= pairs && stages >= 4 * split) split *= 2;
    return mx_launch(grad_kernel<NT, SRC, T>, 2 * (split > 1 ? tiles * split : std::min(tiles, pairs)), S::warps * 32,
                     S::smem, 2 * split, s, x_map, y_map, p, out, split);
}

template <typename T>
cudaError_t by_source(const costa_mx_dense &dY, const costa_mx_matrix &Q, float alpha, float beta,
                      const costa_mx_dense &dW, int sms, cudaStream_t s) {
    if (dY.type == COSTA_MX_F32) return launch<128, kF32, T>(dY, Q, alpha, beta, dW, sms, s);
    if (reinterpret_cast<uint64_t>(dY.ptr) % 16 || dY.ld % 8) return launch<128, kBf16, T>(dY, Q, alpha, beta, dW, sms, s);
    if (mx_ceil(dY.cols, 256) * mx_ceil(Q.cols, 2 * kCols) < sms / 2)
        return launch<128, kDirect, T>(dY, Q, alpha, beta, dW, sms, s);
    return launch<256, kDirect, T>(dY, Q, alpha, beta, dW, sms, s);
}

}  // namespace
}  // namespace mx

cudaError_t launch_mx_weight_grad(const costa_mx_dense &dY, const costa_mx_matrix &Q, float alpha, float beta,
                                  const costa_mx_dense &dW, cudaStream_t s) {
    if (dY.rows == 0) return launch_mx_scale(beta, dW, s);
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    return dW.type == COSTA_MX_F32 ? mx::by_source<float>(dY, Q, alpha, beta, dW, sms, s)
                                   : mx::by_source<__nv_bfloat16>(dY, Q, alpha, beta, dW, sms, s);
}

cudaError_t mx_grad_failures(unsigned *count) {
    return cudaMemcpyFromSymbol(count, mx::g_failed, sizeof *count);
}

}  // namespace costa
