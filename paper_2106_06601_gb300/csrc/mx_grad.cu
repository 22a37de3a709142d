// dW = alpha dY^T X + beta dW with X (m x k) from its 8-bit checkpoint and dY
// (m x n) in bf16 or f32, on the tensor cores' bf16 products.
//
// A checkpoint's value is an integer below 2^7 times a power of two: exact in
// bf16.  An f32 gradient is cut into three bf16 parts of 8 bits each (by
// truncation, so no part overflows), all of which are multiplied.  So every
// product is that of the values, and only the sums round.
//
// A pair of thread blocks takes a tile of 256 columns of X (the lanes of tensor
// memory, 128 in each block: neighbouring elements of a row of dW) and NT
// columns of dY, half of which each block holds, and runs over the tokens in
// stages of 64.  Warps load X's codes and turn them into bf16 in the tensor
// cores' layout.  dY comes by bulk copies as it is where it is bf16 with 16-byte
// aligned rows (kDirect); else more warps load, cut and store it.
//
// The tensor cores' sums truncate: of each term what lies below some 2^-25 of the
// largest.  For values of one sign that is about 1.3e-8 of the sum for each product
// over 16 tokens (1.3e-5 after 1024).  So a sum takes kProducts of them at most, in
// one of two places in tensor memory; eight warps add each to sums in registers,
// rounded to nearest, while the next one builds.  An f32 gradient's second and third
// parts have a sum of their own: beside the first parts' their 16 bits were cut off,
// term by term (errors 2.2e-6 of the sum at any number of tokens, now 4e-8; 777 x
// 1000 x 1531 15.2 -> 15.6 us, 4096 x 8192 x 4096 632 -> 622).  Values of one sign
// whose magnitudes spread over 2^8 and 2^24: 4e-7 and 1.8e-6 in bf16, 1.3e-7 and
// 8e-7 in f32.
//
// GB300: 4096 x 8192 x 4096 bf16 190 us (1.45 PFLOP/s, 75% of the library
// products' rate), 16384 tokens 803 us (1.37); the same with an odd stride 476
// us, f32 622 us (three products each: 1.33 PFLOP/s of them), f32 with an odd
// stride 694 us.  What bounds it: the conversions' logical operations, at half
// rate (ALU pipe 56% busy), shared memory, which the operands and the converted
// codes share (56%; f32 59%), and the issue slots (58%; 62%): 24 or 28 warps hide
// no more of their latency, and the tensor pipe is 64% (56%) busy.  Spilt, around
// the roles' loops: 40 to 76 bytes a thread (f32 92).
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
constexpr int kMaxSplit = 4;

__device__ unsigned g_failed;

struct Params {
    const uint8_t *codes, *scales;
    int64_t ldx, pitch;  // bytes of their rows
    int64_t width;       // bytes of a row of codes that are there
    const void *dy;      // not kDirect
    int64_t ldy;
    int64_t m, n;
    int n_tiles, k_tiles;
};

enum Source { kDirect = 0, kBf16 = 1, kF32 = 3 };  // of dY; the number of parts if not direct

template <int NT, int SRC> struct Shape {
    static constexpr bool direct = SRC == kDirect;
    static constexpr int parts = SRC == kF32 ? 3 : 1;
    static constexpr int half = NT / 2;  // columns of dY in a block
    static constexpr int x_bytes = kCols * kTokens * 2, y_part = half * kTokens * 2, y_bytes = parts * y_part;
    static constexpr int operands = x_bytes + y_bytes;  // of a stage, in the tensor cores' layout
    // More stages would leave the L1 cache too little for what the converters load (16384 x 8192 x 4096 bf16, 4, 5, 6,
    // 7 stages: 870, 831, 849, 1004 us; m = 4096 f32, 3, 4, 5: 639, 681, 857; unaligned bf16, 4, 5, 8: 546, 529, 582).
    static constexpr int stages = SRC == kF32 ? 3 : 5;
    static constexpr int smem = stages * operands + 1024;
    // Warpgroups: two for the sums; one for dY's copies and the products; sets of converters, which take turns.
    // (Unaligned bf16, 4096 x 8192 x 4096, 2 and 2, 2 and 3, 3 and 2 sets for X and dY: 508, 519, 469 us.)
    static constexpr int x_sets = SRC == kF32 ? 2 : 3, y_sets = direct ? 0 : 2, groups = 3 + x_sets + y_sets;
    // Registers of a thread: at launch, and then of each.  (Nothing here may call a function that is not inlined: its
    // code would use registers that a warp has given up.)
    static constexpr int at_launch = direct ? 80 : SRC == kF32 ? 72 : 64;
    static constexpr int for_sums = direct ? 168 : 104, for_copies = 24, for_x = 40, for_y = SRC == kF32 ? 96 : 72;
    static_assert(2 * for_sums + for_copies + x_sets * for_x + y_sets * for_y <= groups * at_launch, "registers");
    static_assert(groups * 128 * at_launch <= 65536, "registers");
    // f32: the first parts' products to one sum, the others' to another.
    static constexpr int sums = SRC == kF32 ? 2 : 1, cols = 2 * NT * sums;
    static constexpr int chunk = kProducts / (std::max(1, parts - 1) * (kTokens / 16));  // stages to a sum
    static_assert(smem <= 226 * 1024 && kCols * NT * 4 <= stages * operands, "shared memory");
};

// Codes as bf16 pairs, times the block's unit 2^(s - 133), which is subnormal
// below 2^-126 and NaN for scale byte 255.  With 7 low bits r and sign bit s a
// code is r - 128 s; as bf16, 0x4300 | r is 128 + r, and 0x4300 | 128 s is 128 or
// 256.  Two logical operations and two in bf16 for a pair keep both of their
// pipes, of half rate each, equally busy; floating ones alone (relu(.) / 2 -
// relu(-.) of one fused product each) were slower, 1055 us for 808.
struct Decoder {
    __nv_bfloat162 unit;
    __device__ explicit Decoder(uint32_t s) {
        const uint32_t normal = s == 255 ? 0x7fff7fffu : s * 0x00800080u - 0x03000300u;
        unit = halves(s <= 6 ? 0x10001u << s : normal);
    }
    __device__ uint32_t operator()(uint32_t two) const {  // a code in the low byte of each half; the others' bits may be set
        const uint32_t a = (two & 0x007f007fu) | 0x43004300u, b = (two & 0x00800080u) | 0x43004300u;
        return word(__hmul2(__hsub2(halves(a), halves(b)), unit));
    }
};
// Eight codes, 16 bytes.  The pairs of a word are elements 0, 2 and 1, 3, which
// saves permutations: positions 1 and 2 of each four columns of a tile are
// exchanged until the sums are written out.
__device__ __forceinline__ uint4 decode(const Decoder &d, uint32_t x, uint32_t y) {
    return make_uint4(d(x), d(x >> 8), d(y), d(y >> 8));
}
// The column in a tile whose sum a lane has.
__device__ __forceinline__ int column_of(int lane) { return (lane & ~3) | (lane & 1) << 1 | (lane >> 1 & 1); }

__device__ __forceinline__ void store16(uint32_t at, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// The upper halves of two words: the first 8 bits of two f32 numbers as a bf16 pair.
__device__ __forceinline__ uint32_t upper(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x7632); }
__device__ __forceinline__ void take_upper(uint32_t &a) {  // off a
    a = __float_as_uint(__uint_as_float(a) - __uint_as_float(a & 0xffff0000u));
}

template <int NT, int SRC, typename T>
__global__ void __launch_bounds__(Shape<NT, SRC>::groups * 128, 1)
    grad_kernel(const __grid_constant__ CUtensorMap y_map, const Params p, const Output<T> out, const int split) {
    using S = Shape<NT, SRC>;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::stages + 4];
    __shared__ uint32_t tmem_slot;
    __shared__ uint32_t failed_word;
    volatile uint32_t *failed = &failed_word;
    const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u;
    float *const part_sums = reinterpret_cast<float *>(raw + (ring - smem_addr(raw)));
    const uint32_t bar0 = smem_addr(bars), bar1 = bar0 + 16 * S::stages;
    auto full = [&](int s) { return bar0 + 16 * s; };       // (first block's) both blocks' operands
    auto empty = [&](int s) { return bar0 + 16 * s + 8; };  // products have read the stage
    auto sum_full = [&](int i) { return bar1 + 8 * i; };
    auto sum_empty = [&](int i) { return bar1 + 16 + 8 * i; };  // (first block's)
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rank = static_cast<int>(cluster_rank()), half = rank & 1, lead = rank & ~1, part = rank >> 1;

    if (threadIdx.x == 0) {
        failed_word = 0;
        for (int s = 0; s < S::stages; ++s) {
            bar_init(full(s), S::direct ? 1 + 2 * 4 : 2 * 8);  // converters' warps of both blocks; the copies' bytes
            bar_init(empty(s), 1);
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
    let_next_start();
    after_previous();

    // This block's share of the tokens, in stages; and its tiles.
    const int64_t stages_m = (p.m + kTokens - 1) / kTokens;
    const int s_first = static_cast<int>(stages_m * part / split), s_last = static_cast<int>(stages_m * (part + 1) / split);
    const int tiles = p.n_tiles * p.k_tiles, first = blockIdx.x / (2 * split), stride = gridDim.x / (2 * split);

    // A role's way through the stages of all tiles: every `steps`-th, from its own first.
    Ring<S::stages> at;
    int t = first, st = s_first, n0 = t / p.k_tiles * NT + half * S::half, k0 = t % p.k_tiles * (2 * kCols) + half * kCols;
    auto advance = [&](int steps) {  // whether it came to another tile
        at.next(steps);
        st += steps;
        if (st < s_last) return false;
        do {
            st -= s_last - s_first;
            t += stride;
        } while (st >= s_last && t < tiles);
        n0 = t / p.k_tiles * NT + half * S::half;
        k0 = t % p.k_tiles * (2 * kCols) + half * kCols;
        return true;
    };
    auto stage_done = [&](int s) {  // this warp's part of stage s is in shared memory
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) bar_arrive_at(full(s), lead);
    };

    // Each role takes its registers first, so that its code is laid out for them.
    if (warp < 8) {  // sums; warp w: lanes of quarter w % 4, half of the columns
        more_registers<S::for_sums>();
        const int chunks = (s_last - s_first + S::chunk - 1) / S::chunk;
        const uint32_t from = tmem + (uint32_t(warp % 4 * 32) << 16) + warp / 4 * S::half;
        Ring<2> sum;
        for (; t < tiles; t += stride) {
            float acc[S::half];
#pragma unroll
            for (int i = 0; i < S::half; ++i) acc[i] = 0.0f;
            bool ok = true;
            for (int c = 0; c < chunks && ok; ++c, sum.next()) {
                ok = __all_sync(~0u, bar_wait(sum_full(sum.s), sum.parity, failed));
                fence_after();
                const uint32_t place = from + S::sums * sum.s * NT;
#pragma unroll
                for (int g = 0; g < S::half / 16; ++g) {
                    uint32_t r[16];
                    if constexpr (S::sums == 2) {
                        uint32_t q[16];
                        tmem_ld16(place + NT + g * 16, q);
                        tmem_ld16(place + g * 16, r);
                        tmem_wait_ld(q);
                        tmem_wait_ld(r);
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[g * 16 + i] += __uint_as_float(r[i]) + __uint_as_float(q[i]);
                    } else {
                        tmem_ld16(place + g * 16, r);
                        tmem_wait_ld(r);
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[g * 16 + i] += __uint_as_float(r[i]);
                    }
                }
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_at(sum_empty(sum.s), lead);
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
        if (split > 1) {  // one tile to a cluster
            __syncwarp();
            cluster_sync();  // (the other warps do so below)
            join_split<kMaxSplit>(out, ring, half, 2, part, split, threadIdx.x, 256, int64_t(first / p.k_tiles) * NT,
                                  int64_t(first % p.k_tiles) * (2 * kCols) + half * kCols, NT);
        }
    } else if (warp < 12) {
        fewer_registers<S::for_copies>();
        if (warp == 8) {  // dY as it is
            if (S::direct && elect_one()) {
                for (; t < tiles && !*failed; advance(1)) {
                    if (!bar_wait(empty(at.s), at.parity ^ 1, failed)) break;
                    if (half == 0) bar_expect(full(at.s), 2 * S::y_bytes);
                    const uint32_t to = ring + at.s * S::operands + S::x_bytes;
                    for (int g = 0; g < S::half / 64; ++g)
                        tma_load_2d_at(to + g * (kTokens * 128), &y_map, n0 + g * 64, st * kTokens, full(at.s), lead);
                }
            }
            __syncwarp();
        } else if (warp == 9) {  // products, of both blocks
            if (half == 0 && elect_one()) {
                const uint32_t both = 3u << rank;
                Ring<2> sum;
                for (; t < tiles && !*failed; t += stride) {
                    int in_sum = 0;  // stages
                    for (st = s_first; st < s_last; ++st, at.next()) {
                        if (in_sum == 0 && !bar_wait(sum_empty(sum.s), sum.parity ^ 1, failed)) break;
                        if (!bar_wait(full(at.s), at.parity, failed)) break;
                        fence_after();
                        const uint32_t d = tmem + S::sums * sum.s * NT, from = ring + at.s * S::operands;
                        // 64 columns to a group of kTokens rows of 128 bytes
                        const uint64_t dx = operand_desc(from, kTokens * 128, 1024);
#pragma unroll
                        for (int h = 0; h < S::parts; ++h) {
                            const uint64_t dy = operand_desc(from + S::x_bytes + h * S::y_part, kTokens * 128, 1024);
#pragma unroll
                            for (int q = 0; q < kTokens / 16; ++q)
                                mma_bf16_pair(d + (h > 0 ? NT : 0), dx + 128 * q, dy + 128 * q, idesc_bf16_pair(NT),
                                              in_sum > 0 || h > 1 || q > 0);
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
    } else if (warp < 12 + 4 * S::x_sets) {  // X to bf16: 16 codes of a token to a thread, four times
        fewer_registers<S::for_x>();
        // Lanes 0 to 3 of 8 take the first 64 columns of a token, lanes 4 to 7 the other 64 of its neighbour, whose
        // swizzle differs by one piece: so the stores of 8 lanes fill all banks.
        const int id = threadIdx.x % 128, c = id % 8, row = (id / 8) ^ (c / 4);
        const uint32_t store = (c / 4) * (kTokens * 128) + row * 128 + (((2 * (c % 4)) ^ (row & 7)) << 4);
        const uint8_t *code, *scale;  // this thread's first of a stage
        auto seek = [&] {
            const int64_t tok = int64_t(st) * kTokens + row, col = k0 + c * 16;
            code = p.codes + tok * p.ldx + col;
            scale = p.scales + tok * p.pitch + col / 32;
        };
        const int64_t code_step = S::x_sets * kTokens * p.ldx, scale_step = S::x_sets * kTokens * p.pitch;
        uint4 w[4];
        uint32_t s4[4];
        auto load = [&] {  // a turn's codes and scales, at the end of the turn before it
            const int left = t < tiles && k0 + c * 16 < p.width
                                 ? static_cast<int>(min(p.m - int64_t(st) * kTokens, int64_t(kTokens))) - row : 0;
            if (left > 48) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    w[j] = *reinterpret_cast<const uint4 *>(code + j * (16 * p.ldx));
                    s4[j] = scale[j * (16 * p.pitch)];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    w[j] = make_uint4(0, 0, 0, 0);
                    s4[j] = 0;
                    if (left > 16 * j) {
                        w[j] = *reinterpret_cast<const uint4 *>(code + j * (16 * p.ldx));
                        s4[j] = scale[j * (16 * p.pitch)];
                    }
                }
            }
        };
        const int set = warp / 4 - 3;
        if (set > 0) advance(set);
        seek();
        load();
        while (t < tiles) {
            if (!__all_sync(~0u, bar_wait(empty(at.s), at.parity ^ 1, failed))) break;
            const uint32_t to = ring + at.s * S::operands + store;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Decoder d(s4[j]);
                const uint32_t piece = to + j * (16 * 128);
                store16(piece, decode(d, w[j].x, w[j].y));
                store16(piece ^ 16, decode(d, w[j].z, w[j].w));
            }
            stage_done(at.s);
            if (advance(S::x_sets)) {
                seek();
            } else {
                code += code_step;
                scale += scale_step;
            }
            load();
        }
    } else if constexpr (!S::direct) {  // dY to bf16 parts: 8 columns of a token to a thread, some times
        more_registers<S::for_y>();
        using Y = std::conditional_t<SRC == kF32, float, __nv_bfloat16>;
        const Y *const dy = static_cast<const Y *>(p.dy);
        // Of a stage's 64 tokens a warp takes those of two remainders by 8: their rows are all off 16 bytes by the same.
        // Task j: tokens token(j), 8 lanes to each.
        constexpr int kTasks = 4;
        static_assert(S::half == 64 && kTokens == 64, "8 lanes to a token");
        const int c = lane % 8, rest = warp % 4 * 2;
        auto token = [&](int j) { return rest + j / 2 + 8 * (lane / 8) + 32 * (j % 2); };
        uint32_t off[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
            off[h] = __shfl_sync(~0u, Unaligned<Y, 8>::offset(dy + (rest + h) * p.ldy), 0);
        Unaligned<Y, 8> y[kTasks];
        const Y *first_y;  // this thread's columns of a stage's first token
        int count;         // how many there are
        auto seek = [&] {
            first_y = dy + int64_t(st) * kTokens * p.ldy + n0 + c * 8;
            count = count_from(n0 + c * 8, p.n, 8);
        };
        const int64_t step = S::y_sets * kTokens * p.ldy;
        auto load = [&] {
            const int left = t < tiles ? static_cast<int>(min(p.m - int64_t(st) * kTokens, int64_t(kTokens))) : 0;
            if (left == kTokens && count == 8) {
#pragma unroll
                for (int j = 0; j < kTasks; ++j) y[j].load_whole(first_y + token(j) * p.ldy, off[j / 2]);
            } else {
#pragma unroll
                for (int j = 0; j < kTasks; ++j)
                    y[j].load(first_y + token(j) * p.ldy, off[j / 2], token(j) < left ? count : 0);
            }
        };
        const int set = warp / 4 - 3 - S::x_sets;
        if (set > 0) advance(set);
        seek();
        load();
        while (t < tiles) {
            if (!__all_sync(~0u, bar_wait(empty(at.s), at.parity ^ 1, failed))) break;
            const uint32_t to = ring + at.s * S::operands + S::x_bytes;
#pragma unroll
            for (int j = 0; j < kTasks; ++j) {
                uint32_t w[Unaligned<Y, 8>::kWords];
                y[j].place(off[j / 2], count, w);  // (of a token past the last: zeros)
                const uint32_t line = to + token(j) * 128 + ((c ^ (rest + j / 2)) << 4);
                if constexpr (SRC == kF32) {
#pragma unroll
                    for (int h = 0; h < S::parts; ++h) {
                        store16(line + h * S::y_part,
                                make_uint4(upper(w[0], w[1]), upper(w[2], w[3]), upper(w[4], w[5]), upper(w[6], w[7])));
#pragma unroll
                        for (int i = 0; i < 8 && h < S::parts - 1; ++i) take_upper(w[i]);
                    }
                } else {
                    store16(line, make_uint4(w[0], w[1], w[2], w[3]));
                }
            }
            stage_done(at.s);
            if (advance(S::y_sets))
                seek();
            else
                first_y += step;
            load();
        }
    }
    __syncwarp();

    if (*failed) let_copies_land();
    if (split > 1 && warp >= 8) cluster_sync();
    fence_before();
    __syncthreads();
    cluster_sync();  // neither block leaves, or frees tensor memory, while the other's products run
    if (warp == 9) {
        fence_after();
        tmem_free_pair(tmem, S::cols);
    }
    if (threadIdx.x == 0 && *failed) atomicAdd(&g_failed, 1u);
}

// How a call is laid out: columns of dY in a tile, and the parts of its tokens.
struct Layout {
    int nt, split;
    double ns;
};

// The shortest by what was measured with aligned bf16 dY: a stage of a pair takes
// 375 ns with 128 columns of dY and 450 with 256, joining the parts some 3 and 6
// us, and tiles beyond what the device runs at a time take another round.  (With
// 128 columns of other dY a stage takes about 540, and 700 in f32; they are laid
// out by the same figures, which weigh parts of the tokens a little too low.)  (GPU us with the
// quantisation, 128 and 256 columns: 4096 x 2048 x 2048 55, 36; 4096 x 1024 x
// 4096 60, 41; 512 x 4096 x 4096 32, 26; 4096 x 1024 x 1024 in two parts 21,
// in four 32; 4096 x 512 x 512 in four 14, 17.)
Layout choose(int64_t n, int64_t k, int64_t m, bool wide) {
    Layout best{128, 1, -1.0};
    for (int nt = 128; nt <= (wide ? 256 : 128); nt *= 2)
        for (int split = 1; split <= kMaxSplit; split *= 2) {
            const int64_t stages = mx_ceil(m, kTokens), tiles = mx_ceil(n, nt) * mx_ceil(k, 2 * kCols);
            if (split > 1 && stages < 2 * split) break;
            const double rounds = static_cast<double>(mx_ceil(tiles, mx_clusters(2 * split, 1)));
            // whole rounds where parts are joined; else pairs go on to the next tile
            const double ns = rounds * (mx_ceil(stages, split) * (nt == 128 ? 375.0 : 450.0) + (split > 1 ? nt * 24.0 : 0.0));
            if (best.ns < 0 || ns < best.ns) best = {nt, split, ns};
        }
    return best;
}

template <int NT, int SRC, typename T>
cudaError_t launch(const costa_mx_dense &dY, const costa_mx_matrix &Q, float alpha, float beta, const costa_mx_dense &dW,
                   int split, cudaStream_t s) {
    using S = Shape<NT, SRC>;
    CUtensorMap y_map{};
    if (SRC == kDirect) {
        const cudaError_t e = mx_bf16_map(&y_map, dY.ptr, dY.cols, dY.rows, dY.ld, kTokens);
        if (e != cudaSuccess) return e;
    }
    Params p;
    p.codes = static_cast<const uint8_t *>(Q.codes);
    p.scales = static_cast<const uint8_t *>(Q.scales);
    p.ldx = Q.ld;
    p.pitch = mx_scale_pitch(Q.cols);
    p.width = 32 * mx_blocks(Q.cols);
    p.dy = dY.ptr;
    p.ldy = dY.ld;
    p.m = dY.rows;
    p.n = dY.cols;
    p.n_tiles = static_cast<int>(mx_ceil(dY.cols, NT));
    p.k_tiles = static_cast<int>(mx_ceil(Q.cols, 2 * kCols));
    const Output<T> out{static_cast<T *>(dW.ptr), dW.ld, dW.rows, dW.cols, alpha, beta};
    const int64_t tiles = int64_t(p.n_tiles) * p.k_tiles;
    if (tiles > INT32_MAX / 16) return cudaErrorInvalidValue;
    const int64_t pairs = split > 1 ? tiles * split : std::min<int64_t>(tiles, mx_clusters(2, 1));
    return mx_launch(grad_kernel<NT, SRC, T>, 2 * pairs, S::groups * 128, S::smem, 2 * split, s, y_map, p, out, split);
}

template <typename T>
cudaError_t by_source(const costa_mx_dense &dY, const costa_mx_matrix &Q, float alpha, float beta,
                      const costa_mx_dense &dW, cudaStream_t s) {
    const bool f32 = dY.type == COSTA_MX_F32;
    const bool direct = !f32 && reinterpret_cast<uint64_t>(dY.ptr) % 16 == 0 && dY.ld % 8 == 0;
    const Layout l = choose(dY.cols, Q.cols, dY.rows, direct);
    if (f32) return launch<128, kF32, T>(dY, Q, alpha, beta, dW, l.split, s);
    if (!direct) return launch<128, kBf16, T>(dY, Q, alpha, beta, dW, l.split, s);
    if (l.nt == 128) return launch<128, kDirect, T>(dY, Q, alpha, beta, dW, l.split, s);
    return launch<256, kDirect, T>(dY, Q, alpha, beta, dW, l.split, s);
}

}  // namespace
}  // namespace mx

cudaError_t launch_mx_weight_grad(const costa_mx_dense &dY, const costa_mx_matrix &Q, float alpha, float beta,
                                  const costa_mx_dense &dW, cudaStream_t s) {
    if (dY.rows == 0) return launch_mx_scale(beta, dW, s);
    return dW.type == COSTA_MX_F32 ? mx::by_source<float>(dY, Q, alpha, beta, dW, s)
                                   : mx::by_source<__nv_bfloat16>(dY, Q, alpha, beta, dW, s);
}

cudaError_t mx_grad_failures(unsigned *count) {
    return cudaMemcpyFromSymbol(count, mx::g_failed, sizeof *count);
}

}  // namespace costa
