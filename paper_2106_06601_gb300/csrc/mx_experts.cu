// Tokens sorted by expert, their rows to their places and back, and the gradients.
//
//   place(t, s): the place of token t's s-th expert among all pairs sorted by expert (stably)
//   dispatch    X'[place(t, s)] = X[t]
//   combine     Y[t] = sum_s w_ts Z[place(t, s)];  the same without weights is the gradient of dispatch
//   backward    dZ[place(t, s)] = w_ts dY[t],  dw_ts = <Z[place(t, s)], dY[t]>
//
// The copies read and write each row once, eight elements to a lane; memory bounds
// them.  GB300, 16384 x 4096 bf16 of eight experts: dispatch 176 us, combine 168 us
// (7.2 TB/s), its gradients 333 us (6.9 TB/s), the sort 14 us.  As codes to four
// places 4096 x 4096 take 31 us (floor 20), 50 instructions an element in 77% of the
// issue slots.  The gradients of combine as codes are made anew for each place, as each
// has a weight of its own: 302 us for the batch above (floor 62), with those of the
// weights 402 (floor 220).
#include <algorithm>
#include <type_traits>

#include "costa_internal.h"
#include "mx_rows.cuh"
#include "mx_tc.cuh"

namespace costa {
namespace mx {
namespace {

// ---- the sort ----
//
// A stable counting sort: a warp counts the experts of its pairs; the counts are
// added up over the warps before it, the blocks before its block and the experts
// before; then the warp goes over its pairs again, 32 neighbouring ones at a time,
// and hands out places.  Up to 8192 pairs are one block's, more those of a cluster
// of eight.

constexpr int kSortBlocks = 8, kSortThreads = 1024, kAhead = 16;

struct Sort {
    const int32_t *experts;
    int64_t ld;
    int64_t pairs;
    int top, n_experts, align;
    int32_t *place;
    int64_t ld_place;
    int32_t *starts, *counts;
    int64_t per_warp;  // pairs, a multiple of 32
};

__device__ __forceinline__ int cluster_load_int(const int *at, uint32_t rank) {
    uint32_t a;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(at)), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

template <int BLOCKS> __global__ void __launch_bounds__(kSortThreads) sort_kernel(const Sort p) {
    extern __shared__ int counted[];  // [warps][experts], then the block's totals
    __shared__ int scan[32];
    let_next_start();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32, n = p.n_experts;
    const int rank = BLOCKS > 1 ? static_cast<int>(cluster_rank()) : 0;
    int *const mine = counted + warp * n, *const totals = counted + warps * n;
    for (int i = threadIdx.x; i < warps * n; i += blockDim.x) counted[i] = 0;
    __syncthreads();
    after_previous();
    const int64_t first = (int64_t(rank) * warps + warp) * p.per_warp, last = min(p.pairs, first + p.per_warp);
    // f(expert, pair) for the pairs of this warp; expert n: none.  The experts of kAhead times 32 pairs are asked for
    // together (and stay in registers for the second time, where they are all).
    int ahead[kAhead];
    bool have = false;
    auto each = [&](auto f) {
        for (int64_t from = first; from < last; from += 32 * kAhead) {
            if (!have)
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int64_t i = from + 32 * k + lane;
                    ahead[k] = i >= last ? -1 : p.ld == p.top ? p.experts[i] : p.experts[i / p.top * p.ld + i % p.top];
                }
            have = last - first <= 32 * kAhead;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int64_t i = from + 32 * k;
                if (i >= last) break;
                f(ahead[k] >= 0 && ahead[k] < n ? ahead[k] : n, i + lane);
            }
        }
    };
    each([&](int e, int64_t) {
        if (e < n) atomicAdd(&mine[e], 1);  // (whole numbers: in any order)
    });
    __syncthreads();
    const int e = threadIdx.x;  // there are as many threads as experts at least
    int before = 0, all = 0;
    if (e < n) {
        for (int w = 0; w < warps; ++w) {
            const int here = counted[w * n + e];
            counted[w * n + e] = all;
            all += here;
        }
        totals[e] = all;
    }
    if constexpr (BLOCKS > 1) {
        cluster_sync();
        if (e < n) {
            all = 0;
            for (int b = 0; b < BLOCKS; ++b) {
                const int there = cluster_load_int(totals + e, b);
                before += b < rank ? there : 0;
                all += there;
            }
        }
        cluster_sync();  // no block leaves while another reads its totals
    }
    // The experts' first places.
    const int span = (all + p.align - 1) / p.align * p.align;
    int upto = span;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(~0u, upto, d);
        if (lane >= d) upto += v;
    }
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    for (int w = 0; w < warp; ++w) upto += scan[w];
    const int start = upto - span;
    if (e < n) {
        if (rank == 0) {
            p.starts[e] = start;
            p.counts[e] = all;
            if (e == n - 1) p.starts[n] = upto;
        }
        for (int w = 0; w < warps; ++w) counted[w * n + e] += start + before;
    }
    __syncthreads();
    const int bits = 32 - __clz(n);
    each([&](int to, int64_t i) {
        uint32_t same = ~0u;  // lanes of the same expert, from its digits (131072 pairs: 14 us; counted and handed out by match.any, 28 us)
        for (int b = 0; b < bits; ++b) {
            const uint32_t set = __ballot_sync(~0u, to >> b & 1);
            same &= to >> b & 1 ? set : ~set;
        }
        const int before = __popc(same & ((1u << lane) - 1));
        int at = -1;
        if (to < n) at = mine[to] + before;
        __syncwarp();
        if (to < n && before == 0) mine[to] = at + __popc(same);
        __syncwarp();
        if (i < last) p.place[p.ld_place == p.top ? i : i / p.top * p.ld_place + i % p.top] = at;
    });
}

// ---- rows ----

// Where a token's rows are, for up to 32 of its experts: lane s holds the s-th's place, -1 for none.
struct Places {
    const int32_t *p;
    int64_t ld, rows;  // rows: those that places may name
    int top;
    __device__ int load(int64_t token, int first) const {
        const int s = first + threadIdx.x % 32;
        const int at = s < top ? p[token * ld + s] : -1;
        return at >= 0 && at < rows ? at : -1;
    }
};

constexpr int kWarps = 8;

// A warp's part of the tokens' rows: U groups of eight to a lane.
template <int U> struct Part {
    int64_t token, first;  // first: group
    __device__ Part(int64_t per_token) {
        const int64_t id = int64_t(blockIdx.x) * kWarps + threadIdx.x / 32;
        token = id / per_token;
        first = (id - token * per_token) * (32 * U);
    }
    __device__ int64_t group(int u) const { return first + u * 32 + threadIdx.x % 32; }
    __device__ int64_t col(int u) const { return group(u) * 8; }
};

// Columns of a group of a row that begins `head` elements after a 16-byte boundary: the first group has what comes before
// the next one, the others lie on boundaries; so stores are whole, and loads of rows that lie otherwise take what is in two
// pieces.
struct Span {
    int64_t col;
    int n;
    __device__ Span(int64_t group, int head, int64_t cols)
        : col(group == 0 ? 0 : group * 8 - head), n(group == 0 ? static_cast<int>(min(int64_t(8 - head), cols)) : count_from(col, cols, 8)) {}
};
template <typename T> __device__ __forceinline__ int head_of(const T *row) {
    return static_cast<int>(reinterpret_cast<uint64_t>(row) & 15) / static_cast<int>(sizeof(T));
}

// Rows to rows that lie anyhow.
template <typename T, int U>
__global__ void __launch_bounds__(32 * kWarps) dispatch_any_kernel(const Rows<const T> x, const Places places, const Rows<T> y, int64_t tokens,
                                                                   int64_t cols, int64_t per_token) {
    let_next_start();
    const Part<U> part(per_token);
    if (part.token >= tokens) return;
    after_previous();
    const T *const row = x.at(part.token, 0);
    for (int s0 = 0; s0 < places.top; s0 += 32) {
        const int at = places.load(part.token, s0), n = min(32, places.top - s0);
        for (int s = 0; s < n; ++s) {
            const int to = __shfl_sync(~0u, at, s);
            if (to < 0) continue;
            T *const out = y.at(to, 0);
            const int head = head_of(out);
            Fetched<T, false> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const Span span(part.group(u), head, cols);
                v[u].fetch(row + span.col, span.n);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const Span span(part.group(u), head, cols);
                store_eight<T, true>(out + span.col, 0, span.n, v[u].get(row + span.col, span.n));
            }
        }
    }
}

// Rows to aligned rows, and as codes.
template <typename T, int U, bool ALIGNED>
__global__ void __launch_bounds__(32 * kWarps, 4) dispatch_kernel(const Rows<const T> x, const Places places, const Rows<T> y, const RowCodes q4,
                                                               const RowCodes q8, int64_t tokens, int64_t cols, int64_t per_token) {
    let_next_start();
    const Part<U> part(per_token);
    if (part.token >= tokens) return;
    after_previous();
    Fetched<T, ALIGNED> in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) in[u].fetch(x.at(part.token, part.col(u)), count_from(part.col(u), cols, 8));
    Eight<T> v[U];
    EightCodes<COSTA_MX_E2M1> four[U];
    EightCodes<COSTA_MX_I8> eight[U];
    const int blocks = static_cast<int>((cols + 31) >> 5);
    int col[U];  // (past the row's last block where it would not fit)
#pragma unroll
    for (int u = 0; u < U; ++u) col[u] = static_cast<int>(min(part.col(u), int64_t(INT32_MAX)));
    for (int s0 = 0; s0 < places.top; s0 += 32) {
        const int at = places.load(part.token, s0), n = min(32, places.top - s0);
        if (s0 == 0)
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = in[u].get(x.at(part.token, part.col(u)), count_from(part.col(u), cols, 8));
        if (ALIGNED && y.p)
            for (int s = 0; s < n; ++s) {
                const int to = __shfl_sync(~0u, at, s);
                if (to < 0) continue;
#pragma unroll
                for (int u = 0; u < U; ++u) store_eight<T, true>(y.at(to, part.col(u)), 0, count_from(part.col(u), cols, 8), v[u]);
            }
        if (!q4.codes && !q8.codes) continue;
        if (s0 == 0) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = v[u](i);
                const float largest = block_largest(f);
                if (q4.codes) four[u] = EightCodes<COSTA_MX_E2M1>(f, largest);
                if (q8.codes) eight[u] = EightCodes<COSTA_MX_I8>(f, largest);
            }
        }
        for (int s = 0; s < n; ++s) {
            const int to = __shfl_sync(~0u, at, s);
            if (to < 0) continue;
            const CodeRow<COSTA_MX_E2M1> row4(q4, to);
            const CodeRow<COSTA_MX_I8> row8(q8, to);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (q4.codes) four[u].store(row4, col[u], blocks);
                if (q8.codes) eight[u].store(row8, col[u], blocks);
            }
        }
    }
}

template <typename T, int U, bool ALIGNED>
__global__ void __launch_bounds__(32 * kWarps, sizeof(T) == 2 ? 4 : 1) combine_kernel(const Rows<const T> z, const Places places, const float *w, int64_t ldw,
                                                              const Rows<T> y, int64_t tokens, int64_t cols, int64_t per_token) {
    constexpr int kSlots = (ALIGNED ? 8 : 4) / U;  // rows on their way at a time
    let_next_start();
    const Part<U> part(per_token);
    if (part.token >= tokens) return;
    after_previous();
    const int head = ALIGNED ? 0 : head_of(y.at(part.token, 0));
    int64_t col[U];
    int count[U];
    float sum[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const Span span(part.group(u), head, cols);
        col[u] = span.col;
        count[u] = span.n;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[u][i] = 0.0f;
    }
    for (int s0 = 0; s0 < places.top; s0 += 32) {
        const int at = places.load(part.token, s0), n = min(32, places.top - s0);
        const int lane = threadIdx.x % 32;
        const float weight = w && lane < n ? w[part.token * ldw + s0 + lane] : 1.0f;
        for (int s = 0; s < n; s += kSlots) {
            Fetched<T, ALIGNED> v[kSlots][U];
            int from[kSlots];
#pragma unroll
            for (int k = 0; k < kSlots; ++k) {
                from[k] = __shfl_sync(~0u, at, (s + k) & 31);
                if (s + k >= n) from[k] = -1;
#pragma unroll
                for (int u = 0; u < U; ++u)  // (one without a place: nothing of row 0)
                    v[k][u].fetch(z.at(max(from[k], 0), col[u]), from[k] < 0 ? 0 : count[u]);
            }
#pragma unroll
            for (int k = 0; k < kSlots; ++k) {
                const float f = __shfl_sync(~0u, weight, (s + k) & 31);
                if (from[k] < 0) continue;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const Eight<T> e = v[k][u].get(z.at(from[k], col[u]), count[u]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[u][i] = fmaf(f, e(i), sum[u][i]);
                }
            }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        Eight<T> out;
        out.set(sum[u]);
        store_eight<T, true>(y.at(part.token, col[u]), 0, count[u], out);
    }
}

// Experts of a token whose rows are taken together: as many as 32 registers hold on their way.
template <typename T, bool ALIGNED> constexpr int kBatch = (sizeof(T) == 2 ? 8 : 4) / (ALIGNED ? 1 : 2);

// A token to a block, or (WARP) to a warp of it.
template <typename T, bool WARP, bool ALIGNED>
__global__ void __launch_bounds__(128, 6) combine_backward_kernel(const Rows<const T> dy, const Rows<const T> z, const Places places, const float *w,
                                                                  int64_t ldw, const Rows<T> dz, const RowCodes q4, float *dw, int64_t lddw,
                                                                  int64_t tokens, int64_t cols) {
    constexpr int B = kBatch<T, ALIGNED>;
    __shared__ float sums[4][B];
    let_next_start();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t token = WARP ? int64_t(blockIdx.x) * 4 + warp : blockIdx.x;
    const int first = WARP ? lane : threadIdx.x, step = WARP ? 32 : 128;
    if (WARP && token >= tokens) return;
    after_previous();
    const int rounds = static_cast<int>(((cols + 31) / 32 * 4 + step - 1) / step);
    for (int s0 = 0; s0 < places.top; s0 += B) {
        const int at = places.load(token, s0), n = min(B, places.top - s0);
        const float weight = lane < n ? w[token * ldw + s0 + lane] : 0.0f;
        float dot[B];
#pragma unroll
        for (int s = 0; s < B; ++s) dot[s] = 0.0f;
        for (int j = 0; j < rounds; ++j) {
            const int64_t col = (first + int64_t(j) * step) * 8;
            const int count = count_from(col, cols, 8);
            Fetched<T, ALIGNED> fd, v[B];
            fd.fetch(dy.at(token, col), count);
            if (z.p) {
#pragma unroll
                for (int s = 0; s < B; ++s) {
                    const int from = s < n ? __shfl_sync(~0u, at, s) : -1;
                    v[s].fetch(z.at(max(from, 0), col), from < 0 ? 0 : count);
                }
            }
            const Eight<T> d = fd.get(dy.at(token, col), count);
#pragma unroll
            for (int s = 0; s < B; ++s) {
                if (s >= n) break;
                const int to = __shfl_sync(~0u, at, s);
                const float f = __shfl_sync(~0u, weight, s);
                if (to < 0) continue;
                if (z.p) {
                    const Eight<T> e = v[s].get(z.at(to, col), count);
#pragma unroll
                    for (int i = 0; i < 8; ++i) dot[s] = fmaf(d(i), e(i), dot[s]);
                }
                float out[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) out[i] = f * d(i);
                if (dz.p) {
                    Eight<T> e;
                    e.set(out);
                    store_eight<T, ALIGNED>(dz.at(to, col), 0, count, e);
                }
                if (q4.codes) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i >= count) out[i] = 0.0f;  // (not -0, nor an infinite weight's NaN)
                    EightCodes<COSTA_MX_E2M1>(out, block_largest(out)).store(CodeRow<COSTA_MX_E2M1>(q4, to), static_cast<int>(min(col, int64_t(INT32_MAX))),
                                                                            static_cast<int>((cols + 31) >> 5));
                }
            }
        }
        if (!dw) continue;
#pragma unroll
        for (int s = 0; s < B; ++s) dot[s] = warp_sum(dot[s]);
        if constexpr (WARP) {
#pragma unroll
            for (int s = 0; s < B; ++s)
                if (lane == s && s < n) dw[token * lddw + s0 + s] = dot[s];
        } else {
            if (s0) __syncthreads();  // the batch before has been read
#pragma unroll
            for (int s = 0; s < B; ++s)
                if (lane == s) sums[warp][s] = dot[s];
            __syncthreads();
            if (warp == 0 && lane < n)
                dw[token * lddw + s0 + lane] = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
        }
    }
}

Places places_of(const costa_mx_index &place, int64_t rows) {
    return {place.ptr, place.ld, rows, static_cast<int>(place.cols)};
}

// f(groups of eight to a lane) with few where there are few rows in all, whose latency counts.
template <typename F> cudaError_t by_part(int64_t tokens, int64_t cols, bool aligned, F g) {
    using std::integral_constant;
    const auto f = [&](auto u, int64_t per) { return aligned ? g(u, per, std::true_type()) : g(u, per, std::false_type()); };
    const int64_t eights = aligned ? mx_eights(cols) : std::max(mx_eights(cols), (cols + 14) / 8);
    if (tokens * mx_ceil(eights, 32) <= 152 * 16 || eights <= 32) return f(integral_constant<int, 1>(), mx_ceil(eights, 32));
    return f(integral_constant<int, 2>(), mx_ceil(eights, 64));
}

template <typename T>
cudaError_t dispatch(const costa_mx_dense &X, const costa_mx_index &place, int64_t rows, const costa_mx_dense *Y,
                     const costa_mx_matrix *Q4, const costa_mx_matrix *Q8, cudaStream_t s) {
    return by_part(X.rows, X.cols, aligned16(&X) && aligned16(Y), [&](auto u, int64_t per, auto line) {
        constexpr int U = decltype(u)::value;
        constexpr bool kAligned = decltype(line)::value;
        const int64_t blocks = mx_ceil(X.rows * per, kWarps);
        if (!kAligned && Y) {
            const cudaError_t e = mx_launch(dispatch_any_kernel<T, U>, blocks, 32 * kWarps, 0, 1, s, rows_of<const T>(&X), places_of(place, rows),
                                            rows_of<T>(Y), X.rows, X.cols, per);
            if (e != cudaSuccess || (!Q4 && !Q8)) return e;
        }
        return mx_launch(dispatch_kernel<T, U, kAligned>, blocks, 32 * kWarps, 0, 1, s, rows_of<const T>(&X), places_of(place, rows), rows_of<T>(Y),
                         row_codes_of(Q4), row_codes_of(Q8), X.rows, X.cols, per);
    });
}

template <typename T>
cudaError_t combine(const costa_mx_dense &Z, const costa_mx_index &place, const costa_mx_dense *W, const costa_mx_dense &Y,
                    cudaStream_t s) {
    return by_part(Y.rows, Y.cols, aligned16(&Z) && aligned16(&Y), [&](auto u, int64_t per, auto line) {
        return mx_launch(combine_kernel<T, decltype(u)::value, decltype(line)::value>, mx_ceil(Y.rows * per, kWarps), 32 * kWarps, 0, 1, s, rows_of<const T>(&Z),
                         places_of(place, Z.rows), W ? static_cast<const float *>(W->ptr) : nullptr, W ? W->ld : 0, rows_of<T>(&Y), Y.rows,
                         Y.cols, per);
    });
}

template <typename T>
cudaError_t combine_backward(const costa_mx_dense &dY, const costa_mx_dense *Z, const costa_mx_index &place, int64_t rows,
                             const costa_mx_dense &W, const costa_mx_dense *dZ, const costa_mx_matrix *Q4, const costa_mx_dense *dW,
                             cudaStream_t s) {
    const auto launch = [&](auto warp, auto line) {
        constexpr bool kWarp = decltype(warp)::value;
        return mx_launch(combine_backward_kernel<T, kWarp, decltype(line)::value>, kWarp ? mx_ceil(dY.rows, 4) : dY.rows, 128, 0, 1, s, rows_of<const T>(&dY),
                         rows_of<const T>(Z), places_of(place, rows), static_cast<const float *>(W.ptr), W.ld, rows_of<T>(dZ), row_codes_of(Q4),
                         dW ? static_cast<float *>(dW->ptr) : nullptr, dW ? dW->ld : 0, dY.rows, dY.cols);
    };
    const auto by_line = [&](auto warp) {
        return aligned16(&dY) && aligned16(Z) && aligned16(dZ) ? launch(warp, std::true_type()) : launch(warp, std::false_type());
    };
    return mx_eights(dY.cols) <= 128 ? by_line(std::true_type()) : by_line(std::false_type());
}

}  // namespace
}  // namespace mx

cudaError_t launch_mx_expert_sort(const costa_mx_index &experts, int n_experts, int align, const costa_mx_index &place,
                                  const costa_mx_index &starts, const costa_mx_index &counts, cudaStream_t s) {
    mx::Sort p{experts.ptr, experts.ld, experts.rows * experts.cols, static_cast<int>(experts.cols), n_experts, align,
               place.ptr, place.ld, starts.ptr, counts.ptr, 0};
    const bool many = p.pairs > 8192;
    const int warps = many ? mx::kSortThreads / 32
                           : static_cast<int>(std::max<int64_t>(std::min<int64_t>(mx_ceil(p.pairs, 32), mx::kSortThreads / 32),
                                                                mx_ceil(n_experts, 32)));
    const int blocks = many ? mx::kSortBlocks : 1;
    p.per_warp = mx_ceil(mx_ceil(p.pairs, int64_t(blocks) * warps), 32) * 32;
    const MxShared smem(sizeof(int) * (size_t(warps) + 1) * n_experts, sizeof(int) * (mx::kSortThreads / 32 + 1) * COSTA_MX_MAX_EXPERTS);
    return many ? mx_launch(mx::sort_kernel<mx::kSortBlocks>, blocks, 32 * warps, smem, blocks, s, p)
                : mx_launch(mx::sort_kernel<1>, blocks, 32 * warps, smem, 1, s, p);
}

cudaError_t launch_mx_dispatch(const costa_mx_dense &X, const costa_mx_index &place, int64_t rows, const costa_mx_dense *Y,
                               const costa_mx_matrix *Q4, const costa_mx_matrix *Q8, cudaStream_t s) {
    return X.type == COSTA_MX_F32 ? mx::dispatch<float>(X, place, rows, Y, Q4, Q8, s)
                                  : mx::dispatch<__nv_bfloat16>(X, place, rows, Y, Q4, Q8, s);
}

cudaError_t launch_mx_combine(const costa_mx_dense &Z, const costa_mx_index &place, const costa_mx_dense *W, const costa_mx_dense &Y,
                              cudaStream_t s) {
    return Y.type == COSTA_MX_F32 ? mx::combine<float>(Z, place, W, Y, s) : mx::combine<__nv_bfloat16>(Z, place, W, Y, s);
}

cudaError_t launch_mx_combine_backward(const costa_mx_dense &dY, const costa_mx_dense *Z, const costa_mx_index &place, int64_t rows,
                                       const costa_mx_dense &W, const costa_mx_dense *dZ, const costa_mx_matrix *Q4,
                                       const costa_mx_dense *dW, cudaStream_t s) {
    return dY.type == COSTA_MX_F32 ? mx::combine_backward<float>(dY, Z, place, rows, W, dZ, Q4, dW, s)
                                   : mx::combine_backward<__nv_bfloat16>(dY, Z, place, rows, W, dZ, Q4, dW, s);
}

}  // namespace costa
