// Root-mean-square norm with the residual's addition, and its gradients.
//
//   H = X + R (rounded),  s_i = 1 / sqrt(mean_j h_ij^2 + eps),  y_ij = h_ij s_i w_j
//   dx_ij = s_i (g_ij - u_ij c_i) + dh_ij  with  u = h s, g = dy w, c_i = mean_j g_ij u_ij
//   dw_j = sum_i dy_ij u_ij
//
// Memory bounds large calls, and the latency of one row small ones.  A row stays in
// the registers of a warp (up to 1024 elements, of the gradients 512) or of a thread
// block between its sum and what is written; only the gradients of more than 8192
// columns read dY and H twice.
// GB300, 8192 x 8192 bf16: the norm 92 us (5.8 TB/s, X and R read, H and Y written),
// its gradients 84 us (6.4 TB/s with the join of dW).  As 4- and 8-bit codes 2047 x
// 8192 take 28 us (floor 18.7): 41 instructions an element in 69% of the issue slots,
// between waits for the row's other warps; 100 bytes a thread are spilled at the 64
// registers that let two blocks share an SM.  4096 x 16384: 80 us (floor 79), gradients
// 138 (floor 79).  One row of 4096: 2 us.
#include <algorithm>
#include <type_traits>

#include "costa_internal.h"
#include "mx_rows.cuh"

namespace costa {
namespace mx {
namespace {

constexpr int kWarps = 4;  // of a block whose warps take a row each

// s = 1 / sqrt(sum / n + eps); or where the sum of squares, or that sum, left f32's range, kDown times the same of elements
// kDown = 2^-100 times as large and of kDown^2 eps: the largest element is above 2^56 then (there are 2^15 at most), beside
// which what underflows does not count.
__device__ __forceinline__ float square(float sum, float n, float eps) { return __fdiv_rn(sum, n) + eps; }
constexpr float kDown = 7.888609052210118e-31f;  // 2^-100

// A kernel's MOST: the most threads that share a row; a warp's 32 have a block of kWarps rows.
constexpr int threads_of(int most) { return most == 32 ? 32 * kWarps : most; }

// A sum over the threads that share a row, the same in all of them.  `turn` differs between neighbouring calls.
template <bool WARP> __device__ __forceinline__ float row_sum(float v, float (*sums)[32], int turn) {
    v = warp_sum(v);
    if constexpr (!WARP) {
        const int warps = blockDim.x / 32;
        if (threadIdx.x % 32 == 0) sums[turn][threadIdx.x / 32] = v;
        __syncthreads();
        v = static_cast<int>(threadIdx.x % 32) < warps ? sums[turn][threadIdx.x % 32] : 0.0f;
        v = warp_sum(v);
    }
    return v;
}

template <typename T> struct Forward {
    Rows<const T> x, r;
    Rows<T> h, y;
    const void *w;
    RowCodes q4, q8;
    float *s;
    int64_t lds, rows;
    int cols, w_f32;
    float eps;
};

// How many of eight elements from column `col` on a row has.
__device__ __forceinline__ int count_at(int col, int cols) { return max(0, min(8, cols - col)); }

// The weights of eight columns.
__device__ __forceinline__ void weights_of(const void *w, int f32, int col, int n, float (&v)[8]) {
    if (f32) {
        Eight<float> e;
        e.load(static_cast<const float *>(w) + col, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = e(i);
    } else {
        Eight<__nv_bfloat16> e;
        e.load(static_cast<const __nv_bfloat16 *>(w) + col, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = e(i);
    }
}

// Codes of eight values of a row; whole warps.
template <bool WHOLE = false>
__device__ __forceinline__ void write_codes(const RowCodes &q4, const RowCodes &q8, int64_t row, int col, int cols, const float (&v)[8]) {
    const float largest = block_largest(v);
    const int blocks = (cols + 31) >> 5;
    if (q4.codes) EightCodes<COSTA_MX_E2M1>(v, largest).store<WHOLE>(CodeRow<COSTA_MX_E2M1>(q4, row), col, blocks);
    if (q8.codes) EightCodes<COSTA_MX_I8>(v, largest).store<WHOLE>(CodeRow<COSTA_MX_I8>(q8, row), col, blocks);
}

// C groups of eight elements to a thread.  ALIGNED: the rows of X, R, H and Y lie on 16-byte boundaries.
template <typename T, int C, int MOST, bool ALIGNED>
__global__ void __launch_bounds__(threads_of(MOST)) norm_forward_kernel(const Forward<T> p) {
    constexpr bool WARP = MOST == 32;
    __shared__ float sums[2][32];
    let_next_start();
    const int64_t row = WARP ? int64_t(blockIdx.x) * kWarps + threadIdx.x / 32 : blockIdx.x;
    const int first = WARP ? threadIdx.x % 32 : threadIdx.x, step = WARP ? 32 : blockDim.x;
    after_previous();
    if (WARP && row >= p.rows) return;
    const T *const x_row = p.x.at(row, 0), *const r_row = p.r.at(row, 0);
    T *const h_row = p.h.at(row, 0), *const y_row = p.y.at(row, 0);
    Eight<T> h[C];
    float sum = 0.0f;
    Fetched<T, ALIGNED> x[C], r[C];
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int col = (first + j * step) * 8;
        x[j].fetch(x_row + col, count_at(col, p.cols));
    }
    if (p.r.p) {
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int col = (first + j * step) * 8;
            r[j].fetch(r_row + col, count_at(col, p.cols));
        }
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int col = (first + j * step) * 8;
            const int count = count_at(col, p.cols);
            const Eight<T> a = x[j].get(x_row + col, count), b = r[j].get(r_row + col, count);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = a(i) + b(i);
            h[j].set(v);
            store_eight<T, ALIGNED>(h_row + col, 0, count, h[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int col = (first + j * step) * 8;
            h[j] = x[j].get(x_row + col, count_at(col, p.cols));
        }
    }
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(h[j](i), h[j](i), sum);
    const float n = static_cast<float>(p.cols);
    const float all = square(row_sum<WARP>(sum, sums, 0), n, p.eps);
    float s = __frsqrt_rn(all);
    if (all == INFINITY) {
        sum = 0.0f;
#pragma unroll
        for (int j = 0; j < C; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(h[j](i) * kDown, h[j](i) * kDown, sum);
        s = kDown * __frsqrt_rn(square(row_sum<WARP>(sum, sums, 1), n, p.eps * kDown * kDown));
    }
    if (p.s && first == 0) p.s[row * p.lds] = s;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int col = (first + j * step) * 8;
        const int count = count_at(col, p.cols);
        float w[8], v[8];
        weights_of(p.w, p.w_f32, col, count, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = h[j](i) * s * w[i];
        if (p.y.p) {
            Eight<T> y;
            y.set(v);
            store_eight<T, ALIGNED>(y_row + col, 0, count, y);
        }
        if (p.q4.codes || p.q8.codes) write_codes(p.q4, p.q8, row, col, p.cols, v);
    }
}

template <typename T> struct Backward {
    Rows<const T> dy, h, dh;
    Rows<T> dx;
    const void *w;
    const float *s;
    float *work;  // a row of `pitch` partial sums to a block; null: no dW
    int64_t lds, rows;
    int cols, pitch, w_f32;
};

// Of the widest rows neither dY and H nor the sums of dW fit the registers: the rows are read again (from the L2 cache)
// after their sum is known, and the sums of dW are in shared memory.
template <typename T, int C, int MOST, bool ALIGNED>
__global__ void __launch_bounds__(threads_of(MOST), MOST == 32 ? 4 : MOST == 512 && sizeof(T) == 2 ? 2 : 1) norm_backward_kernel(const Backward<T> p) {
    constexpr bool WARP = MOST == 32, kKeep = WARP || C < 4;
    __shared__ float sums[2][32];
    __shared__ __align__(16) float joined[WARP ? 32 * C * 8 : 4];
    extern __shared__ float4 wide[];  // [C][2][threads]
    let_next_start();
    const int warp = threadIdx.x / 32;
    const int first = WARP ? threadIdx.x % 32 : threadIdx.x, step = WARP ? 32 : blockDim.x;
    const int64_t per = WARP ? kWarps : 1;
    auto wide_at = [&](int j) { return wide + (2 * j) * step + first; };
    after_previous();
    float dw[kKeep ? C : 1][8];
#pragma unroll
    for (int j = 0; j < C; ++j) {
        if constexpr (kKeep) {
#pragma unroll
            for (int i = 0; i < 8; ++i) dw[j][i] = 0.0f;
        } else {
            wide_at(j)[0] = wide_at(j)[step] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
    }
    int turn = 0;
    for (int64_t row = int64_t(blockIdx.x) * per + (WARP ? warp : 0); row < p.rows; row += gridDim.x * per, turn ^= 1) {
        constexpr int kHave = kKeep ? C : 1;
        const T *const dy_row = p.dy.at(row, 0), *const h_row = p.h.at(row, 0), *const dh_row = p.dh.at(row, 0);
        T *const dx_row = p.dx.at(row, 0);
        Fetched<T, ALIGNED> fy[kHave], fh[kHave], fd[kHave];
        Eight<T> dy[kHave], h[kHave];
        auto fetch = [&](int j, int at) {
            const int col = (first + j * step) * 8;
            const int count = count_at(col, p.cols);
            fy[at].fetch(dy_row + col, count);
            fh[at].fetch(h_row + col, count);
        };
        auto fetch_dh = [&](int j, int at) {
            const int col = (first + j * step) * 8;
            if (p.dh.p) fd[at].fetch(dh_row + col, count_at(col, p.cols));
        };
        auto get = [&](int j, int at) {
            const int col = (first + j * step) * 8;
            const int count = count_at(col, p.cols);
            dy[at] = fy[at].get(dy_row + col, count);
            h[at] = fh[at].get(h_row + col, count);
        };
        if constexpr (kKeep) {
#pragma unroll
            for (int j = 0; j < C; ++j) fetch(j, j);
#pragma unroll
            for (int j = 0; j < C; ++j) fetch_dh(j, j);
#pragma unroll
            for (int j = 0; j < C; ++j) get(j, j);
        }
        const float s = p.s[row * p.lds];
        float along = 0.0f;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int at = kKeep ? j : 0;
            if constexpr (!kKeep) {
                fetch(j, 0);
                get(j, 0);
            }
            const int col = (first + j * step) * 8;
            float w[8], t[8];
            weights_of(p.w, p.w_f32, col, count_at(col, p.cols), w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                t[i] = dy[at](i) * (h[at](i) * s);
                along = fmaf(t[i], w[i], along);
            }
            if constexpr (kKeep) {
#pragma unroll
                for (int i = 0; i < 8; ++i) dw[j][i] += t[i];
            } else {
                float4 a = wide_at(j)[0], b = wide_at(j)[step];
                a.x += t[0], a.y += t[1], a.z += t[2], a.w += t[3];
                b.x += t[4], b.y += t[5], b.z += t[6], b.w += t[7];
                wide_at(j)[0] = a;
                wide_at(j)[step] = b;
            }
        }
        along = __fdiv_rn(row_sum<WARP>(along, sums, turn), static_cast<float>(p.cols));
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int at = kKeep ? j : 0;
            if constexpr (!kKeep) {
                fetch(j, 0);
                fetch_dh(j, 0);
                get(j, 0);
            }
            const int col = (first + j * step) * 8;
            const int count = count_at(col, p.cols);
            float w[8], v[8];
            weights_of(p.w, p.w_f32, col, count, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = s * (dy[at](i) * w[i] - h[at](i) * s * along);
            if (p.dh.p) {
                const Eight<T> dh = fd[at].get(dh_row + col, count);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += dh(i);
            }
            Eight<T> dx;
            dx.set(v);
            store_eight<T, ALIGNED>(dx_row + col, 0, count, dx);
        }
    }
    if (!p.work) return;
    if constexpr (WARP) {  // the warps' sums, in their order
        for (int k = 0; k < kWarps; ++k) {
            if (warp == k)
#pragma unroll
                for (int j = 0; j < C; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float &to = joined[(first + 32 * j) * 8 + i];
                        to = k == 0 ? dw[j][i] : to + dw[j][i];
                    }
            __syncthreads();
        }
        for (int k = threadIdx.x; k < p.cols; k += blockDim.x) p.work[int64_t(blockIdx.x) * p.pitch + k] = joined[k];
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int col = (first + j * step) * 8;
            if (col >= p.pitch) continue;
            float4 *const to = reinterpret_cast<float4 *>(p.work + (int64_t(blockIdx.x) * p.pitch + col));
            if constexpr (kKeep) {
                to[0] = make_float4(dw[j][0], dw[j][1], dw[j][2], dw[j][3]);
                to[1] = make_float4(dw[j][4], dw[j][5], dw[j][6], dw[j][7]);
            } else {
                to[0] = wide_at(j)[0];
                to[1] = wide_at(j)[step];
            }
        }
    }
}

// ---- many rows: each block lets its rows follow each other through shared memory ----
//
// A block takes every gridDim.x-th row and has `stages` of them under way: a thread asks for its own two groups of eight of
// the row that comes stages - 1 rows later, by copies of 16 bytes that need no registers and fill with zeros past the
// row's end, before it takes those of this row.  Only it reads them, so that nothing but its own copies is waited for.
// (8192 x 8192 bf16 with a block to a row, loaded to registers: 142 us, so 92; gradients 429 us, so 84.)
// The weights stay in registers.  WHOLE: the rows have all of the block's groups, of which then nothing is checked.

constexpr int kStreamGroups = 2, kStreamThreads = 512;
constexpr int kStreamBytes = 208 * 1024;  // of shared memory, of an SM's blocks

template <typename T, int ARRAYS, bool WHOLE> struct Stream {
    static constexpr int kPieces = sizeof(T) / 2, kPer = 16 / sizeof(T);  // 16-byte pieces of a group, elements of one
    uint4 *base;
    __device__ uint4 *at(int stage, int array, int j, int piece) const {
        return base + (((stage * ARRAYS + array) * kStreamGroups + j) * kPieces + piece) * blockDim.x + threadIdx.x;
    }
    __device__ void fetch(int stage, int array, const T *row, int cols) const {
#pragma unroll
        for (int j = 0; j < kStreamGroups; ++j)
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                const int col = (threadIdx.x + j * blockDim.x) * 8 + k * kPer;
                const int bytes = WHOLE ? 16 : max(0, min(kPer, cols - col)) * static_cast<int>(sizeof(T));
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                                 static_cast<uint32_t>(__cvta_generic_to_shared(at(stage, array, j, k)))),
                             "l"(bytes ? row + col : row), "r"(bytes)
                             : "memory");
            }
    }
    __device__ Eight<T> get(int stage, int array, int j) const {
        Eight<T> x;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const uint4 v = *at(stage, array, j, k);
            x.w[4 * k] = v.x;
            x.w[4 * k + 1] = v.y;
            x.w[4 * k + 2] = v.z;
            x.w[4 * k + 3] = v.w;
        }
        return x;
    }
};
__device__ __forceinline__ void stream_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Until at most `left` (0 to 3) of the rows that this thread asked for are under way.
__device__ __forceinline__ void stream_wait(int left) {
    if (left == 0)
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    else if (left == 1)
        asm volatile("cp.async.wait_group 1;" ::: "memory");
    else if (left == 2)
        asm volatile("cp.async.wait_group 2;" ::: "memory");
    else
        asm volatile("cp.async.wait_group 3;" ::: "memory");
}

template <typename T, bool WHOLE> __global__ void __launch_bounds__(kStreamThreads, 2) norm_forward_stream_kernel(const Forward<T> p, const int stages) {
    __shared__ float sums[3][32];
    extern __shared__ uint4 staged[];
    constexpr int C = kStreamGroups;
    let_next_start();
    const Stream<T, 2, WHOLE> in{staged};
    const int first = threadIdx.x, step = blockDim.x;
    auto count = [&](int col) { return WHOLE ? 8 : count_at(col, p.cols); };
    after_previous();
    auto fetch = [&](int64_t row, int stage) {
        if (row < p.rows) {
            in.fetch(stage, 0, p.x.at(row, 0), p.cols);
            if (p.r.p) in.fetch(stage, 1, p.r.at(row, 0), p.cols);
        }
        stream_commit();
    };
    for (int k = 0; k < stages - 1; ++k) fetch(blockIdx.x + int64_t(k) * gridDim.x, k);
    float w[C][8];
#pragma unroll
    for (int j = 0; j < C; ++j) weights_of(p.w, p.w_f32, (first + j * step) * 8, count_at((first + j * step) * 8, p.cols), w[j]);
    const float n = static_cast<float>(p.cols);
    int stage = 0, turn = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
        fetch(row + int64_t(stages - 1) * gridDim.x, stage == 0 ? stages - 1 : stage - 1);
        stream_wait(stages - 1);
        Eight<T> h[C];
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            h[j] = in.get(stage, 0, j);
            if (p.r.p) {
                const Eight<T> r = in.get(stage, 1, j);
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = h[j](i) + r(i);
                h[j].set(v);
                store_eight<T, true>(p.h.at(row, (first + j * step) * 8), 0, count((first + j * step) * 8), h[j]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(h[j](i), h[j](i), sum);
        }
        stage = stage + 1 == stages ? 0 : stage + 1;
        const float all = square(row_sum<false>(sum, sums, turn), n, p.eps);
        float s = __frsqrt_rn(all);
        if (all == INFINITY) {
            sum = 0.0f;
#pragma unroll
            for (int j = 0; j < C; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fmaf(h[j](i) * kDown, h[j](i) * kDown, sum);
            s = kDown * __frsqrt_rn(square(row_sum<false>(sum, sums, 2), n, p.eps * kDown * kDown));
        }
        if (p.s && first == 0) p.s[row * p.lds] = s;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int col = (first + j * step) * 8;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = h[j](i) * s * w[j][i];
            if (p.y.p) {
                Eight<T> y;
                y.set(v);
                store_eight<T, true>(p.y.at(row, col), 0, count(col), y);
            }
            if (p.q4.codes || p.q8.codes) write_codes<WHOLE>(p.q4, p.q8, row, col, p.cols, v);
        }
    }
}

template <typename T, bool WHOLE> __global__ void __launch_bounds__(kStreamThreads, 1) norm_backward_stream_kernel(const Backward<T> p, const int stages) {
    __shared__ float sums[2][32];
    extern __shared__ uint4 staged[];
    constexpr int C = kStreamGroups;
    let_next_start();
    const Stream<T, 3, WHOLE> in{staged};
    const int first = threadIdx.x, step = blockDim.x;
    auto count = [&](int col) { return WHOLE ? 8 : count_at(col, p.cols); };
    after_previous();
    auto fetch = [&](int64_t row, int stage) {
        if (row < p.rows) {
            in.fetch(stage, 0, p.dy.at(row, 0), p.cols);
            in.fetch(stage, 1, p.h.at(row, 0), p.cols);
            if (p.dh.p) in.fetch(stage, 2, p.dh.at(row, 0), p.cols);
        }
        stream_commit();
    };
    for (int k = 0; k < stages - 1; ++k) fetch(blockIdx.x + int64_t(k) * gridDim.x, k);
    float w[C][8], dw[C][8];
#pragma unroll
    for (int j = 0; j < C; ++j) {
        weights_of(p.w, p.w_f32, (first + j * step) * 8, count_at((first + j * step) * 8, p.cols), w[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = 0.0f;
    }
    int stage = 0, turn = 0;
    float s_next = p.s[blockIdx.x * p.lds];
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
        const float s = s_next;
        if (row + gridDim.x < p.rows) s_next = p.s[(row + gridDim.x) * p.lds];
        fetch(row + int64_t(stages - 1) * gridDim.x, stage == 0 ? stages - 1 : stage - 1);
        stream_wait(stages - 1);
        Eight<T> dy[C], h[C];
        float along = 0.0f;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            dy[j] = in.get(stage, 0, j);
            h[j] = in.get(stage, 1, j);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float t = dy[j](i) * (h[j](i) * s);
                dw[j][i] += t;
                along = fmaf(t, w[j][i], along);
            }
        }
        along = __fdiv_rn(row_sum<false>(along, sums, turn), static_cast<float>(p.cols));
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int col = (first + j * step) * 8;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = s * (dy[j](i) * w[j][i] - h[j](i) * s * along);
            if (p.dh.p) {
                const Eight<T> dh = in.get(stage, 2, j);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += dh(i);
            }
            Eight<T> dx;
            dx.set(v);
            store_eight<T, true>(p.dx.at(row, col), 0, count(col), dx);
        }
        stage = stage + 1 == stages ? 0 : stage + 1;
    }
    if (!p.work) return;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int col = (first + j * step) * 8;
        if (col >= p.pitch) continue;
        float4 *const to = reinterpret_cast<float4 *>(p.work + (int64_t(blockIdx.x) * p.pitch + col));
        to[0] = make_float4(dw[j][0], dw[j][1], dw[j][2], dw[j][3]);
        to[1] = make_float4(dw[j][4], dw[j][5], dw[j][6], dw[j][7]);
    }
}

// The gradients for rows that lie anyhow with respect to 16 bytes.  The blocks' number is a multiple of the elements in 16
// bytes, so that all rows of a block lie alike, in each matrix its own way.  They come to shared memory as they lie; a
// thread's groups of eight lie as those of the output do, and are taken from where they are in the inputs' rows.  (8192 x
// 4097 f32: 118 us, from registers 202 us; the norm itself gains nothing by it.)

template <typename T, int ARRAYS> struct Windows {
    static constexpr int kPieces = sizeof(T) / 2, kPer = 16 / sizeof(T), kWords = Eight<T>::kWords;
    uint4 *base;
    int pieces, cols;  // of a row (and one before and after it); of the matrices
    __device__ Windows(uint4 *staged, int n) : base(staged), pieces(kStreamGroups * kPieces * blockDim.x + 2), cols(n) {}
    __device__ static int head_of(const T *row) { return static_cast<int>(reinterpret_cast<uint64_t>(row) & 15) / static_cast<int>(sizeof(T)); }
    __device__ uint4 *at(int stage, int array) const { return base + (stage * ARRAYS + array) * pieces + 1; }
    __device__ void fetch(int stage, int array, const T *row) const {
        const int head = head_of(row);
#pragma unroll
        for (int i = 0; i < kStreamGroups * kPieces; ++i) {
            const int q = threadIdx.x + i * blockDim.x, bytes = max(0, min(kPer, cols + head - q * kPer)) * static_cast<int>(sizeof(T));
            if (bytes)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                                 static_cast<uint32_t>(__cvta_generic_to_shared(at(stage, array) + q))),
                             "l"(row - head + q * kPer), "r"(bytes)
                             : "memory");
        }
    }
    // Columns col .. col + 7 of a row that begins `head` elements after a boundary; 0 for those that it has not.  (col + head)
    // modulo the elements in 16 bytes is the same in all threads.
    __device__ Eight<T> get(int stage, int array, int col, int head) const {
        const int e = col + head, off = e & (kPer - 1);
        const uint4 *const from = at(stage, array) + (e - off) / kPer;
        uint32_t c[kWords + 4];
#pragma unroll
        for (int k = 0; k <= kPieces; ++k) {
            if (k == kPieces && off == 0) break;
            const uint4 v = from[k];
            c[4 * k] = v.x;
            c[4 * k + 1] = v.y;
            c[4 * k + 2] = v.z;
            c[4 * k + 3] = v.w;
        }
        Eight<T> x;
        const uint32_t bytes = off * sizeof(T), bits = (bytes & 2) * 8;
        if (bytes == 0) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) x.w[i] = c[i];
        } else if (bytes < 4) {
            from_word<T, 0>(c, bits, x.w);
        } else if (bytes < 8) {
            from_word<T, 1>(c, bits, x.w);
        } else if (bytes < 12) {
            from_word<T, 2>(c, bits, x.w);
        } else {
            from_word<T, 3>(c, bits, x.w);
        }
        if (__builtin_expect(col < 0 || col + 8 > cols, 0)) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < 0 || col + i >= cols) {
                    if constexpr (sizeof(T) == 4)
                        x.w[i] = 0;
                    else
                        x.w[i / 2] &= i % 2 ? 0xffffu : 0xffff0000u;
                }
        }
        return x;
    }
    __device__ void store(T *row, int col, const Eight<T> &x) const {
        if (__builtin_expect(col >= 0 && col + 8 <= cols, 1)) {
#pragma unroll
            for (int j = 0; j < kWords; j += 4)
                reinterpret_cast<uint4 *>(row + col)[j / 4] = make_uint4(x.w[j], x.w[j + 1], x.w[j + 2], x.w[j + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i >= 0 && col + i < cols) row[col + i] = from_float<T>(x(i));
        }
    }
    __device__ void weights(const void *w, int f32, int col, float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool in = col + i >= 0 && col + i < cols;
            v[i] = !in ? 0.0f : f32 ? static_cast<const float *>(w)[col + i] : to_float(static_cast<const __nv_bfloat16 *>(w)[col + i]);
        }
    }
};

template <typename T> __global__ void __launch_bounds__(kStreamThreads, 1) norm_backward_windows_kernel(const Backward<T> p, const int stages) {
    __shared__ float sums[2][32];
    extern __shared__ uint4 staged[];
    constexpr int C = kStreamGroups;
    let_next_start();
    const Windows<T, 3> in(staged, p.cols);
    after_previous();
    const int dy_head = in.head_of(p.dy.at(blockIdx.x, 0)), h_head = in.head_of(p.h.at(blockIdx.x, 0));
    const int dh_head = in.head_of(p.dh.at(blockIdx.x, 0)), out_head = in.head_of(p.dx.at(blockIdx.x, 0));
    auto col_of = [&](int j) { return static_cast<int>(threadIdx.x + j * blockDim.x) * 8 - out_head; };
    auto fetch = [&](int64_t row, int stage) {
        if (row < p.rows) {
            in.fetch(stage, 0, p.dy.at(row, 0));
            in.fetch(stage, 1, p.h.at(row, 0));
            if (p.dh.p) in.fetch(stage, 2, p.dh.at(row, 0));
        }
        stream_commit();
    };
    for (int k = 0; k < stages - 1; ++k) fetch(blockIdx.x + int64_t(k) * gridDim.x, k);
    float w[C][8], dw[C][8];
#pragma unroll
    for (int j = 0; j < C; ++j) {
        in.weights(p.w, p.w_f32, col_of(j), w[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = 0.0f;
    }
    int stage = 0, turn = 0;
    float s_next = p.s[blockIdx.x * p.lds];
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
        const float s = s_next;
        if (row + gridDim.x < p.rows) s_next = p.s[(row + gridDim.x) * p.lds];
        stream_wait(stages - 2);
        __syncthreads();
        fetch(row + int64_t(stages - 1) * gridDim.x, stage == 0 ? stages - 1 : stage - 1);
        Eight<T> dy[C], h[C];
        float along = 0.0f;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            dy[j] = in.get(stage, 0, col_of(j), dy_head);
            h[j] = in.get(stage, 1, col_of(j), h_head);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float t = dy[j](i) * (h[j](i) * s);
                dw[j][i] += t;
                along = fmaf(t, w[j][i], along);
            }
        }
        along = __fdiv_rn(row_sum<false>(along, sums, turn), static_cast<float>(p.cols));
#pragma unroll
        for (int j = 0; j < C; ++j) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = s * (dy[j](i) * w[j][i] - h[j](i) * s * along);
            if (p.dh.p) {
                const Eight<T> dh = in.get(stage, 2, col_of(j), dh_head);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += dh(i);
            }
            Eight<T> dx;
            dx.set(v);
            in.store(p.dx.at(row, 0), col_of(j), dx);
        }
        stage = stage + 1 == stages ? 0 : stage + 1;
    }
    if (!p.work) return;
    float *const to = p.work + int64_t(blockIdx.x) * p.pitch;
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col_of(j) + i >= 0 && col_of(j) + i < p.cols) to[col_of(j) + i] = dw[j][i];
}

// dW = the blocks' partial sums, joined in one order: 32 columns to a block, each thread adds every 32nd block's of four.
template <typename T> __global__ void __launch_bounds__(256) norm_join_kernel(const float *work, int64_t pitch, int parts, int64_t cols, T *dw) {
    __shared__ float4 sums[32][8];
    let_next_start();
    after_previous();
    const int line = threadIdx.x / 8, four = threadIdx.x % 8;
    const float4 *const from = reinterpret_cast<const float4 *>(work + int64_t(blockIdx.x) * 32) + four;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 10
    for (int k = line; k < parts; k += 32) {
        const float4 v = from[k * (pitch / 4)];
        sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
    }
    sums[line][four] = sum;
    __syncthreads();
    const int64_t col = int64_t(blockIdx.x) * 32 + threadIdx.x;
    if (threadIdx.x >= 32 || col >= cols) return;
    const float *const mine = &reinterpret_cast<const float *>(sums)[threadIdx.x];
    float part[4] = {};
#pragma unroll
    for (int k = 0; k < 32; ++k) part[k % 4] += mine[32 * k];
    dw[col] = from_float<T>((part[0] + part[1]) + (part[2] + part[3]));
}

// How a row is laid out: groups of eight to a thread, and threads (32: a warp).
struct Shape {
    int c, threads;
};

// A warp up to `most` groups (16384 x 1000 bf16: 22 us, by blocks 28 us; gradients, whose sums of dW fill a warp's registers
// by then, 46 and 41 us).  Else a block, with few groups to a thread where there are few rows and latency counts.
constexpr int kForwardMost = 128, kBackwardMost = 64;
Shape shape_of(int64_t cols, int64_t rows, int most) {
    const int64_t eights = mx_eights(cols);
    if (eights <= most) return {eights <= 32 ? 1 : eights <= 64 ? 2 : 4, 32};
    const int c = rows <= 304 && eights <= 1024 ? 1 : eights <= 1024 ? 2 : 4;
    return {c, static_cast<int>(mx_ceil(mx_ceil(eights, c), 32) * 32)};
}

// Threads for rows of windows: their groups, begun up to 16 bytes early.
template <typename T> int window_threads(int64_t cols) {
    return static_cast<int>(mx_ceil(mx_ceil(cols + 16 / sizeof(T), 8 * kStreamGroups), 32) * 32);
}
// Blocks to an SM and rows under way in each (two at least), for rows of `arrays` matrices, by shared memory and 1024 threads.
// (The gradients' 128 registers leave room for 512 threads: of two blocks of more than 256 each the second then waits for the
// first; 8192 x 5120 bf16 68 us, floor 49, where 4096 columns take 47, floor 40.)
struct Under {
    int blocks, stages;
    MxShared bytes;
};
Under under_way(int threads, int arrays, int size, int most_blocks) {
    const size_t stage = size_t(16) * arrays * (kStreamGroups * (size / 2) * threads + 2);  // (windows need two pieces more)
    int blocks = std::max(1, std::min(most_blocks, 1024 / threads));
    while (blocks > 1 && kStreamBytes / (blocks * stage) < 3) --blocks;
    const int stages = static_cast<int>(std::min<size_t>(4, kStreamBytes / (blocks * stage)));
    return {blocks, stages, MxShared(stage * stages, kStreamBytes)};
}
static_assert(kStreamBytes / (16 * 3 * (kStreamGroups * 2 * kStreamThreads + 2)) >= 2, "two rows of the widest");

// Whether rows of this shape come through shared memory, where they lie aligned (or as windows).
bool streams(const Shape &s) { return s.c == kStreamGroups && s.threads > 32; }

// f(groups of eight to a thread, most threads, aligned) for a shape; MOST: a warp's groups.
template <int MOST, typename F> cudaError_t with_shape(const Shape &s, bool aligned, F g) {
    using std::integral_constant;
    using One = integral_constant<int, 1>;
    using Two = integral_constant<int, 2>;
    using Four = integral_constant<int, 4>;
    const auto f = [&](auto c, auto most) { return aligned ? g(c, most, std::true_type()) : g(c, most, std::false_type()); };
    if (s.threads == 32) {
        const integral_constant<int, 32> warp;
        if constexpr (MOST > 64)
            if (s.c == 4) return f(Four(), warp);
        return s.c == 1 ? f(One(), warp) : f(Two(), warp);
    }
    if (s.c == 1) return f(One(), integral_constant<int, 1024>());
    if (s.c == 2) return g(Two(), integral_constant<int, 512>(), std::false_type());
    return f(Four(), integral_constant<int, 1024>());
}

template <typename T>
cudaError_t forward(const costa_mx_dense &X, const costa_mx_dense *R, const costa_mx_dense &W, float eps,
                    const costa_mx_dense *H, const costa_mx_dense *Y, const costa_mx_matrix *Q4, const costa_mx_matrix *Q8,
                    const costa_mx_dense *S, cudaStream_t s) {
    const Shape shape = shape_of(X.cols, X.rows, kForwardMost);
    const Forward<T> p{rows_of<const T>(&X), rows_of<const T>(R), rows_of<T>(H), rows_of<T>(Y), W.ptr, row_codes_of(Q4),
                       row_codes_of(Q8), S ? static_cast<float *>(S->ptr) : nullptr, S ? S->ld : 0, X.rows, static_cast<int>(X.cols),
                       W.type == COSTA_MX_F32, eps};
    const bool aligned = aligned16(&X) && aligned16(R) && aligned16(H) && aligned16(Y);
    if (streams(shape) && aligned) {
        const Under u = under_way(shape.threads, 2, sizeof(T), 8);
        const auto launch = [&](auto whole) {
            return mx_launch(norm_forward_stream_kernel<T, decltype(whole)::value>, std::min<int64_t>(X.rows, 152 * u.blocks), shape.threads,
                             u.bytes, 1, s, p, u.stages);
        };
        return X.cols == shape.threads * 8 * kStreamGroups ? launch(std::true_type()) : launch(std::false_type());
    }
    return with_shape<kForwardMost>(shape, aligned, [&](auto c, auto most, auto line) {
        constexpr int C = decltype(c)::value, kMost = decltype(most)::value;
        return mx_launch(norm_forward_kernel<T, C, kMost, decltype(line)::value>, kMost == 32 ? mx_ceil(X.rows, kWarps) : X.rows,
                         kMost == 32 ? 32 * kWarps : shape.threads, 0, 1, s, p);
    });
}

template <typename T>
cudaError_t backward(const costa_mx_dense &dY, const costa_mx_dense &H, const costa_mx_dense &S, const costa_mx_dense &W,
                     const costa_mx_dense *dH, const costa_mx_dense &dX, const costa_mx_dense *dW, void *work, cudaStream_t s) {
    const Shape shape = shape_of(H.cols, H.rows, kBackwardMost);
    const int64_t pitch = mx_eights(H.cols) * 8;
    const Backward<T> p{rows_of<const T>(&dY), rows_of<const T>(&H), rows_of<const T>(dH), rows_of<T>(&dX), W.ptr,
                        static_cast<const float *>(S.ptr), dW ? static_cast<float *>(work) : nullptr, S.ld, H.rows,
                        static_cast<int>(H.cols), static_cast<int>(pitch), W.type == COSTA_MX_F32};
    int64_t parts = 0;
    cudaError_t e = cudaSuccess;
    const int most_blocks = static_cast<int>(mx_norm_parts(H.cols) / 152), window = window_threads<T>(H.cols);
    const bool aligned = aligned16(&dY) && aligned16(&H) && aligned16(dH) && aligned16(&dX);
    if (streams(shape) && aligned) {
        const Under u = under_way(shape.threads, 3, sizeof(T), most_blocks);
        parts = std::min<int64_t>(H.rows, 152 * u.blocks);
        const auto launch = [&](auto whole) {
            return mx_launch(norm_backward_stream_kernel<T, decltype(whole)::value>, parts, shape.threads, u.bytes, 1, s, p, u.stages);
        };
        e = H.cols == shape.threads * 8 * kStreamGroups ? launch(std::true_type()) : launch(std::false_type());
    } else if (streams(shape) && window <= kStreamThreads) {
        const Under u = under_way(window, 3, sizeof(T), most_blocks);
        parts = std::min<int64_t>(H.rows / 8 * 8, 152 * u.blocks);
        e = mx_launch(norm_backward_windows_kernel<T>, parts, window, u.bytes, 1, s, p, u.stages);
    } else if (H.rows > 0) {
        e = with_shape<kBackwardMost>(shape, aligned, [&](auto c, auto most, auto line) {
            constexpr int C = decltype(c)::value, kMost = decltype(most)::value;
            const int threads = kMost == 32 ? 32 * kWarps : shape.threads;
            constexpr size_t kWide = kMost == 32 || C < 4 ? 0 : sizeof(float) * 8 * C;  // of a thread
            const MxShared wide(kWide * threads, kWide * kMost);
            parts = std::min<int64_t>(kMost == 32 ? mx_ceil(H.rows, kWarps) : H.rows, mx_norm_parts(H.cols));
            return mx_launch(norm_backward_kernel<T, C, kMost, decltype(line)::value>, parts, threads, wide, 1, s, p);
        });
    }
    if (e != cudaSuccess || !dW) return e;
    const auto join = [&](auto *to) {
        using D = std::remove_pointer_t<decltype(to)>;
        return mx_launch(norm_join_kernel<D>, mx_ceil(H.cols, 32), 256, 0, 1, s, p.work, pitch, static_cast<int>(parts),
                         H.cols, to);
    };
    return dW->type == COSTA_MX_F32 ? join(static_cast<float *>(dW->ptr)) : join(static_cast<__nv_bfloat16 *>(dW->ptr));
}

}  // namespace
}  // namespace mx

cudaError_t launch_mx_norm_forward(const costa_mx_dense &X, const costa_mx_dense *R, const costa_mx_dense &W, float eps,
                                   const costa_mx_dense *H, const costa_mx_dense *Y, const costa_mx_matrix *Q4,
                                   const costa_mx_matrix *Q8, const costa_mx_dense *S, cudaStream_t s) {
    return X.type == COSTA_MX_F32 ? mx::forward<float>(X, R, W, eps, H, Y, Q4, Q8, S, s)
                                  : mx::forward<__nv_bfloat16>(X, R, W, eps, H, Y, Q4, Q8, S, s);
}

cudaError_t launch_mx_norm_backward(const costa_mx_dense &dY, const costa_mx_dense &H, const costa_mx_dense &S,
                                    const costa_mx_dense &W, const costa_mx_dense *dH, const costa_mx_dense &dX,
                                    const costa_mx_dense *dW, void *work, cudaStream_t s) {
    return H.type == COSTA_MX_F32 ? mx::backward<float>(dY, H, S, W, dH, dX, dW, work, s)
                                  : mx::backward<__nv_bfloat16>(dY, H, S, W, dH, dX, dW, work, s);
}

}  // namespace costa
