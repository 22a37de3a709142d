// Tensor-core plumbing of the low-bit products: mbarriers with bounded waits,
// bulk copies, tensor memory, and the descriptors of tcgen05.mma.
#pragma once

#include <cstdint>

#include <cuda.h>

#include "mx_device.cuh"
#include "mx_host.h"

namespace costa {
namespace mx {

__device__ __forceinline__ uint32_t smem_addr(const void *p) {
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// An arrival at the same barrier of another block of the cluster.  What it
// announces is read by tensor cores, not by threads: the writer's
// fence.proxy.async (or tcgen05 fence) before it orders that, and a release at
// cluster scope would only stall the warp (measured: 2000 cycles each).
__device__ __forceinline__ void bar_arrive_at(uint32_t bar, uint32_t rank) {
    asm volatile(
        "{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\t"
        "mbarrier.arrive.shared::cluster.b64 _, [a];\n\t}" ::"r"(bar),
        "r"(rank)
        : "memory");
}
// Whether the phase of this parity is complete; the thread may be suspended for
// some milliseconds until it is (a thread that asks again and again takes issue
// slots from the others).
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t p;
    asm volatile(
        "{\n\t.reg .pred q;\n\tmbarrier.try_wait.parity.shared::cta.b64 q, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(p)
        : "r"(bar), "r"(parity), "r"(4000000u)
        : "memory");
    return p != 0;
}

// Every wait ends: after kWaitClocks (some seconds; the longest sound wait, for
// the products over the largest k, is below) it gives up and marks the block as
// failed, which ends the block's other waits too.  A failed block computes
// nothing more, lets its copies in flight land, frees its tensor memory and
// leaves; costa_mx_failures tells the host.
constexpr long long kWaitClocks = 8000000000ll;

__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t *failed) {
    if (bar_try(bar, parity)) return true;
    const long long start = clock64();
    while (!bar_try(bar, parity))
        if (*failed || clock64() - start > kWaitClocks) {
            *failed = 1;
            return false;
        }
    return true;
}

// A place in a ring of N stages and the parity of its barriers' current phase.
template <int N> struct Ring {
    int s = 0;
    uint32_t parity = 0;
    __device__ void next(int steps = 1) {  // fewer than N
        if ((s += steps) >= N) {
            s -= N;
            parity ^= 1;
        }
    }
};

// Some milliseconds, far longer than any copy in flight takes.
__device__ __forceinline__ void let_copies_land() {
    const long long start = clock64();
    while (clock64() - start < 10000000) __nanosleep(1000);
}

// ---- copies into shared memory ----

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
// The same box only as far as the L2: no data reach the block, so this may run before after_previous().
__device__ __forceinline__ void tma_prefetch_2d(const CUtensorMap *map, int x, int y) {
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}
// The same, counted at the barrier of block `rank` (of this pair of blocks).
__device__ __forceinline__ void tma_load_2d_at(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar,
                                               uint32_t rank) {
    asm volatile(
        "{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\t"
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, "
        "%3}], [a];\n\t}" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar), "r"(rank)
        : "memory");
}
// bytes: a multiple of 16; both addresses 16-byte aligned
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}

// ---- tensor memory ----

__device__ __forceinline__ void tmem_alloc(uint32_t *slot, uint32_t cols) {  // one whole warp
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(slot)), "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t *slot, uint32_t cols) {  // one warp of each block
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(slot)), "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void tmem_free_pair(uint32_t addr, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// To the barriers of the blocks in `mask` (bits are ranks in the cluster).
__device__ __forceinline__ void mma_commit_pair(uint32_t bar, uint32_t mask) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                     bar),
                 "h"(static_cast<uint16_t>(mask))
                 : "memory");
}
// 16 columns of this warp's 32 lanes, one lane to a thread
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
        "[%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}
// Waits for the loads so far; r, of one of them, is not used before.
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}

// ---- descriptors ----

// Shared-memory operand: 128-byte swizzle; strides in bytes.  K-major rows of
// 128 bytes: sbo = 1024 (8 rows), lbo unused.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t lbo, uint32_t sbo) {
    return uint64_t((addr >> 4) & 0x3fff) | uint64_t(lbo >> 4) << 16 | uint64_t(sbo >> 4) << 32 | uint64_t(1) << 46 |
           uint64_t(2) << 61;
}
// 32 rows of 16 bytes without swizzle (a tile of scales)
__device__ __forceinline__ uint64_t scales_desc(uint32_t addr) {
    return uint64_t((addr >> 4) & 0x3fff) | uint64_t(128 >> 4) << 32 | uint64_t(1) << 46;
}
// A tile of scales to 4 columns of tensor memory, the same for each quarter of its lanes.
__device__ __forceinline__ void scales_to_tmem(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

// D[128 x n] += A B^T over 64 elements of E2M1 with a scale for each 32.
__device__ __forceinline__ void mma_e2m1(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(uint32_t(accumulate))
        : "memory");
}
// The same for D[256 x n] by a pair of blocks: each holds 128 rows of A (with
// their scales) and of D, half of B's rows, and the scales of all of them.
__device__ __forceinline__ void scales_to_tmem_pair(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_e2m1_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa,
                                              uint32_t sfb, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(uint32_t(accumulate))
        : "memory");
}
// E2M1 x E2M1, scales of exponents only, m x n; which half of the scales' 4 bytes: 0 or 2.
__device__ __forceinline__ constexpr uint32_t idesc_e2m1(int m, int n, int half) {
    return uint32_t(half) << 4 | 1u << 7 | 1u << 10 | uint32_t(n >> 3) << 17 | 1u << 23 | uint32_t(m >> 4) << 24 |
           uint32_t(half) << 29;
}

// D[256 x n] += A B^T over 16 elements of bf16, both operands MN-major, by a
// pair of blocks: each holds 128 rows of A and of D, and half of B's rows.
__device__ __forceinline__ void mma_bf16_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(accumulate))
        : "memory");
}
// bf16 x bf16 to f32, 256 rows, both operands MN-major.
__device__ __forceinline__ constexpr uint32_t idesc_bf16_pair(int n) {
    return 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | uint32_t(n >> 3) << 17 | uint32_t(256 >> 4) << 24;
}

// ---- registers and clusters ----

// More (or fewer) registers for each thread of this warpgroup, from those that
// the block was launched with.
template <int N> __device__ __forceinline__ void more_registers() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N> __device__ __forceinline__ void fewer_registers() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 cluster_load(uint32_t addr, uint32_t rank) {
    uint32_t a;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a));
    return v;
}

// ---- the way out of tensor memory ----

// An output of row-major rows, `rows` x `cols`: out = alpha sum + beta out.
template <typename T> struct Output {
    T *p;
    int64_t ld, rows, cols;
    float alpha, beta;
    __device__ void put(int64_t row, int64_t col, float sum) const {
        T *at = p + row * ld + col;
        float v = alpha * sum;
        if (beta != 0.0f) v += beta * to_float(*at);
        *at = from_float<T>(v);
    }
    // The sums sum(0) .. sum(15) of 16 rows of a column, one by one: for a caller that holds many more.
    template <typename F> __device__ void put_each(int64_t row, int64_t col, F sum) const {
        if (col >= cols || row >= rows) return;
        T *at = p + row * ld + col;
        const int n = static_cast<int>(min(int64_t(16), rows - row));
#pragma unroll
        for (int i = 0; i < 16; ++i, at += ld)
            if (i < n) {
                float v = alpha * sum(i);
                if (beta != 0.0f) v += beta * to_float(*at);
                *at = from_float<T>(v);
            }
    }
    // The same, with what they are added to read first.
    template <typename F> __device__ void put16(int64_t row, int64_t col, F sum) const {
        if (col >= cols || row >= rows) return;
        T *at = p + row * ld + col;
        if (beta == 0.0f && row + 16 <= rows) {
#pragma unroll
            for (int i = 0; i < 16; ++i, at += ld) *at = from_float<T>(alpha * sum(i));
            return;
        }
        const int n = static_cast<int>(min(int64_t(16), rows - row));
        float old[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) old[i] = beta != 0.0f && i < n ? beta * to_float(at[i * ld]) : 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i, at += ld)
            if (i < n) *at = from_float<T>(alpha * sum(i) + old[i]);
    }
};

// Joins the partial sums of `split` <= MAX blocks of a cluster (at shared
// address `part` of the blocks first, first + step, ...), in that order; each of
// them, the index-th, writes a share with `threads` threads, of which this is
// the tid-th.  A cluster_sync() comes before this, and one after it before any
// block leaves.
template <int MAX, typename T>
__device__ __forceinline__ void join_split(const Output<T> &out, uint32_t part, int first, int step, int index, int split,
                                           int tid, int threads, int64_t row0, int64_t col0, int tile_rows) {
    // Four neighbouring columns at a time, and two such groups of all blocks on their way together: another block's
    // shared memory is some 700 cycles away.
    const int groups = static_cast<int>(min(int64_t(tile_rows), out.rows - row0)) * 32, stride = split * threads;
    for (int g = index * threads + tid; g < groups; g += 2 * stride) {
        float4 v[2][MAX];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < MAX; ++r)
                if (r < split && g + h * stride < groups) v[h][r] = cluster_load(part + 16 * (g + h * stride), first + r * step);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = g + h * stride;
            if (at >= groups) break;
            float4 sum = v[h][0];
#pragma unroll
            for (int r = 1; r < MAX; ++r)
                if (r < split) {
                    sum.x += v[h][r].x;
                    sum.y += v[h][r].y;
                    sum.z += v[h][r].z;
                    sum.w += v[h][r].w;
                }
            const int64_t row = row0 + at / 32, col = col0 + at % 32 * 4;
            const float each[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + i < out.cols) out.put(row, col + i, each[i]);
        }
    }
}

}  // namespace mx
}  // namespace costa
