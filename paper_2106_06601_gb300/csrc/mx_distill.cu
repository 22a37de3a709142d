// Distillation from a teacher's top logits: the loss of each row of logits and its
// gradient.
//
//   p = softmax(t / tau) over the K named columns,  q = softmax(z / tau) over all
//   loss = tau^2 sum_k p_k (log p_k - log q_k),     dz_j = g tau (q_j - p_j)
//
// A row lies in the registers of a block's threads, or of a cluster's of up to eight: each warp takes its largest logit m
// and s = sum exp((z - m) / tau), the pairs (m, s) are brought to one, log q_k = (z_k - m) / tau - log s, and the gradient
// is written as g tau q throughout, then again where the teacher names a column.  So a row is read once, its exponentials
// are computed twice, and several blocks to an SM overlap one's loads with another's sums and stores.  Longer rows are
// read twice.  4096 x 131072 bf16 takes 366 to 369 us, 5.8 TB/s; 13 instructions a logit, five of them conversions from and to
// bf16 and exponentials.  A ring in shared memory that read the next row ahead was no faster: reads are not what waits.
#include <algorithm>
#include <type_traits>

#include "costa_internal.h"
#include "mx_rows.cuh"
#include "mx_tc.cuh"

namespace costa {
namespace mx {
namespace {

// Groups of eight logits that a thread has at a time: 64 registers, or 32 in blocks of 1024 threads.
template <typename T, int THREADS> constexpr int kGroups = (THREADS == 1024 ? 32 : 64) / Eight<T>::kWords;
// Blocks of an SM at least: 640 threads of 102 registers (4096 x 131072 bf16: 366 us, with 512 of 128 418 us, with 768 of 85
// 373 us); f32 that has to be shifted needs more.
template <typename T, int THREADS, bool WHOLE>
constexpr int kLeastBlocks = THREADS == 1024 ? 1 : (WHOLE || sizeof(T) == 2 ? 640 : 512) / THREADS;
constexpr int kMostBlocks = 8;  // of a cluster

template <typename T> struct Distill {
    Rows<const T> z;
    Rows<T> dz;
    const int32_t *ids;
    int64_t ld_ids;
    const void *t;
    int64_t ld_t;
    int t_f32, top;
    float *loss, *stats;
    const float *g;
    int64_t ld_loss, ld_stats, ld_g;
    int64_t rows, cols;
    float scale, scale_low;  // log2(e) / tau, in two parts
    float tau;
    int64_t per;  // groups of a row to a block
};

template <int THREADS> struct Shared {
    float m[32], s[32], tm[32], ts[32], loss[32];
    float2 peers[kMostBlocks];
    bool some;   // whether the row names any column
    int own[32];  // of each warp's entries, those of columns in this block's part of the row; they come first in
    int id[THREADS];
    float p[THREADS], z[THREADS];
};

// 2^(d scale), that is exp(d / tau), for d <= 0 (or NaN).  For f32 logits the exponent's rounding, which would be some
// 1e-6 of the result at d = -20, is made up for.
template <typename T> __device__ __forceinline__ float exponential(float d, float scale, float low) {
    float e;
    if constexpr (sizeof(T) == 2) {
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(d * scale));
        return e;
    } else {
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(d) : "f"(-1e30f));  // so that the product's rounding is a number
        const float y = d * scale, rest = fmaf(d, low, fmaf(d, scale, -y));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(y));
        return fmaf(e, rest * 0.693147182f, e);
    }
}

// A pair (largest, sum of exponentials to it), joined over the warp's lanes.
template <typename T> __device__ __forceinline__ void join_warp(float &m, float &s, float scale, float low) {
    float top = m;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
    const float at = top == -INFINITY ? 0.0f : top;
    s = warp_sum(s == 0.0f ? 0.0f : s * exponential<T>(m - at, scale, low));
    m = top;
}
// The same over the warps' pairs of a block, or over a cluster's blocks'; after a barrier.
template <typename T> __device__ __forceinline__ void join_pairs(const float *ms, const float *ss, int n, float &m, float &s, float scale, float low) {
    const int lane = threadIdx.x % 32;
    m = lane < n ? ms[lane] : -INFINITY;
    s = lane < n ? ss[lane] : 0.0f;
    join_warp<T>(m, s, scale, low);
}

// Pairs of 32-bit numbers, which one instruction takes.
struct Two {
    uint64_t v;
    __device__ Two() {}
    __device__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ void get(float &a, float &b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ Two operator+(Two a, Two b) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Two operator*(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Two fma_two(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// exp((z - at) / tau) of two logits, but for a factor 2^rest that all of them lack: 2^(z scale - c) with c = at scale
// rounded to an integer, so that one operation of one rounding gives the exponent.
struct Powers {
    Two scale, minus;
    float rest;
    __device__ Powers(float at, float scale_) : scale(scale_, scale_) {
        const float c = rintf(at * scale_);
        minus = Two(-c, -c);
        rest = fmaf(-at, scale_, c);
    }
    __device__ Two operator()(Two z) const {
        float a, b;
        fma_two(z, scale, minus).get(a, b);
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
        return Two(a, b);
    }
    __device__ float lacking() const {
        float f;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(f) : "f"(rest));
        return f;
    }
};
// A largest logit this far from 0 (the type's lowest number in a row that is masked with it, say) leaves no such integer:
// its logits are taken less it before.
__device__ __forceinline__ bool far_off(float m, float scale) { return fabsf(m) * scale > 0x1p20f && fabsf(m) != INFINITY; }
__device__ __forceinline__ void less(Eight<float> &x, float m) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x.w[i] = __float_as_uint(x(i) - m);
}
__device__ __forceinline__ void less(Eight<__nv_bfloat16> &x, float m) {  // the next smaller number is 2^12 units of the exponent away
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x(i) == m ? 0.0f : x(i) - INFINITY;
    x.set(v);
}

// Logits 2 i and 2 i + 1 of a group.
template <typename T> __device__ __forceinline__ Two two_of(const Eight<T> &x, int i) { return Two(x(2 * i), x(2 * i + 1)); }

// The largest of a group's logits, and `m`.
struct Largest {
    float f;
    uint32_t pair;
    __device__ Largest() : f(-INFINITY), pair(0xff80ff80u) {}
    __device__ void take(const Eight<__nv_bfloat16> &x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("max.bf16x2 %0, %0, %1;" : "+r"(pair) : "r"(x.w[i]));
    }
    __device__ void take(const Eight<float> &x) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f = fmaxf(f, x(i));
    }
    __device__ float get() const { return fmaxf(f, fmaxf(low_of(pair), high_of(pair))); }
};

// A part of a row, in groups of eight: `groups` ones from the row's first-th on.  Groups lie on 16-byte boundaries, or
// (shift) that many elements before them: as those of a gradient do that lies otherwise than the logits with respect to
// 16 bytes.  I counts elements from the part's beginning.
template <typename T, typename I = int> struct Line {
    static constexpr int kPer = 16 / sizeof(T);
    int64_t from, to;  // the part's columns
    const T *z;        // on a 16-byte boundary: `shift` elements after the part's beginning
    I lo, hi;          // its first and last elements that are the row's
    I reach;           // pieces that begin (at z) before it hold some of the row
    bool ragged;       // some of its groups are so in part
    __device__ Line(const T *row, int64_t cols, int64_t first, int64_t groups, int shift = 0) {
        const int head = static_cast<int>(reinterpret_cast<uint64_t>(row) & 15) / static_cast<int>(sizeof(T));
        const int64_t begin = first * 8 - head - shift;
        z = row + (begin + shift);
        lo = static_cast<I>(max(int64_t(0), -begin));
        hi = cols == 0 ? 0 : static_cast<I>(max(int64_t(0), min(cols - begin, groups * 8)));
        reach = cols == 0 ? 0 : static_cast<I>(max(int64_t(0), min(cols - begin - shift, groups * 8)));
        from = begin + lo;
        to = begin + hi;
        ragged = lo != 0 || hi % 8 != 0;
    }
    // The group at `at`, by the whole 16-byte pieces that hold some of the row (that begin before `end`); or -infinity.
    __device__ void load(I at, I end, Eight<T> &x) const {
        constexpr uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
        for (int j = 0; j < Eight<T>::kWords / 4; ++j) {
            uint4 v = make_uint4(none, none, none, none);
            if (at + j * kPer < end) v = *reinterpret_cast<const uint4 *>(z + at + j * kPer);
            x.w[4 * j] = v.x;
            x.w[4 * j + 1] = v.y;
            x.w[4 * j + 2] = v.z;
            x.w[4 * j + 3] = v.w;
        }
    }
    // What is not the row's to -infinity.
    __device__ void cut(I at, Eight<T> &x) const {
        if (at >= lo && at + 8 <= hi) return;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at + i < lo || at + i >= hi) {
                if constexpr (sizeof(T) == 4)
                    x.w[i] = 0xff800000u;
                else
                    x.w[i / 2] = i % 2 ? (x.w[i / 2] & 0xffffu) | 0xff800000u : (x.w[i / 2] & 0xffff0000u) | 0xff80u;
            }
    }
    // Values of a group, `to` for the part's first.
    __device__ void store(T *to, I at, const Eight<T> &x) const {
        if (at >= lo && at + 8 <= hi) {
#pragma unroll
            for (int j = 0; j < Eight<T>::kWords; j += 4)
                reinterpret_cast<uint4 *>(to + at)[j / 4] = make_uint4(x.w[j], x.w[j + 1], x.w[j + 2], x.w[j + 3]);
        } else if (at < hi) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (at + i >= lo && at + i < hi) to[at + i] = from_float<T>(x(i));
        }
    }
};

// The gradient of a group: exponentials times a factor.
template <typename T> __device__ __forceinline__ Eight<T> gradient(const Eight<T> &x, const Powers &e, Two factor) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) (e(two_of(x, i)) * factor).get(v[2 * i], v[2 * i + 1]);
    Eight<T> out;
    out.set(v);
    return out;
}

// How far a row `to` lies after `row` with respect to 16 bytes, in elements.
template <typename T> __device__ __forceinline__ int shift_of(const T *row, const T *to) {
    return static_cast<int>((reinterpret_cast<uint64_t>(to) - reinterpret_cast<uint64_t>(row)) & 15) / static_cast<int>(sizeof(T));
}

// A part's groups in a block of THREADS threads; the j-th of this thread lies at element at(j).  WHOLE: all of the row's
// groups are whole and lie on 16-byte boundaries, those of the gradient too.
//
// Else groups lie as those of the gradient do: they begin `shift` elements before a 16-byte boundary of the logits, so each
// takes the last ones of the 16 bytes before its own from the lane before.  A warp's groups then all follow each other, 32
// times `rounds`, and only its first lane has to read those for itself.
template <typename T, int THREADS, bool WHOLE> struct Part {
    static constexpr int G = kGroups<T, THREADS>, kWords = Eight<T>::kWords, kPer = 16 / sizeof(T), kStep = WHOLE ? THREADS * 8 : 256;
    const Line<T> line;
    const int rounds, base, shift, room;  // room: elements before this thread's first group that the row has
    __device__ Part(const T *row, int64_t cols, int64_t first, int64_t groups, int shift_)
        : line(row, cols, first, groups, shift_), rounds((static_cast<int>(groups) + THREADS - 1) / THREADS),
          base((WHOLE ? threadIdx.x : threadIdx.x / 32 * rounds * 32 + threadIdx.x % 32) * 8), shift(shift_), room(first > 0 ? kPer : base) {}
    __device__ int at(int j) const { return base + j * kStep; }
    __device__ bool none(int j) const { return WHOLE ? j * kStep >= line.hi : j >= rounds; }  // for no thread
    __device__ void load(Eight<T> (&x)[G]) const {
        if constexpr (WHOLE) {
#pragma unroll
            for (int j = 0; j < G; ++j) line.load(at(j), line.hi, x[j]);
        } else {
            uint4 before = make_uint4(0, 0, 0, 0);
            if (shift && threadIdx.x % 32 == 0 && room > 0 && base < line.hi)
                before = *reinterpret_cast<const uint4 *>(line.z + base - kPer);
#pragma unroll
            for (int j = 0; j < G; ++j) line.load(at(j), j < rounds ? line.reach : 0, x[j]);
            if (shift) {
#pragma unroll
                for (int j = G - 1; j >= 0; --j) {
                    if (j >= rounds) continue;
                    uint32_t c[kWords + 4];  // the 16 bytes before, and mine
                    const bool last = threadIdx.x % 32 == 31;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t mine = x[j].w[kWords - 4 + i];
                        c[i] = __shfl_sync(~0u, j > 0 && last ? x[j > 0 ? j - 1 : 0].w[kWords - 4 + i] : mine, (threadIdx.x + 31) % 32);
                    }
                    if (j == 0 && threadIdx.x % 32 == 0) c[0] = before.x, c[1] = before.y, c[2] = before.z, c[3] = before.w;
#pragma unroll
                    for (int i = 0; i < kWords; ++i) c[4 + i] = x[j].w[i];
                    const int bytes = 16 - shift * static_cast<int>(sizeof(T));  // to where the group begins among them
                    const uint32_t bits = (bytes & 2) * 8;
                    if (bytes < 4)
                        from_word<T, 0>(c, bits, x[j].w);
                    else if (bytes < 8)
                        from_word<T, 1>(c, bits, x[j].w);
                    else if (bytes < 12)
                        from_word<T, 2>(c, bits, x[j].w);
                    else
                        from_word<T, 3>(c, bits, x[j].w);
                }
            }
        }
    }
    __device__ void cut(Eight<T> (&x)[G]) const {
        if constexpr (!WHOLE) {
            if (!line.ragged && shift == 0) return;  // (what was shifted beyond a part's end is the next one's)
#pragma unroll
            for (int j = 0; j < G; ++j)
                if (j < rounds) line.cut(at(j), x[j]);
        }
    }
    // The gradient of the part, or zeros.
    __device__ void write(T *dz, const Eight<T> (&x)[G], const Powers &e, float factor, bool some) const {
        factor *= e.lacking();
        const Two two(factor, factor);
        T *const to = dz + (line.from - line.lo);
        if (__builtin_expect(!some, 0)) {
            Eight<T> zeros;
            zeros.clear();
#pragma unroll
            for (int j = 0; j < G; ++j)
                if (!none(j)) line.store(to, at(j), zeros);
            return;
        }
#pragma unroll
        for (int j = 0; j < G; ++j) {
            if (none(j)) break;
            const Eight<T> out = gradient(x[j], e, two);
            if constexpr (WHOLE) {
                if (at(j) < line.hi)
#pragma unroll
                    for (int k = 0; k < kWords; k += 4)
                        reinterpret_cast<uint4 *>(to + at(j))[k / 4] = make_uint4(out.w[k], out.w[k + 1], out.w[k + 2], out.w[k + 3]);
            } else {
                line.store(to, at(j), out);
            }
        }
    }
};

// An entry of the teacher's, of which there are no more than threads.  It is asked for before the row's logits are, and the
// logit of its column once that is known, which is put down when the row's logits have been taken.
template <typename T> struct Entry {
    int id;
    float t, p;
    T z;
    bool has_z, own;
    __device__ void ask(const Distill<T> &d, int64_t row) {
        const int k = threadIdx.x;
        id = -1;
        t = -INFINITY;
        p = 0.0f;
        has_z = own = false;
        if (k >= d.top) return;
        id = d.ids[row * d.ld_ids + k];
        const int64_t at = row * d.ld_t + k;
        t = d.t_f32 ? static_cast<const float *>(d.t)[at] : to_float(static_cast<const __nv_bfloat16 *>(d.t)[at]);
    }
};

// The sum of the entries' exponentials, this entry's probability, and whether its column is one of from .. to - 1; its logit
// is asked for then, or always (all).  Warps without entries pass by.  put_down() and a barrier come after it.
template <typename T, int N>
__device__ __forceinline__ float teacher(const Distill<T> &d, int64_t row, Shared<N> &sh, Entry<T> &e, bool all, int64_t from, int64_t to) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
    float tm = -INFINITY, ts = 0.0f, power = 0.0f;
    if (warp * 32 < d.top) {
        const bool names = e.id >= 0 && e.id < d.cols && e.t != -INFINITY;
        e.own = names && e.id >= from && e.id < to;
        e.has_z = names && (all || e.own);
        if (e.has_z) e.z = *d.z.at(row, e.id);
        tm = names ? fmaxf(e.t, -INFINITY) : -INFINITY;  // (not NaN)
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) tm = fmaxf(tm, __shfl_xor_sync(~0u, tm, k));
        power = names ? exponential<float>(e.t - (tm == -INFINITY ? 0.0f : tm), d.scale, d.scale_low) : 0.0f;
        ts = warp_sum(power);
    }
    const float mine = tm;
    if (d.top > 32) {  // several warps have some
        if (lane == 0) {
            sh.tm[warp] = tm;
            sh.ts[warp] = ts;
        }
        __syncthreads();
        if (warp * 32 < d.top) join_pairs<float>(sh.tm, sh.ts, warps, tm, ts, d.scale, d.scale_low);
    }
    if (threadIdx.x == 0) sh.some = ts != 0.0f;
    if (mine != -INFINITY)
        e.p = power * __fdiv_rn(exponential<float>(mine - tm, d.scale, d.scale_low), ts);
    else if (power != 0.0f)
        e.p = power;  // NaN
    e.t -= tm;
    return ts;
}
template <typename T, int N> __device__ __forceinline__ void put_down(const Distill<T> &d, Shared<N> &sh, const Entry<T> &e) {
    if (static_cast<int>(threadIdx.x) / 32 * 32 >= d.top) return;
    const int lane = threadIdx.x % 32;
    const uint32_t own = __ballot_sync(~0u, e.own);
    if (e.own) {
        const int at = (threadIdx.x - lane) + __popc(own & ((1u << lane) - 1));
        sh.id[at] = e.id;
        sh.p[at] = e.p;
        sh.z[at] = to_float(e.z);
    }
    if (lane == 0) sh.own[threadIdx.x / 32] = __popc(own);
}

// The warps' parts of the loss over tau, to shared memory; a barrier, and write_loss() by a thread.  tau times a logarithm
// of a probability is the logit's distance less tau log s: nothing is divided, so no tau takes it out of range.
template <typename T, int N> __device__ __forceinline__ void loss_part(const Distill<T> &d, Shared<N> &sh, const Entry<T> &e, float m, float s, float ts) {
    const int warp = threadIdx.x / 32;
    if (warp * 32 >= d.top) return;
    // (where p underflows its term counts nothing)
    const float term = e.p != 0.0f ? e.p * ((e.t - (to_float(e.z) - m)) + d.tau * (logf(s) - logf(ts))) : 0.0f;
    const float sum = warp_sum(term);
    if (threadIdx.x % 32 == 0) sh.loss[warp] = sum;
}
template <typename T, int N> __device__ __forceinline__ void write_loss(const Distill<T> &d, int64_t row, const Shared<N> &sh, float m, float s) {
    float sum = 0.0f;
    for (int w = 0; w * 32 < d.top; ++w) sum += sh.loss[w];
    d.loss[row * d.ld_loss] = sh.some ? d.tau * sum : 0.0f;
    d.stats[row * d.ld_stats] = m;
    d.stats[row * d.ld_stats + 1] = s;
}

// The gradient at the own columns, once for each of them (the first entry that names it adds the others'), after the rest
// is written and a barrier.
template <typename T, int N> __device__ __forceinline__ void named(const Distill<T> &d, int64_t row, const Shared<N> &sh, float m, float inverse, float slope) {
    const int mine = threadIdx.x;
    if (mine >= d.top || mine % 32 >= sh.own[mine / 32]) return;
    const int id = sh.id[mine];
    bool first = true;
    float sum = 0.0f;
    for (int w = 0; w * 32 < d.top; ++w)
        for (int j = w * 32, end = j + sh.own[w]; j < end; ++j)
            if (sh.id[j] == id) {
                first = first && j >= mine;
                sum += sh.p[j];
            }
    if (!first) return;
    const float q = exponential<T>(sh.z[mine] - m, d.scale, d.scale_low) * inverse;
    *d.dz.at(row, id) = from_float<T>(slope * (q - sum));
}

__device__ __forceinline__ void cluster_store(const float2 *at, uint32_t rank, float2 v) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(at)), "r"(rank));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(a), "f"(v.x), "f"(v.y) : "memory");
}

// All blocks of a cluster have started once every one of them has arrived, which each does first of all.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }

// A row's pair from its blocks' warps', after a barrier and with one.  The first warp brings a block's together.
template <typename T, int N> __device__ __forceinline__ void join_row(const Distill<T> &p, Shared<N> &sh, int blocks, int rank, float &m, float &s) {
    const int lane = threadIdx.x % 32;
    if (threadIdx.x < 32) join_pairs<T>(sh.m, sh.s, blockDim.x / 32, m, s, p.scale, p.scale_low);
    if (blocks == 1) {
        if (threadIdx.x == 0) sh.peers[0] = make_float2(m, s);
        __syncthreads();
        m = sh.peers[0].x;
        s = sh.peers[0].y;
    } else {
        cluster_wait();
        if (static_cast<int>(threadIdx.x) < blocks) cluster_store(&sh.peers[rank], threadIdx.x, make_float2(m, s));
        cluster_sync();
        const float2 v = lane < blocks ? sh.peers[lane] : make_float2(-INFINITY, 0.0f);
        m = v.x;
        s = v.y;
        join_warp<T>(m, s, p.scale, p.scale_low);
    }
}

// A row's loss and gradient by a block or a cluster of 2^log_blocks, each thread up to kGroups groups.  Latency bounds it:
// half of the issue slots and 86% of the memory's rate are used, the barriers of a cluster lie between a row's two passes.
template <typename T, bool WHOLE, int THREADS>
__global__ void __launch_bounds__(THREADS, (kLeastBlocks<T, THREADS, WHOLE>)) distill_kernel(const Distill<T> p, const int log_blocks) {
    __shared__ Shared<THREADS> sh;
    constexpr int G = kGroups<T, THREADS>;
    const int blocks = 1 << log_blocks;
    if (blocks > 1) cluster_arrive();
    let_next_start();
    const int rank = blocks > 1 ? static_cast<int>(cluster_rank()) : 0, warp = threadIdx.x / 32;
    const int64_t row = blockIdx.x >> log_blocks;
    after_previous();
    Entry<T> mine;
    mine.ask(p, row);
    float g;  // here, not after the barriers
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(g) : "l"(p.g + row * p.ld_g));
    const Part<T, THREADS, WHOLE> part(p.z.at(row, 0), p.cols, rank * p.per, p.per,
                                         WHOLE ? 0 : shift_of<T>(p.z.at(row, 0), p.dz.at(row, 0)));
    Eight<T> x[G];
    part.load(x);
    const float ts = teacher(p, row, sh, mine, rank == 0, part.line.from, part.line.to);  // (the first block takes the loss)
    part.cut(x);
    Largest largest;
#pragma unroll
    for (int j = 0; j < G; ++j) largest.take(x[j]);
    float m = largest.get(), s;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
    const float own = m;  // the warp's
    const bool far = far_off(own, p.scale);
    if (__builtin_expect(far, 0))
#pragma unroll
        for (int j = 0; j < G; ++j) less(x[j], own);
    {
        const Powers e(far || own == -INFINITY ? 0.0f : own, p.scale);
        Two sum(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < G; ++j) {
            if (part.none(j)) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum = sum + e(two_of(x[j], i));
        }
        float a, b;
        sum.get(a, b);
        s = warp_sum(a + b) * e.lacking();
        if (threadIdx.x % 32 == 0) {
            sh.m[warp] = own;
            sh.s[warp] = s;
        }
    }
    put_down(p, sh, mine);
    __syncthreads();
    join_row(p, sh, blocks, rank, m, s);
    const float inverse = __fdiv_rn(1.0f, s), slope = p.tau * g;
    // (so that the compiler does not keep the logits of the first pass in 32 bits)
#pragma unroll
    for (int j = 0; j < G; ++j)
#pragma unroll
        for (int i = 0; i < Eight<T>::kWords; ++i) asm volatile("" : "+r"(x[j].w[i]));
    // From the warp's largest where it has been taken off, or the row's leaves no exponent.
    const bool none = far || own == -INFINITY, apart = none || far_off(m, p.scale);
    const float factor = apart ? slope * inverse * exponential<T>(own - m, p.scale, p.scale_low) : slope * inverse;
    part.write(p.dz.at(row, 0), x, Powers(none ? 0.0f : apart ? own : m, p.scale), factor, sh.some);
    if (rank == 0) loss_part(p, sh, mine, m, s, ts);
    __syncthreads();
    if (rank == 0 && threadIdx.x == blockDim.x - 1) write_loss(p, row, sh, m, s);
    named(p, row, sh, m, inverse, slope);
}

// Loss and statistics of a row by a block or a cluster of 2^log_blocks: each thread goes over its groups, with its own
// largest logit so far, and asks for the next ones before it takes those that it has.  4096 x 32000 bf16: 45 us, 5.8 TB/s;
// what is left are the pauses between a block's rows.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) distill_loss_kernel(const Distill<T> p, const int log_blocks) {
    __shared__ Shared<THREADS> sh;
    constexpr int G = 16 / Eight<T>::kWords;
    const int blocks = 1 << log_blocks;
    if (blocks > 1) cluster_arrive();
    let_next_start();
    const int rank = blocks > 1 ? static_cast<int>(cluster_rank()) : 0, warp = threadIdx.x / 32;
    const int64_t row = blockIdx.x >> log_blocks;
    after_previous();
    Entry<T> mine;
    mine.ask(p, row);
    const Line<T, int64_t> line(p.z.at(row, 0), p.cols, rank * p.per, p.per);
    constexpr int kStep = THREADS * 8;
    int64_t at = threadIdx.x * 8;
    Eight<T> next[G];
#pragma unroll
    for (int j = 0; j < G; ++j) line.load(at + j * kStep, line.hi, next[j]);
    const float ts = teacher(p, row, sh, mine, rank == 0, line.from, line.to);
    float m = -INFINITY, s = 0.0f;
    for (; at < line.hi; at += G * kStep) {
        Eight<T> x[G];
#pragma unroll
        for (int j = 0; j < G; ++j) {
            x[j] = next[j];
            line.load(at + (G + j) * kStep, line.hi, next[j]);
        }
        Largest largest;
#pragma unroll
        for (int j = 0; j < G; ++j) {
            if (line.ragged) line.cut(at + j * kStep, x[j]);
            largest.take(x[j]);
        }
        const float top = fmaxf(m, largest.get()), about = top == -INFINITY ? 0.0f : top;
        if (top > m) s *= exponential<T>(m - about, p.scale, p.scale_low);
        m = top;
        const bool far = far_off(about, p.scale);
        if (__builtin_expect(far, 0))
#pragma unroll
            for (int j = 0; j < G; ++j) less(x[j], about);
        const Powers e(far ? 0.0f : about, p.scale);
        Two sum(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < G; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum = sum + e(two_of(x[j], i));
        float a, b;
        sum.get(a, b);
        s = fmaf(a + b, e.lacking(), s);
    }
    __syncwarp();
    join_warp<T>(m, s, p.scale, p.scale_low);
    if (threadIdx.x % 32 == 0) {
        sh.m[warp] = m;
        sh.s[warp] = s;
    }
    put_down(p, sh, mine);
    __syncthreads();
    join_row(p, sh, blocks, rank, m, s);
    if (rank != 0) return;
    loss_part(p, sh, mine, m, s, ts);
    __syncthreads();
    if (threadIdx.x == THREADS - 1) write_loss(p, row, sh, m, s);
}

// The gradient of a part of a row, from its statistics.  4096 x 32000 bf16: 77 us, 6.8 TB/s, at memory speed.
template <typename T, bool WHOLE, int THREADS>
__global__ void __launch_bounds__(THREADS, (kLeastBlocks<T, THREADS, WHOLE>)) distill_backward_kernel(const Distill<T> p, const unsigned parts) {
    __shared__ Shared<THREADS> sh;
    let_next_start();
    const unsigned row_ = blockIdx.x / parts;
    const int64_t row = row_;
    after_previous();
    Entry<T> mine;
    mine.ask(p, row);
    const Part<T, THREADS, WHOLE> part(p.z.at(row, 0), p.cols, int64_t(blockIdx.x - row_ * parts) * p.per, p.per,
                                         WHOLE ? 0 : shift_of<T>(p.z.at(row, 0), p.dz.at(row, 0)));
    Eight<T> x[kGroups<T, THREADS>];
    part.load(x);
    const float m = p.stats[row * p.ld_stats], s = p.stats[row * p.ld_stats + 1], slope = p.tau * p.g[row * p.ld_g];
    teacher(p, row, sh, mine, false, part.line.from, part.line.to);
    put_down(p, sh, mine);
    __syncthreads();
    const float inverse = __fdiv_rn(1.0f, s);
    const bool far = far_off(m, p.scale);
    if (__builtin_expect(far, 0))
#pragma unroll
        for (int j = 0; j < kGroups<T, THREADS>; ++j) less(x[j], m);
    part.write(p.dz.at(row, 0), x, Powers(far ? 0.0f : m, p.scale), slope * inverse, sh.some);
    __syncthreads();
    named(p, row, sh, m, inverse, slope);
}

// ---- launches ----

// Groups that a row may touch.
template <typename T> int64_t groups_of(const Distill<T> &p, bool whole) {
    constexpr int kMore = 16 / sizeof(T) - 1;  // elements before the row, and of the shift
    return mx_ceil(p.cols + (whole ? 0 : 2 * kMore), 8);
}

template <typename T> cudaError_t launch_loss(Distill<T> p, bool whole, cudaStream_t s) {
    const int64_t groups = groups_of(p, whole);
    int log_blocks = 0;
    while ((1 << log_blocks) < kMostBlocks && p.rows << (log_blocks + 1) <= 304 && groups >= 256 << log_blocks) ++log_blocks;
    p.per = mx_ceil(groups, 1 << log_blocks);
    const auto launch = [&](auto threads) {
        return mx_launch(distill_loss_kernel<T, decltype(threads)::value>, p.rows << log_blocks, threads, 0, 1 << log_blocks, s, p, log_blocks);
    };
    // Rows that fill the SMs 16 at a time each take two warps: fewer wait for each other (4096 x 32000 bf16: 45 us, with
    // eight warps 50 us).
    if (p.rows >= 16 * 152 && p.top <= 64) return launch(std::integral_constant<int, 64>());
    return p.top <= 256 ? launch(std::integral_constant<int, 256>()) : launch(std::integral_constant<int, 1024>());
}

template <typename T, bool WHOLE> cudaError_t launch_backward(Distill<T> p, cudaStream_t s) {
    const int64_t groups = groups_of(p, WHOLE);
    const auto launch = [&](auto threads) {
        constexpr int N = decltype(threads)::value;
        // more parts where there are few rows
        const int64_t parts = std::max(mx_ceil(groups, N * kGroups<T, N>), std::min<int64_t>(mx_ceil(groups, N), 608 / p.rows));
        p.per = mx_ceil(groups, parts);
        return mx_launch(distill_backward_kernel<T, WHOLE, N>, p.rows * parts, N, 0, 1, s, p, static_cast<unsigned>(parts));
    };
    return p.top <= 128 ? launch(std::integral_constant<int, 128>()) : launch(std::integral_constant<int, 1024>());
}

// In one kernel where a cluster of blocks of 128 threads holds a row (five of them overlap on an SM) and they are no fewer
// than the teacher's entries; else in two (1000 x 200000 f32: 357 us, by a cluster of blocks of 512 threads 545 us).  More
// entries take blocks of 1024 threads, one to an SM: 4096 x 32000 bf16 with 128 entries 102 us, with 200 250 us.
template <typename T, bool WHOLE> cudaError_t launch_both(Distill<T> p, cudaStream_t s) {
    using std::integral_constant;
    constexpr int kMost = 128;
    const int64_t groups = groups_of(p, WHOLE);
    if (groups > kMost * kGroups<T, kMost> * kMostBlocks || p.top > kMost) {
        const cudaError_t e = launch_loss(p, WHOLE, s);
        return e == cudaSuccess ? launch_backward<T, WHOLE>(p, s) : e;
    }
    int log_blocks = 0;
    while (groups > int64_t(kMost) * kGroups<T, kMost> << log_blocks) ++log_blocks;
    // few rows: more blocks, and fewer groups to a thread
    while ((1 << log_blocks) < kMostBlocks && p.rows << (log_blocks + 1) <= 152 && groups >= 256 << log_blocks) ++log_blocks;
    p.per = mx_ceil(groups, 1 << log_blocks);
    const int64_t threads = p.rows << log_blocks <= 304 ? p.per : mx_ceil(p.per, kGroups<T, kMost>);
    const auto launch = [&](auto n) {
        return mx_launch(distill_kernel<T, WHOLE, decltype(n)::value>, p.rows << log_blocks, n, 0, 1 << log_blocks, s, p, log_blocks);
    };
    return threads <= 64 && p.top <= 64 ? launch(integral_constant<int, 64>()) : launch(integral_constant<int, kMost>());
}

template <typename T>
cudaError_t distill(const costa_mx_dense &Z, const costa_mx_index &ids, const costa_mx_dense &L, float tau, const costa_mx_dense *loss,
                    const costa_mx_dense &stats, const costa_mx_dense *G, const costa_mx_dense *dZ, cudaStream_t s) {
    const double scale = 1.4426950408889634 / static_cast<double>(tau);
    Distill<T> p{};
    p.z = rows_of<const T>(&Z);
    p.dz = rows_of<T>(dZ);
    p.ids = ids.ptr;
    p.ld_ids = ids.ld;
    p.t = L.ptr;
    p.ld_t = L.ld;
    p.t_f32 = L.type == COSTA_MX_F32;
    p.top = static_cast<int>(ids.cols);
    if (loss) {
        p.loss = static_cast<float *>(loss->ptr);
        p.ld_loss = loss->ld;
    }
    p.stats = static_cast<float *>(stats.ptr);
    p.ld_stats = stats.ld;
    if (G) {
        p.g = static_cast<const float *>(G->ptr);
        p.ld_g = G->ld;
    }
    p.rows = Z.rows;
    p.cols = Z.cols;
    p.scale = static_cast<float>(scale);
    p.scale_low = static_cast<float>(scale - static_cast<double>(p.scale));
    p.tau = tau;
    const bool whole = aligned16(&Z) && aligned16(dZ) && p.cols % 8 == 0;
    if (!loss) return whole ? launch_backward<T, true>(p, s) : launch_backward<T, false>(p, s);
    if (!dZ || p.cols == 0) return launch_loss(p, whole, s);  // (no columns: nothing of a gradient to write)
    return whole ? launch_both<T, true>(p, s) : launch_both<T, false>(p, s);
}

}  // namespace
}  // namespace mx

cudaError_t launch_mx_distill(const costa_mx_dense &Z, const costa_mx_index &ids, const costa_mx_dense &L, float tau,
                              const costa_mx_dense *loss, const costa_mx_dense &stats, const costa_mx_dense *G, const costa_mx_dense *dZ,
                              cudaStream_t s) {
    return Z.type == COSTA_MX_F32 ? mx::distill<float>(Z, ids, L, tau, loss, stats, G, dZ, s)
                                  : mx::distill<__nv_bfloat16>(Z, ids, L, tau, loss, stats, G, dZ, s);
}

}  // namespace costa
