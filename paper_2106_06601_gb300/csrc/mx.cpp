// Entry points of the low-bit matrices: every check of arguments, then one
// launch.  Nothing is kept between calls.
#include <cuda.h>
#include <cuda_runtime_api.h>

#include <cstdarg>
#include <cstdio>

#include "costa_internal.h"
#include "mx.h"
#include "mx_host.h"

namespace {

using namespace costa;

constexpr int64_t kMaxExtent = (int64_t(1) << 31) - 256, kMaxLd = int64_t(1) << 38;
constexpr int64_t kMaxElements = int64_t(1) << 48;  // rows * ld

costa_status bad(costa_status s, const char *fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return report_error(s, buf);
}

costa_status done(cudaError_t e, const char *what) {
    return e == cudaSuccess ? COSTA_OK : bad(COSTA_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

int64_t esize(const costa_mx_dense &d) { return d.type == COSTA_MX_F32 ? 4 : 2; }

costa_status check_dense(const costa_mx_dense *d, const char *name) {
    if (!d) return bad(COSTA_ERR_INVALID_ARG, "%s is null", name);
    if (d->type != COSTA_MX_F32 && d->type != COSTA_MX_BF16)
        return bad(COSTA_ERR_INVALID_ARG, "%s: unknown type %d", name, d->type);
    if (d->reserved != 0) return bad(COSTA_ERR_INVALID_ARG, "%s: reserved is not 0", name);
    if (d->rows < 0 || d->cols < 0 || d->rows > kMaxExtent || d->cols > kMaxExtent)
        return bad(COSTA_ERR_INVALID_ARG, "%s: extents %lld x %lld out of range", name, (long long)d->rows,
                   (long long)d->cols);
    if (d->rows == 0 || d->cols == 0) return COSTA_OK;
    if (d->ld < d->cols || d->ld >= kMaxLd)
        return bad(COSTA_ERR_LAYOUT, "%s: ld %lld for %lld columns", name, (long long)d->ld, (long long)d->cols);
    if (d->ld > kMaxElements / d->rows)
        return bad(COSTA_ERR_LAYOUT, "%s: %lld rows of %lld elements leave the address space", name,
                   (long long)d->rows, (long long)d->ld);
    if (!d->ptr) return bad(COSTA_ERR_INVALID_ARG, "%s: null pointer", name);
    if (reinterpret_cast<uint64_t>(d->ptr) % esize(*d))
        return bad(COSTA_ERR_LAYOUT, "%s: pointer not aligned to its elements", name);
    return COSTA_OK;
}

int64_t least_ld(int format, int64_t cols) { return mx_blocks(cols) * (format == COSTA_MX_E2M1 ? 16 : 32); }

int64_t scale_bytes_of(int format, int64_t rows, int64_t cols) {
    return format == COSTA_MX_E2M1 ? mx_ceil(rows, 128) * mx_scale_tiles(cols) * 512 : rows * mx_scale_pitch(cols);
}

costa_status check_matrix(const costa_mx_matrix *q, const char *name) {
    if (!q) return bad(COSTA_ERR_INVALID_ARG, "%s is null", name);
    if (q->format != COSTA_MX_E2M1 && q->format != COSTA_MX_I8)
        return bad(COSTA_ERR_INVALID_ARG, "%s: unknown format %d", name, q->format);
    if (q->reserved != 0) return bad(COSTA_ERR_INVALID_ARG, "%s: reserved is not 0", name);
    if (q->rows < 0 || q->cols < 0 || q->rows > kMaxExtent || q->cols > kMaxExtent)
        return bad(COSTA_ERR_INVALID_ARG, "%s: extents %lld x %lld out of range", name, (long long)q->rows,
                   (long long)q->cols);
    if (q->rows == 0 || q->cols == 0) return COSTA_OK;
    if (q->ld < least_ld(q->format, q->cols) || q->ld % 16 || q->ld >= kMaxLd)
        return bad(COSTA_ERR_LAYOUT, "%s: ld %lld bytes for %lld columns (a multiple of 16, %lld at least)", name,
                   (long long)q->ld, (long long)q->cols, (long long)least_ld(q->format, q->cols));
    if (q->ld > kMaxElements / q->rows)
        return bad(COSTA_ERR_LAYOUT, "%s: %lld rows of %lld bytes leave the address space", name, (long long)q->rows,
                   (long long)q->ld);
    if (!q->codes || !q->scales) return bad(COSTA_ERR_INVALID_ARG, "%s: null pointer", name);
    if (reinterpret_cast<uint64_t>(q->codes) % 16 || reinterpret_cast<uint64_t>(q->scales) % 16)
        return bad(COSTA_ERR_LAYOUT, "%s: codes and scales must be 16-byte aligned", name);
    return COSTA_OK;
}

using AttrsFn = CUresult (*)(unsigned int, CUpointer_attribute *, void **, CUdeviceptr);

AttrsFn attrs_fn() {
    static const AttrsFn fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q{};
        if (cudaGetDriverEntryPointByVersion("cuPointerGetAttributes", &f, 12000, cudaEnableDefault, &q) !=
                cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<AttrsFn>(f);
    }();
    return fn;
}

// Whether the bytes [p, p + bytes) are memory of the current device: in one
// allocation, or in mappings that follow each other without a gap (as a pool
// that grows by mapping more memory has).  Host and managed memory is refused:
// the products' bulk copies take device memory.
costa_status check_bytes(const void *p, int64_t bytes, int dev, const char *name) {
    AttrsFn fn = attrs_fn();
    if (!fn) return bad(COSTA_ERR_CUDA, "no CUDA driver");
    CUdeviceptr a = reinterpret_cast<CUdeviceptr>(p);
    const CUdeviceptr end = a + static_cast<uint64_t>(bytes);
    for (int mappings = 0; a < end; ++mappings) {
        unsigned int type = 0, managed = 0;
        int ordinal = -1;
        CUdeviceptr start = 0;
        size_t size = 0;
        CUpointer_attribute what[5] = {CU_POINTER_ATTRIBUTE_MEMORY_TYPE, CU_POINTER_ATTRIBUTE_DEVICE_ORDINAL,
                                       CU_POINTER_ATTRIBUTE_RANGE_START_ADDR, CU_POINTER_ATTRIBUTE_RANGE_SIZE,
                                       CU_POINTER_ATTRIBUTE_IS_MANAGED};
        void *out[5] = {&type, &ordinal, &start, &size, &managed};
        const bool known = fn(5, what, out, a) == CUDA_SUCCESS && type != 0;
        if (mappings == 0 && (!known || type != CU_MEMORYTYPE_DEVICE || managed))
            return bad(COSTA_ERR_LAYOUT, "%s: not device memory", name);
        if (!known || type != CU_MEMORYTYPE_DEVICE || managed || size == 0 || a < start || a >= start + size ||
            mappings > 65536)
            return bad(COSTA_ERR_LAYOUT, "%s: %lld bytes from its pointer leave the allocation", name, (long long)bytes);
        if (ordinal != dev)
            return bad(COSTA_ERR_LAYOUT, "%s: memory of device %d, not of the current device %d", name, ordinal, dev);
        a = start + size;
    }
    return COSTA_OK;
}

// Access checks of a call's matrices, after all other checks.
struct Access {
    int dev = -1;
    costa_status st = COSTA_OK;
    Access() {
        const cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) {
            cudaGetLastError();
            st = done(e, "cudaGetDevice");
        }
    }
    Access &dense(const costa_mx_dense *d, const char *name) {
        if (st == COSTA_OK && d && d->rows > 0 && d->cols > 0)
            st = check_bytes(d->ptr, ((d->rows - 1) * d->ld + d->cols) * esize(*d), dev, name);
        return *this;
    }
    Access &codes(const costa_mx_matrix *q, const char *name) {
        if (st != COSTA_OK || !q || q->rows == 0 || q->cols == 0) return *this;
        st = check_bytes(q->codes, (q->rows - 1) * q->ld + least_ld(q->format, q->cols), dev, name);
        if (st == COSTA_OK) st = check_bytes(q->scales, scale_bytes_of(q->format, q->rows, q->cols), dev, name);
        return *this;
    }
};

costa_status same_extents(int64_t r1, int64_t c1, const char *n1, int64_t r2, int64_t c2, const char *n2) {
    if (r1 == r2 && c1 == c2) return COSTA_OK;
    return bad(COSTA_ERR_SHAPE, "%s is %lld x %lld, %s %lld x %lld", n1, (long long)r1, (long long)c1, n2, (long long)r2,
               (long long)c2);
}

#define COSTA_MX_CHECK(call)               \
    do {                                   \
        const costa_status st_ = (call);   \
        if (st_ != COSTA_OK) return st_;   \
    } while (0)

}  // namespace

extern "C" {

costa_status costa_mx_sizes(costa_mx_format format, int64_t rows, int64_t cols, int64_t *ld, int64_t *code_bytes,
                            int64_t *scale_bytes) {
    if (format != COSTA_MX_E2M1 && format != COSTA_MX_I8)
        return bad(COSTA_ERR_INVALID_ARG, "unknown format %d", static_cast<int>(format));
    if (rows < 0 || cols < 0 || rows > kMaxExtent || cols > kMaxExtent)
        return bad(COSTA_ERR_INVALID_ARG, "extents %lld x %lld out of range", (long long)rows, (long long)cols);
    if (ld) *ld = least_ld(format, cols);
    if (code_bytes) *code_bytes = rows * least_ld(format, cols);
    if (scale_bytes) *scale_bytes = cols ? scale_bytes_of(format, rows, cols) : 0;
    return COSTA_OK;
}

costa_status costa_mx_quantize(const costa_mx_dense *X, costa_op op, const costa_mx_matrix *Q, void *stream) {
    COSTA_MX_CHECK(check_dense(X, "X"));
    COSTA_MX_CHECK(check_matrix(Q, "Q"));
    if (op != COSTA_OP_N && op != COSTA_OP_T && op != COSTA_OP_C)
        return bad(COSTA_ERR_INVALID_ARG, "unknown op %d", static_cast<int>(op));
    const bool n = op == COSTA_OP_N;
    COSTA_MX_CHECK(same_extents(Q->rows, Q->cols, "Q", n ? X->rows : X->cols, n ? X->cols : X->rows, "op(X)"));
    if (X->rows == 0 || X->cols == 0) return COSTA_OK;
    COSTA_MX_CHECK(Access().dense(X, "X").codes(Q, "Q").st);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return done(n ? launch_mx_quantize_n(*X, *Q, s) : launch_mx_quantize_t(*X, nullptr, *Q, s), "costa_mx_quantize");
}

costa_status costa_mx_quantize_both(const costa_mx_dense *X, const costa_mx_matrix *QN, const costa_mx_matrix *QT,
                                    void *stream) {
    COSTA_MX_CHECK(check_dense(X, "X"));
    COSTA_MX_CHECK(check_matrix(QN, "QN"));
    COSTA_MX_CHECK(check_matrix(QT, "QT"));
    if (QN->format != QT->format) return bad(COSTA_ERR_DTYPE, "QN and QT have different formats");
    COSTA_MX_CHECK(same_extents(QN->rows, QN->cols, "QN", X->rows, X->cols, "X"));
    COSTA_MX_CHECK(same_extents(QT->rows, QT->cols, "QT", X->cols, X->rows, "X's transpose"));
    if (X->rows == 0 || X->cols == 0) return COSTA_OK;
    COSTA_MX_CHECK(Access().dense(X, "X").codes(QN, "QN").codes(QT, "QT").st);
    return done(launch_mx_quantize_t(*X, QN, *QT, static_cast<cudaStream_t>(stream)), "costa_mx_quantize_both");
}

costa_status costa_mx_dequantize(const costa_mx_matrix *Q, const costa_mx_dense *Y, void *stream) {
    COSTA_MX_CHECK(check_matrix(Q, "Q"));
    COSTA_MX_CHECK(check_dense(Y, "Y"));
    COSTA_MX_CHECK(same_extents(Q->rows, Q->cols, "Q", Y->rows, Y->cols, "Y"));
    if (Q->rows == 0 || Q->cols == 0) return COSTA_OK;
    COSTA_MX_CHECK(Access().codes(Q, "Q").dense(Y, "Y").st);
    return done(launch_mx_dequantize(*Q, *Y, static_cast<cudaStream_t>(stream)), "costa_mx_dequantize");
}

costa_status costa_mx_product(const costa_mx_matrix *A, const costa_mx_matrix *B, float alpha, float beta,
                              const costa_mx_dense *C, void *stream) {
    COSTA_MX_CHECK(check_matrix(A, "A"));
    COSTA_MX_CHECK(check_matrix(B, "B"));
    COSTA_MX_CHECK(check_dense(C, "C"));
    if (A->format != COSTA_MX_E2M1 || B->format != COSTA_MX_E2M1)
        return bad(COSTA_ERR_DTYPE, "costa_mx_product takes E2M1 codes");
    if (A->cols != B->cols)
        return bad(COSTA_ERR_SHAPE, "A has %lld columns, B %lld", (long long)A->cols, (long long)B->cols);
    COSTA_MX_CHECK(same_extents(C->rows, C->cols, "C", A->rows, B->rows, "A B^T"));
    if (C->rows == 0 || C->cols == 0) return COSTA_OK;
    COSTA_MX_CHECK(Access().codes(A, "A").codes(B, "B").dense(C, "C").st);
    return done(launch_mx_product(*A, *B, alpha, beta, *C, static_cast<cudaStream_t>(stream)), "costa_mx_product");
}

costa_status costa_mx_act_forward(costa_mx_act act, const costa_mx_dense *X, const costa_mx_dense *G,
                                  const costa_mx_dense *Y, const costa_mx_matrix *QX, const costa_mx_matrix *QG,
                                  void *stream) {
    if (act != COSTA_MX_SILU && act != COSTA_MX_GELU && act != COSTA_MX_RELU)
        return bad(COSTA_ERR_INVALID_ARG, "unknown activation %d", static_cast<int>(act));
    COSTA_MX_CHECK(check_dense(X, "X"));
    COSTA_MX_CHECK(check_dense(Y, "Y"));
    COSTA_MX_CHECK(check_matrix(QX, "QX"));
    if ((G == nullptr) != (QG == nullptr)) return bad(COSTA_ERR_INVALID_ARG, "G and QG go together");
    if (G) {
        COSTA_MX_CHECK(check_dense(G, "G"));
        COSTA_MX_CHECK(check_matrix(QG, "QG"));
    }
    if (X->type != Y->type || (G && G->type != X->type)) return bad(COSTA_ERR_DTYPE, "X, G and Y have different types");
    if (QX->format != COSTA_MX_I8 || (QG && QG->format != COSTA_MX_I8))
        return bad(COSTA_ERR_DTYPE, "checkpoints of activations are I8 codes");
    COSTA_MX_CHECK(same_extents(Y->rows, Y->cols, "Y", X->rows, X->cols, "X"));
    COSTA_MX_CHECK(same_extents(QX->rows, QX->cols, "QX", X->rows, X->cols, "X"));
    if (G) {
        COSTA_MX_CHECK(same_extents(G->rows, G->cols, "G", X->rows, X->cols, "X"));
        COSTA_MX_CHECK(same_extents(QG->rows, QG->cols, "QG", X->rows, X->cols, "X"));
    }
    if (X->rows == 0 || X->cols == 0) return COSTA_OK;
    COSTA_MX_CHECK(Access().dense(X, "X").dense(G, "G").dense(Y, "Y").codes(QX, "QX").codes(QG, "QG").st);
    return done(launch_mx_act_forward(act, *X, G, *Y, *QX, QG, static_cast<cudaStream_t>(stream)),
                "costa_mx_act_forward");
}

costa_status costa_mx_act_backward(costa_mx_act act, const costa_mx_matrix *QX, const costa_mx_matrix *QG,
                                   const costa_mx_dense *dY, const costa_mx_dense *dX, const costa_mx_dense *dG,
                                   void *stream) {
    if (act != COSTA_MX_SILU && act != COSTA_MX_GELU && act != COSTA_MX_RELU)
        return bad(COSTA_ERR_INVALID_ARG, "unknown activation %d", static_cast<int>(act));
    COSTA_MX_CHECK(check_matrix(QX, "QX"));
    COSTA_MX_CHECK(check_dense(dY, "dY"));
    COSTA_MX_CHECK(check_dense(dX, "dX"));
    if ((QG == nullptr) != (dG == nullptr)) return bad(COSTA_ERR_INVALID_ARG, "QG and dG go together");
    if (QG) {
        COSTA_MX_CHECK(check_matrix(QG, "QG"));
        COSTA_MX_CHECK(check_dense(dG, "dG"));
    }
    if (dY->type != dX->type || (dG && dG->type != dY->type))
        return bad(COSTA_ERR_DTYPE, "dY, dX and dG have different types");
    if (QX->format != COSTA_MX_I8 || (QG && QG->format != COSTA_MX_I8))
        return bad(COSTA_ERR_DTYPE, "checkpoints of activations are I8 codes");
    COSTA_MX_CHECK(same_extents(dY->rows, dY->cols, "dY", QX->rows, QX->cols, "QX"));
    COSTA_MX_CHECK(same_extents(dX->rows, dX->cols, "dX", QX->rows, QX->cols, "QX"));
    if (QG) {
        COSTA_MX_CHECK(same_extents(QG->rows, QG->cols, "QG", QX->rows, QX->cols, "QX"));
        COSTA_MX_CHECK(same_extents(dG->rows, dG->cols, "dG", QX->rows, QX->cols, "QX"));
    }
    if (QX->rows == 0 || QX->cols == 0) return COSTA_OK;
    COSTA_MX_CHECK(Access().codes(QX, "QX").codes(QG, "QG").dense(dY, "dY").dense(dX, "dX").dense(dG, "dG").st);
    return done(launch_mx_act_backward(act, *QX, QG, *dY, *dX, dG, static_cast<cudaStream_t>(stream)),
                "costa_mx_act_backward");
}

costa_status costa_mx_weight_grad(const costa_mx_dense *dY, const costa_mx_matrix *QX, float alpha, float beta,
                                  const costa_mx_dense *dW, void *stream) {
    COSTA_MX_CHECK(check_dense(dY, "dY"));
    COSTA_MX_CHECK(check_matrix(QX, "QX"));
    COSTA_MX_CHECK(check_dense(dW, "dW"));
    if (QX->format != COSTA_MX_I8) return bad(COSTA_ERR_DTYPE, "costa_mx_weight_grad takes I8 codes");
    if (dY->rows != QX->rows)
        return bad(COSTA_ERR_SHAPE, "dY has %lld rows, QX %lld", (long long)dY->rows, (long long)QX->rows);
    COSTA_MX_CHECK(same_extents(dW->rows, dW->cols, "dW", dY->cols, QX->cols, "dY^T X"));
    if (dW->rows == 0 || dW->cols == 0) return COSTA_OK;
    COSTA_MX_CHECK(Access().dense(dY, "dY").codes(QX, "QX").dense(dW, "dW").st);
    return done(launch_mx_weight_grad(*dY, *QX, alpha, beta, *dW, static_cast<cudaStream_t>(stream)),
                "costa_mx_weight_grad");
}

costa_status costa_mx_failures(int64_t *count) {
    if (!count) return bad(COSTA_ERR_INVALID_ARG, "count is null");
    unsigned a = 0, b = 0;
    cudaError_t e = cudaDeviceSynchronize();  // the copies alone would not wait for non-blocking streams
    if (e == cudaSuccess) e = mx_product_failures(&a);
    if (e == cudaSuccess) e = mx_grad_failures(&b);
    if (e != cudaSuccess) return done(e, "costa_mx_failures");
    *count = int64_t(a) + b;
    return COSTA_OK;
}

}  // extern "C"
