"""Low-bit matrices, without a GPU: storage sizes, refusals before any device
work, and the tests' own definitions against hand-worked values."""
import numpy as np
import pytest

from tests import _mx

costa = pytest.importorskip("paper_2106_06601_gb300")

P = 1 << 40  # an aligned address that nothing dereferences: every call below is refused before it is looked up


def refused(status, fn, *a, **k):
    with pytest.raises(costa.CostaError) as e:
        fn(*a, **k)
    assert costa.STATUS_NAMES[e.value.status] == status, str(e.value)


def D(rows, cols, dtype="f32", ptr=P, ld=None):
    return costa.costa_mx_dense(dtype, rows, cols, ptr, cols if ld is None else ld)


def Q(rows, cols, fmt="e2m1", ptr=P, scales=P, ld=None):
    return costa.costa_mx_matrix(fmt, rows, cols, ptr, scales, _mx.sizes(fmt, rows, cols)[0] if ld is None else ld)


@pytest.mark.parametrize("fmt", ["e2m1", "i8"])
@pytest.mark.parametrize("rows, cols", [(1, 1), (1, 32), (3, 33), (128, 128), (129, 129), (1000, 4096), (5, 0), (0, 5)])
def test_sizes(fmt, rows, cols):
    assert costa.costa_mx_sizes(fmt, rows, cols) == _mx.sizes(fmt, rows, cols)


def test_sizes_refusals():
    refused("INVALID_ARG", costa.costa_mx_sizes, "i8", -1, 4)
    refused("INVALID_ARG", costa.costa_mx_sizes, "i8", 4, 1 << 31)


def test_definitions():
    # largest magnitude 6: E = 0; halfway cases go to the even code
    x = np.zeros((1, 32))
    x[0, :10] = [6, -0.25, 0.75, 1.25, -1.75, 2.5, 3.5, 5.0, 0.2, -7.0]
    got = _mx.rounded("e2m1", x)[0, :10]
    assert got.tolist() == [6, 0, 1, 1, -2, 2, 4, 4, 0, -6]
    x = np.zeros((1, 33))
    x[0, :4] = [1.0, 0.5 / 64, 1.5 / 64, 2.0 - 2 ** -10]  # E = 0 in the first block
    x[0, 32] = 2.0 ** -140
    c, s = _mx.quantize("i8", x)
    assert c[0, :4].tolist() == [64, 0, 2, 127] and s.tolist() == [[127, 0]] and c[0, 32] == 0
    x[0, 5] = np.inf
    c, s = _mx.quantize("i8", x)
    assert s[0, 0] == 255 and not c[0, :32].any() and np.isnan(_mx.rounded("i8", x)[0, :32]).all()


def test_dense_refusals():
    q = Q(4, 40)
    call = costa.costa_mx_quantize
    refused("INVALID_ARG", call, None, "N", q)
    refused("INVALID_ARG", call, D(4, 40), "N", None)
    refused("INVALID_ARG", call, D(4, 40, ptr=0), "N", q)
    refused("LAYOUT", call, D(4, 40, ptr=P + 2), "N", q)
    refused("LAYOUT", call, D(4, 40, dtype="bf16", ptr=P + 1), "N", q)
    refused("LAYOUT", call, D(4, 40, ld=39), "N", q)
    refused("LAYOUT", call, D(4, 40, ld=1 << 38), "N", q)
    refused("LAYOUT", call, D(1 << 20, 40, ld=1 << 37), "N", Q(1 << 20, 40))
    refused("INVALID_ARG", call, D(-1, 40), "N", q)
    refused("INVALID_ARG", call, D(1 << 31, 40), "N", q)
    refused("INVALID_ARG", call, D(4, 40)[:-8] + b"\7\0\0\0\0\0\0\0", "N", q)  # type 7
    refused("INVALID_ARG", call, D(4, 40)[:-4] + b"\1\0\0\0", "N", q)           # reserved
    refused("SHAPE", call, D(4, 41), "N", q)
    refused("SHAPE", call, D(4, 40), "T", q)


def test_matrix_refusals():
    x = D(4, 40)
    call = costa.costa_mx_quantize
    refused("INVALID_ARG", call, x, "N", Q(4, 40, ptr=0))
    refused("INVALID_ARG", call, x, "N", Q(4, 40, scales=0))
    refused("LAYOUT", call, x, "N", Q(4, 40, ptr=P + 8))
    refused("LAYOUT", call, x, "N", Q(4, 40, scales=P + 4))
    refused("LAYOUT", call, x, "N", Q(4, 40, ld=16))
    refused("LAYOUT", call, x, "N", Q(4, 40, ld=40))
    refused("LAYOUT", call, x, "N", Q(4, 40, fmt="i8", ld=32))
    refused("INVALID_ARG", call, x, "N", Q(4, 40)[:-8] + b"\2\0\0\0\0\0\0\0")
    refused("INVALID_ARG", call, x, "N", Q(4, 40)[:-4] + b"\1\0\0\0")


def test_call_refusals():
    refused("DTYPE", costa.costa_mx_quantize_both, D(4, 40), Q(4, 40), Q(40, 4, "i8"))
    refused("SHAPE", costa.costa_mx_quantize_both, D(4, 40), Q(4, 40), Q(4, 40))
    refused("SHAPE", costa.costa_mx_dequantize, Q(4, 40), D(4, 41))
    refused("DTYPE", costa.costa_mx_product, Q(4, 40, "i8"), Q(5, 40), D(4, 5))
    refused("SHAPE", costa.costa_mx_product, Q(4, 40), Q(5, 41), D(4, 5))
    refused("SHAPE", costa.costa_mx_product, Q(4, 40), Q(5, 40), D(5, 4))
    f, b = costa.costa_mx_act_forward, costa.costa_mx_act_backward
    q = Q(4, 40, "i8")
    refused("DTYPE", f, "silu", D(4, 40), None, D(4, 40), Q(4, 40), None)
    refused("DTYPE", f, "silu", D(4, 40), None, D(4, 40, "bf16"), q, None)
    refused("DTYPE", f, "silu", D(4, 40), D(4, 40, "bf16"), D(4, 40), q, q)
    refused("INVALID_ARG", f, "silu", D(4, 40), D(4, 40), D(4, 40), q, None)
    refused("INVALID_ARG", f, "silu", D(4, 40), None, D(4, 40), q, q)
    refused("SHAPE", f, "silu", D(4, 40), None, D(4, 41), q, None)
    refused("SHAPE", f, "silu", D(4, 40), D(4, 41), D(4, 40), q, q)
    refused("DTYPE", b, "gelu", Q(4, 40), None, D(4, 40), D(4, 40), None)
    refused("INVALID_ARG", b, "gelu", q, q, D(4, 40), D(4, 40), None)
    refused("DTYPE", b, "gelu", q, None, D(4, 40), D(4, 40, "bf16"), None)
    refused("SHAPE", b, "gelu", q, None, D(5, 40), D(4, 40), None)
    refused("SHAPE", b, "gelu", q, q, D(4, 40), D(4, 40), D(4, 39))
    refused("DTYPE", costa.costa_mx_weight_grad, D(4, 6), Q(4, 40), D(6, 40))
    refused("SHAPE", costa.costa_mx_weight_grad, D(5, 6), q, D(6, 40))
    refused("SHAPE", costa.costa_mx_weight_grad, D(4, 6), q, D(40, 6))
    lib = costa.library()
    assert lib.costa_mx_act_forward(9, D(4, 40), None, D(4, 40), q, None, None) == 1
    assert lib.costa_mx_quantize(D(4, 40), 5, Q(4, 40), None) == 1


def test_empty_matrices_need_no_device():
    costa.costa_mx_quantize(D(0, 40, ptr=0), "N", Q(0, 40, ptr=0, scales=0))
    costa.costa_mx_quantize(D(4, 0, ptr=0), "T", Q(0, 4, ptr=0, scales=0))
    costa.costa_mx_product(Q(0, 40, ptr=0, scales=0), Q(5, 40), D(0, 5, ptr=0))
    costa.costa_mx_weight_grad(D(4, 0, ptr=0), Q(4, 40, "i8"), D(0, 40, ptr=0))
