"""Low-bit matrices on the GPU against their definitions in 64 bits: codes and
scales bit for bit; products, activations and gradients within bounds that
follow from 32-bit sums and one rounding; nothing written outside the outputs."""
import math

import numpy as np
import pytest

from tests import _mx

torch = pytest.importorskip("torch")
costa = pytest.importorskip("paper_2106_06601_gb300")

pytestmark = pytest.mark.gpu

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = {"f32": 2.0 ** -24, "bf16": 2.0 ** -9}  # half a unit in the last place, relative
GUARD = 0xA5


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.fixture(autouse=True)
def no_wait_gave_up():
    yield
    assert costa.costa_mx_failures() == 0


class Dense:
    """A row-major matrix in a buffer with `shift` elements before it and `pad`
    after each row; every other byte is a guard that has to stay."""

    def __init__(self, rows, cols, dtype, values=None, pad=0, shift=0):
        self.rows, self.cols, self.dtype, self.ld, self.shift = rows, cols, dtype, cols + pad, shift
        n = shift + rows * self.ld + 16
        es = 4 if dtype == "f32" else 2
        raw = torch.full((n * es,), GUARD, dtype=torch.uint8, device="cuda")
        self.flat = raw.view(TORCH[dtype])
        self.view = torch.as_strided(self.flat, (rows, cols), (self.ld, 1), shift)
        if values is not None:
            self.view.copy_(torch.from_numpy(np.ascontiguousarray(values)).to("cuda"))
        self.before = raw.clone()

    @property
    def c(self):
        return costa.costa_mx_dense(self.dtype, self.rows, self.cols, self.view.data_ptr(), self.ld)

    def numpy(self):
        """The values as float64, after a look at the guards."""
        kept = self.before.view(TORCH[self.dtype]).clone()
        torch.as_strided(kept, (self.rows, self.cols), (self.ld, 1), self.shift).copy_(self.view)
        assert torch.equal(kept.view(torch.uint8), self.flat.view(torch.uint8)), "written outside the matrix"
        return self.view.double().cpu().numpy()


class Codes:
    def __init__(self, fmt, rows, cols, pad=0, packed=None):
        self.fmt, self.rows, self.cols = fmt, rows, cols
        least, _, ns = _mx.sizes(fmt, rows, cols)
        self.ld = least + pad
        if packed is None:
            self.codes = torch.full((rows * self.ld + 32,), GUARD, dtype=torch.uint8, device="cuda")
            self.scales = torch.full((ns + 32,), GUARD, dtype=torch.uint8, device="cuda")
        else:
            self.codes, self.scales = (torch.from_numpy(p.reshape(-1).copy()).to("cuda") for p in packed)

    @property
    def c(self):
        return costa.costa_mx_matrix(self.fmt, self.rows, self.cols, self.codes.data_ptr(), self.scales.data_ptr(),
                                     self.ld)

    def check(self, x):
        """The codes of x, and guards elsewhere."""
        want = _mx.pack(self.fmt, *_mx.quantize(self.fmt, x), self.cols, self.ld, fill=GUARD)
        codes, scales = self.codes.cpu().numpy(), self.scales.cpu().numpy()
        n = self.rows * self.ld
        assert np.array_equal(scales[:-32], want[1])
        assert np.array_equal(codes[:n].reshape(self.rows, self.ld), want[0])
        assert (codes[n:] == GUARD).all() and (scales[-32:] == GUARD).all()


def matrix(rng, rows, cols, dtype, scale=1.0):
    """Values of several magnitudes, rows and blocks of zeros among them."""
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 7, (rows, cols)))
    x *= np.where(rng.random((rows, 1)) < 0.1, 0.0, scale)
    x[:, cols // 2:cols // 2 + 32][rng.random((rows, x[:, cols // 2:cols // 2 + 32].shape[1])) < 0.5] = 0.0
    x = x.astype(np.float32)
    return _mx.bf16(x) if dtype == "bf16" else x


def codes_of(fmt, x, pad=0):
    """x's codes made by the definition, and their values."""
    packed = _mx.pack(fmt, *_mx.quantize(fmt, x), x.shape[1], _mx.sizes(fmt, *x.shape)[0] + pad, fill=GUARD)
    return Codes(fmt, *x.shape, pad=pad, packed=packed), _mx.rounded(fmt, x)


def close(got, want, tol):
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = np.isnan(want) | (np.abs(got - want) <= tol) | (got == want)
    if not ok.all():
        bad = np.argwhere(~ok)
        i = tuple(bad[0])
        raise AssertionError(f"{len(bad)} of {ok.size} off, first {i}: {got[i]} for {want[i]}, allowed {tol[i]}")


SHAPES = [(1, 1), (1, 32), (1, 4096), (2, 33), (5, 8), (31, 31), (33, 64), (64, 96), (127, 129), (128, 128),
          (256, 64), (257, 65), (300, 1000), (1000, 300), (40, 2056)]


@pytest.mark.parametrize("rows, cols", SHAPES)
@pytest.mark.parametrize("fmt", ["e2m1", "i8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad, shift, qpad", [(0, 0, 0), (3, 1, 16), (8, 8, 0)])
def test_quantize(rows, cols, fmt, dtype, pad, shift, qpad):
    rng = np.random.default_rng([rows, cols, pad])
    x = matrix(rng, rows, cols, dtype)
    X = Dense(rows, cols, dtype, x, pad, shift)
    n, t = Codes(fmt, rows, cols, qpad), Codes(fmt, cols, rows, qpad)
    costa.costa_mx_quantize(X.c, "N", n.c, stream())
    costa.costa_mx_quantize(X.c, "T", t.c, stream())
    n.check(x)
    t.check(x.T)
    n2, t2 = Codes(fmt, rows, cols, qpad), Codes(fmt, cols, rows, qpad)
    costa.costa_mx_quantize_both(X.c, n2.c, t2.c, stream())
    n2.check(x)
    t2.check(x.T)
    Y = Dense(rows, cols, dtype, None, pad, shift)
    costa.costa_mx_dequantize(n.c, Y.c, stream())
    assert np.array_equal(Y.numpy(), _mx.rounded(fmt, x))


@pytest.mark.parametrize("fmt", ["e2m1", "i8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_special_values(fmt, dtype):
    """Ties, the largest and the smallest numbers, signed zeros, and blocks with infinities and NaN."""
    tiny, big = 2.0 ** -126, 2.0 ** 127 * (2 - 2.0 ** -7)
    rows = [np.arange(32) * 0.25, np.arange(32) / 64 + 1.0 / 128, -np.arange(32) * 0.125, np.full(32, big),
            np.full(32, -tiny), np.arange(32) * tiny / 128, np.arange(32) * tiny * 0.75, np.zeros(32), -np.zeros(32),
            np.where(np.arange(32) == 7, np.nan, 1.0), np.where(np.arange(32) == 31, np.inf, 1.0),
            np.where(np.arange(32) == 0, -np.inf, 0.0), np.where(np.arange(32) % 2, big, tiny),
            np.exp2(np.arange(32) - 140.0), np.exp2(-np.arange(32.0)) * 1.99, np.full(32, 2.0 ** -133)]
    x = np.array(rows, np.float32)
    x = _mx.bf16(x) if dtype == "bf16" else x
    x = np.concatenate([x, np.roll(x, 5, 0)], 1)
    X = Dense(*x.shape, dtype, x)
    n, t = Codes(fmt, *x.shape), Codes(fmt, *x.T.shape)
    costa.costa_mx_quantize_both(X.c, n.c, t.c, stream())
    n.check(x)
    t.check(x.T)
    Y = Dense(*x.shape, dtype)
    costa.costa_mx_dequantize(n.c, Y.c, stream())
    assert np.array_equal(Y.numpy(), _mx.rounded(fmt, x), equal_nan=True)


PRODUCTS = [(1, 1, 1), (1, 128, 32), (1, 300, 64), (2, 7, 33), (3, 130, 96), (8, 64, 128), (13, 501, 2200), (17, 129, 160),
            (64, 64, 64), (127, 255, 257), (128, 128, 1024), (129, 257, 4096), (200, 1000, 777), (300, 520, 8200),
            (1000, 33, 513), (5, 4096, 31), (16, 256, 16384), (513, 7000, 160), (700, 13000, 1100),
            (750, 4090, 96), (260, 2048, 4100), (90, 16000, 700)]


@pytest.mark.parametrize("m, n, k", PRODUCTS)
@pytest.mark.parametrize("dtype, alpha, beta, pad, qpad", [("f32", 1.0, 0.0, 0, 0), ("bf16", 1.0, 0.0, 0, 0),
                                                           ("f32", -0.75, 0.3, 3, 16), ("bf16", 2.0, 1.0, 1, 48)])
def test_product(m, n, k, dtype, alpha, beta, pad, qpad):
    rng = np.random.default_rng([m, n, k])
    A, a = codes_of("e2m1", matrix(rng, m, k, "f32"), qpad)
    B, b = codes_of("e2m1", matrix(rng, n, k, "f32", 0.02), qpad)
    c = matrix(rng, m, n, dtype)
    C = Dense(m, n, dtype, c if beta else np.full((m, n), np.nan), pad, pad)
    costa.costa_mx_product(A.c, B.c, C.c, alpha, beta, stream())
    check_product(C, a, b, c, np.float64(np.float32(alpha)), np.float64(np.float32(beta)), dtype, k)


def check_product(C, a, b, c, alpha, beta, dtype, terms):
    """The products are exact; each of `terms` additions in 32 bits, truncating or rounding, is off by 2^-23 of what
    the sum of magnitudes bounds; then alpha, beta and the output's rounding."""
    want = alpha * (a @ b.T) + (beta * c if beta else 0.0)
    mag = np.abs(alpha) * (np.abs(a) @ np.abs(b).T)
    tol = mag * (terms + 2) * 2.0 ** -23 + (3 * 2.0 ** -24 * np.abs(beta * c) if beta else 0.0) + 1e-38
    close(C.numpy(), want, tol + 2 * EPS[dtype] * (np.abs(want) + tol))


def test_product_without_columns():
    A, B = Codes("e2m1", 3, 0), Codes("e2m1", 5, 0)
    c = np.arange(15, dtype=np.float32).reshape(3, 5)
    C = Dense(3, 5, "f32", c)
    costa.costa_mx_product(A.c, B.c, C.c, 1.0, 0.5, stream())
    assert np.array_equal(C.numpy(), c * 0.5)
    costa.costa_mx_product(A.c, B.c, C.c, 1.0, 0.0, stream())
    assert not C.numpy().any()


def one_sign(rng, rows, k, repeat=1):
    """`rows` x k codes of one sign whose blocks' scales spread over 2^8, and their values; the rows `repeat` times."""
    codes = rng.integers(1, 8, (rows, k), np.uint8)
    scales = (127 - rng.integers(0, 9, (rows, -(-k // 32)))).astype(np.uint8)
    padded = np.pad(codes, ((0, 0), (0, -k % 32)))
    q = Codes("e2m1", rows, k, packed=_mx.pack("e2m1", padded, scales, k))
    if repeat > 1:  # whole bands of 128 rows
        q.rows, q.codes, q.scales = rows * repeat, q.codes.repeat(repeat), q.scales.repeat(repeat)
    unit = torch.exp2(torch.from_numpy(scales).cuda().double() - 127).repeat_interleave(32, 1)[:, :k]
    return q, torch.from_numpy(_mx.GRID).cuda()[torch.from_numpy(codes).cuda().long()] * unit


@pytest.mark.parametrize("m, repeat, k", [(3, 1, 2000), (3, 1, 1 << 19), (3, 160, 66000), (30, 160, 66000), (60, 160, 66000),
                                          (120, 160, 66000), (260, 128, 66000), (260, 128, 8193), (260, 128, 8448),
                                          (5, 3, 8200), (20, 160, 16640)])
def test_product_sums_of_one_sign(m, repeat, k):
    """Each product of 64 elements cuts less than 2^-23 off the growing sum, of 8192 elements at most: 64.5 units of 2^-23,
    however large k is; then one rounding for each sum of a tile and up to 7 for the parts of k."""
    rng = np.random.default_rng([m, k])
    (A, a), (B, b) = one_sign(rng, m, k), one_sign(rng, 128, k, repeat)
    n = 128 * repeat
    for alpha, beta, kind in ((1.0, 0.0, "f32"), (0.5, 2.0, "f32"), (1.0, 0.0, "bf16")):
        C = torch.ones(m + 1, n, device="cuda", dtype=TORCH[kind])
        costa.costa_mx_product(A.c, B.c, costa.costa_mx_dense(kind, m, n, C.data_ptr(), n), alpha, beta, stream())
        assert (C[m] == 1).all()
        want = (alpha * (a @ b.t()) + beta).repeat(1, repeat)
        units = 2 * 64.5 + k / 8192 / 2 + 7 + 3
        off = (C[:m].double() - want).abs() / want
        assert off.max().item() <= units * 2.0 ** -24 + (2.0 ** -8 if kind == "bf16" else 0)


def test_product_nan_stays_in_its_rows():
    """A block of NaN reaches its own row of C and no other; so does one in B for columns."""
    rng = np.random.default_rng(3)
    x, w = matrix(rng, 70, 300, "f32"), matrix(rng, 90, 300, "f32")
    x[:, :8], w[:, :8] = 1.0, 1.0
    x[4, 70], w[11, 299], w[80, 0] = np.nan, np.inf, -np.inf
    (A, a), (B, b) = codes_of("e2m1", x), codes_of("e2m1", w)
    C = Dense(70, 90, "f32")
    costa.costa_mx_product(A.c, B.c, C.c, stream=stream())
    got = C.numpy()
    nan = np.zeros((70, 90), bool)
    nan[4], nan[:, 11], nan[:, 80] = True, True, True
    assert np.array_equal(np.isnan(got), nan)
    close(np.where(nan, 0, got), np.where(nan, 0, np.nan_to_num(a) @ np.nan_to_num(b).T),
          302 * 2.0 ** -23 * (np.abs(np.nan_to_num(a)) @ np.abs(np.nan_to_num(b)).T) + 1e-38)


def test_product_small_and_large_scales():
    """Scales at both ends of their range, where the products still fit 32 bits."""
    rng = np.random.default_rng(5)
    a_codes, b_codes = rng.integers(0, 16, (40, 256), np.uint8), rng.integers(0, 16, (50, 256), np.uint8)
    sa = rng.integers(60, 100, (40, 8)).astype(np.uint8)
    sb = rng.integers(60, 100, (50, 8)).astype(np.uint8)
    sa[3], sb[7] = 0, 250  # 2^-127 and 2^123: their product is in range
    A = Codes("e2m1", 40, 256, packed=_mx.pack("e2m1", a_codes, sa, 256))
    B = Codes("e2m1", 50, 256, packed=_mx.pack("e2m1", b_codes, sb, 256))
    a, b = _mx.values("e2m1", a_codes, sa, 256), _mx.values("e2m1", b_codes, sb, 256)
    C = Dense(40, 50, "f32")
    costa.costa_mx_product(A.c, B.c, C.c, stream=stream())
    close(C.numpy(), a @ b.T, 258 * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T) + 2.0 ** -126)


ACT_SHAPES = [(1, 1), (1, 4096), (3, 33), (16, 257), (70, 1000), (33, 64)]


@pytest.mark.parametrize("rows, cols", ACT_SHAPES)
@pytest.mark.parametrize("name", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gated, pad", [(False, 0), (True, 0), (True, 3), (False, 1)])
def test_act(rows, cols, name, dtype, gated, pad):
    rng = np.random.default_rng([rows, cols, pad])
    x, g, dy = (matrix(rng, rows, cols, dtype) for _ in range(3))
    X, Y, dY, dX = (Dense(rows, cols, dtype, v, pad, pad) for v in (x, None, dy, None))
    G, dG = (Dense(rows, cols, dtype, g, pad, pad), Dense(rows, cols, dtype, None, pad, pad)) if gated else (None, None)
    qx, qg = Codes("i8", rows, cols, 16), Codes("i8", rows, cols) if gated else None
    c = lambda v: v.c if v is not None else None
    costa.costa_mx_act_forward(name, X.c, c(G), Y.c, qx.c, c(qg), stream())
    qx.check(x)
    if gated:
        qg.check(g)
    costa.costa_mx_act_backward(name, qx.c, c(qg), dY.c, dX.c, c(dG), stream())
    # the functions within 8 units of 32 bits of their largest term; the slope's terms are at most 1 + |x|
    unit = 16 * 2.0 ** -24
    x, g, dy = (v.astype(np.float64) for v in (x, g, dy))
    one = np.abs(g) if gated else 1.0
    y = _mx.act(name, x)[0] * (g if gated else 1.0)
    close(Y.numpy(), y, unit * np.abs(x) * one + 2 * EPS[dtype] * np.abs(y) + 1e-38)
    xr, gr = _mx.rounded("i8", x), _mx.rounded("i8", g) if gated else 1.0
    back, slope = _mx.act(name, xr)
    dx = dy * gr * slope
    close(dX.numpy(), dx, np.abs(dy * gr) * unit * (1 + np.abs(xr)) + 2 * EPS[dtype] * np.abs(dx) + 1e-38)
    if gated:
        close(dG.numpy(), dy * back, np.abs(dy) * unit * np.abs(xr) + 2 * EPS[dtype] * np.abs(dy * back) + 1e-38)


@pytest.mark.parametrize("rows, cols", ACT_SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("over", ["first", "second"])
def test_act_in_place(rows, cols, dtype, pad, over):
    """Y over X or G, dX or dG over dY: the same bits, checkpoints too, as with storage of their own."""
    rng = np.random.default_rng([rows, cols, pad])
    x, g, dy = (matrix(rng, rows, cols, dtype) for _ in range(3))
    dense = lambda v=None: Dense(rows, cols, dtype, v, pad, pad)

    def run(in_place):
        X, G, dY = dense(x), dense(g), dense(dy)
        Y = dense() if not in_place else X if over == "first" else G
        dX = dY if in_place and over == "first" else dense()
        dG = dY if in_place and over == "second" else dense()
        qx, qg = Codes("i8", rows, cols), Codes("i8", rows, cols)
        costa.costa_mx_act_forward("silu", X.c, G.c, Y.c, qx.c, qg.c, stream())
        costa.costa_mx_act_backward("silu", qx.c, qg.c, dY.c, dX.c, dG.c, stream())
        qx.check(x)
        qg.check(g)
        return [v.numpy() for v in (Y, dX, dG)]

    for got, want in zip(run(True), run(False)):
        assert np.array_equal(got, want)


# Rows that are whole blocks apart (the usual rounding up of a stride), so that a row's first block follows the cut one
# of the row before it as if they were one run; 32 more; and 16, where rows are whole groups apart.
ROW_ENDS = [(2, 13), (16, 13), (31, 31), (64, 33), (20, 40), (33, 48), (64, 90), (16, 257), (70, 300), (9, 480), (5, 4099),
            (64, 2777)]


def apart(cols, more):
    return -cols % (16 if more == "groups" else 32) + (32 if more == "more" else 0)


@pytest.mark.parametrize("rows, cols", ROW_ENDS)
@pytest.mark.parametrize("fmt", ["e2m1", "i8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("more", ["blocks", "more", "groups"])
@pytest.mark.parametrize("shift", [0, 1])
def test_dequantize_rows_whole_blocks_apart(rows, cols, fmt, dtype, more, shift):
    x = matrix(np.random.default_rng([rows, cols]), rows, cols, "bf16")  # whose codes' values are exact in either type
    q, want = codes_of(fmt, x)
    Y = Dense(rows, cols, dtype, None, apart(cols, more), shift)
    costa.costa_mx_dequantize(q.c, Y.c, stream())
    assert np.array_equal(Y.numpy(), want)


@pytest.mark.parametrize("rows, cols", ROW_ENDS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("more", ["blocks", "more", "groups"])
@pytest.mark.parametrize("shift", [0, 1])
def test_act_rows_whole_blocks_apart(rows, cols, dtype, gated, more, shift):
    """The same bits as in rows without gaps, guards around them, in storage of their own and in place."""
    rng = np.random.default_rng([rows, cols])
    x, g, dy = (matrix(rng, rows, cols, dtype) for _ in range(3))

    def run(pad, shift, in_place):
        dense = lambda v=None: Dense(rows, cols, dtype, v, pad, shift)
        X, dY, qx = dense(x), dense(dy), Codes("i8", rows, cols)
        Y, dX = (X, dY) if in_place else (dense(), dense())
        G, dG, qg = (dense(g), dense(), Codes("i8", rows, cols)) if gated else (None, None, None)
        c = lambda v: v.c if v is not None else None
        costa.costa_mx_act_forward("silu", X.c, c(G), Y.c, qx.c, c(qg), stream())
        costa.costa_mx_act_backward("silu", qx.c, c(qg), dY.c, dX.c, c(dG), stream())
        qx.check(x)
        if gated:
            qg.check(g)
        return [v.numpy() for v in (Y, dX, dG) if v is not None]

    want = run(0, 0, False)
    for in_place in (False, True):
        for got, w in zip(run(apart(cols, more), shift, in_place), want):
            assert np.array_equal(got, w)


def act_terms(name, x):
    """act(x), its slope, and the slope's terms' magnitudes, each accurate to its own size in the tails too."""
    x = x.astype(np.float64)
    if name == "silu":
        e = np.exp(-np.abs(x))
        s, c = np.where(x < 0, e, 1.0) / (1 + e), np.where(x < 0, 1.0, e) / (1 + e)
        return x * s, s + x * s * c, s + np.abs(x) * s * c
    cdf = 0.5 * np.vectorize(math.erfc, otypes=[float])(-x / math.sqrt(2))
    density = np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    return x * cdf, cdf + x * density, cdf + np.abs(x) * density


def act_points(rng):
    """Both tails to where the functions underflow, the middle, and arguments down to the smallest."""
    tails = np.linspace(-100, 100, 4001), np.linspace(-14, 14, 4001), rng.uniform(-2, 2, 4001)
    small = np.exp2(-np.arange(0, 149.0))
    x = np.concatenate([*tails, small, -small])
    return np.resize(x, (96, 128)).astype(np.float32)


# The errors in units of 2^-24 of the value.  f32: SiLU: e^-|x| 4 (the library's 2 units in the last place), 1 + e^-|x| 1
# more, its reciprocal 2, two products 2.  GELU: the polynomial's argument 3, of which 2.3 times reach the value, its sum
# 4, the fit 1, two products 2, e^(-x^2 / 2) 5.  A gate's product 1.  So 10 and 19 with all of them; slopes have two such
# terms and a sum.  Where e^-|x| or e^(-x^2 / 2) is subnormal it is off by up to 2^-148.
# bf16: the argument of the exponential, |x| or x^2 / 2, below 88 is rounded by 1.5 or 2.5 units of itself, the GELU's fit
# is 79 units off: 2^8 and 2^9 with the rest.  What is below 2^-126 may be 0.
ACT_UNITS = {"f32": {"silu": 10, "gelu": 19}, "bf16": {"silu": 256, "gelu": 512}}
FLUSH = {"f32": 2.0 ** -148, "bf16": 2.0 ** -126}


def check_act(got, want, tol, dtype):
    """One rounding to the output's type, half a unit in its last place or of its least number, after `tol`."""
    half, least = (2.0 ** -24, 2.0 ** -150) if dtype == "f32" else (2.0 ** -8, 2.0 ** -134)
    close(got, want, tol + half * (np.abs(want) + tol) + least)


@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_act_is_accurate_in_the_tails(name, dtype):
    """Y to its own size, not to that of X."""
    x = act_points(np.random.default_rng(21))
    x = _mx.bf16(x) if dtype == "bf16" else x
    X, Y, q = Dense(*x.shape, dtype, x), Dense(*x.shape, dtype), Codes("i8", *x.shape)
    costa.costa_mx_act_forward(name, X.c, None, Y.c, q.c, None, stream())
    want = act_terms(name, x)[0]
    check_act(Y.numpy(), want, ACT_UNITS[dtype][name] * 2.0 ** -24 * np.abs(want) + np.abs(x) * FLUSH[dtype], dtype)


@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_act_gradient_is_accurate_in_the_tails(name, dtype):
    x = act_points(np.random.default_rng(22))
    x[np.abs(x) > (80 if name == "silu" else 12.5)] = 0  # (slopes below 2^-110)
    x = np.sort(x.reshape(-1)).reshape(x.shape)  # like with like: a block's step is 2^-7 of its largest
    qx, xr = codes_of("i8", x)
    dX = Dense(*x.shape, dtype)
    costa.costa_mx_act_backward(name, qx.c, None, Dense(*x.shape, dtype, np.ones(x.shape)).c, dX.c, None, stream())
    _, want, terms = act_terms(name, xr)
    check_act(dX.numpy(), want, (2 * ACT_UNITS[dtype][name] + 2) * 2.0 ** -24 * terms, dtype)


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_act_gradient_against_differences(name):
    """Central differences of the forward pass at the checkpoint's values, in 64 bits on the definition's side and
    through the kernel: the slope is that of the function that the forward pass computes."""
    x = np.linspace(-6, 6, 96, dtype=np.float32).reshape(3, 32)
    qx, xr = codes_of("i8", x)
    one = Dense(3, 32, "f32", np.ones((3, 32)))
    dX = Dense(3, 32, "f32")
    costa.costa_mx_act_backward(name, qx.c, None, one.c, dX.c, None, stream())
    h = 2.0 ** -6
    ends = []
    for d in (-h, h):
        X, Y, q = Dense(3, 32, "f32", (xr + d).astype(np.float32)), Dense(3, 32, "f32"), Codes("i8", 3, 32)
        costa.costa_mx_act_forward(name, X.c, None, Y.c, q.c, None, stream())
        ends.append(Y.numpy())
    slope = (ends[1] - ends[0]) / (2 * h)
    # third derivatives are below 2: h^2 / 3; each Y off by at most 16 units of 32 bits of 6
    close(dX.numpy(), slope, np.full((3, 32), h * h / 3 + 6 * 16 * 2.0 ** -24 / h + 1e-5))


@pytest.mark.parametrize("name", ["silu", "gelu", "relu"])
def test_act_nan(name):
    x = np.zeros((2, 64), np.float32)
    x[0, 3] = np.nan
    X, Y, q = Dense(2, 64, "f32", x), Dense(2, 64, "f32"), Codes("i8", 2, 64)
    costa.costa_mx_act_forward(name, X.c, None, Y.c, q.c, None, stream())
    q.check(x)
    assert np.array_equal(np.isnan(Y.numpy()), np.isnan(x))
    dY, dX = Dense(2, 64, "f32", np.ones((2, 64))), Dense(2, 64, "f32")
    costa.costa_mx_act_backward(name, q.c, None, dY.c, dX.c, None, stream())
    want = np.zeros((2, 64), bool)
    want[0, :32] = True
    assert np.array_equal(np.isnan(dX.numpy()), want)


GRADS = [(1, 1, 1), (1, 128, 64), (3, 5, 33), (17, 129, 96), (31, 64, 257), (64, 64, 64), (65, 300, 100), (128, 256, 256),
         (200, 130, 520), (777, 100, 153), (4100, 72, 40), (33, 1000, 24), (5000, 8, 300), (130, 5000, 2100),
         (200, 5000, 2600)]


@pytest.mark.parametrize("m, n, k", GRADS)
@pytest.mark.parametrize("ytype, wtype, alpha, beta, pad, qpad", [
    ("bf16", "f32", 1.0, 0.0, 0, 0), ("f32", "f32", 1.0, 0.0, 0, 0), ("bf16", "bf16", 0.5, 1.0, 3, 16),
    ("f32", "bf16", 1.0, 0.0, 1, 0), ("bf16", "f32", -1.5, 0.3, 8, 32), ("f32", "f32", 1.0, 1.0, 4, 0)])
def test_weight_grad(m, n, k, ytype, wtype, alpha, beta, pad, qpad):
    rng = np.random.default_rng([m, n, k])
    dy = matrix(rng, m, n, ytype, 1e-3)
    dY = Dense(m, n, ytype, dy, pad, pad)
    q, x = codes_of("i8", matrix(rng, m, k, "f32"), qpad)
    w = matrix(rng, n, k, wtype)
    dW = Dense(n, k, wtype, w if beta else np.full((n, k), np.nan), pad, 0)
    costa.costa_mx_weight_grad(dY.c, q.c, dW.c, alpha, beta, stream())
    # f32 gradients may be summed in three parts
    check_product(dW, dy.T.astype(np.float64), x.T, w, np.float64(np.float32(alpha)), np.float64(np.float32(beta)), wtype,
                  3 * m)


@pytest.mark.parametrize("m, n, k", [(64, 40, 70), (500, 130, 260), (2048, 130, 260), (2048, 1500, 1000)])
@pytest.mark.parametrize("pad", [0, 1])
def test_weight_grad_f32_sums_of_one_sign(m, n, k, pad):
    """Full 24-bit gradients, values in 1 .. 2: products of the first 8 bits are multiples of 2^-13 below 4, of which 256
    sum exactly; the others' sums are 2^-7 of those, of whose 17 terms each of 32 products cuts below 2^-24: 2.2 units of
    2^-24 on average over the growing sum.  Then one rounding of either sum's total, one for each 256 tokens (half a unit
    of a sum that grows: 8 at most of 2048), and up to 3 where parts of the tokens are joined."""
    rng = np.random.default_rng([m, n])
    dy = (1 + rng.random((m, n))).astype(np.float32)
    q, x = codes_of("i8", rng.uniform(1, 1.98, (m, k)).astype(np.float32))
    dW = Dense(n, k, "f32")
    costa.costa_mx_weight_grad(Dense(m, n, "f32", dy, pad).c, q.c, dW.c, stream=stream())
    want = dy.T.astype(np.float64) @ x
    close(dW.numpy(), want, (2.2 + 1 + min(8, m / 512) + 3) * 2.0 ** -24 * want)


@pytest.mark.parametrize("m, n, k", [(1000, 130, 260), (65536, 130, 260), (32768, 520, 1030)])
@pytest.mark.parametrize("pad", [0, 1])
def test_weight_grad_bf16_sums_of_one_sign(m, n, k, pad):
    """A sum of 32 products over 16 tokens cuts 17 terms of each below 2^-24 of the growing sum (280 units of 2^-24), and
    each 512 tokens are joined with one rounding: far below 17 m / 32 units of one long sum."""
    rng = np.random.default_rng([m, n])
    size = lambda: np.exp2(-rng.integers(0, 4, (m, 1)))
    dy = _mx.bf16(((1 + rng.random((m, n))) * size()).astype(np.float32))
    x = torch.from_numpy(((1 + rng.random((m, k))) * size()).astype(np.float32)).to("cuda")
    q, xr = Codes("i8", m, k), torch.empty(m, k, device="cuda")
    as_dense = lambda a: costa.costa_mx_dense("f32", m, k, a.data_ptr(), k)
    costa.costa_mx_quantize(as_dense(x), "N", q.c, stream())
    costa.costa_mx_dequantize(q.c, as_dense(xr), stream())
    dY, dW = Dense(m, n, "bf16", dy, pad), Dense(n, k, "f32")
    costa.costa_mx_weight_grad(dY.c, q.c, dW.c, stream=stream())
    want = dy.T.astype(np.float64) @ xr.double().cpu().numpy()
    close(dW.numpy(), want, (280 + m / 1024 + 3) * 2.0 ** -24 * want)


def test_weight_grad_without_tokens():
    w = np.arange(12, dtype=np.float32).reshape(3, 4)
    dW, q = Dense(3, 4, "f32", w), Codes("i8", 0, 4)
    costa.costa_mx_weight_grad(costa.costa_mx_dense("bf16", 0, 3, 0, 3), q.c, dW.c, 1.0, 2.0, stream())
    assert np.array_equal(dW.numpy(), w * 2)
    costa.costa_mx_weight_grad(costa.costa_mx_dense("bf16", 0, 3, 0, 3), q.c, dW.c, 1.0, 0.0, stream())
    assert not dW.numpy().any()


@pytest.mark.parametrize("ytype", ["f32", "bf16"])
def test_weight_grad_small_and_large(ytype):
    """Scales at both ends, where the checkpoint's values are subnormal or near the largest, and gradients to match."""
    rng = np.random.default_rng(9)
    m, n, k = 96, 40, 96
    codes = rng.integers(-127, 128, (m, k)).astype(np.int8)
    s = rng.integers(120, 134, (m, 3)).astype(np.uint8)
    s[:, 0], s[:, 2] = rng.integers(0, 8, m), rng.integers(240, 254, m)
    x = _mx.values("i8", codes, s, k)
    q = Codes("i8", m, k, packed=_mx.pack("i8", codes, s, k, fill=GUARD))
    for scale, cols in ((2.0 ** 60, slice(0, 32)), (1.0, slice(32, 64)), (2.0 ** -60, slice(64, 96))):
        dy = matrix(rng, m, n, ytype, scale)
        dW = Dense(n, k, "f32")
        costa.costa_mx_weight_grad(Dense(m, n, ytype, dy).c, q.c, dW.c, stream=stream())
        got, d = dW.numpy()[:, cols], dy.T.astype(np.float64)
        mag = np.abs(d) @ np.abs(x[:, cols])
        close(got, d @ x[:, cols], 3 * (m + 2) * 2.0 ** -23 * mag + 1e-38)


def test_weight_grad_nan_stays_in_its_columns():
    rng = np.random.default_rng(4)
    x = matrix(rng, 50, 100, "f32")
    x[7, 40] = np.nan
    dy = np.ones((50, 20), np.float32)
    dy[:, 3] = 0
    dy[2, 5] = np.inf
    q, xr = codes_of("i8", x)
    dW = Dense(20, 100, "f32")
    costa.costa_mx_weight_grad(Dense(50, 20, "f32", dy).c, q.c, dW.c, stream=stream())
    got = dW.numpy()
    with np.errstate(invalid="ignore"):
        want = np.einsum("tn,tk->nk", dy.astype(np.float64), xr)
    assert np.isnan(got[:, 32:64]).all()
    rest = np.r_[0:32, 64:100]
    others = np.r_[0:5, 6:20]
    assert np.isfinite(got[np.ix_(others, rest)]).all()
    assert not np.isfinite(got[5, rest]).any()
    close(got[np.ix_(others, rest)], want[np.ix_(others, rest)],
          (150 * 2.0 ** -23 * (np.abs(dy.T) @ np.abs(np.nan_to_num(xr))))[np.ix_(others, rest)] + 1e-38)


def test_weight_grad_against_differences():
    """<dW, V> is the derivative of sum(dY * (X W^T)) along V: differences of that (linear) function in 64 bits."""
    rng = np.random.default_rng(6)
    m, n, k = 60, 30, 50
    dy, w, v = rng.standard_normal((m, n)).astype(np.float32), rng.standard_normal((n, k)), rng.standard_normal((n, k))
    q, x = codes_of("i8", matrix(rng, m, k, "f32"))
    dW = Dense(n, k, "f32")
    costa.costa_mx_weight_grad(Dense(m, n, "f32", dy).c, q.c, dW.c, stream=stream())
    f = lambda u: float(np.sum(dy.astype(np.float64) * (x @ u.T)))
    diff = (f(w + v) - f(w - v)) / 2
    mag = float(np.sum((np.abs(dy).T.astype(np.float64) @ np.abs(x)) * np.abs(v)))
    assert abs(float(np.sum(dW.numpy() * v)) - diff) <= mag * 3 * (m + 2) * 2.0 ** -23


def test_repeated_calls_give_the_same_bits():
    rng = np.random.default_rng(8)
    A, _ = codes_of("e2m1", matrix(rng, 9, 5000, "f32"))
    B, _ = codes_of("e2m1", matrix(rng, 700, 5000, "f32"))
    q, _ = codes_of("i8", matrix(rng, 3000, 90, "f32"))
    dY = Dense(3000, 70, "f32", matrix(rng, 3000, 70, "f32"))
    seen = []
    for _ in range(3):
        C, dW = Dense(9, 700, "f32"), Dense(70, 90, "f32")
        costa.costa_mx_product(A.c, B.c, C.c, stream=stream())
        costa.costa_mx_weight_grad(dY.c, q.c, dW.c, stream=stream())
        seen.append((C.numpy(), dW.numpy()))
    for c, w in seen[1:]:
        assert np.array_equal(c, seen[0][0]) and np.array_equal(w, seen[0][1])


def test_streams_and_graph():
    """A layer's step on a side stream, then captured in a graph and replayed on other inputs."""
    rng = np.random.default_rng(11)
    m, n, k = 40, 200, 160
    side = torch.cuda.Stream()
    X, w = Dense(m, k, "bf16", matrix(rng, m, k, "bf16")), matrix(rng, n, k, "f32")
    B, b = codes_of("e2m1", w)
    qx, q8, C, dW = Codes("e2m1", m, k), Codes("i8", m, k), Dense(m, n, "f32"), Dense(n, k, "f32")
    dy = matrix(rng, m, n, "bf16")
    dY = Dense(m, n, "bf16", dy)

    def step():
        s = stream()
        costa.costa_mx_quantize(X.c, "N", qx.c, s)
        costa.costa_mx_quantize(X.c, "N", q8.c, s)
        costa.costa_mx_product(qx.c, B.c, C.c, stream=s)
        costa.costa_mx_weight_grad(dY.c, q8.c, dW.c, stream=s)

    def check(x):
        check_product(C, _mx.rounded("e2m1", x), b, None, 1.0, 0.0, "f32", k)
        check_product(dW, dy.T.astype(np.float64), _mx.rounded("i8", x).T, None, 1.0, 0.0, "f32", 3 * m)

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    check(X.numpy())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        X.view.copy_(torch.from_numpy(matrix(rng, m, k, "bf16")))
        graph.replay()
        torch.cuda.synchronize()
        check(X.view.double().cpu().numpy())


def test_two_streams_at_once():
    """Products of every tile size and gradients of every source on two streams, which share SMs and tensor memory."""
    rng = np.random.default_rng(13)
    work = []
    for m, n, k in ((3, 900, 700), (30, 900, 700), (60, 2000, 500), (120, 900, 700), (700, 5000, 300)):
        A, a = codes_of("e2m1", matrix(rng, m, k, "f32"))
        B, b = codes_of("e2m1", matrix(rng, n, k, "f32"))
        C = Dense(m, n, "f32")
        work.append((lambda A=A, B=B, C=C: costa.costa_mx_product(A.c, B.c, C.c, stream=stream()),
                     lambda C=C, a=a, b=b, k=k: check_product(C, a, b, None, 1.0, 0.0, "f32", k)))
    for m, n, k, kind, pad in ((300, 200, 300, "bf16", 0), (300, 200, 300, "bf16", 1), (300, 200, 300, "f32", 0),
                               (200, 2600, 2100, "bf16", 0)):
        dy = matrix(rng, m, n, kind)
        dY, dW = Dense(m, n, kind, dy, pad), Dense(n, k, "f32")
        q, x = codes_of("i8", matrix(rng, m, k, "f32"))
        work.append((lambda dY=dY, q=q, dW=dW: costa.costa_mx_weight_grad(dY.c, q.c, dW.c, stream=stream()),
                     lambda dW=dW, dy=dy, x=x, m=m: check_product(dW, dy.T.astype(np.float64), x.T, None, 1.0, 0.0,
                                                                  "f32", 3 * m)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(4):
        for i, (call, _) in enumerate(work):  # a call stays on its stream; its neighbour runs beside it
            with torch.cuda.stream(streams[i % 2]):
                call()
    torch.cuda.synchronize()
    for _, check in work:
        check()


def test_failures_waits_for_all_streams():
    """The count is that of all calls so far, those on non-blocking streams too."""
    A, B = (Codes("e2m1", 4096, 4096) for _ in range(2))
    for q in (A, B):
        q.codes.zero_()
        q.scales.zero_()
    C = torch.empty(4096, 4096, device="cuda")
    c = costa.costa_mx_dense("f32", 4096, 4096, C.data_ptr(), 4096)
    assert costa.costa_mx_failures() == 0  # (a first call may wait for other reasons)
    side, done = torch.cuda.Stream(), torch.cuda.Event()
    for _ in range(200):  # some 10 ms
        costa.costa_mx_product(A.c, B.c, c, stream=side.cuda_stream)
    done.record(side)
    assert costa.costa_mx_failures() == 0
    assert done.query()


def test_storage_refusals():
    """Host memory and matrices that leave their allocation are refused before any kernel runs."""
    host = np.zeros(4096, np.uint8)
    x = torch.zeros(64, 64, device="cuda")
    q = Codes("e2m1", 64, 64)
    n = costa.costa_kernel_launch_count()
    at = -(-host.ctypes.data // 16) * 16
    pinned = torch.zeros(4096, dtype=torch.uint8).pin_memory()
    for bad in (costa.costa_mx_dense("f32", 4, 64, at, 64),
                costa.costa_mx_dense("f32", 4, 64, pinned.data_ptr(), 64),
                costa.costa_mx_dense("f32", 4, 64, x.data_ptr(), 1 << 33)):
        with pytest.raises(costa.CostaError) as e:
            costa.costa_mx_quantize(bad, "N", costa.costa_mx_matrix("e2m1", 4, 64, q.codes.data_ptr(),
                                                                    q.scales.data_ptr(), 32), stream())
        assert costa.STATUS_NAMES[e.value.status] == "LAYOUT"
    with pytest.raises(costa.CostaError) as e:
        costa.costa_mx_quantize(costa.costa_mx_dense("f32", 64, 64, x.data_ptr(), 64), "N",
                                costa.costa_mx_matrix("e2m1", 64, 64, q.codes.data_ptr(), at, 32), stream())
    assert costa.STATUS_NAMES[e.value.status] == "LAYOUT"
    assert costa.costa_kernel_launch_count() == n


def test_offsets_beyond_32_bits():
    """Matrices of more than 2^32 elements: codes beyond 2 GB, dense rows beyond 8 GB."""
    rows, cols = 70000, 65536
    least, nc, ns = _mx.sizes("e2m1", rows, cols)
    x = torch.randn(rows, 256, device="cuda", dtype=torch.bfloat16).repeat(1, cols // 256)
    codes = torch.empty(nc, dtype=torch.uint8, device="cuda")
    scales = torch.empty(ns, dtype=torch.uint8, device="cuda")
    Q = costa.costa_mx_matrix("e2m1", rows, cols, codes.data_ptr(), scales.data_ptr(), least)
    costa.costa_mx_quantize(costa.costa_mx_dense("bf16", rows, cols, x.data_ptr(), cols), "N", Q, stream())
    at = [0, 1, 127, 33333, 65535, 65536, 69999]
    picked = x[at].double().cpu().numpy()
    want = _mx.rounded("e2m1", picked)
    got = codes.view(rows, least)[at].cpu().numpy()
    assert np.array_equal(got, _mx.pack("e2m1", *_mx.quantize("e2m1", picked), cols)[0])
    token, t = codes_of("e2m1", matrix(np.random.default_rng(2), 2, cols, "f32"))
    C = Dense(2, rows, "f32")
    costa.costa_mx_product(token.c, Q, C.c, stream=stream())
    close(C.numpy()[:, at], t @ want.T, (cols + 2) * 2.0 ** -23 * (np.abs(t) @ np.abs(want).T))
    del x
    y = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16)
    costa.costa_mx_dequantize(Q, costa.costa_mx_dense("bf16", rows, cols, y.data_ptr(), cols), stream())
    assert np.array_equal(y[at].double().cpu().numpy(), want)
