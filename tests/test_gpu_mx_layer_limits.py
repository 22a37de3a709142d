"""Norm, experts' rows and distillation at the limits of what their calls take, and where their kernels change."""
import threading

import numpy as np
import pytest

from tests import _mx_layer as ref

torch = pytest.importorskip("torch")
costa = pytest.importorskip("paper_2106_06601_gb300")

from tests.test_gpu_mx import Dense, close, matrix, stream  # noqa: E402
from tests.test_gpu_mx_layer import Index, places, rounded, workspace  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 3, 700])
@pytest.mark.parametrize("top", [1, 2, 128, 129, 200, 1024])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_without_columns_with_a_gradient(rows, top, dtype):
    """No entry names one of no columns: no loss, and a gradient of no elements."""
    L, S, G = Dense(rows, 1, "f32"), Dense(rows, 2, "f32"), Dense(rows, 1, "f32", np.ones((rows, 1)))
    T, at = Dense(rows, top, "f32", np.ones((rows, top))), Index(rows, top, np.zeros((rows, top), np.int32))
    none = costa.costa_mx_dense(dtype, rows, 0, 0, 0)
    costa.costa_mx_distill_forward(none, at.c, T.c, 1.0, L.c, S.c, G.c, none, stream())
    assert not L.numpy().any()
    assert (S.numpy() == [-np.inf, 0.0]).all()
    costa.costa_mx_distill_backward(none, at.c, T.c, 1.0, S.c, G.c, none, stream())


@pytest.mark.parametrize("n, pairs", [(372, 9000), (372, 1024), (384, 992), (384, 961), (371, 9000), (373, 9000), (385, 992), (1024, 9000)])
def test_expert_sort_of_48_kb(n, pairs):
    """Counts of 48 KB of shared memory, with what the kernel has besides."""
    rng = np.random.default_rng([n, pairs])
    e = rng.integers(0, n, (pairs, 1)).astype(np.int32)
    E, place, starts, counts = Index(pairs, 1, e), Index(pairs, 1), Index(1, n + 1), Index(1, n)
    costa.costa_mx_expert_sort(E.c, n, 1, place.c, starts.c, counts.c, stream())
    for got, want in zip((place, starts, counts), ref.sort(e, n, 1)):
        assert np.array_equal(got.numpy().reshape(want.shape), want)


@pytest.mark.parametrize("rows, cols", [(3, 12288), (310, 12288), (305, 11265), (3, 11900), (2, 11264), (2, 12289), (4, 16384)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 3])
def test_norm_backward_of_48_kb(rows, cols, dtype, pad):
    """Sums of dW of 48 KB of shared memory, with what the kernel has besides."""
    rng = np.random.default_rng([rows, cols, pad])
    x, dy = matrix(rng, rows, cols, dtype), matrix(rng, rows, cols, dtype)
    w = rounded(1 + 0.1 * rng.standard_normal((1, cols)), dtype)
    X, W, Y, S = Dense(rows, cols, dtype, x, pad), Dense(1, cols, dtype, w), Dense(rows, cols, dtype, None, pad), Dense(rows, 1, "f32")
    costa.costa_mx_norm_forward(X.c, None, W.c, 1e-5, None, Y.c, S=S.c, stream=stream())
    dY, dX, dW, work = Dense(rows, cols, dtype, dy, pad), Dense(rows, cols, dtype, None, pad), Dense(1, cols, "f32"), workspace(rows, cols)
    costa.costa_mx_norm_backward(dY.c, X.c, S.c, W.c, None, dX.c, dW.c, work.data_ptr(), work.numel() - 32, stream())
    h, w, dy = x.astype(np.float64), w.astype(np.float64), dy.astype(np.float64)
    y, s = ref.norm(h, w, np.float64(np.float32(1e-5)))
    close(Y.numpy(), y, ref.norm_tol(y, dtype))
    dx, dw, mean = ref.norm_grad(dy, h, s, w)
    tol_x, tol_w = ref.norm_grad_tol(dx, dw, dy, h, s, w, np.zeros_like(h), mean, dtype, "f32", rows)
    close(dX.numpy(), dx, tol_x)
    close(dW.numpy(), dw, tol_w)


def test_calls_of_unlike_sizes_from_several_threads():
    """Host threads whose calls need shared memory of unlike sizes of the same kernels, each on its own stream and storage,
    do not refuse each other's."""
    rng = np.random.default_rng(3)

    class Job:
        def __init__(self, rows, cols, n):
            self.stream, self.failed = torch.cuda.Stream(), []
            x, e = matrix(rng, rows, cols, "bf16"), rng.integers(0, n, (1030, 1)).astype(np.int32)
            X, Y, dX, W = Dense(rows, cols, "bf16", x), Dense(rows, cols, "bf16"), Dense(rows, cols, "bf16"), Dense(1, cols, "bf16", np.ones((1, cols)))
            S, dW, work = Dense(rows, 1, "f32"), Dense(1, cols, "f32"), workspace(rows, cols)
            E, place, starts, counts = Index(1030, 1, e), Index(1030, 1), Index(1, n + 1), Index(1, n)
            self.kept, self.outputs = (X, W, E, work), (Y, S, dX, dW, place, starts, counts)
            st = self.stream.cuda_stream
            # (arguments made once: Python's lock is held while they are, and calls would hardly meet)
            self.calls = [
                (costa.costa_mx_norm_forward, (X.c, None, W.c, 1e-5, None, Y.c, None, None, S.c, st)),
                (costa.costa_mx_norm_backward, (Y.c, X.c, S.c, W.c, None, dX.c, dW.c, work.data_ptr(), work.numel() - 32, st)),
                (costa.costa_mx_expert_sort, (E.c, n, 1, place.c, starts.c, counts.c, st))]

        def many(self, start, times):
            start.wait()
            try:
                for _ in range(times):
                    for call, args in self.calls:
                        call(*args)
            except costa.CostaError as err:
                self.failed.append(str(err))

        def results(self):
            return [v.numpy() for v in self.outputs]

    # rows through shared memory as they lie and as windows, sums of dW there; and sorts by some more experts
    jobs = [Job(*sizes) for sizes in ((310, 3000, 400), (305, 6144, 1024), (310, 2777, 500), (312, 6001, 800), (1, 12800, 450), (1, 30000, 700))]
    torch.cuda.synchronize()
    alone = []
    for job in jobs:
        job.many(threading.Barrier(1), 1)
        torch.cuda.synchronize()
        assert not job.failed
        alone.append(job.results())
    start = threading.Barrier(len(jobs))
    threads = [threading.Thread(target=job.many, args=(start, 3000)) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not [job.failed for job in jobs if job.failed]
    for job, want in zip(jobs, alone):
        for a, b in zip(job.results(), want):
            assert np.array_equal(a, b)


@pytest.mark.parametrize("rows, cols", [(3, 1), (2, 2), (9, 33), (5, 600), (3, 4100), (310, 1200), (310, 1203), (3, 9000)])
@pytest.mark.parametrize("eps", [2.0 ** 127, 2.0 ** 126, 2.0 ** 100, 2.0 ** 90, 1e-6])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("res", [False, True])
def test_norm_of_a_large_eps(rows, cols, eps, dtype, res):
    """An eps of any size counts also where the squares, their sum or it and their mean leave f32's range."""
    rng = np.random.default_rng([rows, cols])
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(50, 64, (rows, 1)))
    x[0], x[1] = 2.0 ** 64, 1.875 * 2.0 ** 63  # of one column the mean leaves the range; it and eps do
    x = rounded(x, dtype)
    eps = np.float32(eps)
    W, w = Dense(1, cols, "f32", np.full((1, cols), 2.0 ** 40)), np.full((1, cols), 2.0 ** 40)
    X, Y, S, H = Dense(rows, cols, dtype, x), Dense(rows, cols, dtype), Dense(rows, 1, "f32"), Dense(rows, cols, dtype)
    R = Dense(rows, cols, dtype, np.zeros((rows, cols)))
    costa.costa_mx_norm_forward(X.c, R.c if res else None, W.c, eps, H.c if res else None, Y.c, S=S.c, stream=stream())
    h = x.astype(np.float64)
    y, s = ref.norm(h, w, np.float64(eps))
    close(S.numpy(), s, 1.01 * ref.S_UNITS * ref.U * s)
    close(Y.numpy(), y, ref.norm_tol(y, dtype))
    dy = rounded(rng.standard_normal((rows, cols)), dtype)
    dY, dX, dW, work = Dense(rows, cols, dtype, dy), Dense(rows, cols, dtype), Dense(1, cols, "f32"), workspace(rows, cols)
    costa.costa_mx_norm_backward(dY.c, X.c, S.c, W.c, None, dX.c, dW.c, work.data_ptr(), work.numel() - 32, stream())
    dx, dw, mean = ref.norm_grad(dy.astype(np.float64), h, s, w)
    tol_x, tol_w = ref.norm_grad_tol(dx, dw, dy.astype(np.float64), h, s, w, np.zeros_like(h), mean, dtype, "f32", rows)
    close(dX.numpy(), dx, tol_x)
    close(dW.numpy(), dw, tol_w)


@pytest.mark.parametrize("tokens, cols, top, rows", [(3, 33, 2, 9), (50, 900, 3, 200), (130, 1027, 8, 1200), (64, 4096, 9, 700), (9, 2777, 33, 300)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad, pad_dz", [(0, 0), (3, 3), (8, 1), (1, 8)])
def test_weights_gradient_by_itself_and_over_z(tokens, cols, top, rows, dtype, pad, pad_dz):
    """dweights is added up in one order, whatever else is written: its bits are the same with dZ beside it, alone, and with
    dZ over Z, which a read of Z after its overwriting would change."""
    rng = np.random.default_rng([tokens, cols, pad])
    at = places(rng, tokens, top, rows)
    z, dy = matrix(rng, rows, cols, dtype), matrix(rng, tokens, cols, dtype)
    Z, dY = Dense(rows, cols, dtype, z, pad), Dense(tokens, cols, dtype, dy, pad)
    place, W = Index(tokens, top, at), Dense(tokens, top, "f32", rng.standard_normal((tokens, top)).astype(np.float32))
    beside, alone, over = (Dense(tokens, top, "f32") for _ in range(3))
    costa.costa_mx_combine_backward(dY.c, Z.c, place.c, W.c, Dense(rows, cols, dtype, None, pad_dz).c, None, beside.c, stream())
    costa.costa_mx_combine_backward(dY.c, Z.c, place.c, W.c, None, None, alone.c, stream())
    costa.costa_mx_combine_backward(dY.c, Z.c, place.c, W.c, Z.c, None, over.c, stream())
    assert np.array_equal(alone.numpy(), beside.numpy())
    assert np.array_equal(over.numpy(), beside.numpy())
