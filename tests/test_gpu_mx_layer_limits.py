"""Norm, experts' rows and distillation at the limits of what their calls take, and where their kernels change."""

import numpy as np
import pytest


torch = pytest.importorskip("torch")
costa = pytest.importorskip("paper_2106_06601_gb300")

from tests.test_gpu_mx import Dense, stream  # noqa: E402
from tests.test_gpu_mx_layer import Index  # noqa: E402

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
