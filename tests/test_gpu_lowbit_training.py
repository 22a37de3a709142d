"""The low-bit training step: its gradients against those that plain 64-bit products of the same codes give, and the
update of weights held in a block-cyclic layout."""
import numpy as np
import pytest

from tests import _mx

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2106_06601_gb300")

pytestmark = pytest.mark.gpu


def test_step_matches_its_definition():
    from paper_2106_06601_gb300 import lowbit_training as lt
    tokens, width, hidden, lr = 96, 72, 136, 0.25
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    x = torch.randn(tokens, width, generator=gen, device="cuda").bfloat16()
    dy = (torch.randn(tokens, width, generator=gen, device="cuda") * 1e-2).bfloat16()
    layer = lt.Layer(width, hidden)
    before = [w.dense.double().cpu().numpy().copy() for w in (layer.gate, layer.up, layer.down)]
    y, kept = layer.forward(x)
    dx = layer.backward(dy, kept)
    layer.update(lr)
    for w in (layer.gate, layer.up, layer.down):  # what the ranks hold now
        w.gather()
    torch.cuda.synchronize()

    f = lambda t: t.double().cpu().numpy()
    q4, q8 = lambda a: _mx.rounded("e2m1", a), lambda a: _mx.rounded("i8", a)
    b16 = lambda a: _mx.bf16(a.astype(np.float32)).astype(np.float64)
    wg, wu, wd = before
    X, DY = f(x), f(dy)
    p, u = b16(q4(X) @ q4(wg).T), b16(q4(X) @ q4(wu).T)
    h = b16(_mx.act("silu", p)[0] * u)
    # Each intermediate is rounded to bf16 on both sides from sums that differ by 32-bit rounding: a value at a rounding
    # boundary may differ by one unit of bf16 (2^-8), and a code made from it by one step (1/4 of the largest in a block
    # in 4 bits).  Few do: the norms are compared, at 2^-5, eight units of bf16.
    near = lambda got, want: np.linalg.norm(got - want) <= 2.0 ** -5 * np.linalg.norm(want)
    assert near(f(y), q4(h) @ q4(wd).T)
    back, slope = _mx.act("silu", q8(p))
    dh = b16(q4(DY) @ q4(wd.T).T)
    dp, du = b16(dh * q8(u) * slope), b16(dh * back)
    assert near(f(dx), q4(dp) @ q4(wg.T).T + q4(du) @ q4(wu.T).T)
    for w, old, grad in ((layer.gate, wg, dp.T @ q8(X)), (layer.up, wu, du.T @ q8(X)), (layer.down, wd, DY.T @ q8(h))):
        assert near(f(w.grad), grad)
        # the update is one fma in f32 of the very gradient
        want = old - lr * f(w.grad)
        assert np.abs(f(w.dense) - want).max() <= 2.0 ** -23 * np.abs(want).max()


def test_training_lowers_the_loss():
    from paper_2106_06601_gb300 import lowbit_training as lt
    losses = lt.run(steps=12, tokens=256, width=128, hidden=256)
    assert all(np.isfinite(losses)) and losses[-1] < losses[0]
