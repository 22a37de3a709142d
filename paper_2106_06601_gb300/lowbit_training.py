"""Training steps of a gated layer on low-bit matrices, its weights held by ranks in block-cyclic layouts.

    H = silu(X Wg^T) * (X Wu^T),  Y = H Wd^T,  loss = mean (Y - T)^2 / 2

A step shows the low-bit operators and the reshuffle together:
  - each weight is gathered from its ranks into one dense matrix (costa_transform) and quantised to 4 bits in both
    orders in one pass: one for the forward product, one for the gradient of its input;
  - the forward pass quantises its inputs to 4 bits for the products, and keeps X, H and the two inputs of the
    activation in 8 bits for the backward pass;
  - the backward pass takes the activation's gradients and every weight's gradient from those checkpoints, and the
    inputs' gradients from 4-bit products with the weights' other order, the second one added to the first (beta = 1);
  - each weight's gradient goes back to its ranks as the update W = -lr * dW + 1 * W, one costa_transform.

    python -m paper_2106_06601_gb300.lowbit_training [--steps 20] [--tokens 512] [--width 256] [--hidden 768]
"""
from __future__ import annotations

import argparse

import torch

import paper_2106_06601_gb300 as costa

RANKS, GRID, BLOCK = 4, 2, 32


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _dense(a: torch.Tensor) -> bytes:
    kind = {torch.float32: "f32", torch.bfloat16: "bf16"}[a.dtype]
    return costa.costa_mx_dense(kind, a.shape[0], a.shape[1], a.data_ptr(), a.stride(0))


class Codes:
    """Storage of a matrix of codes."""

    def __init__(self, fmt: str, rows: int, cols: int):
        ld, code_bytes, scale_bytes = costa.costa_mx_sizes(fmt, rows, cols)
        self.codes = torch.empty(code_bytes, dtype=torch.uint8, device="cuda")
        self.scales = torch.empty(scale_bytes, dtype=torch.uint8, device="cuda")
        self.matrix = costa.costa_mx_matrix(fmt, rows, cols, self.codes.data_ptr(), self.scales.data_ptr(), ld)


def _quantized(a: torch.Tensor, fmt: str) -> Codes:
    q = Codes(fmt, *a.shape)
    costa.costa_mx_quantize(_dense(a), "N", q.matrix, stream=_stream())
    return q


def _product(a: Codes, b: Codes, out: torch.Tensor, beta: float = 0.0) -> torch.Tensor:
    costa.costa_mx_product(a.matrix, b.matrix, _dense(out), beta=beta, stream=_stream())
    return out


def _one_block(a: torch.Tensor):
    """The layout of a dense row-major matrix that rank 0 holds."""
    return costa.costa_layout_create("f32", RANKS, [0, a.shape[0]], [0, a.shape[1]], [0], [a.data_ptr()], [a.stride(0)],
                                     [costa.ORDERS["R"]])


class Weight:
    """An n x k matrix in a block-cyclic layout, with what a step makes of it."""

    def __init__(self, n: int, k: int, gen: torch.Generator):
        self.dense = torch.randn(n, k, generator=gen, device="cuda") / k ** 0.5
        self.grad = torch.empty_like(self.dense)
        per = GRID * BLOCK
        local = lambda extent, r: extent // per * BLOCK + min(max(extent % per - r * BLOCK, 0), BLOCK)
        sizes = [(local(n, i), local(k, j)) for i in range(GRID) for j in range(GRID)]
        self.ranks = [torch.zeros(max(1, c * r), device="cuda") for r, c in sizes]
        self.layout = costa.costa_layout_create_block_cyclic(
            "f32", n, k, BLOCK, BLOCK, GRID, GRID, "R", None, [r.data_ptr() for r in self.ranks],
            [max(1, r) for r, _ in sizes])
        self.gathered, self.update_from = _one_block(self.dense), _one_block(self.grad)
        self.q, self.q_t = Codes("e2m1", n, k), Codes("e2m1", k, n)
        costa.costa_transform(self.layout, self.gathered, "N", 1.0, 0.0, relabel=False, stream=_stream())

    def gather(self) -> None:
        costa.costa_transform(self.gathered, self.layout, "N", 1.0, 0.0, relabel=False, stream=_stream())
        costa.costa_mx_quantize_both(_dense(self.dense), self.q.matrix, self.q_t.matrix, stream=_stream())

    def take_gradient(self, dy: torch.Tensor, x: Codes) -> None:
        costa.costa_mx_weight_grad(_dense(dy), x.matrix, _dense(self.grad), stream=_stream())

    def update(self, lr: float) -> None:
        costa.costa_transform(self.layout, self.update_from, "N", -lr, 1.0, relabel=False, stream=_stream())


class Layer:
    def __init__(self, width: int, hidden: int, seed: int = 1):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.gate, self.up, self.down = Weight(hidden, width, gen), Weight(hidden, width, gen), Weight(width, hidden, gen)

    def forward(self, x: torch.Tensor):
        """(Y, checkpoints)."""
        new = lambda cols: torch.empty(x.shape[0], cols, dtype=torch.bfloat16, device="cuda")
        hidden, width = self.gate.dense.shape
        for w in (self.gate, self.up, self.down):
            w.gather()
        q = _quantized(x, "e2m1")
        p, u, h = _product(q, self.gate.q, new(hidden)), _product(q, self.up.q, new(hidden)), new(hidden)
        p8, u8 = Codes("i8", *p.shape), Codes("i8", *u.shape)
        costa.costa_mx_act_forward("silu", _dense(p), _dense(u), _dense(h), p8.matrix, u8.matrix, stream=_stream())
        y = _product(_quantized(h, "e2m1"), self.down.q, new(width))
        return y, (_quantized(x, "i8"), p8, u8, _quantized(h, "i8"))

    def backward(self, dy: torch.Tensor, kept) -> torch.Tensor:
        """dX; the weights' gradients stay with the weights."""
        x8, p8, u8, h8 = kept
        hidden, width = self.gate.dense.shape
        new = lambda cols: torch.empty(dy.shape[0], cols, dtype=torch.bfloat16, device="cuda")
        self.down.take_gradient(dy, h8)
        dh = _product(_quantized(dy, "e2m1"), self.down.q_t, new(hidden))
        dp, du = new(hidden), new(hidden)
        costa.costa_mx_act_backward("silu", p8.matrix, u8.matrix, _dense(dh), _dense(dp), _dense(du), stream=_stream())
        self.gate.take_gradient(dp, x8)
        self.up.take_gradient(du, x8)
        dx = _product(_quantized(dp, "e2m1"), self.gate.q_t, new(width))
        return _product(_quantized(du, "e2m1"), self.up.q_t, dx, beta=1.0)

    def update(self, lr: float) -> None:
        for w in (self.gate, self.up, self.down):
            w.update(lr)


def run(steps: int = 20, tokens: int = 512, width: int = 256, hidden: int = 768, lr: float = 0.5) -> list[float]:
    """The loss before each step."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    x = torch.randn(tokens, width, generator=gen, device="cuda").bfloat16()
    target = torch.tanh(x.float() @ torch.randn(width, width, generator=gen, device="cuda") / width ** 0.5)
    layer = Layer(width, hidden)
    losses = []
    for _ in range(steps):
        y, kept = layer.forward(x)
        off = y.float() - target
        losses.append(off.square().mean().div(2))
        layer.backward((off / tokens).bfloat16(), kept)  # of the mean over tokens of the sum over columns
        layer.update(lr)
    return [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--hidden", type=int, default=768)
    ap.add_argument("--lr", type=float, default=0.5)
    a = ap.parse_args()
    for i, loss in enumerate(run(a.steps, a.tokens, a.width, a.hidden, a.lr)):
        print(f"step {i:3d}  loss {loss:.5f}")


if __name__ == "__main__":
    main()
