"""Softmax cross entropy of users against an item table and its gradients, against the formula in 64 bits.

Bounds.  Vectors are 8-bit codes over a step of 1/16, whose products and sums 32 bits hold exactly, so that the logits are exact and the bounds of
tests/logits_helpers.py hold for log p and p.  An entry g = f (p - [v = t]) is off by |f| d_p and three roundings of 32 bits, and enters the products
rounded to bf16 (2^-8 of itself; for fp32 gradients as two bf16: 2^-16).  The tensor cores add 16 products at a time to a sum of 32 bits and
cut off: at most two last places (2^-22) of the sum of the terms' sizes for each 16 products, and for each part that is added with rounding.
A bf16 result is rounded once more.
"""
import numpy as np
import pytest
import torch

from paper_2204_04179_b200 import binding
from tests.logits_helpers import DEV, DT, INF, U, Rows, context, near

pytestmark = pytest.mark.gpu

# N, V, d, elements between the rows' ends and the next
SIZES = [(1, 1, 8, 0), (2, 3, 8, 8), (1, 255, 16, 0), (3, 256, 64, 0), (64, 257, 72, 8), (127, 1000, 104, 0), (128, 300, 768, 0), (129, 513, 64, 16),
         (5, 10_007, 768, 0), (300, 2603, 256, 0), (257, 5000, 1000, 24), (700, 777, 64, 0), (3000, 70, 32, 0), (2, 100_003, 8, 0), (40, 30_522, 136, 0)]


def codes(rng, rows, d, pad):
    x = np.clip(np.round(rng.standard_normal((rows, d)) * 30), -127, 127) / 16
    buf = torch.full((rows, d + pad), float("nan"), dtype=torch.bfloat16, device=DEV)
    buf[:, :d] = torch.from_numpy(x).to(torch.bfloat16)
    return buf[:, :d], x


def gradient(rows, d, pad, dtype):
    """A buffer of NaN whose elements behind the rows must stay."""
    buf = torch.full((rows + 1, d + pad), float("nan"), dtype=DT[dtype], device=DEV)
    return buf, buf[:rows, :d]


def untouched(buf, rows, d):
    return bool(buf[rows:].isnan().all()) and bool(buf[:, d:].isnan().all())


def workspace(N, V, d, dtype, size):
    least, best = binding.Gram.score_loss_workspace(N, V, d, DT[dtype])
    assert 0 < least <= best
    n = {"least": least, "between": (least + best) // 2, "best": best}[size]
    return torch.full((n + 256,), 255, dtype=torch.uint8, device=DEV)[:n]       # NaN in every type


class Plain:
    """The loss and its gradients in 64 bits with their bounds, from exact logits."""

    def __init__(self, u, w, bias, targets, weight, scale, dtype):
        z = u @ w.T + (bias if bias is not None else 0.0)
        self.r = r = Rows(z, scale)
        N = len(z)
        t = targets.astype(np.int64)
        at = np.arange(N), np.maximum(t, 0)
        self.loss = np.where(t >= 0, -r.logp[at], 0.0)
        self.d_loss = np.where(t >= 0, np.where(np.isfinite(r.logp[at]), r.d_logp[at], 0.0), 0.0)
        f = np.where((t < 0) | np.isneginf(r.logp[at]), 0.0, weight) * r.scale
        delta = r.p.copy()
        delta[at] -= 1.0
        g = f[:, None] * delta
        step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -16
        exact = np.abs(f)[:, None] * r.d_p + 3 * U * np.abs(g)
        off = exact + step * (np.abs(g) + exact)
        K = 1 if dtype == "bf16" else 2
        cut = lambda n: (K * n / 16 + 8 + K * n / 2048 + 32) * 2.0 ** -22   # noqa: E731
        last = 2.0 ** -8 if dtype == "bf16" else U
        self.dU, self.dI, self.db = g @ w, g.T @ u, g.sum(0)
        tiny = 1e-37
        self.d_dU = (off + cut(g.shape[1]) * np.abs(g)) @ np.abs(w) + last * np.abs(self.dU) + tiny
        self.d_dI = (off + cut(N) * np.abs(g)).T @ np.abs(u) + last * np.abs(self.dI) + tiny
        self.d_dU += last * self.d_dU
        self.d_dI += last * self.d_dI
        self.d_db = (exact + (N / 8 + 48) * U * np.abs(g)).sum(0) + tiny


def inputs(rng, N, V, d, pad, bias, none=0.2):
    users, u = codes(rng, N, d, pad)
    items, w = codes(rng, V, d, pad)
    b = None
    if bias:
        b = np.round(rng.standard_normal(V) * 20 * 256) / 256
        b[rng.random(V) < 0.05] = -INF
        b[rng.integers(V)] = 0.0
    targets = np.where(rng.random(N) < none, -1, rng.integers(0, V, N)).astype(np.int32)
    weight = np.where(rng.random(N) < 0.1, 0.0, rng.random(N) + 0.5).astype(np.float32)
    on = lambda x: None if x is None else torch.from_numpy(x).to(DEV)   # noqa: E731
    return users, items, u, w, b, targets, weight, dict(bias=on(None if b is None else b.astype(np.float32)), weight=on(weight)), on(targets)


@pytest.mark.parametrize("size", ["least", "between", "best"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V,d,pad", SIZES)
def test_loss_and_gradients(N, V, d, pad, dtype, size):
    rng = np.random.default_rng(N + V + d)
    users, items, u, w, b, targets, weight, more, t = inputs(rng, N, V, d, pad, bias=(N + V) % 2 == 0 or N > 100)
    scale = 0.05 if d > 32 else 0.3
    want = Plain(u, w, b, targets, weight.astype(np.float64), scale, dtype)
    g = context()
    got = []
    for _ in range(2):
        loss = torch.full((N,), float("nan"), device=DEV)
        (bu, du), (bi, di) = gradient(N, d, pad, dtype), gradient(V, d, pad, dtype)
        db = torch.full((V,), float("nan"), device=DEV)
        g.score_loss(users, items, t, loss, workspace(N, V, d, dtype, size), scale=scale, dusers=du, ditems=di, dbias=db, **more)
        g.sync()
        assert untouched(bu, N, d) and untouched(bi, V, d)
        got.append((loss, du, di, db))
    near(loss, want.loss, want.d_loss, "loss")
    near(du, want.dU, want.d_dU, "dusers")
    near(di, want.dI, want.d_dI, "ditems")
    near(db, want.db, want.d_db, "dbias")
    assert all(torch.equal(x, y) for x, y in zip(*got))
    g.close()
