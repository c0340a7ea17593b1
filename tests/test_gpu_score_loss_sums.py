"""gram_score_loss: bf16 gradients whose sums take several accumulators, and what the rounding of a target's entry leaves in its user's gradient."""
import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, U, context, near
from tests.test_gpu_score_loss import gradient, untouched, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,V", [(70_000, 66_000), (66_000, 70_000)])
def test_sums_of_more_than_65_536_products(N, V):
    """Against the formula in 64 bits, 1000 users at a time.  Vectors are codes, so that logits are exact.  As in tests/test_gpu_score_loss.py: p is off by
    (2^-22 + (V / 128 + 64) u + 3 u Y) of itself from its sum, and the roundings of y, log s and the power of two (Y, |y| <= 2 max |scale z|, log s <= 12);
    g is rounded to bf16; the tensor cores cut off at most 2^-22 of the terms' sizes for each 16 products, and as much for each accumulator and part."""
    d, scale = 16, float(np.float32(0.3))
    gen = torch.Generator(device=DEV).manual_seed(N)
    codes = lambda n: torch.randint(-16, 17, (n, d), device=DEV, generator=gen).to(torch.bfloat16) / 8   # noqa: E731
    users, items = codes(N), codes(V)
    t = torch.randint(-1, V, (N,), dtype=torch.int32, device=DEV, generator=gen)
    weight = torch.rand(N, device=DEV, generator=gen) + 0.5
    loss, (bu, du), (bi, di), db = torch.empty(N, device=DEV), gradient(N, d, 8, "bf16"), gradient(V, d, 8, "bf16"), torch.empty(V, device=DEV)
    g = context()
    g.score_loss(users, items, t, loss, workspace(N, V, d, "bf16", "best"), scale=scale, weight=weight, dusers=du, ditems=di, dbias=db)
    g.sync()
    assert untouched(bu, N, d) and untouched(bi, V, d)
    w, most = items.double(), 0.0
    dI, size, dB, sizeB = torch.zeros_like(w), torch.zeros_like(w), torch.zeros_like(w[:, 0]), torch.zeros_like(w[:, 0])
    cut = lambda n: (n / 16 + 8 + n / 2048 + 32) * 2.0 ** -22   # noqa: E731
    step, last = 2.0 ** -8, 2.0 ** -8
    for at in range(0, N, 1000):
        rows = slice(at, min(N, at + 1000))
        u, real, to = users[rows].double(), t[rows] >= 0, t[rows].clamp(min=0).long()
        z = scale * (u @ w.T)
        y = float(z.abs().max()) * 2
        off_p = 2.0 ** -21 + (V / 128 + 64 + 3 * y + 4 * (y + 12) + 4 * 12 + 2 * (y + 12)) * U
        lp = torch.log_softmax(z, 1)
        here = torch.arange(len(u), device=DEV)
        assert bool(((loss[rows].double() + torch.where(real, lp[here, to], 0.0)).abs() <= off_p).all())
        f = torch.where(real, weight[rows].double() * scale, 0.0)[:, None]
        e = lp.exp()
        exact = f * e * off_p
        e[here, to] -= 1.0
        e *= f
        exact += 3 * U * e.abs()
        off = exact + step * (e.abs() + exact)
        want = e @ w
        bound = (off + cut(V) * e.abs()) @ w.abs()
        bound += last * (want.abs() + bound)
        most = max(most, float(((du[rows].double() - want).abs() - bound).max()))
        dI += e.T @ u
        size += (off + cut(N) * e.abs()).T @ u.abs()
        dB += e.sum(0)
        sizeB += (exact + (N / 8 + 48) * U * e.abs()).sum(0)
    assert most <= 1e-37, most
    assert bool(((di.double() - dI).abs() <= size + last * (dI.abs() + size) + 1e-37).all())
    assert bool(((db.double() - dB).abs() <= sizeB).all())
    g.close()


def to_bf16(x):
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


# by lanes; a row a block (no bias' gradient, up to 16 384 items); logits in L2; logits formed again, in tiles of half the width and whole ones
@pytest.mark.parametrize("N,V,bias", [(1, 3000, True), (4, 3000, False), (5, 3000, False), (300, 5000, False), (5, 3000, True), (70, 20_000, False), (400, 9000, True), (600, 2000, True),
                                      (3000, 9000, False)])
def test_what_rounding_leaves_of_the_targets_entry(N, V, bias):
    """All items but one are zeros, so that a row of dusers is its target's entry times that item, in which 64 bits, rounded once, must be met: the entry's
    own rounding to bf16 would show.  32 bits: p and its factors are off by less than 2^-19 of the entry, its products' sum by 2^-20."""
    d, rng = 64, np.random.default_rng(N)
    at = V // 3
    u, w = np.round(rng.standard_normal((N, d)) * 16) / 64, np.zeros((V, d))
    w[at] = np.round(rng.standard_normal(d) * 100 + 30) / 128
    w[at] = to_bf16(w[at])
    weight = (rng.random(N) + 0.5).astype(np.float32)
    z = u @ w[at]
    entry = weight.astype(np.float64) * (np.exp(z) / (np.exp(z) + V - 1) - 1)
    want = entry[:, None] * w[at]

    def off(got):
        near_by = np.abs(want) * (1 + 2.0 ** -18)
        half = np.exp2(np.floor(np.log2(np.maximum(near_by, 1e-30))) - 8)        # half a step
        return np.abs(got - want) - half - 2.0 ** -18 * np.abs(want)

    assert N < 5 or (off(to_bf16(to_bf16(entry)[:, None] * w[at])) > 0).mean() > 0.1        # an entry that is rounded first would be seen
    on = lambda x: torch.from_numpy(x).to(DEV)   # noqa: E731
    for size in ("least", "best"):
        loss, du, di = torch.empty(N, device=DEV), gradient(N, d, 0, "bf16")[1], gradient(V, d, 0, "bf16")[1]
        g = context()
        g.score_loss(on(u).to(torch.bfloat16), on(w).to(torch.bfloat16), torch.full((N,), at, dtype=torch.int32, device=DEV), loss, workspace(N, V, d, "bf16", size), weight=on(weight),
                     dusers=du, ditems=di, dbias=torch.empty(V, device=DEV) if bias else None)
        g.sync()
        near(loss, np.log(np.exp(z) + V - 1) - z, 1e-4, "loss")
        assert float(off(du.double().cpu().numpy()).max()) <= 0
        g.close()
