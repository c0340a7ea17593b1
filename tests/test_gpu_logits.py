"""Answers read from rows of logits, their gradient, and distillation, against plain forms in 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, DT, INF, U, Rows, answers, buffer, check_answers, context, near, place
from paper_2204_04179_b200 import binding

pytestmark = pytest.mark.gpu

# N, V, type, elements between the rows' ends and the next, elements ahead of the first row
SIZES = [(1, 1, "f32", 0, 0), (2, 1, "bf16", 3, 1), (3, 2, "f32", 0, 1), (4, 7, "bf16", 0, 0), (5, 31, "bf16", 2, 3),
         (300, 64, "f32", 0, 0), (7, 257, "f32", 3, 2), (600, 130, "bf16", 1, 0), (130, 1025, "bf16", 7, 5), (9, 2603, "f32", 0, 0),
         (33, 2048, "bf16", 0, 0), (40, 4099, "f32", 1, 3), (200, 8192, "f32", 0, 0), (2, 10_000, "f32", 0, 0), (1, 10_007, "bf16", 0, 1),
         (160, 16_384, "bf16", 0, 0), (3, 30_522, "bf16", 6, 0), (310, 30_522, "bf16", 0, 0), (5, 30_522, "f32", 0, 0), (75, 33_001, "f32", 0, 0),
         (4, 100_000, "f32", 0, 0), (1, 100_003, "f32", 0, 3), (20, 131_073, "bf16", 0, 0), (2, 262_147, "f32", 5, 0), (1, 600_011, "bf16", 0, 0)]


def _draw(N, V, seed, masked=0.05):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((N, V)) * 3
    z[rng.random((N, V)) < masked] = -INF
    z[:, 0] = np.where(np.isneginf(z).all(1), 0.5, z[:, 0])
    return rng, z


def _special(V, lowest):
    """Rows where a softmax or a selection goes wrong first."""
    rng = np.random.default_rng(V)
    rows = [np.full(V, -INF), np.full(V, lowest), np.full(V, 2.5), np.linspace(-30, 30, V), np.linspace(30, -30, V),
            np.where(np.arange(V) == V - 1, 1.0, -INF), np.where(np.arange(V) % 2 == 0, lowest, -INF),
            np.where(np.arange(V) % 3 == 0, 4.0, -4.0), rng.integers(-3, 4, V).astype(float),
            np.where(np.arange(V) == V // 2, 3.0e38, -3.0e38), np.where(np.arange(V) % 2 == 0, 0.0, -0.0),
            np.where(np.arange(V) < V // 2, lowest, rng.standard_normal(V)), np.full(V, -3.0e38) + 0 * rng.standard_normal(V)]
    return np.stack(rows)


def _targets(rng, N, V, C):
    return np.where(rng.random((N, C)) < 0.2, -1, rng.integers(0, V, (N, C))).astype(np.int32)


@pytest.mark.parametrize("k", [0, 1, 10, 128])
@pytest.mark.parametrize("N,V,dtype,pad,offset", SIZES)
def test_logprobs(N, V, dtype, pad, offset, k):
    rng, z = _draw(N, V, V + k)
    C = {0: 1, 1: 3, 10: 0, 128: 7}[k]
    scale = {0: 1.0, 1: 0.5, 10: 1.25, 128: 1.0}[k]
    view, z = place(z, dtype, pad, offset)
    targets = _targets(rng, N, V, C) if C else None
    g = context()
    out = answers(N, C, k)
    t = torch.from_numpy(targets).to(DEV) if C else None
    g.logprobs(view, scale=scale, targets=t, **out)
    g.sync()
    check_answers(out, Rows(z, scale), targets, k)
    again = answers(N, C, k)
    g.logprobs(view, scale=scale, targets=t, **again)
    g.sync()
    assert all(out[x] is None or torch.equal(out[x], again[x]) for x in out)
    g.close()


@pytest.mark.parametrize("scale", [1.0, 0.25, 3.0])
@pytest.mark.parametrize("V", [1, 3, 64, 300, 2603, 5000, 20_001, 70_000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logprobs_of_rows_that_go_wrong_first(dtype, V, scale):
    lowest = float(torch.finfo(DT[dtype]).min)
    view, z = place(_special(V, lowest), dtype, 1, 0)
    g = context()
    targets = np.stack([np.zeros(len(z)), np.full(len(z), V - 1), np.full(len(z), V // 2)], 1).astype(np.int32)
    for k in (5, 100):
        out = answers(len(z), 3, k)
        g.logprobs(view, scale=scale, targets=torch.from_numpy(targets).to(DEV), **out)
        g.sync()
        r = Rows(z, scale)
        with np.errstate(all="ignore"):                 # a difference that leaves 32 bits is -inf there
            r.logp = np.where(r.logp < -float(np.finfo(np.float32).max), -INF, r.logp)
        check_answers(out, r, targets, k)
    g.close()


@pytest.mark.parametrize("V", [5, 700, 9000, 40_000])
def test_a_row_with_nan_or_infinity_keeps_to_itself(V):
    rng, z = _draw(9, V, 3)
    z[1, V // 2] = np.nan
    z[4, V - 1] = INF
    z[6] = -INF
    z[6, V - 1] = np.nan
    view, _ = place(z, "f32")
    g = context()
    out = answers(9, 1, 4)
    t = torch.zeros(9, 1, dtype=torch.int32, device=DEV)
    g.logprobs(view, targets=t, **out)
    bad = [1, 4, 6]
    good = [n for n in range(9) if n not in bad]
    for x in ("entropy", "logp"):
        assert torch.isnan(out[x][bad]).all(), x
    assert torch.isnan(out["stats"][bad, 1]).all()
    assert out["top_ids"][4, 0] == V - 1
    ids = out["top_ids"].cpu().numpy()
    assert ((ids >= -1) & (ids < V)).all()
    part = {x: out[x][good] for x in out}
    check_answers(part, Rows(z[good].astype(np.float32).astype(np.float64), 1.0), np.zeros((6, 1), np.int32), 4)
    dz, loss = torch.full((9, V), 7.0, device=DEV), torch.empty(9, device=DEV)
    tl = torch.zeros(9, 2, device=DEV)
    g.distill(view, torch.tensor([[0, 1]] * 9, dtype=torch.int32, device=DEV), tl, loss, dlogits=dz)
    assert torch.isnan(loss[[1, 4]]).all() and torch.isfinite(loss[good]).all()
    assert torch.isnan(dz[[1, 4]]).all() and torch.isfinite(dz[good]).all()
    assert loss[6] == 0 and (dz[6] == 0).all()           # both of the teacher's entries are masked out there
    g.sync()
    g.close()


def _backward_reference(r, targets, dlogp, dH, dtype):
    """(gradient by the formula, its bound) in 64 bits."""
    N, V, C = len(r.z), r.V, 0 if targets is None else targets.shape[1]
    gsum, at, mag = np.zeros(N), np.zeros((N, V)), np.zeros((N, V))
    for c in range(C):
        live = (targets[:, c] >= 0) & ~np.isneginf(r.at(r.z, targets[:, c:c + 1], -INF)[:, 0])
        gl = np.where(live, dlogp[:, c].astype(float), 0.0)
        np.add.at(at, (np.arange(N), np.maximum(targets[:, c], 0)), gl)
        np.add.at(mag, (np.arange(N), np.maximum(targets[:, c], 0)), np.abs(gl))
        gsum += gl
    lp = np.where(r.p > 0, r.logp, 0.0)
    h = np.zeros(N) if dH is None else dH.astype(float)
    inner = gsum[:, None] + h[:, None] * (lp + r.H[:, None])
    want = r.scale * np.where(np.isneginf(r.z), 0.0, at - r.p * inner)
    # log p from rounded statistics: 2 u |log s| more; the factor's own roundings: d_logp |h| + 8 u of its parts
    size = np.abs(gsum)[:, None] + np.abs(h)[:, None] * (np.abs(lp) + r.H[:, None])
    d_lp = r.d_logp + 2 * U * np.abs(np.where(r.empty, 0, r.log_s))[:, None]
    bound = r.scale * (r.d_p * size + r.p * (np.abs(h)[:, None] * d_lp + (16 + C) * U * size + C * U * mag.sum(1, keepdims=True)) + (8 + C) * U * mag) + 1e-37
    if dtype == "bf16":
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    return want, bound


@pytest.mark.parametrize("what", ["both", "tokens", "entropy"])
@pytest.mark.parametrize("N,V,dtype,pad,offset", SIZES)
def test_logprobs_backward(N, V, dtype, pad, offset, what):
    rng, z = _draw(N, V, V + 1)
    if N > 2:
        z[1] = -INF
    scale, C = {"both": (0.5, 7), "tokens": (1.0, 1), "entropy": (1.25, 0)}[what]
    view, z = place(z, dtype, pad, offset)
    r = Rows(z, scale)
    stats = np.stack([r.m, r.log_s], 1).astype(np.float32)
    H = r.H.astype(np.float32)
    targets = _targets(rng, N, V, C) if C else None
    if C > 2:
        targets[:, 2] = targets[:, 1]                    # the same token twice
    dlogp = rng.standard_normal((N, C)).astype(np.float32) if C else None
    dH = rng.standard_normal(N).astype(np.float32) if what != "tokens" else None
    if N > 4 and C:
        targets[3] = -1                                  # a row with nothing given
    up = lambda a: None if a is None else torch.from_numpy(a).to(DEV)  # noqa: E731
    want, bound = _backward_reference(r, targets, dlogp, dH, dtype)
    g = context()
    for same in (False, True):
        if same:
            dz = view
        else:
            flat, dz = buffer(N, V, dtype, pad, offset)
        g.logprobs_backward(view, up(stats), dz, scale=scale, targets=up(targets), dlogp=up(dlogp), entropy=up(H), dentropy=up(dH))
        g.sync()
        near(dz, want, bound, f"gradient, in place {same}")
        assert (dz[torch.from_numpy(np.isneginf(z)).to(DEV)] == 0).all()
        if not same:                                     # nothing around the rows was touched
            torch.as_strided(flat, (N, V), (V + pad, 1), offset).fill_(float("nan"))
            assert torch.isnan(flat).all()
    g.close()


def test_logprobs_backward_against_differences():
    """Central differences of the forward call: the step of 2^-4 leaves |f'''| / 6 2^-8 <= 2^-8 / 6 sum |coefficients| per token and
    twice that for the entropy; the values' own errors of about 2^-20 are divided by the step."""
    N, V, C, scale, step = 3, 24, 2, 0.8, 2.0 ** -4
    rng, z = _draw(N, V, 5, masked=0.0)
    z = np.round(z * 8) / 8
    targets = _targets(rng, N, V, C)
    dlogp, dH = rng.standard_normal((N, C)).astype(np.float32), rng.standard_normal(N).astype(np.float32)
    g = context()
    up = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    many = np.repeat(z[None], 2 * V, 0)                   # [2 V, N, V]: each place moved up and down
    for v in range(V):
        many[2 * v, :, v] += step
        many[2 * v + 1, :, v] -= step
    rows = torch.from_numpy(many.reshape(-1, V)).float().to(DEV)
    out = answers(len(rows), C)
    g.logprobs(rows, scale=scale, targets=up(np.tile(targets, (2 * V, 1))), **out)
    f = (out["logp"].double().cpu().numpy().reshape(2 * V, N, C) * dlogp).sum(2) + out["entropy"].double().cpu().numpy().reshape(2 * V, N) * dH
    want = ((f[0::2] - f[1::2]) / (2 * step)).T
    view = torch.from_numpy(z).float().to(DEV)
    out = answers(N, C)
    g.logprobs(view, scale=scale, targets=up(targets), **out)
    dz = torch.empty_like(view)
    g.logprobs_backward(view, out["stats"], dz, scale=scale, targets=up(targets), dlogp=up(dlogp), entropy=out["entropy"], dentropy=up(dH))
    bound = (2.0 ** -8 / 6 + 2.0 ** -15) * (np.abs(dlogp).sum(1) + 2 * np.abs(dH))[:, None]
    near(dz, want, bound, "differences")
    g.sync()
    g.close()


def _distill_reference(r, ids, a, weight):
    """(loss, its bound, gradient, its bound) in 64 bits."""
    N, k = ids.shape
    loss, d_loss = np.zeros(N), np.zeros(N)
    want, bound = np.zeros_like(r.p), np.zeros_like(r.p)
    for n in range(N):
        use = [j for j in range(k) if ids[n, j] >= 0 and r.z[n, ids[n, j]] > -INF and a[n, j] > -INF]
        if not use:
            continue
        x = r.scale * (a[n, use] - a[n, use].max())
        lq = x - np.log(np.exp(x).sum())
        q = np.exp(lq)
        at = ids[n, use]
        loss[n] = (q * (lq - r.logp[n, at])).sum()
        # q's logarithm as log p's bound with V = k; each factor and the sum of k terms
        dlq = 2.0 ** -22 + (k + 80) * U * (1 + np.abs(x) + np.abs(lq))
        d_loss[n] = (q * (dlq + r.d_logp[n, at]) + q * np.abs(lq - r.logp[n, at]) * (dlq + 2.0 ** -21 + (k + 8) * U)).sum() + 1e-37
        g = r.p[n].copy()
        b = r.d_p[n] + 4 * U * r.p[n]
        np.subtract.at(g, at, q)
        np.add.at(b, at, q * (dlq + 2.0 ** -21 + (k + 4) * U))
        w = abs(float(weight[n])) * r.scale
        want[n], bound[n] = float(weight[n]) * r.scale * g, w * (b + 4 * U * np.abs(g)) + 1e-37
    return loss, d_loss, want, bound


@pytest.mark.parametrize("k", [1, 10, 64, 128])
@pytest.mark.parametrize("N,V,dtype,pad,offset", SIZES)
def test_distill(N, V, dtype, pad, offset, k):
    rng, z = _draw(N, V, V + k)
    if N > 2:
        z[1] = -INF
    view, z = place(z, dtype, pad, offset)
    scale = {1: 1.0, 10: 0.5, 64: 1.25, 128: 0.7}[k]
    r = Rows(z, scale)
    ids = np.where(rng.random((N, k)) < 0.15, -1, rng.integers(0, V, (N, k))).astype(np.int32)   # small V: the same place many times
    a = (rng.standard_normal((N, k)) * 3).astype(np.float32)
    a[rng.random((N, k)) < 0.05] = -INF
    weight = rng.random(N).astype(np.float32)
    if N > 4:
        ids[3], weight[4] = -1, 0.0
    up = lambda x: torch.from_numpy(x).to(DEV)  # noqa: E731
    loss, d_loss, want, bound = _distill_reference(r, ids, a.astype(float), weight)
    if dtype == "bf16":
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    g = context()
    got = torch.full((N,), float("nan"), device=DEV)
    g.distill(view, up(ids), up(a), got, scale=scale)
    near(got, loss, d_loss, "loss alone")
    for same in (False, True):
        if same:
            dz = view
        else:
            flat, dz = buffer(N, V, dtype, pad, offset)
        got = torch.full((N,), float("nan"), device=DEV)
        g.distill(view, up(ids), up(a), got, scale=scale, weight=up(weight), dlogits=dz)
        g.sync()
        near(got, loss, d_loss, "loss")
        near(dz, want, bound, f"gradient, in place {same}")
        if N > 4:
            assert (dz[3] == 0).all() and (dz[4] == 0).all()
        if not same:
            torch.as_strided(flat, (N, V), (V + pad, 1), offset).fill_(float("nan"))
            assert torch.isnan(flat).all()
    g.close()


@pytest.mark.parametrize("pad_out,offset_out", [(0, 0), (1, 0), (3, 2), (8, 5)])
@pytest.mark.parametrize("V", [100, 5001, 50_000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_into_rows_of_another_stride(dtype, V, pad_out, offset_out):
    N, k = 6, 5
    rng, z = _draw(N, V, V)
    view, z = place(z, dtype, 2, 1)
    r = Rows(z, 1.0)
    ids = rng.integers(0, V, (N, k)).astype(np.int32)
    a = rng.standard_normal((N, k)).astype(np.float32)
    up = lambda x: torch.from_numpy(x).to(DEV)  # noqa: E731
    _, _, want, bound = _distill_reference(r, ids, a.astype(float), np.ones(N))
    g = context()
    _, tight = buffer(N, V, dtype, 2, 1)
    flat, dz = buffer(N, V, dtype, pad_out, offset_out)
    loss = torch.empty(N, device=DEV)
    g.distill(view, up(ids), up(a), loss, dlogits=dz)
    g.distill(view, up(ids), up(a), loss, dlogits=tight)
    near(dz, want, bound + (2.0 ** -8 * np.abs(want) * 1.01 if dtype == "bf16" else 0), "gradient")
    assert torch.equal(dz, tight)
    stats, H = up(np.stack([r.m, r.log_s], 1).astype(np.float32)), up(r.H.astype(np.float32))
    t, dl, dh = up(ids[:, :1].copy()), up(a[:, :1].copy()), up(a[:, 1].copy())
    for out in (dz, tight):
        g.logprobs_backward(view, stats, out, targets=t, dlogp=dl, entropy=H, dentropy=dh)
    assert torch.equal(dz, tight)
    g.sync()
    dz.fill_(float("nan"))
    assert torch.isnan(flat).all()
    g.close()


def test_distill_against_differences():
    """As for the log probabilities: |f'''| / 6 2^-8 with the loss's third derivative at most 1."""
    N, V, k, scale, step = 3, 20, 4, 0.8, 2.0 ** -4
    rng, z = _draw(N, V, 8, masked=0.0)
    z = np.round(z * 8) / 8
    ids = np.stack([rng.permutation(V)[:k] for _ in range(N)]).astype(np.int32)
    a = rng.standard_normal((N, k)).astype(np.float32)
    up = lambda x: torch.from_numpy(x).to(DEV)  # noqa: E731
    many = np.repeat(z[None], 2 * V, 0)
    for v in range(V):
        many[2 * v, :, v] += step
        many[2 * v + 1, :, v] -= step
    rows = torch.from_numpy(many.reshape(-1, V)).float().to(DEV)
    g = context()
    loss = torch.empty(len(rows), device=DEV)
    g.distill(rows, up(np.tile(ids, (2 * V, 1))), up(np.tile(a, (2 * V, 1))), loss, scale=scale)
    f = loss.double().cpu().numpy().reshape(2 * V, N)
    want = ((f[0::2] - f[1::2]) / (2 * step)).T
    view = torch.from_numpy(z).float().to(DEV)
    dz, loss = torch.empty_like(view), torch.empty(N, device=DEV)
    g.distill(view, up(ids), up(a), loss, scale=scale, dlogits=dz)
    near(dz, want, 2.0 ** -8 / 6 + 2.0 ** -15, "differences")
    g.sync()
    g.close()


# V, type, elements between rows, elements ahead, k: as many rows as give each one a warp (the few are repeated)
MANY = [(1, "f32", 0, 0, 1), (7, "bf16", 1, 1, 5), (300, "f32", 0, 0, 128), (1000, "bf16", 0, 3, 128), (1029, "f32", 3, 1, 10), (2500, "f32", 0, 0, 32),
        (3001, "bf16", 2, 5, 16), (5000, "f32", 0, 0, 31), (10_001, "bf16", 0, 0, 20), (16_384, "f32", 0, 0, 16), (16_381, "f32", 2, 3, 10),
        (32_760, "bf16", 1, 7, 3), (20_000, "bf16", 0, 0, 0)]


def _tiled(few, N, dtype, pad, offset):
    base, z = place(few, dtype)
    flat, view = buffer(N, few.shape[1], dtype, pad, offset)
    view.copy_(base.repeat(-(-N // len(few)), 1)[:N])
    return flat, view, z


def _same(a, n, what, bound=None):
    """Each group of n rows holds, to the bit, what the first n hold; within twice `bound` of it where one is given (repeated rows
    of another alignment, whose sums take another order)."""
    a = torch.nan_to_num(a.double(), nan=1.25e40, posinf=1.5e40, neginf=-1.5e40)
    wide = lambda x: x.repeat(-(-len(a) // n), *[1] * (x.dim() - 1))[:len(a)]  # noqa: E731
    if bound is None:
        assert torch.equal(a, wide(a[:n])), what
    else:
        bound = torch.from_numpy(np.broadcast_to(np.where(np.isfinite(bound), bound, 0.0), a[:n].shape).copy()).to(a.device)
        assert ((a - wide(a[:n])).abs() <= 2 * wide(bound)).all(), what


@pytest.mark.parametrize("V,dtype,pad,offset,k", MANY)
def test_logprobs_of_many_rows(V, dtype, pad, offset, k):
    N = 2400
    few = np.concatenate([_special(V, float(torch.finfo(DT[dtype]).min)), _draw(6, V, V)[1]])
    n = len(few)
    flat, view, z = _tiled(few, N, dtype, pad, offset)
    targets = _targets(np.random.default_rng(V), n, V, 3)
    g = context()
    out = answers(N, 3, k)
    g.logprobs(view, scale=0.5, targets=torch.from_numpy(np.tile(targets, (N // n + 1, 1))[:N].copy()).to(DEV), **out)
    g.sync()
    r = Rows(z, 0.5)
    check_answers({x: None if out[x] is None else out[x][:n] for x in out}, r, targets, k)
    aligned = (V + pad) * view.element_size() % 16 == 0
    bounds = dict(stats=np.stack([np.zeros(n), r.d_log_s], 1), entropy=r.d_H, logp=r.at(r.d_logp, targets, 0.0))
    if k:
        bounds["top_logp"] = r.at(r.d_logp, r.top(k), 0.0)
    for x in out:
        if out[x] is not None:
            _same(out[x], n, x, None if aligned else bounds.get(x))
    view[5] = float("nan")                               # of one warp's row; its neighbours in the block keep theirs
    view[6, V - 1] = INF
    again = answers(N, 0, k)
    g.logprobs(view, scale=0.5, **again)
    g.sync()
    assert torch.isnan(again["entropy"][5:7]).all() and torch.isnan(again["stats"][5:7, 1]).all()
    rest = [i for i in range(N) if i not in (5, 6)]
    for x in ("stats", "entropy", "top_logp", "top_ids"):
        assert again[x] is None or torch.equal(again[x][rest], out[x][rest])
    if k:
        ids = again["top_ids"].cpu().numpy()
        assert ids[6, 0] == V - 1 and ((ids >= -1) & (ids < V)).all()
    g.close()


@pytest.mark.parametrize("order", ["ascending", "descending", "equal", "few values", "one warp's places"])
@pytest.mark.parametrize("V,dtype,k", [(9000, "f32", 16), (5000, "f32", 32), (500, "f32", 128), (30_000, "bf16", 12), (20_000, "f32", 128), (90_000, "f32", 100)])
def test_alternatives_that_crowd_together(V, dtype, k, order):
    """Rows whose better logits fall to few threads, or tie, with a warp, a block and a cluster a row."""
    i = np.arange(V)
    z = {"ascending": i / 256.0, "descending": -i / 256.0, "equal": np.zeros(V), "few values": (i % 7) * 0.5,
         "one warp's places": np.where(i // 4 % 32 == 3, 8.0 + (i % 11) / 16.0, -(i % 97) / 64.0)}[order]
    for N in (1, 200, 2400):
        flat, view, want = _tiled(z[None], N, dtype, 0, 0)
        g = context()
        out = answers(N, 0, k)
        g.logprobs(view, **out)
        g.sync()
        check_answers({x: None if out[x] is None else out[x][:1] for x in out}, Rows(want, 1.0), None, k)
        for x in ("stats", "entropy", "top_logp", "top_ids"):
            _same(out[x], 1, x)
        g.close()


@pytest.mark.parametrize("k", [1, 17, 128])
@pytest.mark.parametrize("V,dtype,pad,offset", [(1, "f32", 0, 0), (9, "bf16", 0, 1), (700, "f32", 0, 0), (1999, "bf16", 3, 5), (2048, "f32", 0, 0),
                                                (3000, "f32", 0, 0), (2999, "f32", 1, 3), (6000, "bf16", 2, 1), (6144, "bf16", 0, 0),
                                                (5000, "f32", 0, 0), (10_001, "bf16", 3, 1)])
def test_gradients_of_many_rows(V, dtype, pad, offset, k):
    N = 2400
    rng, few = _draw(16, V, V + k)
    few[1] = -INF
    few[2] = np.where(np.arange(V) % 2 == 0, float(torch.finfo(DT[dtype]).min), -INF)
    n = len(few)
    flat, view, z = _tiled(few, N, dtype, pad, offset)
    r = Rows(z, 0.5)
    ids = np.where(rng.random((n, k)) < 0.15, -1, rng.integers(0, V, (n, k))).astype(np.int32)
    a = (rng.standard_normal((n, k)) * 3).astype(np.float32)
    weight = rng.random(n).astype(np.float32)
    ids[3], weight[4] = -1, 0.0
    up = lambda x: torch.from_numpy(np.concatenate([x] * (N // n)).copy()).to(DEV)  # noqa: E731
    loss, d_loss, want, bound = _distill_reference(r, ids, a.astype(float), weight)
    if dtype == "bf16":
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    g = context()
    got = torch.full((N,), float("nan"), device=DEV)
    out, dz = buffer(N, V, dtype, pad, offset)
    g.distill(view, up(ids), up(a), got, scale=0.5, weight=up(weight), dlogits=dz)
    g.sync()
    near(got[:n], loss, d_loss, "loss")
    near(dz[:n], want, bound, "gradient")
    aligned = (V + pad) * view.element_size() % 16 == 0
    _same(got, n, "loss", None if aligned else d_loss)
    _same(dz, n, "gradient", None if aligned else bound)
    stats, H = np.stack([r.m, r.log_s], 1).astype(np.float32), r.H.astype(np.float32)
    dh = rng.standard_normal(n).astype(np.float32)
    there = dz.clone()
    g.logprobs_backward(view, up(stats), dz, scale=0.5, targets=up(ids), dlogp=up(a), entropy=up(H), dentropy=up(dh))
    g.sync()
    want, bound = _backward_reference(r, ids, a, dh, dtype)
    near(dz[:n], want, bound, "backward")
    _same(dz, n, "backward", None if aligned else bound)
    g.distill(view, up(ids), up(a), got, scale=0.5, weight=up(weight), dlogits=view)      # in place
    g.sync()
    assert torch.equal(view, there)
    dz.fill_(float("nan"))
    assert torch.isnan(out).all()
    g.close()


@pytest.mark.parametrize("blocks", [1, 2, 4])
def test_with_smaller_clusters(blocks):
    """Where the device places no cluster of 8, or none at all, rows are cut into fewer slices."""
    N, V, k = 5, 70_001, 40
    rng, z = _draw(N, V, 2)
    z[1] = -INF
    view, z = place(z, "f32", 2, 1)
    r = Rows(z, 0.5)
    ids = rng.integers(0, V, (N, k)).astype(np.int32)
    a = rng.standard_normal((N, k)).astype(np.float32)
    up = lambda x: torch.from_numpy(x).to(DEV)  # noqa: E731
    loss, d_loss, want, bound = _distill_reference(r, ids, a.astype(float), np.ones(N))
    g = context()
    g.selftest_cluster_blocks(blocks)
    out = answers(N, k, k)
    g.logprobs(view, scale=0.5, targets=up(ids), **out)
    g.sync()
    check_answers(out, r, ids, k)
    dz, got = torch.empty(N, V, device=DEV), torch.empty(N, device=DEV)
    dl, dh = up(a), up(a[:, 0].copy())
    g.logprobs_backward(view, out["stats"], dz, scale=0.5, targets=up(ids), dlogp=dl, entropy=out["entropy"], dentropy=dh)
    whole, back = context(), torch.empty_like(dz)
    whole.logprobs_backward(view, out["stats"], back, scale=0.5, targets=up(ids), dlogp=dl, entropy=out["entropy"], dentropy=dh)
    whole.sync()
    g.sync()
    assert torch.equal(dz, back)
    whole.close()
    g.distill(view, up(ids), up(a), got, scale=0.5, dlogits=view)
    g.sync()
    near(got, loss, d_loss, "loss")
    near(view, want, bound, "gradient")
    g.close()


def test_a_teachers_alternatives_are_its_students_lists():
    """What gram_logprobs writes goes into gram_distill as it stands; a student that equals its teacher over a pool of k has no loss."""
    _, z = _draw(8, 100, 4)
    z[2] = -INF
    view, z = place(z, "f32")
    g = context()
    out = answers(8, 0, 100)
    g.logprobs(view, **out)
    loss, dz = torch.empty(8, device=DEV), torch.empty_like(view)
    g.distill(view, out["top_ids"], out["top_logp"], loss, dlogits=dz)
    g.sync()
    r = Rows(z, 1.0)
    assert (loss.abs().double().cpu().numpy() <= 4 * r.d_logp.max(1)).all()
    near(dz, np.zeros_like(z), 4 * r.d_p + 8 * U * r.p, "gradient")
    g.close()


def test_rows_past_2_to_the_31_elements():
    ld, V = (1 << 30) + 8, 1000
    flat = torch.empty(2 * ld + V, dtype=torch.bfloat16, device=DEV)
    view = flat.as_strided((3, V), (ld, 1))
    _, z = _draw(3, V, 1)
    view.copy_(torch.from_numpy(z).to(torch.bfloat16))
    z = view.double().cpu().numpy()
    g = context()
    out = answers(3, 0, 3)
    g.logprobs(view, **out)
    r = Rows(z, 1.0)
    check_answers(out, r, None, 3)
    ids, loss = out["top_ids"].clone(), torch.empty(3, device=DEV)
    g.distill(view, ids, torch.zeros(3, 3, device=DEV), loss, dlogits=view)
    _, _, want, bound = _distill_reference(r, ids.cpu().numpy(), np.zeros((3, 3)), np.ones(3))
    near(view, want, bound + 2.0 ** -8 * np.abs(want) * 1.01, "gradient")
    g.sync()
    g.close()


def test_tokens_out_of_range_are_recorded_and_count_as_none():
    _, z = _draw(4, 50, 1)
    view, z = place(z, "f32")
    g = context()
    t = torch.tensor([[3], [50], [-2], [2 ** 31 - 1]], dtype=torch.int32, device=DEV)
    out = answers(4, 1)
    g.logprobs(view, targets=t, **out)
    with pytest.raises(binding.GramError) as e:
        g.sync()
    assert e.value.status == 2
    assert (out["logp"][1:] == 0).all()
    dz = torch.full_like(view, 7.0)
    g.logprobs_backward(view, out["stats"], dz, targets=t, dlogp=torch.ones(4, 1, device=DEV))
    with pytest.raises(binding.GramError):
        g.sync()
    assert (dz[1:] == 0).all() and (dz[0] != 0).any()
    loss = torch.empty(4, device=DEV)
    g.distill(view, t, torch.zeros(4, 1, device=DEV), loss, dlogits=dz)
    with pytest.raises(binding.GramError):
        g.sync()
    assert (loss[1:] == 0).all() and (dz[1:] == 0).all() and (dz[0] != 0).any()
    g.sync()
    g.close()


def test_no_rows():
    g = context()
    view = torch.empty(0, 10, device=DEV)
    g.logprobs(view, **answers(0, 0, 2))
    g.logprobs_backward(view, torch.empty(0, 2, device=DEV), torch.empty(0, 10, device=DEV))
    g.distill(view, torch.empty(0, 2, dtype=torch.int32, device=DEV), torch.empty(0, 2, device=DEV), torch.empty(0, device=DEV))
    g.sync()
    g.close()


def test_on_another_stream_behind_its_work():
    N, V = 64, 20_000
    _, z = _draw(N, V, 6)
    want = torch.from_numpy(z).float().to(DEV)
    view = torch.zeros_like(want)
    g = context()
    out, dz, loss = answers(N, 0, 3), torch.empty_like(want), torch.empty(N, device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a = torch.randn(4096, 4096, device=DEV)
        for _ in range(20):
            a = a @ a * 1e-3
        view.copy_(want)
        g.logprobs(view, **out)
        g.distill(view, out["top_ids"], out["top_logp"], loss, dlogits=dz)
        view.zero_()                                     # the calls have read it by then
    g.sync(s)
    check_answers(out, Rows(want.double().cpu().numpy(), 1.0), None, 3)
    assert torch.isfinite(dz).all() and torch.isfinite(loss).all()
    g.close()


def test_refusals():
    g = context()
    z = torch.zeros(4, 16, device=DEV)
    f, i = torch.zeros(4, 200, device=DEV), torch.zeros(4, 200, dtype=torch.int32, device=DEV)
    st = torch.zeros(4, 2, device=DEV)
    L, P = binding.lib(), lambda t: C.c_void_p(0 if t is None else t.data_ptr())  # noqa: E731

    def refused(status, fn, *args):
        assert fn(g._h, *args) == status, fn
        assert L.gram_last_error(g._h)

    def logprobs(p=P(z), dtype=0, ld=16, N=4, V=16, scale=1.0, t=None, nc=0, lp=None, ti=None, tl=None, k=0):
        return (p, C.c_int(dtype), C.c_int64(ld), C.c_int64(N), C.c_int32(V), C.c_float(scale), P(t), C.c_int32(nc), P(lp), P(st), P(None),
                P(tl), P(ti), C.c_int32(k), C.c_void_p(0))
    for bad in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(V=0), dict(N=-1), dict(ld=15),
                dict(dtype=2), dict(p=P(None)), dict(p=C.c_void_p(z.data_ptr() + 2)), dict(nc=129, t=i, lp=f), dict(nc=-1), dict(k=129, ti=i, tl=f),
                dict(nc=1, t=i), dict(nc=1, lp=f), dict(k=1, ti=i), dict(k=1, tl=f), dict(N=1 << 31, ld=1 << 40), dict(ld=1 << 62)):
        refused(1, L.gram_logprobs, *logprobs(**bad))

    def backward(dz=P(f), ld_out=16, stats=P(st), H=None, dh=None, t=None, nc=0, dl=None):
        return (P(z), C.c_int(0), C.c_int64(16), C.c_int64(4), C.c_int32(16), C.c_float(1.0), P(t), C.c_int32(nc), stats, P(H), P(dl), P(dh), dz,
                C.c_int64(ld_out), C.c_void_p(0))
    for bad in (dict(dz=P(None)), dict(ld_out=8), dict(stats=P(None)), dict(dh=f), dict(nc=1, t=i), dict(nc=1, dl=f), dict(nc=129, t=i, dl=f),
                dict(dz=C.c_void_p(z.data_ptr() + 64)), dict(dz=P(z), ld_out=17), dict(dz=C.c_void_p(f.data_ptr() + 1))):
        refused(1, L.gram_logprobs_backward, *backward(**bad))

    def distill(ids=i, a=f, k=2, loss=f, dz=None, ld_out=16, scale=1.0):
        return (P(z), C.c_int(0), C.c_int64(16), C.c_int64(4), C.c_int32(16), C.c_float(scale), P(ids), P(a), C.c_int32(k), P(loss), P(None),
                dz or P(None), C.c_int64(ld_out), C.c_void_p(0))
    for bad in (dict(ids=None), dict(a=None), dict(loss=None), dict(k=0), dict(k=129), dict(scale=0.0), dict(dz=P(f), ld_out=3),
                dict(dz=C.c_void_p(z.data_ptr() + 4))):
        refused(1, L.gram_distill, *distill(**bad))
    g.logprobs(z, stats=st)                              # the context stays usable
    g.sync()
    assert abs(float(st[0, 1]) - np.log(16)) < 1e-6
    g.close()
