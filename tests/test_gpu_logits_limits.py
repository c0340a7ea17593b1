"""Logits and scales at the ends of their types, rows of NaN, and what else a softmax goes wrong on first, in each form of the calls
on rows of logits: a warp a row, a block, and a cluster of blocks."""
import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, DT, INF, Rows, answers, check_answers, context, near, place
from tests.test_gpu_logits import _backward_reference, _distill_reference, _special
from paper_2204_04179_b200 import binding

pytestmark = pytest.mark.gpu

LARGEST = float(np.finfo(np.float32).max)
# N, V, type: a warp a row, a block (rows of 24 KB, more than two of them per block that the GPU holds), a cluster
FORMS = [(2400, 700, "f32"), (2400, 1501, "bf16"), (1200, 6000, "f32"), (1200, 12_003, "bf16"), (14, 20_001, "f32"), (14, 40_000, "bf16")]


def _up(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _tile(x, N):
    return np.concatenate([x] * -(-N // len(x)))[:N]


# ------------------------------ a teacher whose logits are large in size ------------------------------
def _teachers(k):
    """Rows of a teacher's logits, k each: all alike at a large size, near one another there, and mixed with ordinary ones."""
    i = np.arange(k)
    rows = [np.full(k, -1e9), np.full(k, -LARGEST), np.full(k, 1e12), np.full(k, LARGEST), np.full(k, -6e6), -6e6 - 0.5 * (i % 7),
            6e6 + 0.5 * (i % 5), 1e12 + 65536.0 * (i % 3), np.where(i % 2 == 0, -1e9, -2e9), np.where(i == k // 2, 1.5, -LARGEST),
            np.where(i % 3 == 0, LARGEST, -LARGEST), np.where(i == 0, -1e9, -INF), np.full(k, -INF), np.sin(i)]
    return np.stack(rows).astype(np.float32)


@pytest.mark.parametrize("k", [1, 10, 128])
@pytest.mark.parametrize("N,V,dtype", FORMS)
def test_distill_from_a_teacher_of_large_logits(N, V, dtype, k):
    """Only an entry at -inf takes no part: loss and gradient are those of the definition at any finite size."""
    a = _teachers(k)
    n = len(a)
    rng = np.random.default_rng(V + k)
    few = rng.standard_normal((n, V)) * 3
    few[rng.random((n, V)) < 0.05] = -INF
    few[:, 0] = 0.25
    base, z = place(few, dtype)
    ids = rng.integers(0, V, (n, k)).astype(np.int32)
    ids[:, 0] = 0                                        # one entry of every row is there in any case
    weight = rng.random(n).astype(np.float32) + 0.5
    r = Rows(z, 0.5)
    loss, d_loss, want, bound = _distill_reference(r, ids, a.astype(float), weight)
    if dtype == "bf16":
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    view = base.repeat(-(-N // n), 1)[:N].contiguous()
    g = context()
    got, dz = torch.full((N,), float("nan"), device=DEV), torch.full_like(view, float("nan"))
    args = _up(_tile(ids, N)), _up(_tile(a, N)), got
    g.distill(view, *args, scale=0.5, weight=_up(_tile(weight, N)), dlogits=dz)
    g.sync()
    for first in range(0, N, n):
        m = min(n, N - first)
        near(got[first:first + m], loss[:m], d_loss[:m], "loss")
        if first < 2 * n or first + n >= N:
            near(dz[first:first + m], want[:m], bound[:m], "gradient")
    g.distill(view, *args, scale=0.5, weight=_up(_tile(weight, N)), dlogits=view)        # in place
    g.sync()
    assert torch.equal(view, dz)
    g.close()


def test_distill_from_a_teacher_of_large_logits_against_differences():
    """Central differences of the loss, whose third derivative is 1 at most: the step of 2^-4 leaves 2^-8 / 6, the values' errors of
    about 2^-20 are divided by it."""
    k, V, scale, step = 4, 20, 0.8, 2.0 ** -4
    a = _teachers(k)
    N = len(a)
    rng = np.random.default_rng(8)
    z = np.round(rng.standard_normal((N, V)) * 24) / 8
    ids = np.stack([rng.permutation(V)[:k] for _ in range(N)]).astype(np.int32)
    many = np.repeat(z[None], 2 * V, 0)
    for v in range(V):
        many[2 * v, :, v] += step
        many[2 * v + 1, :, v] -= step
    rows = _up(many.reshape(-1, V).astype(np.float32))
    g = context()
    loss = torch.empty(len(rows), device=DEV)
    g.distill(rows, _up(np.tile(ids, (2 * V, 1))), _up(np.tile(a, (2 * V, 1))), loss, scale=scale)
    f = loss.double().cpu().numpy().reshape(2 * V, N)
    want = ((f[0::2] - f[1::2]) / (2 * step)).T
    view = _up(z.astype(np.float32))
    dz, loss = torch.empty_like(view), torch.empty(N, device=DEV)
    g.distill(view, _up(ids), _up(a), loss, scale=scale, dlogits=dz)
    near(dz, want, 2.0 ** -8 / 6 + 2.0 ** -15, "differences")
    g.sync()
    g.close()


# ------------------------------ log probabilities that leave 32 bits ------------------------------
@pytest.mark.parametrize("scale", [0.5, 2.0, 10.0, 1e6])
@pytest.mark.parametrize("N,V,dtype", FORMS + [(3, 4, "f32")])
def test_log_probabilities_beyond_32_bits(N, V, dtype, scale):
    """Rows of logits near the type's lowest value, the largest among them too: an entry whose log probability leaves 32 bits has
    -inf, never NaN."""
    lowest = float(torch.finfo(DT[dtype]).min)
    i = np.arange(V)
    few = np.stack([np.where(i % 2 == 0, -1e38, lowest), np.where(i == V - 1, -2e38, lowest), np.where(i % 3 == 0, 1e38, lowest)])
    base, z = place(few, dtype)
    view = base.repeat(-(-N // 3), 1)[:N].contiguous()
    targets = np.tile(np.array([[0, 1, V - 1]], np.int32), (3, 1))
    r = Rows(z, scale)
    with np.errstate(all="ignore"):
        r.logp = np.where(r.logp < -LARGEST, -INF, r.logp)
    g = context()
    out = answers(N, 3, V if V <= 128 else 128)
    g.logprobs(view, scale=scale, targets=_up(_tile(targets, N)), **out)
    g.sync()
    k = out["top_ids"].shape[1]
    for first in (0, N - N % 3 - 3):
        check_answers({x: out[x][first:first + 3] for x in out}, r, targets, k)
    g.close()


# ------------------------------ scales far from 1 ------------------------------
SCALES = [1e-30, 3e-24, 1e-12, 3e7, 1e9, 1e17, 1e30]


def _rows_of_scales(V, dtype):
    """Rows with masked places: ordinary ones, ones whose largest logit is 0, and those of _special."""
    rng = np.random.default_rng(V)
    z = rng.standard_normal((4, V)) * 3
    z[rng.random((4, V)) < 0.3] = -INF
    z[2] = np.where(np.isneginf(z[2]), -INF, -np.abs(z[2]))
    z[2, V // 2] = 0.0
    z[3] = np.where(np.arange(V) % 2 == 0, 0.0, -INF)
    return np.concatenate([z, _special(V, float(torch.finfo(DT[dtype]).min))])


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("N,V,dtype", FORMS + [(17, 3, "f32"), (17, 130, "bf16")])
def test_scales_far_from_one(N, V, dtype, scale):
    """A masked place has no weight, and an entry's share is that of the definition, however small or large the scale is."""
    base, z = place(_rows_of_scales(V, dtype), dtype)
    n, k, nc = len(z), 8, 3
    N = max(N, n)
    rng = np.random.default_rng(V)
    view = base.repeat(-(-N // n), 1)[:N].contiguous()
    r = Rows(z, scale)
    with np.errstate(all="ignore"):                      # what leaves 32 bits is -inf there
        r.logp = np.where(r.logp < -LARGEST, -INF, r.logp)
    targets = np.where(rng.random((n, nc)) < 0.2, -1, rng.integers(0, V, (n, nc))).astype(np.int32)
    g = context()
    with_top, without = answers(N, nc, k), answers(N, nc)
    for out in (with_top, without):
        g.logprobs(view, scale=scale, targets=_up(_tile(targets, N)), **out)
        g.sync()
        for first in {0, N // n // 2 * n, (N // n - 1) * n}:
            check_answers({x: None if out[x] is None else out[x][first:first + n] for x in out}, r, targets, k if out is with_top else 0)
    # gradients: powers below 2^-126 are 0, which with the scale ahead of them is scale 1e-37 at most
    stats, H = np.stack([r.m, r.log_s], 1).astype(np.float32), r.H.astype(np.float32)
    dlogp, dH = rng.standard_normal((n, nc)).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    more = lambda bound, want: (bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want) if dtype == "bf16" else bound) + r.scale * 1e-37  # noqa: E731
    dz = torch.full_like(view, float("nan"))
    g.logprobs_backward(view, _up(_tile(stats, N)), dz, scale=scale, targets=_up(_tile(targets, N)), dlogp=_up(_tile(dlogp, N)),
                        entropy=_up(_tile(H, N)), dentropy=_up(_tile(dH, N)))
    g.sync()
    want, bound = _backward_reference(r, targets, dlogp, dH, "f32")
    near(dz[:n], want, more(bound, want), "gradient")
    assert (dz[:n][torch.from_numpy(np.isneginf(z)).to(DEV)] == 0).all()
    a = rng.standard_normal((n, nc)).astype(np.float32)
    a[:, 1] = a[:, 0]
    loss = torch.empty(N, device=DEV)
    with np.errstate(all="ignore"):
        want_loss, d_loss, want, bound = _distill_reference(r, targets, a.astype(float), np.ones(n))
    g.distill(view, _up(_tile(targets, N)), _up(_tile(a, N)), loss, scale=scale, dlogits=dz)
    g.sync()
    fits = np.abs(want_loss) < LARGEST
    near(loss[:n][torch.from_numpy(fits).to(DEV)], want_loss[fits], d_loss[fits], "loss")
    near(dz[:n], want, more(bound, want), "gradient of distillation")
    g.close()


@pytest.mark.parametrize("scale", SCALES[::2])
@pytest.mark.parametrize("N,V", [(5, 3000), (300, 30_522), (700, 12_500)])
def test_scores_of_scales_far_from_one(N, V, scale):
    """Of small whole numbers, whose products are exact in any order: as logits that are written, and as lists of candidates."""
    d, k = 8, 5
    rng = np.random.default_rng(N)
    u, w = rng.integers(-3, 4, (N, d)).astype(float), rng.integers(-3, 4, (V, d)).astype(float)
    bias = np.where(rng.random(V) < 0.3, -INF, np.round(rng.standard_normal(V) * 256) / 256)
    bias[0] = 0.0
    targets = rng.integers(0, V, (N, 2)).astype(np.int32)
    r = Rows(u @ w.T + bias, scale)
    with np.errstate(all="ignore"):
        r.logp = np.where(r.logp < -LARGEST, -INF, r.logp)
    g = context()
    for kk in (k, 0):
        out = answers(N, 2, kk)
        g.score_logprobs(_up(u).to(torch.bfloat16), _up(w).to(torch.bfloat16), bias=_up(bias.astype(np.float32)), scale=scale, targets=_up(targets), **out)
        g.sync()
        check_answers(out, r, targets, kk)
    g.close()


def test_scales_that_are_refused():
    """Beyond 1e-30 and 1e30 differences of finite logits, and their gradients, leave 32 bits."""
    g = context()
    z, st = torch.zeros(4, 16, device=DEV), torch.zeros(4, 2, device=DEV)
    for scale in (9e-31, 1.1e30, 1e-45, 3e38):
        for call in (lambda: g.logprobs(z, scale=scale, stats=st), lambda: g.logprobs_backward(z, st, z, scale=scale),
                     lambda: g.distill(z, torch.zeros(4, 1, dtype=torch.int32, device=DEV), st[:, :1].contiguous(), st[:, 0].contiguous(), scale=scale),
                     lambda: g.score_logprobs(z.to(torch.bfloat16), z.to(torch.bfloat16), scale=scale, stats=st)):
            with pytest.raises(binding.GramError) as e:
                call()
            assert e.value.status == 1
    g.sync()
    g.close()


# ------------------------------ rows that hold NaN or +inf ------------------------------
@pytest.mark.parametrize("asked", ["none", "sum of 0", "tokens", "entropy", "no tokens"])
@pytest.mark.parametrize("N,V,dtype", FORMS + [(9, 5, "f32"), (9, 700, "bf16")])
def test_gradients_of_rows_with_nan_or_infinity(N, V, dtype, asked):
    """Their statistics and gradients are NaN whatever is asked of them, and those of the other rows as always."""
    rng = np.random.default_rng(V)
    n = 7
    few = rng.standard_normal((n, V)) * 3
    few[1, V // 2], few[4, V - 1], few[6] = np.nan, INF, -INF
    few[6, V - 1] = np.nan
    base, z = place(few, dtype)
    view = base.repeat(-(-N // n), 1)[:N].contiguous()
    bad, good = [1, 4, 6], [0, 2, 3, 5]
    targets = np.zeros((n, 2), np.int32)
    targets[:, 1] = V - 1
    dlogp = np.ones((n, 2), np.float32)
    dH = np.full(n, 0.5, np.float32) if asked == "entropy" else None
    if asked == "none":
        targets[:] = -1
    if asked == "sum of 0":
        dlogp[:, 1] = -1.0
    if asked == "no tokens":
        targets = dlogp = None
    g = context()
    out = answers(N, 0, 3)
    g.logprobs(view, **out)
    g.sync()
    stats = out["stats"][:n].cpu().numpy()
    assert np.isnan(stats[bad]).all() and np.isfinite(stats[good]).all()
    r = Rows(z[good], 1.0)
    entropy = out["entropy"][:n].cpu().numpy()
    stats[good], entropy[good] = np.stack([r.m, r.log_s], 1), r.H
    stats, entropy = _up(_tile(stats, N)), _up(_tile(entropy, N))
    dz = torch.full_like(view, 7.0)
    t, dl, dh = (_up(None if x is None else _tile(x, N)) for x in (targets, dlogp, dH))
    g.logprobs_backward(view, stats, dz, targets=t, dlogp=dl, entropy=entropy, dentropy=dh)
    g.sync()
    assert torch.isnan(dz[:n][bad]).all()
    want, bound = _backward_reference(r, None if targets is None else targets[good], None if dlogp is None else dlogp[good],
                                      None if dH is None else dH[good], dtype)
    near(dz[:n][good], want, bound, "gradient of the other rows")
    g.logprobs_backward(view, stats, view, targets=t, dlogp=dl, entropy=entropy, dentropy=dh)
    g.sync()
    assert torch.equal(torch.nan_to_num(view, nan=1e3), torch.nan_to_num(dz, nan=1e3))
    g.close()


@pytest.mark.parametrize("N,V", [(6, 900), (300, 30_522), (700, 12_500)])
def test_scores_with_nan_have_nan_statistics(N, V):
    rng = np.random.default_rng(1)
    users = torch.from_numpy(rng.integers(-3, 4, (N, 16)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    items = torch.from_numpy(rng.integers(-3, 4, (V, 16)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    users[3, 5] = float("nan")
    g = context()
    for k in (0, 4):
        out = answers(N, 0, k)
        g.score_logprobs(users, items, scale=0.05, **out)
        g.sync()
        assert torch.isnan(out["stats"][3]).all() and torch.isnan(out["entropy"][3])
        assert torch.isfinite(out["stats"][[0, 1, 2, 4, 5]]).all()
    g.close()


# ------------------------------ rows of 2^31 - 1 elements ------------------------------
@pytest.mark.parametrize("dtype,offset", [("bf16", 3), ("f32", 1)])
def test_a_row_of_the_most_elements(dtype, offset):
    """Places, vectors and single elements at the row's end count to 2^31 - 1 without leaving 32 bits; nothing behind the row is
    touched.  Places of -4 and a few hundred others, the last ones among them.  A thread of eight blocks adds up V / 2^10 elements, 16 or
    32 of them at a time: the sum is off by less than V 2^-14 u = 2^-7 of itself."""
    V, k, scale = 2 ** 31 - 1, 10, 0.5
    rng = np.random.default_rng(1)
    at = np.unique(np.concatenate([np.arange(V - 20, V), np.arange(20), rng.integers(0, V, 300)]))
    value = rng.permutation(len(at)) / 64.0               # exact in bf16 up to 4
    value = np.where(value < 4, value, -4.0)
    value[-1] = 3.875                                     # in the last place
    flat = torch.full((V + offset + 64,), -4.0, dtype=DT[dtype], device=DEV)
    flat[:offset], flat[offset + V:] = 9.0, 9.0
    row = flat[offset:offset + V].view(1, V)
    where = _up(at.astype(np.int64))
    row[0, where] = _up(value).to(DT[dtype])
    y = scale * (value - value.max())
    base = np.exp(scale * (-4.0 - value.max()))
    s = (V - len(at)) * base + np.exp(y).sum()
    order = np.lexsort((at, -value))[:k]
    g = context()
    out = answers(1, 2, k)
    targets = _up(np.array([[V - 1, at[len(at) // 2]]], np.int32))
    g.logprobs(row, scale=scale, targets=targets, **out)
    g.sync()
    assert out["top_ids"][0].tolist() == at[order].tolist()
    near(out["stats"][0], np.array([value.max(), np.log(s)]), np.array([0.0, 2.0 ** -6]), "statistics")
    near(out["logp"][0], np.array([y[-1], y[len(at) // 2]]) - np.log(s), 2.0 ** -6, "log p")
    p = np.exp(y) / s
    loss, ids = torch.empty(1, device=DEV), np.concatenate([at[-1:], at[:1]]).astype(np.int32)[None]
    g.distill(row, _up(ids), torch.zeros(1, 2, device=DEV), loss, scale=scale, dlogits=row)      # in place
    g.sync()
    want = p.copy()
    want[[-1, 0]] -= 0.5
    near(row[0, where], scale * want, 2.0 ** -6 * scale * np.abs(want), "gradient")
    rest = row[0, 21:10 ** 9 + 7:9973]
    rest = rest[(rest - float(scale * base / s)).abs() > 2.0 ** -6 * float(scale * base / s)]
    assert len(rest) <= 300                               # those of other values
    assert (flat[:offset] == 9).all() and (flat[offset + V:] == 9).all()
    row.fill_(-4.0)
    row[0, where] = _up(value).to(DT[dtype])
    g.logprobs_backward(row, out["stats"], row, scale=scale, targets=targets[:, :1].contiguous(), dlogp=torch.ones(1, 1, device=DEV))
    g.sync()
    want = -p
    want[-1] += 1.0
    near(row[0, where], scale * want, 2.0 ** -6 * scale * np.abs(want), "gradient of log p")
    assert (flat[:offset] == 9).all() and (flat[offset + V:] == 9).all()
    g.close()


def test_tables_of_too_many_items_are_refused():
    g = context()
    u, st = torch.zeros(4, 8, dtype=torch.bfloat16, device=DEV), torch.zeros(4, 2, device=DEV)
    P = lambda t: t.data_ptr()  # noqa: E731
    for V in (2 ** 31 - 1, 2 ** 31 - 127, 1_857_283_073):    # refused before anything is read
        assert binding.lib().gram_score_logprobs(g._h, P(u), 8, P(u), 8, None, 4, V, 8, 1.0, None, 0, None, P(st), None, None, None, 0, 0) == 4
    g.sync()
    g.close()


# ------------------------------ a gradient beside its logits ------------------------------
@pytest.mark.parametrize("N,V", [(5, 64), (2400, 300), (7, 20_001)])
def test_gradients_beside_their_logits(N, V):
    """Logits and gradients as the halves of one buffer's rows do not overlap, whichever comes first; what does is refused."""
    rng = np.random.default_rng(V)
    z = rng.standard_normal((N, V))
    a, ids = rng.standard_normal((N, 4)).astype(np.float32), rng.integers(0, V, (N, 4)).astype(np.int32)
    g = context()
    r = Rows(z.astype(np.float32).astype(np.float64), 1.0)
    _, _, want, bound = _distill_reference(r, ids, a.astype(float), np.ones(N))
    back, back_bound = _backward_reference(r, ids[:, :1], a[:, :1], None, "f32")
    stats, loss = _up(np.stack([r.m, r.log_s], 1).astype(np.float32)), torch.empty(N, device=DEV)
    flat = torch.zeros(N * (2 * V + 4) + 8, device=DEV)
    both = flat[:N * (2 * V + 3)].view(N, 2 * V + 3)
    left, right, middle = both[:, :V], both[:, V + 3:], both[:, V:2 * V]
    for logits, dz in ((left, right), (right, left), (left, middle)):
        logits.copy_(_up(z.astype(np.float32)))
        g.distill(logits, _up(ids), _up(a), loss, dlogits=dz)
        g.sync()
        near(dz, want, bound, "gradient")
        g.logprobs_backward(logits, stats, dz, targets=_up(ids[:, :1]), dlogp=_up(a[:, :1]))
        g.sync()
        near(dz, back, back_bound, "gradient of log p")
        assert torch.equal(logits, _up(z.astype(np.float32)))
    wide = flat[1:].as_strided((N, V), (2 * V + 4, 1))                    # rows of another distance run into the logits
    for logits, dz in ((left, both[:, V - 1:2 * V - 1]), (right, both[:, 4:V + 4]), (left, both[:, 1:V + 1]), (right, wide)):
        with pytest.raises(binding.GramError) as e:
            g.distill(logits, _up(ids), _up(a), loss, dlogits=dz)
        assert e.value.status == 1
    g.sync()
    g.close()
