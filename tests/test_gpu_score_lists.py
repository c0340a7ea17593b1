"""Scores whose candidates are listed (more logits than are written and read again): equal ones in all row tiles, rows of large
logits, and products that 32 bits round."""
import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, INF, U, Rows, answers, check_answers, context, near

pytestmark = pytest.mark.gpu


def _up(x, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV).to(dtype)


# ------------------------------ equal logits ------------------------------
def _check_alike(out, z, scale, k):
    """All users have the one row z of logits."""
    check_answers({x: None if out[x] is None else out[x][-1:] for x in out}, Rows(z[None], scale), None, k)
    assert (out["top_ids"] == out["top_ids"][-1:]).all()


@pytest.mark.parametrize("start", [1280, 1281, 20_000, 99_990])
@pytest.mark.parametrize("N", [300, 512, 4096])
def test_equal_scores_from_a_place_on(N, start):
    """The best are equal and begin within the table: the first k of them, in every row tile."""
    V, d = 100_000, 8
    g = context()
    users, items = torch.zeros(N, d, dtype=torch.bfloat16, device=DEV), torch.ones(V, d, dtype=torch.bfloat16, device=DEV)
    for low, k in ((low, k) for low in (-1.0, -INF) for k in (1, 10, 34, 128)):
        z = np.where(np.arange(V) < start, low, 0.0)
        out = answers(N, 0, k)
        g.score_logprobs(users, items, bias=_up(z), scale=0.5, **out)
        g.sync()
        _check_alike(out, z, 0.5, k)
    g.close()


@pytest.mark.parametrize("N", [300, 4096])
@pytest.mark.parametrize("plateau", [1, 700, 3000, 40_000])
@pytest.mark.parametrize("order", [1, -1])
def test_plateaus_of_scores(order, plateau, N):
    """Scores that rise or fall over the table in steps, longer than a list or a run, or of single items."""
    V, d = 100_000, 8
    z = order * (np.arange(V) // plateau) / 64.0
    g = context()
    users, items = torch.zeros(N, d, dtype=torch.bfloat16, device=DEV), torch.ones(V, d, dtype=torch.bfloat16, device=DEV)
    for k in (1, 10, 34, 128):
        out = answers(N, 0, k)
        g.score_logprobs(users, items, bias=_up(z), scale=0.5, **out)
        g.sync()
        _check_alike(out, z, 0.5, k)
    g.close()


@pytest.mark.parametrize("k", [1, 10, 34, 128])
@pytest.mark.parametrize("N,V", [(300, 30_522), (512, 100_000), (700, 12_500), (3000, 20_011)])
def test_whole_number_scores(N, V, k):
    """A few dozen values over the whole table, different for each user: the order by value and place, exactly."""
    d = 8
    rng = np.random.default_rng(N + k)
    users, items = _up(rng.integers(-1, 2, (N, d)).astype(np.float32)), _up(rng.integers(-1, 2, (V, d)).astype(np.float32))
    g = context()
    out = answers(N, 0, k)
    g.score_logprobs(users.to(torch.bfloat16), items.to(torch.bfloat16), scale=0.5, **out)
    g.sync()
    place = torch.arange(V, device=DEV)
    for n in range(0, N, 500):
        key = ((users[n:n + 500].double() @ items.double().T).long() << 32) - place
        assert torch.equal(out["top_ids"][n:n + 500].long(), (-key.topk(k, dim=1).values) & 0xFFFFFFFF), n
    g.close()


# ------------------------------ rows of large logits ------------------------------
@pytest.mark.parametrize("size,common", [(1e7, False), (1e10, False), (1e18, False), (1e7, True), (1e10, True)])
@pytest.mark.parametrize("k", [0, 10, 128])
@pytest.mark.parametrize("N,V,d", [(300, 30_522, 768), (700, 12_500, 72)])
def test_scores_of_large_vectors(N, V, d, k, size, common):
    """Logits so large that 32 bits hold no fraction of theirs, and of which 128 items are offered: the answers belong to one set of
    logits.  The best item's log probability is then -log s to the bit, the 128 probabilities add up to 1, and the entropy is theirs.
    Bounds: a log probability is off by 2^-22 + (V / 128 + 64) u < 2e-5 and 4 u of its difference to the best; with
    sum p |y| <= 128 / e < 48 the sum of the probabilities by less than 1e-4 and the entropy by less than 2e-3."""
    rng = np.random.default_rng(N + k)
    step = 1.0 if common else np.sqrt(size / np.sqrt(d))
    users = _up(rng.standard_normal((N, d)) * step, torch.bfloat16)
    items = _up(rng.standard_normal((V, d)) * step, torch.bfloat16)
    if common:                                           # the size is all items' alike, their differences those of the other columns
        users[:, 0] = items[:, 0] = float(np.sqrt(size))
    offered = np.sort(rng.permutation(V)[:128]).astype(np.int32)
    bias = np.full(V, -INF)
    bias[offered] = 0.0
    targets = np.tile(offered, (N, 1))
    g = context()
    for scale in (1.0, 4.0 / size, 1e8 / size):
        out = answers(N, 128, k)
        g.score_logprobs(users, items, bias=_up(bias), scale=scale, targets=_up(targets, torch.int32), **out)
        g.sync()
        logp, log_s, entropy = out["logp"].double().cpu().numpy(), out["stats"][:, 1].double().cpu().numpy(), out["entropy"].double().cpu().numpy()
        assert np.isfinite(log_s).all() and (log_s >= 0).all() and (log_s <= np.log(128) + 1e-4).all()
        if scale * size >= 1e7:                          # others have sums of the products' own order
            assert np.array_equal(logp.max(1), -log_s)
            p = np.exp(logp)
            assert (np.abs(p.sum(1) - 1) <= 1e-4).all()
            assert (np.abs(-np.where(p > 0, p * logp, 0.0).sum(1) - entropy) <= 2e-3).all()
        u, w = users.double().cpu().numpy(), items[torch.from_numpy(offered).to(DEV).long()].double().cpu().numpy()
        dz = 2 * d * U * (np.abs(u) @ np.abs(w).T).max()
        z = u @ w.T
        near(out["stats"][:, 0], z.max(1), dz, "m")
        if k:
            ids, top = out["top_ids"].cpu().numpy(), out["top_logp"].double().cpu().numpy()
            where = np.searchsorted(offered, ids)
            assert np.array_equal(offered[where], ids) and all(len(set(row)) == k for row in ids)
            best = -np.sort(-z, 1)[:, :k]
            assert (np.abs(np.take_along_axis(z, where, 1) - best) <= 2 * dz).all()
            if scale * size >= 1e7:
                assert np.array_equal(top, np.take_along_axis(logp, where, 1))
    g.close()


# ------------------------------ products that 32 bits round ------------------------------
@pytest.mark.parametrize("k", [0, 1, 10, 50, 128])
@pytest.mark.parametrize("N,V,d", [(300, 30_522, 768), (300, 30_522, 64), (257, 40_000, 100), (1000, 10_007, 1000), (1600, 5500, 328), (64, 140_001, 768)])
def test_listed_scores_of_any_vectors(N, V, d, k):
    """A sum of d products of bf16 values in 32 bits is off by at most d u times the sum of their sizes, however it is ordered.  The bar that
    the sample of the table gives is reached by k entries of the main pass as well, whatever the width of their tiles."""
    rng = np.random.default_rng(d + k)
    pad = -d % 8
    users = torch.nn.functional.pad(_up(rng.standard_normal((N, d)), torch.bfloat16), (0, pad), value=float("nan"))[:, :d]
    items = torch.nn.functional.pad(_up(rng.standard_normal((V, d)) * 0.2, torch.bfloat16), (0, pad), value=float("nan"))[:, :d]
    targets = rng.integers(0, V, (N, 2)).astype(np.int32)
    scale = float(2.0 / np.sqrt(d))
    g = context()
    out = answers(N, 2, k)
    g.score_logprobs(users, items, scale=scale, targets=_up(targets, torch.int32), **out)
    g.sync()
    u, w = users.double(), items.double()
    dz = 2 * d * U * float((u.abs() @ w.abs().T).max())
    r = Rows((u @ w.T).cpu().numpy(), scale)
    check_answers(out, r, targets, 0, dz)
    if k:
        ids = out["top_ids"].cpu().numpy().astype(np.int64)
        assert (ids >= 0).all() and all(len(set(row)) == k for row in ids)
        best = -np.sort(-r.z, 1)[:, :k]
        assert (np.abs(np.take_along_axis(r.z, ids, 1) - best) <= 2 * dz).all()
        top = out["top_logp"].double().cpu().numpy()
        assert (top[:, 1:] <= top[:, :-1]).all()
        near(top, np.take_along_axis(r.logp, ids, 1), np.take_along_axis(r.d_logp, ids, 1) + 4 * r.scale * dz, "log p of alternatives")
    g.close()


@pytest.mark.parametrize("d", [72, 768, 1000])
def test_a_product_is_the_same_in_every_pass_and_tile(d):
    """What the bars rest on: the sum of a user and an item does not depend on the item's place in the table, on the width of its tile, on
    the other users, nor on whether logits are written, listed or only summed.  The largest logit of a row shows it to the bit."""
    N, V = 300, 30_522
    rng = np.random.default_rng(d)
    users, items = _up(rng.standard_normal((N, d)), torch.bfloat16), _up(rng.standard_normal((V, d)), torch.bfloat16)
    g = context()
    want = None
    for shift in (0, 1, 128, 4000, 20_011):
        table = items.roll(shift, 0)
        for k in (0, 1, 10, 40, 128):
            for rows in (slice(0, N), slice(40, N), slice(0, 20), slice(250, 270)):
                out = answers(len(range(*rows.indices(N))), 0, k)
                g.score_logprobs(users[rows], table, scale=0.1, **out)
                g.sync()
                want = out["stats"][:, 0] if want is None else want
                assert torch.equal(out["stats"][:, 0], want[rows]), (shift, k, rows)
    g.close()
