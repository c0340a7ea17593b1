"""Answers over an item table from the vectors themselves, against plain forms in 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, INF, U, Rows, answers, check_answers, context
from paper_2204_04179_b200 import binding

pytestmark = pytest.mark.gpu

# N, V, d, elements between the rows' ends and the next (users, items)
SIZES = [(1, 1, 8, 0, 0), (2, 3, 8, 8, 0), (1, 255, 16, 0, 16), (3, 256, 64, 0, 0), (64, 257, 72, 0, 8), (127, 1000, 100, 4, 28),
         (128, 300, 768, 0, 0), (129, 513, 64, 8, 0), (5, 10_007, 768, 0, 0), (300, 2603, 256, 0, 0), (1, 40_000, 128, 0, 0),
         (257, 5000, 1000, 24, 24), (700, 777, 64, 0, 0), (40, 30_522, 64, 0, 0), (20_000, 70, 32, 0, 0), (2, 200_003, 8, 0, 0)]
# more logits than are written and read again: candidates are listed
LISTED = [(300, 30_522, 64, 0, 0), (257, 40_000, 128, 24, 24), (1000, 10_007, 72, 0, 8), (90, 100_003, 8, 8, 0), (1600, 5500, 32, 0, 0)]


def _codes(rng, rows, d, pad):
    """8-bit codes over a step of 1/16 in bf16: every sum of their products is exact in 32 bits up to d = 1040."""
    x = np.clip(np.round(rng.standard_normal((rows, d)) * 30), -127, 127) / 16
    buf = torch.full((rows, d + pad), float("nan"), dtype=torch.bfloat16, device=DEV)
    buf[:, :d] = torch.from_numpy(x).to(torch.bfloat16)
    return buf[:, :d], x


@pytest.mark.parametrize("k", [0, 1, 10, 128])
@pytest.mark.parametrize("N,V,d,pad_u,pad_i", SIZES + LISTED)
def test_score_of_codes(N, V, d, pad_u, pad_i, k):
    rng = np.random.default_rng(N + V + k)
    users, u = _codes(rng, N, d, pad_u)
    items, w = _codes(rng, V, d, pad_i)
    bias = np.round(rng.standard_normal(V) * 20 * 256) / 256 if k != 1 else None
    if bias is not None:
        bias[rng.random(V) < 0.03] = -INF
    z = u @ w.T + (bias if bias is not None else 0.0)
    nc = {0: 1, 1: 0, 10: 5, 128: 128}[k]
    targets = np.where(rng.random((N, nc)) < 0.2, -1, rng.integers(0, V, (N, nc))).astype(np.int32) if nc else None
    scale = 0.05 if d > 32 else 0.3
    g = context()
    t = torch.from_numpy(targets).to(DEV) if nc else None
    b = torch.from_numpy(bias).float().to(DEV) if bias is not None else None
    out, again = answers(N, nc, k), answers(N, nc, k)
    for o in (out, again):
        g.score_logprobs(users, items, bias=b, scale=scale, targets=t, **o)
        g.sync()
    check_answers(out, Rows(z, scale), targets, k)
    assert all(out[x] is None or torch.equal(out[x], again[x]) for x in out)
    g.close()


@pytest.mark.parametrize("N,V,d", [(1, 3000, 768), (130, 1111, 200), (64, 20_000, 768)])
def test_score_of_any_vectors(N, V, d):
    """A sum of d products of bf16 values in 32 bits is off by at most d u times the sum of their sizes, however it is ordered."""
    rng = np.random.default_rng(d)
    users = torch.from_numpy(rng.standard_normal((N, d))).to(torch.bfloat16).to(DEV)
    items = torch.from_numpy(rng.standard_normal((V, d)) * 0.2).to(torch.bfloat16).to(DEV)
    u, w = users.double().cpu().numpy(), items.double().cpu().numpy()
    targets = rng.integers(0, V, (N, 2)).astype(np.int32)
    g = context()
    out = answers(N, 2, 3)
    g.score_logprobs(users, items, scale=0.7, targets=torch.from_numpy(targets).to(DEV), **out)
    g.sync()
    dz = 2 * d * U * (np.abs(u) @ np.abs(w).T).max()
    r = Rows(u @ w.T, 0.7)
    check_answers(out, r, targets, 0, dz)
    z = r.z
    ids = out["top_ids"].cpu().numpy()
    best = -np.sort(-z, 1)[:, :3]
    assert (np.abs(np.take_along_axis(z, ids.astype(np.int64), 1) - best) <= 2 * dz).all()
    g.close()


@pytest.mark.parametrize("N,V", [(1, 3000), (70, 3000), (200, 3000), (300, 30_000)])
def test_score_with_ties_and_nothing_left(N, V):
    d = 64
    rng = np.random.default_rng(N)
    users, u = _codes(rng, N, d, 0)
    items, w = _codes(rng, 5, d, 0)
    items = items.repeat(V // 5, 1)                       # every item a fifth of V times
    w = np.tile(w, (V // 5, 1))
    g = context()
    for k in (1, 30, 128):
        out = answers(N, 0, k)
        g.score_logprobs(users, items, scale=0.1, **out)
        check_answers(out, Rows(u @ w.T, 0.1), None, k)
        out = answers(N, 1, k)
        t = torch.zeros(N, 1, dtype=torch.int32, device=DEV)
        g.score_logprobs(users, items, bias=torch.full((V,), -INF, device=DEV), targets=t, **out)
        check_answers(out, Rows(np.full((N, V), -INF), 1.0), np.zeros((N, 1), np.int32), k)
        one = torch.full((V,), -INF, device=DEV)
        one[V - 7] = 0.0
        g.score_logprobs(users, items, bias=one, targets=t, **out)
        z = u @ w.T + one.double().cpu().numpy()
        check_answers(out, Rows(z, 1.0), np.zeros((N, 1), np.int32), k)
        zero = torch.zeros_like(users)                    # all logits equal
        g.score_logprobs(zero, items, targets=t, **out)
        check_answers(out, Rows(np.zeros((N, V)), 1.0), np.zeros((N, 1), np.int32), k)
    g.sync()
    g.close()


@pytest.mark.parametrize("N,V,k", [(128, 3000, 64), (128, 3000, 65), (63, 3000, 128), (65, 3000, 128), (129, 3000, 64), (1, 8_500_000, 10), (1, 8_300_000, 10),
                                   (64, 32_768, 0), (64, 32_769, 0), (65, 32_768, 0),
                                   (2560, 3000, 10), (2561, 3000, 10), (5000, 3000, 1), (1792, 4100, 10), (1793, 4100, 10), (900, 10_000, 64), (900, 10_000, 65),
                                   (1000, 2000, 0), (1100, 2000, 0)])
def test_score_where_the_way_changes(N, V, k):
    """Few logits are written and read again, in turns where the table is small; else candidates are listed."""
    d = 8
    rng = np.random.default_rng(N + k)
    users, u = _codes(rng, N, d, 0)
    items, w = _codes(rng, V, d, 0)
    targets = np.where(rng.random((N, 2)) < 0.2, -1, rng.integers(0, V, (N, 2))).astype(np.int32)
    g = context()
    out = answers(N, 2, k)
    g.score_logprobs(users, items, scale=0.3, targets=torch.from_numpy(targets).to(DEV), **out)
    g.sync()
    check_answers(out, Rows(u @ w.T, 0.3), targets, k)
    g.close()


@pytest.mark.parametrize("N,V", [(3, 500), (200, 500), (200, 50_000)])
def test_items_out_of_range_are_recorded_and_count_as_none(N, V):
    rng = np.random.default_rng(N)
    users, u = _codes(rng, N, 64, 0)
    items, w = _codes(rng, V, 64, 0)
    t = np.zeros((N, 1), np.int32)
    t[1], t[2] = V, -2
    g = context()
    for k in (0, 3):
        out = answers(N, 1, k)
        g.score_logprobs(users, items, scale=0.05, targets=torch.from_numpy(t).to(DEV), **out)
        with pytest.raises(binding.GramError) as e:
            g.sync()
        assert e.value.status == 2
        check_answers(out, Rows(u @ w.T, 0.05), np.where((t < 0) | (t >= V), -1, t), k)
    g.sync()
    g.close()


def test_score_on_another_stream_behind_its_work():
    rng = np.random.default_rng(7)
    for N in (20, 300, 2000):
        users, u = _codes(rng, N, 64, 0)
        items, w = _codes(rng, 5000, 64, 0)
        late = torch.zeros_like(users)
        g = context()
        out = answers(N, 0, 3)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            a = torch.randn(4096, 4096, device=DEV)
            for _ in range(20):
                a = a @ a * 1e-3
            late.copy_(users)
            g.score_logprobs(late, items, scale=0.05, **out)
            late.zero_()
        g.sync(s)
        check_answers(out, Rows(u @ w.T, 0.05), None, 3)
        g.close()


@pytest.mark.parametrize("order", [1, -1])
def test_score_of_a_sorted_table(order):
    """Items in ascending and descending order of their score: every one, or none, is better than those before it."""
    V, d = 50_000, 8
    x = np.zeros((V, d))
    x[:, 0], x[:, 1] = np.arange(V) // 250, np.arange(V) % 250 / 256     # both exact in bf16
    x = x[::order]
    items = torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).to(DEV)
    for N in (1, 140, 200):
        users = torch.zeros(N, d, dtype=torch.bfloat16, device=DEV)
        users[:, :2] = 1.0
        g = context()
        out = answers(N, 0, 100)
        g.score_logprobs(users, items, scale=0.5, **out)
        g.sync()
        check_answers(out, Rows(np.tile(x.sum(1), (N, 1)), 0.5), None, 100)
        g.close()


@pytest.mark.parametrize("N,V", [(140, 900), (300, 30_522)])
def test_nan_in_a_vector_stays_with_its_rows(N, V):
    d = 64
    rng = np.random.default_rng(1)
    users, u = _codes(rng, N, d, 0)
    items, w = _codes(rng, V, d, 0)
    users[3, 5] = float("nan")
    g = context()
    out = answers(N, 0, 4)
    g.score_logprobs(users, items, scale=0.05, **out)
    g.sync()
    assert torch.isnan(out["entropy"][3]) and torch.isnan(out["stats"][3, 1])
    keep = [n for n in range(N) if n != 3]
    check_answers({x: None if out[x] is None else out[x][keep] for x in out}, Rows(u[keep] @ w.T, 0.05), None, 4)
    g.close()


def test_refusals():
    g = context()
    u = torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV)
    w = torch.zeros(50, 64, dtype=torch.bfloat16, device=DEV)
    st = torch.zeros(4, 2, device=DEV)
    i = torch.zeros(4, 200, dtype=torch.int32, device=DEV)
    L, P = binding.lib(), lambda t: C.c_void_p(0 if t is None else t.data_ptr())  # noqa: E731

    def call(pu=P(u), ldu=64, pi=P(w), ldi=64, N=4, V=50, d=64, scale=1.0, nc=0, t=None, k=0, ti=None):
        return L.gram_score_logprobs(g._h, pu, C.c_int64(ldu), pi, C.c_int64(ldi), P(None), C.c_int64(N), C.c_int32(V), C.c_int32(d), C.c_float(scale),
                                     P(t), C.c_int32(nc), P(None), P(st), P(None), P(None), P(ti), C.c_int32(k), C.c_void_p(0))
    for bad in (dict(pu=P(None)), dict(pi=P(None)), dict(d=0), dict(ldu=56), dict(ldi=63), dict(V=0), dict(N=-1), dict(scale=0.0),
                dict(nc=1, t=i), dict(k=1, ti=i), dict(k=129), dict(nc=129)):
        assert call(**bad) == 1, bad
    for bad in (dict(ldu=65), dict(ldi=68), dict(pu=C.c_void_p(u.data_ptr() + 2)), dict(pi=C.c_void_p(w.data_ptr() + 8))):
        assert call(**bad) == 4, bad
    assert call(N=0, pu=P(None)) == 0 and call() == 0
    g.sync()
    assert abs(float(st[0, 1]) - np.log(50)) < 1e-6
    g.close()
