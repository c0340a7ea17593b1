"""gram_score_loss where it can go wrong: parts of the gradients, rows that take no part, masks that leave nothing, special values, far scales,
other streams and captured calls, calls whose copies stop, and what is refused."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2204_04179_b200 import binding
from tests.logits_helpers import DEV, DT, INF, Rows, context, near
from tests.test_gpu_score_loss import Plain, codes, gradient, inputs, untouched, workspace

pytestmark = pytest.mark.gpu

PARTS = ["dusers", "ditems", "dbias"]


def outputs(N, V, d, dtype, ask):
    made = dict(dusers=lambda: gradient(N, d, 0, dtype)[1], ditems=lambda: gradient(V, d, 0, dtype)[1], dbias=lambda: torch.full((V,), float("nan"), device=DEV))
    return {k: made[k]() if k in ask else None for k in PARTS}


@pytest.mark.parametrize("ask", [[], ["dusers"], ["ditems"], ["dbias"], ["dusers", "ditems"], ["dusers", "dbias"], ["ditems", "dbias"]])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V,d", [(1, 3000, 256), (7, 20_000, 64), (60, 257, 72), (300, 1500, 64), (700, 300, 128), (1, 16_384, 8), (3, 16_385, 8),
                                   (4, 100, 1032), (2, 700_001, 8), (9, 16_384, 16), (513, 1000, 64)])
def test_each_part_alone(N, V, d, dtype, ask):
    rng = np.random.default_rng(N + V)
    users, items, u, w, b, targets, weight, more, t = inputs(rng, N, V, d, 0, bias=V % 2 == 1, none=0.1)
    scale = 0.05
    want = Plain(u, w, b, targets, weight.astype(np.float64), scale, dtype)
    g = context()
    loss, out = torch.full((N,), float("nan"), device=DEV), outputs(N, V, d, dtype, ask)
    g.score_loss(users, items, t, loss, workspace(N, V, d, dtype, "between"), scale=scale, **more, **out)
    g.sync()
    near(loss, want.loss, want.d_loss, "loss")
    for name, exact, bound in (("dusers", want.dU, want.d_dU), ("ditems", want.dI, want.d_dI), ("dbias", want.db, want.d_db)):
        if out[name] is not None:
            near(out[name], exact, bound, name)
    g.close()


def test_without_weights_and_over_one_item():
    g = context()
    rng = np.random.default_rng(1)
    for N, V in ((5, 1), (300, 1), (4, 9)):
        users, u = codes(rng, N, 16, 0)
        items, w = codes(rng, V, 16, 0)
        targets = rng.integers(0, V, N).astype(np.int32)
        want = Plain(u, w, None, targets, np.ones(N), 0.3, "f32")
        loss, out = torch.empty(N, device=DEV), outputs(N, V, 16, "f32", PARTS)
        g.score_loss(users, items, torch.from_numpy(targets).to(DEV), loss, workspace(N, V, 16, "f32", "best"), scale=0.3, **out)
        g.sync()
        near(loss, want.loss, want.d_loss, "loss")
        near(out["dusers"], want.dU, want.d_dU, "dusers")
        near(out["ditems"], want.dI, want.d_dI, "ditems")
        near(out["dbias"], want.db, want.d_db, "dbias")
    g.close()


def test_no_users():
    g = context()
    V, d = 50, 16
    users, items = torch.empty(0, d, dtype=torch.bfloat16, device=DEV), torch.randn(V, d, device=DEV).to(torch.bfloat16)
    for dtype in ("bf16", "f32"):
        (buf, di), db = gradient(V, d, 8, dtype), torch.full((V,), float("nan"), device=DEV)
        g.score_loss(users, items, torch.empty(0, dtype=torch.int32, device=DEV), torch.empty(0, device=DEV), workspace(0, V, d, dtype, "least"),
                     dusers=torch.empty(0, d, dtype=DT[dtype], device=DEV), ditems=di, dbias=db)
        g.sync()
        assert bool((di == 0).all()) and bool((db == 0).all()) and untouched(buf, V, d)
    g.close()


@pytest.mark.parametrize("N,V", [(4, 500), (40, 500), (40, 20_000), (300, 9000), (600, 9000), (1500, 400)])
def test_rows_that_take_no_part(N, V):
    """Rows of a padded batch hold NaN and infinities; targets of -1, weights of 0 and targets that the bias takes out."""
    d, rng = 64, np.random.default_rng(N)
    for dtype in ("bf16", "f32"):
        users, items, u, w, b, targets, weight, more, t = inputs(rng, N, V, d, 0, bias=True, none=0.3)
        gone = np.nonzero(np.isneginf(b))[0]
        targets[::7] = gone[0]
        t = torch.from_numpy(targets).to(DEV)
        idle = (targets < 0) | (weight == 0)
        off = torch.from_numpy(np.nonzero(idle)[0]).to(DEV)
        users[off[::3]] = float("nan")
        users[off[1::3]] = INF
        want = Plain(u, w, b, targets, weight.astype(np.float64), 0.05, dtype)
        g = context()
        loss, out = torch.empty(N, device=DEV), outputs(N, V, d, dtype, PARTS)
        g.score_loss(users, items, t, loss, workspace(N, V, d, dtype, "between"), scale=0.05, **more, **out)
        g.sync()
        none, real = torch.from_numpy(targets < 0).to(DEV), torch.from_numpy(~idle).to(DEV)
        assert bool((loss[none] == 0).all())
        near(loss[real], want.loss[~idle], want.d_loss[~idle], "loss")
        assert N == 4 or np.isposinf(want.loss[~idle]).any()
        near(out["dusers"], want.dU, want.d_dU, "dusers")
        near(out["ditems"], want.dI, want.d_dI, "ditems")
        near(out["dbias"], want.db, want.d_db, "dbias")
        nothing = torch.from_numpy(idle | np.isposinf(want.loss)).to(DEV)
        assert bool((out["dusers"][nothing] == 0).all())
        g.close()


@pytest.mark.parametrize("N,V", [(2, 300), (5, 300), (5, 40_000), (600, 2000)])
def test_nothing_left(N, V):
    """A bias that takes all items out: every target is taken out, nothing has a gradient."""
    g = context()
    users, items = torch.randn(N, 32, device=DEV).to(torch.bfloat16), torch.randn(V, 32, device=DEV).to(torch.bfloat16)
    loss, out = torch.empty(N, device=DEV), outputs(N, V, 32, "bf16", PARTS)
    t = torch.arange(N, dtype=torch.int32, device=DEV)
    t[1] = -1
    for ask in (PARTS, PARTS[:2]):
        g.score_loss(users, items, t, loss, workspace(N, V, 32, "bf16", "best"), bias=torch.full((V,), -INF, device=DEV), **{k: out[k] for k in ask})
        g.sync()
        assert bool((loss[t >= 0] == INF).all()) and float(loss[1]) == 0.0
        assert all(bool((out[k] == 0).all()) for k in ask)
    g.close()


@pytest.mark.parametrize("value", [float("nan"), INF])
@pytest.mark.parametrize("N,V", [(4, 300), (5, 300), (5, 40_000), (600, 2000)])
def test_a_row_that_holds_nan_or_infinity(N, V, value):
    g = context()
    users, items = torch.randn(N, 32, device=DEV).to(torch.bfloat16), torch.rand(V, 32, device=DEV).to(torch.bfloat16)
    users[2, 3] = value
    t = torch.arange(N, dtype=torch.int32, device=DEV)
    for ask in (PARTS, PARTS[:2]):
        loss, out = torch.empty(N, device=DEV), outputs(N, V, 32, "f32", ask)
        g.score_loss(users, items, t, loss, workspace(N, V, 32, "f32", "best"), **out)
        g.sync()
        others = torch.arange(N, device=DEV) != 2
        assert bool(loss[2].isnan()) and bool(loss[others].isfinite().all())
        assert bool(out["dusers"][2].isnan().all()) and bool(out["dusers"][others].isfinite().all())
        assert bool(out["ditems"].isnan().all()) and (out["dbias"] is None or bool(out["dbias"].isnan().all()))
    g.close()


@pytest.mark.parametrize("ask", [PARTS, PARTS[:2]])
@pytest.mark.parametrize("N,V,scale", [(4, 500, 1e-30), (4, 500, 1e30), (4, 500, 3e4), (9, 500, 1e-30), (9, 500, 1e30), (9, 500, 3e4), (600, 2000, 1e-30), (600, 2000, 1e30), (600, 2000, 3e4), (4, 30_000, 1e30),
                                       (9, 30_000, 1e30)])
def test_far_scales(N, V, scale, ask):
    """Whole numbers of a few bits, so that logits are exact and rows have either one largest entry or several equal ones."""
    rng = np.random.default_rng(V)
    u, w = rng.integers(-2, 3, (N, 16)).astype(np.float64), rng.integers(-2, 3, (V, 16)).astype(np.float64)
    users, items = (torch.from_numpy(x).to(torch.bfloat16).to(DEV) for x in (u, w))
    targets = np.argmax(u @ w.T, 1).astype(np.int32)
    weight = np.full(N, 1e-30 if scale > 1e20 else 1.0, np.float32)
    want = Plain(u, w, None, targets, weight.astype(np.float64), scale, "f32")
    g = context()
    loss, out = torch.empty(N, device=DEV), outputs(N, V, 16, "f32", ask)
    g.score_loss(users, items, torch.from_numpy(targets).to(DEV), loss, workspace(N, V, 16, "f32", "best"), scale=scale, weight=torch.from_numpy(weight).to(DEV), **out)
    g.sync()
    near(loss, want.loss, want.d_loss, "loss")
    near(out["dusers"], want.dU, want.d_dU, "dusers")
    near(out["ditems"], want.dI, want.d_dI, "ditems")
    g.close()


def test_against_differences():
    """Central differences of the loss in 64 bits, h = 1e-4: their own error is h^2 / 6 times a third derivative, here below 1e-6 of the sizes."""
    N, V, d, scale = 9, 700, 24, 0.7
    rng = np.random.default_rng(3)
    users, items = (torch.from_numpy(rng.standard_normal((n, d)) * 0.5).to(torch.bfloat16).to(DEV) for n in (N, V))
    u, w, b = users.double().cpu().numpy(), items.double().cpu().numpy(), rng.standard_normal(V).astype(np.float32).astype(np.float64)
    targets, weight = rng.integers(0, V, N).astype(np.int32), rng.random(N).astype(np.float32)

    def total(u, w, b):
        x = scale * (u @ w.T + b)
        m = x.max(1, keepdims=True)
        return (weight.astype(np.float64) * (np.log(np.exp(x - m).sum(1)) + m[:, 0] - x[np.arange(N), targets])).sum()

    g = context()
    loss, out = torch.empty(N, device=DEV), outputs(N, V, d, "f32", PARTS)
    on = lambda x: torch.from_numpy(x).to(DEV)   # noqa: E731
    g.score_loss(users, items, on(targets), loss, workspace(N, V, d, "f32", "best"), bias=on(b.astype(np.float32)), scale=scale, weight=on(weight), **out)
    g.sync()
    h = 1e-4
    for k, (grad, at) in enumerate((("dusers", (2, 5)), ("dusers", (8, 0)), ("ditems", (int(targets[0]), 3)), ("ditems", (699, 23)), ("dbias", (int(targets[1]),)), ("dbias", (5,)))):
        args = [u, w, b]
        which = PARTS.index(grad)
        values = []
        for sign in (1, -1):
            x = [a.copy() for a in args]
            x[which][at] += sign * h
            values.append(total(*x))
        want = (values[0] - values[1]) / (2 * h)
        assert abs(float(out[grad][at]) - want) <= 2e-5 * abs(want) + 1e-6, (grad, at)
    g.close()


def test_a_target_out_of_range():
    g = context()
    users, items = torch.randn(3, 16, device=DEV).to(torch.bfloat16), torch.randn(90, 16, device=DEV).to(torch.bfloat16)
    for N, ask in ((3, PARTS), (3, PARTS[:2]), (3, [])):
        for bad in (90, -2, 2 ** 31 - 1):
            loss, out = torch.empty(N, device=DEV), outputs(N, 90, 16, "f32", ask)
            g.score_loss(users, items, torch.tensor([1, bad, 2], dtype=torch.int32, device=DEV), loss, workspace(N, 90, 16, "f32", "best"), **out)
            with pytest.raises(binding.GramError, match="GRAM_ERR_ID_RANGE"):
                g.sync()
            assert float(loss[1]) == 0.0 and (out["dusers"] is None or bool((out["dusers"][1] == 0).all()))
            g.sync()
    g.close()


@pytest.mark.parametrize("N,V", [(2, 4000), (20, 4000), (600, 4000), (3000, 700)])
def test_another_stream_and_a_captured_call(N, V):
    """The same bits from another stream, and from a captured call whose inputs have changed since."""
    d = 64
    g = context()
    users, items = torch.randn(N, d, device=DEV).to(torch.bfloat16), torch.randn(V, d, device=DEV).to(torch.bfloat16)
    t, ws = torch.randint(0, V, (N,), dtype=torch.int32, device=DEV), workspace(N, V, d, "bf16", "between")

    def call(stream=None):
        loss, out = torch.zeros(N, device=DEV), outputs(N, V, d, "bf16", PARTS)
        return [loss, *out.values()], lambda: g.score_loss(users, items, t, loss, ws, scale=0.2, stream=stream, **out)

    first, run = call()
    run()
    g.sync()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    second, run = call(side)
    run()
    g.sync(side)
    assert all(torch.equal(x, y) for x, y in zip(first, second))
    third, run = call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    users.copy_(users.flip(0))
    t.copy_(t.flip(0))
    graph.replay()
    g.sync()
    assert torch.equal(first[0].flip(0), third[0]) and torch.equal(first[1].flip(0), third[1])
    users.copy_(users.flip(0))
    t.copy_(t.flip(0))
    graph.replay()
    g.sync()
    assert all(torch.equal(x, y) for x, y in zip(first, third))
    g.close()


@pytest.mark.parametrize("N,V,d", [(3, 5000, 64), (64, 30_000, 72), (700, 900, 264)])
def test_two_calls_at_once_and_the_workspaces_end(N, V, d):
    """Two contexts on two streams, each with a workspace of its own; the bytes behind a workspace stay."""
    calls = []
    for seed in (0, 1):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        users, items = torch.randn(N, d, device=DEV, generator=gen).to(torch.bfloat16), torch.randn(V, d, device=DEV, generator=gen).to(torch.bfloat16)
        t, ws = torch.randint(0, V, (N,), dtype=torch.int32, device=DEV, generator=gen), workspace(N, V, d, "f32", ("least", "best")[seed])
        g, stream = context(), torch.cuda.Stream()
        made = [(torch.zeros(N, device=DEV), outputs(N, V, d, "f32", PARTS)) for _ in range(4)]
        calls.append((g, stream, ws, made, lambda i, g=g, u=users, w=items, t=t, ws=ws, made=made, s=stream: g.score_loss(u, w, t, made[i][0], ws, stream=s, **made[i][1])))
    torch.cuda.synchronize()
    for g, stream, _, _, run in calls:
        run(0)
        g.sync(stream)
    for i in (1, 2, 3):
        for _, _, _, _, run in calls:
            run(i)
    for g, stream, ws, made, _ in calls:
        g.sync(stream)
        for loss, out in made[1:]:
            assert torch.equal(loss, made[0][0]) and all(torch.equal(out[k], made[0][1][k]) for k in PARTS)
        assert bool((ws._base[ws.numel():] == 255).all())
        g.close()


def test_more_than_2_31_entries_of_g():
    """All of g in one piece of 4.6 GB against pieces of 256 MB: entries of g are the same, sums are added in another order.  Of 16 products at a time up to
    two last places (2^-22) of the sum of the terms' sizes are cut off, so each side is off by n / 16 2^-22 times it; then both are rounded (2^-8 each).
    The sizes: over a row sum |g| <= 2 scale; over a column scale (sum p + targets there), where sum p is what db tells."""
    N, V, d = 25_600, 90_000, 16
    gen = torch.Generator(device=DEV).manual_seed(3)
    users, items = torch.randn(N, d, device=DEV, generator=gen).to(torch.bfloat16), torch.randn(V, d, device=DEV, generator=gen).to(torch.bfloat16)
    t = torch.randint(0, V, (N,), dtype=torch.int32, device=DEV, generator=gen)
    g, got = context(), []
    for room in (6 << 30, g.score_loss_workspace(N, V, d, torch.bfloat16)[1]):
        loss, out = torch.empty(N, device=DEV), outputs(N, V, d, "bf16", PARTS)
        g.score_loss(users, items, t, loss, torch.empty(room, dtype=torch.uint8, device=DEV), scale=0.3, **out)
        g.sync()
        got.append((loss, out))
    assert torch.equal(got[0][0], got[1][0])
    z = 0.3 * users[-1].double() @ items.double().T
    assert abs(float(got[0][0][-1]) - float(torch.logsumexp(z, 0) - z[t[-1].long()])) <= 1e-4
    hits = torch.bincount(t.long(), minlength=V).double()
    column = got[1][1]["dbias"].double() + 2 * 0.3 * hits
    size = dict(dusers=2 * 0.3 * items.abs().max().double() * V / 16, ditems=(column * users.abs().max().double() * N / 16)[:, None])
    for k in PARTS:
        x, y = got[0][1][k].double(), got[1][1][k].double()
        # db: no more than 800 + 8 additions of 32 bits in a row either way, roundings of 2^-24 of sum |g|
        bound = 2 * 810 * 2.0 ** -24 * column if k == "dbias" else 2 * 2.0 ** -22 * size[k] + 2.0 ** -7 * y.abs() * (1 + 2.0 ** -7)
        assert bool(((x - y).abs() <= bound).all()), (k, float(((x - y).abs() - bound).max()))
    g.close()


@pytest.mark.parametrize("tile", [0, 1])
@pytest.mark.parametrize("N,V,dtype", [(20, 30_000, "bf16"), (300, 30_000, "bf16"), (300, 30_000, "f32"), (40_000, 300, "f32")])
def test_copies_that_stop(N, V, dtype, tile):
    """The copies of every product give up at a tile: the status says so, nothing outside the results is written, and the context works on."""
    rng = np.random.default_rng(5)
    users, items, u, w, b, targets, weight, more, t = inputs(rng, N, V, 16, 0, bias=True)
    g = context()
    ws = workspace(N, V, 16, dtype, "best")

    def call():
        (bu, du), (bi, di), loss = gradient(N, 16, 8, dtype), gradient(V, 16, 8, dtype), torch.full((N + 64,), -9.0, device=DEV)
        db = torch.full((V + 64,), -9.0, device=DEV)
        g.score_loss(users, items, t, loss[:N], ws, scale=0.3, dusers=du, ditems=di, dbias=db[:V], **more)
        return bu, bi, loss, db

    g.selftest_ring_rows(tile)
    bu, bi, loss, db = call()
    with pytest.raises(binding.GramError, match="GRAM_ERR_TIMEOUT"):
        g.sync()
    assert untouched(bu, N, 16) and untouched(bi, V, 16) and bool((loss[N:] == -9).all()) and bool((db[V:] == -9).all())
    g.selftest_ring_rows(-1)
    bu, bi, loss, db = call()
    g.sync()
    want = Plain(u, w, b, targets, weight.astype(np.float64), 0.3, dtype)
    near(loss[:N], want.loss, want.d_loss, "loss")
    near(bi[:V, :16], want.dI, want.d_dI, "ditems")
    g.close()


def test_refusals():
    """What the library refuses, with its status; nothing is launched."""
    g = context()
    N, V, d = 6, 300, 24
    users, items = torch.zeros(N, d, device=DEV, dtype=torch.bfloat16), torch.zeros(V, d, device=DEV, dtype=torch.bfloat16)
    t, loss = torch.zeros(N, dtype=torch.int32, device=DEV), torch.zeros(N, device=DEV)
    du, di = torch.zeros(N, d, device=DEV), torch.zeros(V, d, device=DEV)
    least, best = g.score_loss_workspace(N, V, d, torch.float32)
    ws = torch.zeros(best + 256, dtype=torch.uint8, device=DEV)
    launches = g.launch_count()

    def refused(match, users=users, items=items, t=t, loss=loss, ws=ws[:best], **more):
        with pytest.raises(binding.GramError, match=match):
            g.score_loss(users, items, t, loss, ws, **more)

    refused("GRAM_ERR_WORKSPACE.*bytes is needed", ws=ws[:least - 256], dusers=du, ditems=di, dbias=torch.zeros(V, device=DEV))
    refused("GRAM_ERR_WORKSPACE", ws=ws[:64])
    refused("GRAM_ERR_ARG.*null workspace", ws=ws[:0])
    refused("GRAM_ERR_ARG.*256-byte", ws=ws[16:])
    for scale in (0.0, -1.0, 1e31, float("nan"), INF):
        refused("GRAM_ERR_ARG.*scale", scale=scale)
    odd = lambda n: torch.zeros(n, d + 4, device=DEV, dtype=torch.bfloat16)[:, :d]   # noqa: E731
    refused("GRAM_ERR_UNSUPPORTED.*rows a multiple of 8", users=odd(N))
    refused("GRAM_ERR_UNSUPPORTED.*rows a multiple of 8", items=odd(V))
    refused("GRAM_ERR_UNSUPPORTED.*rows a multiple of 16 bytes", ditems=odd(V))
    refused("GRAM_ERR_UNSUPPORTED.*rows a multiple of 16 bytes", dusers=torch.zeros(N, d + 1, device=DEV)[:, :d])
    flat = torch.zeros(N * d + 8, device=DEV)
    refused("GRAM_ERR_UNSUPPORTED.*16-byte aligned", dusers=flat[1:1 + N * d].view(N, d))
    narrow = [x[:, :20] for x in (users, items, du)]
    refused("GRAM_ERR_UNSUPPORTED.*multiple of 8", users=narrow[0], items=narrow[1], dusers=narrow[2])
    with pytest.raises(binding.GramError):
        g.score_loss_workspace(-1, V, d, torch.float32)
    with pytest.raises(binding.GramError):
        g.score_loss_workspace(N, 0, d, torch.float32)
    with pytest.raises(binding.GramError):
        g.score_loss_workspace(N, V, d, torch.float16)
    h = g._h
    L = binding.lib()
    p = lambda x: x.data_ptr()   # noqa: E731
    args = [h, p(users), d, p(items), d, None, N, V, d, 1.0, p(t), None, p(loss), 0, None, 0, None, 0, None, p(ws), best, 0]
    for at, bad, status in ((1, None, 1), (2, d - 8, 1), (3, None, 1), (6, -1, 1), (6, 2 ** 31, 1), (7, 0, 1), (8, 0, 1), (10, None, 1), (12, None, 1), (19, None, 1),
                            (20, -1, 1), (1, p(users) + 2, 4), (0, None, 1)):
        assert L.gram_score_loss(*[bad if i == at else x for i, x in enumerate(args)]) == status, (at, bad)
    assert L.gram_score_loss(*[{13: 7, 14: p(du), 15: d}.get(i, x) for i, x in enumerate(args)]) == 1       # an unknown type
    assert g.launch_count() == launches
    g.score_loss(narrow[0], narrow[1], t, loss, ws[:best])                                                   # the loss alone takes any width
    g.sync()
    g.close()
