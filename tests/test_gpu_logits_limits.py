"""Logits and scales at the ends of their types, rows of NaN, and what else a softmax goes wrong on first, in each form of the calls
on rows of logits: a warp a row, a block, and a cluster of blocks."""
import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, DT, INF, Rows, answers, check_answers, context, near, place
from tests.test_gpu_logits import _distill_reference

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
