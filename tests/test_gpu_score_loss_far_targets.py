"""gram_score_loss where a target's log probability leaves 32 bits: its loss is +inf, but only a target that the bias takes out (-inf) takes no part
in the gradients."""
import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, INF, context, near
from tests.test_gpu_score_loss import Plain, workspace
from tests.test_gpu_score_loss_limits import PARTS, outputs

pytestmark = pytest.mark.gpu

LARGEST = float(np.finfo(np.float32).max)
# up to four users, few users, many users, more users than items
SIZES = [(4, 500), (9, 500), (70, 9000), (600, 2000), (3000, 70)]


def check(u, w, bias, targets, weight, scale, ask):
    N, V, d = len(u), len(w), u.shape[1]
    on = lambda x, t=torch.float32: None if x is None else torch.from_numpy(x).to(DEV).to(t)   # noqa: E731
    want = Plain(u, w, bias, targets, weight.astype(np.float64), scale, "f32")
    g = context()
    loss, out = torch.empty(N, device=DEV), outputs(N, V, d, "f32", ask)
    g.score_loss(on(u, torch.bfloat16), on(w, torch.bfloat16), on(targets, torch.int32), loss, workspace(N, V, d, "f32", "best"), bias=on(bias), scale=scale,
                 weight=on(weight), **out)
    g.sync()
    near(loss, np.where(want.loss > LARGEST, INF, want.loss), want.d_loss, "loss")
    near(out["dusers"], want.dU, want.d_dU, "dusers")
    near(out["ditems"], want.dI, want.d_dI, "ditems")
    if out["dbias"] is not None:
        near(out["dbias"], want.db, want.d_db, "dbias")
    g.close()
    return want


@pytest.mark.parametrize("ask", [PARTS, PARTS[:2]])
@pytest.mark.parametrize("N,V", SIZES)
def test_differences_that_the_scale_takes_out_of_32_bits(N, V, ask):
    """Whole numbers times a power of two, so that logits are exact, and rows that have one largest entry or several equal ones."""
    rng = np.random.default_rng(N)
    u, w = (rng.integers(-2, 3, (n, 16)).astype(np.float64) * 2.0 ** 16 for n in (N, V))
    targets = rng.integers(0, V, N).astype(np.int32)
    targets[::3] = np.argmax(u @ w.T, 1)[::3]
    want = check(u, w, None, targets, np.full(N, 1e-30, np.float32), 1e30, ask)
    assert (want.loss > LARGEST).sum() >= N // 3


@pytest.mark.parametrize("ask", [PARTS, PARTS[:2]])
@pytest.mark.parametrize("scale", [1.0, 1.25])
@pytest.mark.parametrize("N,V", SIZES)
def test_targets_masked_by_the_types_lowest_value(N, V, scale, ask):
    rng = np.random.default_rng(V)
    u, w = (rng.integers(-8, 9, (n, 16)).astype(np.float64) / 8 for n in (N, V))
    bias = np.round(rng.standard_normal(V) * 16).astype(np.float32) / 16
    bias[::3], bias[1::6] = -LARGEST, -INF
    targets = rng.integers(0, V // 3, N).astype(np.int32) * 3
    targets[::4] = 1
    targets[3::4] = 5
    with np.errstate(over="ignore"):
        check(u, w, bias, targets, rng.random(N).astype(np.float32) + 0.5, scale, ask)
