"""gram_score_loss of few users over tables whose logits are not kept, of gradients 16 bytes' odd multiples apart, and of vectors of any length."""
import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, DT, context, near
from tests.test_gpu_score_loss import Plain, inputs, workspace
from tests.test_gpu_score_loss_limits import PARTS, outputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", ["least", "best"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V,d", [(1, 8_500_000, 8), (3, 2_900_001, 8), (9, 1_000_003, 16), (33, 262_145, 24), (100, 90_001, 72), (128, 65_537, 64)])
def test_few_users_whose_logits_are_not_kept(N, V, d, dtype, size):
    """More than 32 MB of logits: tiles of 256 users of which few are there, copied in boxes of their number."""
    rng = np.random.default_rng(N)
    users, items, u, w, b, targets, weight, more, t = inputs(rng, N, V, d, 0, bias=N % 2 == 1, none=0.1 if N > 3 else 0.0)
    want = Plain(u, w, b, targets, weight.astype(np.float64), 0.1, dtype)
    g = context()
    got = []
    for _ in range(2):
        loss, out = torch.empty(N, device=DEV), outputs(N, V, d, dtype, PARTS)
        g.score_loss(users, items, t, loss, workspace(N, V, d, dtype, size), scale=0.1, **more, **out)
        g.sync()
        got.append((loss, *out.values()))
    near(loss, want.loss, want.d_loss, "loss")
    near(out["dusers"], want.dU, want.d_dU, "dusers")
    near(out["ditems"], want.dI, want.d_dI, "ditems")
    near(out["dbias"], want.db, want.d_db, "dbias")
    assert all(torch.equal(x, y) for x, y in zip(*got))
    g.close()


@pytest.mark.parametrize("dtype,pad,offset", [("f32", 4, 0), ("f32", 0, 4), ("f32", 12, 12), ("bf16", 8, 8), ("bf16", 0, 8)])
@pytest.mark.parametrize("N,V,d", [(1, 700, 40), (3, 700, 40), (9, 700, 264), (70, 9000, 64), (600, 2000, 64), (3000, 70, 40)])
def test_gradients_at_odd_multiples_of_16_bytes(N, V, d, dtype, pad, offset):
    """Rows and addresses that are a multiple of 16 bytes, but not of 32."""
    rng = np.random.default_rng(N + d)
    users, items, u, w, b, targets, weight, more, t = inputs(rng, N, V, d, 8, bias=True)
    want = Plain(u, w, b, targets, weight.astype(np.float64), 0.1, dtype)
    g, flats, grads = context(), [], []
    for n in (N, V):
        flat = torch.full((offset + n * (d + pad) + 64,), float("nan"), dtype=DT[dtype], device=DEV)
        flats.append(flat)
        grads.append(flat[offset:].as_strided((n, d), (d + pad, 1)))
    loss = torch.empty(N, device=DEV)
    g.score_loss(users, items, t, loss, workspace(N, V, d, dtype, "between"), scale=0.1, dusers=grads[0], ditems=grads[1], **more)
    g.sync()
    near(loss, want.loss, want.d_loss, "loss")
    near(grads[0], want.dU, want.d_dU, "dusers")
    near(grads[1], want.dI, want.d_dI, "ditems")
    for flat, x in zip(flats, grads):
        x.fill_(float("nan"))
        assert bool(flat.isnan().all())
    g.close()


@pytest.mark.parametrize("N,V,d", [(3, 500, 1), (3, 500, 20), (20, 3000, 7), (700, 3000, 13), (700, 90, 65), (100, 90_001, 3)])
def test_the_loss_and_the_bias_of_vectors_of_any_length(N, V, d):
    """Without gradients of vectors d may be any number; what lies behind a row (NaN) takes no part."""
    rng = np.random.default_rng(d)
    users, items, u, w, b, targets, weight, more, t = inputs(rng, N, V, d, -d % 8 + 8, bias=True)
    want = Plain(u, w, b, targets, weight.astype(np.float64), 0.1, "bf16")
    g = context()
    for ask in ([], ["dbias"]):
        loss, out = torch.empty(N, device=DEV), outputs(N, V, d, "bf16", ask)
        g.score_loss(users, items, t, loss, workspace(N, V, d, "bf16", "best"), scale=0.1, **more, **out)
        g.sync()
        near(loss, want.loss, want.d_loss, "loss")
        if ask:
            near(out["dbias"], want.db, want.d_db, "dbias")
    g.close()
