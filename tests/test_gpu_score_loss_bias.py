"""gram_score_loss asked for the bias' gradient alone: no entry of g is kept."""
import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, context, near
from tests.test_gpu_score_loss import Plain, inputs, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,V", [(3, 4000), (100, 3000), (600, 3000), (3000, 600)])
def test_the_workspace_holds_no_entry_of_g(N, V):
    """Sums of 32 rows or more, 4 bytes each, and 36 bytes a row: far less than the two bytes for each user and item that g would take."""
    d, rng = 64, np.random.default_rng(N)
    users, items, u, w, b, targets, weight, more, t = inputs(rng, N, V, d, 0, bias=True)
    want = Plain(u, w, b, targets, weight.astype(np.float64), 0.05, "bf16")
    g, ws = context(), workspace(N, V, d, "bf16", "best")
    loss, db = torch.empty(N, device=DEV), torch.full((V,), float("nan"), device=DEV)
    g.score_loss(users, items, t, loss, ws, scale=0.05, dbias=db, **more)
    g.sync()
    near(loss, want.loss, want.d_loss, "loss")
    near(db, want.db, want.d_db, "dbias")
    assert int((ws != 255).sum()) <= (N + 31) // 32 * (V + 255) * 4 + 36 * N
    g.close()
