"""gram_score_loss of vectors as long as nothing but memory bounds."""
import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, context, near
from tests.test_gpu_score_loss import Plain, workspace
from tests.test_gpu_score_loss_limits import PARTS, outputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V", [(1, 3), (3, 2), (5, 2)])
def test_more_columns_than_a_grid_counts(N, V, dtype):
    """65 535 blocks of 256 columns and 8 more.  Zeros but for the first and last 512 columns, whose products 32 bits hold exactly."""
    d, edge = 65_535 * 256 + 8, 512
    rng = np.random.default_rng(N + V)
    at = np.r_[0:edge, d - edge:d]
    u, w = (np.clip(np.round(rng.standard_normal((n, 2 * edge)) * 30), -127, 127) / 16 for n in (N, V))
    users, items = (torch.zeros(n, d, dtype=torch.bfloat16, device=DEV) for n in (N, V))
    for full, x in ((users, u), (items, w)):
        full[:, torch.from_numpy(at).to(DEV)] = torch.from_numpy(x).to(DEV).to(torch.bfloat16)
    targets = rng.integers(0, V, N).astype(np.int32)
    want = Plain(u, w, None, targets, np.ones(N), 0.01, dtype)
    g = context()
    loss, out = torch.empty(N, device=DEV), outputs(N, V, d, dtype, PARTS)
    g.score_loss(users, items, torch.from_numpy(targets).to(DEV), loss, workspace(N, V, d, dtype, "best"), scale=0.01, **out)
    g.sync()
    near(loss, want.loss, want.d_loss, "loss")
    near(out["dbias"], want.db, want.d_db, "dbias")
    for name, exact, bound in (("dusers", want.dU, want.d_dU), ("ditems", want.dI, want.d_dI)):
        near(out[name][:, torch.from_numpy(at).to(DEV)], exact, bound, name)
        assert bool((out[name][:, edge:d - edge] == 0).all())
    g.close()
