"""Scores when the copies of a run give up (the kernel decides so itself at a tile): the error is reported, nothing outside the
answers is touched, and the context stays usable."""
import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, Rows, answers, check_answers, context
from paper_2204_04179_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tile", [0, 1, 3])
@pytest.mark.parametrize("N,V,k", [(20, 100_000, 5), (300, 30_522, 0), (300, 30_522, 10), (700, 12_500, 128), (300, 40_000, 50)])
def test_scores_give_up(N, V, k, tile):
    """Written logits, sums alone, and lists, joined by blocks and by warps.  What lies in the workspace when copies stop is what other
    calls left there: floating-point numbers of both signs, and keys."""
    rng = np.random.default_rng(N + k)
    d = 16
    u, w = rng.integers(-3, 4, (N, d)).astype(np.float32), rng.integers(-3, 4, (V, d)).astype(np.float32)
    users, items = (torch.from_numpy(x).to(torch.bfloat16).to(DEV) for x in (u, w))
    targets = rng.integers(0, V, (N, 2)).astype(np.int32)
    t = torch.from_numpy(targets).to(DEV)
    g = context()

    def call(scale=0.3):
        out = answers(N, 2, k)
        around = {x: None if y is None else torch.full((y.numel() + 64,), -9, dtype=y.dtype, device=DEV) for x, y in out.items()}
        out = {x: None if y is None else around[x][32:-32].view(y.shape) for x, y in out.items()}
        g.score_logprobs(users, items, scale=scale, targets=t, **out)
        return out, around

    many = torch.randn(2000, 64, device=DEV).to(torch.bfloat16)           # 32 MB of logits of either sign
    g.score_logprobs(many, torch.randn(4000, 64, device=DEV).to(torch.bfloat16), **answers(2000, 0, 1))
    g.sync()
    for scale in (0.3, 1e9):                                              # at the second one rows are summed again
        g.selftest_ring_rows(tile)
        _, around = call(scale)
        with pytest.raises(binding.GramError, match="GRAM_ERR_TIMEOUT"):
            g.sync()
        for y in around.values():
            assert y is None or ((y[:32] == -9).all() and (y[-32:] == -9).all())
        g.selftest_ring_rows(-1)
    out, _ = call()
    g.sync()
    check_answers(out, Rows((u @ w.T).astype(np.float64), 0.3), targets, k)
    g.close()
