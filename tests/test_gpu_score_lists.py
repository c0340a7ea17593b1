"""Scores whose candidates are listed (more logits than are written and read again): equal ones in all row tiles."""
import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, INF, Rows, answers, check_answers, context

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
