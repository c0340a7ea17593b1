"""gram_score_loss refuses arrays that it would overwrite while it reads them, and takes what lies side by side in rows of one buffer."""
import numpy as np
import pytest
import torch

from paper_2204_04179_b200 import binding
from tests.logits_helpers import DEV, context, near
from tests.test_gpu_score_loss import Plain, inputs, workspace

pytestmark = pytest.mark.gpu

N, V, d = 40, 300, 64


def arrays():
    zeros = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device=DEV)   # noqa: E731
    return dict(users=zeros(N, d, dtype=torch.bfloat16), items=zeros(V, d, dtype=torch.bfloat16), targets=zeros(N, dtype=torch.int32), loss=zeros(N), workspace=workspace(N, V, d, "f32", "best"),
                bias=zeros(V), weight=zeros(N), dusers=zeros(N, d), ditems=zeros(V, d), dbias=zeros(V))


CASES = {
    "loss over weight": (lambda a: dict(loss=a["weight"]), "d_loss overlaps d_weight"),
    "loss over targets": (lambda a: dict(loss=a["targets"].view(torch.float32)), "d_loss overlaps d_targets"),
    "dbias over bias": (lambda a: dict(dbias=a["bias"]), "d_dbias overlaps d_bias"),
    "loss in dbias": (lambda a: dict(loss=a["dbias"][V - N:]), "d_loss overlaps d_dbias"),
    "dusers in ditems": (lambda a: dict(dusers=a["ditems"][7:7 + N]), "d_dusers overlaps d_ditems"),
    "dusers over users": (lambda a: dict(dusers=a["users"], ditems=a["ditems"].to(torch.bfloat16)), "d_dusers overlaps d_users"),
    "ditems over items": (lambda a: dict(ditems=a["items"], dusers=a["dusers"].to(torch.bfloat16)), "d_ditems overlaps d_items"),
    "loss in the workspace": (lambda a: dict(loss=a["workspace"][:4 * N].view(torch.float32)), "d_loss overlaps d_workspace"),
    "weight in the workspace's end": (lambda a: dict(weight=a["workspace"][-4 * N - (a["workspace"].numel() % 4):][:4 * N].view(torch.float32)), "d_workspace overlaps d_weight"),
    "rows that reach into the others'": (lambda a: (lambda b: dict(users=b[:, :d], dusers=b[:, d - 8:2 * d - 8], ditems=a["ditems"].to(torch.bfloat16)))(torch.zeros(N, 2 * d, dtype=torch.bfloat16, device=DEV)),
                                         "d_dusers overlaps d_users"),
    "dbias in a row of ditems": (lambda a: (lambda b: dict(ditems=b[:, :d], dbias=b.view(-1)[50:50 + V]))(torch.zeros(V, d + 8, device=DEV)), "d_ditems overlaps d_dbias"),
}


@pytest.mark.parametrize("name", sorted(CASES))
def test_refused(name):
    more, message = CASES[name]
    a = arrays()
    a.update(more(a))
    g = context()
    launches = g.launch_count()
    with pytest.raises(binding.GramError) as e:
        g.score_loss(**a)
    assert e.value.status == 1 and message in str(e.value)
    assert g.launch_count() == launches
    g.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_one_buffer(dtype):
    """Users beside their gradient and items beside theirs, the statistics in the gaps of neither: the same bits as from arrays of their own."""
    rng = np.random.default_rng(0)
    users, items, u, w, b, targets, weight, more, t = inputs(rng, N, V, d, 0, bias=True)
    want = Plain(u, w, b, targets, weight.astype(np.float64), 0.1, dtype)
    kind, wide = (torch.bfloat16, 1) if dtype == "bf16" else (torch.float32, 2)
    g, grads, vectors = context(), [], []
    flat = torch.full((N + V, d * (1 + wide)), float("nan"), dtype=torch.bfloat16, device=DEV)
    for rows, x in ((flat[:N], users), (flat[N:], items)):
        rows[:, :d] = x
        vectors.append(rows[:, :d])
        grads.append(rows.view(kind)[:, d // wide:] if wide == 1 else rows[:, d:].view(kind))
    loss, db = torch.empty(N, device=DEV), torch.empty(V, device=DEV)
    g.score_loss(vectors[0], vectors[1], t, loss, workspace(N, V, d, dtype, "best"), scale=0.1, dusers=grads[0], ditems=grads[1], dbias=db, **more)
    g.sync()
    near(loss, want.loss, want.d_loss, "loss")
    near(grads[0], want.dU, want.d_dU, "dusers")
    near(grads[1], want.dI, want.d_dI, "ditems")
    assert torch.equal(vectors[0], users) and torch.equal(vectors[1], items)
    g.close()
