"""An encoder that learns against the whole pool and is answered from in 8 bits: its gradient and the answers against the formulas."""
import numpy as np
import pytest
import torch

from tests import gram_helpers as gh
from paper_2204_04179_b200 import binding, distill, pool, synth

pytestmark = pytest.mark.gpu


def learner(n_items, users, history, seed):
    _, shape = distill.shapes(n_items=n_items, users=users, history=history)
    return shape, pool.Learner(shape, synth.item_tokens(seed, n_items, shape.l_t, shape.vocab), seed, 0.0, torch.device("cuda:0"))


def test_the_learners_gradient():
    """The gradient of the pool's encodings in 64 bits, taken through the same backward pass, whose operands are bf16: 2e-2 of a tensor's largest
    entry is the bound that the step's gradients in bf16 are held to; the loss is off by the roundings of 32 bits."""
    V, N, L, scale = 257, 61, 5, 0.1
    shape, e = learner(V, N, L, 4)
    rng = np.random.default_rng(0)
    hist = torch.from_numpy(rng.integers(0, V, (N, L)).astype(np.int32)).cuda()
    clicks = torch.from_numpy(np.where(rng.random(N) < 0.1, -1, rng.integers(0, V, N)).astype(np.int32)).cuda()
    loss = e.gradient(hist, clicks, scale)
    got = synth.unflatten(e.gram.get_grads(binding.GRAM_MODULE_CE), synth.encoder_param_spec(shape))
    H = e.H.double()
    items, users = e.H.to(torch.bfloat16).double(), H[hist.long()].mean(1).to(torch.bfloat16).double()
    lp = torch.log_softmax(scale * users @ items.T, 1)
    at, real = clicks.clamp(min=0).long()[:, None], (clicks >= 0)[:, None]
    assert float((loss.double() - torch.where(real, -lp.gather(1, at), 0.0)[:, 0]).abs().max()) <= 1e-4
    dz = torch.where(real, scale / N * (lp.exp() - torch.zeros_like(lp).scatter_(1, at, 1.0)), 0.0)
    G = dz.T @ users
    G.index_add_(0, hist.long().flatten(), (dz @ items / L).repeat_interleave(L, 0))
    e.gram.zero_grads(binding.GRAM_MODULE_CE)
    e.gram.encoder_backward(G.float().contiguous(), e.pool, V)
    want = synth.unflatten(e.gram.get_grads(binding.GRAM_MODULE_CE), synth.encoder_param_spec(shape))
    err, name = gh.worst_rel_err(got, want)
    assert err <= 2e-2, (err, name)
    e.gram.close()


def test_answers_from_the_table_in_8_bits():
    """A code is off by half a step of its row's scale (and the roundings of 32 bits), so a logit by at most
    sum |u| s_i / 2 + sum |w| s_u / 2 + d s_u s_i / 4 over the step sizes."""
    V, N = 1003, 37
    shape, e = learner(V, N, 5, 7)
    hist = torch.from_numpy(np.random.default_rng(1).integers(0, V, (N, 5)).astype(np.int32)).cuda()
    e.encode()
    users = e.users(hist)
    table = pool.Table(e.gram, e.H)
    z = table.logits(users)
    u, w = users.double(), e.H.double()
    su, sw = u.abs().amax(1, keepdim=True) / 127, w.abs().amax(1) / 127
    bound = u.abs().sum(1, keepdim=True) * sw / 2 + w.abs().sum(1) * su / 2 + u.shape[1] * su * sw / 4
    assert bool(((z.double() - u @ w.T).abs() <= bound * (1 + 1e-5)).all())
    clicks = torch.from_numpy(np.random.default_rng(2).integers(0, V, N).astype(np.int32)).cuda()
    logp, ids = table.answer(users, clicks, 10, 0.2)
    e.gram.sync()
    lp = torch.log_softmax(0.2 * z.double(), 1)
    assert float((logp.double() - lp.gather(1, clicks.long()[:, None])[:, 0]).abs().max()) <= 1e-4
    assert torch.equal(ids.long(), torch.sort(z, dim=1, descending=True, stable=True).indices[:, :10])
    e.gram.close()


def test_the_example_runs():
    loss, logp = pool.main(["--items", "500", "--users", "60", "--steps", "3"])
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(logp).all())
