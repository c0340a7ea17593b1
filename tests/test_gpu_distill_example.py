"""A student encoder learning a teacher's answers over the pool: its gradient against the formulas, and its loss over some steps."""
import numpy as np
import pytest
import torch

from tests import gram_helpers as gh
from paper_2204_04179_b200 import binding, distill, synth

pytestmark = pytest.mark.gpu


def test_the_students_gradient():
    """The gradient of the pool's encodings in 64 bits, taken through the same backward pass: what is left between the two is the
    rounding of the logits' gradient to bf16 and of what follows from it (2^-9 an operand; 2e-2 of a tensor's largest entry is the
    bound that the step's gradients in bf16 are held to)."""
    big, small = distill.shapes(n_items=256, users=64, history=5)
    dev, scale, of_clicks, of_entropy = torch.device("cuda:0"), 0.1, 0.5, 0.2
    student = distill.Student(small, synth.item_tokens(3, 256, small.l_t, small.vocab), 4, 0.0, dev)
    rng = np.random.default_rng(0)
    hist = torch.from_numpy(rng.integers(0, 256, (64, 5)).astype(np.int32)).to(dev)
    clicks = torch.from_numpy(rng.integers(0, 256, 64).astype(np.int32)).to(dev)
    ids = torch.from_numpy(np.stack([rng.permutation(256)[:8] for _ in range(64)]).astype(np.int32)).to(dev)
    a = torch.from_numpy(rng.standard_normal((64, 8)).astype(np.float32) * 10).to(dev)
    loss, logp, entropy = student.gradient(hist, clicks, ids, a, scale, of_clicks, of_entropy)
    got = synth.unflatten(student.gram.get_grads(binding.GRAM_MODULE_CE), synth.encoder_param_spec(small))
    # 64 bits, from the rounded vectors that the products took
    H = student.H.double()
    items = student.H.to(torch.bfloat16).double()
    users = H[hist.long()].mean(1).to(torch.bfloat16).double()
    lp = torch.log_softmax(scale * users @ items.T, 1)
    p, q = lp.exp(), torch.softmax(scale * a.double(), 1)
    ent = -(p * lp).sum(1)
    want_loss = (q * (q.log() - lp.gather(1, ids.long()))).sum(1)
    at = torch.zeros_like(p).scatter_add_(1, ids.long(), q)
    click = torch.zeros_like(p).scatter_(1, clicks.long()[:, None], 1.0)
    dz = scale / 64 * (p - at - of_clicks * (click - p) + of_entropy * p * (lp + ent[:, None]))
    G = dz.T @ users
    G.index_add_(0, hist.long().flatten(), (dz @ items / 5).repeat_interleave(5, 0))
    for x, y in ((loss, want_loss), (logp, lp.gather(1, clicks.long()[:, None])[:, 0]), (entropy, ent)):
        assert float((x.double() - y).abs().max()) <= 1e-4
    student.gram.zero_grads(binding.GRAM_MODULE_CE)
    student.gram.encoder_backward(G.float().contiguous(), student.pool, 256)
    want = synth.unflatten(student.gram.get_grads(binding.GRAM_MODULE_CE), synth.encoder_param_spec(small))
    err, name = gh.worst_rel_err(got, want)
    assert err <= 2e-2, (err, name)
    student.gram.close()


def test_the_student_comes_nearer():
    first, last = distill.main(["--items", "504", "--users", "64", "--steps", "12", "--k", "16"])
    assert np.isfinite(last) and last < first
