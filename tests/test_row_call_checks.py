"""What the binding refuses of the calls on rows of logits before the library sees it: tensors that the kernels would read past or
could not read at all (no GPU needed for these)."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2204_04179_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F, I, H = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 8, dtype=torch.bfloat16)


class OnDevice(torch.Tensor):
    """A host tensor that says it lies in device memory."""
    is_cuda = True


def _on(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


D, DI, DH = _on(4, 8), _on(4, 2, dtype=torch.int32), _on(4, 8, dtype=torch.bfloat16)
CALLS = {
    "logits on the host": (lambda g: g.logprobs(F), "logits: device or pinned host memory"),
    "logits in half precision": (lambda g: g.logprobs(F.half()), "logits: float32 or bfloat16"),
    "columns apart": (lambda g: g.logprobs(torch.zeros(8, 4).t()), "logits: the elements of a row must be contiguous"),
    "a vector of logits": (lambda g: g.logprobs(F[0]), "logits: a matrix"),
    "given tokens on the host": (lambda g: g.logprobs(D, targets=I, logp=_on(4, 2)), "targets: device or pinned host memory"),
    "a vector of given tokens": (lambda g: g.logprobs(D, targets=DI[:, 0], logp=_on(4, 1)), "targets: a matrix"),
    "given tokens in 64 bits": (lambda g: g.logprobs(D, targets=_on(4, 2, dtype=torch.int64), logp=_on(4, 2)), "targets: a contiguous array of 8"),
    "short statistics": (lambda g: g.logprobs(D, stats=_on(4, 1)), "stats: a contiguous array of 8"),
    "alternatives without IDs": (lambda g: g.logprobs(D, top_logp=_on(4, 2)), "top_logp: a contiguous array of 0"),
    "statistics in another order": (lambda g: g.logprobs_backward(D, _on(2, 4).t(), D), "stats: a contiguous array of 8"),
    "statistics on the host": (lambda g: g.logprobs_backward(D, torch.zeros(4, 2), D), "stats: device or pinned host memory"),
    "a gradient of another shape": (lambda g: g.logprobs_backward(D, _on(4, 2), _on(4, 7)), "dlogits: torch.float32 (4, 8)"),
    "a gradient of another type": (lambda g: g.logprobs_backward(D, _on(4, 2), DH), "dlogits: torch.float32 (4, 8)"),
    "a gradient on the host": (lambda g: g.logprobs_backward(D, _on(4, 2), F), "dlogits: device or pinned host memory"),
    "a teacher of another length": (lambda g: g.distill(D, DI, _on(4, 3), _on(4)), "teacher_logits: a contiguous array of 8"),
    "a teacher on the host": (lambda g: g.distill(D, I, _on(4, 2), _on(4)), "teacher_ids: device or pinned host memory"),
    "a short loss": (lambda g: g.distill(D, DI, _on(4, 2), _on(3)), "loss: a contiguous array of 4"),
    "a distillation's gradient of another shape": (lambda g: g.distill(D, DI, _on(4, 2), _on(4), dlogits=_on(5, 8)), "dlogits: torch.float32"),
    "vectors in 32 bits": (lambda g: g.score_logprobs(D, D), "users and items: bfloat16"),
    "vectors of two lengths": (lambda g: g.score_logprobs(DH, _on(9, 16, dtype=torch.bfloat16)), "users and items: bfloat16"),
    "items on the host": (lambda g: g.score_logprobs(DH, H), "items: device or pinned host memory"),
    "a short bias": (lambda g: g.score_logprobs(DH, DH, bias=_on(3)), "bias: a contiguous array of 4"),
}


def _refused(case):
    call, message = CALLS[case]
    try:
        call(object.__new__(_NoContext))
    except binding.GramError as e:
        return e.status == 1 and message in str(e), str(e)
    return False, "not refused"


class _NoContext(binding.Gram):
    _h = None

    def _ck(self, st):
        pass

    def close(self):
        pass


@pytest.mark.parametrize("case", CALLS)
def test_refused(case):
    fine, what = _refused(case)
    assert fine, what


def test_refused_without_assertions():
    """The checks are not statements that `python -O` leaves out."""
    code = "from tests import test_row_call_checks as t; bad = [c for c in t.CALLS if not t._refused(c)[0]]; print(bad); raise SystemExit(len(bad))"
    r = subprocess.run([sys.executable, "-O", "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


@pytest.mark.gpu
def test_pinned_host_memory():
    z = torch.arange(32, dtype=torch.float32).view(4, 8).pin_memory()
    stats = torch.empty(4, 2).pin_memory()
    cfg = binding.GramConfig()
    cfg.n_items, cfg.P_max, cfg.d = 1, 1, 8
    g = binding.Gram(cfg)
    g.logprobs(z, stats=stats)
    g.sync()
    assert stats[:, 0].tolist() == [7.0, 15.0, 23.0, 31.0]
    g.close()
