"""Sizes past what the calls over a pool count with are refused, not wrapped around."""
import pytest
import torch

from paper_2204_04179_b200 import binding
from tests.logits_helpers import DEV, context

LONGEST = 2 ** 31 - 256


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V,d", [(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 256), (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 30), (2 ** 31 - 1, 5, 2 ** 19 + 8), (5, 2 ** 31 - 1, 2 ** 19 + 8),
                                   (4, 4, 2 ** 31 - 255), (1, 1, 2 ** 31 - 1)])
def test_workspaces_of_petabytes_are_refused(N, V, d, dtype):
    with pytest.raises(binding.GramError) as e:
        binding.Gram.score_loss_workspace(N, V, d, dtype)
    assert e.value.status == 4


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V,d", [(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 19), (3, 2 ** 19, 2 ** 31 - 256), (2 ** 31 - 1, 7, 2 ** 19)])
def test_the_largest_workspaces(N, V, d, dtype):
    """Users and items of 2^50 elements still have sizes that 64 bits hold: what each row needs, and a part of the summed gradient, at least."""
    least, best = binding.Gram.score_loss_workspace(N, V, d, dtype)
    assert 4 * min(N, V) * d + 2 * N * d < least <= best < 2 ** 62


@pytest.mark.gpu
@pytest.mark.parametrize("d", [LONGEST + 1, 2 ** 31 - 1])
def test_vectors_too_long_to_count(d):
    """Refused before anything is launched or read (the buffers are far smaller than these sizes)."""
    g = context()
    L, h = binding.lib(), g._h
    x = torch.zeros(1024, dtype=torch.bfloat16, device=DEV)
    t, f = torch.zeros(8, dtype=torch.int32, device=DEV), torch.zeros(64, device=DEV)
    ws = torch.zeros(4096, dtype=torch.uint8, device=DEV)
    p = lambda a: a.data_ptr()   # noqa: E731
    launches = g.launch_count()
    assert L.gram_score_loss(h, p(x), d, p(x), d, None, 1, 1, d, 1.0, p(t), None, p(f), 0, None, 0, None, 0, None, p(ws), 4096, 0) == 4
    assert L.gram_score_logprobs(h, p(x), d, p(x), d, None, 1, 1, d, 1.0, p(t), 1, p(f), None, None, None, None, 0, 0) == 4
    assert g.launch_count() == launches
    g.close()


def _far(rows, cols, dtype):
    from tests.test_row_call_checks import OnDevice
    return torch.empty(rows, cols, dtype=dtype, device="meta").as_subclass(OnDevice)


PAST = 2 ** 32 + 16                                       # 16 in 32 bits
B, F, I8 = torch.bfloat16, torch.float32, torch.int8
CALLS = {
    "items": lambda g: g.score_loss(_far(4, 8, B), _far(PAST, 8, B), None, None, None),
    "users": lambda g: g.score_logprobs(_far(PAST, 8, B), _far(9, 8, B)),
    "longer vectors": lambda g: g.score_loss(_far(4, PAST, B), _far(9, PAST, B), None, None, None),
    "rows": lambda g: g.quantize_rows(_far(4, PAST, F), _far(4, PAST, I8), None),
    "codes' channels": lambda g: g.gemm_i8(_far(4, 16, I8), None, _far(PAST, 16, I8), None, _far(4, PAST, F)),
    "codes of longer rows": lambda g: g.gemm_i8(_far(4, PAST, I8), None, _far(9, PAST, I8), None, _far(4, 9, F)),
    "logits": lambda g: g.logprobs(_far(4, PAST, F)),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_sizes_that_leave_32_bits_are_refused(name):
    """The library takes these sizes in 32 bits, where they would be other, smaller ones."""
    from tests.test_row_call_checks import _NoContext
    with pytest.raises(binding.GramError) as e:
        CALLS[name](object.__new__(_NoContext))
    assert e.value.status == 1 and "2^31 - 1" in str(e.value)


@pytest.mark.parametrize("N,V,d", [(4, PAST, 8), (4, 9, PAST), (PAST, 9, 8)])
def test_workspaces_of_sizes_that_leave_32_bits_are_refused(N, V, d):
    with pytest.raises(binding.GramError) as e:
        binding.Gram.score_loss_workspace(N, V, d, B)
    assert e.value.status == 1
