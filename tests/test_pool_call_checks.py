"""What the binding refuses of the loss over a pool and of tables in 8 bits before the library sees it, and the sizes of workspaces (no GPU needed)."""
import pytest
import torch

from paper_2204_04179_b200 import binding
from tests.test_row_call_checks import _NoContext, _on

H = lambda *shape: _on(*shape, dtype=torch.bfloat16)   # noqa: E731
I8 = lambda *shape: _on(*shape, dtype=torch.int8)   # noqa: E731
T, LOSS, WS = _on(4, dtype=torch.int32), _on(4), _on(4096, dtype=torch.uint8)
CALLS = {
    "vectors in 32 bits": (lambda g: g.score_loss(_on(4, 8), H(9, 8), T, LOSS, WS), "users and items: bfloat16"),
    "vectors of two lengths": (lambda g: g.score_loss(H(4, 8), H(9, 16), T, LOSS, WS), "users and items: bfloat16"),
    "items on the host": (lambda g: g.score_loss(H(4, 8), torch.zeros(9, 8, dtype=torch.bfloat16), T, LOSS, WS), "items: device or pinned host memory"),
    "targets in 64 bits": (lambda g: g.score_loss(H(4, 8), H(9, 8), _on(4, dtype=torch.int64), LOSS, WS), "targets: a contiguous array of 4"),
    "targets on the host": (lambda g: g.score_loss(H(4, 8), H(9, 8), torch.zeros(4, dtype=torch.int32), LOSS, WS), "targets: device or pinned host memory"),
    "a short loss": (lambda g: g.score_loss(H(4, 8), H(9, 8), T, _on(3), WS), "loss: a contiguous array of 4"),
    "a short weight": (lambda g: g.score_loss(H(4, 8), H(9, 8), T, LOSS, WS, weight=_on(5)), "weight: a contiguous array of 4"),
    "a bias of the users": (lambda g: g.score_loss(H(4, 8), H(9, 8), T, LOSS, WS, bias=_on(4)), "bias: a contiguous array of 9"),
    "a gradient of another shape": (lambda g: g.score_loss(H(4, 8), H(9, 8), T, LOSS, WS, ditems=_on(4, 8)), "ditems: shape (9, 8)"),
    "gradients of two types": (lambda g: g.score_loss(H(4, 8), H(9, 8), T, LOSS, WS, dusers=_on(4, 8), ditems=H(9, 8)), "dusers and ditems: one type"),
    "a gradient on the host": (lambda g: g.score_loss(H(4, 8), H(9, 8), T, LOSS, WS, dusers=torch.zeros(4, 8)), "dusers: device or pinned host memory"),
    "a gradient of the bias in bf16": (lambda g: g.score_loss(H(4, 8), H(9, 8), T, LOSS, WS, dbias=H(9)), "dbias: a contiguous array of 9"),
    "a workspace of floats": (lambda g: g.score_loss(H(4, 8), H(9, 8), T, LOSS, _on(4096)), "workspace: a contiguous array of 4096"),
    "a workspace on the host": (lambda g: g.score_loss(H(4, 8), H(9, 8), T, LOSS, torch.zeros(4096, dtype=torch.uint8)), "workspace: device or pinned host memory"),
    "rows in half precision": (lambda g: g.quantize_rows(_on(4, 8, dtype=torch.float16), I8(4, 8), LOSS), "x: float32 or bfloat16"),
    "codes of another shape": (lambda g: g.quantize_rows(_on(4, 8), I8(4, 16), LOSS), "codes: shape (4, 8)"),
    "codes without a sign": (lambda g: g.quantize_rows(_on(4, 8), _on(4, 8, dtype=torch.uint8), LOSS), "codes: int8 rows"),
    "codes on the host": (lambda g: g.quantize_rows(_on(4, 8), torch.zeros(4, 8, dtype=torch.int8), LOSS), "codes: int8 rows"),
    "a scale for each column": (lambda g: g.quantize_rows(_on(4, 8), I8(4, 8), _on(8)), "scale: a contiguous array of 4"),
    "operands of two lengths": (lambda g: g.gemm_i8(I8(4, 16), LOSS, I8(9, 32), _on(9), _on(4, 9)), "A, B and C: [M, K], [N, K] and [M, N]"),
    "a result of another shape": (lambda g: g.gemm_i8(I8(4, 16), LOSS, I8(9, 16), _on(9), _on(9, 4)), "A, B and C: [M, K], [N, K] and [M, N]"),
    "a result in 8 bits": (lambda g: g.gemm_i8(I8(4, 16), LOSS, I8(9, 16), _on(9), I8(4, 9)), "C: float32 or bfloat16"),
    "an operand in bf16": (lambda g: g.gemm_i8(H(4, 16), LOSS, I8(9, 16), _on(9), _on(4, 9)), "A: int8 rows"),
    "columns apart": (lambda g: g.gemm_i8(I8(4, 16), LOSS, torch.zeros(16, 9, dtype=torch.int8).t(), _on(9), _on(4, 9)), "B: int8 rows"),
    "a vector": (lambda g: g.gemm_i8(I8(16), LOSS, I8(9, 16), _on(9), _on(1, 9)), "A: a matrix"),
    "one scale for all": (lambda g: g.gemm_i8(I8(4, 16), _on(1), I8(9, 16), _on(9), _on(4, 9)), "scale_a: a contiguous array of 4"),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_refused(name):
    call, message = CALLS[name]
    with pytest.raises(binding.GramError) as e:
        call(object.__new__(_NoContext))
    assert e.value.status == 1 and message in str(e.value), str(e.value)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V,d", [(0, 1, 1), (1, 1, 8), (1, 100_000, 768), (64, 100_000, 768), (4096, 100_000, 768), (25_600, 10_000, 768), (300, 2603, 64), (2 ** 31 - 1, 100, 8),
                                   (5, 1_857_283_072, 8)])
def test_workspaces(N, V, d, dtype):
    """The least holds one piece of 256 items (or users, where these are more) beside what every row needs; the best one of 256 MB of g."""
    least, best = binding.Gram.score_loss_workspace(N, V, d, dtype)
    n, planes = max(N, 1), (4, 6) if dtype == torch.float32 else (2, 2)
    short = min(n, V)
    fixed = 36 * n + 2 * n * d + 4 * ((short + 255) // 256 * 256) * d
    assert fixed + planes[0] * 256 * short <= least <= fixed + 6 * 256 * (short + 256) + 8 * 32 * (short + 256) + 4096
    assert least <= best <= max(2 * least, fixed * 33 + (257 << 20) * 17 // 16 + (planes[1] + 1) * 256 * (short + 256))


def test_longest_rows():
    import re
    import os
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gram.h")).read()
    assert binding.GRAM_I8_K_MAX == int(re.search(r"GRAM_I8_K_MAX = (\d+)", text).group(1)) and binding.GRAM_I8_K_MAX * 128 * 128 < 2 ** 31
