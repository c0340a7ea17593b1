"""Products of tables in 8 bits whose results lie in rows of a wider buffer: what is beside them and behind them stays."""
import pytest
import torch

from tests.logits_helpers import DEV, DT, context
from tests.test_gpu_i8_limits import check, operands

pytestmark = pytest.mark.gpu


# channels held in shared memory (K up to 768) and fetched with each tile; the last channels end in every place of 16 bytes, of a box and of a tile
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [64, 900])
@pytest.mark.parametrize("N", [1, 2, 3, 5, 7, 9, 31, 33, 63, 65, 66, 97, 127, 129, 191, 193, 253, 254, 255, 257, 289, 511, 999, 1000, 1001])
def test_results_beside_other_columns(N, K, dtype):
    M, more = 300, 24
    A, sa, B, sb, bias = operands(M, N, K, N)
    width = (N + more + 7) // 8 * 8
    flat = torch.full((M * width + 64,), -9.0, dtype=DT[dtype], device=DEV)
    C = flat[:M * width].view(M, width)[:, :N]
    g = context()
    g.gemm_i8(A, sa, B, sb, C, bias=bias)
    g.sync()
    check(C, A, sa, B, sb, bias)
    C.fill_(-9.0)
    assert bool((flat == -9.0).all())
    g.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [64, 900])
@pytest.mark.parametrize("M", [129, 160, 161, 257])
def test_results_at_a_buffers_end(M, K, dtype):
    """The last row ends at its last element, with another array directly behind it."""
    N, width = 77, 80
    A, sa, B, sb, bias = operands(M, N, K, M)
    flat = torch.full(((M - 1) * width + N + 40,), -9.0, dtype=DT[dtype], device=DEV)
    C = flat.as_strided((M, N), (width, 1))
    g = context()
    g.gemm_i8(A, sa, B, sb, C, bias=bias)
    g.sync()
    check(C, A, sa, B, sb, bias)
    C.fill_(-9.0)
    assert bool((flat == -9.0).all())
    g.close()
