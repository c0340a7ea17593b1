"""Products of tables in 8 bits where pairs of SMs hold one tile of channels after another: whole rounds of tiles, and the rest that is cut evenly."""
import pytest
import torch

from tests.logits_helpers import DEV, DT, U, context
from tests.test_gpu_i8 import rows_of

pytestmark = pytest.mark.gpu


# tiles of 256 channels and of 256 tokens over 74 pairs: 235 and 2 (three rounds and 13 columns), 223 and 3 (three and one), 149 and 8 (two and one), 296 and 1 (four,
# nothing left), 75 and 5 (one and one)
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(300, 60_001, 40), (700, 57_000, 768), (2000, 38_100, 200), (129, 75_776, 128), (1100, 19_200, 700)])
def test_rounds_of_held_channels(M, N, K, dtype, bias):
    """Sums are exact; the conversion and three operations are rounded: 4 u of the product's size, u of the result, and the result's own rounding."""
    gen = torch.Generator(device=DEV).manual_seed(M)
    room = -K % 16
    (_, A), (_, B) = rows_of(M, K, room, torch.int8, 77), rows_of(N, K, room, torch.int8, 77)
    A.copy_(torch.randint(-127, 128, (M, K), dtype=torch.int8, device=DEV, generator=gen))
    B.copy_(torch.randint(-127, 128, (N, K), dtype=torch.int8, device=DEV, generator=gen))
    sa = torch.rand(M, device=DEV, generator=gen) + 0.1
    sb = (torch.arange(N, device=DEV) % 1021 + 1).float() * (torch.rand(N, device=DEV, generator=gen) + 0.5) * 0.01        # of each channel its own
    c = torch.randn(N, device=DEV, generator=gen) * 1000 if bias else None
    flat, C = rows_of(M, N, -N % 8, DT[dtype], float("nan"))
    g = context()
    g.gemm_i8(A, sa, B, sb, C, bias=c)
    g.sync()
    for at in range(0, N, 8192):
        cols = slice(at, min(N, at + 8192))
        product = (A.double() @ B[cols].double().T) * sa.double()[:, None] * sb[cols].double()
        want = product if c is None else product + c[cols].double()
        bound = (4 * U * product.abs() + U * want.abs()) * 1.01 + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0.0)
        assert bool(((C[:, cols].double() - want).abs() <= bound).all()), at
    C.fill_(float("nan"))
    assert bool(flat.isnan().all())                   # nothing between the rows or behind them
    g.close()
