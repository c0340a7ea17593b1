"""gram_quantize_rows and gram_gemm_i8 where they can go wrong: no rows, addresses and strides, far rows, special scales, other streams and
captured calls, copies that stop, and what is refused."""
import numpy as np
import pytest
import torch

from paper_2204_04179_b200 import binding
from tests.logits_helpers import DEV, DT, U, context, near
from tests.test_gpu_i8 import plain_codes

pytestmark = pytest.mark.gpu


def operands(M, N, K, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    room = (K + 15) // 16 * 16
    A, B = (torch.randint(-127, 128, (n, room), dtype=torch.int8, device=DEV, generator=g)[:, :K] for n in (M, N))
    return A, torch.rand(M, device=DEV, generator=g) + 0.1, B, torch.rand(N, device=DEV, generator=g) + 0.1, torch.randn(N, device=DEV, generator=g)


def check(C, A, sa, B, sb, bias):
    product = (A.double() @ B.double().T) * sa.double()[:, None] * sb.double()
    want = product + (0.0 if bias is None else bias.double())
    bound = (4 * U * product.abs() + U * want.abs()) * 1.01 + (2.0 ** -8 * want.abs() if C.dtype == torch.bfloat16 else 0.0)
    near(C, want.cpu().numpy(), bound.cpu().numpy(), "C")


def test_no_rows():
    g = context()
    g.quantize_rows(torch.empty(0, 8, device=DEV), torch.empty(0, 16, dtype=torch.int8, device=DEV)[:, :8], torch.empty(0, device=DEV))
    A, sa, B, sb, _ = operands(1, 20, 16)
    g.gemm_i8(A[:0], sa[:0], B, sb, torch.empty(0, 20, device=DEV))
    g.sync()
    g.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (0, 1), (8, 8), (4, 4), (2, 6), (3, 5)])
@pytest.mark.parametrize("M,N,K", [(5, 300, 100), (200, 300, 100), (200, 300, 900), (700, 77, 768)])
def test_any_address_and_stride_of_the_result(M, N, K, offset, pad, dtype):
    A, sa, B, sb, bias = operands(M, N, K, offset + pad)
    scales = torch.zeros(M + N + N + 3, device=DEV)                     # at odd addresses too
    for at, x in ((1, sa), (M + 2, sb), (M + N + 3, bias)):
        scales[at:at + len(x)] = x
    sa, sb, bias = scales[1:1 + M], scales[M + 2:M + 2 + N], scales[M + N + 3:]
    flat = torch.full((offset + M * (N + pad) + 64,), float("nan"), dtype=DT[dtype], device=DEV)
    C = flat[offset:].as_strided((M, N), (N + pad, 1))
    g = context()
    g.gemm_i8(A, sa, B, sb, C, bias=bias)
    g.sync()
    check(C, A, sa, B, sb, bias)
    C.fill_(float("nan"))
    assert bool(flat.isnan().all())
    g.close()


@pytest.mark.parametrize("offset", [0, 1])
def test_rows_far_apart(offset):
    """Operands and result whose last rows lie past 2^31 elements."""
    M, N, K, ld = 2100, 40, 48, 1 << 20
    A0, sa, B, sb, bias = operands(M, N, K)
    A = torch.zeros(M * ld, dtype=torch.int8, device=DEV).as_strided((M, K), (ld, 1))
    A.copy_(A0)
    C = torch.zeros(M * ld + 8, dtype=torch.bfloat16, device=DEV)[offset:].as_strided((M, N), (ld, 1))
    g = context()
    g.gemm_i8(A, sa, B, sb, C, bias=bias)
    g.sync()
    check(C, A, sa, B, sb, bias)
    C.zero_()
    g.gemm_i8(B, sb, A, sa, torch.empty(N, M, device=DEV))              # as channels
    x = torch.randn(M, K, device=DEV)
    codes, scale = A, torch.empty(M, device=DEV)
    g.quantize_rows(x, codes, scale)
    g.sync()
    want, want_scale = plain_codes(x)
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scale.cpu().numpy(), want_scale)
    g.close()


def test_rows_of_nan_and_zeros_on_their_way():
    """A row with NaN or infinity is NaN in every product, a row of zeros leaves the bias."""
    g = context()
    x = torch.randn(300, 64, device=DEV)
    x[3, 5], x[7], x[200, 0] = float("nan"), 0.0, float("inf")
    codes, scale = torch.empty(300, 64, dtype=torch.int8, device=DEV), torch.empty(300, device=DEV)
    g.quantize_rows(x, codes, scale)
    _, _, B, sb, bias = operands(1, 90, 64)
    for rows in (slice(0, 20), slice(0, 300)):
        C = torch.empty(len(codes[rows]), 90, device=DEV)
        g.gemm_i8(codes[rows], scale[rows].contiguous(), B, sb, C, bias=bias)
        g.sync()
        nan = C.isnan().all(1)
        assert nan.nonzero().flatten().tolist() == [i for i in (3, 200) if i < len(C)] and bool(C[~nan].isfinite().all())
        assert torch.equal(C[7], bias)
    g.close()


def test_the_longest_rows():
    """Codes of -128, at the length whose sum still fits 32 bits."""
    g = context()
    K = binding.GRAM_I8_K_MAX
    A, B = (torch.full((n, K + 1), -128, dtype=torch.int8, device=DEV)[:, :K] for n in (130, 3))
    one = lambda n: torch.ones(n, device=DEV)   # noqa: E731
    for M in (1, 130):
        C = torch.empty(M, 4, device=DEV)[:, :3]
        g.gemm_i8(A[:M], one(M), B, one(3), C)
        g.sync()
        assert bool((C == float(np.float32(K * 128 * 128))).all())
    g.close()


@pytest.mark.parametrize("M,N,K", [(3, 900, 64), (400, 900, 768), (400, 900, 800)])
def test_another_stream_and_a_captured_call(M, N, K):
    g = context()
    A, sa, B, sb, bias = operands(M, N, K)
    C = torch.zeros(3, M, N, device=DEV)
    g.gemm_i8(A, sa, B, sb, C[0], bias=bias)
    g.sync()
    side = torch.cuda.Stream()
    g.gemm_i8(A, sa, B, sb, C[1], bias=bias, stream=side)
    g.sync(side)
    x, scale = torch.randn(M, K, device=DEV), torch.empty(M, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.quantize_rows(x, A, scale)
        g.gemm_i8(A, scale, B, sb, C[2], bias=bias)
    assert torch.equal(C[0], C[1])
    for _ in range(2):
        x.copy_(torch.randn(M, K, device=DEV))
        graph.replay()
        g.sync()
        assert np.array_equal(A.cpu().numpy(), plain_codes(x)[0])
        check(C[2], A, scale, B, sb, bias)
    g.close()


@pytest.mark.parametrize("tile", [0, 1])
@pytest.mark.parametrize("M,N,K,pad", [(3, 100_000, 64, 0), (6000, 3000, 256, 0), (6000, 3000, 1000, 0), (6000, 3000, 64, 1)])
def test_copies_that_stop(M, N, K, pad, tile):
    g = context()
    A, sa, B, sb, bias = operands(M, N, K)
    flat = torch.full((M, N + pad + 8), -9.0, device=DEV)
    C = flat[:, :N] if not pad else flat.view(-1)[:M * (N + pad)].view(M, N + pad)[:, :N]
    g.selftest_ring_rows(tile)
    g.gemm_i8(A, sa, B, sb, C, bias=bias)
    with pytest.raises(binding.GramError, match="GRAM_ERR_TIMEOUT"):
        g.sync()
    g.selftest_ring_rows(-1)
    g.gemm_i8(A, sa, B, sb, C, bias=bias)
    g.sync()
    check(C, A, sa, B, sb, bias)
    C.fill_(-9.0)
    assert bool((flat == -9.0).all())
    g.close()


def test_refusals():
    g = context()
    A, sa, B, sb, bias = operands(4, 30, 48)
    C = torch.zeros(4, 30, device=DEV)
    x, codes, scale = torch.zeros(4, 48, device=DEV), torch.zeros(4, 48, dtype=torch.int8, device=DEV), torch.zeros(4, device=DEV)
    L, h, p = binding.lib(), g._h, lambda t: t.data_ptr()   # noqa: E731
    launches = g.launch_count()
    args = [h, p(A), 48, p(sa), p(B), 48, p(sb), None, p(C), 0, 30, 4, 30, 48, 0]
    for at, bad, status in ((0, None, 1), (1, None, 1), (2, 32, 1), (2, 56, 4), (1, p(A) + 8, 4), (3, None, 1), (4, None, 1), (4, p(B) + 1, 4), (5, 47, 1), (5, 50, 4), (6, None, 1),
                            (8, None, 1), (8, p(C) + 2, 1), (9, 5, 1), (10, 29, 1), (11, -1, 1), (11, 2 ** 31, 1), (12, 0, 1), (13, 0, 1), (13, binding.GRAM_I8_K_MAX + 1, 1)):
        assert L.gram_gemm_i8(*[bad if i == at else v for i, v in enumerate(args)]) == status, (at, bad)
    args = [h, p(x), 0, 48, 4, 48, p(codes), 48, p(scale), 0]
    for at, bad in ((0, None), (1, None), (1, p(x) + 2), (2, 9), (3, 47), (4, -1), (4, 2 ** 31), (5, 0), (6, None), (7, 47), (8, None)):
        assert L.gram_quantize_rows(*[bad if i == at else v for i, v in enumerate(args)]) == 1, (at, bad)
    assert g.launch_count() == launches
    g.close()
