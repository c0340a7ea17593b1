"""Rows in 8 bits and their products, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

from tests.logits_helpers import DEV, DT, U, context, near

pytestmark = pytest.mark.gpu


def rows_of(n, d, pad, dtype, fill):
    flat = torch.full((n * (d + pad) + 64,), fill, dtype=dtype, device=DEV)
    return flat, flat[:n * (d + pad)].view(n, d + pad)[:, :d]


def plain_codes(x):
    """The definition in numpy's fp32: quotients and products are rounded as the device rounds them."""
    x = x.float().cpu().numpy()
    top = np.abs(x).max(1)
    with np.errstate(all="ignore"):
        inv = np.where(top < np.float32(1e-30), np.float32(0), np.float32(127) / top).astype(np.float32)
        scale = np.where(top < np.float32(1e-30), np.float32(0), top / np.float32(127)).astype(np.float32)
        codes = np.clip(np.rint(x * inv[:, None]), -127, 127)
    bad = ~np.isfinite(top)
    scale[bad] = np.nan
    codes[bad] = 0
    return codes.astype(np.int8), scale


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad,pad_codes", [(1, 1, 0, 0), (3, 7, 1, 9), (8, 16, 0, 0), (5, 33, 3, 15), (64, 768, 0, 0), (17, 768, 8, 16), (9, 1000, 1, 24), (2, 1024, 0, 0),
                                               (3, 1025, 7, 1), (4, 5000, 8, 8), (2, 100_003, 5, 5), (70_001, 24, 0, 8)])
def test_codes_of_rows(n, d, pad, pad_codes, dtype):
    g = torch.Generator(device=DEV).manual_seed(n + d)
    _, x = rows_of(n, d, pad, DT[dtype], float("nan"))
    x.copy_(torch.randn(n, d, device=DEV, generator=g) * torch.logspace(-32, 30, n, device=DEV)[:, None])
    flat, codes = rows_of(n, d, pad_codes, torch.int8, 99)
    scale = torch.full((n,), float("nan"), device=DEV)
    gram = context()
    gram.quantize_rows(x, codes, scale)
    gram.sync()
    want, want_scale = plain_codes(x)
    assert np.array_equal(codes.cpu().numpy(), want)
    assert np.array_equal(scale.cpu().numpy(), want_scale)
    kept = flat.clone()
    kept[:n * (d + pad_codes)].view(n, d + pad_codes)[:, :d] = 99
    assert bool((kept == 99).all())                   # nothing between the rows or behind them
    gram.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_codes_of_special_rows(dtype):
    """Zeros, the least sizes, ties, the type's largest value, infinities and NaN."""
    inf, nan, top = float("inf"), float("nan"), torch.finfo(DT[dtype]).max
    rows = [[0.0, -0.0, 0.0, 0.0], [1e-38, -1e-31, 0.0, 0.0], [2e-30, -1e-30, 0.0, 1e-38], [127.0, 0.5, 1.5, -2.5], [top, -top, 0.0, top / 2], [inf, 1.0, 0.0, 0.0],
            [-inf, inf, 0.0, 0.0], [nan, 1.0, 0.0, 0.0], [0.0, 0.0, 0.0, nan], [-1.0, 0.25, 0.0, 1e-30]]
    gram = context()
    for width in (4, 40):                             # lanes that hold one piece, and several
        x = torch.tensor(rows, device=DEV).repeat(1, width // 4).to(DT[dtype]).contiguous()
        codes, scale = torch.full((len(rows), width), 99, dtype=torch.int8, device=DEV), torch.full((len(rows),), 7.0, device=DEV)
        gram.quantize_rows(x, codes, scale)
        gram.sync()
        want, want_scale = plain_codes(x)
        assert np.array_equal(codes.cpu().numpy(), want)
        assert np.array_equal(scale.cpu().numpy(), want_scale, equal_nan=True)
    gram.close()


# M, N, K, elements between C's rows' ends and the next
PRODUCTS = [(1, 1, 1, 0), (1, 16, 16, 0), (2, 255, 100, 1), (7, 257, 128, 3), (32, 1000, 129, 0), (33, 300, 768, 5), (64, 513, 64, 0), (65, 2304, 768, 0), (128, 100, 2048, 1),
            (129, 4001, 96, 0), (256, 256, 256, 0), (257, 700, 4096, 2), (1000, 999, 777, 0), (1, 100_003, 768, 0), (3000, 20, 40, 7), (5, 64, 131_071, 0)]


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K,pad", PRODUCTS)
def test_product(M, N, K, pad, dtype, bias):
    """The sum is exact; its conversion, two products (or one and a multiply-add) are rounded: 4 u of the product's size, u of the result, and the
    result's own rounding."""
    rng = np.random.default_rng(M + N + K)
    lo = -128 if K == 131_071 else -127               # the whole range of the type, at the longest sum
    a, b = rng.integers(lo, 128, (M, K)).astype(np.int8), rng.integers(lo, 128, (N, K)).astype(np.int8)
    if K == 131_071:
        a[0], b[0] = -128, -128
    sa, sb = rng.random(M).astype(np.float32) + 0.1, (rng.random(N).astype(np.float32) + 0.1) * 0.01
    c = rng.standard_normal(N).astype(np.float32) * 10 if bias else None
    room = (K + 15) // 16 * 16 - K
    (_, A), (_, B) = rows_of(M, K, room, torch.int8, 77), rows_of(N, K, room + 16, torch.int8, 77)
    A.copy_(torch.from_numpy(a))
    B.copy_(torch.from_numpy(b))
    on = lambda x: None if x is None else torch.from_numpy(x).to(DEV)   # noqa: E731
    flat, C = rows_of(M, N, pad, DT[dtype], float("nan"))
    gram = context()
    gram.gemm_i8(A, on(sa), B, on(sb), C, bias=on(c))
    gram.sync()
    product = (A.double() @ B.double().T).cpu().numpy() * sa.astype(np.float64)[:, None] * sb.astype(np.float64)
    want = product + (c.astype(np.float64) if bias else 0.0)
    near(C, want, (4 * U * np.abs(product) + U * np.abs(want)) * 1.01 + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0.0), "C")
    C.fill_(float("nan"))
    assert bool(flat.isnan().all())                   # nothing between the rows or behind them
    gram.close()
