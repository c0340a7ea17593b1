"""Codes of rows as long as a call allows, 2^31 - 1 elements: the walks over a row end with it, whose last elements are its largest."""
import pytest
import torch

from tests.logits_helpers import DEV, DT, context

pytestmark = pytest.mark.gpu

LONGEST = 2 ** 31 - 1


@pytest.mark.parametrize("cols,dtype,offset", [(LONGEST, "bf16", 0), (LONGEST, "f32", 1)])
def test_the_longest_rows_of_all(cols, dtype, offset):
    """Whole numbers in [-64, 64] and 127 at the end: codes are the values themselves.  offset 1: an address that takes single loads and stores."""
    piece = 1 << 28
    pattern = (torch.arange(piece, device=DEV, dtype=torch.int32) % 129 - 64).to(torch.int8)
    x = torch.empty(cols + offset + 64, dtype=DT[dtype], device=DEV)
    codes = torch.full((cols + offset + 64,), 99, dtype=torch.int8, device=DEV)
    row, out = x[offset:offset + cols].view(1, cols), codes[offset:offset + cols].view(1, cols)
    for at in range(0, cols, piece):
        row[0, at:at + piece] = pattern[:min(piece, cols - at)]
    row[0, -3:] = torch.tensor([-127.0, 5.0, 127.0], device=DEV)
    x[offset + cols:] = float("nan")
    scale = torch.zeros(1, device=DEV)
    g = context()
    g.quantize_rows(row, out, scale)
    g.sync()
    assert float(scale) == 1.0 and out[0, -3:].tolist() == [-127, 5, 127]
    for at in range(0, cols - 3, piece):
        n = min(piece, cols - 3 - at)
        assert torch.equal(out[0, at:at + n], pattern[:n])
    assert bool((codes[:offset] == 99).all()) and bool((codes[offset + cols:] == 99).all())
    g.close()
