"""Rows of the products that are not like the others: those that no source names, those that offsets outside or out of order
make."""
import math

import pytest
import torch

from layer_util import DEV, offsets, place_in
from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.gpu

# rows, n: few rows (16 bits and 8), tiles of 64 x 128 (8 bits), 128 x 128, large
SHAPES = [(6, 40), (24, 8200), (300, 2056), (1500, 2056), (3080, 4104)]


@pytest.mark.parametrize("rows,n,layout", [(*s, "wide") for s in SHAPES] + [(*s, "odd") for s in SHAPES[:3]])         # "odd": the plain kernel
def test_rows_without_a_source_are_zeros_whatever_the_weights_hold(rows, n, layout):
    g = torch.Generator().manual_seed(rows)
    k = 144
    source = torch.arange(rows, dtype=torch.int32)
    none = torch.tensor([0, 3, rows - 1])
    source[none] = torch.tensor([-1, rows, 2 ** 31 - 1], dtype=torch.int32)
    offset = offsets([rows - 2, 2])
    w = torch.randn(2 * n, k, generator=g)
    w[5, 7], w[n - 1, 3], w[n + 2, k - 1], w[2 * n - 1] = math.inf, math.nan, -math.inf, math.inf
    x = torch.randn(rows, k, generator=g)
    y = torch.full((rows, n), 7.0, dtype=torch.bfloat16, device=DEV)
    named = torch.ones(rows, dtype=torch.bool)
    named[none] = False
    bad = torch.zeros(rows, n, dtype=torch.bool)
    bad[:-2, 5], bad[:-2, n - 1], bad[-2:, 2], bad[-2:, n - 1] = True, True, True, True
    bad[~named] = False

    def check():
        got = y.cpu()
        assert (got[~named] == 0).all()
        assert torch.equal(~torch.isfinite(got), bad)

    B.csr5_grouped_gemm(place_in(x.bfloat16(), layout), place_in(w.bfloat16(), layout).unflatten(0, (2, n)), offset, y, source=source.to(DEV))
    check()
    # 8 bits: a NaN in the values, infinite scales
    w8 = torch.randn(2 * n, k, generator=g).to(torch.float8_e4m3fn)
    code = w8.view(torch.uint8)
    code[5, 7], code[n - 1, 3], code[n + 2, k - 1], code[2 * n - 1] = 0x7f, 0xff, 0x7f, 0x7f
    ws = torch.ones(2, n, 2)
    ws[0, 5, 0], ws[1, n - 1] = math.inf, math.nan
    for dtype in (torch.bfloat16, torch.float32):
        y = torch.full((rows, n), 7.0, dtype=dtype, device=DEV)
        B.csr5_grouped_gemm_f8(place_in(x.to(torch.float8_e4m3fn), layout), torch.ones(rows, 2, device=DEV), place_in(w8, layout).unflatten(0, (2, n)),
                               ws.to(DEV), offset, y, w_rows=1, source=source.to(DEV))
        check()
