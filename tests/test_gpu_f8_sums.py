"""How products in 8 bits add up: in 32 bits where their results are float32, within the stated bound where they have 16."""
import pytest
import torch

from layer_util import DEV, EPS32, TINY, U, place_in, room, untouched
from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.gpu
ids = lambda t: str(t).replace("torch.", "")  # noqa: E731

# rows, n: few rows (16 and 32 of them, 16 and 32 columns), tiles of 64 x 128, 128 x 128 and, for 16-bit results, 192 x 256
SHAPES = [(3, 1032), (5, 8200), (24, 1032), (24, 8200), (300, 2056), (1500, 2056), (3080, 4104)]
DEPTHS = [16, 48, 128, 272, 400]        # the last blocks have 16, 48, 128, 16 and 16 products


def spread(scale, rows, k):
    """Scales by rows, or by 128 of them, as one for each value."""
    by = 1 if scale.shape[0] == rows else 128
    return scale.double().repeat_interleave(by, 0)[:rows].repeat_interleave(128, 1)[:, :k]


def cancelling(gen, m, n, k):
    """In every eight neighbouring products two are 448 * 448 and cancel; the others are small."""
    def small(rows):
        return torch.tensor([-2.0, -1.0, 1.0, 2.0])[torch.randint(0, 4, (rows, k), generator=gen)]
    x, w = small(m), small(n)
    first = torch.randint(0, 8, (k // 8,), generator=gen)
    at = torch.arange(0, k, 8)
    a, b = at + first, at + (first + torch.randint(1, 8, (k // 8,), generator=gen)) % 8
    sign = torch.where(torch.rand(n, k // 8, generator=gen) < 0.5, -448.0, 448.0)
    x[:, a] = x[:, b] = 448.0
    w[:, a], w[:, b] = sign, -sign
    return x, w


def scales(gen, rows, blocks):
    """Powers of two, the last block's larger than all others."""
    s = 2.0 ** torch.randint(-2, 3, (rows, blocks), generator=gen)
    s[:, -1] = 16.0
    return s


def gemm(x, xs, w, ws, w_rows, dtype, layout):
    m, n = x.shape[0], w.shape[0]
    big, y = room(m, n, dtype, layout)
    B.csr5_gemm_f8(place_in(x.to(torch.float8_e4m3fn), layout), xs.to(DEV), place_in(w.to(torch.float8_e4m3fn), layout), ws.to(DEV), y, w_rows=w_rows)
    untouched(big, m, n, layout)
    return y.double().cpu()


@pytest.mark.parametrize("k", DEPTHS)
@pytest.mark.parametrize("m,n", SHAPES)
def test_float32_results_have_sums_in_32_bits(m, n, k):
    """Products are whole numbers, any sum of some of 32 of them is below 2^20, and the blocks' scaled sums are multiples of 2^-4
    below 2^18: exact in 32 bits, in any order."""
    g = torch.Generator().manual_seed(m + n + k)
    x, w = cancelling(g, m, n, k)
    xs = scales(g, m, -(-k // 128))
    for w_rows in (128, 1):
        ws = scales(g, -(-n // w_rows), -(-k // 128))
        want = (x.double() * spread(xs, m, k)) @ (w.double() * spread(ws, n, k)).T
        for layout in ("wide", "odd") if m < 100 else ("wide",):
            assert torch.equal(gemm(x, xs, w, ws, w_rows, torch.float32, layout), want), (w_rows, layout)


def codes(gen, rows, k):
    """Any finite e4m3 values."""
    b = torch.randint(0, 254, (rows, k), generator=gen)
    return (b + (b >= 127)).to(torch.uint8).view(torch.float8_e4m3fn).float()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=ids)
@pytest.mark.parametrize("k", [16, 272])
@pytest.mark.parametrize("m,n", SHAPES)
@pytest.mark.parametrize("make", [cancelling, lambda g, m, n, k: (codes(g, m, k), codes(g, n, k))], ids=["cancelling", "any"])
def test_16_bit_results_are_within_the_stated_bound(make, m, n, k, dtype):
    g = torch.Generator().manual_seed(m + n + k + 1)
    x, w = (v[:rows] for v, rows in zip(make(g, m, n, k), (m, n)))
    blocks = -(-k // 128)
    xs, ws = scales(g, m, blocks) * 2.0 ** -12, scales(g, -(-n // 128), blocks)        # float16 holds the results
    y = gemm(x, xs, w, ws, 128, dtype, "wide")
    some = torch.randint(0, n, (256,), generator=g)
    xd, wd = x.double() * spread(xs, m, k), (w.double() * spread(ws, n, k))[some]
    xb, wb = (torch.maximum(v.abs().double(), torch.tensor(2.0 ** -6)) * s for v, s in ((x, spread(xs, m, k)), (w, spread(ws, n, k))))
    want, size, cut = xd @ wd.T, xd.abs() @ wd.abs().T, torch.zeros(m, 256, dtype=torch.float64)
    for c in range(0, k, 8):
        most = torch.zeros_like(cut)
        for i in range(c, c + 8):
            most = torch.maximum(most, xb[:, i, None] * wb[some][:, i])
        cut += most * 2.0 ** -10
    slack = (cut + (k + 8) * EPS32 * size) * (1 + 2 * U[dtype])
    off = (y[:, some] - want).abs()
    assert (off <= U[dtype] * want.abs() + slack + TINY[dtype]).all(), (off / slack).max()
