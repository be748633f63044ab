"""Products of few rows over depths that take several turns of a workgroup's wavefronts.  Whole numbers and scales of powers of
two: every sum is exact in 32 bits, so results equal the definition's, rounded once."""
import pytest
import torch

from layer_util import DEV, offsets, place_in, room, untouched
from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]
ids = lambda t: str(t).replace("torch.", "")  # noqa: E731

# a dense product is one group; 16 rows and fewer on average, and more
GROUPS = {"3": [3], "16": [16], "24": [24], "ragged": [3, 0, 9, 1], "pairs": [20, 30]}


def whole(gen, rows, k, most):
    return torch.randint(-most, most + 1, (rows, k), generator=gen).float()


def sources(gen, rows, x_rows, by_source):
    """What each row reads, -1: zeros."""
    if not by_source:
        return torch.arange(rows), None
    s = torch.randint(0, x_rows, (rows,), generator=gen, dtype=torch.int32)
    s[rows // 2] = x_rows
    return torch.where(s < x_rows, s, -1).long(), s.to(DEV)


def expected(x, named, w, sizes, rows):
    out, at = torch.full((rows, w.shape[1]), 77.0, dtype=torch.float64), 0
    taken = x.double()[named.clamp(min=0)] * (named >= 0)[:, None]
    for g, c in enumerate(sizes):
        out[at:at + c] = taken[at:at + c] @ w[g].double().T
        at += c
    return out


@pytest.mark.parametrize("dtype", HALF, ids=ids)
@pytest.mark.parametrize("by_source", [False, True])
@pytest.mark.parametrize("k", [1016, 1024, 1032, 2048, 2056, 3080])         # a turn is 1024
@pytest.mark.parametrize("groups", GROUPS)
def test_16_bits(groups, k, by_source, dtype):
    sizes, n = GROUPS[groups], 1028
    rows = sum(sizes)
    g = torch.Generator().manual_seed(k + rows)
    x, w = whole(g, rows + 2, k, 2), whole(g, len(sizes) * n, k, 2)
    named, source = sources(g, rows, rows + 2, by_source)
    big, y = room(rows, n, dtype, "wide")
    B.csr5_grouped_gemm(place_in(x.to(dtype), "wide"), place_in(w.to(dtype), "wide").unflatten(0, (len(sizes), n)), offsets(sizes), y, source=source)
    untouched(big, rows, n, "wide")
    assert torch.equal(y.cpu(), expected(x, named, w.unflatten(0, (len(sizes), n)), sizes, rows).to(dtype))


@pytest.mark.parametrize("dtype", HALF + [torch.float32], ids=ids)
@pytest.mark.parametrize("w_rows", [128, 1])
@pytest.mark.parametrize("k", [2032, 2048, 2064, 4096, 4240, 8320])         # a turn is 2048, with 32 columns to a workgroup 4096
@pytest.mark.parametrize("n", [1028, 8200])                                 # 16 columns and 32, the last ones fewer
@pytest.mark.parametrize("m", [3, 16, 24])
def test_8_bits(m, n, k, w_rows, dtype):
    g = torch.Generator().manual_seed(m + n + k + w_rows)
    blocks = -(-k // 128)
    x, w = whole(g, m, k, 2), whole(g, n, k, 2)
    xs, ws = (2.0 ** torch.randint(-2, 3, (r, blocks), generator=g) for r in (m, -(-n // w_rows)))
    big, y = room(m, n, dtype, "wide")
    B.csr5_gemm_f8(place_in(x.to(torch.float8_e4m3fn), "wide"), xs.to(DEV), place_in(w.to(torch.float8_e4m3fn), "wide"), ws.to(DEV), y, w_rows=w_rows)
    untouched(big, m, n, "wide")
    seen = x * xs.repeat_interleave(128, 1)[:, :k], w * ws.repeat_interleave(w_rows, 0)[:n].repeat_interleave(128, 1)[:, :k]
    assert torch.equal(y.cpu(), (seen[0].double() @ seen[1].double().T).to(dtype))


@pytest.mark.parametrize("w_rows", [128, 1])
@pytest.mark.parametrize("by_source", [False, True])
@pytest.mark.parametrize("k", [2064, 4240])
@pytest.mark.parametrize("n", [1028, 4104])
@pytest.mark.parametrize("groups", ["ragged", "pairs"])
def test_8_bits_grouped(groups, n, k, by_source, w_rows):
    sizes = GROUPS[groups]
    rows, e, blocks = sum(sizes), len(sizes), -(-k // 128)
    g = torch.Generator().manual_seed(n + k + rows)
    x, w = whole(g, rows + 2, k, 2), whole(g, e * n, k, 2)
    named, source = sources(g, rows, rows + 2, by_source)
    xs, ws = 2.0 ** torch.randint(-2, 3, (rows + 2, blocks), generator=g), 2.0 ** torch.randint(-2, 3, (e, -(-n // w_rows), blocks), generator=g)
    big, y = room(rows, n, torch.bfloat16, "wide")
    B.csr5_grouped_gemm_f8(place_in(x.to(torch.float8_e4m3fn), "wide"), xs.to(DEV), place_in(w.to(torch.float8_e4m3fn), "wide").unflatten(0, (e, n)),
                           ws.to(DEV), offsets(sizes), y, w_rows=w_rows, source=source)
    untouched(big, rows, n, "wide")
    seen_x = x * xs.repeat_interleave(128, 1)[:, :k]
    seen_w = w.unflatten(0, (e, n)) * ws.repeat_interleave(w_rows, 1)[:, :n].repeat_interleave(128, 2)[:, :, :k]
    assert torch.equal(y.cpu(), expected(seen_x, named, seen_w, sizes, rows).to(torch.bfloat16))
