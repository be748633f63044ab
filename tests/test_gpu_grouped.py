"""Products grouped by expert and products in 8 bits against their definitions in 64 bits."""
import math

import pytest
import torch

from layer_util import DEV, EPS32, close, matrix, meaning, offsets, place_in, quantised, room, untouched
from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]
ids = lambda t: str(t).replace("torch.", "")  # noqa: E731

GROUPS = {
    "one": [1],
    "singles": [1, 0, 1, 1, 0],
    "edges": [127, 128, 129, 0, 15, 16, 17],
    "large": [255, 1, 257, 0, 64],
    "lopsided": [0, 0, 700, 3, 0],
    "none": [0, 0, 0],
}
SHAPES = [(1, 1, "plain"), (17, 33, "odd"), (128, 64, "plain"), (136, 200, "wide"), (264, 328, "plain"), (300, 129, "odd"), (512, 640, "plain")]


def experts(gen, groups, n, k, dtype, layout, scale=1.0):
    """Weights [groups, n, k], a view whose surroundings are NaN unless "plain"."""
    if layout == "plain":
        return (torch.randn(groups, n, k, generator=gen) * scale).to(dtype).to(DEV)
    flat = matrix(gen, groups * n, k, dtype, layout, scale)
    return flat.unflatten(0, (groups, n))


def source_for(gen, rows, x_rows, bad=True):
    s = torch.randint(0, x_rows, (rows,), generator=gen, dtype=torch.int32)
    if bad and rows > 4:
        s[1], s[3] = -1, x_rows             # rows of zeros
    return s


def taken(x, source, rows):
    """The rows of x that the products see, in 64 bits."""
    x = x.double().cpu()
    if source is None:
        return x[:rows]
    s = source.long()
    there = (s >= 0) & (s < x.shape[0])
    return x[torch.where(there, s, 0)] * there[:, None]


def spans(sizes):
    at = 0
    for g, c in enumerate(sizes):
        yield g, at, at + c
        at += c


@pytest.mark.parametrize("dtype", HALF, ids=ids)
@pytest.mark.parametrize("groups", GROUPS)
@pytest.mark.parametrize("n,k,layout", SHAPES)
def test_grouped(dtype, groups, n, k, layout):
    sizes = GROUPS[groups]
    g = torch.Generator().manual_seed(n * k)
    rows, tail = sum(sizes), 3                              # rows in no group stay as they are
    offset = offsets(sizes)
    w = experts(g, len(sizes), n, k, dtype, layout)
    wc = w.double().cpu()
    x = matrix(g, rows + tail, k, dtype, layout)
    source = source_for(g, rows + tail, rows + tail)
    for s in (None, source):
        big, y = room(rows + tail, n, dtype, layout)
        B.csr5_grouped_gemm(x, w, offset, y, source=None if s is None else s.to(DEV))
        untouched(big, rows + tail, n, layout)
        xc = taken(x, s, rows + tail)
        ref, size = torch.full((rows + tail, n), 77.0, dtype=torch.float64).to(dtype).double(), torch.zeros(rows + tail, n, dtype=torch.float64)
        for i, a, b in spans(sizes):
            ref[a:b], size[a:b] = xc[a:b] @ wc[i].T, xc[a:b].abs() @ wc[i].T.abs()
        close(y, ref, dtype, (k + 8) * EPS32 * size, "y")
        dy = matrix(g, rows + tail, n, dtype, layout)
        dyc = dy.double().cpu()
        big, dx = room(rows + tail, k, dtype, layout)
        B.csr5_grouped_gemm_dx(dy, w, offset, dx)
        untouched(big, rows + tail, k, layout)
        ref, size = torch.full((rows + tail, k), 77.0, dtype=torch.float64).to(dtype).double(), torch.zeros(rows + tail, k, dtype=torch.float64)
        for i, a, b in spans(sizes):
            ref[a:b], size[a:b] = dyc[a:b] @ wc[i], dyc[a:b].abs() @ wc[i].abs()
        close(dx, ref, dtype, (n + 8) * EPS32 * size, "dx")
        big, dw = room(len(sizes) * n, k, dtype, layout)
        B.csr5_grouped_gemm_dw(dy, x, offset, dw.unflatten(0, (len(sizes), n)), source=None if s is None else s.to(DEV))
        untouched(big, len(sizes) * n, k, layout)
        ref, size = torch.zeros(len(sizes) * n, k, dtype=torch.float64), torch.zeros(len(sizes) * n, k, dtype=torch.float64)
        for i, a, b in spans(sizes):
            ref[i * n:(i + 1) * n], size[i * n:(i + 1) * n] = dyc[a:b].T @ xc[a:b], dyc[a:b].T.abs() @ xc[a:b].abs()
        close(dw, ref, dtype, (max(sizes) + 8) * EPS32 * size, "dw")


@pytest.mark.parametrize("dtype", HALF, ids=ids)
def test_grouped_gradients_are_those_of_differences(dtype):
    """With small whole numbers every sum is exact, and so is a difference of the (linear) product: it has to equal the
    gradients' prediction bit by bit."""
    g = torch.Generator().manual_seed(11)
    sizes, n, k = [3, 0, 20, 1], 24, 40
    rows, groups = sum(sizes), 4
    draw = lambda *shape: torch.randint(-1, 2, shape, generator=g).to(dtype).to(DEV)  # noqa: E731
    x, w, dy, offset = draw(9, k), draw(groups, n, k), draw(rows, n), offsets(sizes)
    source = source_for(g, rows, 9, bad=False).to(DEV)

    def product(x, w):
        y = torch.zeros(rows, n, dtype=dtype, device=DEV)
        B.csr5_grouped_gemm(x, w, offset, y, source=source)
        return y.double()

    dx, dw = torch.zeros(rows, k, dtype=dtype, device=DEV), torch.zeros_like(w)
    B.csr5_grouped_gemm_dx(dy, w, offset, dx)
    B.csr5_grouped_gemm_dw(dy, x, offset, dw, source=source)
    for _ in range(3):
        ex, ew = draw(9, k), draw(groups, n, k)
        moved = ((product(x + ex, w) - product(x, w)) * dy.double()).sum()
        assert moved == (dx.double() * ex[source.long()].double()).sum()
        moved = ((product(x, w + ew) - product(x, w)) * dy.double()).sum()
        assert moved == (dw.double() * ew.double()).sum()


@pytest.mark.parametrize("offset", [[0, 5, 3, 9, 40], [-4, 2, 2, 1000, 6], [9, 9, 9, 9, 9], [0, 0, 0, 0, 30]])
def test_offsets_outside_stay_inside(offset):
    """Clamped to the rows; a group that ends before it begins is empty."""
    g = torch.Generator().manual_seed(0)
    rows, n, k = 30, 32, 48
    x, w = matrix(g, rows, k, torch.bfloat16), experts(g, 4, n, k, torch.bfloat16, "plain")
    o = torch.tensor(offset, dtype=torch.int32, device=DEV)
    big, y = room(rows, n, torch.bfloat16)
    B.csr5_grouped_gemm(x, w, o, y)
    untouched(big, rows, n, "plain")
    dw = torch.empty(4, n, k, dtype=torch.bfloat16, device=DEV)
    B.csr5_grouped_gemm_dw(y, x, o, dw)
    c = [min(max(v, 0), rows) for v in offset]
    for i in range(4):
        if c[i + 1] <= c[i]:
            assert (dw[i] == 0).all()


def test_masked_rows_do_not_spread():
    """A NaN or infinity in a row of x stays in that row's results; rows in no group are not read."""
    g = torch.Generator().manual_seed(0)
    for k in (64, 72, 100, 128):
        x, w = matrix(g, 40, k, torch.bfloat16), experts(g, 2, 256, k, torch.bfloat16, "plain")
        offset = offsets([17, 20])
        x[5], x[38] = math.nan, math.nan
        y = torch.zeros(40, 256, dtype=torch.bfloat16, device=DEV)
        B.csr5_grouped_gemm(x, w, offset, y)
        bad = torch.isnan(y).any(1).cpu()
        assert bad[5] and bad.sum() == 1 and (y[37:] == 0).all()
        dy = matrix(g, 40, 256, torch.bfloat16)
        dy[37:] = math.inf
        x[5] = 0
        dw = torch.empty(2, 256, k, dtype=torch.bfloat16, device=DEV)
        B.csr5_grouped_gemm_dw(dy, x, offset, dw)
        assert torch.isfinite(dw).all()


# ---------------------------------------------------------------------------------------------------------------- 8 bits
def f8_operand(gen, rows, k, block_rows, layout):
    q, scale = quantised(torch.randn(rows, k, generator=gen) * 2, block_rows)
    return place_in(q, layout), scale.to(DEV), meaning(q, scale, block_rows)


F8_SHAPES = [(1, 1, 1, "plain"), (5, 33, 17, "odd"), (16, 128, 128, "plain"), (17, 130, 144, "wide"), (33, 257, 260, "plain"), (129, 384, 512, "wide"),
             (200, 129, 399, "odd"), (260, 264, 1040, "plain"), (8, 1024, 2048, "plain")]


@pytest.mark.parametrize("dtype", HALF + [torch.float32], ids=ids)
@pytest.mark.parametrize("w_rows", [128, 1])
@pytest.mark.parametrize("m,n,k,layout", F8_SHAPES)
def test_f8(dtype, w_rows, m, n, k, layout):
    g = torch.Generator().manual_seed(m + n + k)
    x, xs, xc = f8_operand(g, m, k, 1, layout)
    w, ws, wc = f8_operand(g, n, k, w_rows, layout)
    ref, slack = xc @ wc.T, (k + 8) * EPS32 * (xc.abs() @ wc.T.abs())
    for scales in (xs, xs.T.contiguous().T):                            # in either order
        big, y = room(m, n, dtype, layout)
        B.csr5_gemm_f8(x, scales, w, ws, y, w_rows=w_rows)
        untouched(big, m, n, layout)
        close(y, ref, dtype, slack)


@pytest.mark.parametrize("w_rows", [128, 1])
@pytest.mark.parametrize("groups", GROUPS)
@pytest.mark.parametrize("n,k,layout", [(33, 17, "odd"), (128, 128, "plain"), (264, 400, "wide"), (384, 512, "plain")])
def test_grouped_f8(w_rows, groups, n, k, layout):
    sizes = GROUPS[groups]
    g = torch.Generator().manual_seed(n + k)
    rows, tail, x_rows = sum(sizes), 2, max(sum(sizes) // 2, 1)
    operands = [f8_operand(g, n, k, w_rows, "plain") for _ in sizes]
    flat = place_in(torch.cat([o[0].cpu() for o in operands]), layout)
    w, ws = flat.unflatten(0, (len(sizes), n)), torch.stack([o[1] for o in operands])
    x, xs, xc = f8_operand(g, x_rows, k, 1, layout)
    source = source_for(g, rows + tail, x_rows)
    xs[0] = 1e30 if x_rows > 1 else 1.0     # a large scale belongs to its row alone
    xc = meaning(x.cpu(), xs.cpu(), 1)
    big, y = room(rows + tail, n, torch.bfloat16, layout)
    B.csr5_grouped_gemm_f8(x, xs, w, ws, offsets(sizes), y, w_rows=w_rows, source=source.to(DEV))
    untouched(big, rows + tail, n, layout)
    seen = taken(xc, source, rows + tail)
    ref, size = torch.full((rows + tail, n), 77.0, dtype=torch.float64), torch.zeros(rows + tail, n, dtype=torch.float64)
    ref = ref.to(torch.bfloat16).double()
    for i, a, b in spans(sizes):
        ref[a:b], size[a:b] = seen[a:b] @ operands[i][2].T, seen[a:b].abs() @ operands[i][2].T.abs()
    close(y, ref, torch.bfloat16, (k + 8) * EPS32 * size)


def test_products_of_depth_zero_are_zero():
    y = torch.full((5, 40), 7.0, dtype=torch.bfloat16, device=DEV)
    x, w = torch.empty(5, 0, dtype=torch.bfloat16, device=DEV), torch.empty(2, 40, 0, dtype=torch.bfloat16, device=DEV)
    B.csr5_grouped_gemm(x, w, offsets([2, 3]), y)
    assert (y == 0).all()
    y.fill_(7.0)
    e = lambda *s: torch.empty(*s, device=DEV)  # noqa: E731
    B.csr5_gemm_f8(x.to(torch.float8_e4m3fn), e(5, 0), w[0].to(torch.float8_e4m3fn), e(1, 0), y)
    assert (y == 0).all()


# ---------------------------------------------------------------------------------------------------------------- large tiles
TALL = [700, 0, 1301]


@pytest.mark.parametrize("dtype", HALF, ids=ids)
@pytest.mark.parametrize("n,k", [(5640, 264), (5632, 40), (264, 5640), (2056, 2056)])
def test_grouped_in_large_tiles(dtype, n, k):
    """Enough rows and columns for the large tiles: of y with many columns, of dx with a large depth's, of dw."""
    g = torch.Generator().manual_seed(n)
    rows, groups = sum(TALL), len(TALL)
    offset, w, x = offsets(TALL), experts(g, groups, n, k, dtype, "wide", k ** -0.5), matrix(g, rows, k, dtype, "wide")
    source = source_for(g, rows, rows)
    dy = matrix(g, rows, n, dtype, "wide")
    big_y, y = room(rows, n, dtype, "wide")
    big_x, dx = room(rows, k, dtype, "wide")
    big_w, dw = room(groups * n, k, dtype, "wide")
    B.csr5_grouped_gemm(x, w, offset, y, source=source.to(DEV))
    B.csr5_grouped_gemm_dx(dy, w, offset, dx)
    B.csr5_grouped_gemm_dw(dy, x, offset, dw.unflatten(0, (groups, n)), source=source.to(DEV))
    for big, r, c in ((big_y, rows, n), (big_x, rows, k), (big_w, groups * n, k)):
        untouched(big, r, c, "wide")
    xc, wc, dyc = taken(x, source, rows), w.double().cpu(), dy.double().cpu()
    for i, a, b in spans(TALL):
        close(y[a:b], xc[a:b] @ wc[i].T, dtype, (k + 8) * EPS32 * (xc[a:b].abs() @ wc[i].T.abs()), "y")
        close(dx[a:b], dyc[a:b] @ wc[i], dtype, (n + 8) * EPS32 * (dyc[a:b].abs() @ wc[i].abs()), "dx")
        close(dw[i * n:(i + 1) * n], dyc[a:b].T @ xc[a:b], dtype, (b - a + 8) * EPS32 * (dyc[a:b].T.abs() @ xc[a:b].abs()), "dw")


@pytest.mark.parametrize("w_rows", [128, 1])
@pytest.mark.parametrize("n,k", [(5640, 272), (5632, 1040)])
def test_f8_in_large_tiles(w_rows, n, k):
    g = torch.Generator().manual_seed(n + k)
    rows, groups = sum(TALL), len(TALL)
    x, xs, xc = f8_operand(g, rows, k, 1, "wide")
    operands = [f8_operand(g, n, k, w_rows, "plain") for _ in range(groups)]
    w, ws = torch.stack([o[0] for o in operands]), torch.stack([o[1] for o in operands])
    source = source_for(g, rows, rows)
    for s in (None, source):
        big, y = room(rows, n, torch.bfloat16, "wide")
        B.csr5_grouped_gemm_f8(x, xs, w, ws, offsets(TALL), y, w_rows=w_rows, source=None if s is None else s.to(DEV))
        untouched(big, rows, n, "wide")
        seen = taken(xc, s, rows)
        for i, a, b in spans(TALL):
            close(y[a:b], seen[a:b] @ operands[i][2].T, torch.bfloat16, (k + 8) * EPS32 * (seen[a:b].abs() @ operands[i][2].T.abs()))


@pytest.mark.parametrize("n", [64, 5632])
def test_rows_past_32_bits(n):
    """A source may name rows whose bytes from the beginning of x do not fit 32 bits."""
    g = torch.Generator().manual_seed(n)
    x_rows, k, rows, sizes = 70_000, 256, 2000, [1200, 800]
    source = torch.randint(0, x_rows, (rows,), generator=g, dtype=torch.int32)
    source[:5] = torch.tensor([x_rows - 1, 0, 65_535, 65_536, 65_537])
    names = source.long().to(DEV)
    offset = offsets(sizes)
    some = torch.cat([torch.arange(0, 40), torch.arange(1190, 1230), torch.arange(1990, 2000)])
    wide = torch.zeros(x_rows, 65_536, dtype=torch.uint8, device=DEV)          # rows 64 KiB apart: 4.6e9 bytes
    values = (torch.randn(rows, k, generator=g)).to(torch.bfloat16)
    x = wide.view(torch.bfloat16)[:, :k]
    x[names] = values.to(DEV)
    xc = x[names].double().cpu()
    w = experts(g, 2, n, k, torch.bfloat16, "plain")
    y, dw = torch.empty(rows, n, dtype=torch.bfloat16, device=DEV), torch.empty_like(w)
    B.csr5_grouped_gemm(x, w, offset, y, source=source.to(DEV))
    B.csr5_grouped_gemm_dw(y, x, offset, dw, source=source.to(DEV))
    wc = w.double().cpu()
    for i, a, b in spans(sizes):
        at = some[(some >= a) & (some < b)]
        close(y[at.to(DEV)], xc[at] @ wc[i].T, torch.bfloat16, (k + 8) * EPS32 * (xc[at].abs() @ wc[i].T.abs()), "y")
        yc = y[a:b, :64].double().cpu()
        close(dw[i, :64], yc.T @ xc[a:b], torch.bfloat16, (b - a + 8) * EPS32 * (yc.T.abs() @ xc[a:b].abs()), "dw")
    q, scale = quantised(torch.randn(rows, k, generator=g), 1)
    x8, xs = wide[:, :k], torch.zeros(x_rows, 2, device=DEV)
    x8[names], xs[names] = q.view(torch.uint8).to(DEV), scale.to(DEV)
    xc = meaning(x8[names].cpu().view(torch.float8_e4m3fn), xs[names].cpu(), 1)
    w8, ws, w8c = f8_operand(g, n, k, 128, "plain")
    B.csr5_grouped_gemm_f8(x8, xs, torch.stack([w8, w8]), torch.stack([ws, ws]), offset, y, source=source.to(DEV))
    close(y[some.to(DEV)], xc[some] @ w8c.T, torch.bfloat16, (k + 8) * EPS32 * (xc[some].abs() @ w8c.T.abs()), "f8")


def test_products_on_another_stream_and_in_a_graph():
    """The calls go to the given stream, and captured ones give the same on every replay."""
    g = torch.Generator().manual_seed(8)
    sizes, n, k = [5, 0, 300, 40], 256, 384
    rows = sum(sizes)
    x, w, offset = matrix(g, rows, k, torch.bfloat16), experts(g, 4, n, k, torch.bfloat16, "plain"), offsets(sizes)
    y, dx, dw = torch.empty(rows, n, dtype=torch.bfloat16, device=DEV), torch.empty_like(x), torch.empty_like(w)
    q, scale = torch.empty(rows, k, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(rows, 3, device=DEV)
    w8, ws, _ = f8_operand(g, n, k, 128, "plain")
    y8 = torch.empty_like(y)

    def work():
        B.csr5_grouped_gemm(x, w, offset, y)
        B.csr5_grouped_gemm_dx(y, w, offset, dx)
        B.csr5_grouped_gemm_dw(y, x, offset, dw)
        B.csr5_quantise(x, q, scale)
        B.csr5_gemm_f8(q, scale, w8, ws, y8)

    outs = (y, dx, dw, q.view(torch.uint8), scale, y8)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        work()
    s.synchronize()
    first = [t.clone() for t in outs]
    work()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for turn in range(3):
        x.copy_(torch.randn(rows, k, generator=g))
        work()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), turn


@pytest.mark.parametrize("sizes", [[3, 2], [700, 600]])
def test_sources_of_no_rows(sizes):
    """x has no rows, so no source names one: zeros, and nothing of x or its scales is read."""
    rows, n, k = sum(sizes), 8192, 256
    source = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    w = torch.ones(2, n, k, dtype=torch.bfloat16, device=DEV)
    y = torch.ones(rows, n, dtype=torch.bfloat16, device=DEV)
    B.csr5_grouped_gemm(w[0, :0], w, offsets(sizes), y, source=source)
    assert not y.any()
    y.fill_(1)
    w8, ws = w.to(torch.float8_e4m3fn), torch.ones(2, n // 128, 2, device=DEV)
    B.csr5_grouped_gemm_f8(w8[0, :0], ws[0, :0], w8, ws, offsets(sizes), y, source=source)
    assert not y.any()
    dw = torch.ones_like(w)
    B.csr5_grouped_gemm_dw(y, w[0, :0], offsets(sizes), dw, source=source)
    assert not dw.any()


@pytest.mark.parametrize("w_rows", [128, 1])
@pytest.mark.parametrize("sizes,n,k", [([200], 5640, 272), ([513], 2056, 1040), ([70, 0, 130, 65], 2048, 528)])
def test_f8_in_tiles_of_64_rows(sizes, n, k, w_rows):
    """More rows and columns than go for few, fewer than fill the card with larger tiles."""
    g = torch.Generator().manual_seed(n + k)
    rows, groups = sum(sizes), len(sizes)
    x, xs, xc = f8_operand(g, rows, k, 1, "wide")
    operands = [f8_operand(g, n, k, w_rows, "plain") for _ in range(groups)]
    w, ws = torch.stack([o[0] for o in operands]), torch.stack([o[1] for o in operands])
    source = source_for(g, rows, rows)
    for s in (None, source):
        big, y = room(rows, n, torch.float16, "wide")
        B.csr5_grouped_gemm_f8(x, xs, w, ws, offsets(sizes), y, w_rows=w_rows, source=None if s is None else s.to(DEV))
        untouched(big, rows, n, "wide")
        seen = taken(xc, s, rows)
        for i, a, b in spans(sizes):
            close(y[a:b], seen[a:b] @ operands[i][2].T, torch.float16, (k + 8) * EPS32 * (seen[a:b].abs() @ operands[i][2].T.abs()))


# ---------------------------------------------------------------------------------------------------------------- where steps end
ENDS = [1, 63, 64, 65, 127, 128, 129, 0, 192, 193, 256, 257, 320, 321]


@pytest.mark.parametrize("n,k", [(136, 264), (1024, 1032)])
@pytest.mark.parametrize("by_source", [False, True])
def test_dw_of_groups_that_end_about_a_step(n, k, by_source):
    g = torch.Generator().manual_seed(n + by_source)
    rows, groups = sum(ENDS), len(ENDS)
    dy, x = matrix(g, rows, n, torch.bfloat16), matrix(g, rows, k, torch.bfloat16)
    source = source_for(g, rows, rows) if by_source else None
    big, dw = room(groups * n, k, torch.bfloat16, "wide")
    B.csr5_grouped_gemm_dw(dy, x, offsets(ENDS), dw.unflatten(0, (groups, n)), source=None if source is None else source.to(DEV))
    untouched(big, groups * n, k, "wide")
    xc, dyc = taken(x, source, rows), dy.double().cpu()
    for i, a, b in spans(ENDS):
        close(dw[i * n:(i + 1) * n], dyc[a:b].T @ xc[a:b], torch.bfloat16, (b - a + 8) * EPS32 * (dyc[a:b].T.abs() @ xc[a:b].abs()), ENDS[i])


@pytest.mark.parametrize("depth", [8, 56, 64, 72, 128, 136, 184, 192, 200, 256, 264, 320, 328])
def test_depths_that_end_about_a_step(depth):
    """y and dx of that depth, in 128 x 128 tiles and (192 of them) larger ones."""
    g = torch.Generator().manual_seed(depth)
    for rows, cols in ((300, 2056), (3080, 4104)):
        offset = offsets([rows])
        for turned in (False, True):
            x = matrix(g, rows, depth, torch.bfloat16)
            w = experts(g, 1, *((depth, cols) if turned else (cols, depth)), torch.bfloat16, "plain")
            big, y = room(rows, cols, torch.bfloat16, "wide")
            (B.csr5_grouped_gemm_dx if turned else B.csr5_grouped_gemm)(x, w, offset, y)
            untouched(big, rows, cols, "wide")
            xc, wc = x.double().cpu(), w[0].double().cpu() if turned else w[0].double().cpu().T
            close(y, xc @ wc, torch.bfloat16, (depth + 8) * EPS32 * (xc.abs() @ wc.abs()), (rows, turned))


@pytest.mark.parametrize("depth", [16, 48, 64, 112, 128, 144, 256, 272, 384, 400, 512, 528, 640])
def test_f8_depths_that_end_about_a_step(depth):
    """In tiles of 64 x 128, of 128 x 128 and (192 of them) of 192 x 256.  Whole numbers up to 4 with scales of powers of two:
    every sum is exact, in the 8-bit instruction as well, so only y is rounded (not at all in float32)."""
    g = torch.Generator().manual_seed(depth)

    def operand(rows, by):
        q = torch.randint(-4, 5, (rows, depth), generator=g).float()
        scale = 2.0 ** torch.randint(-2, 3, (-(-rows // by), -(-depth // 128)), generator=g)
        seen = q * scale.repeat_interleave(by, 0)[:rows].repeat_interleave(128, 1)[:, :depth]
        return q.to(torch.float8_e4m3fn).to(DEV), scale.to(DEV), seen.double()

    for rows, n in ((300, 2056), (1500, 2056), (3080, 4104)):
        x, xs, xc = operand(rows, 1)
        for w_rows in (128, 1):
            w, ws, wc = operand(n, w_rows)
            big, y = room(rows, n, torch.float32, "wide")
            B.csr5_gemm_f8(x, xs, w, ws, y, w_rows=w_rows)
            untouched(big, rows, n, "wide")
            assert torch.equal(y.double().cpu(), xc @ wc.T), (rows, w_rows)
