"""The router, the way back to the tokens, the norm and the quantisation against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

from layer_util import DEV, EPS32, close, matrix, place_in, quantised, room, untouched
from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]
ids = lambda t: str(t).replace("torch.", "")  # noqa: E731


# ---------------------------------------------------------------------------------------------------------------- router
def route_reference(logits, k):
    """expert, weight, offset, source, place by definition, and how far each weight's exponent reaches."""
    v = logits.double().numpy()
    t, e = v.shape
    expert, weight, reach = np.full((t, k), -1), np.zeros((t, k)), np.zeros((t, k))
    for i in range(t):
        order = sorted((-v[i, j], j) for j in range(e) if not math.isnan(v[i, j]) and v[i, j] > -math.inf)[:k]
        for j, (_, at) in enumerate(order):
            expert[i, j] = at
        if order:
            top = -order[0][0]
            if math.isinf(top):
                weight[i] = math.nan
            else:
                part = [math.exp(-m - top) for m, _ in order]
                weight[i, :len(part)] = np.array(part) / sum(part)
                reach[i, :len(part)] = [m + top for m, _ in order]
        if np.isnan(v[i]).any():
            weight[i] = math.nan
    flat = expert.reshape(-1)
    rows = [p for g in range(e) for p in np.nonzero(flat == g)[0]]
    offset = np.concatenate([[0], np.cumsum([int((flat == g).sum()) for g in range(e)])])
    source, place = np.full(t * k, -1), np.full(t * k, -1)
    for r, p in enumerate(rows):
        source[r], place[p] = p // k, r
    return expert, weight, offset, source, place.reshape(t, k), reach


def route(logits, k, stream=None):
    t, e = logits.shape
    i32 = dict(dtype=torch.int32, device=DEV)
    out = dict(expert=torch.full((t, k), 7777, **i32), weight=torch.full((t, k), 7.0, device=DEV), offset=torch.full((e + 1,), 7777, **i32),
               source=torch.full((t * k,), 7777, **i32), place=torch.full((t, k), 7777, **i32))
    ws = torch.full((B.csr5_route_workspace_bytes(t, e, k),), 255, dtype=torch.uint8, device=DEV)
    B.csr5_route(logits, k, *out.values(), workspace=ws, stream=stream)
    return out


def check_route(logits, k):
    got = {n: v.cpu().numpy() for n, v in route(logits, k).items()}
    expert, weight, offset, source, place, reach = route_reference(logits.cpu(), k)
    assert np.array_equal(got["expert"], expert)
    assert np.array_equal(got["offset"], offset)
    assert np.array_equal(got["place"], place)
    assert np.array_equal(got["source"], source)
    # exp within 2 units in the last place, its argument within half a unit, a sum of k, a quotient
    bound = (k + 8 + reach) * EPS32 * weight + 2.0 ** -126
    assert np.array_equal(np.isnan(got["weight"]), np.isnan(weight))
    ok = ~np.isnan(weight)
    assert (np.abs(got["weight"] - weight)[ok] <= bound[ok]).all()


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("tokens,experts,k", [(0, 8, 2), (1, 1, 1), (1, 64, 8), (3, 65, 1), (63, 60, 6), (64, 128, 8), (65, 7, 7),
                                              (130, 33, 32), (300, 256, 8), (1000, 16, 2), (4500, 160, 6), (77, 1000, 5), (70, 1024, 32)])
def test_route(dtype, tokens, experts, k):
    g = torch.Generator().manual_seed(tokens + experts)
    check_route((torch.randn(tokens, experts, generator=g) * 2).to(dtype).to(DEV), k)


@pytest.mark.parametrize("tokens", [5, 200])
def test_route_masks_ties_and_strides(tokens):
    g = torch.Generator().manual_seed(3)
    v = torch.randint(-2, 3, (tokens, 48), generator=g).float()         # many ties; -0 and 0 are equal
    v[:, 5] = -0.0
    v[:, 40:] = -math.inf
    v[1] = -math.inf                                                    # nothing left
    v[2, 3:] = -math.inf                                                # fewer than k left
    v[3] = torch.finfo(torch.float32).min                               # the type's lowest value is a value
    v[4] = 1.0
    v[-1, 7] = math.nan
    v[0, 9] = math.inf
    check_route(place_in(v, "odd"), 6)
    check_route(place_in(v.to(torch.bfloat16), "wide"), 6)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("tokens,experts,k,layout", [(1, 1, 1, "plain"), (5, 60, 6, "odd"), (33, 256, 8, "wide"), (9, 1024, 32, "plain")])
def test_route_backward(dtype, tokens, experts, k, layout):
    g = torch.Generator().manual_seed(experts)
    logits = (torch.randn(tokens, experts, generator=g)).to(DEV)
    logits[0, k // 2:] = -math.inf
    r = route(logits, k)
    dweight = torch.randn(tokens, k, generator=g).to(DEV)
    big, out = room(tokens, experts, dtype, layout)
    B.csr5_route_backward(r["expert"], r["weight"], dweight, out)
    untouched(big, tokens, experts, layout)
    expert, w, d = r["expert"].cpu().long(), r["weight"].double().cpu(), dweight.double().cpu()
    ref, slack = torch.zeros(tokens, experts, dtype=torch.float64), torch.zeros(tokens, experts, dtype=torch.float64)
    for t in range(tokens):
        for j in range(k):
            if expert[t, j] >= 0:
                ref[t, expert[t, j]] = w[t, j] * (d[t, j] - (w[t] * d[t]).sum())
                slack[t, expert[t, j]] = (k + 4) * EPS32 * w[t, j] * (d[t, j].abs() + (w[t] * d[t]).abs().sum())
    close(out, ref, dtype, slack)


def test_route_gradient_is_that_of_differences():
    """The formula against central differences of the definition, in 64 bits; step 1e-5: off by 1e-10 at most."""
    g = torch.Generator().manual_seed(9)
    logits, d = torch.randn(12, dtype=torch.float64, generator=g), torch.randn(4, dtype=torch.float64, generator=g)
    top = torch.topk(logits, 4).indices

    def loss(v):
        return float((torch.softmax(v[top], 0) * d).sum())

    w = torch.softmax(logits[top], 0)
    formula = torch.zeros(12, dtype=torch.float64)
    formula[top] = w * (d - (w * d).sum())
    for e in range(12):
        step = torch.zeros(12, dtype=torch.float64)
        step[e] = 1e-5
        assert abs((loss(logits + step) - loss(logits - step)) / 2e-5 - float(formula[e])) < 1e-8
    r = route(logits.float()[None].to(DEV), 4)
    out = torch.empty(1, 12, device=DEV)
    B.csr5_route_backward(r["expert"], r["weight"], d.float()[None].to(DEV), out)
    # logits and d rounded to 32 bits, then the kernel's own error: some units in the last place of the magnitudes
    assert (out[0].double().cpu() - formula).abs().max() < 64 * EPS32 * float(d.abs().sum())


# ---------------------------------------------------------------------------------------------------------------- combine
def pairs(tokens, k, rows, seed):
    """place: distinct rows in some order, some pairs without one."""
    rng = np.random.default_rng(seed)
    place = rng.permutation(max(rows, tokens * k))[:tokens * k].astype(np.int64)
    place[place >= rows] = -1
    place[rng.random(tokens * k) < 0.1] = -1
    return torch.from_numpy(place.reshape(tokens, k).astype(np.int32))


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("tokens,k,n,layout", [(1, 1, 1, "plain"), (3, 2, 17, "odd"), (7, 8, 512, "wide"), (5, 4, 2048, "plain"), (4, 3, 2049, "odd"), (9, 32, 40, "wide"), (2, 0, 24, "plain")])
def test_combine_and_backward(dtype, tokens, k, n, layout):
    g = torch.Generator().manual_seed(n)
    rows = tokens * k + 3
    place = pairs(tokens, k, rows, n).to(DEV)
    place_cpu = place.cpu().long()
    z, dy, res = (matrix(g, r, n, dtype, layout) for r in (rows, tokens, tokens))
    weight = torch.rand(tokens, k, generator=g).to(DEV)
    zc = torch.cat([z.double().cpu(), torch.zeros(1, n, dtype=torch.float64)])[place_cpu]       # a pair without a row: zeros
    wc = weight.double().cpu()
    for w, r in ((weight, res), (None, None), (weight, None)):
        big, y = room(tokens, n, dtype, layout)
        B.csr5_combine(z, place, y, weight=w, residual=r)
        untouched(big, tokens, n, layout)
        terms = zc * (wc[:, :, None] if w is not None else 1)
        base = r.double().cpu() if r is not None else torch.zeros(tokens, n, dtype=torch.float64)
        close(y, base + terms.sum(1), dtype, (k + 2) * EPS32 * (base.abs() + terms.abs().sum(1)), "y")
    big, dz = room(rows, n, dtype, layout)
    before = dz.clone()
    dweight = torch.full((tokens, k), 7.0, device=DEV)
    B.csr5_combine_backward(dy, z, place, weight, dz, dweight)
    untouched(big, rows, n, layout)
    ref, dyc = before.double().cpu(), dy.double().cpu()
    for t in range(tokens):
        for j in range(k):
            if place_cpu[t, j] >= 0:
                ref[place_cpu[t, j]] = wc[t, j] * dyc[t]
    close(dz, ref, dtype, EPS32 * ref.abs(), "dz")
    terms = dyc[:, None, :] * zc
    close(dweight, terms.sum(2), torch.float32, (n + 2) * EPS32 * terms.abs().sum(2), "dweight")


def test_combine_in_place_and_beyond_the_rows():
    """y may be the residual, dz may be z; places outside the rows are no rows."""
    g = torch.Generator().manual_seed(1)
    z, y = matrix(g, 10, 64, torch.float32), matrix(g, 4, 64, torch.float32)
    place = torch.tensor([[0, 10], [-5, 3], [2 ** 31 - 1, -2 ** 31], [9, 1]], dtype=torch.int32, device=DEV)
    w = torch.rand(4, 2, generator=g).to(DEV)
    zc, wc = z.double().cpu(), w.double().cpu()
    ref = y.double().cpu()
    for t, j, r in ((0, 0, 0), (1, 1, 3), (3, 0, 9), (3, 1, 1)):
        ref[t] += wc[t, j] * zc[r]
    B.csr5_combine(z, place, y, weight=w, residual=y)
    close(y, ref, torch.float32, 4 * EPS32 * 10)
    dy, dweight = matrix(g, 4, 64, torch.float32), torch.full((4, 2), 7.0, device=DEV)
    keep = z.clone()
    B.csr5_combine_backward(dy, z, place, w, z, dweight)
    want = torch.zeros(4, 2, dtype=torch.float64)
    for t, j, r in ((0, 0, 0), (1, 1, 3), (3, 0, 9), (3, 1, 1)):
        want[t, j] = (dy[t].double().cpu() * zc[r]).sum()
        assert torch.equal(z[r], w[t, j] * dy[t])
    assert torch.equal(z[2], keep[2])
    close(dweight, want, torch.float32, 66 * EPS32 * 64 * 4)


# ---------------------------------------------------------------------------------------------------------------- 8 bits
def check_f8(q, scale, ref, slack):
    """q times scale is ref within half a step of e4m3, the scale that of the largest magnitude; slack: relative error of
    the values that were quantised."""
    q, scale, ref = q.float().double().cpu(), scale.double().cpu(), ref.double().cpu()
    rows, n = ref.shape
    for b in range(scale.shape[1]):
        part, got, s = ref[:, b * 128:(b + 1) * 128], q[:, b * 128:(b + 1) * 128], scale[:, b:b + 1]
        want = (part.abs().amax(1, keepdim=True) / 448).clamp(min=2.0 ** -126)
        assert ((s - want).abs() <= (slack + 2 * EPS32) * want).all()
        # half a step: 2^-4 of a normal value, 2^-10 below the smallest normal
        bound = torch.maximum(2.0 ** -4 * part.abs(), 2.0 ** -10 * s) * (1 + 1e-4) + 2 * slack * part.abs()
        assert ((got * s - part).abs() <= bound).all()


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,n,layout", [(1, 1, "plain"), (3, 128, "plain"), (129, 130, "odd"), (5, 1000, "wide"), (257, 384, "plain"), (130, 2049, "odd")])
def test_quantise(dtype, block_rows, rows, n, layout):
    g = torch.Generator().manual_seed(rows * n)
    x = matrix(g, rows, n, dtype, layout, scale=3.0)
    if rows > 2:
        x[2] = 0                                                        # blocks of zeros
        x[1] *= 2.0 ** -12
    big, q = room(rows, n, torch.float8_e4m3fn, layout)
    scale = torch.full((-(-n // 128), -(-rows // block_rows)), 7.0, device=DEV).T       # any layout: here block by block
    B.csr5_quantise(x, q, scale, block_rows=block_rows)
    ref_q, ref_scale = quantised(x.cpu(), block_rows)
    close(scale, ref_scale, torch.float32, EPS32 * ref_scale.double())
    # the quotient is off by 2 units in the last place: another neighbour only next to the middle between two
    got, want = q.float().cpu(), ref_q.float()
    assert (got != want).float().mean() <= 1e-3
    assert ((got - want).abs() <= 0.126 * want.abs() + 2.0 ** -9).all()
    left = {"plain": 0, "wide": 16, "odd": 1}[layout]
    mask = torch.ones(big.shape, dtype=torch.bool, device=DEV)
    mask[1:1 + rows, left:left + n] = False
    assert (big.view(torch.uint8)[mask] == torch.tensor(77.0).to(torch.float8_e4m3fn).view(torch.uint8).item()).all()
    if dtype is torch.float32 and block_rows == 1:
        check_f8(q, scale, x, 0.0)


def test_quantise_infinity_and_nan_show():
    x = torch.ones(4, 256, device=DEV)
    x[0, 3], x[1, 200], x[2, 100] = math.inf, math.nan, 3.0e38
    q, scale = torch.empty(4, 256, dtype=torch.uint8, device=DEV), torch.empty(4, 2, device=DEV)
    B.csr5_quantise(x, q, scale)
    s = scale.cpu()
    assert math.isinf(s[0, 0]) and math.isnan(s[1, 1]) and s[1, 0] == 1 / torch.tensor(448.0) and math.isfinite(s[2, 0])
    value = q.view(torch.float8_e4m3fn).float()[2, :128].cpu() * s[2, 0]
    assert value[100] == pytest.approx(3.0e38, rel=1e-6) and (value[:100] == 0).all()


# ---------------------------------------------------------------------------------------------------------------- norm
NORMS = [(1, 1, "plain"), (3, 8, "plain"), (2, 511, "odd"), (5, 1024, "wide"), (4, 2048, "plain"), (3, 2056, "plain"), (2, 4096, "plain"), (3, 5000, "odd"),
         (2, 8192, "wide"), (2, 9000, "plain"), (1, 20000, "odd"), (2, 32768, "plain"), (1100, 384, "plain")]


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rows,n,layout", NORMS)
def test_rmsnorm(dtype, rows, n, layout):
    g = torch.Generator().manual_seed(n)
    x, res = matrix(g, rows, n, dtype, layout), matrix(g, rows, n, dtype, layout, scale=2.0)
    gain = (1 + 0.3 * torch.randn(n, generator=g)).to(dtype).to(DEV)
    eps = 1e-5
    for r, w in ((res, gain), (None, None)):
        outs = {name: room(rows, n, t, layout) for name, t in (("h", dtype), ("y", dtype), ("q", torch.float8_e4m3fn))}
        scale, rstd = torch.full((rows, -(-n // 128)), 7.0, device=DEV), torch.full((rows,), 7.0, device=DEV)
        B.csr5_rmsnorm(x, w, eps, residual=r, h=outs["h"][1], y=outs["y"][1], q=outs["q"][1], scale=scale, rstd=rstd)
        h = x.double().cpu() + (0 if r is None else r.double().cpu())
        ref_rstd = (h.square().mean(1) + eps).rsqrt()
        y = h * ref_rstd[:, None] * (1 if w is None else w.double().cpu())
        off = (n + 8) * EPS32               # of the sum of squares, relative; half of it for the root, then some roundings
        for big, _ in (outs["h"], outs["y"]):
            untouched(big, rows, n, layout)
        close(outs["h"][1], h, dtype, EPS32 * h.abs(), "h")
        close(rstd, ref_rstd, torch.float32, off * ref_rstd, "rstd")
        close(outs["y"][1], y, dtype, off * y.abs(), "y")
        check_f8(outs["q"][1], scale, y, off)


def test_rmsnorm_in_place_and_single_outputs():
    g = torch.Generator().manual_seed(5)
    x, res = matrix(g, 6, 640, torch.bfloat16), matrix(g, 6, 640, torch.bfloat16)
    h, y = torch.empty_like(x), torch.empty_like(x)
    B.csr5_rmsnorm(x, None, 1e-6, residual=res, h=h, y=y)
    x2, res2 = x.clone(), res.clone()
    B.csr5_rmsnorm(x2, None, 1e-6, residual=res2, h=res2, y=x2)         # the residual stream and the input in place
    assert torch.equal(res2, h) and torch.equal(x2, y)
    only = torch.empty(6, device=DEV)
    B.csr5_rmsnorm(x, None, 1e-6, residual=res, rstd=only)
    assert torch.isfinite(only).all()
    zero = torch.zeros(2, 640, dtype=torch.bfloat16, device=DEV)
    q, s = torch.full((2, 640), 5, dtype=torch.uint8, device=DEV), torch.empty(2, 5, device=DEV)
    B.csr5_rmsnorm(zero, None, 1e-6, q=q, scale=s)
    assert (q == 0).all() and (s == 2.0 ** -126).all()
    bad = x.clone()
    bad[3, 7] = math.nan
    B.csr5_rmsnorm(bad, None, 1e-6, y=y)
    assert torch.isnan(y[3]).all() and torch.isfinite(y[:3]).all()


def norm_gradients(h, gain, rstd, dy, extra):
    v, u = h * rstd[:, None], dy * gain
    inner = (u * v).mean(1, keepdim=True)
    return rstd[:, None] * (u - v * inner) + extra, (dy * v).sum(0)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rows,n,layout", NORMS + [(0, 64, "plain")])
def test_rmsnorm_backward(dtype, rows, n, layout):
    g = torch.Generator().manual_seed(n + 1)
    h, dy, extra = (matrix(g, rows, n, dtype, layout) for _ in range(3))
    gain = (1 + 0.3 * torch.randn(n, generator=g)).to(dtype).to(DEV)
    rstd = (h.double().square().mean(1) + 1e-5).rsqrt().float()
    ws = torch.full((B.csr5_rmsnorm_workspace_bytes(rows, n),), 255, dtype=torch.uint8, device=DEV)
    hc, dyc, rc = h.double().cpu(), dy.double().cpu(), rstd.double().cpu()
    for w, e in ((gain, extra), (None, None)):
        big, dh = room(rows, n, dtype, layout)
        dgain = torch.full((n,), 7.0, device=DEV)
        B.csr5_rmsnorm_backward(h, w, rstd, dy, dh, dgain, ws, residual_grad=e)
        untouched(big, rows, n, layout)
        wc = torch.ones(n, dtype=torch.float64) if w is None else w.double().cpu()
        ec = torch.zeros(rows, n, dtype=torch.float64) if e is None else e.double().cpu()
        ref, ref_gain = norm_gradients(hc, wc, rc, dyc, ec)
        size, size_gain = norm_gradients(hc.abs(), wc.abs(), rc, dyc.abs(), ec.abs())
        v = (hc * rc[:, None]).abs()
        size = rc[:, None] * ((dyc * wc).abs() + v * ((dyc * wc).abs() * v).mean(1, keepdim=True)) + ec.abs()
        close(dh, ref, dtype, (n + 16) * EPS32 * size, "dh")
        close(dgain, ref_gain, torch.float32, (rows + 8) * EPS32 * size_gain, "dgain")
    alone = torch.empty_like(dh)
    B.csr5_rmsnorm_backward(h, None, rstd, dy, alone)
    assert torch.equal(alone, dh)
    both = dy.clone()
    B.csr5_rmsnorm_backward(h, None, rstd, both, both)                  # in place
    assert torch.equal(both, dh)


def test_rmsnorm_gradient_is_that_of_differences():
    """The formula against central differences of the definition in 64 bits (step 1e-5: off by about 1e-10)."""
    g = torch.Generator().manual_seed(2)
    h, gain, dy = torch.randn(3, 10, dtype=torch.float64, generator=g), torch.randn(10, dtype=torch.float64, generator=g), torch.randn(3, 10, dtype=torch.float64, generator=g)

    def loss(h, gain):
        return float((h * (h.square().mean(1, keepdim=True) + 1e-5).rsqrt() * gain * dy).sum())

    dh, dgain = norm_gradients(h, gain, (h.square().mean(1) + 1e-5).rsqrt(), dy, torch.zeros_like(h))
    for i in range(3):
        for j in range(10):
            step = torch.zeros_like(h)
            step[i, j] = 1e-5
            assert abs((loss(h + step, gain) - loss(h - step, gain)) / 2e-5 - float(dh[i, j])) < 1e-8
    for j in range(10):
        step = torch.zeros_like(gain)
        step[j] = 1e-5
        assert abs((loss(h, gain + step) - loss(h, gain - step)) / 2e-5 - float(dgain[j])) < 1e-8


# ---------------------------------------------------------------------------------------------------------------- streams
def test_other_stream_and_graph():
    """The calls go to the given stream, and a captured layer's front end gives the same on every replay."""
    g = torch.Generator().manual_seed(4)
    s = torch.cuda.Stream()
    logits = torch.randn(500, 64, generator=g).to(DEV)
    want = route(logits, 4)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        got = route(logits, 4)
    s.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in got)
    x, gain = matrix(g, 500, 512, torch.bfloat16), torch.ones(512, dtype=torch.bfloat16, device=DEV)
    y, dh, dgain, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(512, device=DEV), torch.empty(500, device=DEV)
    nws = torch.empty(B.csr5_rmsnorm_workspace_bytes(500, 512), dtype=torch.uint8, device=DEV)
    ws = torch.empty(B.csr5_route_workspace_bytes(500, 64, 4), dtype=torch.uint8, device=DEV)

    def work():
        B.csr5_rmsnorm(x, gain, 1e-6, y=y, rstd=rstd)
        B.csr5_rmsnorm_backward(x, gain, rstd, y, dh, dgain, nws)
        B.csr5_route(logits, 4, *got.values(), workspace=ws)

    with torch.cuda.stream(s):
        work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for turn in range(3):
        logits.copy_(torch.randn(500, 64, generator=g))
        x.copy_(torch.randn(500, 512, generator=g))
        work()
        torch.cuda.synchronize()
        want = [t.clone() for t in (*got.values(), y, dh, dgain)]
        for t in (*got.values(), y, dh, dgain):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (*got.values(), y, dh, dgain))), turn



# ---------------------------------------------------------------------------------------------------------------- very many rows
def test_more_rows_than_one_dimension_of_a_grid_holds():
    """A wavefront (or more) per row: 2^32 threads and more.  Every row is one of four, so the last ones are known."""
    rows, n = 2 ** 26 + 3, 8
    four = torch.tensor([[1, 2, 3, 4, 5, 6, 7, 8], [0] * 8, [-8, 4, 0, 1, 2, 0, 0, 0.5], [2] * 8], dtype=torch.bfloat16, device=DEV)
    x = four.repeat(rows // 4 + 1, 1)[:rows]
    ends = [0, 1, 2, 3, 2 ** 20 - 1, 2 ** 20, 2 ** 20 + 1, 2 ** 24 + 2, 2 ** 26 - 1, 2 ** 26, 2 ** 26 + 1, 2 ** 26 + 2]
    y = torch.full_like(x, 9)
    B.csr5_rmsnorm(x, None, 1e-6, y=y)
    small = torch.empty_like(four)
    B.csr5_rmsnorm(four, None, 1e-6, y=small)
    assert torch.equal(y, small.repeat(rows // 4 + 1, 1)[:rows])
    place = torch.arange(rows, dtype=torch.int32, device=DEV).flip(0).view(rows, 1)
    y.fill_(9)
    B.csr5_combine(x, place, y)
    assert torch.equal(y, x.flip(0))
    weight, dweight = torch.full((rows, 1), 2.0, device=DEV), torch.full((rows, 1), 9.0, device=DEV)
    y.fill_(9)
    B.csr5_combine_backward(x, x, place, weight, y, dweight)
    assert torch.equal(y, 2 * x.flip(0))
    for r in ends:
        assert dweight[r].item() == (x[r].float() * x[rows - 1 - r].float()).sum().item()
    del place
    expert = torch.arange(rows, dtype=torch.int32, device=DEV).remainder_(n).view(rows, 1)
    y.fill_(9)
    B.csr5_route_backward(expert, weight, dweight, y)
    want = torch.zeros_like(y).scatter_(1, expert.long(), (-2 * dweight).to(torch.bfloat16))
    assert torch.equal(y, want)
    del want
    del expert, weight, dweight
    rows = 2 ** 28 + 5
    x = four.repeat(rows // 4 + 1, 1)[:rows]
    q, scale = torch.full((rows, n), 9, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn), torch.full((rows, 1), 9.0, device=DEV)
    B.csr5_quantise(x, q, scale)
    small_q, small_scale = torch.empty(4, n, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(4, 1, device=DEV)
    B.csr5_quantise(four, small_q, small_scale)
    for r in ends + [2 ** 28 - 1, 2 ** 28, 2 ** 28 + 4]:
        assert torch.equal(q[r].view(torch.uint8), small_q[r % 4].view(torch.uint8)) and scale[r].item() == small_scale[r % 4].item()
    assert not (scale == 9).any()
