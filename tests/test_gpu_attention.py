"""Attention over packed sequences, and its gradients, against the definitions in 64 bits (GPU)."""
import math

import pytest
import torch

import attention_util as A
from layer_util import DEV
from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16

# queries and keys of each sequence
LENGTHS = {
    "one": [(1, 1)],
    "small": [(3, 3), (0, 0), (1, 1), (17, 17), (2, 2)],
    "edges": [(31, 31), (32, 32), (33, 33), (63, 63), (64, 64), (65, 65), (127, 127), (128, 128), (129, 129)],
    "long": [(700, 700), (1, 1), (257, 257)],
    "more keys": [(5, 77), (130, 200), (1, 300), (64, 65), (0, 9), (33, 1000)],
    "more queries": [(77, 5), (200, 130), (300, 1), (65, 64), (9, 0), (150, 0), (400, 33)],
}


def packed(lengths, heads, kv, d, dtype, layout="plain", seed=0, behind=3):
    gen = torch.Generator().manual_seed(seed)
    qo, ko = A.pointer([a for a, _ in lengths]), A.pointer([b for _, b in lengths])
    rows, k_rows = int(qo[-1]) + behind, int(ko[-1]) + behind
    return dict(q=A.heads(gen, rows, heads, d, dtype, layout, scale=1.5), k=A.heads(gen, k_rows, kv, d, dtype, layout), v=A.heads(gen, k_rows, kv, d, dtype, layout),
                qo=qo, ko=ko, out=A.heads(gen, rows, heads, d, dtype, layout, fill=77.0), lse=torch.full((heads, rows), 77.0, device=DEV), rows=rows, k_rows=k_rows, gen=gen)


def forward(p, causal, scale=None):
    p["out"].fill_(77.0), p["lse"].fill_(77.0)
    around = A.whole(p["out"]).clone()
    B.csr5_attention(p["q"], p["k"], p["v"], p["qo"], p["ko"], p["out"], lse=p["lse"], scale=scale, causal=causal)
    d = p["q"].shape[2]
    A.check_forward(p["q"], p["k"], p["v"], A.sequences(p["qo"]), A.sequences(p["ko"]), p["out"], p["lse"], d ** -0.5 if scale is None else scale, causal)
    end = int(p["qo"][-1])
    assert bool((p["out"][end:] == 77).all()) and bool((p["lse"][:, end:] == 77).all())
    got = A.whole(p["out"]).clone()
    p["out"][:end] = 77.0
    assert torch.equal(A.whole(p["out"]).nan_to_num(5.0), around.nan_to_num(5.0))          # nothing around the rows was written
    A.whole(p["out"]).copy_(got)


def backward(p, causal, layout="plain", scale=None):
    q, k, v = p["q"], p["k"], p["v"]
    heads, kv, d = q.shape[1], k.shape[1], q.shape[2]
    dout = A.heads(p["gen"], p["rows"], heads, d, q.dtype, layout)
    dq, dk, dv = (A.heads(p["gen"], rows, h, d, q.dtype, layout, fill=77.0) for rows, h in ((p["rows"], heads), (p["k_rows"], kv), (p["k_rows"], kv)))
    space = torch.full((B.csr5_attention_backward_workspace_bytes(p["rows"], heads),), 255, dtype=torch.uint8, device=DEV)
    B.csr5_attention_backward(dout, q, k, v, p["out"], p["lse"], p["qo"], p["ko"], dq, dk, dv, space, scale=scale, causal=causal)
    A.check_backward(q, k, v, dout, p["out"], p["lse"], A.sequences(p["qo"]), A.sequences(p["ko"]), dq, dk, dv, d ** -0.5 if scale is None else scale, causal)
    end, k_end = int(p["qo"][-1]), int(p["ko"][-1])
    assert bool((dq[end:] == 77).all()) and bool((dk[k_end:] == 77).all()) and bool((dv[k_end:] == 77).all())
    for t, n in ((dq, end), (dk, k_end), (dv, k_end)):
        t[:n] = 77.0
        left = A.whole(t)
        assert bool(((left == 77) | left.isnan()).all())                                   # nothing around the rows was written


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", list(LENGTHS))
@pytest.mark.parametrize("dtype,heads,kv,d", [(BF16, 4, 2, 128), (F16, 3, 3, 64), (BF16, 8, 1, 80)])
def test_lengths(dtype, heads, kv, d, name, causal):
    p = packed(LENGTHS[name], heads, kv, d, dtype)
    forward(p, causal)
    backward(p, causal)


@pytest.mark.parametrize("layout", ["plain", "beside", "major", "odd"])
@pytest.mark.parametrize("d", [1, 7, 8, 16, 33, 64, 72, 96, 127, 128])
def test_sizes_of_heads_and_strides(d, layout):
    p = packed([(70, 70), (5, 40), (40, 5)], 4, 2, d, F16 if d % 16 else BF16, layout, seed=d)
    forward(p, True)
    backward(p, True, layout)


@pytest.mark.parametrize("heads,kv", [(1, 1), (5, 1), (7, 7), (14, 2), (16, 1), (40, 8)])
def test_heads_that_share(heads, kv):
    p = packed([(50, 50), (9, 170), (1, 64)], heads, kv, 64, BF16, seed=heads)
    forward(p, True)
    backward(p, True)


# Few workgroups: their wavefronts share rows' keys, four or two of them; more: none do.  Short sequences, and few heads that share keys or many, have kernels
# of their own in the gradients of keys.
EVERY = [("one wavefront to a row", [(700, 700), (300, 300), (520, 600), (64, 64), (33, 1)], 16, 16), ("two", [(700, 700), (300, 300), (520, 600), (64, 64), (33, 1)], 8, 8),
         ("four", [(450, 450), (129, 300)], 2, 2), ("short ones", [(90, 90)] * 21 + [(5, 200), (70, 3)], 8, 2), ("many heads to one", [(260, 260), (31, 64)], 16, 1),
         ("five heads to one", [(130, 131), (64, 64)], 10, 2)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F16, 64), (BF16, 96), (F16, 88)])
@pytest.mark.parametrize("name,lengths,heads,kv", EVERY, ids=[e[0] for e in EVERY])
def test_every_kernel(name, lengths, heads, kv, dtype, d, causal):
    p = packed(lengths, heads, kv, d, dtype, seed=17)
    forward(p, causal)
    backward(p, causal)


@pytest.mark.parametrize("scale", [1e-3, 0.5, 4.0])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_scales(scale, dtype):
    """Flat softmaxes, and those that are nearly one key's."""
    p = packed([(150, 150), (20, 90)], 4, 4, 64, dtype, seed=3)
    forward(p, True, scale)
    backward(p, True, scale=scale)


def test_many_sequences():
    lengths = [((7 * i) % 23, (7 * i) % 23 + (i % 5) * 9) for i in range(301)]
    p = packed(lengths, 2, 1, 64, BF16, seed=1)
    forward(p, True)
    backward(p, True)


def test_scores_that_grow_and_are_far_apart():
    """The running maximum rises with every key, or falls off at once: sums are rescaled in every tile, or never."""
    for sign in (1.0, -1.0):
        p = packed([(300, 300)], 2, 1, 64, BF16, seed=2)
        p["q"].fill_(1.0)
        p["k"].copy_((sign * torch.arange(p["k_rows"], device=DEV) * 0.125)[:, None, None].expand_as(p["k"]))
        forward(p, False)
        forward(p, True)
        backward(p, True)


@pytest.mark.parametrize("heads,kv", [(4, 2), (16, 8), (32, 16), (3, 3)])
@pytest.mark.parametrize("bad", [math.nan, -math.inf])
def test_what_the_mask_hides_does_not_show_in_any_kernel(bad, heads, kv):
    """As below, with more workgroups: 150 rows and 20 short sequences."""
    m, d = 150, 128
    lengths = [(m, m)] + [(30, 30)] * 20
    for at in (70, 149):
        clean, p = (packed(lengths, heads, kv, d, BF16, seed=5) for _ in range(2))
        p["k"][at], p["v"][at] = bad, bad
        for x in (clean, p):
            B.csr5_attention(x["q"], x["k"], x["v"], x["qo"], x["ko"], x["out"], lse=x["lse"])
        other = [i for i in range(m + 600) if not at <= i < m]
        assert torch.equal(p["out"][other], clean["out"][other]) and torch.equal(p["lse"][:, other], clean["lse"][:, other])
        grads = []
        for x, k, q in ((clean, clean["k"], clean["q"]), (clean, p["k"], clean["q"]), (clean, clean["k"], clean["q"].clone())):
            if len(grads) == 2:
                q[at] = bad
            dout = A.heads(torch.Generator().manual_seed(9), x["rows"], heads, d, BF16)
            dq, dk, dv = (A.heads(x["gen"], r, h, d, BF16, fill=0.0) for r, h in ((x["rows"], heads), (x["k_rows"], kv), (x["k_rows"], kv)))
            space = torch.full((B.csr5_attention_backward_workspace_bytes(x["rows"], heads),), 255, dtype=torch.uint8, device=DEV)
            B.csr5_attention_backward(dout, q, k, x["v"], x["out"], x["lse"], x["qo"], x["ko"], dq, dk, dv, space)
            grads.append((dq, dk, dv))
        (dq, dk, dv), (eq, ek, ev), (fq, fk, fv) = grads
        assert torch.equal(dq[other], eq[other]) and not bool(torch.isfinite(eq[at:m].float()).any())          # a key: the rows before it, and other sequences
        keys = [i for i in range(m + 600) if not (i <= at)]
        assert torch.equal(dk[keys], fk[keys]) and torch.equal(dv[keys], fv[keys]) and not bool(torch.isfinite(fk[:at + 1].float()).any())      # a query: the keys after it


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_the_mask_hides_does_not_show(bad, d):
    """Keys and values that a row does not see, and in the gradients rows that do not see a key, hold what is not finite."""
    m = 150
    for at in (0, 40, 149):
        p = packed([(m, m), (30, 30)], 4, 2, d, BF16, seed=5)
        clean = packed([(m, m), (30, 30)], 4, 2, d, BF16, seed=5)
        p["k"][at], p["v"][at] = bad, bad
        for x in (p, clean):
            B.csr5_attention(x["q"], x["k"], x["v"], x["qo"], x["ko"], x["out"], lse=x["lse"])
        sees = list(range(at, m))
        other = [i for i in range(m + 30) if i not in sees]
        assert torch.equal(p["out"][other], clean["out"][other]) and torch.equal(p["lse"][:, other], clean["lse"][:, other])
        assert not bool(torch.isfinite(p["out"][at + 1:m].float()).any()) or bad == -math.inf
        # the gradients: rows from `at` on are not finite, so are all of dq there and the keys that they see
        grads = []
        for x, value in ((clean, 1.0), (clean, bad)):
            dout = A.heads(torch.Generator().manual_seed(9), x["rows"], 4, d, BF16)
            dout[at] = dout[at] * value
            dq, dk, dv = (A.heads(x["gen"], r, h, d, BF16, fill=0.0) for r, h in ((x["rows"], 4), (x["k_rows"], 2), (x["k_rows"], 2)))
            space = torch.empty(B.csr5_attention_backward_workspace_bytes(x["rows"], 4), dtype=torch.uint8, device=DEV)
            B.csr5_attention_backward(dout, x["q"], x["k"], x["v"], x["out"], x["lse"], x["qo"], x["ko"], dq, dk, dv, space)
            grads.append((dq, dk, dv))
        (dq, dk, dv), (eq, ek, ev) = grads
        rest = [i for i in range(m + 30) if i != at]
        assert torch.equal(dq[rest], eq[rest])
        unseen = list(range(at + 1, m + 30))
        assert torch.equal(dk[unseen], ek[unseen]) and torch.equal(dv[unseen], ev[unseen])
        assert not bool(torch.isfinite(ev[:at + 1].float()).any())


def test_a_value_that_is_infinite_where_it_is_seen():
    p = packed([(90, 90)], 2, 1, 64, BF16, seed=6)
    p["v"][33, 0, 5], p["v"][50, 0, 5], p["v"][20, 0, 7] = math.inf, -math.inf, -math.inf
    B.csr5_attention(p["q"], p["k"], p["v"], p["qo"], p["ko"], p["out"], lse=p["lse"])
    out = p["out"].float()[:90]
    assert bool(torch.isfinite(out[:33, :, 5]).all()) and bool((out[33:50, :, 5] == math.inf).all()) and bool(out[50:, :, 5].isnan().all())
    assert bool(torch.isfinite(out[:20, :, 7]).all()) and bool((out[20:, :, 7] == -math.inf).all())
    others = [c for c in range(64) if c not in (5, 7)]
    assert bool(torch.isfinite(out[:, :, others]).all())


def test_scores_of_minus_infinity_and_rows_of_nothing_else():
    p = packed([(40, 40)], 2, 1, 64, F16, seed=7)
    p["q"].abs_()
    p["k"][3] = -math.inf
    B.csr5_attention(p["q"], p["k"], p["v"], p["qo"], p["ko"], p["out"], lse=p["lse"])
    k, v = torch.cat([p["k"][:3], p["k"][4:]]), torch.cat([p["v"][:3], p["v"][4:]])
    want, lse, slack, lse_slack, *_ = A.forward_of(p["q"][10:40, 0].double(), k[:39, 0].double(), v[:39, 0].double(), 30, 39, 0.125, True, F16)
    A.bounded(p["out"][10:40, 0], want, slack, F16, "out")
    A.bounded(p["lse"][0, 10:40], lse, lse_slack, torch.float32, "lse")


def test_differences():
    """The gradients against differences of the definition, in 64 bits, along random directions."""
    p = packed([(45, 45), (20, 61)], 4, 2, 64, F16, seed=8, behind=0)
    forward(p, True)
    gen = p["gen"]
    dout = A.heads(gen, p["rows"], 4, 64, F16)
    dq, dk, dv = torch.empty_like(p["q"]), torch.empty_like(p["k"]), torch.empty_like(p["v"])
    space = torch.empty(B.csr5_attention_backward_workspace_bytes(p["rows"], 4), dtype=torch.uint8, device=DEV)
    B.csr5_attention_backward(dout, p["q"], p["k"], p["v"], p["out"], p["lse"], p["qo"], p["ko"], dq, dk, dv, space)

    def loss(q, k, v):
        total = 0.0
        for (a, b), (c, e) in zip(A.sequences(p["qo"]), A.sequences(p["ko"])):
            for h in range(4):
                o = A.forward_of(q[a:b, h], k[c:e, h // 2], v[c:e, h // 2], b - a, e - c, 0.125, True, F16)[0]
                total += float((o * dout[a:b, h].double()).sum())
        return total
    q, k, v = (p[n].double() for n in "qkv")
    for i, (x, g) in enumerate(((q, dq), (k, dk), (v, dv))):
        way = torch.randn(x.shape, generator=gen).double().to(DEV)
        step = 1e-5
        args = [q, k, v]
        up, down = list(args), list(args)
        up[i], down[i] = x + step * way, x - step * way
        slope = (loss(*up) - loss(*down)) / (2 * step)
        got = float((g.double() * way).sum())
        # the gradient's roundings are 2^-10 of a value at most (p or ds, then the result) and, as errors of values that are taken at
        # random signs, add up as the root of the sum of squares: 6 of those is what a difference may be; the difference's own error is step^2 * third derivatives
        assert abs(got - slope) <= 6 * 2.0 ** -10 * float((g.double() * way).square().sum().sqrt()) + 6 * 2.0 ** -10 * float(g.double().square().sum().sqrt()), (i, got, slope)


def test_offsets_out_of_order_stay_within_the_arrays():
    """Offsets that shrink, pass the end or lie before the beginning: rows that no sequence has stay, nothing else is written."""
    p = packed([(60, 60), (60, 60), (60, 60)], 2, 1, 64, BF16, seed=4)
    for qo, ko in (([0, 100, 50, 120], [0, 50, 100, 120]), ([-5, 60, 1000, 2000], [0, 60, 120, 5000]), ([0, 60, 120, 180], [180, 120, 60, 0])):
        p["qo"].copy_(torch.tensor(qo)), p["ko"].copy_(torch.tensor(ko))
        B.csr5_attention(p["q"], p["k"], p["v"], p["qo"], p["ko"], p["out"], lse=p["lse"])
        dq, dk, dv = torch.empty_like(p["q"]), torch.empty_like(p["k"]), torch.empty_like(p["v"])
        space = torch.empty(B.csr5_attention_backward_workspace_bytes(p["rows"], 2), dtype=torch.uint8, device=DEV)
        B.csr5_attention_backward(p["out"], p["q"], p["k"], p["v"], p["out"], p["lse"], p["qo"], p["ko"], dq, dk, dv, space)
    torch.cuda.synchronize()


def test_another_stream_twice_the_same_and_replayed():
    p = packed([(300, 300), (77, 500), (1, 1)], 8, 2, 128, BF16, seed=11)
    dout = A.heads(p["gen"], p["rows"], 8, 128, BF16)
    dq, dk, dv = torch.empty_like(p["q"]), torch.empty_like(p["k"]), torch.empty_like(p["v"])
    space = torch.empty(B.csr5_attention_backward_workspace_bytes(p["rows"], 8), dtype=torch.uint8, device=DEV)

    def both(stream=None):
        B.csr5_attention(p["q"], p["k"], p["v"], p["qo"], p["ko"], p["out"], lse=p["lse"], stream=stream)
        B.csr5_attention_backward(dout, p["q"], p["k"], p["v"], p["out"], p["lse"], p["qo"], p["ko"], dq, dk, dv, space, stream=stream)

    def results():
        torch.cuda.synchronize()
        end, k_end = int(p["qo"][-1]), int(p["ko"][-1])
        return [t.clone() for t in (p["out"][:end], p["lse"][:, :end], dq[:end], dk[:k_end], dv[:k_end])]
    both()
    first = results()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    assert all(torch.equal(a, b) for a, b in zip(first, results()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i in range(3):
        p["q"].copy_(A.heads(torch.Generator().manual_seed(50 + i), p["rows"], 8, 128, BF16))
        if i == 1:
            p["qo"].copy_(A.pointer([100, 250, 28])), p["ko"].copy_(A.pointer([300, 400, 101]))
        both()
        want = results()
        for t in (p["out"], p["lse"], dq, dk, dv):
            t.fill_(3.0)
        graph.replay()
        got = results()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_nothing_to_do():
    e = lambda *shape, dtype=BF16: torch.empty(*shape, dtype=dtype, device=DEV)  # noqa: E731
    zero, two = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    B.csr5_attention(e(0, 4, 64), e(0, 2, 64), e(0, 2, 64), zero, zero, e(0, 4, 64), lse=e(4, 0, dtype=torch.float32))
    out, lse = e(5, 4, 64).fill_(3), e(4, 5, dtype=torch.float32).fill_(3)
    B.csr5_attention(e(5, 4, 64), e(0, 2, 64), e(0, 2, 64), two, two, out, lse=lse)
    assert bool((out == 3).all()) and bool((lse == 3).all())
    one = torch.tensor([0, 5], dtype=torch.int32, device=DEV)
    B.csr5_attention(e(5, 4, 64), e(0, 2, 64), e(0, 2, 64), one, two[:2], out, lse=lse)      # five queries, no key
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    dk = e(6, 2, 64).fill_(3)
    dv = dk.clone()
    B.csr5_attention_backward(e(0, 4, 64), e(0, 4, 64), e(6, 2, 64), e(6, 2, 64), e(0, 4, 64), e(4, 0, dtype=torch.float32), two[:2], torch.tensor([0, 6], dtype=torch.int32, device=DEV),
                              e(0, 4, 64), dk, dv, None)                                     # six keys, no query
    assert bool((dk == 0).all()) and bool((dv == 0).all())


@pytest.mark.parametrize("scale", [2.0 ** -100, 1.5e-38, 2.0 ** -126, 2.0 ** -140, 2.0 ** -149])
@pytest.mark.parametrize("lengths,heads,kv", [([(1, 90), (2, 400)], 4, 2), ([(150, 150)], 4, 2), ([(150, 150)] + [(40, 40)] * 20, 8, 8), ([(150, 150)] + [(40, 40)] * 20, 32, 16)])
def test_the_smallest_scales(lengths, heads, kv, scale):
    """Scores that are all but 0 in units of which 8 powers of two are past the largest number: means of the values."""
    p = packed(lengths, heads, kv, 64, BF16, seed=12)
    forward(p, True, scale)
    backward(p, True, scale=scale)


def test_no_query_heads():
    """Keys that no head of queries shares have gradients of 0, as those that no query sees."""
    e = lambda *shape, dtype=BF16: torch.empty(*shape, dtype=dtype, device=DEV)  # noqa: E731
    dk = e(150, 2, 64).fill_(3)
    dv = dk.clone()
    offset, k_offset = torch.tensor([0, 5, 7], dtype=torch.int32, device=DEV), torch.tensor([0, 90, 140], dtype=torch.int32, device=DEV)
    none = e(7, 0, 64)
    B.csr5_attention_backward(none, none, e(150, 2, 64), e(150, 2, 64), none, e(0, 7, dtype=torch.float32), offset, k_offset, none, dk, dv, None)
    assert bool((dk[:140] == 0).all()) and bool((dv[:140] == 0).all()) and bool((dk[140:] == 3).all()) and bool((dv[140:] == 3).all())
