"""Attention and its gradients in sizes that fill the GPU, whose kernels have a row's keys in one wavefront, against the definitions in 64 bits (GPU)."""
import math

import pytest
import torch

import attention_util as A
import test_gpu_attention as packed_tests
import test_gpu_attention_paged as paged_tests
from layer_util import DEV
from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16

PACKED = {
    "same": [(420, 420), (300, 300), (64, 64), (129, 129), (31, 31)],
    "more keys": [(300, 520), (129, 300), (33, 400), (64, 65), (0, 9), (257, 257)],
    "more queries": [(520, 300), (300, 129), (90, 1), (65, 64), (70, 0), (128, 128)],
}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", list(PACKED))
@pytest.mark.parametrize("dtype,d,heads,kv", [(BF16, 128, 64, 32), (F16, 128, 40, 40), (BF16, 64, 32, 32), (F16, 64, 64, 32), (BF16, 96, 40, 40), (F16, 80, 48, 24), (F16, 64, 56, 56)])
def test_packed(dtype, d, heads, kv, name, causal):
    p = packed_tests.packed(PACKED[name], heads, kv, d, dtype, seed=31)
    assert A.forward_kernel(p["rows"], len(PACKED[name]), heads, kv) == ("many", 1)
    packed_tests.forward(p, causal)
    packed_tests.backward(p, causal)


@pytest.mark.parametrize("layout", ["beside", "major", "odd"])
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F16, 72), (BF16, 33), (F16, 64), (BF16, 100), (F16, 9)])
def test_strides(dtype, d, layout):
    """Rows of any addresses, and heads of other than 64, 96 and 128 values."""
    heads, kv = 64, 32
    p = packed_tests.packed(PACKED["same"], heads, kv, d, dtype, layout, seed=32)
    assert A.forward_kernel(p["rows"], len(PACKED["same"]), heads, kv) == ("many", 1)
    packed_tests.forward(p, True)
    packed_tests.backward(p, True, layout)


@pytest.mark.parametrize("heads,kv", [(64, 8), (80, 5), (96, 32)])
def test_many_heads_to_one(heads, kv):
    lengths = [(430, 430), (520, 700), (300, 300), (77, 77)]
    p = packed_tests.packed(lengths, heads, kv, 64, BF16, seed=33)
    assert A.forward_kernel(p["rows"], len(lengths), heads, kv) == ("many", 1)
    packed_tests.forward(p, True)
    packed_tests.backward(p, True)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_values_that_are_not_finite_where_they_are_hidden(bad):
    """Against the definition, in which what the mask hides does not count, whatever it holds."""
    heads, kv, d = 64, 32, 128
    for dtype in (BF16, F16):
        p = packed_tests.packed(PACKED["same"], heads, kv, d, dtype, seed=34)
        p["v"][70, :, 5], p["v"][419, :, 11], p["k"][400] = bad, bad, math.nan
        p["out"].fill_(77.0), p["lse"].fill_(77.0)
        B.csr5_attention(p["q"], p["k"], p["v"], p["qo"], p["ko"], p["out"], lse=p["lse"])
        assert not bool(torch.isfinite(p["out"][400:420].float()).any()) and bool(torch.isfinite(p["out"][:70].float()).all())
        A.check_forward(p["q"][:400], p["k"][:400], p["v"][:400], [(0, 400)], [(0, 400)], p["out"][:400], p["lse"][:, :400], d ** -0.5, True, "before")



CHUNKS = {"split": [(500, 900), (1, 700), (300, 300), (129, 1500), (64, 64)], "whole": [(260, 400), (1, 70), (300, 300), (70, 501)]}


@pytest.mark.parametrize("name", list(CHUNKS))
@pytest.mark.parametrize("page,layout", [(1, "plain"), (16, "plain"), (64, "plain"), (16, "major"), (32, "odd")])
@pytest.mark.parametrize("dtype,d,heads,kv", [(BF16, 128, 64, 32), (F16, 64, 64, 64), (F16, 128, 56, 56), (BF16, 80, 64, 32)])
def test_chunks(dtype, d, heads, kv, page, layout, name):
    p = paged_tests.batch(CHUNKS[name], heads, kv, d, dtype, page, layout, seed=35)
    rows, n = p["q"].shape[0], len(CHUNKS[name])
    assert A.forward_kernel(rows, n, heads, kv) == ("many", 1)
    assert A.is_split(rows, n, heads, kv, p["table"].shape[1] * page) == (name == "split") == (paged_tests.space(p).numel() > 0)
    paged_tests.check(p)


@pytest.mark.parametrize("page", [1, 16, 64])
@pytest.mark.parametrize("heads,kv,sides", [(8, 8, 4), (24, 24, 2), (64, 64, 1)])
def test_chunks_by_every_number_of_wavefronts(heads, kv, sides, page):
    lengths = [(500, 900), (1, 700), (300, 300), (129, 1500), (64, 64)]
    p = paged_tests.batch(lengths, heads, kv, 64, BF16, page, seed=36)
    assert A.forward_kernel(p["q"].shape[0], len(lengths), heads, kv) == ("many", sides)
    paged_tests.check(p)


@pytest.mark.parametrize("heads,kv,sides", [(16, 16, 4), (40, 40, 2), (64, 64, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_by_every_number_of_wavefronts(heads, kv, sides, causal):
    lengths = [(300, 300), (257, 400), (64, 64)]
    p = packed_tests.packed(lengths, heads, kv, 64, F16, seed=37)
    assert A.forward_kernel(p["rows"], len(lengths), heads, kv) == ("many", sides)
    packed_tests.forward(p, causal)
    packed_tests.backward(p, causal)


def guarded(rows, heads, d, margin=64):
    """A view [rows, heads, d] of 77 within a longer array of 77, and the array."""
    whole = torch.full(((rows + 2 * margin) * heads * d,), 77.0, dtype=BF16, device=DEV)
    return whole[margin * heads * d:(margin + rows) * heads * d].view(rows, heads, d), whole


@pytest.mark.parametrize("heads,kv", [(2, 1), (24, 24), (96, 48)])
def test_offsets_out_of_order_write_within_their_sequences(heads, kv):
    """Offsets that shrink, pass the end or lie before the beginning: well-formed sequences among them have their results, rows in none stay, and
    nothing beside the arrays or the workspace is written."""
    rows, d = 183, 64
    for qo, ko, q_spans, k_spans in (
            ([-5, 60, 1000, 2000], [0, 60, 120, 5000], [(0, 60), (60, 183), (183, 183)], [(0, 60), (60, 120), (120, 183)]),
            ([0, 60, 120, 180], [180, 120, 60, 0], [(0, 60), (60, 120), (120, 180)], [(180, 180), (120, 120), (60, 60)]),
            ([0, 100, 50, 120], [0, 50, 100, 120], None, None)):
        gen = torch.Generator().manual_seed(38)
        q, k, v, dout = (A.heads(gen, rows, h, d, BF16) for h in (heads, kv, kv, heads))
        offset = [torch.tensor(o, dtype=torch.int32, device=DEV) for o in (qo, ko)]
        (out, out_all), (dq, dq_all), (dk, dk_all), (dv, dv_all) = (guarded(rows, h, d) for h in (heads, heads, kv, kv))
        lse_all = torch.full((heads * (rows + 400),), 77.0, device=DEV)
        lse = lse_all[heads * 200:heads * (200 + rows)].view(heads, rows)
        need = B.csr5_attention_backward_workspace_bytes(rows, heads)
        space = torch.full((need + 8192,), 123, dtype=torch.uint8, device=DEV)
        B.csr5_attention(q, k, v, *offset, out, lse=lse)
        forward = out.clone(), lse.clone()
        B.csr5_attention_backward(dout, q, k, v, out, lse, *offset, dq, dk, dv, space[4096:4096 + need])
        assert bool((space[:4096] == 123).all()) and bool((space[4096 + need:] == 123).all())
        assert torch.equal(out, forward[0]) and torch.equal(lse, forward[1])
        if q_spans:
            A.check_forward(q, k, v, q_spans, k_spans, out, lse, d ** -0.5, True)
            A.check_backward(q, k, v, dout, out, lse, q_spans, k_spans, dq, dk, dv, d ** -0.5, True)
        end = (max(b for _, b in q_spans), max(b for _, b in k_spans) if ko[0] == 0 else 0) if q_spans else (120, 120)
        assert bool((out[end[0]:] == 77).all()) and bool((lse[:, end[0]:] == 77).all()) and bool((dq[end[0]:] == 77).all())
        assert bool((dk[end[1]:] == 77).all()) and bool((dv[end[1]:] == 77).all())
        for view, whole in ((out, out_all), (dq, dq_all), (dk, dk_all), (dv, dv_all), (lse, lse_all)):
            view.fill_(77.0)
            assert bool((whole == 77).all())


FORMS = {("few", 1): ([(5, 70), (1, 300), (8, 8), (3, 131)], 4, 2), ("few", 2): ([(13, 70), (11, 300), (16, 16)], 4, 2), ("few", 4): ([(30, 70), (25, 300), (31, 31)], 4, 2),
         ("many", 4): ([(130, 200), (65, 65)], 4, 2), ("many", 2): ([(130, 200), (65, 65)], 60, 60), ("many", 1): ([(130, 200), (65, 65)], 128, 128)}


@pytest.mark.parametrize("layout", ["plain", "odd"])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("form", list(FORMS), ids=lambda f: f"{f[0]} {f[1]}")
def test_every_form(form, dtype, d, layout):
    """Each compiled kernel once: by rows and wavefronts, type, size of heads, rows in 16 bytes or not, packed and paged."""
    lengths, heads, kv = FORMS[form]
    p = packed_tests.packed(lengths, heads, kv, d, dtype, layout, seed=39)
    assert A.forward_kernel(p["rows"], len(lengths), heads, kv) == form
    packed_tests.forward(p, True)
    packed_tests.backward(p, True, layout)
    p = paged_tests.batch(lengths, heads, kv, d, dtype, 16, layout, seed=40)
    assert A.forward_kernel(p["q"].shape[0], len(lengths), heads, kv) == form
    paged_tests.check(p)
