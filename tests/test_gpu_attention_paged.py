"""Attention of new tokens over a paged cache, against the definition in 64 bits (GPU)."""
import math

import pytest
import torch

import attention_util as A
from layer_util import DEV
from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16

# new tokens and cached ones (the new among them) of each request
BATCHES = {
    "one": [(1, 1)],
    "single": [(1, 5), (1, 64), (1, 300), (1, 1), (1, 65), (1, 0), (1, 129)],
    "few": [(3, 3), (2, 700), (0, 40), (5, 33), (1, 256)],
    "chunks": [(40, 40), (1, 900), (130, 400), (64, 64), (17, 500)],
    "more queries than keys": [(20, 7), (1, 0), (90, 33)],
    "long": [(1, 5000), (2, 3333)],
}


def batch(lengths, heads, kv, d, dtype, page, layout="plain", seed=0, width=None, behind=2):
    gen = torch.Generator().manual_seed(seed)
    qo, spans = A.pointer([a for a, _ in lengths]), A.sequences(A.pointer([b for _, b in lengths]))
    rows, k_rows = int(qo[-1]) + behind, spans[-1][1]
    k, v = A.heads(gen, k_rows, kv, d, dtype), A.heads(gen, k_rows, kv, d, dtype)
    k_cache, v_cache, table, length = A.paged(gen, k, v, spans, page, layout, width=width)
    return dict(q=A.heads(gen, rows, heads, d, dtype, layout, scale=1.5), k=k, v=v, spans=spans, qo=qo, k_cache=k_cache, v_cache=v_cache, table=table, length=length,
                out=A.heads(gen, rows, heads, d, dtype, layout, fill=77.0), lse=torch.full((heads, rows), 77.0, device=DEV), page=page)


def space(p):
    need = B.csr5_attention_paged_workspace_bytes(p["q"].shape[0], p["q"].shape[1], p["k"].shape[1], p["q"].shape[2], p["table"].shape[0], p["table"].shape[1] * p["page"])
    return torch.full((need,), 255, dtype=torch.uint8, device=DEV)


def call(p, **more):
    B.csr5_attention_paged(p["q"], p["k_cache"], p["v_cache"], p["qo"], p["length"], p["table"], p["out"], space(p), lse=p["lse"], **more)


def check(p, **more):
    call(p, **more)
    A.check_forward(p["q"], p["k"], p["v"], A.sequences(p["qo"]), p["spans"], p["out"], p["lse"], p["q"].shape[2] ** -0.5, True)
    end = int(p["qo"][-1])
    assert bool((p["out"][end:] == 77).all()) and bool((p["lse"][:, end:] == 77).all())


@pytest.mark.parametrize("name", list(BATCHES))
@pytest.mark.parametrize("dtype,heads,kv,d,page", [(BF16, 8, 2, 128, 16), (F16, 4, 4, 64, 64), (BF16, 16, 1, 80, 1), (F16, 7, 1, 128, 256), (BF16, 40, 8, 96, 32)])
def test_batches(dtype, heads, kv, d, page, name):
    check(batch(BATCHES[name], heads, kv, d, dtype, page))


@pytest.mark.parametrize("layout", ["plain", "major", "odd"])
@pytest.mark.parametrize("d", [1, 9, 48, 127, 128])
def test_sizes_of_heads_and_strides(d, layout):
    check(batch([(1, 70), (6, 130), (1, 3)], 6, 3, d, F16 if d % 2 else BF16, 8, layout, seed=d))
    check(batch([(1, 70), (70, 130), (1, 3)], 6, 3, d, F16 if d % 2 else BF16, 8, layout, seed=d))


@pytest.mark.parametrize("heads,kv", [(16, 16), (8, 8), (4, 2)])
@pytest.mark.parametrize("page", [1, 16, 64])
def test_chunks_by_every_kernel(page, heads, kv):
    """One, two or four wavefronts to a row, pages of less than a load's rows, of some of them and of whole tiles; the keys split and not."""
    check(batch([(500, 900), (1, 700), (300, 300), (129, 1500), (64, 64)], heads, kv, 128, BF16, page, seed=9))
    check(batch([(260, 400), (1, 70), (300, 300)], heads, kv, 64, F16, page, seed=10))


@pytest.mark.parametrize("width", [40, 400, 5000])
def test_tables_much_wider_than_the_histories(width):
    check(batch([(1, 600), (4, 130), (1, 0), (1, 1), (2, 639)], 16, 2, 64, BF16, 16, seed=1, width=width))


def test_many_requests():
    check(batch([(1, 3 + 11 * (i % 17)) for i in range(150)], 8, 2, 64, BF16, 16, seed=2))
    check(batch([(i % 4, 3 + 11 * (i % 17)) for i in range(150)], 2, 1, 64, F16, 16, seed=2))


def test_pages_of_none_are_zeros():
    p = batch([(1, 100), (3, 90)], 4, 2, 64, BF16, 16, seed=3)
    for s, page, value in ((0, 2, -1), (1, 0, 10 ** 6), (1, 5, -2 ** 31)):
        p["table"][s, page] = value
        a = p["spans"][s][0] + page * 16
        b = min(a + 16, p["spans"][s][1])
        p["k"][a:b], p["v"][a:b] = 0.0, 0.0
    check(p)


def test_lengths_past_the_table_end_with_it():
    p = batch([(1, 64), (5, 48)], 4, 2, 64, BF16, 16, seed=4)
    assert p["table"].shape[1] == 4
    p["length"][0] = 10 ** 9
    p["length"][1] = -3
    p["spans"][1] = (p["spans"][1][0], p["spans"][1][0])
    check(p)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_the_mask_hides_does_not_show(bad):
    """The rest of a last page is NaN in all of these tests; here also tokens that a chunk's earlier ones do not see."""
    for new, heads in ((6, 4), (100, 4)):
        p = batch([(new, 130), (1, 40)], heads, 2, 64, BF16, 16, seed=5)
        call(p)
        clean, clean_lse = p["out"].clone(), p["lse"].clone()
        page, place = int(p["table"][0, 127 // 16]), 127 % 16
        p["k_cache"][page, place], p["v_cache"][page, place] = bad, bad
        call(p)
        sees = [new - 3, new - 2, new - 1]
        rest = [i for i in range(new + 1) if i not in sees]
        assert torch.equal(p["out"][rest], clean[rest]) and torch.equal(p["lse"][:, rest], clean_lse[:, rest])
        assert not bool(torch.isfinite(p["out"][sees].float()).any())


def test_a_cache_past_32_bits():
    """Pages that begin 2^31 values and 2^32 bytes into the cache."""
    page, kv, d = 64, 8, 128
    pages = 2 ** 31 // (page * kv * d) + 40
    if torch.cuda.mem_get_info()[0] < 3 * pages * page * kv * d * 2:
        pytest.skip("not enough memory")
    gen = torch.Generator().manual_seed(6)
    k_cache = torch.empty(pages, page, kv, d, dtype=BF16, device=DEV)
    v_cache = torch.empty(pages, page, kv, d, dtype=BF16, device=DEV)
    k, v = A.heads(gen, 200, kv, d, BF16), A.heads(gen, 200, kv, d, BF16)
    table = torch.tensor([[pages - 1, 3, pages - 30, pages - 7]], dtype=torch.int32, device=DEV)
    for i, at in enumerate(table[0].tolist()):
        rows = min(64, 200 - 64 * i)
        k_cache[at, :rows], v_cache[at, :rows] = k[64 * i:64 * i + rows], v[64 * i:64 * i + rows]
    for new in (1, 90):
        q = A.heads(gen, new, 16, d, BF16)
        p = dict(q=q, k=k, v=v, spans=[(0, 200)], qo=A.pointer([new]), k_cache=k_cache, v_cache=v_cache, table=table, length=torch.tensor([200], dtype=torch.int32, device=DEV),
                 out=torch.empty_like(q), lse=torch.empty(16, new, device=DEV), page=page)
        check(p)


def test_another_stream_twice_the_same_and_replayed():
    """Two graphs with workspaces of their own, replayed in turn with eager calls between, while the requests go on."""
    p = batch([(1, 1500), (1, 77), (1, 900), (1, 4)], 16, 2, 128, BF16, 16, seed=7, width=120)
    q = batch([(30, 1500), (1, 77), (90, 900), (2, 4)], 16, 2, 128, BF16, 16, seed=8)
    graphs, keep = [], []
    for x in (p, q):
        call(x)
        torch.cuda.synchronize()
        first = x["out"].clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(x)
        torch.cuda.synchronize()
        assert torch.equal(first, x["out"])
        own = space(x)
        keep.append(own)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.csr5_attention_paged(x["q"], x["k_cache"], x["v_cache"], x["qo"], x["length"], x["table"], x["out"], own, lse=x["lse"])
        graphs.append(graph)
    for turn in range(3):
        for x in (p, q):
            x["q"].mul_(0.9)
            x["length"].sub_(turn)
        want = []
        for x in (p, q):
            call(x)
            want.append((x["out"].clone(), x["lse"].clone()))
            x["out"].fill_(3.0), x["lse"].fill_(3.0)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for x, (out, lse) in zip((p, q), want):
            end = int(x["qo"][-1])
            assert torch.equal(x["out"][:end], out[:end]) and torch.equal(x["lse"][:, :end], lse[:, :end])


@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** -126, 2.0 ** -149])
@pytest.mark.parametrize("lengths", [[(1, 1500), (3, 700), (1, 1)], [(300, 1500), (100, 100)]])
def test_the_smallest_scales(lengths, scale):
    """Scores of which 8 powers of two are past the largest number, with the keys split."""
    p = batch(lengths, 8, 4, 64, BF16, 16, seed=12)
    assert space(p).numel() > 0
    call(p, scale=scale)
    A.check_forward(p["q"], p["k"], p["v"], A.sequences(p["qo"]), p["spans"], p["out"], p["lse"], scale, True)
