"""Rotary positions, to rows and into a paged cache, against the definition in 64 bits (GPU)."""
import math

import pytest
import torch

import attention_util as A
from layer_util import DEV, U
from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
I32 = torch.int32


def turned(x, position, frequency, axis, interleaved, inverse):
    """x [tokens, heads, d] turned, in 64 bits, and the bound of the error before the last rounding."""
    x = x.double()
    pairs = frequency.numel()
    angle = torch.zeros(x.shape[0], pairs, dtype=torch.float64, device=x.device)
    for i in range(pairs):
        if 0 <= int(axis[i]) < position.shape[0]:
            angle[:, i] = position[int(axis[i])].double() * frequency[i].double()
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None] * (-1 if inverse else 1)
    first, second = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
    a, b = x[..., first], x[..., second]
    y, slack = x.clone(), torch.zeros_like(x)
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    # cosine and sine in 32 bits, of an angle that is reduced in 64 and rounded to 32: within 3 * 2^-24 * pi; two products and a sum: 3 * 2^-24
    both = (a.abs() + b.abs()) * 14 * 2.0 ** -24
    slack[..., first], slack[..., second] = both, both
    return y, slack


def case(tokens, heads, kv, d, rot, axes, dtype, layout="plain", seed=0, far=1 << 20):
    gen = torch.Generator().manual_seed(seed)
    q, k, v = (A.heads(gen, tokens, h, d, dtype, layout) for h in (heads, kv, kv))
    position = torch.randint(0, far, (axes, tokens), generator=gen).to(I32).to(DEV)
    frequency = (10000.0 ** (-torch.arange(rot // 2) / max(rot // 2, 1))).float().to(DEV)
    axis = torch.randint(0, axes, (rot // 2,), generator=gen).to(I32).to(DEV)
    return gen, q, k, v, position, frequency, axis


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,kv,d,rot,axes,dtype,layout", [
    (1, 1, 1, 2, 2, 1, BF16, "plain"), (5, 4, 2, 128, 128, 1, BF16, "plain"), (33, 28, 4, 128, 96, 3, BF16, "beside"), (7, 3, 3, 64, 64, 2, F16, "major"),
    (9, 5, 1, 80, 80, 2, F32, "plain"), (4, 2, 2, 33, 20, 1, F32, "odd"), (300, 2, 1, 96, 48, 3, F16, "odd"), (6, 2, 1, 64, 0, 1, BF16, "plain"), (3, 2, 2, 512, 512, 4, BF16, "plain"),
    (11, 6, 2, 72, 36, 2, F16, "beside"), (1, 64, 8, 128, 128, 1, BF16, "plain"), (13, 4, 4, 40, 24, 1, BF16, "plain"),
])
def test_rows(tokens, heads, kv, d, rot, axes, dtype, layout, interleaved, inverse):
    gen, q, k, v, position, frequency, axis = case(tokens, heads, kv, d, rot, axes, dtype, layout)
    q_out, k_out = A.heads(gen, tokens, heads, d, dtype, layout, fill=77.0), A.heads(gen, tokens, kv, d, dtype, layout, fill=77.0)
    B.csr5_rotary(q, k, position, frequency, q_out, k_out=k_out, axis=axis, interleaved=interleaved, inverse=inverse)
    for x, y in ((q, q_out), (k, k_out)):
        want, slack = turned(x, position, frequency, axis, interleaved, inverse)
        A.bounded(y, want, slack, dtype, "turned")
        y.fill_(77.0)
        rest = A.whole(y)
        assert bool(((rest == 77) | rest.isnan()).all())
    # in place, and without keys
    want, slack = turned(q, position, frequency, axis, interleaved, inverse)
    B.csr5_rotary(q, None, position, frequency, q, axis=axis, interleaved=interleaved, inverse=inverse)
    A.bounded(q, want, slack, dtype, "in place")


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,d,page,layout", [(BF16, 128, 16, "plain"), (F16, 64, 1, "major"), (F32, 80, 64, "plain"), (BF16, 33, 8, "odd"), (BF16, 96, 256, "major")])
def test_into_the_cache(dtype, d, page, layout, interleaved):
    tokens, heads, kv, pages = 37, 6, 2, -(-50 // page) + 3
    gen, q, k, v, position, frequency, axis = case(tokens, heads, kv, d, d // 4 * 2, 2, dtype, "beside", seed=1)
    shape = {"plain": (pages, page, kv, d), "major": (pages, kv, page, d), "odd": (pages, page, kv, d + 4)}[layout]
    caches = []
    for _ in range(2):
        c = torch.full(shape, 77.0, dtype=dtype, device=DEV)
        caches.append(c.transpose(1, 2) if layout == "major" else c[..., 1:1 + d] if layout == "odd" else c)
    slot = torch.randperm(pages * page, generator=gen)[:tokens].to(I32)
    slot[5], slot[20], slot[36], slot[9] = -1, pages * page, 2 ** 31 - 1, -2 ** 31
    slot = slot.to(DEV)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    B.csr5_rotary(q, k, position, frequency, q_out, k_out=k_out, axis=axis, interleaved=interleaved, v=v, slot=slot, k_cache=caches[0], v_cache=caches[1])
    want, slack = turned(k, position, frequency, axis, interleaved, False)
    A.bounded(k_out, want, slack, dtype, "beside the cache")
    written = torch.zeros(pages, page, dtype=torch.bool, device=DEV)
    for t, at in enumerate(slot.tolist()):
        if 0 <= at < pages * page:
            A.bounded(caches[0][at // page, at % page], want[t], slack[t], dtype, "key")
            assert torch.equal(caches[1][at // page, at % page], v[t])
            written[at // page, at % page] = True
    for c in caches:
        c[written] = 77.0
        assert bool((A.whole(c) == 77).all())
    again = [torch.full_like(c, 5.0) for c in caches]
    B.csr5_rotary(q, k, position, frequency, q_out, axis=axis, interleaved=interleaved, v=v, slot=slot, k_cache=again[0], v_cache=again[1])
    at = slot.tolist()[0]
    A.bounded(again[0][at // page, at % page], want[0], slack[0], dtype, "without rows")


def test_far_positions_and_axes_of_none():
    tokens, d = 9, 64
    gen, q, _, _, _, frequency, _ = case(tokens, 2, 1, d, d, 1, F32, seed=2)
    position = torch.tensor([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 999983, 123456789, 7, 65537]], dtype=I32, device=DEV)
    frequency[:4] = torch.tensor([1.0, 0.7, 1e-8, 3.0])
    out = torch.empty_like(q)
    B.csr5_rotary(q, None, position[0], frequency, out)
    want, slack = turned(q, position, frequency, torch.zeros(32, dtype=I32), False, False)
    A.bounded(out, want, slack, F32, "far")
    axis = torch.zeros(32, dtype=I32, device=DEV)
    axis[3], axis[8], axis[20] = -1, 1, 2 ** 31 - 1
    B.csr5_rotary(q, None, position, frequency, out, axis=axis)
    want, slack = turned(q, position, frequency, axis, False, False)
    A.bounded(out, want, slack, F32, "axes of none")
    assert torch.equal(out[..., [3, 35, 8, 40, 20, 52]], q[..., [3, 35, 8, 40, 20, 52]])


def test_back_and_forth_and_the_gradient():
    """The inverse undoes it, and is its transpose: <turn(x), y> = <x, inverse(y)>."""
    _, q, k, _, position, frequency, axis = case(50, 4, 4, 128, 96, 3, F32, seed=3)
    a, b, c = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    B.csr5_rotary(q, None, position, frequency, a, axis=axis)
    B.csr5_rotary(a, None, position, frequency, b, axis=axis, inverse=True)
    assert float((b - q).abs().max()) <= 2 * 30 * 2.0 ** -24 * 2 * float(q.abs().max())
    B.csr5_rotary(k, None, position, frequency, c, axis=axis, inverse=True)
    left, right = (a.double() * k.double()).sum(), (q.double() * c.double()).sum()
    size = (a.double() * k.double()).square().sum().sqrt()
    assert abs(float(left - right)) <= 40 * 2.0 ** -24 * float(size) * 8


def test_replayed():
    gen, q, k, v, position, frequency, axis = case(40, 4, 2, 128, 128, 1, BF16, seed=4)
    caches = [torch.zeros(8, 16, 2, 128, dtype=BF16, device=DEV) for _ in range(2)]
    slot = torch.randperm(128, generator=gen)[:40].to(I32).to(DEV)
    out = torch.empty_like(q)
    run = lambda: B.csr5_rotary(q, k, position, frequency, out, axis=axis, v=v, slot=slot, k_cache=caches[0], v_cache=caches[1])  # noqa: E731
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        position.add_(1), slot.add_(1).remainder_(128)
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in (out, *caches)]
        out.zero_()
        caches[0][slot.long() // 16, slot.long() % 16] = 0
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (out, *caches)))


def test_nothing_to_do():
    e = lambda *shape, dtype=BF16: torch.empty(*shape, dtype=dtype, device=DEV)  # noqa: E731
    B.csr5_rotary(e(0, 4, 64), e(0, 2, 64), e(0, dtype=I32), e(32, dtype=F32), e(0, 4, 64), k_out=e(0, 2, 64))
    q = e(3, 4, 64).normal_()
    out = e(3, 4, 64)
    B.csr5_rotary(q, None, torch.zeros(3, dtype=I32, device=DEV), e(0, dtype=F32), out)
    assert torch.equal(q, out) and U and math.pi


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,kv,d,rot,axes,dtype,layout", [
    (1024, 4, 2, 128, 128, 1, BF16, "plain"), (1025, 3, 1, 128, 96, 3, BF16, "beside"), (1027, 2, 2, 64, 64, 2, F16, "major"), (2050, 5, 1, 80, 80, 2, F32, "plain"), (1030, 2, 1, 512, 512, 1, F32, "plain"),
    (1999, 1, 1, 40, 16, 1, F16, "plain"), (1026, 2, 2, 33, 20, 1, F32, "odd"),
])
def test_prompts(tokens, heads, kv, d, rot, axes, dtype, layout, interleaved):
    """From 1024 tokens on, of which four are a workgroup's: to rows, in place, back, and into the cache."""
    gen, q, k, v, position, frequency, axis = case(tokens, heads, kv, d, rot, axes, dtype, layout, seed=5)
    wants = {inverse: [turned(x, position, frequency, axis, interleaved, inverse) for x in (q, k)] for inverse in (False, True)}
    for inverse in (False, True):
        q_out, k_out = A.heads(gen, tokens, heads, d, dtype, layout, fill=77.0), A.heads(gen, tokens, kv, d, dtype, layout, fill=77.0)
        B.csr5_rotary(q, k, position, frequency, q_out, k_out=k_out, axis=axis, interleaved=interleaved, inverse=inverse)
        for y, (want, slack) in zip((q_out, k_out), wants[inverse]):
            A.bounded(y, want, slack, dtype, ("turned", inverse))
            y.fill_(77.0)
            rest = A.whole(y)
            assert bool(((rest == 77) | rest.isnan()).all())
    page, pages = 16, tokens // 16 + 9
    caches = [torch.full((pages, page, kv, d), 77.0, dtype=dtype, device=DEV) for _ in range(2)]
    slot = torch.randperm(pages * page, generator=gen)[:tokens].to(I32)
    for i, none in ((0, -1), (5, pages * page), (1000, 2 ** 31 - 1), (tokens - 1, -2 ** 31), (tokens - 2, -7)):
        slot[i] = none
    slot = slot.to(DEV)
    q_before = q.clone()
    B.csr5_rotary(q, k, position, frequency, q, axis=axis, interleaved=interleaved, v=v, slot=slot, k_cache=caches[0], v_cache=caches[1])
    A.bounded(q, *wants[False][0], dtype, "in place")
    q.copy_(q_before)
    there = (slot >= 0) & (slot < pages * page)
    at = slot[there].long()
    want, slack = wants[False][1]
    A.bounded(caches[0][at // page, at % page], want[there], slack[there], dtype, "keys")
    assert torch.equal(caches[1][at // page, at % page], v[there])
    for c in caches:
        c[at // page, at % page] = 77.0
        assert bool((c == 77).all())
