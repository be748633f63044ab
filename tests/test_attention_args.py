"""Refusals of the attention's calls: in C on the host, before anything is launched (dummy addresses), and of tensors (without memory); no GPU."""
import os

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_1503_05032_amd import binding as B
from paper_1503_05032_amd import build as libbuild

pytestmark = pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
P = 4096        # a plausible, aligned address that is never read
BF16, F16, F32, I32, U8 = torch.bfloat16, torch.float16, torch.float32, torch.int32, torch.uint8
H, Z = B.Heads(P, 512, 128), B.Heads(None, 0, 0)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        libbuild.build(verbose=False)
    return B.load()


def test_pages_refusals(lib):
    def rc(requests=0, width=4, ring=8, page=16, tokens=0, fresh=P, length=P, table=P, ldt=4, pool=P, state=P, offset=P, position=P, slot=P, length_out=P, state_out=P):
        return lib.csr5_pages(requests, width, ring, page, tokens, fresh, length, table, ldt, pool, state, offset, position, slot, length_out, state_out, None)
    for bad in (dict(requests=-1), dict(width=-1), dict(ring=-1), dict(tokens=-1), dict(page=0), dict(page=-16), dict(page=48), dict(state=None), dict(offset=None), dict(state_out=None),
                dict(requests=2, fresh=None), dict(requests=2, length=None), dict(requests=2, length_out=None), dict(requests=2, table=None), dict(requests=2, ldt=3), dict(pool=None),
                dict(tokens=3, position=None), dict(tokens=3, slot=None), dict(fresh=P + 2), dict(offset=P + 1), dict(slot=P + 2)):
        assert rc(**bad) == B.CSR5_EINVAL, bad
    assert rc(requests=2 ** 31 - 1) == B.CSR5_ERANGE and rc(tokens=2 ** 31 - 1) == B.CSR5_ERANGE and rc(width=2 ** 20, page=2 ** 11, ldt=2 ** 20) == B.CSR5_ERANGE


def test_rotary_refusals(lib):
    cache = B.Cache(P, 4096, 256, 128)

    def rc(tokens=3, heads=4, kv=2, d=128, rot=128, dtype=B.CSR5_DTYPE_BF16, axes=1, position=P, ldp=3, frequency=P, axis=None, q=H, q_out=H, k=B.Heads(P, 256, 128),
           k_out=B.Heads(P, 256, 128), v=Z, slot=None, pages=0, page=0, kc=B.Cache(), vc=B.Cache()):
        return lib.csr5_rotary(tokens, heads, kv, d, rot, dtype, axes, position, ldp, frequency, axis, 0, 0, q, q_out, k, k_out, v, slot, pages, page, kc, vc, None)
    for bad in (dict(tokens=-1), dict(heads=-1), dict(kv=-1), dict(d=-1), dict(rot=-2), dict(rot=130), dict(rot=3), dict(dtype=0), dict(dtype=9), dict(axes=-1), dict(position=None),
                dict(frequency=None), dict(ldp=2), dict(position=P + 2), dict(axis=P + 1), dict(q=Z), dict(q_out=Z), dict(k=Z), dict(q=B.Heads(P + 1, 512, 128)), dict(q=B.Heads(P, -1, 128)),
                dict(q_out=B.Heads(P, 511, 128)), dict(q_out=B.Heads(P, 512, 127)), dict(q_out=B.Heads(P, 0, 128)), dict(k_out=B.Heads(P, 128, 128)),
                dict(slot=P, pages=2, page=16, v=Z, kc=cache, vc=cache), dict(slot=P, pages=2, page=16, v=H, kc=B.Cache(), vc=cache), dict(slot=P, pages=2, page=12, v=H, kc=cache, vc=cache),
                dict(slot=P, pages=2, page=16, v=H, kc=B.Cache(P, 4095, 256, 128), vc=cache), dict(slot=P, pages=2, page=16, v=H, kc=B.Cache(P, 0, 256, 128), vc=cache), dict(slot=P + 2, pages=0, page=16, v=H)):
        assert rc(**bad) == B.CSR5_EINVAL, bad
    assert rc(d=513, rot=0, q=B.Heads(P, 4000, 600), q_out=B.Heads(P, 4000, 600)) == B.CSR5_ERANGE and rc(tokens=2 ** 31 - 1, ldp=2 ** 31) == B.CSR5_ERANGE and rc(heads=70000) == B.CSR5_ERANGE
    assert rc(tokens=0) == B.CSR5_OK and rc(d=0, rot=0) == B.CSR5_OK and rc(heads=0, kv=0) == B.CSR5_OK


def test_attention_refusals(lib):
    K = B.Heads(P, 256, 128)

    def fwd(n=2, rows=3, k_rows=5, heads=4, kv=2, d=128, dtype=B.CSR5_DTYPE_BF16, qo=P, ko=P, scale=0.1, q=H, k=K, v=K, out=H, lse=P):
        return lib.csr5_attention(n, rows, k_rows, heads, kv, d, dtype, qo, ko, scale, 1, q, k, v, out, lse, None)
    common = (dict(n=-1), dict(rows=-1), dict(heads=-1), dict(kv=-1), dict(d=-1), dict(heads=3), dict(kv=0), dict(dtype=B.CSR5_DTYPE_F32), dict(dtype=B.CSR5_DTYPE_F64), dict(dtype=9), dict(scale=0.0),
              dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(q=Z), dict(qo=None), dict(qo=P + 2), dict(lse=P + 2), dict(q=B.Heads(P + 1, 512, 128)), dict(out=B.Heads(P, 128, 128)),
              dict(out=B.Heads(P, 512, 64)), dict(out=Z))
    for bad in (*common, dict(k_rows=-1), dict(k=Z), dict(v=Z), dict(ko=None), dict(ko=P + 1)):
        assert fwd(**bad) == B.CSR5_EINVAL, bad
    for far in (dict(d=129), dict(rows=2 ** 30 + 1), dict(k_rows=2 ** 30 + 1), dict(heads=65536, kv=1), dict(n=2 ** 31 - 1)):
        assert fwd(**far) == B.CSR5_ERANGE, far
    for nothing in (dict(n=0, qo=None, ko=None), dict(rows=0), dict(heads=0, kv=0)):
        assert fwd(**nothing) == B.CSR5_OK, nothing

    def back(n=2, rows=3, k_rows=5, heads=4, kv=2, d=128, scale=0.1, qo=P, ko=P, dout=H, q=H, k=K, v=K, out=H, lse=P, dq=H, dk=K, dv=K, ws=P, wsb=1 << 20):
        return lib.csr5_attention_backward(n, rows, k_rows, heads, kv, d, B.CSR5_DTYPE_F16, qo, ko, scale, 1, dout, q, k, v, out, lse, dq, dk, dv, ws, wsb, None)
    for bad in (dict(n=-1), dict(heads=3), dict(scale=0.0), dict(dout=Z), dict(q=Z), dict(k=Z), dict(v=Z), dict(out=Z), dict(lse=None), dict(lse=P + 1), dict(dq=Z), dict(dk=Z), dict(dv=Z), dict(qo=None), dict(ko=None),
                dict(dq=B.Heads(P, 0, 128)), dict(dk=B.Heads(P, 256, 0)), dict(dv=B.Heads(P, 200, 128)), dict(ws=P + 2)):
        assert back(**bad) == B.CSR5_EINVAL, bad
    need = B.csr5_attention_backward_workspace_bytes(3, 4)
    assert need > 0 and back(wsb=need - 1) == B.CSR5_ENOMEM and back(ws=None) == B.CSR5_ENOMEM and back(d=200) == B.CSR5_ERANGE
    assert B.csr5_attention_backward_workspace_bytes(0, 4) == 0 and back(n=0) == B.CSR5_OK and back(rows=0, k_rows=0, ws=None) == B.CSR5_OK

    cache = B.Cache(P, 4096, 256, 128)

    def paged(n=2, rows=3, heads=4, kv=2, d=128, dtype=B.CSR5_DTYPE_BF16, qo=P, length=P, table=P, width=6, ldt=6, pages=9, page=16, scale=0.1, q=H, k=cache, v=cache, out=H, lse=P, ws=None, wsb=0):
        return lib.csr5_attention_paged(n, rows, heads, kv, d, dtype, qo, length, table, width, ldt, pages, page, scale, q, k, v, out, lse, ws, wsb, None)
    for bad in (*common, dict(width=-1), dict(pages=-1), dict(page=0), dict(page=24), dict(table=None), dict(ldt=5), dict(length=None), dict(length=P + 2), dict(k=B.Cache()), dict(v=B.Cache()), dict(k=B.Cache(P, -1, 256, 128))):
        assert paged(**bad) == B.CSR5_EINVAL, bad
    assert paged(width=2 ** 27, ldt=2 ** 27) == B.CSR5_ERANGE and paged(n=0) == B.CSR5_OK and paged(rows=0) == B.CSR5_OK
    need = B.csr5_attention_paged_workspace_bytes(3, 4, 2, 128, 2, 400 * 16)
    assert need > 0 and paged(width=400, ldt=400) == B.CSR5_ENOMEM and paged(width=400, ldt=400, ws=P, wsb=need - 1) == B.CSR5_ENOMEM and paged(width=400, ldt=400, ws=P + 2, wsb=need) == B.CSR5_EINVAL
    assert B.csr5_attention_paged_workspace_bytes(3, 4, 3, 128, 2, 6400) == 0 and B.csr5_attention_paged_workspace_bytes(3, 4, 2, 128, 2, 2 ** 31) == 0


# ---------------------------------------------------------------------------------------------------------------------
# tensors
# ---------------------------------------------------------------------------------------------------------------------
def tensors(device="cuda:0", **shapes):
    with FakeTensorMode():
        return {name: torch.empty(*shape, dtype=dtype, device=device) for name, (dtype, *shape) in shapes.items()}


CALLS = {
    "csr5_pages": (dict(fresh=(I32, 3), length=(I32, 3), table=(I32, 3, 4), pool=(I32, 9), state=(I32, 2), offset=(I32, 4), position=(I32, 7), slot=(I32, 7), length_out=(I32, 3), state_out=(I32, 2)), dict(page=16)),
    "csr5_rotary": (dict(q=(BF16, 5, 4, 64), k=(BF16, 5, 2, 64), position=(I32, 2, 5), frequency=(F32, 32), q_out=(BF16, 5, 4, 64), k_out=(BF16, 5, 2, 64), axis=(I32, 32), v=(BF16, 5, 2, 64), slot=(I32, 5),
                         k_cache=(BF16, 3, 16, 2, 64), v_cache=(BF16, 3, 16, 2, 64)), {}),
    "csr5_attention": (dict(q=(F16, 5, 4, 64), k=(F16, 6, 2, 64), v=(F16, 6, 2, 64), q_offset=(I32, 3), k_offset=(I32, 3), out=(F16, 5, 4, 64), lse=(F32, 4, 5)), {}),
    "csr5_attention_backward": (dict(dout=(F16, 5, 4, 64), q=(F16, 5, 4, 64), k=(F16, 6, 2, 64), v=(F16, 6, 2, 64), out=(F16, 5, 4, 64), lse=(F32, 4, 5), q_offset=(I32, 3), k_offset=(I32, 3), dq=(F16, 5, 4, 64),
                                     dk=(F16, 6, 2, 64), dv=(F16, 6, 2, 64), workspace=(U8, 4096)), {}),
    "csr5_attention_paged": (dict(q=(BF16, 5, 4, 64), k_cache=(BF16, 3, 16, 2, 64), v_cache=(BF16, 3, 16, 2, 64), q_offset=(I32, 3), length=(I32, 2), table=(I32, 2, 4), out=(BF16, 5, 4, 64), workspace=(U8, 64),
                                  lse=(F32, 4, 5)), {}),
}
# dimensions that may have any size, as nothing else says what it is
FREE = {("csr5_pages", "table", 1), ("csr5_pages", "pool", 0), ("csr5_attention_backward", "workspace", 0), ("csr5_attention_paged", "workspace", 0), ("csr5_attention_paged", "table", 1), ("csr5_rotary", "position", 0),
        ("csr5_rotary", "frequency", 0), ("csr5_pages", "slot", 0)}


class Stream:
    cuda_stream = 4096

    def __init__(self, gpu):
        self.device_index = gpu


def run(call, here, more, gpu=0):
    return getattr(B, call)(**here, **more, stream=Stream(gpu), check=False)


@pytest.mark.parametrize("call", CALLS)
def test_tensors_that_do_not_fit_are_refused(lib, call):
    shapes, more = CALLS[call]
    here = tensors(**shapes)
    assert run(call, here, more) == B.CSR5_EINVAL               # everything fits: the library's own refusal of tensors without memory
    for name, (dtype, *shape) in shapes.items():
        other = {BF16: F32, F16: BF16, F32: I32, I32: F32, U8: I32}[dtype]
        with pytest.raises(ValueError):
            run(call, here | tensors(**{name: (other, *shape)}), more)
        for i in range(len(shape)):
            if (call, name, i) not in FREE:
                with pytest.raises(ValueError):
                    run(call, here | tensors(**{name: (dtype, *shape[:i], shape[i] - 1, *shape[i + 1:])}), more)
        if len(shape) > 2:
            with pytest.raises(ValueError, match="contiguous"):
                run(call, here | {name: tensors(t=(dtype, *shape[:-2], shape[-1], shape[-2]))["t"].transpose(-1, -2)}, more)
        with pytest.raises(ValueError, match="GPU"):
            run(call, here | tensors("cuda:1", **{name: (dtype, *shape)}), more)
        with pytest.raises(ValueError):
            run(call, here | {name: 4096}, more)
    with pytest.raises(ValueError, match="stream is one of GPU 1"):
        run(call, here, more, gpu=1)


def test_rotary_takes_a_cache_or_rows(lib):
    shapes, _ = CALLS["csr5_rotary"]
    here = tensors(**shapes)
    without = lambda *names: {k: v for k, v in here.items() if k not in names}  # noqa: E731
    for names in (("v",), ("slot",), ("k_cache",), ("v_cache", "slot")):
        with pytest.raises(ValueError, match="all or none"):
            run("csr5_rotary", without(*names), {})
    with pytest.raises(ValueError, match="k: needs"):
        run("csr5_rotary", without("k_out", "v", "slot", "k_cache", "v_cache"), {})
    with pytest.raises(ValueError, match="k: needed"):
        run("csr5_rotary", without("k") | {"k": None}, {})
    assert run("csr5_rotary", without("k_out"), {}) == B.CSR5_EINVAL
    with pytest.raises(ValueError, match="frequency"):
        run("csr5_rotary", here | tensors(frequency=(F32, 33)), {})
    with pytest.raises(ValueError):
        run("csr5_rotary", here | {"axis": 3}, {})


def test_scale_is_a_number(lib):
    shapes, _ = CALLS["csr5_attention"]
    here = tensors(**shapes)
    with pytest.raises(ValueError, match="scale"):
        run("csr5_attention", here, {"scale": "much"})


def test_scales_past_the_range_of_scores(lib):
    """Scores are held times log2 e: a scale that is past 2^128 in that is refused."""
    K = B.Heads(P, 256, 128)
    top = 2.0 ** 128 * (1 - 2.0 ** -24)
    past, below = top / 1.4426, top / 1.4427
    assert lib.csr5_attention(2, 3, 5, 4, 2, 128, B.CSR5_DTYPE_BF16, P, P, past, 1, H, K, K, H, P, None) == B.CSR5_EINVAL
    assert lib.csr5_attention(0, 3, 5, 4, 2, 128, B.CSR5_DTYPE_BF16, P, P, below, 1, H, K, K, H, P, None) == B.CSR5_OK
    assert lib.csr5_attention_backward(2, 3, 5, 4, 2, 128, B.CSR5_DTYPE_F16, P, P, past, 1, H, H, K, K, H, P, H, K, K, P, 1 << 20, None) == B.CSR5_EINVAL
    cache = B.Cache(P, 4096, 256, 128)
    assert lib.csr5_attention_paged(2, 3, 4, 2, 128, B.CSR5_DTYPE_BF16, P, P, P, 6, 6, 9, 16, past, H, cache, cache, H, P, None, 0, None) == B.CSR5_EINVAL


def test_heads_of_keys_without_queries(lib):
    K, N = B.Heads(P, 256, 128), B.Heads(None, 0, 0)
    back = lambda n, kv, ko=P, dk=K: lib.csr5_attention_backward(n, 3, 5, 0, kv, 128, B.CSR5_DTYPE_F16, P, ko, 0.1, 1, N, N, K, K, N, None, N, dk, K, None, 0, None)  # noqa: E731
    assert back(0, 2) == B.CSR5_OK and back(2, 2, ko=None) == B.CSR5_EINVAL and back(2, 2, dk=N) == B.CSR5_EINVAL and back(2, 65536, dk=B.Heads(P, 2 ** 24, 128)) == B.CSR5_ERANGE


def test_pages_outputs_that_overlap(lib):
    """No output of a step may be another array of it, or share a word with one: workgroups read the inputs while others write."""
    sizes = dict(fresh=3, length=3, table=12, pool=8, state=2, offset=4, position=5, slot=5, length_out=3, state_out=2)
    place, at = {}, P
    for name, words in sizes.items():
        place[name] = at
        at += 4 * words
    written = ("table", "pool", "offset", "position", "slot", "length_out", "state_out")

    def rc(**over):
        p = place | over
        return lib.csr5_pages(3, 4, 8, 16, 5, p["fresh"], p["length"], p["table"], 4, p["pool"], p["state"], p["offset"], p["position"], p["slot"], p["length_out"], p["state_out"], None)
    for name in written:
        for other in sizes:
            if other != name:
                for shift in (0, 4 * (sizes[other] - 1), -4 * (sizes[name] - 1)):
                    assert rc(**{name: place[other] + shift}) == B.CSR5_EINVAL, (name, other, shift)
