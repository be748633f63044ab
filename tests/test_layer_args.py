"""Refusals of the calls of a layer of experts: on the host, before anything is launched (dummy addresses, no GPU)."""
import os

import pytest
import torch

from paper_1503_05032_amd import binding as B
from paper_1503_05032_amd import build as libbuild

P = 4096        # a plausible, aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        libbuild.build(verbose=False)
    return B.load()


def test_route_refusals(lib):
    def rc(tokens=4, experts=8, k=2, dtype=B.CSR5_DTYPE_F32, logits=P, ld=8, expert=P, weight=P, offset=P, source=P, place=P, ws=P, wsb=1 << 20):
        return lib.csr5_route(tokens, experts, k, dtype, logits, ld, expert, weight, offset, source, place, ws, wsb, None)
    assert rc(tokens=-1) == B.CSR5_EINVAL and rc(dtype=B.CSR5_DTYPE_F64) == B.CSR5_EINVAL and rc(dtype=9) == B.CSR5_EINVAL
    assert rc(k=0) == B.CSR5_ERANGE and rc(k=9) == B.CSR5_ERANGE and rc(experts=1025, ld=1025) == B.CSR5_ERANGE
    assert rc(experts=64, k=33, ld=64) == B.CSR5_ERANGE and rc(tokens=2 ** 31 - 1) == B.CSR5_ERANGE
    assert rc(ld=7) == B.CSR5_EINVAL and rc(logits=None) == B.CSR5_EINVAL and rc(logits=P + 2) == B.CSR5_EINVAL
    for name in ("expert", "weight", "offset", "source", "place"):
        assert rc(**{name: None}) == B.CSR5_EINVAL, name
    need = B.csr5_route_workspace_bytes(5000, 64, 4)
    assert need > 0 and B.csr5_route_workspace_bytes(8, 64, 4) == 0 and B.csr5_route_workspace_bytes(8, 2000, 4) == 0
    assert rc(tokens=5000, experts=64, k=4, ld=64, wsb=need - 1) == B.CSR5_ENOMEM
    assert rc(tokens=5000, experts=64, k=4, ld=64, ws=None) == B.CSR5_ENOMEM
    assert rc(tokens=5000, experts=64, k=4, ld=64, ws=P + 1, wsb=need) == B.CSR5_EINVAL
    back = lambda tokens=4, k=2, w=P, ld=8: lib.csr5_route_backward(tokens, 8, k, 1, P, w, P, P, ld, None)  # noqa: E731
    assert back(k=9) == B.CSR5_ERANGE and back(w=None) == B.CSR5_EINVAL and back(ld=1) == B.CSR5_EINVAL and back(tokens=0) == B.CSR5_OK


def test_combine_refusals(lib):
    def rc(tokens=4, k=2, rows=8, n=16, dtype=2, z=P, ldz=16, place=P, res=None, ldr=0, y=P, ldy=16):
        return lib.csr5_combine(tokens, k, rows, n, dtype, z, ldz, place, P, res, ldr, y, ldy, None)
    assert rc(k=-1) == B.CSR5_EINVAL and rc(dtype=0) == B.CSR5_EINVAL and rc(z=None) == B.CSR5_EINVAL and rc(place=None) == B.CSR5_EINVAL
    assert rc(ldz=15) == B.CSR5_EINVAL and rc(ldy=15) == B.CSR5_EINVAL and rc(res=P, ldr=3) == B.CSR5_EINVAL and rc(y=P + 1) == B.CSR5_EINVAL
    assert rc(tokens=2 ** 30, k=4) == B.CSR5_ERANGE and rc(tokens=0) == B.CSR5_OK and rc(n=0) == B.CSR5_OK
    back = lambda dz=P, w=P, lddz=16, tokens=4: lib.csr5_combine_backward(tokens, 2, 8, 16, 2, P, 16, P, 16, P, w, dz, lddz, P, None)  # noqa: E731
    assert back(dz=None) == B.CSR5_EINVAL and back(w=None) == B.CSR5_EINVAL and back(lddz=8) == B.CSR5_EINVAL and back(tokens=0) == B.CSR5_OK


def test_product_refusals(lib):
    def fwd(groups=2, rows=8, n=16, k=32, dtype=2, offset=P, x=P, x_rows=8, ldx=32, source=None, w=P, ldw=32, y=P, ldy=16):
        return lib.csr5_grouped_gemm(groups, rows, n, k, dtype, offset, x, x_rows, ldx, source, w, ldw, 512, y, ldy, None)
    for bad in (dict(groups=-1), dict(rows=-1), dict(n=-1), dict(k=-1), dict(dtype=1), dict(dtype=7), dict(offset=None), dict(offset=P + 2), dict(x=None),
                dict(x_rows=7), dict(x_rows=-1, source=P), dict(ldx=31), dict(ldw=31), dict(ldy=15), dict(w=None), dict(y=None), dict(x=P + 1), dict(source=P + 1)):
        assert fwd(**bad) == B.CSR5_EINVAL, bad
    for nothing in (dict(groups=0, offset=None), dict(rows=0), dict(n=0)):
        assert fwd(**nothing) == B.CSR5_OK, nothing
    dx = lambda dtype=2, dy=P, ldd=32: lib.csr5_grouped_gemm_dx(2, 8, 16, 32, dtype, P, dy, 16, P, 32, 512, P, ldd, None)  # noqa: E731
    assert dx(dtype=1) == B.CSR5_EINVAL and dx(dy=None) == B.CSR5_EINVAL and dx(ldd=31) == B.CSR5_EINVAL
    dw = lambda x_rows=8, lddw=32, dw=P: lib.csr5_grouped_gemm_dw(2, 8, 16, 32, 2, P, P, 16, P, x_rows, 32, None, dw, lddw, 512, None)  # noqa: E731
    assert dw(x_rows=3) == B.CSR5_EINVAL and dw(lddw=31) == B.CSR5_EINVAL and dw(dw=None) == B.CSR5_EINVAL


def test_f8_refusals(lib):
    def f8(m=8, n=16, k=32, dtype=2, x=P, ldx=32, xs=P, w=P, ldw=32, ws=P, w_rows=128, y=P, ldy=16):
        return lib.csr5_gemm_f8(m, n, k, dtype, x, ldx, xs, 1, 1, w, ldw, ws, w_rows, 1, 1, y, ldy, None)
    for bad in (dict(m=-1), dict(dtype=0), dict(x=None), dict(xs=None), dict(ws=None), dict(xs=P + 2), dict(w_rows=64), dict(ldx=31), dict(ldw=31),
                dict(ldy=15), dict(y=P + 1)):
        assert f8(**bad) == B.CSR5_EINVAL, bad
    assert f8(m=0) == B.CSR5_OK and f8(n=0) == B.CSR5_OK
    grouped = lambda w_rows=128, offset=P: lib.csr5_grouped_gemm_f8(2, 8, 16, 32, 2, offset, P, 8, 32, P, 1, 1, None, P, 32, 512, P, w_rows, 1, 1, 1, P, 16, None)  # noqa: E731
    assert grouped(w_rows=2) == B.CSR5_EINVAL and grouped(offset=None) == B.CSR5_EINVAL
    quantise = lambda rows=4, block=1, dtype=2, scale=P, ldq=16: lib.csr5_quantise(rows, 16, block, dtype, P, 16, P, ldq, scale, 1, 1, None)  # noqa: E731
    assert quantise(rows=-1) == B.CSR5_EINVAL and quantise(block=64) == B.CSR5_EINVAL and quantise(dtype=0) == B.CSR5_EINVAL
    assert quantise(scale=None) == B.CSR5_EINVAL and quantise(ldq=8) == B.CSR5_EINVAL and quantise(rows=0) == B.CSR5_OK


def test_norm_refusals(lib):
    def norm(rows=4, n=16, dtype=2, x=P, ldx=16, res=None, ldr=0, h=None, y=P, ldy=16, q=None, scale=None):
        return lib.csr5_rmsnorm(rows, n, dtype, x, ldx, res, ldr, P, 1e-6, h, 16, y, ldy, q, 16, scale, 1, 1, None, None)
    for bad in (dict(rows=-1), dict(dtype=0), dict(x=None), dict(ldx=15), dict(res=P, ldr=4), dict(ldy=3), dict(q=P), dict(x=P + 1)):
        assert norm(**bad) == B.CSR5_EINVAL, bad
    assert norm(n=B.CSR5_NORM_MAX_N + 1, ldx=1 << 20, ldy=1 << 20) == B.CSR5_ERANGE and norm(rows=0) == B.CSR5_OK and norm(n=0) == B.CSR5_OK
    need = B.csr5_rmsnorm_workspace_bytes(4, 16)
    assert need > 0 and B.csr5_rmsnorm_workspace_bytes(4, B.CSR5_NORM_MAX_N + 1) == 0
    back = lambda wsb=need, ws=P, rstd=P, ld=16: lib.csr5_rmsnorm_backward(4, 16, 2, P, ld, P, rstd, P, 16, None, 0, P, 16, P, ws, wsb, None)  # noqa: E731
    assert back(wsb=need - 1) == B.CSR5_ENOMEM and back(ws=None) == B.CSR5_ENOMEM and back(rstd=None) == B.CSR5_EINVAL and back(ld=8) == B.CSR5_EINVAL


def test_tensors_that_do_not_fit_are_refused():
    z = torch.zeros
    with pytest.raises(ValueError, match="dtype"):
        B.csr5_rmsnorm(z(2, 8, dtype=torch.float64), None, 1e-6)
    with pytest.raises(ValueError, match="GPU"):
        B.csr5_rmsnorm(z(2, 8), None, 1e-6)
    with pytest.raises(ValueError, match="both"):
        B.csr5_rmsnorm(z(2, 8), None, 1e-6, q=z(2, 8, dtype=torch.uint8))
    with pytest.raises(ValueError, match="shape"):
        B._matrix(z(2, 8), torch.float32, 2, 9, "x")
    with pytest.raises(ValueError, match="dtype"):
        B._matrix(z(2, 8), None, 2, 8, "q")
    with pytest.raises(ValueError, match="shape"):
        B._experts(z(2, 8, 4), torch.float32, 2, 8, 5, "w")
    with pytest.raises(ValueError, match="needs"):
        B._source(None, 5, 4)


def test_sizes_that_32_bits_do_not_count(lib):
    big = 2 ** 31 - 1
    assert lib.csr5_combine(1, 1, 1, big, 2, P, big, P, P, None, 0, P, big, None) == B.CSR5_ERANGE
    assert lib.csr5_combine_backward(1, 1, 1, big, 2, P, big, P, big, P, P, P, big, P, None) == B.CSR5_ERANGE
    for rows, n in ((big, 16), (4, big)):
        assert lib.csr5_quantise(rows, n, 1, 2, P, n, P, n, P, 1, 1, None) == B.CSR5_ERANGE
    for groups, rows, n, k in ((big, 8, 16, 32), (2, big, 16, 32), (2, 8, big, 32), (2, 8, 16, big)):
        assert lib.csr5_grouped_gemm(groups, rows, n, k, 2, P, P, rows, k, None, P, k, 512, P, n, None) == B.CSR5_ERANGE
        assert lib.csr5_grouped_gemm_dx(groups, rows, n, k, 2, P, P, n, P, k, 512, P, k, None) == B.CSR5_ERANGE
        assert lib.csr5_grouped_gemm_dw(groups, rows, n, k, 2, P, P, n, P, rows, k, None, P, k, 512, None) == B.CSR5_ERANGE
        assert lib.csr5_grouped_gemm_f8(groups, rows, n, k, 2, P, P, rows, k, P, 1, 1, None, P, k, 512, P, 128, 1, 1, 1, P, n, None) == B.CSR5_ERANGE
    for m, n, k in ((big, 16, 32), (8, big, 32), (8, 16, big)):
        assert lib.csr5_gemm_f8(m, n, k, 2, P, k, P, 1, 1, P, k, P, 128, 1, 1, P, n, None) == B.CSR5_ERANGE
