"""Rows at addresses of 16 bytes that are not multiples of 32 give what aligned rows give, in every type."""
import pytest
import torch

from layer_util import DEV
from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]
ids = lambda t: str(t).replace("torch.", "")  # noqa: E731


def calls(rows, n, dtype, at, seed):
    """Every call that moves rows about, of rows that begin `at` values into wider ones; what it wrote."""
    g = torch.Generator().manual_seed(seed)

    def wide(r):
        big = torch.zeros(r, n + 16, dtype=dtype, device=DEV)
        big[:, at:at + n] = torch.randn(r, n, generator=g).to(dtype)
        return big[:, at:at + n]

    x, residual, dy, z = wide(rows), wide(rows), wide(rows), wide(3 * rows)
    gain = wide(1)[0]
    place, weight = torch.randperm(3 * rows, generator=g).int().view(rows, 3).to(DEV), torch.rand(rows, 3, generator=g).to(DEV)
    h, y, s, dh, dz = wide(rows), wide(rows), wide(rows), wide(rows), wide(3 * rows)
    q, scale, rstd = torch.empty(rows, n + 16, dtype=torch.uint8, device=DEV)[:, 8:8 + n], torch.empty(rows, -(-n // 128), device=DEV), torch.empty(rows, device=DEV)
    dgain, dweight = torch.empty(n, device=DEV), torch.empty(rows, 3, device=DEV)
    B.csr5_rmsnorm(x, gain, 1e-6, residual=residual, h=h, y=y, rstd=rstd)
    B.csr5_rmsnorm_backward(h, gain, rstd, dy, dh, dgain, torch.empty(B.csr5_rmsnorm_workspace_bytes(rows, n), dtype=torch.uint8, device=DEV), residual_grad=residual)
    B.csr5_quantise(x, q, scale)
    B.csr5_combine(z, place, s, weight=weight, residual=residual)
    B.csr5_combine_backward(dy, z, place, weight, dz, dweight)
    return [t.clone() for t in (h, y, rstd, dh, dgain, q, scale, s, dz, dweight)]


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("n", [8, 136, 4096, 12000])
def test_16_bytes_are_enough(n, dtype):
    narrow = 16 // torch.empty((), dtype=dtype).element_size()
    for i, (a, b) in enumerate(zip(calls(37, n, dtype, 0, n), calls(37, n, dtype, narrow, n))):
        assert torch.equal(a, b), i
