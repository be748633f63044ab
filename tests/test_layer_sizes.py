"""Products that take more threads than a launch has are refused on the host (dummy addresses, no GPU)."""
import pytest

from paper_1503_05032_amd import binding as B

P = 4096        # a plausible, aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    return B.load()


@pytest.mark.parametrize("groups,rows", [(2 ** 24, 2 ** 24), (2 ** 27, 8)])
@pytest.mark.parametrize("n,k", [(32, 16), (33, 17)])          # 16-byte rows; the plain kernel
def test_too_many_threads(lib, groups, rows, n, k):
    assert lib.csr5_grouped_gemm(groups, rows, n, k, 2, P, P, rows, k, None, P, k, n * k, P, n, None) == B.CSR5_ERANGE
    assert lib.csr5_grouped_gemm_dx(groups, rows, n, k, 2, P, P, n, P, k, n * k, P, k, None) == B.CSR5_ERANGE
    assert lib.csr5_grouped_gemm_dw(groups, rows, n, k, 2, P, P, n, P, rows, k, None, P, k, n * k, None) == B.CSR5_ERANGE
    assert lib.csr5_grouped_gemm_f8(groups, rows, n, k, 2, P, P, rows, k, P, 1, 1, None, P, k, n * k, P, 128, 1, 1, 1, P, n, None) == B.CSR5_ERANGE
