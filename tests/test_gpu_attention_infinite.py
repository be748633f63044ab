"""Attention and its gradients where keys or queries have one infinite value, as where a bias is carried as one more value of both: against the
definition in 64 bits, in which a score of -inf has weight 0, and a row of nothing else is one that sees no key (GPU).

In the definition STANDIN takes the place of -inf: it makes the score of such a key -1400 or less, whose weight is 0 in 64 bits as well.  The values of the
gradients that are sums of 0 times infinity are NaN and looked at apart."""
import math

import pytest
import torch

import attention_util as A
from layer_util import DEV
from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
STANDIN = -32768.0

# One sequence of 150 and others, which make up to 128, up to 320 and more workgroups of 128 rows.
SHAPES = {"four wavefronts to a row": ([(150, 150), (40, 40)], 4, 2), "two": ([(150, 150)] + [(40, 40)] * 20, 8, 8), "one": ([(150, 150)] + [(40, 40)] * 20, 32, 16)}
TYPES = [(BF16, 128), (F16, 64), (BF16, 80)]


class Case:
    """Random rows; the last value of queries is 1, of keys `last`.  `finite` is the same with STANDIN for -inf."""

    def __init__(self, name, dtype, d, last, gone=(), lost=()):
        lengths, heads, kv = SHAPES[name]
        gen = torch.Generator().manual_seed(21)
        self.qo, self.ko = A.pointer([a for a, _ in lengths]), A.pointer([b for _, b in lengths])
        rows = int(self.qo[-1])
        self.q, self.k, self.v, self.dout = (A.heads(gen, rows, h, d, dtype) for h in (heads, kv, kv, heads))
        self.q[..., -1], self.k[..., -1] = 1.0, last
        self.finite_q, self.finite_k, self.without = self.q.clone(), self.k.clone(), self.k.clone()
        for x, value in ((self.q, -math.inf), (self.finite_q, STANDIN)):
            x[list(lost), :, -1] = value
        for x, value in ((self.k, -math.inf), (self.finite_k, STANDIN)):
            x[list(gone), :, -1] = value
        self.without[list(gone)] = 0.0
        self.scale, self.shared, self.dtype, self.gone, self.lost = d ** -0.5, heads // kv, dtype, gone, lost

    def run(self, causal):
        q, k, v = self.q, self.k, self.v
        self.out, self.lse = torch.empty_like(q), torch.empty(q.shape[1], q.shape[0], device=DEV)
        B.csr5_attention(q, k, v, self.qo, self.ko, self.out, lse=self.lse, causal=causal)
        self.dq, self.dk, self.dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        space = torch.full((B.csr5_attention_backward_workspace_bytes(q.shape[0], q.shape[1]),), 255, dtype=torch.uint8, device=DEV)
        B.csr5_attention_backward(self.dout, q, k, v, self.out, self.lse, self.qo, self.ko, self.dq, self.dk, self.dv, space, causal=causal)
        # rows all of whose scores are -inf
        self.nothing = []
        for a, b in A.sequences(self.qo):
            for i in range(a, b):
                if i in self.lost or all(j in self.gone for j in range(a, i + 1 if causal else b)):
                    self.nothing.append(i)

    def check_forward(self, causal):
        nothing = torch.zeros(self.q.shape[0], dtype=torch.bool, device=DEV)
        nothing[self.nothing] = True
        for a, b in A.sequences(self.qo):
            rest = ~nothing[a:b]
            for h in range(self.q.shape[1]):
                one = lambda k: A.forward_of(self.finite_q[a:b, h].double(), k[a:b, h // self.shared].double(), self.v[a:b, h // self.shared].double(), b - a, b - a, self.scale, causal, self.dtype)  # noqa: E731,B023
                want, lse, slack, *_ = one(self.finite_k)
                lse_slack = one(self.without)[3]                # keys that do not count add no error
                A.bounded(self.out[a:b, h][rest], want[rest], slack[rest], self.dtype, ("out", a, h))
                A.bounded(self.lse[h, a:b][rest], lse[rest], lse_slack[rest], torch.float32, ("lse", a, h))
        assert bool((self.out[nothing] == 0).all()) and bool((self.lse[:, nothing] == -math.inf).all())

    def check_backward(self, causal, dq_nan, dk_nan):
        """dq_nan, dk_nan: rows and keys whose last value of dq and dk is a sum with 0 times infinity."""
        for a, b in A.sequences(self.qo):
            for hk in range(self.k.shape[1]):
                dk = dv = 0.0
                dk_slack = dv_slack = 0.0
                for h in range(hk * self.shared, (hk + 1) * self.shared):
                    (x, xs), (y, ys), (z, zs) = A.gradients_of(self.finite_q[a:b, h].double(), self.finite_k[a:b, hk].double(), self.v[a:b, hk].double(), self.dout[a:b, h].double(), self.out[a:b, h].double(),
                                                               self.lse[h, a:b].double(), self.scale, causal, self.dtype)
                    self.compare(self.dq[a:b, h], x, xs, [i - a for i in dq_nan if a <= i < b], ("dq", a, h))
                    dk, dk_slack, dv, dv_slack = dk + y, dk_slack + ys, dv + z, dv_slack + zs
                self.compare(self.dk[a:b, hk], dk, dk_slack, [i - a for i in dk_nan if a <= i < b], ("dk", a, hk))
                self.compare(self.dv[a:b, hk], dv, dv_slack, [], ("dv", a, hk))

    def compare(self, got, want, slack, nan, what):
        want = want.clone()
        want[nan, -1] = math.nan
        A.bounded(got, want, slack, self.dtype, what)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("name", list(SHAPES))
def test_keys_with_one_value_of_minus_infinity(name, dtype, d, causal):
    """In the tiles that the diagonal crosses, in those before them, and without a mask."""
    gone = [3, 37, 38, 70, 101, 149, 160]
    case = Case(name, dtype, d, 0.0, gone=gone)
    case.run(causal)
    assert not case.nothing
    case.check_forward(causal)
    case.check_backward(causal, [i for i in range(190) if (i >= 3 if i < 150 else i >= 160) or not causal], [])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("name", list(SHAPES))
def test_rows_that_see_such_keys_only(name, dtype, d, causal):
    """The first rows under the mask, and all of a sequence: they have no part in any gradient."""
    case = Case(name, dtype, d, 0.0, gone=[0, 1, 2, *range(150, 190)])
    case.run(causal)
    assert case.nothing == [*(range(3) if causal else []), *range(150, 190)]
    case.check_forward(causal)
    case.check_backward(causal, range(190), [])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("name", list(SHAPES))
def test_queries_with_one_value_of_minus_infinity(name, dtype, d, causal):
    """All their scores are -inf, in tiles with a mask and without."""
    case = Case(name, dtype, d, 0.5, lost=[2, 40, 101, 170])
    case.run(causal)
    assert case.nothing == [2, 40, 101, 170]
    case.check_forward(causal)
    case.check_backward(causal, [], [j for j in range(190) if (j <= 101 if j < 150 else j <= 170) or not causal])
