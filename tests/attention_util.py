"""Helpers of the attention's tests: inputs, the definitions in 64 bits, and error bounds.

Bounds.  A score, a sum of d products in 32 bits, is off by delta = (d + 8) * 2^-23 * scale * sum |q||k|.  So p = exp(score - c) is
off by eps_p = delta + 2^-21 + 2^-21 * (|score| + |c|) relatively: the score's error, an exponential within 2^-21, and its argument
in 32 bits; one below 2^-126, the smallest normal number of 32 bits, may be 0, which is 2^-126 absolutely.  One rounding to the type adds U (2^-8 in BF16, 2^-11 in F16; there also 2^-25 absolutely, below the smallest
normal number), and a sum of n terms n * 2^-23 of their magnitudes, joined parts and rescaling by factors within 2^-21 among them."""
import math

import torch

from layer_util import DEV, EPS32, U

TINY16 = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def bounded(got, ref, slack, dtype, what):
    """|got - ref| <= slack and one rounding of the result to `dtype`; what is not finite has to be the same."""
    got, ref, slack = got.double(), ref.double(), slack.double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(got[~fine].nan_to_num(nan=0.0), ref[~fine].nan_to_num(nan=0.0)), (what, "not finite")
    bound = U[dtype] * ref.abs() + slack * (1 + 2 * U[dtype]) + TINY16.get(dtype, 0.0)
    bad = fine & ~((got - ref).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), [int(i) for i in bad.nonzero()[0]], float(got[bad][0]), float(ref[bad][0]), float(bound[bad][0]))


def forward_of(q, k, v, m, n, scale, causal, dtype):
    """out, lse and their slack of one head of one sequence, q [m, d], k and v [n, d] in 64 bits.  Masked keys do not count, whatever they hold."""
    d = q.shape[1]
    j, i = torch.arange(n, device=q.device), torch.arange(m, device=q.device)[:, None]
    see = (j <= i + n - m) if causal else torch.ones(m, n, dtype=torch.bool, device=q.device)
    score = torch.where(see, scale * (q @ k.T), -math.inf)
    lse = torch.logsumexp(score, 1) if n else torch.full((m,), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.where(see, torch.exp(score - torch.where(lse == -math.inf, 0.0, lse)[:, None]), 0.0)
    out = weighted(p, v, see)
    size = torch.where(see, score.abs(), 0.0).amax(1) if n else torch.zeros(m, dtype=torch.float64, device=q.device)
    delta = torch.where(see, (d + 8) * EPS32 * scale * (q.abs() @ k.abs().T), 0.0).amax(1) if n else size
    eps = delta + 2.0 ** -21 + 2.0 ** -21 * 2 * size
    slack = (p @ v.nan_to_num(0.0, 0.0, 0.0).abs()) * (2 * eps + U[dtype] + 2 * (n + 64) * EPS32)[:, None]
    if dtype is torch.float16 and n:
        slack = slack + n * 2.0 ** -25 * v.nan_to_num(0.0, 0.0, 0.0).abs().amax()
    return out, lse, slack, delta + 2.0 ** -21 * (2 + lse.nan_to_num(0.0, 0.0, 0.0).abs() + 2 * size) + n * EPS32, p, see, eps


def weighted(p, v, see):
    """sum_j p_ij v_j over what is seen only, so that a masked value that is not finite does not show."""
    if bool(torch.isfinite(v).all()):
        return p @ v
    return torch.where(see[:, :, None], p[:, :, None] * v[None], 0.0).sum(1)


def sequences(offset):
    e = offset.tolist()
    return list(zip(e, e[1:]))


def check_forward(q, k, v, q_spans, k_spans, out, lse, scale, causal, what=""):
    """out [rows, heads, d] and lse [heads, rows] (or None) of packed keys against the definition."""
    dtype, shared = q.dtype, q.shape[1] // k.shape[1]
    for s, ((a, b), (c, e)) in enumerate(zip(q_spans, k_spans)):
        for h in range(q.shape[1]):
            want, want_lse, slack, lse_slack, *_ = forward_of(q[a:b, h].double(), k[c:e, h // shared].double(), v[c:e, h // shared].double(), b - a, e - c, scale, causal, dtype)
            bounded(out[a:b, h], want, slack, dtype, (what, "out", s, h))
            if lse is not None:
                bounded(lse[h, a:b], want_lse, lse_slack, torch.float32, (what, "lse", s, h))


def gradients_of(q, k, v, dout, out, lse, scale, causal, dtype):
    """dq, and this head's parts of dk and dv, with their slack: the formulas from `out` and `lse` as they are given."""
    (m, d), n = q.shape, k.shape[0]
    j, i = torch.arange(n, device=q.device), torch.arange(m, device=q.device)[:, None]
    see = (j <= i + n - m) if causal else torch.ones(m, n, dtype=torch.bool, device=q.device)
    score = torch.where(see, scale * (q @ k.T), -math.inf)
    base = torch.where(lse == -math.inf, 0.0, lse)[:, None]
    p = torch.where(see, torch.exp(score - base), 0.0)
    dp, delta = dout @ v.T, (dout * out).sum(1, keepdim=True)
    ds = torch.where(see, p * (dp - delta), 0.0)
    tiny = TINY16[dtype]
    eps = (d + 8) * EPS32 * scale * (q.abs() @ k.abs().T) + 2.0 ** -21 + 2.0 ** -21 * (torch.where(see, score.abs(), 0.0) + base.abs())
    eps_dp = (d + 8) * EPS32 * (dout.abs() @ v.abs().T + (dout.abs() * out.abs()).sum(1, keepdim=True))
    err_p = torch.where(see, p * (eps + U[dtype]) + tiny, 0.0)
    err_ds = torch.where(see, p * eps_dp * (1 + U[dtype]) + ds.abs() * (eps + U[dtype] + 2.0 ** -21) + tiny + 2.0 ** -126 * (dp - delta).abs(), 0.0)
    more = lambda count: (count + 64) * EPS32                           # noqa: E731  a sum's own error
    dq, dq_slack = scale * (ds @ k), scale * ((err_ds + more(n) * ds.abs()) @ k.abs())
    dk, dk_slack = scale * (ds.T @ q), scale * ((err_ds + more(m * 16) * ds.abs()).T @ q.abs())
    dv, dv_slack = p.T @ dout, (err_p + more(m * 16) * p).T @ dout.abs()
    return (dq, dq_slack), (dk, dk_slack), (dv, dv_slack)


def check_backward(q, k, v, dout, out, lse, q_spans, k_spans, dq, dk, dv, scale, causal, what=""):
    dtype, shared = q.dtype, q.shape[1] // k.shape[1]
    for s, ((a, b), (c, e)) in enumerate(zip(q_spans, k_spans)):
        for hk in range(k.shape[1]):
            keys, values = k[c:e, hk].double(), v[c:e, hk].double()
            sums = [torch.zeros(e - c, q.shape[2], dtype=torch.float64, device=q.device) for _ in range(4)]
            for h in range(hk * shared, (hk + 1) * shared):
                (x, xs), *rest = gradients_of(q[a:b, h].double(), keys, values, dout[a:b, h].double(), out[a:b, h].double(), lse[h, a:b].double(), scale, causal, dtype)
                bounded(dq[a:b, h], x, xs, dtype, (what, "dq", s, h))
                sums = [t + u for t, u in zip(sums, [u for pair in rest for u in pair])]
            bounded(dk[c:e, hk], sums[0], sums[1], dtype, (what, "dk", s, hk))
            bounded(dv[c:e, hk], sums[2], sums[3], dtype, (what, "dv", s, hk))


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def heads(gen, rows, heads_, d, dtype, layout="plain", scale=1.0, fill=None):
    """Random rows of heads.  layout: "plain"; "beside": heads of a wider row, as of one product for queries, keys and values; "major":
    heads outside, rows inside; "odd": at an odd address with odd strides.  What surrounds a view is NaN.  fill: that value instead of random ones."""
    v = (torch.randn(rows, heads_, d, generator=gen) * scale).to(dtype) if fill is None else torch.full((rows, heads_, d), fill, dtype=dtype)
    if layout == "plain":
        return v.to(DEV)
    if layout == "beside":
        big = torch.full((rows + 1, heads_ + 3, -(-d // 8) * 8 + 8), math.nan, dtype=dtype, device=DEV)
        view = big[:rows, 2:2 + heads_, :d]
    elif layout == "major":
        big = torch.full((heads_, rows + 2, -(-d // 8) * 8), math.nan, dtype=dtype, device=DEV)
        view = big[:, 1:1 + rows, :d].transpose(0, 1)
    else:
        assert layout == "odd"
        big = torch.full((rows + 1, heads_ + 1, d + 3 + d % 2), math.nan, dtype=dtype, device=DEV)
        view = big[:rows, :heads_, 1:1 + d]
    view.copy_(v)
    return view


def whole(view):
    """The values of the array that a view of heads() lies in."""
    return torch.as_strided(view, (view.untyped_storage().nbytes() // view.element_size(),), (1,), 0)


def pointer(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device=DEV)


def paged(gen, k, v, k_spans, page, layout="plain", spare=3, width=None):
    """Packed keys and values [rows, kv_heads, d] scattered over the pages of a cache that is NaN elsewhere: k_cache, v_cache, table, length."""
    lengths = [b - a for a, b in k_spans]
    held = [-(-n // page) for n in lengths]
    pages, kv, d = sum(held) + spare, k.shape[1], k.shape[2]
    order = torch.randperm(pages, generator=gen).tolist()
    width = max(held + [1]) if width is None else width
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)

    def empty():
        if layout == "plain":
            return torch.full((pages, page, kv, d), math.nan, dtype=k.dtype, device=DEV)
        if layout == "major":                                            # heads outside the tokens of a page
            return torch.full((pages, kv, page, d), math.nan, dtype=k.dtype, device=DEV).transpose(1, 2)
        return torch.full((pages, page, kv, d + 3 + d % 2), math.nan, dtype=k.dtype, device=DEV)[..., 1:1 + d]
    k_cache, v_cache = empty(), empty()
    for s, (a, b) in enumerate(k_spans):
        for p in range(held[s]):
            table[s, p] = order.pop()
            rows = min(page, b - a - p * page)
            k_cache[int(table[s, p]), :rows] = k[a + p * page:a + p * page + rows]
            v_cache[int(table[s, p]), :rows] = v[a + p * page:a + p * page + rows]
    return k_cache, v_cache, table.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------------------------------------------------------------
# Which kernel a call takes: the library's rule (plan_of in attention.hip, csr5_attention_backward), so that a test can say which one it means
# ---------------------------------------------------------------------------------------------------------------------
def sides(rows, n, heads_, kv):
    """Wavefronts that share a row's keys, in the kernels for many rows."""
    groups = ((rows * (heads_ // kv) >> 7) + n) * kv
    return 4 if groups <= 128 else 2 if groups <= 320 else 1


def forward_kernel(rows, n, heads_, kv):
    each = -(-rows // n) * (heads_ // kv)
    return ("few", 1 if each <= 16 else 2 if each <= 32 else 4) if each <= 64 else ("many", sides(rows, n, heads_, kv))


def is_split(rows, n, heads_, kv, most):
    """Whether the attention over a cache takes its keys by parts; most: what the table could hold."""
    kind, size = forward_kernel(rows, n, heads_, kv)
    shift = {("few", 1): 4, ("few", 2): 5, ("few", 4): 6, ("many", 1): 7, ("many", 2): 6, ("many", 4): 5}[kind, size]
    groups = ((rows * (heads_ // kv) >> shift) + n) * kv
    return max(-(-(most * groups // 2048) // 128) * 128, 256 if kind == "few" else 512) < most
