"""What a layer of experts in a large language model has libcsr5 do, as measurable cases.

The router's choice is a sparse matrix of tokens x experts with k entries per row.  Grouped by expert it is that matrix
in CSR (`offset` is its row pointer), the experts' products are a block-sparse product over those offsets, and the way
back to the tokens is a sparse times dense product.  Kinds of case, each ONE pass through an operator by the calls that
`paper_1503_05032_amd.binding` offers:

  "norm"          root-mean-square norm of x + residual, normalised output in 16 bits or in 8 bits with scales
  "norm_back"     its gradients
  "route"         the k largest logits of each token, their softmax, the grouping by expert
  "combine_train" the weighted sum of the experts' rows per token, and the gradients down to the logits
  "grouped"       products grouped by expert over ragged groups
  "grouped_back"  their gradients with respect to the rows and to the weights
  "f8"            product in 8-bit floating point (e4m3) with a scale for each block of 128, from quantised or 16-bit rows
  "f8_grouped"    the same, grouped by expert

Sizes are generic ones of such layers: hidden sizes of 1 to 8 thousand, 8 to 256 experts, 1 to 8 of them per token, and
from a few tokens (one step of serving) to some ten thousand (a prompt, a training step).
"""
import math

import torch

own = False                     # False: `run` computes the plain forms; True: it calls the library

DEVICE = "cuda:0"
BLOCK = 128                     # values that share a scale
F8_MAX = 448.0                  # largest finite e4m3 value
SCALE_MIN = 2.0 ** -126         # smallest scale: a block of zeros has it
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------
def listed():
    cases = {
        # one step of serving for 16 sequences: the smallest call, all latency; 8-bit output for the next product
        "norm_decode": dict(kind="norm", rows=16, n=4096, dtype="bf16", out="f8"),
        # a long prompt, 8-bit output
        "norm_prefill": dict(kind="norm", rows=16384, n=4096, dtype="bf16", out="f8"),
        # a training step's way back, an odd number of rows, half precision
        "norm_back": dict(kind="norm_back", rows=8191, n=2560, dtype="f16"),
        # routing one step of serving: many experts, logits in single precision
        "route_decode": dict(kind="route", tokens=24, experts=128, k=8, dtype="f32", masked=False),
        # routing a long prompt with padding and experts that are out of service
        "route_prefill": dict(kind="route", tokens=32768, experts=256, k=8, dtype="bf16", masked=True),
        # training: back from the experts' rows to the tokens, and the gradients of rows, weights and logits
        "combine_train": dict(kind="combine_train", tokens=8192, experts=64, k=4, n=2048, dtype="bf16"),
        # one step of serving: one or two rows per expert, the weights are read once
        "grouped_decode": dict(kind="grouped", tokens=16, experts=64, k=4, n=1536, depth=2048, dtype="bf16"),
        # a long prompt: the largest product in 16 bits
        "grouped_prefill": dict(kind="grouped", tokens=16384, experts=32, k=4, n=2816, depth=2048, dtype="bf16"),
        # a training step's way back over ragged groups, odd number of tokens
        "grouped_back": dict(kind="grouped_back", tokens=8191, experts=16, k=2, n=2048, depth=2304, dtype="bf16"),
        # serving a few sequences in 8 bits, rows quantised by what came before
        "f8_decode": dict(kind="f8", rows=8, n=8192, depth=4096, w_rows=128, dtype="bf16", quantise=False),
        # a prompt in 8 bits from 16-bit rows: quantise, multiply
        "f8_prefill": dict(kind="f8", rows=8000, n=8192, depth=4096, w_rows=128, dtype="bf16", quantise=True),
        # a prompt through the experts in 8 bits, ragged groups
        "f8_grouped": dict(kind="f8_grouped", tokens=4096, experts=64, k=8, n=2048, depth=2048, dtype="bf16"),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _tokens(rng, lo, hi):
    """Any number of tokens, mostly odd: what prompts have."""
    return _log_int(rng, lo, hi) | 1


def _size(rng, lo, hi):
    """A hidden size: an odd multiple of 128, or of 16 for one in four."""
    unit = rng.choice([128, 128, 128, 16])
    return unit * (_log_int(rng, lo // unit, hi // unit) | 1)


def draw(rng):
    kind = rng.choice(["norm", "norm_back", "route", "combine_train", "grouped", "grouped", "grouped_back", "f8", "f8", "f8_grouped"])
    half = rng.choice(["bf16", "bf16", "f16"])
    if kind == "norm":
        return dict(kind=kind, rows=_tokens(rng, 1, 12000), n=_size(rng, 1000, 8000), dtype=half, out=rng.choice(["f8", "f8", "same"]))
    if kind == "norm_back":
        return dict(kind=kind, rows=_tokens(rng, 64, 8000), n=_size(rng, 1000, 6000), dtype=half)
    if kind in ("route", "combine_train"):
        experts = rng.choice([8, 16, 60, 64, 128, 160, 256])
        k = rng.choice([1, 2, 4, 6, 8])
        if kind == "route":
            return dict(kind=kind, tokens=_tokens(rng, 1, 40000), experts=experts, k=k, dtype=rng.choice(["bf16", "f32"]), masked=rng.random() < 0.5)
        return dict(kind=kind, tokens=_tokens(rng, 64, 24000 // k), experts=experts, k=k, n=_size(rng, 1000, 5000), dtype=half)
    n, depth = _size(rng, 1000, 5000), _size(rng, 1000, 5000)
    if kind == "f8":
        rows = _tokens(rng, 1, 8000) if rng.random() < 0.6 else _tokens(rng, 1, 64)
        quantise = rng.random() < 0.5
        w_rows = rng.choice([128, 128, 1])
        return dict(kind=kind, rows=rows, n=n, depth=depth, w_rows=w_rows, dtype=half, quantise=quantise)
    experts = rng.choice([8, 16, 24, 32, 60, 64])
    k = rng.choice([1, 2, 4, 8])
    most = 1.2e11 / (n * depth)                     # rows in all: a drawn case stays under the largest listed one
    tokens = _tokens(rng, 64 if kind == "grouped_back" else 1, max(128, int(most / k)))
    return dict(kind=kind, tokens=tokens, experts=experts, k=k, n=n, depth=depth, dtype=half)


# ---------------------------------------------------------------------------------------------------------------
# inputs, drawn on the GPU
# ---------------------------------------------------------------------------------------------------------------
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _logits(c, g):
    """Logits of a router in use: experts of uneven popularity; masked: 1 of 16 experts out of service, 1 token of 32 padding."""
    t, e = c["tokens"], c["experts"]
    out = _randn(g, t, e) * 1.5 + _randn(g, e) * 0.7
    if c.get("masked"):
        out[:, e - e // 16:] = -math.inf
        out[t - t // 32:] = -math.inf
    return out


def _plan(c, g):
    """The grouping of a router's choice, and the largest group."""
    t, e, k = c["tokens"], c["experts"], c["k"]
    weight, expert = torch.topk(torch.softmax(_logits(c, g), 1), k, dim=1)
    weight = weight / weight.sum(1, keepdim=True)
    order = torch.sort(expert.reshape(-1), stable=True).indices
    count = torch.bincount(expert.reshape(-1), minlength=e)
    offset = torch.zeros(e + 1, dtype=torch.int32, device=DEVICE)
    offset[1:] = torch.cumsum(count, 0)
    place = torch.empty_like(order)
    place[order] = torch.arange(t * k, device=DEVICE)
    return dict(expert=expert.int(), weight=weight, offset=offset, source=(order // k).int(), place=place.view(t, k).int(), most=int(count.max()))


def _per_row(scale, rows):
    """Scales per 128 rows as scales of each of the rows."""
    return scale.repeat_interleave(BLOCK, -2)[..., :rows, :]


def _quantised(x, block_rows):
    """e4m3 values and scales of x[..., rows, n] per block of block_rows x 128, in float32 arithmetic."""
    rows, n = x.shape[-2:]
    pad = torch.nn.functional.pad(x.float(), (0, -n % BLOCK, 0, -rows % block_rows))
    tiles = pad.unflatten(-1, (-1, BLOCK)).unflatten(-3, (-1, block_rows))
    scale = (tiles.abs().amax((-3, -1)) / F8_MAX).clamp(min=SCALE_MIN)
    q = (tiles / scale[..., None, :, None]).clamp(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn)
    return q.flatten(-2, -1).flatten(-3, -2)[..., :rows, :n].contiguous(), scale


def _blocks(n):
    return -(-n // BLOCK)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    kind, dt = c["kind"], TYPES[c["dtype"]]
    s = dict(kind=kind, case=c)
    empty = lambda *shape, dtype=dt: torch.empty(*shape, dtype=dtype, device=DEVICE)  # noqa: E731
    if kind in ("norm", "norm_back"):
        r, n = c["rows"], c["n"]
        s.update(gain=(1 + 0.2 * _randn(g, n)).to(dt))
        if kind == "norm":
            # a residual stream has channels that are much larger than the rest
            wide = 1 + 9 * (torch.rand(n, generator=g, device=DEVICE) < 0.01)
            s.update(x=_randn(g, r, n).to(dt), residual=(2 * _randn(g, r, n) * wide).to(dt), h=empty(r, n), rstd=empty(r, dtype=torch.float32))
            if c["out"] == "f8":
                s.update(q=empty(r, n, dtype=torch.float8_e4m3fn), scale=empty(r, _blocks(n), dtype=torch.float32))
            else:
                s.update(y=empty(r, n))
        else:
            h = (2 * _randn(g, r, n)).to(dt)
            s.update(h=h, rstd=torch.rsqrt(h.float().square().mean(1) + EPS), dy=_randn(g, r, n).to(dt), residual_grad=_randn(g, r, n).to(dt),
                     dh=empty(r, n), dgain=empty(n, dtype=torch.float32))
        return s
    if kind == "route":
        t, e, k = c["tokens"], c["experts"], c["k"]
        i32 = torch.int32
        s.update(logits=_logits(c, g).to(dt), expert=empty(t, k, dtype=i32), weight=empty(t, k, dtype=torch.float32), offset=empty(e + 1, dtype=i32),
                 source=empty(t * k, dtype=i32), place=empty(t, k, dtype=i32))
        return s
    if kind == "f8":
        m, n, d = c["rows"], c["n"], c["depth"]
        w8, w_scale = _quantised(_randn(g, n, d) / math.sqrt(d), c["w_rows"])
        s.update(w8=w8, w_scale=w_scale, y=empty(m, n))
        x = _randn(g, m, d)
        if c["quantise"]:
            s.update(x=x.to(dt), x8=empty(m, d, dtype=torch.float8_e4m3fn), x_scale=empty(m, _blocks(d), dtype=torch.float32))
        else:
            x8, x_scale = _quantised(x, 1)
            s.update(x8=x8, x_scale=x_scale)
        return s
    plan = _plan(c, g)
    s.update(plan)
    t, p, e, n = c["tokens"], c["tokens"] * c["k"], c["experts"], c["n"]
    if kind == "combine_train":
        f32 = torch.float32
        s.update(z=_randn(g, p, n).to(dt), dy=_randn(g, t, n).to(dt), y=empty(t, n), dz=empty(p, n), dweight=empty(t, c["k"], dtype=f32),
                 dlogits=empty(t, e))
        return s
    d = c["depth"]
    w = _randn(g, e, n, d) / math.sqrt(d)
    if kind == "f8_grouped":
        w8, w_scale = _quantised(w, BLOCK)
        x8, x_scale = _quantised(_randn(g, t, d), 1)
        s.update(w8=w8, w_scale=w_scale, x8=x8, x_scale=x_scale, y=empty(p, n))
        return s
    s.update(w=w.to(dt), x=_randn(g, t, d).to(dt), y=empty(p, n))
    if kind == "grouped_back":
        s.update(dy=_randn(g, p, n).to(dt), dx=empty(p, d), dw=empty(e, n, d))
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    return (_kernels if own else _plain)(s)


_library = None


def _kernels(s):
    global _library
    if _library is None:
        from paper_1503_05032_amd import binding
        _library = binding
    B, kind = _library, s["kind"]
    if kind == "norm":
        y, q, scale = s.get("y"), s.get("q"), s.get("scale")
        B.csr5_rmsnorm(s["x"], s["gain"], EPS, residual=s["residual"], h=s["h"], y=y, q=q, scale=scale, rstd=s["rstd"])
        return [s["h"], s["rstd"]] + ([y] if q is None else [q, scale])
    if kind == "norm_back":
        if "workspace" not in s:
            s["workspace"] = torch.empty(B.csr5_rmsnorm_workspace_bytes(*s["h"].shape), dtype=torch.uint8, device=DEVICE)
        B.csr5_rmsnorm_backward(s["h"], s["gain"], s["rstd"], s["dy"], s["dh"], s["dgain"], s["workspace"], residual_grad=s["residual_grad"])
        return [s["dh"], s["dgain"]]
    if kind == "route":
        if "workspace" not in s:
            s["workspace"] = torch.empty(B.csr5_route_workspace_bytes(*s["logits"].shape, s["case"]["k"]), dtype=torch.uint8, device=DEVICE)
        B.csr5_route(s["logits"], s["case"]["k"], s["expert"], s["weight"], s["offset"], s["source"], s["place"], s["workspace"])
        return [s["expert"], s["weight"], s["offset"], s["source"], s["place"]]
    if kind == "combine_train":
        B.csr5_combine(s["z"], s["place"], s["y"], weight=s["weight"])
        B.csr5_combine_backward(s["dy"], s["z"], s["place"], s["weight"], s["dz"], s["dweight"])
        B.csr5_route_backward(s["expert"], s["weight"], s["dweight"], s["dlogits"])
        return [s["y"], s["dz"], s["dweight"], s["dlogits"]]
    if kind == "grouped":
        B.csr5_grouped_gemm(s["x"], s["w"], s["offset"], s["y"], source=s["source"])
        return s["y"]
    if kind == "grouped_back":
        B.csr5_grouped_gemm_dx(s["dy"], s["w"], s["offset"], s["dx"])
        B.csr5_grouped_gemm_dw(s["dy"], s["x"], s["offset"], s["dw"], source=s["source"])
        return [s["dx"], s["dw"]]
    if kind == "f8":
        if not s["case"]["quantise"]:
            B.csr5_gemm_f8(s["x8"], s["x_scale"], s["w8"], s["w_scale"], s["y"], w_rows=s["case"]["w_rows"])
            return s["y"]
        B.csr5_quantise(s["x"], s["x8"], s["x_scale"])
        B.csr5_gemm_f8(s["x8"], s["x_scale"], s["w8"], s["w_scale"], s["y"], w_rows=s["case"]["w_rows"])
        return [s["x8"], s["x_scale"], s["y"]]
    B.csr5_grouped_gemm_f8(s["x8"], s["x_scale"], s["w8"], s["w_scale"], s["offset"], s["y"], source=s["source"])
    return s["y"]


def _padded(offset, most):
    """Rows of each group side by side: index[group, i] into the rows, and whether there is such a row."""
    first, count = offset[:-1, None].long(), (offset[1:] - offset[:-1])[:, None]
    i = torch.arange(most, device=DEVICE)[None]
    there = i < count
    return torch.where(there, first + i, 0), there


def _grouped(x, w, offset, most):
    """x[rows, d] times w[group][n, d] transposed, for the rows of each group."""
    index, there = _padded(offset, most)
    y = torch.bmm(x[index], w.transpose(1, 2).contiguous())
    out = torch.empty(x.shape[0], w.shape[1], device=DEVICE)
    out[index[there]] = y[there]
    return out


def _dequantised(q, scale):
    d = q.shape[-1]
    return q.float() * scale.repeat_interleave(BLOCK, -1)[..., :d]


def _plain(s):
    kind, c = s["kind"], s["case"]
    dt = TYPES[c["dtype"]]
    if kind == "norm":
        h = s["x"].float() + s["residual"].float()
        rstd = torch.rsqrt(h.square().mean(1) + EPS)
        y = h * rstd[:, None] * s["gain"].float()
        if c["out"] == "f8":
            return [h.to(dt), rstd, *_quantised(y, 1)]
        return [h.to(dt), rstd, y.to(dt)]
    if kind == "norm_back":
        r = s["rstd"][:, None]
        unit, dy = s["h"].float() * r, s["dy"].float()
        u = dy * s["gain"].float()
        dh = r * (u - unit * (u * unit).mean(1, keepdim=True)) + s["residual_grad"].float()
        return [dh.to(dt), (dy * unit).sum(0)]
    if kind == "route":
        k, e, t = c["k"], c["experts"], c["tokens"]
        top, index = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
        top, index = top[:, :k], index[:, :k]
        there = top > -math.inf
        expert = torch.where(there, index, -1)
        part = torch.where(there, torch.exp(top - torch.where(there[:, :1], top[:, :1], 0)), 0)
        weight = part / part.sum(1, keepdim=True).clamp(min=1)          # the largest is exp(0): no sum of a row is under 1
        key = torch.where(there, index, e).reshape(-1)
        order = torch.sort(key, stable=True).indices
        offset = torch.zeros(e + 1, dtype=torch.int32, device=DEVICE)
        offset[1:] = torch.cumsum((key[:, None] == torch.arange(e, device=DEVICE)).sum(0), 0)
        pair = torch.arange(t * k, device=DEVICE)
        place = torch.empty_like(pair)
        place[order] = pair
        place = torch.where(there, place.view(t, k), -1)
        source = torch.where(pair < offset[e], order // k, -1)
        return [expert.int(), weight, offset, source.int(), place.int()]
    if kind == "combine_train":
        place, weight, dy = s["place"].long(), s["weight"], s["dy"].float()
        z = s["z"].float()[place]
        y = (weight[:, :, None] * z).sum(1)
        dz = torch.empty(s["z"].shape, device=DEVICE)
        dz[place] = weight[:, :, None] * dy[:, None, :]
        dweight = (dy[:, None, :] * z).sum(2)
        dlogits = torch.zeros(c["tokens"], c["experts"], device=DEVICE)
        dlogits.scatter_(1, s["expert"].long(), weight * (dweight - (weight * dweight).sum(1, keepdim=True)))
        return [y.to(dt), dz.to(dt), dweight, dlogits.to(dt)]
    if kind == "grouped":
        return _grouped(s["x"].float()[s["source"]], s["w"].float(), s["offset"], s["most"]).to(dt)
    if kind == "grouped_back":
        dy, x = s["dy"].float(), s["x"].float()[s["source"]]
        dx = _grouped(dy, s["w"].float().transpose(1, 2), s["offset"], s["most"])
        index, there = _padded(s["offset"], s["most"])
        dw = torch.bmm((dy[index] * there[:, :, None]).transpose(1, 2).contiguous(), x[index])
        return [dx.to(dt), dw.to(dt)]
    if kind == "f8":
        x8, x_scale = _quantised(s["x"], 1) if c["quantise"] else (s["x8"], s["x_scale"])
        w_scale = _per_row(s["w_scale"], c["n"]) if c["w_rows"] == BLOCK else s["w_scale"]
        y = (_dequantised(x8, x_scale) @ _dequantised(s["w8"], w_scale).T).to(dt)
        return [x8, x_scale, y] if c["quantise"] else y
    x = _dequantised(s["x8"], s["x_scale"])[s["source"]]
    return _grouped(x, _dequantised(s["w8"], _per_row(s["w_scale"], c["n"])), s["offset"], s["most"]).to(dt)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    c, kind = case, case["kind"]
    size = 4 if c["dtype"] == "f32" else 2
    if kind == "norm":
        r, n = c["rows"], c["n"]
        y = r * (n + 4 * _blocks(n)) if c["out"] == "f8" else r * n * size
        return {"bytes": 3 * r * n * size + n * size + 4 * r + y, "flops": 6 * r * n}
    if kind == "norm_back":
        r, n = c["rows"], c["n"]
        return {"bytes": 4 * r * n * size + n * size + 4 * r + 4 * n, "flops": 9 * r * n}
    if kind == "route":
        t, e, k = c["tokens"], c["experts"], c["k"]
        return {"bytes": t * e * size + 16 * t * k + 4 * (e + 1), "flops": t * e + 4 * t * k}
    if kind == "combine_train":
        t, e, k, n = c["tokens"], c["experts"], c["k"], c["n"]
        return {"bytes": 2 * t * k * n * size + 2 * t * n * size + 16 * t * k + t * e * size, "flops": 5 * t * k * n}
    n, d = c["n"], c["depth"]
    if kind == "f8":
        m = c["rows"]
        w_scales = 4 * _blocks(d) * (_blocks(n) if c["w_rows"] == BLOCK else n)
        rows = m * d * 2 if c["quantise"] else 0                     # read in 16 bits; its 8-bit form is an output
        return {"bytes": rows + m * d + 4 * m * _blocks(d) + n * d + w_scales + m * n * size, "flops": 2 * m * n * d}
    t, e, k = c["tokens"], c["experts"], c["k"]
    p = t * k
    used = e * (1 - (1 - 1 / e) ** p)                                # experts that have a row, as evenly drawn ones do
    if kind == "f8_grouped":
        return {"bytes": t * (d + 4 * _blocks(d)) + used * (n * d + 4 * _blocks(n) * _blocks(d)) + p * n * size + 4 * p, "flops": 2 * p * n * d}
    if kind == "grouped":
        return {"bytes": (t * d + used * n * d + p * n) * size + 4 * p, "flops": 2 * p * n * d}
    return {"bytes": (p * n + used * n * d + p * d + t * d + e * n * d) * size + 4 * p, "flops": 4 * p * n * d}


# ---------------------------------------------------------------------------------------------------------------
# the definition, in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _values(q, scale, row_block):
    """What 8-bit values stand for, column block by column block."""
    out = q.double()
    for b in range(scale.shape[-1]):
        sc = scale[..., b].double()
        rows = sc if row_block == 1 else sc[..., torch.arange(q.shape[-2], device=DEVICE) // row_block]
        out[..., b * BLOCK:(b + 1) * BLOCK] *= rows[..., None]
    return out


def _each_group(s):
    o = s["offset"].tolist()
    return [(g, a, b) for g, (a, b) in enumerate(zip(o, o[1:])) if b > a]


def exact(case, seed):
    s, c = prepare(case, seed), case
    kind = c["kind"]
    d = {name: t.double() for name, t in s.items() if torch.is_tensor(t) and t.is_floating_point() and "8" not in name}
    if kind == "norm":
        h = d["x"] + d["residual"]
        rstd = (h.pow(2).sum(1) / c["n"] + EPS) ** -0.5
        y = h * d["gain"] * rstd.view(-1, 1)
        if c["out"] == "same":
            return [h, rstd, y]
        scale = torch.stack([y[:, b * BLOCK:(b + 1) * BLOCK].abs().max(1).values for b in range(_blocks(c["n"]))], 1) / F8_MAX
        scale = scale.clamp(min=SCALE_MIN)
        return [h, rstd, y / scale[:, torch.arange(c["n"], device=DEVICE) // BLOCK], scale]
    if kind == "norm_back":
        rstd, unit = d["rstd"].view(-1, 1), d["h"] * d["rstd"].view(-1, 1)
        inner = (d["dy"] * d["gain"] * unit).sum(1, keepdim=True) / c["n"]
        return [rstd * d["dy"] * d["gain"] - rstd * unit * inner + d["residual_grad"], (d["dy"] * unit).sum(0)]
    if kind == "route":
        # the k largest by k rounds of taking the first maximum
        left, rounds = d["logits"].clone(), []
        for _ in range(c["k"]):
            best = left.max(1).values
            rounds.append(best)
            left.scatter_(1, (left == best[:, None]).int().argmax(1, keepdim=True), -math.inf)
        top = torch.stack(rounds, 1)
        weight = torch.nan_to_num(torch.softmax(top, 1), nan=0.0)
        return [None, weight, None, None, None]
    if kind == "combine_train":
        t, k = c["tokens"], c["k"]
        y, dweight = torch.zeros_like(d["dy"]), torch.zeros_like(d["weight"])
        dz = torch.zeros_like(d["z"])
        dlogits = torch.zeros(t, c["experts"], dtype=torch.float64, device=DEVICE)
        for j in range(k):
            row, w = s["place"][:, j].long(), d["weight"][:, j:j + 1]
            y += w * d["z"][row]
            dz[row] = w * d["dy"]
            dweight[:, j] = (d["dy"] * d["z"][row]).sum(1)
        mean = (d["weight"] * dweight).sum(1)
        for j in range(k):
            dlogits[torch.arange(t, device=DEVICE), s["expert"][:, j].long()] = d["weight"][:, j] * (dweight[:, j] - mean)
        return [y, dz, dweight, dlogits]
    if kind == "f8":
        w = _values(s["w8"], s["w_scale"], c["w_rows"])
        if not c["quantise"]:
            return _values(s["x8"], s["x_scale"], 1) @ w.T
        # the product is that of the quantised rows, which have no value without rounding; what they stand for has
        scale = torch.stack([d["x"][:, b * BLOCK:(b + 1) * BLOCK].abs().max(1).values for b in range(_blocks(c["depth"]))], 1) / F8_MAX
        scale = scale.clamp(min=SCALE_MIN)
        return [d["x"] / scale[:, torch.arange(c["depth"], device=DEVICE) // BLOCK], scale, None]
    if kind == "f8_grouped":
        x, out = _values(s["x8"], s["x_scale"], 1), torch.zeros(s["y"].shape, dtype=torch.float64, device=DEVICE)
        for g, a, b in _each_group(s):
            out[a:b] = x[s["source"][a:b].long()] @ _values(s["w8"][g], s["w_scale"][g], BLOCK).T
        return out
    if kind == "grouped":
        out = torch.zeros(s["y"].shape, dtype=torch.float64, device=DEVICE)
        for g, a, b in _each_group(s):
            out[a:b] = d["x"][s["source"][a:b].long()] @ d["w"][g].T
        return out
    dx, dw = torch.zeros(s["dx"].shape, dtype=torch.float64, device=DEVICE), torch.zeros(s["dw"].shape, dtype=torch.float64, device=DEVICE)
    for g, a, b in _each_group(s):
        dx[a:b] = d["dy"][a:b] @ d["w"][g]
        dw[g] = d["dy"][a:b].T @ d["x"][s["source"][a:b].long()]
    return [dx, dw]
