"""The attention beside a layer of experts, as measurable cases: what stands between one layer of experts and the next.

Packed sequences are rows one after the other with a row pointer (`offset`) as a sparse matrix in CSR has one; a cache of
keys and values is pages that a table names, request by request.  Kinds of case, each ONE pass through an operator by the
calls that `paper_1503_05032_amd.binding` offers:

  "pages"         page tables, the row pointer, positions and cache slots of a step of serving, from its requests' lengths
  "rotary"        rotary positions over one or several axes (time, height, width), to rows or on into the paged cache;
                  backwards the gradient
  "attend"        attention over packed sequences, grouped heads
  "attend_train"  the same and its gradients
  "paged"         attention of the new tokens, one or a chunk for each request, over the paged cache

Sizes are generic: 64 to 128 values to a head, 1 to 16 query heads that share keys and values, one token to some ten
thousand, pages of 16 to 256 tokens.
"""
import math
import random

import torch

own = False                     # False: `run` computes the plain forms; True: it calls the library

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------
def listed():
    cases = {
        # one step of serving for 48 requests, one new token each, some of them over: all latency
        "pages_decode": dict(kind="pages", requests=48, low=1, high=1, cached=4000, page=16, over=0.1, slack=1.0),
        # admission of many prompts at once while the pool runs out
        "pages_prefill": dict(kind="pages", requests=700, low=1, high=90, cached=900, page=32, over=0.05, slack=0.9),
        # one step of serving, straight into the cache
        "rotary_decode": dict(kind="rotary", tokens=24, heads=32, kv_heads=8, d=128, rot=128, axes=1, interleaved=False, dtype="bf16", page=64, inverse=False),
        # a long prompt of text, image and video tokens: three axes, part of each head
        "rotary_prefill": dict(kind="rotary", tokens=16384, heads=28, kv_heads=4, d=128, rot=96, axes=3, interleaved=True, dtype="bf16", page=0, inverse=False),
        # a training step's way back, half precision, an odd number of tokens
        "rotary_back": dict(kind="rotary", tokens=8191, heads=16, kv_heads=16, d=64, rot=64, axes=2, interleaved=False, dtype="f16", page=0, inverse=True),
        # many short prompts in one call
        "attend_short": dict(kind="attend", sequences=37, low=1, high=420, cross=0, heads=16, kv_heads=4, d=128, causal=True, dtype="bf16"),
        # long prompts: the largest call
        "attend_long": dict(kind="attend", sequences=3, low=1500, high=8001, cross=0, heads=32, kv_heads=8, d=128, causal=True, dtype="bf16"),
        # a training step over packed documents
        "train_packed": dict(kind="attend_train", sequences=5, low=300, high=2801, cross=0, heads=20, kv_heads=5, d=128, causal=True, dtype="bf16"),
        # a training step that looks both ways, small heads, half precision
        "train_both_ways": dict(kind="attend_train", sequences=9, low=17, high=1025, cross=0, heads=12, kv_heads=12, d=64, causal=False, dtype="f16"),
        # one step of serving for few requests with short histories
        "paged_decode": dict(kind="paged", requests=8, new_low=1, new_high=1, low=200, high=2200, heads=32, kv_heads=8, d=128, page=16, dtype="bf16"),
        # one step of serving for a full batch with long histories
        "paged_decode_long": dict(kind="paged", requests=48, new_low=1, new_high=1, low=3000, high=24000, heads=64, kv_heads=8, d=128, page=64, dtype="bf16"),
        # chunks of prompts beside single tokens
        "paged_chunk": dict(kind="paged", requests=6, new_low=1, new_high=700, low=2000, high=12000, heads=32, kv_heads=4, d=128, page=32, dtype="bf16"),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["pages", "rotary", "rotary", "attend", "attend", "attend_train", "attend_train", "paged", "paged", "paged"])
    half = rng.choice(["bf16", "bf16", "f16"])
    if kind == "pages":
        high = _log_int(rng, 1, 400)
        return dict(kind=kind, requests=_log_int(rng, 1, 60000 // (high + 59)), low=rng.choice([1, high]), high=high, cached=_log_int(rng, 1, 8000), page=rng.choice([1, 16, 32, 64, 256]),
                    over=rng.choice([0.0, 0.1, 0.3]), slack=rng.choice([0.5, 0.9, 1.0, 2.0]))
    shared, d = rng.choice([1, 2, 4, 5, 7, 8, 16]), rng.choice([64, 80, 96, 128, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 6, 8])
    heads = shared * kv_heads
    if kind == "rotary":
        page = rng.choice([0, 0, 16, 64])
        rot = rng.choice([d, d, d // 2])
        tokens = _log_int(rng, 1, max(2, min(30000, 16384 * 32 * 128 // ((heads + kv_heads) * d)))) | 1
        return dict(kind=kind, tokens=tokens, heads=heads, kv_heads=kv_heads, d=d, rot=rot, axes=rng.choice([1, 1, 2, 3]), interleaved=rng.random() < 0.4, dtype=half if rng.random() < 0.8 else "f32",
                    page=page, inverse=page == 0 and rng.random() < 0.4)
    if kind == "paged":
        requests = _log_int(rng, 1, 64)
        new_high = rng.choice([1, 1, 1, _log_int(rng, 2, 12), _log_int(rng, 12, 900)])
        # queries times keys, and the cache, stay under the largest listed ones
        high = _log_int(rng, 64, int(max(65, min(60000, 6e5 / requests, 8e10 / (requests * new_high * heads * d)))))
        low = rng.choice([1, max(1, high // 3), high])
        return dict(kind=kind, requests=requests, new_low=rng.choice([1, new_high]), new_high=new_high, low=low, high=high, heads=heads, kv_heads=kv_heads, d=d, page=rng.choice([16, 32, 64, 128]), dtype=half)
    sequences = _log_int(rng, 1, 40)
    most = 1.2e11 if kind == "attend_train" else 3.5e11        # sequences * high^2 * heads * d
    high = _log_int(rng, 16, int(min(6000, math.sqrt(most / (sequences * heads * d)))))
    low = rng.choice([0, 1, max(1, high // 3), high])
    return dict(kind=kind, sequences=sequences, low=low, high=high, cross=rng.choice([0, 0, 0, high // 2, -(high // 3)]), heads=heads, kv_heads=kv_heads, d=d, causal=rng.random() < 0.75, dtype=half)


# ---------------------------------------------------------------------------------------------------------------
# inputs, drawn on the GPU
# ---------------------------------------------------------------------------------------------------------------
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _spread(count, low, high):
    """`count` lengths from low to high, evenly spread, both ends among them."""
    if count == 1:
        return [high]
    return [low + (high - low) * i // (count - 1) for i in range(count)]


def _requests(c):
    """Cached and new tokens of each request, -1 new ones where it is over: the same for every seed but for their order."""
    n, fixed = c["requests"], random.Random(5)
    fresh = _spread(n, c["low"], c["high"])
    for r in fixed.sample(range(n), int(c["over"] * n)):
        fresh[r] = -1
    return [(fixed.randint(0, c["cached"]), f) for f in fresh]


def _lengths(c):
    """Queries and keys of each sequence: the same for every seed but for their order."""
    if c["kind"] == "paged":
        new = _spread(c["requests"], c["new_low"], c["new_high"])
        old = _spread(c["requests"], c["low"], c["high"])
        random.Random(5).shuffle(old)                   # many new tokens meet long and short histories
        return [(a, a + b) for a, b in zip(new, old)]
    return [(a, max(0, a + (c["cross"] if a else 0))) for a in _spread(c["sequences"], c["low"], c["high"])]


def _row_pointer(lengths):
    return torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32, device=DEVICE)


def _pages_in_use(rng, g, held, page, extra):
    """A table of pages scattered over a cache for requests that hold so many pages, and the pages that are left."""
    total = sum(held) + extra
    order = torch.randperm(total, generator=g, device=DEVICE).int()
    width = max(max(held), 1)
    row = torch.repeat_interleave(torch.arange(len(held), device=DEVICE), torch.tensor(held, device=DEVICE))
    first = torch.tensor([sum(held[:i]) for i in range(len(held))], device=DEVICE)
    table = torch.full((len(held), width), -1, dtype=torch.int32, device=DEVICE)
    at = torch.arange(sum(held), device=DEVICE)
    table[row, at - first[row]] = order[:sum(held)]
    return table, order[sum(held):], total


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    rng = random.Random(int(seed))
    kind = c["kind"]
    s = dict(kind=kind, case=c)
    i32, f32 = torch.int32, torch.float32
    if kind == "pages":
        page = c["page"]
        requests = _requests(c)
        rng.shuffle(requests)
        length, fresh = [x for x, _ in requests], [f for _, f in requests]
        n = len(requests)
        held = [-(-x // page) for x in length]
        need = sum(max(0, -(-(x + max(f, 0)) // page) - h) for x, f, h in zip(length, fresh, held))
        table, left, total = _pages_in_use(rng, g, held, page, int(need * c["slack"]) + 3)
        room = torch.full((n, max(held) + -(-c["high"] // page) + 1), -1, dtype=i32, device=DEVICE)
        room[:, :table.shape[1]] = table
        first = rng.randrange(total)                    # the free pages are a ring that begins anywhere
        pool = torch.full((total,), -1, dtype=i32, device=DEVICE)
        pool[(first + torch.arange(left.numel(), device=DEVICE)) % total] = left
        tokens = sum(max(f, 0) for f in fresh) + 7      # a padded batch
        empty = lambda *shape: torch.empty(*shape, dtype=i32, device=DEVICE)  # noqa: E731
        s.update(fresh=torch.tensor(fresh, dtype=i32, device=DEVICE), length=torch.tensor(length, dtype=i32, device=DEVICE), table=room, pool=pool,
                 state=torch.tensor([first, left.numel()], dtype=i32, device=DEVICE), offset=empty(n + 1), position=empty(tokens), slot=empty(tokens), length_out=empty(n), state_out=empty(2))
        return s
    dt, d, heads, kv = TYPES[c["dtype"]], c["d"], c["heads"], c["kv_heads"]
    empty = lambda *shape, dtype=dt: torch.empty(*shape, dtype=dtype, device=DEVICE)  # noqa: E731
    if kind == "rotary":
        t, pairs = c["tokens"], c["rot"] // 2
        # queries, keys and values side by side, as one product gives them
        qkv = _randn(g, t, heads + 2 * kv, d).to(dt)
        base = torch.randint(0, 1 << 17, (1,), generator=g, device=DEVICE)
        at = torch.arange(t, device=DEVICE)
        axes = [base + at, (at // 37) % 61, at % 37][:c["axes"]] if c["axes"] > 1 else [base + at]
        s.update(q=qkv[:, :heads], k=qkv[:, heads:heads + kv], v=qkv[:, heads + kv:], position=torch.stack(axes).int(),
                 frequency=(10000.0 ** (-torch.arange(pairs, device=DEVICE, dtype=torch.float64) / pairs)).float(),
                 axis=(torch.arange(pairs, device=DEVICE) * c["axes"] // pairs).int(), q_out=empty(t, heads, d))
        if c["page"]:
            pages = 2 * -(-t // c["page"]) + 2
            slot = torch.randperm(pages * c["page"], generator=g, device=DEVICE)[:t].int()
            slot[t - t // 16:] = -1                     # padding
            s.update(k_cache=_randn(g, pages, c["page"], kv, d).to(dt), v_cache=_randn(g, pages, c["page"], kv, d).to(dt), slot=slot)
        else:
            s.update(k_out=empty(t, kv, d))
        return s
    lengths = _lengths(c)
    rng.shuffle(lengths)
    lq, lk = [a for a, _ in lengths], [b for _, b in lengths]
    rows = sum(lq)
    s.update(q_offset=_row_pointer(lq), most_q=max(lq), most_k=max(lk), scale=d ** -0.5)
    if kind == "paged":
        page = c["page"]
        held = [-(-x // page) for x in lk]
        table, _, pages = _pages_in_use(rng, g, held, page, 5)
        s.update(q=(1.5 * _randn(g, rows, heads, d)).to(dt), k_cache=_randn(g, pages, page, kv, d).to(dt), v_cache=_randn(g, pages, page, kv, d).to(dt), table=table,
                 length=torch.tensor(lk, dtype=i32, device=DEVICE), out=empty(rows, heads, d), lse=empty(heads, rows, dtype=f32))
        return s
    s.update(q=(1.5 * _randn(g, rows, heads, d)).to(dt), k=_randn(g, sum(lk), kv, d).to(dt), v=_randn(g, sum(lk), kv, d).to(dt), k_offset=_row_pointer(lk), out=empty(rows, heads, d),
             lse=empty(heads, rows, dtype=f32))
    if kind == "attend_train":
        s.update(dout=_randn(g, rows, heads, d).to(dt), dq=empty(rows, heads, d), dk=empty(sum(lk), kv, d), dv=empty(sum(lk), kv, d))
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
    B, kind, c = _library, s["kind"], s["case"]
    if kind == "pages":
        B.csr5_pages(s["fresh"], s["length"], s["table"], s["pool"], s["state"], c["page"], s["offset"], s["position"], s["slot"], s["length_out"], s["state_out"])
        return [s["offset"], s["position"], s["slot"], s["length_out"], s["state_out"], s["table"], s["pool"]]
    if kind == "rotary":
        if c["page"]:
            B.csr5_rotary(s["q"], s["k"], s["position"], s["frequency"], s["q_out"], axis=s["axis"], interleaved=c["interleaved"], v=s["v"], slot=s["slot"], k_cache=s["k_cache"], v_cache=s["v_cache"])
            return [s["q_out"], s["k_cache"], s["v_cache"]]
        B.csr5_rotary(s["q"], s["k"], s["position"], s["frequency"], s["q_out"], k_out=s["k_out"], axis=s["axis"], interleaved=c["interleaved"], inverse=c["inverse"])
        return [s["q_out"], s["k_out"]]
    if kind == "paged":
        if "workspace" not in s:
            longest = s["table"].shape[1] * c["page"]
            s["workspace"] = torch.empty(B.csr5_attention_paged_workspace_bytes(s["q"].shape[0], c["heads"], c["kv_heads"], c["d"], c["requests"], longest), dtype=torch.uint8, device=DEVICE)
        B.csr5_attention_paged(s["q"], s["k_cache"], s["v_cache"], s["q_offset"], s["length"], s["table"], s["out"], s["workspace"], lse=s["lse"], scale=s["scale"])
        return [s["out"], s["lse"]]
    B.csr5_attention(s["q"], s["k"], s["v"], s["q_offset"], s["k_offset"], s["out"], lse=s["lse"], scale=s["scale"], causal=c["causal"])
    if kind == "attend":
        return [s["out"], s["lse"]]
    if "workspace" not in s:
        s["workspace"] = torch.empty(B.csr5_attention_backward_workspace_bytes(s["q"].shape[0], c["heads"]), dtype=torch.uint8, device=DEVICE)
    B.csr5_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["q_offset"], s["k_offset"], s["dq"], s["dk"], s["dv"], s["workspace"], scale=s["scale"], causal=c["causal"])
    return [s["out"], s["lse"], s["dq"], s["dk"], s["dv"]]


def _plain_pages(s):
    page = s["case"]["page"]
    fresh, length, table, pool = s["fresh"].long(), s["length"].long(), s["table"].long(), s["pool"].long()
    first, count, ring = s["state"][0].long(), s["state"][1].long(), pool.numel()
    width, tokens = table.shape[1], s["slot"].numel()
    new, over = fresh.clamp(min=0), fresh < 0
    held, wanted = (length + page - 1) // page, (length + new + page - 1) // page
    fits = wanted <= width
    need = torch.where(fits, wanted - held, 0)
    upto = torch.cumsum(need, 0)
    served = fits & ~over & ((upto <= count) | (need == 0))
    offset = torch.zeros(fresh.numel() + 1, dtype=torch.int64, device=DEVICE)
    offset[1:] = torch.cumsum(new, 0)
    took = torch.where(served, need, 0)
    # new pages into the tables
    column = torch.arange(width, device=DEVICE)
    fill = served[:, None] & (column >= held[:, None]) & (column < wanted[:, None])
    at = (first + (upto - need)[:, None] + column - held[:, None]) % ring
    table = torch.where(fill, pool[at], table)
    # pages of the requests that are over go behind the last free one
    back = over[:, None] & (column < held[:, None])
    rank = torch.cumsum(back.flatten().long(), 0).view(back.shape) - 1
    pool_out = pool.clone()
    pool_out[((first + count + rank) % ring)[back]] = table[back]
    # tokens
    t = torch.arange(tokens, device=DEVICE)
    r = (t[:, None] >= offset[None, 1:]).sum(1)
    there = t < offset[-1]
    r = torch.where(there, r, 0)
    position = torch.where(there, length[r] + t - offset[r], 0)
    has = there & served[r]
    p = torch.where(has, position, 0)
    slot = torch.where(has, table[r, p // page] * page + p % page, -1)
    length_out = torch.where(over, 0, torch.where(served, length + new, length))
    state_out = torch.stack([(first + took.sum()) % ring, count - took.sum() + back.sum()])
    return [x.int() for x in (offset, position, slot, length_out, state_out, table, pool_out)]


def _plain_rotary(s):
    c = s["case"]
    rot, pairs, dt = c["rot"], c["rot"] // 2, TYPES[c["dtype"]]
    angle = s["position"].double()[s["axis"].long()].T * s["frequency"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if c["inverse"]:
        sin = -sin

    def turn(x):
        x = x.float()
        a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if c["interleaved"] else (x[..., :pairs], x[..., pairs:rot])
        a, b = a * cos - b * sin, a * sin + b * cos
        turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
        return torch.cat([turned, x[..., rot:]], -1).to(dt)

    q, k = turn(s["q"]), turn(s["k"])
    if not c["page"]:
        return [q, k]
    named = s["slot"] >= 0
    slot = s["slot"][named].long()
    s["k_cache"].view(-1, *k.shape[1:])[slot] = k[named]
    s["v_cache"].view(-1, *k.shape[1:])[slot] = s["v"][named]
    return [q, s["k_cache"], s["v_cache"]]


def _padded(offset, most):
    """Rows of each sequence side by side: index[sequence, i] into the rows, and whether there is such a row."""
    count = (offset[1:] - offset[:-1])[:, None]
    i = torch.arange(most, device=DEVICE)[None]
    there = i < count
    return torch.where(there, offset[:-1, None].long() + i, 0), there


def _plain_attention(s):
    """Sequence by sequence side by side, padded: [sequences * kv_heads, queries of the heads that share, keys]."""
    c, paged, train = s["case"], s["kind"] == "paged", s["kind"] == "attend_train"
    heads, kv, d, dt, scale = c["heads"], c["kv_heads"], c["d"], TYPES[c["dtype"]], s["scale"]
    shared, most_q, most_k, rows = heads // kv, s["most_q"], s["most_k"], s["q"].shape[0]
    index, there = _padded(s["q_offset"], most_q)
    n = index.shape[0]

    def of_queries(x):                                  # [rows, heads, d] -> [n * kv, shared * most_q, d]
        x = x.float()[index] * there[:, :, None, None]
        return x.view(n, most_q, kv, shared, d).permute(0, 2, 3, 1, 4).reshape(n * kv, shared * most_q, d)

    def to_queries(x, like):                            # and back
        out = torch.empty(rows, heads, like, device=DEVICE)
        x = x.view(n, kv, shared, most_q, like).permute(0, 3, 1, 2, 4).reshape(n, most_q, heads, like)
        out[index[there]] = x[there]
        return out

    if paged:
        page = c["page"]
        i = torch.arange(most_k, device=DEVICE)
        k_there = i[None] < s["length"][:, None]
        k_index = torch.where(k_there, s["table"].long()[:, i // page] * page + i % page, 0)
        k_rows, v_rows, last = s["k_cache"].view(-1, kv, d), s["v_cache"].view(-1, kv, d), s["length"]
    else:
        k_index, k_there = _padded(s["k_offset"], most_k)
        k_rows, v_rows, last = s["k"], s["v"], s["k_offset"][1:] - s["k_offset"][:-1]

    def of_keys(x):                                     # -> [n * kv, most_k, d]
        return (x[k_index].float() * k_there[:, :, None, None]).permute(0, 2, 1, 3).reshape(n * kv, most_k, d)

    def to_keys(x):
        out = torch.empty(k_rows.shape, device=DEVICE)
        out[k_index[k_there]] = x.view(n, kv, most_k, d).permute(0, 2, 1, 3)[k_there]
        return out

    q, k, v = of_queries(s["q"]), of_keys(k_rows), of_keys(v_rows)
    mask = k_there[:, None, :].expand(n, most_q, most_k)
    if paged or c["causal"]:
        before = last - (s["q_offset"][1:] - s["q_offset"][:-1])
        mask = mask & (torch.arange(most_k, device=DEVICE) <= torch.arange(most_q, device=DEVICE)[:, None] + before[:, None, None])
    mask = mask[:, None, None].expand(n, kv, shared, most_q, most_k)
    score = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(scale)
    score.view(mask.shape).masked_fill_(~mask, -math.inf)
    top = score.amax(2, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    p = score.sub_(top).exp_()
    total = p.sum(2, keepdim=True)
    p = p.div_(total.clamp(min=1e-30))
    out = to_queries(torch.bmm(p, v), d)
    lse = to_queries(top + torch.log(total), 1)[:, :, 0].T.contiguous()
    if not train:
        return [out.to(dt), lse]
    dout = of_queries(s["dout"])
    o = of_queries(out.to(dt))                          # what a training step keeps
    dv = torch.bmm(p.transpose(1, 2).contiguous(), dout)
    ds = torch.bmm(dout, v.transpose(1, 2).contiguous()).sub_((dout * o).sum(2, keepdim=True)).mul_(p).mul_(scale)
    dq = to_queries(torch.bmm(ds, k), d)
    dk = torch.bmm(ds.transpose(1, 2).contiguous(), q)
    return [out.to(dt), lse, dq.to(dt), to_keys(dk).to(dt), to_keys(dv).to(dt)]


def _plain(s):
    if s["kind"] == "pages":
        return _plain_pages(s)
    return _plain_rotary(s) if s["kind"] == "rotary" else _plain_attention(s)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    c, kind = case, case["kind"]
    if kind == "pages":
        n, page = c["requests"], c["page"]
        tokens = sum(max(f, 0) for _, f in _requests(c))
        moved = sum(-(-x // page) if f < 0 else -(-(x + f) // page) - -(-x // page) for x, f in _requests(c))
        return {"bytes": 4 * (4 * n + 2 * tokens + 2 * moved + 5), "flops": 8 * tokens}
    size = 4 if c["dtype"] == "f32" else 2
    heads, kv, d = c["heads"], c["kv_heads"], c["d"]
    if kind == "rotary":
        t = c["tokens"]
        rows = heads + kv * (2 if c["page"] else 1)
        return {"bytes": 2 * t * rows * d * size + 4 * t * c["axes"] + 4 * c["rot"], "flops": 3 * t * (heads + kv) * c["rot"]}
    lengths = _lengths(c)
    seen = 0
    for q, k in lengths:
        rows = min(q, k)                                # with a causal mask the last of the queries see something
        seen += rows * (k - rows) + rows * (rows + 1) // 2 if kind == "paged" or c["causal"] else q * k
    q_rows, k_rows = sum(q for q, _ in lengths), sum(k for _, k in lengths)
    bytes_ = 2 * q_rows * heads * d * size + 2 * k_rows * kv * d * size + 8 * len(lengths)
    if kind == "paged":
        return {"bytes": bytes_ + 4 * q_rows * heads + 4 * k_rows // c["page"], "flops": 4 * seen * heads * d}
    if kind == "attend":
        return {"bytes": bytes_ + 4 * q_rows * heads, "flops": 4 * seen * heads * d}
    return {"bytes": bytes_ + 4 * q_rows * heads + (2 * q_rows * heads + 2 * k_rows * kv) * d * size, "flops": 14 * seen * heads * d}


# ---------------------------------------------------------------------------------------------------------------
# the definition, in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _served(s):
    """A step of serving, request by request: whole numbers, in which nothing is rounded."""
    page, tokens = s["case"]["page"], s["slot"].numel()
    table, pool, (first, count) = s["table"].tolist(), s["pool"].tolist(), s["state"].tolist()
    free = [pool[(first + i) % len(pool)] for i in range(count)]
    behind, taken, asked = first + count, 0, 0
    offset, position, slot, length_out = [0], [], [], []
    for row, have, new in zip(table, s["length"].tolist(), s["fresh"].tolist()):
        held = -(-have // page)
        if new < 0:
            for p in row[:held]:
                pool[behind % len(pool)] = p
                behind += 1
            length_out.append(0)
            offset.append(offset[-1])
            continue
        want = -(-(have + new) // page)
        fits = want <= len(row)
        asked += want - held if fits else 0
        served = fits and (asked <= count or want == held)
        if served:
            row[held:want] = free[asked - (want - held):asked]
            taken += want - held
        length_out.append(have + new if served else have)
        offset.append(offset[-1] + new)
        position += range(have, have + new)
        slot += [row[i // page] * page + i % page if served else -1 for i in range(have, have + new)]
    position += [0] * (tokens - len(position))
    slot += [-1] * (tokens - len(slot))
    state = [(first + taken) % len(pool), behind - first - taken]
    return [torch.tensor(x, dtype=torch.int32, device=DEVICE) for x in (offset, position, slot, length_out, state, table, pool)]


def exact(case, seed):
    s, c = prepare(case, seed), case
    kind = c["kind"]
    if kind == "pages":
        return _served(s)
    heads, kv, d = c["heads"], c["kv_heads"], c["d"]
    if kind == "rotary":
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE), s["position"].double()[s["axis"].long()].T * s["frequency"].double())[:, None]
        turn = turn.conj() if c["inverse"] else turn

        def turned(x):
            y = x.double().clone()
            pair = y[..., :c["rot"]].unflatten(-1, (-1, 2)) if c["interleaved"] else y[..., :c["rot"]].unflatten(-1, (2, -1)).transpose(-1, -2)
            z = torch.view_as_real(torch.complex(pair[..., 0].contiguous(), pair[..., 1].contiguous()) * turn)
            y[..., :c["rot"]] = (z if c["interleaved"] else z.transpose(-1, -2)).flatten(-2)
            return y
        q, k = turned(s["q"]), turned(s["k"])
        if not c["page"]:
            return [q, k]
        k_cache, v_cache = s["k_cache"].double().view(-1, kv, d), s["v_cache"].double().view(-1, kv, d)
        for t, at in enumerate(s["slot"].tolist()):
            if at >= 0:
                k_cache[at], v_cache[at] = k[t], s["v"][t].double()
        return [q, k_cache.view(s["k_cache"].shape), v_cache.view(s["v_cache"].shape)]
    train, shared = kind == "attend_train", heads // kv
    f64 = dict(dtype=torch.float64, device=DEVICE)
    rows = s["q"].shape[0]
    out, lse = torch.zeros(rows, heads, d, **f64), torch.empty(heads, rows, **f64)
    if train:
        dq, dk, dv = torch.zeros(rows, heads, d, **f64), torch.zeros(s["k"].shape, **f64), torch.zeros(s["k"].shape, **f64)
    edges = s["q_offset"].tolist()
    for i, (a, b) in enumerate(zip(edges, edges[1:])):
        if a == b:
            continue
        if kind == "paged":
            n = int(s["length"][i])
            j = torch.arange(n, device=DEVICE)
            page, place = s["table"][i, j // c["page"]].long(), j % c["page"]
            keys, values = s["k_cache"][page, place], s["v_cache"][page, place]
        else:
            lo, hi = int(s["k_offset"][i]), int(s["k_offset"][i + 1])
            n, keys, values = hi - lo, s["k"][lo:hi], s["v"][lo:hi]
        if n == 0:
            lse[:, a:b] = -math.inf
            continue
        for h in range(heads):
            q, k, v = s["q"][a:b, h].double(), keys[:, h // shared].double(), values[:, h // shared].double()
            x = (q @ k.T) * s["scale"]
            if kind == "paged" or c["causal"]:
                hidden = torch.triu(torch.ones_like(x, dtype=torch.bool), diagonal=n - (b - a) + 1)
                x = torch.where(hidden, -math.inf, x)
            norm = torch.logsumexp(x, 1)
            lse[h, a:b] = norm
            p = torch.nan_to_num(torch.exp(x - norm[:, None]), nan=0.0)
            o = p @ v
            out[a:b, h] = o
            if train:
                do = s["dout"][a:b, h].double()
                dp = do @ v.T
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) * s["scale"]
                dq[a:b, h] = ds @ k
                dk[lo:hi, h // shared] += ds.T @ q
                dv[lo:hi, h // shared] += p.T @ do
    return [out, lse, dq, dk, dv] if train else [out, lse]
