"""The attention beside a layer of experts, from the library's operators: trained over packed sequences, served from a paged cache.

    u = norm(x + residual)                  csr5_rmsnorm
    queries, keys and values of u           csr5_grouped_gemm (one group)
    turned by their positions               csr5_rotary: in place, or keys and values on into the cache
    attention                               csr5_attention, or csr5_attention_paged over the cache
    back to the width                       csr5_grouped_gemm (one group)

What comes out goes, with x + residual for its residual, into the next layer (`layer.Layer`), which adds the two.  A step of serving begins with
`Cache.step`: csr5_pages finds the pages of the requests' new tokens, for all layers at once.  `python -m paper_1503_05032_amd.attention`
trains attention and a layer of experts to follow another pair, and then serves a prompt in chunks."""
from __future__ import annotations

import torch

from . import binding as B
from .layer import Layer


class Attention:
    """`heads` query heads of `d` values, `kv_heads` of keys and values, for tokens of `width` values."""

    def __init__(self, width, heads, kv_heads, d, dtype=torch.bfloat16, eps=1e-6, theta=10000.0, device="cuda:0", generator=None):
        def normal(*shape):
            return torch.randn(*shape, generator=generator).to(device)
        self.width, self.heads, self.kv_heads, self.d, self.dtype, self.eps = width, heads, kv_heads, d, dtype, eps
        self.gain = torch.ones(width, dtype=dtype, device=device)
        self.into = (normal(1, (heads + 2 * kv_heads) * d, width) * width ** -0.5).to(dtype)
        self.back = (normal(1, width, heads * d) * (heads * d) ** -0.5).to(dtype)
        self.frequency = (theta ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().to(device)

    def parameters(self):
        return {"gain": self.gain, "into": self.into, "back": self.back}

    def _empty(self, *shape, dtype=None):
        return torch.empty(*shape, dtype=dtype or self.dtype, device=self.gain.device)

    def _queries(self, x, residual):
        """The norm, and queries, keys and values side by side in one row of each token."""
        tokens = x.shape[0]
        s = {"h": self._empty(tokens, self.width), "u": self._empty(tokens, self.width), "rstd": self._empty(tokens, dtype=torch.float32),
             "rows": torch.arange(2, dtype=torch.int32, device=x.device).mul_(tokens)}
        B.csr5_rmsnorm(x, self.gain, self.eps, residual=residual, h=s["h"], y=s["u"], rstd=s["rstd"])
        s["qkv"] = self._empty(tokens, (self.heads + 2 * self.kv_heads) * self.d)
        B.csr5_grouped_gemm(s["u"], self.into, s["rows"], s["qkv"])
        return s

    def _split(self, qkv):
        return qkv.view(-1, self.heads + 2 * self.kv_heads, self.d).split([self.heads, self.kv_heads, self.kv_heads], dim=1)

    def forward(self, x, offset, position, residual=None):
        """Causal attention within each sequence [offset[s], offset[s + 1]) of x [tokens, width], and what `backward` needs; s["h"] is x + residual.
        Tokens in no sequence (before offset[0], or behind the last) get z = 0 and, in `backward`, the gradient of h alone; they have no part in the parameters'."""
        s = self._queries(x, residual)
        q, k, v = self._split(s["qkv"])
        B.csr5_rotary(q, k, position, self.frequency, q, k_out=k)
        tokens = x.shape[0]
        # the attention leaves rows in no sequence as they are, and the products go over all
        out = torch.zeros(tokens, self.heads, self.d, dtype=self.dtype, device=x.device)
        lse, z = self._empty(self.heads, tokens, dtype=torch.float32), self._empty(tokens, self.width)
        B.csr5_attention(q, k, v, offset, offset, out, lse=lse)
        B.csr5_grouped_gemm(out.view(tokens, -1), self.back, s["rows"], z)
        s.update(offset=offset, position=position, out=out, lse=lse)
        return z, s

    def backward(self, dz, s, dh=None):
        """The gradient of x (and of the residual: the same) from those of z and of h, and the parameters', by name."""
        tokens = dz.shape[0]
        dout, dback = self._empty(tokens, self.heads * self.d), torch.empty_like(self.back)
        B.csr5_grouped_gemm_dx(dz, self.back, s["rows"], dout)
        B.csr5_grouped_gemm_dw(dz, s["out"].view(tokens, -1), s["rows"], dback)
        dqkv = torch.zeros_like(s["qkv"])                   # as `out`
        (q, k, v), (dq, dk, dv) = self._split(s["qkv"]), self._split(dqkv)
        space = self._empty(B.csr5_attention_backward_workspace_bytes(tokens, self.heads), dtype=torch.uint8)
        B.csr5_attention_backward(dout.view(tokens, self.heads, self.d), q, k, v, s["out"], s["lse"], s["offset"], s["offset"], dq, dk, dv, space)
        B.csr5_rotary(dq, dk, s["position"], self.frequency, dq, k_out=dk, inverse=True)
        du, dinto = self._empty(tokens, self.width), torch.empty_like(self.into)
        B.csr5_grouped_gemm_dx(dqkv, self.into, s["rows"], du)
        B.csr5_grouped_gemm_dw(dqkv, s["u"], s["rows"], dinto)
        dx, dgain = self._empty(tokens, self.width), self._empty(self.width, dtype=torch.float32)
        space = self._empty(B.csr5_rmsnorm_workspace_bytes(tokens, self.width), dtype=torch.uint8)
        B.csr5_rmsnorm_backward(s["h"], self.gain, s["rstd"], du, dx, dgain=dgain, workspace=space, residual_grad=dh)
        return dx, {"gain": dgain, "into": dinto, "back": dback}

    def serve(self, x, cache, layer, residual=None):
        """Attention of the step's new tokens x [tokens, width] over the cache of this layer; also x + residual."""
        s = self._queries(x, residual)
        q, k, v = self._split(s["qkv"])
        k_cache, v_cache = cache.k[layer], cache.v[layer]
        B.csr5_rotary(q, k, cache.position, self.frequency, q, v=v, slot=cache.slot, k_cache=k_cache, v_cache=v_cache)
        tokens = x.shape[0]
        out, z = torch.zeros(tokens, self.heads, self.d, dtype=self.dtype, device=x.device), self._empty(tokens, self.width)
        need = B.csr5_attention_paged_workspace_bytes(tokens, self.heads, self.kv_heads, self.d, cache.requests, cache.table.shape[1] * cache.page)
        B.csr5_attention_paged(q, k_cache, v_cache, cache.offset, cache.length, cache.table, out, self._empty(need, dtype=torch.uint8))
        B.csr5_grouped_gemm(out.view(tokens, -1), self.back, s["rows"], z)
        return z, s["h"]


class Cache:
    """Keys and values of `layers` layers: `pages` pages of `page` tokens, for `requests` requests of up to `width` pages each."""

    def __init__(self, layers, pages, page, requests, width, kv_heads, d, dtype=torch.bfloat16, device="cuda:0"):
        ints = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device=device)  # noqa: E731
        self.page, self.requests = page, requests
        self.k, self.v = (torch.zeros(layers, pages, page, kv_heads, d, dtype=dtype, device=device) for _ in range(2))
        self.table, self.pool = ints(requests, width).fill_(-1), torch.arange(pages, dtype=torch.int32, device=device)
        self.length, self.state, self.offset = ints(requests), torch.tensor([0, pages], dtype=torch.int32, device=device), ints(requests + 1)
        self._length, self._state = ints(requests), ints(2)

    def step(self, fresh, tokens):
        """The pages of fresh[r] new tokens (int32; below 0: the request is over) of each request, `tokens` (or fewer) in all: positions,
        slots and row pointer for `Attention.serve`.  A request that gets no pages keeps its length."""
        self.position, self.slot = (torch.empty(tokens, dtype=torch.int32, device=fresh.device) for _ in range(2))
        B.csr5_pages(fresh, self.length, self.table, self.pool, self.state, self.page, self.offset, self.position, self.slot, self._length, self._state)
        self.length.copy_(self._length)
        self.state.copy_(self._state)


def train(pair, teacher, steps=30, tokens=384, rate=0.05, generator=None):
    """Steps of momentum by the mean square of pair - teacher over packed sequences of random tokens; the losses."""
    parts = [part.parameters() for part in pair]
    master = [{name: p.float() for name, p in part.items()} for part in parts]
    speed = [{name: torch.zeros_like(p) for name, p in part.items()} for part in master]
    device, dtype = pair[0].gain.device, pair[0].dtype
    x = torch.randn(tokens, pair[0].width, generator=generator).to(device=device, dtype=dtype)
    offset = torch.tensor([0, tokens // 3, tokens // 3 + 1, tokens], dtype=torch.int32, device=device)
    at = torch.arange(tokens, dtype=torch.int32, device=device)
    position = at - offset[torch.bucketize(at, offset, right=True).clamp(max=3) - 1]

    def run(attention, layer):
        z, a = attention.forward(x, offset, position)
        y, b = layer.forward(z, residual=a["h"])
        return y, a, b
    want = run(*teacher)[0].float()
    losses = []
    for _ in range(steps):
        y, a, b = run(*pair)
        off = y.float() - want
        losses.append(off.square().mean().item())
        dz, layer_grads = pair[1].backward((off / tokens).to(dtype), b)
        _, grads = pair[0].backward(dz, a, dh=dz)
        for part, m, s, g in zip(parts, master, speed, (grads, layer_grads)):
            for name, p in part.items():
                s[name].mul_(0.9).add_(g[name].float())
                m[name].sub_(rate * s[name])
                p.copy_(m[name])
    return losses


def main():
    g = torch.Generator().manual_seed(1)
    make = lambda: (Attention(width=512, heads=8, kv_heads=2, d=64, generator=g), Layer(width=512, inner=256, experts=8, k=2, generator=g))  # noqa: E731
    teacher, pair = make(), make()
    pair[1].router.copy_(teacher[1].router)
    losses = train(pair, teacher, generator=g)
    print(f"loss {losses[0]:.4f} before, {losses[-1]:.4f} after {len(losses)} steps")
    attention, _ = pair
    x = torch.randn(100, 512, generator=g).to(device=attention.gain.device, dtype=attention.dtype)
    whole = torch.tensor([0, 100], dtype=torch.int32, device=x.device)
    want, _ = attention.forward(x, whole, torch.arange(100, dtype=torch.int32, device=x.device))
    cache = Cache(layers=1, pages=16, page=16, requests=1, width=8, kv_heads=2, d=64)
    done = 0
    for count in (60, 39, 1):
        cache.step(torch.tensor([count], dtype=torch.int32, device=x.device), count)
        got, _ = attention.serve(x[done:done + count], cache, 0)
        off = (got.float() - want[done:done + count].float()).norm() / want[done:done + count].float().norm()
        print(f"tokens {done} to {done + count - 1} served: {off.item():.4f} from training")
        done += count


if __name__ == "__main__":
    main()
