"""A layer of experts, from the library's operators: trained in 16 bits, served in 8.

    u = norm(x + residual)              csr5_rmsnorm
    which experts, with which weights   csr5_grouped_gemm (one group) and csr5_route
    up and down in each expert          csr5_grouped_gemm over the rows grouped by expert, or csr5_grouped_gemm_f8
    h + sum of the weighted experts     csr5_combine

Between the two products stands silu(a) * b of the halves a and b of the first one's columns; torch computes it, and the
update of the parameters.  `python -m paper_1503_05032_amd.layer` trains a small layer to follow another one and then serves it."""
from __future__ import annotations

import torch

from . import binding as B


class Layer:
    """`experts` experts of `inner` values, `k` of them for each token of `width` values."""

    def __init__(self, width, inner, experts, k, dtype=torch.bfloat16, eps=1e-6, device="cuda:0", generator=None):
        def normal(*shape):
            return torch.randn(*shape, generator=generator).to(device)
        self.width, self.inner, self.experts, self.k, self.dtype, self.eps = width, inner, experts, k, dtype, eps
        self.gain = torch.ones(width, dtype=dtype, device=device)
        self.router = (normal(1, experts, width) * width ** -0.5).to(dtype)
        self.up = (normal(experts, 2 * inner, width) * width ** -0.5).to(dtype)
        self.down = (normal(experts, width, inner) * inner ** -0.5).to(dtype)

    def parameters(self):
        return {"gain": self.gain, "router": self.router, "up": self.up, "down": self.down}

    def _empty(self, *shape, dtype=None):
        return torch.empty(*shape, dtype=dtype or self.dtype, device=self.gain.device)

    def _route(self, u):
        """The pairs of token and expert, grouped by expert."""
        tokens, pairs = u.shape[0], u.shape[0] * self.k
        ints = lambda *shape: self._empty(*shape, dtype=torch.int32)
        logits = self._empty(tokens, self.experts)
        all_rows = torch.arange(2, dtype=torch.int32, device=u.device).mul_(tokens)       # [0, tokens], without a copy that waits
        B.csr5_grouped_gemm(u, self.router, all_rows, logits)
        expert, place, source, offset = ints(tokens, self.k), ints(tokens, self.k), ints(pairs), ints(self.experts + 1)
        weight = self._empty(tokens, self.k, dtype=torch.float32)
        space = self._empty(B.csr5_route_workspace_bytes(tokens, self.experts, self.k), dtype=torch.uint8)
        B.csr5_route(logits, self.k, expert, weight, offset, source, place, workspace=space)
        return {"all_rows": all_rows, "expert": expert, "weight": weight, "offset": offset, "source": source, "place": place}

    def forward(self, x, residual=None):
        """The layer of x [tokens, width], and what `backward` needs."""
        tokens, pairs = x.shape[0], x.shape[0] * self.k
        h, u, rstd = self._empty(tokens, self.width), self._empty(tokens, self.width), self._empty(tokens, dtype=torch.float32)
        B.csr5_rmsnorm(x, self.gain, self.eps, residual=residual, h=h, y=u, rstd=rstd)
        s = self._route(u)
        wide, z, y = self._empty(pairs, 2 * self.inner), self._empty(pairs, self.width), self._empty(tokens, self.width)
        B.csr5_grouped_gemm(u, self.up, s["offset"], wide, source=s["source"])
        a, b = wide.float().chunk(2, dim=1)
        act = (torch.nn.functional.silu(a) * b).to(self.dtype)
        B.csr5_grouped_gemm(act, self.down, s["offset"], z)
        B.csr5_combine(z, s["place"], y, weight=s["weight"], residual=h)
        s.update(h=h, u=u, rstd=rstd, wide=wide, act=act, z=z)
        return y, s

    def backward(self, dy, s):
        """The gradient of x (and of the residual: the same), and those of the parameters, by name."""
        tokens, pairs = dy.shape[0], dy.shape[0] * self.k
        dz, dweight = self._empty(pairs, self.width), self._empty(tokens, self.k, dtype=torch.float32)
        B.csr5_combine_backward(dy, s["z"], s["place"], s["weight"], dz, dweight)
        dact, ddown = self._empty(pairs, self.inner), torch.empty_like(self.down)
        B.csr5_grouped_gemm_dx(dz, self.down, s["offset"], dact)
        B.csr5_grouped_gemm_dw(dz, s["act"], s["offset"], ddown)
        a, b = s["wide"].float().chunk(2, dim=1)
        sig, da = torch.sigmoid(a), dact.float()
        dwide = torch.cat([da * b * sig * (1 + a * (1 - sig)), da * a * sig], dim=1).to(self.dtype)
        dpairs, dup = self._empty(pairs, self.width), torch.empty_like(self.up)
        B.csr5_grouped_gemm_dx(dwide, self.up, s["offset"], dpairs)
        B.csr5_grouped_gemm_dw(dwide, s["u"], s["offset"], dup, source=s["source"])
        dlogits, drouter = self._empty(tokens, self.experts), torch.empty_like(self.router)
        B.csr5_route_backward(s["expert"], s["weight"], dweight, dlogits)
        from_router, du, dx = (self._empty(tokens, self.width) for _ in range(3))
        B.csr5_grouped_gemm_dx(dlogits, self.router, s["all_rows"], from_router)
        B.csr5_grouped_gemm_dw(dlogits, s["u"], s["all_rows"], drouter)
        B.csr5_combine(dpairs, s["place"], du, residual=from_router)                 # each token's k rows, added up
        dgain = self._empty(self.width, dtype=torch.float32)
        space = self._empty(B.csr5_rmsnorm_workspace_bytes(tokens, self.width), dtype=torch.uint8)
        B.csr5_rmsnorm_backward(s["h"], self.gain, s["rstd"], du, dx, dgain=dgain, workspace=space, residual_grad=dy)
        return dx, {"gain": dgain, "router": drouter, "up": dup, "down": ddown}

    def for_serving(self):
        """The experts in 8 bits, a scale for each block of 128 x 128: laid out once, for `serve`."""
        def eight(w):
            q = torch.empty_like(w, dtype=torch.float8_e4m3fn)
            scale = self._empty(w.shape[0], -(-w.shape[1] // 128), -(-w.shape[2] // 128), dtype=torch.float32)
            for i in range(w.shape[0]):
                B.csr5_quantise(w[i], q[i], scale[i], block_rows=128)
            return q, scale
        return eight(self.up) + eight(self.down)

    def serve(self, x, eight, residual=None):
        """The layer of x with the experts in 8 bits: `forward` without what training keeps."""
        up, up_scale, down, down_scale = eight
        tokens, pairs, blocks = x.shape[0], x.shape[0] * self.k, lambda n: -(-n // 128)
        f8, f32 = torch.float8_e4m3fn, torch.float32
        h, u = self._empty(tokens, self.width), self._empty(tokens, self.width)
        q, scale = self._empty(tokens, self.width, dtype=f8), self._empty(tokens, blocks(self.width), dtype=f32)
        B.csr5_rmsnorm(x, self.gain, self.eps, residual=residual, h=h, y=u, q=q, scale=scale)
        s = self._route(u)
        wide, z, y = self._empty(pairs, 2 * self.inner), self._empty(pairs, self.width), self._empty(tokens, self.width)
        B.csr5_grouped_gemm_f8(q, scale, up, up_scale, s["offset"], wide, source=s["source"])
        a, b = wide.float().chunk(2, dim=1)
        act = (torch.nn.functional.silu(a) * b).to(self.dtype)
        q, scale = self._empty(pairs, self.inner, dtype=f8), self._empty(pairs, blocks(self.inner), dtype=f32)
        B.csr5_quantise(act, q, scale)
        B.csr5_grouped_gemm_f8(q, scale, down, down_scale, s["offset"], z)
        B.csr5_combine(z, s["place"], y, weight=s["weight"], residual=h)
        return y


def train(layer, teacher, steps=40, tokens=512, rate=0.1, generator=None):
    """Steps of momentum by the mean square of layer - teacher, on one batch of random tokens; the losses."""
    master = {name: p.float() for name, p in layer.parameters().items()}
    speed = {name: torch.zeros_like(p) for name, p in master.items()}
    x = torch.randn(tokens, layer.width, generator=generator).to(device=layer.gain.device, dtype=layer.dtype)
    want, _ = teacher.forward(x)
    losses = []
    for _ in range(steps):
        y, saved = layer.forward(x)
        off = y.float() - want.float()
        losses.append(off.square().mean().item())
        _, grads = layer.backward((off / tokens).to(layer.dtype), saved)
        for name, p in layer.parameters().items():
            speed[name].mul_(0.9).add_(grads[name].float())
            master[name].sub_(rate * speed[name])
            p.copy_(master[name])
    return losses


def main():
    g = torch.Generator().manual_seed(1)
    make = lambda: Layer(width=512, inner=256, experts=8, k=2, generator=g)
    teacher, layer = make(), make()
    layer.router.copy_(teacher.router)
    losses = train(layer, teacher, generator=g)
    print(f"loss {losses[0]:.4f} before, {losses[-1]:.4f} after {len(losses)} steps")
    x = torch.randn(64, layer.width, generator=g).to(device=layer.gain.device, dtype=layer.dtype)
    eight = layer.for_serving()
    want, _ = layer.forward(x)
    for tokens in (1, 64):
        got = layer.serve(x[:tokens], eight).float()
        print(f"{tokens} tokens served in 8 bits: {((got - want[:tokens].float()).norm() / want[:tokens].float().norm()).item():.4f} from 16 bits")


if __name__ == "__main__":
    main()
