"""Helpers of the tests of a layer of experts: inputs, the definitions in 64 bits on the CPU, and error bounds.

U[type] is the largest relative error of one rounding to the type (half a unit in the last place).  Sums in 32 bits of
`terms` terms are off by at most terms * 2^-23 times the sum of the terms' magnitudes: every addition of partial sums
loses at most 2^-23 of them, whether it rounds or cuts."""
import math

import numpy as np
import torch

from paper_1503_05032_amd import binding as B

DEV = "cuda:0"
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}     # absolute, for results near 0
EPS32 = 2.0 ** -23


def close(got, ref, dtype, slack, what=""):
    """|got - ref| <= one rounding to `dtype` of the result, plus `slack` (from the sums) grown by that rounding."""
    got, ref = got.double().cpu(), ref.double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    bound = U[dtype] * ref.abs() + slack * (1 + 2 * U[dtype]) + TINY[dtype]
    bad = ~((got - ref).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), [int(i) for i in bad.nonzero()[0]], float(got[bad][0]), float(ref[bad][0]), float(bound[bad][0]))


def matrix(gen, rows, cols, dtype, layout="plain", scale=1.0):
    """Random rows on the GPU.  layout: "plain"; "wide": a view into wider rows that keeps 16-byte alignment; "odd": one
    that does not.  What surrounds a view is NaN, so that a kernel that reads it shows."""
    v = (torch.randn(rows, cols, generator=gen) * scale).to(dtype)
    return place_in(v, layout)


def place_in(v, layout):
    rows, cols = v.shape
    if layout == "plain":
        return v.to(DEV).contiguous()
    left, right = (16, 16 + -cols % 16) if layout == "wide" else (1, 2 + cols % 2)
    if v.dtype is torch.float8_e4m3fn:
        big = torch.full((rows + 2, left + cols + right), 0x7f, dtype=torch.uint8).view(v.dtype)
        big.view(torch.uint8)[1:1 + rows, left:left + cols] = v.view(torch.uint8)
    else:
        big = torch.full((rows + 2, left + cols + right), math.nan, dtype=v.dtype)
        big[1:1 + rows, left:left + cols] = v
    return big.to(DEV)[1:1 + rows, left:left + cols]


def room(rows, cols, dtype, layout="plain"):
    """Uninitialised output of the same layouts, filled with a value that no kernel writes there; check with untouched()."""
    left, right = {"plain": (0, 0), "wide": (16, 16 + -cols % 16), "odd": (1, 2 + cols % 2)}[layout]
    big = torch.full((rows + 2, left + cols + right), 77.0, device=DEV).to(dtype)
    return big, big[1:1 + rows, left:left + cols]


def untouched(big, rows, cols, layout):
    """Nothing around the output was written."""
    left = {"plain": 0, "wide": 16, "odd": 1}[layout]
    mask = torch.ones(big.shape, dtype=torch.bool, device=DEV)
    mask[1:1 + rows, left:left + cols] = False
    assert bool((big.float()[mask] == torch.tensor(77.0).to(big.dtype).float().item()).all())


def offsets(sizes):
    return torch.tensor([0] + list(np.cumsum(sizes)), dtype=torch.int32, device=DEV)


def quantised(x, block_rows):
    """e4m3 values and scales from the definition, in 64 bits."""
    rows, n = x.shape
    x = x.double()
    q = torch.zeros(rows, n, dtype=torch.float8_e4m3fn)
    scale = torch.zeros(-(-rows // block_rows), -(-n // 128), dtype=torch.float64)
    for i in range(scale.shape[0]):
        for b in range(scale.shape[1]):
            part = x[i * block_rows:(i + 1) * block_rows, b * 128:(b + 1) * 128]
            scale[i, b] = max(float(part.abs().max()) / 448.0, 2.0 ** -126)
            q[i * block_rows:(i + 1) * block_rows, b * 128:(b + 1) * 128] = (part / scale[i, b]).float().to(torch.float8_e4m3fn)
    return q, scale.float()


def meaning(q, scale, block_rows):
    """What 8-bit values stand for, in 64 bits."""
    rows, n = q.shape
    full = scale.double().repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :n]
    return q.float().double() * full


assert B.CSR5_F8_BLOCK == 128
