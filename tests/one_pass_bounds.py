"""The bound of the one-pass kernels' outputs in bf16, and inputs at which a kernel that took the weights in bf16 alone would miss it.

The weights p of the second product are split, p = high + low + r: high is p rounded to bf16, off by at most 2^-8 p, low is the rest rounded, so that
|r| <= 2^-8 2^-8 p.  Both products are summed in fp32, 2 n terms whose additions are off by at most a step of 2^-23 each: 4 n 2^-24 in all, of
which the common bound has n.  So the common bound without the half step of rounded weights, and (2^-16 + 3 n 2^-24) sum p |v| more."""
import math

import torch

from cache_ops_util import attention


def one_pass_attention(q, k, v, visible, weight=None):
    out, p, tol, _ = attention(q, k, v, visible, weight, rounded_p=False)
    mass = p @ torch.where(visible.any(0)[:, None], v.double().abs(), 0.0)
    split = 2.0 ** -16 + 3 * k.shape[0] * 2.0 ** -24 if q.dtype == torch.bfloat16 else 0.0
    return out, p, tol + split * mass


def _awkward(d, scale):
    """A bf16 number x for which e^(-x scale / sqrt d), 0.3 .. 1, lies as far from every bf16 number as any of that kind does."""
    x = torch.arange(1, 1 << 12, dtype=torch.float64) / 256
    x = x[x.bfloat16().double() == x]
    p = torch.exp(-x * scale / math.sqrt(d))
    off = ((p - p.bfloat16().double()) / p).abs() * ((p > 0.3) & (p < 0.95))
    return float(x[off.argmax()])


def awkward_inputs(rows, d, g, m, seed=0):
    """q [g, m, d], k, v [rows, d] in bf16, every other row with weight 1 and the others, of opposite sign, with one that bf16 does not hold: head h's
    outputs of the dims j with j % g = h are what its weight is off by."""
    q, k, v = torch.zeros(g, m, d), torch.zeros(rows, d), torch.zeros(rows, d)
    scales = [1.0 + h / 8 for h in range(g)]
    for h in range(g):
        q[h, :, h] = 1.0                                   # head h reads channel h
        k[1::2, h] = -_awkward(d, scales[h]) * 1.0
        q[h, :, h] *= scales[h]
    for j in range(d):
        h = j % g
        p = torch.exp(-torch.tensor(_awkward(d, scales[h]), dtype=torch.float64) * scales[h] / math.sqrt(d))
        v[0::2, j], v[1::2, j] = float(p.bfloat16()), -1.0
    sign = torch.where(torch.rand(d, generator=torch.Generator().manual_seed(seed)) < 0.5, -1.0, 1.0)
    return q.bfloat16(), k.bfloat16(), (v * sign).bfloat16()
