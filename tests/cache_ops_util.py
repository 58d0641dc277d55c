"""Definitions in 64 bits of the operators on caller-held caches, with bounds on what a right kernel may be off by."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def attention(q, k, v, visible, weight=None, rounded_p=False):
    """q [r, d] over k, v [n, d] of one stream; visible [r, n]; weight [n].  Returns out [r, d], p [r, n] and bounds on their
    errors, element by element.

    A logit sums d products in fp32: it is off by at most dx = (d + 4) 2^-24 sum |q k| / sqrt d, and the base-2 exponent's product
    and exponential add 2^-22 and |x| 2^-22.  A weight's numerator and its denominator are off by e^dx each, the sums of n terms by
    n 2^-24.  Where the second product takes the weights in bf16 (rounded_p), each adds half a step of its own; the result is rounded
    to its type."""
    r, d = q.shape
    n = k.shape[0]
    out, p = torch.zeros(r, d, dtype=torch.float64, device=q.device), torch.zeros(r, n, dtype=torch.float64, device=q.device)
    if n == 0:
        return out, p, out, p
    qd, kd, vd = q.double(), k.double(), v.double()
    z = qd @ kd.T / math.sqrt(d)
    if weight is not None:
        z = z + weight.double().log()
        visible = visible & (weight > 0)
    z = z.masked_fill(~visible, -math.inf)
    sees = visible.any(-1)
    p[sees] = torch.softmax(z[sees], -1)
    out = p @ torch.where(visible.any(0)[:, None], vd, 0.0)
    size = (qd.abs() @ kd.abs().T / math.sqrt(d)).masked_fill(~visible, 0.0)
    dx = ((d + 4) * 2.0 ** -24 * size + 2.0 ** -22 * (1 + z.masked_fill(~visible, 0.0).abs())).amax(-1, keepdim=True)
    rel = 2 * dx + (n + 64) * 2.0 ** -24
    mass = p @ torch.where(visible.any(0)[:, None], vd.abs(), 0.0)
    half = HALF_STEP[q.dtype]
    return out, p, half * out.abs() + (rel + (half if rounded_p else 0.0)) * mass + 1e-30, rel * p


def scored(q, k, v, n, score, n_scored, decay):
    """One stream: q [g, m, d], k and v [cap, d] with n rows in use, score [cap] or None."""
    g, m, d = q.shape
    j, i = torch.arange(m, device=q.device)[:, None], torch.arange(n, device=q.device)
    visible = (i <= n - m + j).repeat(g, 1)
    out, p, out_tol, p_tol = attention(q.reshape(g * m, d), k[:n], v[:n], visible, rounded_p=True)
    counted = (torch.arange(m, device=q.device) >= m - n_scored).repeat(g)
    old = torch.zeros(n, dtype=torch.float64, device=q.device) if score is None else decay * score[:n].double()
    got = old + p[counted].sum(0)
    tol = p_tol[counted].sum(0) + (g * m + 8) * 2.0 ** -24 * got.abs() + 2.0 ** -23 * old.abs() + 1e-30
    return out.view(g, m, d), got, out_tol.view(g, m, d), tol


def keep_rows(score, pos, n, keep, first, recent):
    """The rows that stay, in the order in which they sit afterwards."""
    s, ps = [float(x) for x in score[:n]], [int(x) for x in pos[:n]]
    newest = max(ps, default=0)
    safe = [p < first or p > newest - recent for p in ps]
    value = [0.0 if safe[i] else -math.inf if s[i] != s[i] else s[i] for i in range(n)]
    nan = [s[i] != s[i] and not safe[i] for i in range(n)]
    best = set(sorted(range(n), key=lambda i: (not safe[i], nan[i], -value[i], i))[:keep])
    late = iter(sorted(i for i in best if i >= keep))
    return [i if i in best else next(late) for i in range(min(n, keep))]
