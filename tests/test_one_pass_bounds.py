"""The bound that the one-pass kernels are held to tells a kernel whose weights are bf16 alone from one that splits them.  No device."""
import pytest
import torch

from one_pass_bounds import awkward_inputs, one_pass_attention


@pytest.mark.parametrize("rows,d,g,m", [(64, 128, 1, 1), (64, 64, 4, 1), (2500, 128, 4, 1), (1000, 64, 8, 1), (600, 128, 5, 1), (300, 128, 2, 2), (300, 64, 4, 2)])
def test_weights_in_bf16_alone_miss_the_bound(rows, d, g, m):
    q, k, v = awkward_inputs(rows, d, g, m)
    r, visible = g * m, torch.arange(rows) <= rows - m + torch.arange(m)[:, None]
    out, p, tol = one_pass_attention(q.reshape(r, d), k, v, visible.repeat(g, 1))
    top = p.amax(-1, keepdim=True)
    high = (p / top).bfloat16().double()
    low = (p / top - high).bfloat16().double()
    total = (p / top).sum(-1, keepdim=True)
    split, alone = ((high + low) @ v.double() / total).bfloat16().double(), (high @ v.double() / total).bfloat16().double()
    assert bool(((split - out).abs() <= tol).all())
    worst = ((alone - out).abs() / tol).amax(-1)
    assert bool((worst > 1.5).all()), worst                # every query tells
