"""The one-pass kernels (up to eight query rows a stream) against their own bound, which leaves no room for weights in bf16 alone."""
import pytest
import torch

from one_pass_bounds import awkward_inputs, one_pass_attention
from test_gpu_cache_ops import TYPES, _keys, _lens, _near, _normal

pytestmark = pytest.mark.gpu


def _check(bk, q, k, v, lens, **kw):
    S, g, m, d = q.shape
    out, _ = bk.attn_scored(k, v, q, lens=_lens(lens), **kw)
    for s, n in enumerate(lens):
        visible = (torch.arange(n, device="cuda") <= n - m + torch.arange(m, device="cuda")[:, None]).repeat(g, 1)
        ref, _, tol = one_pass_attention(q[s].reshape(g * m, d), k[s, :n], v[s, :n], visible)
        _near(out[s].reshape(g * m, d), ref, tol, (s, n))


@pytest.mark.parametrize("n_scored", [0, 1])
@pytest.mark.parametrize("rows,d,g,m,streams", [
    (64, 128, 1, 1, 3), (64, 64, 4, 1, 3), (2500, 128, 4, 1, 2), (1000, 64, 8, 1, 5), (600, 128, 5, 1, 300), (300, 128, 2, 2, 4), (300, 64, 4, 2, 1), (128, 64, 7, 1, 700),
])
def test_weights_that_bf16_does_not_hold(cuda_lib, rows, d, g, m, streams, n_scored):
    q, k, v = (x.cuda().unsqueeze(0).expand(streams, *x.shape).contiguous() for x in awkward_inputs(rows, d, g, m, seed=rows))
    _check(cuda_lib, q, k, v, [rows - 2 * (s % 7) for s in range(streams)], n_scored=n_scored)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,g,m,cap,lens", [
    (128, 4, 1, 4000, [4000, 3999, 1, 0, 33]), (64, 3, 1, 7000, [7000, 2048]), (128, 5, 1, 5000, [5000, 17]), (64, 8, 1, 3000, [3000] * 3), (128, 7, 1, 900, [900, 64] * 30),
    (64, 1, 8, 2000, [2000, 5]), (128, 2, 4, 2500, [2500, 2, 128]), (128, 2, 2, 9000, [9000, 3]), (64, 6, 1, 260, [260 - s % 9 for s in range(800)]),
])
def test_one_pass_attention(cuda_lib, dtype, d, g, m, cap, lens):
    t, S = TYPES[dtype], len(lens)
    _check(cuda_lib, _normal(3, S, g, m, d, dtype=t), _keys(1, S, cap, d, dtype=t), _normal(2, S, cap, d, dtype=t), lens)


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,B,H,g,P,cap", [(128, 2, 2, 4, 3000, 500), (64, 1, 3, 8, 5001, 100), (128, 3, 2, 2, 700, 0), (64, 8, 1, 1, 400, 3000), (128, 1, 4, 5, 2000, 40)])
def test_one_pass_prefix(cuda_lib, dtype, d, B, H, g, P, cap, weighted):
    """Few query rows behind a prefix: it and the own rows are read by one launch."""
    t = TYPES[dtype]
    pk, pv, q = _keys(1, H, P, d, dtype=t), _normal(2, H, P, d, dtype=t), _normal(3, B, H * g, d, dtype=t)
    k, v = (_keys(4, B, H, cap, d, dtype=t), _normal(5, B, H, cap, d, dtype=t)) if cap else (None, None)
    w = torch.exp2(torch.arange(P, device="cuda") % 4).expand(H, P).contiguous() if weighted else None
    out = cuda_lib.decode_attn_prefix(pk, pv, k, v, q, weight=w)
    for b in range(B):
        for h in range(H):
            rows, values = (torch.cat([pk[h], k[b, h]]), torch.cat([pv[h], v[b, h]])) if cap else (pk[h], pv[h])
            weight = torch.cat([w[h] if weighted else torch.ones(P, device="cuda"), torch.ones(cap, device="cuda")])
            ref, _, tol = one_pass_attention(q[b, h * g:h * g + g], rows, values, torch.ones(g, len(rows), dtype=torch.bool, device="cuda"), weight)
            _near(out[b, h * g:h * g + g], ref, tol, (b, h))


@pytest.mark.parametrize("g", [4, 8])
def test_prefix_weights_that_bf16_does_not_hold(cuda_lib, g):
    q, k, v = (x.cuda() for x in awkward_inputs(800, 128, g, 1, seed=g))
    pk, pv = k[None].contiguous(), v[None].contiguous()
    out = cuda_lib.decode_attn_prefix(pk, pv, pk[None], pv[None], q[:, 0][None].contiguous())
    ref, _, tol = one_pass_attention(q[:, 0], torch.cat([k, k]), torch.cat([v, v]), torch.ones(g, 1600, dtype=torch.bool, device="cuda"))
    _near(out[0], ref, tol, g)
