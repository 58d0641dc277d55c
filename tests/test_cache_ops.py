"""Host side of the operators on caller-held caches: refusals before anything is launched, and workspaces.  No device."""
import ctypes as C

import pytest

import paper_2502_07861_b200 as bk
from paper_2502_07861_b200.binding import E_INVAL, E_NOMEM, OK

P = 1 << 20        # an aligned address that no refused call touches


def _workspace(name, *args):
    size = C.c_size_t(0)
    return getattr(bk.load(), name + "_workspace")(*args, C.byref(size)), size.value


SCORED = dict(K=P, V=P, lens=P, n_streams=2, capacity=100, q=P, out=P, n_queries=3, group=4, head_dim=128, dtype=1, score_in=P, score_out=P, n_scored=3,
              decay=1.0, workspace=P, workspace_bytes=0, stream=None)
EVICT = dict(K=P, V=P, score=P, pos=P, lens=P, n_streams=2, capacity=100, K_out=2 * P, V_out=2 * P, score_out=2 * P, pos_out=2 * P, lens_out=P, capacity_out=50,
             n_keep=50, n_first=4, n_recent=10, head_dim=64, dtype=0, workspace=P, workspace_bytes=0, stream=None)
PREFIX = dict(K_prefix=P, V_prefix=P, w_prefix=P, prefix_len=200, K=P, V=P, lens=P, capacity=100, q=P, out=P, n_seqs=3, n_kv_heads=2, group=4, head_dim=128,
              dtype=1, workspace=P, workspace_bytes=0, stream=None)
CALLS = {"balancekv_attn_scored": SCORED, "balancekv_cache_evict": EVICT, "balancekv_decode_attn_prefix": PREFIX}


@pytest.mark.parametrize("name,change", [
    ("balancekv_attn_scored", c) for c in (
        dict(K=None), dict(V=None), dict(q=None), dict(out=None), dict(score_out=None), dict(K=P + 8), dict(V=P + 2), dict(q=P + 4), dict(out=P + 8),
        dict(lens=P + 2), dict(score_in=P + 1), dict(score_out=P + 2), dict(workspace=P + 16), dict(n_streams=0), dict(capacity=0), dict(n_queries=0),
        dict(group=0), dict(group=9), dict(head_dim=96), dict(dtype=2), dict(n_scored=-1), dict(n_scored=4), dict(workspace=None, workspace_bytes=1 << 40),
        dict(n_streams=1 << 20, n_queries=1 << 20, n_scored=1), dict(n_streams=1 << 30, capacity=1 << 20))
] + [
    ("balancekv_cache_evict", c) for c in (
        dict(K=None), dict(V=None), dict(score=None), dict(K_out=None), dict(V_out=None), dict(score_out=None), dict(K=P + 8), dict(V_out=2 * P + 4),
        dict(score=P + 2), dict(pos=P + 1), dict(lens_out=P + 2), dict(workspace=P + 64), dict(n_streams=0), dict(capacity=0), dict(n_keep=0),
        dict(capacity_out=49), dict(n_first=-1), dict(n_recent=-1), dict(n_first=41), dict(head_dim=32), dict(dtype=-1), dict(K_out=P), dict(score_out=P),
        dict(K_out=P, V_out=P), dict(K_out=P, V_out=P, score_out=P, pos_out=P), dict(K_out=P, V_out=P, score_out=P, capacity_out=100), dict(pos_out=P),
        dict(workspace=None, workspace_bytes=1 << 40), dict(n_streams=1 << 30, capacity=1 << 20))
] + [
    ("balancekv_decode_attn_prefix", c) for c in (
        dict(K_prefix=None), dict(V_prefix=None), dict(K=None), dict(V=None), dict(q=None), dict(out=None), dict(K_prefix=P + 8), dict(V=P + 2), dict(q=P + 4),
        dict(w_prefix=P + 2), dict(lens=P + 3), dict(workspace=P + 128), dict(prefix_len=0), dict(capacity=-1), dict(n_seqs=0), dict(n_kv_heads=0), dict(group=9),
        dict(head_dim=256), dict(dtype=3), dict(workspace=None, workspace_bytes=1 << 40), dict(n_seqs=1 << 20, n_kv_heads=1 << 10))
])
def test_bad_arguments_are_refused(name, change):
    args = {**CALLS[name], **change}
    assert getattr(bk.load(), name)(*args.values()) == E_INVAL, change


@pytest.mark.parametrize("name", list(CALLS))
def test_small_workspaces_are_refused(name):
    assert getattr(bk.load(), name)(*CALLS[name].values()) == E_NOMEM


def test_workspaces_follow_from_the_arguments():
    rc, one = _workspace("balancekv_attn_scored", 8, 1 << 20, 1, 4, 128, 1, 1)
    assert rc == OK and one > 0
    rc, none = _workspace("balancekv_attn_scored", 1024, 64, 1, 4, 128, 1, 0)
    assert rc == OK and none == 0                          # one split, no scores: nothing to keep between kernels
    assert _workspace("balancekv_attn_scored", 8, 0, 1, 4, 128, 1, 1)[0] == E_INVAL
    assert bk.load().balancekv_attn_scored_workspace(8, 4096, 1, 4, 128, 1, 1, None) == E_INVAL
    rc, out = _workspace("balancekv_cache_evict", 8, 1000, 300, 128, 1, 0)
    rc2, here = _workspace("balancekv_cache_evict", 8, 1000, 300, 128, 1, 1)
    assert rc == rc2 == OK and out > here > 0
    assert _workspace("balancekv_cache_evict", 8, 1000, 0, 128, 1, 0)[0] == E_INVAL
    rc, size = _workspace("balancekv_decode_attn_prefix", 4096, 0, 32, 8, 4, 128, 1)
    assert rc == OK and _workspace("balancekv_decode_attn_prefix", 0, 0, 32, 8, 4, 128, 1)[0] == E_INVAL


def test_tensors_off_the_device_are_refused():
    import torch

    k = torch.zeros(2, 10, 64)
    with pytest.raises(ValueError, match="current CUDA device"):
        bk.attn_scored(k, k, torch.zeros(2, 1, 64))
    with pytest.raises(ValueError, match="current CUDA device"):
        bk.cache_evict(k, k, torch.zeros(2, 10), 5)
    with pytest.raises(ValueError, match="current CUDA device"):
        bk.decode_attn_prefix(k, k, None, None, torch.zeros(3, 2, 64))
    with pytest.raises(ValueError, match="shape"):
        bk.attn_scored(k, k[:1], torch.zeros(2, 1, 64))
    with pytest.raises(ValueError, match="dtype"):
        bk.attn_scored(k, k, torch.zeros(2, 1, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="neither"):
        bk.attn_scored(k.half(), k.half(), torch.zeros(2, 1, 64).half())
    with pytest.raises(ValueError, match="share"):
        bk.decode_attn_prefix(k, k, None, None, torch.zeros(3, 3, 64))


def test_numbers_beyond_32_bits_are_refused():
    import torch

    x, score = torch.zeros(2, 10, 64), torch.zeros(2, 10)
    for change in (dict(n_keep=(1 << 32) + 5), dict(n_keep=5, n_first=1 << 32), dict(n_keep=5, n_recent=-(1 << 32))):
        with pytest.raises(ValueError, match="32 bits"):
            bk.cache_evict(x, x, score, **change)
    with pytest.raises(ValueError, match="32 bits"):
        bk.attn_scored(x, x, torch.zeros(2, 4, 1, 64), n_scored=(1 << 32) + 1)
