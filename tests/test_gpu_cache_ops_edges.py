"""Operators on caller-held caches, at edges of their own: selections whose clusters meet nowhere before the first count."""
import pytest
import torch

from test_gpu_cache_ops import _check_evict, _lens, _normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("cap,streams,keep", [(5000, 3, 700), (16500, 2, 9000), (30000, 40, 1000), (300, 600, 70)])
@pytest.mark.parametrize("with_pos", [False, True])
def test_eviction_without_recent_positions(cuda_lib, cap, streams, keep, with_pos, in_place):
    """No newest position to find: the clusters' first meeting is that of the first histograms."""
    lens = [cap - 7 * (s % 5) for s in range(streams)]
    _check_evict(cuda_lib, "bf16", 64, cap, lens, keep, 3, 0, kind="spread", with_pos=with_pos, in_place=in_place, seed=cap)
    if with_pos:
        return
    _check_evict(cuda_lib, "bf16", 64, cap, lens, keep, 3, 5, kind="spread", with_pos=False, in_place=in_place, seed=cap)


@pytest.mark.parametrize("n_recent", [0, 16])
def test_eviction_call_after_call_beside_other_work(cuda_lib, n_recent):
    """Clusters that begin while the device is full of something else, again and again: the same rows every time."""
    k, v, score = _normal(1, 24, 16000, 64, dtype=torch.bfloat16), _normal(2, 24, 16000, 64, dtype=torch.bfloat16), _normal(3, 24, 16000)
    lens = _lens([16000 - 100 * s for s in range(24)])
    want = cuda_lib.cache_evict(k, v, score, 4000, lens=lens, n_recent=n_recent)
    torch.cuda.synchronize()
    a, side = _normal(4, 2048, 2048), torch.cuda.Stream()
    for _ in range(40):
        with torch.cuda.stream(side):
            a @ a
        got = cuda_lib.cache_evict(k, v, score, 4000, lens=lens, n_recent=n_recent)
        assert all(torch.equal(got[name], want[name]) for name in want)
    torch.cuda.synchronize()
