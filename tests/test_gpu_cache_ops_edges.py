"""Operators on caller-held caches, at edges of their own: selections whose clusters meet nowhere before the first count, queries that are not
numbers."""
import math

import pytest
import torch

from cache_ops_util import scored
from test_gpu_cache_ops import TYPES, _check_evict, _check_scored, _keys, _lens, _near, _normal

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


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,g,cap,m,n_scored,bad", [
    (128, 4, 1000, 1, 1, 0), (64, 8, 9000, 1, 1, 0), (64, 2, 40000, 3, 2, 1), (128, 2, 800, 4, 4, 2), (64, 3, 600, 33, 33, 20),      # one pass
    (128, 4, 1500, 300, 300, 200), (64, 3, 900, 500, 200, 450), (128, 2, 5000, 256, 256, 255), (64, 8, 700, 40, 40, 39),      # tiles of queries
    (128, 4, 1100, 200, 30, 180), (64, 2, 3000, 64, 64, 0),                                # counted queries that stay, and the rows go by
])
def test_a_query_that_is_not_a_number_reaches_every_row_that_it_sees(cuda_lib, dtype, d, g, cap, m, n_scored, bad):
    """What cannot be told comes out as NaN, like a wait that gives up: from a query's own output and the scores of all rows before its own,
    and nowhere else."""
    t, n = TYPES[dtype], cap - 3
    k, v, q = _keys(1, 2, cap, d, dtype=t), _normal(2, 2, cap, d, dtype=t), _normal(3, 2, g, m, d, dtype=t)
    clean = q[0].clone()
    q[0, 0, bad, 5] = math.nan
    out, score = cuda_lib.attn_scored(k, v, q, lens=_lens([n, n]), n_scored=n_scored)
    sees = n - m + bad + 1
    assert bool(out[0, 0, bad].isnan().all())
    if bad >= m - n_scored:
        assert bool(score[0, :sees].isnan().all()), int((~score[0, :sees].isnan()).sum())
    else:
        sees = 0
    for s, queries in enumerate((clean, q[1])):
        ref, got, tol, score_tol = scored(queries, k[s], v[s], n, None, n_scored, 1.0)
        held = torch.ones(g, m, dtype=torch.bool, device="cuda")
        held[0, bad] = s > 0
        _near(out[s][held], ref[held], tol[held], ("out", s))
        first = 0 if s else sees
        _near(score[s, first:n], got[first:], score_tol[first:], ("score", s)) if first < n else None


@pytest.mark.parametrize("streams,cap,g", [(200, 100, 4), (64, 500, 4), (40, 500, 8), (17, 900, 3), (148, 120, 2)])
def test_fp32_streams_about_as_many_as_clusters_run_at_once(cuda_lib, streams, cap, g):
    _check_scored(cuda_lib, "fp32", 128, g, cap, [cap - (13 * s) % 40 for s in range(streams)], 1, 1, seed=streams)


def _busy(stream, cycles=60_000_000):
    """Some 30 ms of work ahead of what comes next on the stream."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(cycles)


def test_tensors_let_go_while_a_call_on_another_stream_waits(cuda_lib):
    """Temporaries passed with ``stream=``: their memory goes to nobody else before the call is over."""
    bk, side, t = cuda_lib, torch.cuda.Stream(), torch.bfloat16
    sizes = [(6, 700, 128), (6, 700, 128), (6, 4, 20, 128), (6, 700), (3, 2, 700, 128), (3, 2, 700, 128), (3, 8, 128)]

    def calls(stream=None):
        k, v, q, score, k2, v2, q2 = (_normal(i, *size, dtype=torch.float32 if len(size) == 2 else t) for i, size in enumerate(sizes))
        lens, w = _lens([700, 3, 0, 650, 128, 77]), _normal(9, 6, 700).abs()[:2].contiguous()
        torch.cuda.synchronize()
        if stream is not None:
            _busy(stream)
        out, new = bk.attn_scored(k, v, q, lens=lens, score=score, score_out=torch.zeros(6, 700, device="cuda"), stream=stream)
        torch.cuda.current_stream().synchronize()          # (score_out's zeros)
        if stream is not None:
            _busy(stream)
        kept = bk.cache_evict(k, v, score, 100, lens=lens, pos=_lens(list(range(4200))).view(6, 700), stream=stream)
        return [out, new, *kept.values(), bk.decode_attn_prefix(k[:2], v[:2], k2, v2, q2, weight=w, stream=stream)]

    want = calls()
    torch.cuda.synchronize()
    want = [x.clone() for x in want]
    got = calls(side)
    noise = [torch.full(size, float("nan"), device="cuda", dtype=dtype) for size in [*sizes, (6,), (6, 700), (2, 700)] for dtype in (t, torch.float32) for _ in range(4)]
    torch.cuda.synchronize()
    del noise
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_call_on_a_stream_within_a_capture(cuda_lib):
    bk, side = cuda_lib, torch.cuda.Stream()
    k, v, q = _normal(1, 4, 900, 64), _normal(2, 4, 900, 64), _normal(3, 4, 2, 64)
    want = [x.clone() for x in bk.attn_scored(k, v, q)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        got = bk.attn_scored(k, v, q, stream=side)
        here.wait_stream(side)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
