"""Operators on caller-held caches against their definitions in 64 bits, at the sizes and masks where they can go wrong.
Whatever a call has no business to read holds NaN, whatever it has no business to write is looked at afterwards."""
import math

import pytest
import torch

from cache_ops_util import attention, keep_rows, scored

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _normal(seed, *shape, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


def _keys(seed, *shape, dtype):
    """Four channels ten times the others and a mean: logits of either sign, some large."""
    k = _normal(seed, *shape) + 0.5 * _normal(seed + 1, *shape[:-2], 1, shape[-1])
    k[..., 3:35:8] *= 10
    return k.to(dtype)


def _poison(x, lens):
    for s, n in enumerate(lens):
        x[s, n:] = math.nan
    return x


def _lens(lens):
    return torch.tensor(lens, dtype=torch.int32, device="cuda")


def _near(got, want, tol, what):
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), (what, float((off / tol).max()), float(off.max()))


def _check_scored(bk, dtype, d, g, cap, lens, m, n_scored, decay=0.75, old=True, seed=0, use_lens=True, **kw):
    t, S = TYPES[dtype], len(lens)
    k, v = _poison(_keys(seed, S, cap, d, dtype=t), lens), _poison(_normal(seed + 5, S, cap, d, dtype=t), lens)
    q = _normal(seed + 7, S, g, m, d, dtype=t)
    before = _poison(_normal(seed + 8, S, cap).abs_(), lens) if old else None
    score_out = torch.full((S, cap), 77.0, device="cuda")
    out, score = bk.attn_scored(k, v, q, lens=_lens(lens) if use_lens else None, score=before, score_out=score_out, n_scored=n_scored, decay=decay, **kw)
    assert score is score_out
    for s, n in enumerate(lens):
        ref, got, tol, score_tol = scored(q[s], k[s], v[s], n, None if before is None else before[s], n_scored, decay)
        _near(out[s], ref, tol, ("out", s, n))
        if n_scored:
            _near(score[s, :n], got, score_tol, ("score", s, n))
        assert bool((score[s, n if n_scored else 0:] == 77.0).all())
        assert bool((out[s, :, :max(0, m - n)] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,g,cap,lens", [
    (128, 4, 700, [700, 1, 0, 63, 64, 65, 129, 699]), (64, 1, 1, [1, 0, 1]), (64, 8, 130, [130, 127, 128, 2]), (128, 5, 5000, [5000, 4097, 333]),
    (128, 7, 65, [65] * 40), (64, 3, 20000, [19999]), (128, 8, 256, [256, 255, 17, 16, 15, 33]), (128, 2, 40, list(range(41)) * 8), (64, 6, 3000, [3000, 0, 2049, 1500]),
])
def test_one_query(cuda_lib, dtype, d, g, cap, lens):
    _check_scored(cuda_lib, dtype, d, g, cap, lens, 1, 1, seed=d + g)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,g,cap,lens,m,n_scored", [
    (128, 4, 300, [300, 299, 128, 1, 0], 128, 128), (64, 2, 1000, [1000, 33, 32, 5, 517], 33, 33), (128, 1, 129, [129, 128, 127], 129, 64),
    (64, 3, 513, [513, 400, 100], 200, 1), (128, 8, 70, [70, 3], 2, 2), (128, 5, 2000, [2000, 1999], 3, 3), (64, 4, 640, [640], 640, 640),
    (128, 4, 1300, [1300, 1217], 257, 100), (128, 3, 4200, [4200, 4095], 65, 65), (64, 8, 900, [900, 130, 131], 130, 7), (128, 2, 512, [512, 256], 256, 256),
    (128, 6, 385, [385, 384, 383, 200], 384, 130), (64, 1, 2300, [2300, 1150], 1150, 1150), (128, 8, 700, [700, 650], 300, 9), (128, 7, 500, [500, 260], 260, 33),
    (64, 5, 400, [400, 399, 100], 150, 64), (128, 8, 330, [330], 330, 1), (128, 8, 1030, [1030, 1024], 1024, 1024),
])
def test_many_queries(cuda_lib, dtype, d, g, cap, lens, m, n_scored):
    _check_scored(cuda_lib, dtype, d, g, cap, lens, m, n_scored, seed=m)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,g,cap,lens,m,n_scored", [
    (128, 2, 60, [60, 4, 3, 1, 0], 4, 2), (64, 2, 40000, [40000, 39999, 2], 4, 3), (128, 1, 9000, [9000, 8999, 7, 8], 8, 8), (64, 4, 30000, [29999], 2, 1),
    (128, 2, 3000, [(61 * s) % 3001 for s in range(300)], 3, 1), (128, 3, 12000, [12000, 100, 11999], 2, 2),
])
def test_a_handful_of_queries(cuda_lib, dtype, d, g, cap, lens, m, n_scored):
    """Up to eight query rows, drafted tokens' say: the one-pass kernels, every query with a limit of its own."""
    _check_scored(cuda_lib, dtype, d, g, cap, lens, m, n_scored, seed=cap)


def test_a_few_more_blocks_of_queries_than_sms(cuda_lib):
    """150 blocks of query rows, whose keys are split so that the last two do not take a second turn alone."""
    _check_scored(cuda_lib, "bf16", 64, 4, 9000, [9000 - 120 * s for s in range(75)], 100, 7, seed=2)


@pytest.mark.parametrize("dtype,cap", [("bf16", 6300000), ("fp32", 3200000)])
def test_offsets_beyond_32_bits(cuda_lib, dtype, cap):
    """The last stream of caches of more than 2^32 bytes, by the one-pass kernels, the tiles and the eviction."""
    t, lens, d = TYPES[dtype], [5, 0, 700], 128
    k, v = torch.zeros(3, cap, d, dtype=t, device="cuda"), torch.zeros(3, cap, d, dtype=t, device="cuda")
    for s, n in enumerate(lens):
        if n:
            k[s, :n], v[s, :n] = _keys(20 + s, n, d, dtype=t), _normal(30 + s, n, d, dtype=t)
        k[s, n:n + 300] = math.nan
        v[s, n:n + 300] = math.nan
    for m, g in ((1, 4), (20, 2)):
        q = _normal(m, 3, g, m, d, dtype=t)
        out, score = cuda_lib.attn_scored(k, v, q, lens=_lens(lens))
        for s, n in enumerate(lens):
            ref, got, tol, score_tol = scored(q[s], k[s], v[s], n, None, m, 1.0)
            _near(out[s], ref, tol, (m, s))
            _near(score[s, :n], got, score_tol, (m, s, "scores"))
            assert not score[s, n:].any()
    rows = keep_rows(score[2, :700].tolist(), range(700), 700, 100, 0, 10)
    kept = cuda_lib.cache_evict(k, v, score, 100, lens=_lens(lens), n_recent=10)
    assert kept["lens"].tolist() == [5, 0, 100] and kept["pos"][2].tolist() == rows
    assert torch.equal(kept["k"][2], k[2, rows]) and torch.equal(kept["v"][2], v[2, rows])
    n_lens = _lens(lens)
    cuda_lib.cache_evict(k, v, score, 100, lens=n_lens, n_recent=10, in_place=True)
    assert n_lens.tolist() == [5, 0, 100]
    assert torch.equal(kept["k"][2], k[2, :100]) and torch.equal(kept["v"][2], v[2, :100]) and torch.equal(kept["score"][2], score[2, :100])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 40, 150])
def test_scores_are_optional(cuda_lib, dtype, m):
    _check_scored(cuda_lib, dtype, 128, 4, 321, [321, 200, 0], m, 0, seed=3)
    _check_scored(cuda_lib, dtype, 64, 2, 321, [321, 200, 0], m, m, old=False, seed=4)
    _check_scored(cuda_lib, dtype, 64, 2, 321, [321, 321], m, m, decay=0.0, use_lens=False, seed=5)


def test_lengths_beyond_the_capacity_count_as_full(cuda_lib):
    k, v, q = _keys(1, 3, 50, 64, dtype=torch.float32), _normal(2, 3, 50, 64), _normal(3, 3, 2, 64)
    out, score = cuda_lib.attn_scored(k, v, q, lens=_lens([50, 51, -1]))
    full, full_score = cuda_lib.attn_scored(k, v, q)
    assert torch.equal(out[:2], full[:2]) and torch.equal(score[:2], full_score[:2])
    assert not out[2].any() and not score[2].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 70])
def test_scores_in_place_and_one_query_without_its_dimension(cuda_lib, dtype, m):
    """A serving loop's call: the scores that it keeps are updated where they are, and repeated calls add up."""
    t = TYPES[dtype]
    k, v, q = _keys(1, 4, 333, 128, dtype=t), _normal(2, 4, 333, 128, dtype=t), _normal(3, 4, 4, m, 128, dtype=t)
    score = torch.zeros(4, 333, device="cuda")
    q = q[:, :, 0].contiguous() if m == 1 else q
    for call in range(3):
        out, got = cuda_lib.attn_scored(k, v, q, score=score)
        assert got is score and out.shape == q.shape
    # every counted query gives each head's row weight 1 in all; sums of 333 terms of which none is off by more than 1e-5
    assert torch.allclose(score.sum(1), torch.full((4,), 3.0 * 4 * m, device="cuda"), rtol=1e-4)
    once = cuda_lib.attn_scored(k, v, q)[1]
    assert torch.allclose(score, 3 * once, rtol=1e-5, atol=1e-12)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 100])
def test_extreme_logits(cuda_lib, dtype, m):
    """Logits of thousands in either sign, a maximum that comes last, equal rows, zero queries."""
    t, d, n = TYPES[dtype], 64, 500
    k = _keys(5, 3, n, d, dtype=torch.float32)
    k[0] *= torch.linspace(0.0, 30.0, n, device="cuda")[:, None]
    k[1] = k[1, :1]
    k, v, q = k.to(t), _normal(6, 3, n, d, dtype=t), _normal(7, 3, 4, m, d, dtype=t)
    q[2] = 0
    out, score = cuda_lib.attn_scored(k, v, q)
    for s in range(3):
        ref, got, tol, score_tol = scored(q[s], k[s], v[s], n, None, m, 1.0)
        _near(out[s], ref, tol, s)
        _near(score[s], got, score_tol, s)


# ---------------------------------------------------------------------------------------------- eviction

def _check_evict(bk, dtype, d, cap, lens, keep, first, recent, *, kind="mixed", with_pos=True, in_place=False, seed=0, cap_out=None):
    t, S = TYPES[dtype], len(lens)
    k, v = _normal(seed, S, cap, d, dtype=t), _normal(seed + 1, S, cap, d, dtype=t)
    score = torch.exp(2 * _normal(seed + 2, S, cap))
    if kind == "equal":
        score[:] = 0.25
    elif kind == "mixed":                                  # many ties, every kind of value
        u = torch.rand(S, cap, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
        score[u < 0.3] = 0.0
        score[u < 0.2] = -0.0
        score[(u > 0.4) & (u < 0.5)] = 1.5
        score[(u > 0.5) & (u < 0.53)] = math.nan
        score[(u > 0.53) & (u < 0.55)] = math.inf
        score[(u > 0.55) & (u < 0.58)] = -math.inf
        score[(u > 0.58) & (u < 0.65)] *= -1
    pos = torch.stack([torch.randperm(2 * cap, generator=torch.Generator().manual_seed(seed + s))[:cap] for s in range(S)]).to(torch.int32).cuda()
    pos = pos if with_pos else None
    where = [keep_rows(score[s].tolist(), pos[s].tolist() if with_pos else range(cap), n, keep, first, recent) for s, n in enumerate(lens)]
    was = [k.clone(), v.clone(), score.clone(), pos.clone() if with_pos else None]
    if in_place:
        n_out = cap
        got = bk.cache_evict(k, v, score, keep, lens=_lens(lens), pos=pos, n_first=first, n_recent=recent, in_place=True)
        assert got["k"] is k and got["score"] is score and got["pos"] is pos
    else:
        n_out = cap_out or min(keep, cap)
        out = {"k": torch.full((S, n_out, d), 7.0, dtype=t, device="cuda"), "v": torch.full((S, n_out, d), 8.0, dtype=t, device="cuda"),
               "score": torch.full((S, n_out), 9.0, device="cuda"), "pos": torch.full((S, n_out), -7, dtype=torch.int32, device="cuda"),
               "lens": torch.full((S,), -1, dtype=torch.int32, device="cuda")}
        got = bk.cache_evict(k, v, score, keep, lens=_lens(lens), pos=pos, n_first=first, n_recent=recent, out=out)
        assert got is out
        assert torch.equal(k, was[0]) and torch.equal(v, was[1])
    assert got["lens"].tolist() == [len(w) for w in where]
    for s, rows in enumerate(where):
        at = torch.tensor(rows, dtype=torch.long, device="cuda")
        n = len(rows)
        for name, old, fill in (("k", was[0], 7.0), ("v", was[1], 8.0), ("score", was[2], 9.0), ("pos", was[3], -7)):
            if got[name] is None:
                continue
            want = old[s][at] if old is not None else at.int()
            assert torch.equal(torch.nan_to_num(got[name][s, :n].float(), 123.0), torch.nan_to_num(want.float(), 123.0)), (name, s)
            if not in_place:
                assert bool((got[name][s, n:] == fill).all()), (name, s)
            else:                                          # rows behind the last are as they were
                assert torch.equal(torch.nan_to_num(got[name][s, n:].float(), 5.0), torch.nan_to_num(old[s, n:].float(), 5.0)), (name, s)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,d,cap,lens,keep,first,recent", [
    ("bf16", 128, 100, [100, 99, 50, 51, 49, 1, 0, 77], 50, 4, 10), ("fp32", 64, 513, [513, 512, 300], 512, 0, 0), ("fp32", 128, 9000, [9000, 8999, 4097], 1000, 3, 64),
    ("bf16", 64, 1, [1, 0], 1, 0, 1), ("bf16", 64, 40000, [40000, 33333], 39999, 1, 1), ("bf16", 128, 5000, [5000, 1234], 1, 0, 0), ("bf16", 64, 300, [300, 200], 1, 0, 1),
    ("fp32", 64, 33000, [33000, 32, 16500], 12345, 8, 200), ("bf16", 128, 64, [64, 30], 100, 10, 20), ("bf16", 64, 2000, [2000, 1999], 70, 30, 40),
])
def test_eviction(cuda_lib, dtype, d, cap, lens, keep, first, recent, in_place):
    _check_evict(cuda_lib, dtype, d, cap, lens, keep, first, recent, in_place=in_place, seed=cap)


@pytest.mark.parametrize("in_place", [False, True])
def test_eviction_of_equal_scores_and_without_positions(cuda_lib, in_place):
    _check_evict(cuda_lib, "bf16", 64, 5000, [5000, 4000, 10], 600, 4, 100, kind="equal", in_place=in_place)
    _check_evict(cuda_lib, "fp32", 64, 700, [700, 650], 600, 4, 100, with_pos=False, in_place=in_place)
    _check_evict(cuda_lib, "fp32", 64, 20000, [20000, 0], 7, 0, 7, kind="spread", with_pos=False, in_place=in_place)


def test_eviction_with_equal_positions(cuda_lib):
    """Positions that occur more than once, all of them the newest: the lowest rows stay."""
    k, v, score = _normal(1, 2, 300, 64), _normal(2, 2, 300, 64), _normal(3, 2, 300)
    pos = torch.full((2, 300), 7, dtype=torch.int32, device="cuda")
    for keep in (50, 299):
        got = cuda_lib.cache_evict(k, v, score, keep, pos=pos, n_recent=1)
        assert torch.equal(got["k"], k[:, :keep]) and torch.equal(got["v"], v[:, :keep]) and torch.equal(got["score"], score[:, :keep])
        assert got["lens"].tolist() == [keep, keep]


@pytest.mark.parametrize("in_place", [False, True])
def test_more_streams_than_ctas_at_once(cuda_lib, in_place):
    """One row over a budget and short streams, by more clusters than the device holds."""
    _check_evict(cuda_lib, "bf16", 64, 33, [33 - s % 3 for s in range(700)], 32, 2, 8, in_place=in_place)
    _check_evict(cuda_lib, "fp32", 128, 2500, [2500 - s % 2 for s in range(200)], 2499, 2, 8, kind="spread", in_place=in_place)


def test_eviction_into_a_larger_cache(cuda_lib):
    _check_evict(cuda_lib, "bf16", 128, 300, [300, 20], 100, 4, 10, cap_out=250)
    _check_evict(cuda_lib, "bf16", 128, 80, [80, 20], 100, 4, 10, cap_out=100)


def test_eviction_from_a_cache_too_long_to_stage(cuda_lib):
    """A cluster's shared memory holds the keys and positions of 196608 rows; longer caches read them again."""
    _check_evict(cuda_lib, "bf16", 64, 200003, [200003], 1000, 2, 50, seed=9)
    _check_evict(cuda_lib, "bf16", 64, 200003, [200000], 150000, 2, 50, with_pos=False, in_place=True, seed=9)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind,cap", [("mixed", 97), ("equal", 97), ("mixed", 5000), ("spread", 33000), ("equal", 20000)])
def test_one_row_over_the_budget(cuda_lib, kind, cap, in_place):
    """Every token's eviction: one row goes, at most one moves; streams that are not over keep all."""
    _check_evict(cuda_lib, "bf16", 64, cap, [cap, cap - 1, cap, cap // 2], cap - 1, 4, 16, kind=kind, in_place=in_place, seed=cap)
    _check_evict(cuda_lib, "fp32", 128, cap, [cap] * 3, cap - 1, 0, 0, kind=kind, with_pos=False, in_place=in_place, seed=cap + 1)
    _check_evict(cuda_lib, "bf16", 128, cap, [cap - 2, cap - 3], cap - 3, 2, 3, kind=kind, in_place=in_place, seed=cap + 2)      # room for two moves more


def test_many_streams_at_once(cuda_lib):
    _check_evict(cuda_lib, "bf16", 64, 90, [(7 * s) % 91 for s in range(500)], 40, 2, 8)


# ---------------------------------------------------------------------------------------------- shared prefix

def _check_prefix(bk, dtype, d, B, H, g, P, cap, lens, weighted, seed=0):
    t = TYPES[dtype]
    pk, pv = _keys(seed, H, P, d, dtype=t), _normal(seed + 1, H, P, d, dtype=t)
    k, v = _keys(seed + 2, B, H, cap, d, dtype=t) if cap else None, _normal(seed + 3, B, H, cap, d, dtype=t) if cap else None
    q = _normal(seed + 4, B, H * g, d, dtype=t)
    w = None
    if weighted:
        w = torch.exp2(torch.floor(3 * torch.rand(H, P, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))) * 1.0
        w[:, P // 3:P // 2] = 0.0                          # rows that count as absent, whatever they hold
        pk[:, P // 3:P // 2] = math.nan
        pv[:, P // 3:P // 2] = math.inf
    if cap:
        for b, n in enumerate(lens or []):
            k[b, :, n:] = math.nan
            v[b, :, n:] = math.nan
    out = bk.decode_attn_prefix(pk, pv, k, v, q, lens=_lens(lens) if lens else None, weight=w)
    for b in range(B):
        n = lens[b] if lens else cap
        for h in range(H):
            kk = torch.nan_to_num(torch.cat([pk[h], k[b, h, :n]] if cap else [pk[h]]))
            vv = torch.nan_to_num(torch.cat([pv[h], v[b, h, :n]] if cap else [pv[h]]), posinf=0.0)
            ww = torch.cat([w[h] if weighted else torch.ones(P, device="cuda"), torch.ones(n if cap else 0, device="cuda")])
            qq = q[b, h * g:(h + 1) * g]
            ref, _, tol, _ = attention(qq, kk, vv, torch.ones(g, kk.shape[0], dtype=torch.bool, device="cuda"), ww, rounded_p=True)
            _near(out[b, h * g:(h + 1) * g], ref, tol, (b, h, n))


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,B,H,g,P,cap,lens", [
    (128, 3, 2, 4, 1000, 77, [77, 0, 40]), (64, 1, 1, 1, 1, 1, [0]), (64, 5, 3, 3, 129, 300, [300, 1, 64, 65, 0]), (128, 2, 2, 8, 5000, 0, None),
    (128, 40, 1, 5, 640, 130, [(17 * b) % 131 for b in range(40)]), (64, 33, 2, 4, 257, 20, None), (128, 17, 2, 7, 2111, 64, [64] * 17), (128, 70, 2, 4, 300, 10, None),
    (64, 130, 1, 6, 200, 33, [b % 34 for b in range(130)]), (128, 9, 8, 2, 128, 128, [128] * 9),
])
def test_shared_prefix(cuda_lib, dtype, d, B, H, g, P, cap, lens, weighted):
    _check_prefix(cuda_lib, dtype, d, B, H, g, P, cap, lens, weighted, seed=B + P)


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,B,H,g,P,cap,lens", [
    (128, 2, 2, 3, 1500, 40, [0, 33]), (64, 1, 3, 8, 3001, 0, None), (128, 4, 1, 2, 33, 2000, [2000, 1, 0, 777]), (64, 300, 2, 1, 127, 3, [b % 4 for b in range(300)]),
])
def test_prefix_much_longer_or_shorter_than_the_own_rows(cuda_lib, dtype, d, B, H, g, P, cap, lens, weighted):
    _check_prefix(cuda_lib, dtype, d, B, H, g, P, cap, lens, weighted, seed=B + P)


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("d,B,H,g,P,cap", [(128, 200, 4, 3, 900, 150), (64, 20, 4, 5, 3000, 900), (128, 33, 2, 4, 5000, 1300), (64, 700, 1, 2, 1500, 60)])
def test_own_rows_beside_the_prefix(cuda_lib, d, B, H, g, P, cap, weighted):
    """Own rows that are read while the prefix's products are formed, call after call in the same memory, with lengths of every kind."""
    for call in range(3):
        _check_prefix(cuda_lib, "bf16", d, B, H, g, P, cap, [(31 * b * (call + 1)) % (cap + 1) for b in range(B)], weighted, seed=B + call)


def test_own_rows_beside_the_prefix_captured(cuda_lib):
    """The same in a graph, several calls in a row, replayed on other queries, rows and lengths than were captured."""
    B, H, g, P, cap, d = 200, 4, 3, 3000, 400, 128
    t = torch.bfloat16

    def inputs(seed):
        return [_keys(seed, H, P, d, dtype=t), _normal(seed + 1, H, P, d, dtype=t), _keys(seed + 2, B, H, cap, d, dtype=t), _normal(seed + 3, B, H, cap, d, dtype=t),
                _normal(seed + 4, B, H * g, d, dtype=t), _lens([(seed + 29 * b) % (cap + 1) for b in range(B)])]

    def calls(x):
        first = cuda_lib.decode_attn_prefix(*x[:5], lens=x[5])
        second = cuda_lib.decode_attn_prefix(*x[:4], first, lens=x[5])         # its queries are what the first call wrote
        return [first, second, cuda_lib.decode_attn_prefix(*x[:4], second, lens=x[5])]

    a, b = inputs(1), inputs(50)
    want = [[y.clone() for y in calls(x)] for x in (a, b)]
    torch.cuda.synchronize()
    held, graph = [x.clone() for x in a], torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls(held)
    for source, w in ((b, want[1]), (a, want[0]), (b, want[1])):
        for x, y in zip(held, source):
            x.copy_(y)
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, w))
    for _ in range(10):
        again = calls(a)
    assert all(torch.equal(x, y) for x, y in zip(again, want[0]))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B", [1, 40, 200])
def test_prefix_whose_rows_are_all_absent(cuda_lib, dtype, B):
    """Weights of zero everywhere, over rows that hold NaN: the own rows alone, and zeros where there are none."""
    t, H, g, P, cap, d = TYPES[dtype], 2, 4, 500, 30, 128
    pk, w = torch.full((H, P, d), math.nan, dtype=t, device="cuda"), torch.zeros(H, P, device="cuda")
    k, v, q = _keys(1, B, H, cap, d, dtype=t), _normal(2, B, H, cap, d, dtype=t), _normal(3, B, H * g, d, dtype=t)
    lens = [0] + [cap] * (B - 1)
    out = cuda_lib.decode_attn_prefix(pk, pk, k, v, q, lens=_lens(lens), weight=w)
    assert not out[0].any()
    for b in range(1, B, 13):
        for h in range(H):
            qq = q[b, h * g:(h + 1) * g]
            ref, _, tol, _ = attention(qq, k[b, h], v[b, h], torch.ones(g, cap, dtype=torch.bool, device="cuda"), rounded_p=True)
            _near(out[b, h * g:(h + 1) * g], ref, tol, (b, h))
    alone = cuda_lib.decode_attn_prefix(pk, pk, None, None, q, weight=w)
    assert bool((alone == 0).all())


# ---------------------------------------------------------------------------------------------- as they are used

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_prompt_then_budgeted_decoding(cuda_lib, dtype):
    """A prompt is attended and scored, cut to a budget, and decoded token by token with one eviction in place per token; every step
    against the definitions on the same bytes."""
    bk, t, S, g, d, n, budget, first, recent = cuda_lib, TYPES[dtype], 4, 4, 128, 300, 96, 4, 16
    k, v, q = _keys(1, S, n, d, dtype=t), _normal(2, S, n, d, dtype=t), _normal(3, S, g, n, d, dtype=t)
    out, score = bk.attn_scored(k, v, q, n_scored=32)
    ref, got, tol, score_tol = scored(q[1], k[1], v[1], n, None, 32, 1.0)
    _near(out[1], ref, tol, "prompt")
    _near(score[1], got, score_tol, "prompt scores")
    room = {"k": torch.zeros(S, budget + 1, d, dtype=t, device="cuda"), "v": torch.zeros(S, budget + 1, d, dtype=t, device="cuda"),
            "score": torch.zeros(S, budget + 1, device="cuda"), "pos": torch.zeros(S, budget + 1, dtype=torch.int32, device="cuda"),
            "lens": torch.zeros(S, dtype=torch.int32, device="cuda")}
    c = bk.cache_evict(k, v, score, budget, n_first=first, n_recent=recent, out=room)
    for s in range(S):
        rows = keep_rows(score[s].tolist(), range(n), n, budget, first, recent)
        assert c["pos"][s, :budget].tolist() == rows and torch.equal(c["k"][s, :budget], k[s][rows])
    for step in range(6):
        c["k"][:, budget] = _keys(50 + step, S, 1, d, dtype=t)[:, 0]
        c["v"][:, budget] = _normal(60 + step, S, d, dtype=t)
        c["pos"][:, budget], c["score"][:, budget], c["lens"][:] = n + step, 0.0, budget + 1
        was = {name: x.clone() for name, x in c.items()}
        qs = _normal(70 + step, S, g, d, dtype=t)
        out, _ = bk.attn_scored(c["k"], c["v"], qs, lens=c["lens"], score=c["score"], decay=0.9)
        bk.cache_evict(c["k"], c["v"], c["score"], budget, lens=c["lens"], pos=c["pos"], n_first=first, n_recent=recent, in_place=True)
        for s in range(S):
            ref, got, tol, score_tol = scored(qs[s][:, None], was["k"][s], was["v"][s], budget + 1, was["score"][s], 1, 0.9)
            _near(out[s], ref[:, 0], tol[:, 0], (step, s))
            kept = [was["pos"][s].tolist().index(p) for p in c["pos"][s, :budget].tolist()]
            _near(c["score"][s, :budget], got[kept], score_tol[kept], (step, s, "scores"))
            assert len(set(kept)) == budget and torch.equal(c["k"][s, :budget], was["k"][s][kept]) and torch.equal(c["v"][s, :budget], was["v"][s][kept])
            gone = (set(range(budget + 1)) - set(kept)).pop()
            safe = (was["pos"][s] < first) | (was["pos"][s] > n + step - recent)
            assert not bool(safe[gone]) and bool((got[gone] <= got[~safe] + 2 * score_tol[~safe]).all())
        assert c["lens"].tolist() == [budget] * S


def test_evicted_rows_in_a_context(cuda_lib):
    """What an eviction keeps goes on as a context's uncompressed rows, positions included."""
    bk, B, H, g, d, n, budget = cuda_lib, 2, 2, 4, 128, 500, 200
    k, v, q = _keys(1, B * H, n, d, dtype=torch.bfloat16), _normal(2, B * H, n, d, dtype=torch.bfloat16), _normal(3, B * H, g, n, d, dtype=torch.bfloat16)
    c = bk.cache_evict(k, v, bk.attn_scored(k, v, q)[1], budget, n_first=4, n_recent=64)
    ctx = bk.Context(n_seqs=B, n_kv_heads=H, n_q_heads=H * g, head_dim=d, dtype="bf16", block=64, levels=0, max_tokens=1024)
    ctx.cache_load_level(0, 0, c["k"].view(B, H, budget, d), c["v"].view(B, H, budget, d), c["pos"].view(B, H, budget))
    qs = _normal(4, B, H * g, d, dtype=torch.bfloat16)
    out = ctx.decode_attn(0, qs).view(B * H, g, d)
    assert torch.equal(ctx.cache_view(0, 0, 1)[3], c["pos"][1])
    here, _ = bk.attn_scored(c["k"], c["v"], qs.view(B * H, g, d))
    for s in range(B * H):
        ref, _, tol, _ = attention(qs.view(B * H, g, d)[s], c["k"][s], c["v"][s], torch.ones(g, budget, dtype=torch.bool, device="cuda"), rounded_p=True)
        _near(out[s], ref, tol, s)
        _near(here[s], ref, tol, s)
    ctx.close()


def test_compressed_prefix_shared_by_a_batch(cuda_lib):
    """A document compressed once by BalanceKV is the prefix of a batch: rows and weights as the context's view gives them."""
    bk, H, g, d, n, B = cuda_lib, 2, 4, 128, 1500, 6
    ctx = bk.Context(n_seqs=1, n_kv_heads=H, n_q_heads=H * g, head_dim=d, dtype="bf16", block=256, levels=2, max_tokens=n)
    ctx.stream_append_layer(0, _keys(1, 1, H, n, d, dtype=torch.bfloat16), _normal(2, 1, H, n, d, dtype=torch.bfloat16))
    ctx.compress()
    views = [ctx.cache_view(0, 0, h) for h in range(H)]
    pk, pv, w = (torch.stack([view[i] for view in views]) for i in range(3))
    q = _normal(3, B, H * g, d, dtype=torch.bfloat16)
    alone = bk.decode_attn_prefix(pk, pv, None, None, q, weight=w)
    one = torch.cat([ctx.decode_attn(0, q[b:b + 1].contiguous()) for b in range(B)])
    k, v = _keys(4, B, H, 50, d, dtype=torch.bfloat16), _normal(5, B, H, 50, d, dtype=torch.bfloat16)
    both = bk.decode_attn_prefix(pk, pv, k, v, q, lens=_lens([50, 0, 3, 49, 50, 1]), weight=w)
    for b, m in enumerate([50, 0, 3, 49, 50, 1]):
        for h in range(H):
            hs = slice(h * g, h * g + g)
            ref, _, tol, _ = attention(q[b, hs], pk[h], pv[h], torch.ones(g, pk.shape[1], dtype=torch.bool, device="cuda"), w[h], rounded_p=True)
            _near(alone[b, hs], ref, tol, (b, h))
            _near(one[b, hs], ref, tol, (b, h, "context"))
            ref, _, tol, _ = attention(q[b, hs], torch.cat([pk[h], k[b, h, :m]]), torch.cat([pv[h], v[b, h, :m]]),
                                       torch.ones(g, pk.shape[1] + m, dtype=torch.bool, device="cuda"), torch.cat([w[h], torch.ones(m, device="cuda")]), rounded_p=True)
            _near(both[b, hs], ref, tol, (b, h, m))
    ctx.close()


def _pass(bk, x, stream=None):
    out, score = bk.attn_scored(x["k"], x["v"], x["q"], lens=x["lens"], score=x["score"], score_out=x["score_out"], stream=stream)
    one, _ = bk.attn_scored(x["k"], x["v"], x["q"][:, :, -1].contiguous(), lens=x["lens"], n_scored=0, stream=stream)
    kept = bk.cache_evict(x["k"], x["v"], score, 100, lens=x["lens"], n_first=2, n_recent=10, stream=stream)
    ahead = bk.decode_attn_prefix(x["k"], x["v"], x["own_k"], x["own_v"], x["own_q"], stream=stream)
    return [out, score, one, *kept.values(), ahead]


def _inputs(seed, dtype):
    t = TYPES[dtype]
    return {"k": _keys(seed, 3, 400, 128, dtype=t), "v": _normal(seed + 1, 3, 400, 128, dtype=t), "q": _normal(seed + 2, 3, 4, 70, 128, dtype=t),
            "lens": _lens([400, 123, 64]), "score": _normal(seed + 3, 3, 400).abs(), "score_out": torch.zeros(3, 400, device="cuda"),
            "own_k": _keys(seed + 4, 5, 3, 30, 128, dtype=t), "own_v": _normal(seed + 5, 5, 3, 30, 128, dtype=t), "own_q": _normal(seed + 6, 5, 12, 128, dtype=t)}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_same_bits_every_time_and_captured(cuda_lib, dtype):
    """Twice the same call gives the same bits, and so does a captured pass, replayed on inputs that changed behind its back."""
    a, b = _inputs(1, dtype), _inputs(30, dtype)
    b["lens"] = _lens([1, 0, 333])
    want_a, want_b = ([x.clone() for x in _pass(cuda_lib, y)] for y in (a, b))
    for x, y in zip(_pass(cuda_lib, a), want_a):
        assert torch.equal(x, y)
    held = {name: x.clone() for name, x in a.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _pass(cuda_lib, held)
    for source, want in ((b, want_b), (a, want_a), (b, want_b)):
        for name in held:
            held[name].copy_(source[name] if name != "score_out" else torch.zeros_like(held[name]))
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y)


@pytest.mark.parametrize("raw", [False, True])
def test_on_a_stream_of_its_own(cuda_lib, raw):
    """Calls on another stream order after what that stream waits for, and their workspaces are not handed on to other work."""
    x = _inputs(5, "bf16")
    want = [y.clone() for y in _pass(cuda_lib, x)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        got = _pass(cuda_lib, x, stream=side.cuda_stream if raw else side)
        noise = [torch.full((1 << 20,), math.nan, device="cuda") for _ in range(4)]
        del noise
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_calls_that_overlap(cuda_lib, dtype):
    """Two streams whose calls run at once, eagerly and as two captured graphs: each has workspaces of its own."""
    inputs = [_inputs(3, dtype), _inputs(40, dtype)]
    inputs[1]["lens"] = _lens([17, 400, 0])
    want = [[y.clone() for y in _pass(cuda_lib, x)] for x in inputs]
    sides = [torch.cuda.Stream() for _ in inputs]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(20):
        for i in (0, 1):
            got[i] = _pass(cuda_lib, inputs[i], stream=sides[i])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(g, w))
    graphs, held = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for graph, x in zip(graphs, inputs):
        with torch.cuda.graph(graph):
            held.append(_pass(cuda_lib, x))
    for _ in range(20):
        for i in (0, 1):
            with torch.cuda.stream(sides[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    for g, w in zip(held, want):
        assert all(torch.equal(x, y) for x, y in zip(g, w))


@pytest.mark.parametrize("dtype,B,cap", [("bf16", 40, 700), ("fp32", 40, 700), ("bf16", 2, 300), ("fp32", 2, 300)])
def test_steps_without_waiting(cuda_lib, dtype, B, cap):
    """A serving loop that never waits: what a step writes (rows, lens, queries, scores) is what the next one's launches see, early as they
    begin.  The same steps with a wait behind every call give the same bits."""
    t, H, g, d = TYPES[dtype], 8, 4, 128
    S = B * H
    pk, pv = _keys(1, H, 500, d, dtype=t), _normal(2, H, 500, d, dtype=t)
    rows, queries = _keys(3, 25, S, d, dtype=t), _normal(4, 25, S, g, d, dtype=t)

    def steps(wait):
        k, v = _keys(5, S, cap, d, dtype=t), _normal(6, S, cap, d, dtype=t)
        score, lens = torch.zeros(S, cap, device="cuda"), _lens([cap - 20 - 7 * (s % 9) for s in range(S)])
        pos, q, results = torch.arange(cap, dtype=torch.int32, device="cuda").repeat(S, 1), torch.empty(S, g, d, dtype=t, device="cuda"), []
        at = torch.arange(S, device="cuda")
        for i in range(25):
            k[at, lens.long()] = rows[i]
            v[at, lens.long()] = rows[i].flip(-1)
            score[at, lens.long()] = 0
            pos[at, lens.long()] = cap + i
            lens += 1
            q.copy_(queries[i])
            out, _ = cuda_lib.attn_scored(k, v, q, lens=lens, score=score, decay=0.9)
            if wait:
                torch.cuda.synchronize()
            cuda_lib.cache_evict(k, v, score, cap - 15, lens=lens, pos=pos, n_first=4, n_recent=20, in_place=True)
            if wait:
                torch.cuda.synchronize()
            ahead = cuda_lib.decode_attn_prefix(pk, pv, k.view(B, H, cap, d), v.view(B, H, cap, d), q.view(B, H * g, d), lens=lens[::H].contiguous())
            if wait:
                torch.cuda.synchronize()
            results += [out, ahead]
        return [*results, k, v, score, lens, pos]

    for a, b in zip(steps(True), steps(False)):
        assert torch.equal(a, b)


def test_refusals_with_a_device(cuda_lib):
    k, q, score = torch.zeros(2, 10, 64, device="cuda"), torch.zeros(2, 3, 64, device="cuda"), torch.zeros(2, 10, device="cuda")
    bk = cuda_lib
    with pytest.raises(ValueError, match="contiguous"):
        bk.attn_scored(k, torch.zeros(2, 64, 10, device="cuda").transpose(1, 2), q)
    with pytest.raises(ValueError, match="lens"):
        bk.attn_scored(k, k, q, lens=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="lens"):
        bk.attn_scored(k, k, q, lens=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(bk.BalanceKVError, match="invalid"):
        bk.attn_scored(k, k, q, n_scored=2)
    with pytest.raises(bk.BalanceKVError, match="invalid"):
        bk.cache_evict(k, k.clone(), score, 5, n_first=3, n_recent=3)
    with pytest.raises(bk.BalanceKVError, match="invalid"):
        bk.cache_evict(k, k.clone(), score, 5, out={"k": k, "v": k.clone(), "score": score.clone()})
    with pytest.raises(ValueError, match="n_keep"):
        bk.cache_evict(k, k.clone(), score, 0)
    with pytest.raises(bk.BalanceKVError, match="invalid"):
        bk.attn_scored(torch.zeros(2 * 10 * 64 + 1, device="cuda")[1:].view(2, 10, 64), k, q)
