"""Attention over the 8-bit cache where scores, scales or the factors between them are at the ends
of their ranges, through every form of it (clusters, the shared line, tcgen05 tiles)."""
import numpy as np
import pytest

import kv8_ref as R
from parity import has_gpu
from test_gpu_kv8 import _cache, _ints, _values

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a CUDA GPU")]

HEADS, KVH, HD = 4, 2, 128
# Tiles of 16 rows, in clusters (caches of 512 and 1024 positions) and on the shared line (2560); and
# tcgen05 tiles, with one accumulator (2 M = 80 rows a KV head) and with two (260).
SMALL = [("bf16", 2, 512), ("bf16", 2, 2560), ("bf16", 40, 1024), ("f32", 2, 1024), ("f32", 40, 2560)]
WIDE = [("bf16", 40, 2560), ("bf16", 130, 2560)]
FORMS = SMALL + WIDE


def _torch():
    import torch
    return torch


def _appended(k, v, seq):
    """A cache of k, v [positions, KVH, HD] and its values in float64."""
    c = _cache(KVH, HD, seq)
    c.append(k[None].contiguous(), v[None].contiguous(), _ints([0]))
    return c, _held(c)


def _held(c):
    return [_values(t) * np.repeat(s.cpu().numpy().astype(np.float64), 64, -1)[..., None]
            for t, s in ((c.k, c.k_scale), (c.v, c.v_scale))]


def _check(c, vals, q, pos, window=0, unit=0.0):
    """unit: the largest value scale in sight, where value scales are far apart.  A probability
    times its value's scale over that unit is an f16 number, off by 2^-25 (half of the smallest
    one's distance) where it is below 2^-14.  The row's largest probability stands there at 2^7 or
    more, and so does their sum; a code is 448 at most: each key's part of the output is off by up
    to 2^-25 448 unit / 2^7."""
    M = q.shape[1]
    got = c.attention(q, _ints([pos]), window=window)
    c.check()
    ref = np.zeros(got.shape)
    mass, size = R.attend(_values(q), vals[0], vals[1], [pos], [M], [0], window, ref)
    tol = R.attend_bound(ref, mass, size, HD, pos + M, got.dtype == _torch().bfloat16)
    tol += (pos + M) * 2.0 ** -32 * 448 * unit
    out = _values(got)
    assert np.isfinite(out).all(), np.argwhere(~np.isfinite(out))[:5]
    assert (np.abs(out - ref) <= tol).all(), np.abs(out - ref).max()


@pytest.mark.parametrize("dtype,M,seq", FORMS)
@pytest.mark.parametrize("how", ["some zeros", "all zeros", "scale of 0"])
def test_zero_keys_and_zero_queries(dtype, M, seq, how):
    """Blocks of zero keys (scale 2^-120, or 0 in a cache that was filled by hand) where rows see
    a part of them, under queries of zeros and small ones: the factor of a score underflows, and
    the keys that a row does not see stay out of it."""
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(41)
    x = torch.randn(400, 2 * KVH, HD, generator=g, device="cuda")
    k, v = x[:, :KVH], x[:, KVH:]
    zero = torch.zeros(400, dtype=torch.bool, device="cuda")
    zero[64:128] = zero[192:256] = True
    if how == "all zeros":
        zero[:] = True
    if how != "scale of 0":
        k[zero] = 0
    c, vals = _appended(k, v, seq)
    if how == "scale of 0":
        c.k_scale[:, :, 1] = c.k_scale[:, :, 3] = 0
        vals = _held(c)
    q = torch.randn(1, M, HEADS, HD, generator=g, device="cuda")
    q[:, 1::4] = 0
    q[:, 2::4] *= 1e-6
    q[:, 3::8] *= 2.0 ** -40
    q = q.to(torch.float32 if dtype == "f32" else torch.bfloat16)
    for pos, window in ((70, 0), (70, 50), (200, 0), (200, 70)):
        _check(c, vals, q, pos, window)


def _direction(M, dtype, size):
    """Queries along the first axis alone."""
    torch = _torch()
    q = torch.zeros(1, M, HEADS, HD, device="cuda")
    q[..., 0] = size
    return q.to(torch.float32 if dtype == "f32" else torch.bfloat16)


@pytest.mark.parametrize("dtype,M,seq", SMALL)
def test_large_scores_in_small_tiles(dtype, M, seq):
    _large_scores(dtype, M, seq)


@pytest.mark.parametrize("dtype,M,seq", WIDE)
def test_large_scores_in_wide_tiles(dtype, M, seq):
    _large_scores(dtype, M, seq)


def _large_scores(dtype, M, seq):
    """Scores whose distance in fp32 is many powers of two: a softmax is a choice there, and its
    outputs stay between the values.  Values that are the same for every key come out as they are
    whatever the probabilities; and one key whose score stands out by half its size is taken alone,
    from both signs, as the running maximum grows key by key."""
    torch = _torch()
    bf16 = dtype == "bf16"
    g = torch.Generator(device="cuda").manual_seed(43)
    k = torch.randn(400, KVH, HD, generator=g, device="cuda")
    w = torch.randn(1, KVH, HD, generator=g, device="cuda").expand(400, KVH, HD)
    same, (_, wv) = _appended(k, w, seq)
    q0 = torch.randn(1, M, HEADS, HD, generator=g, device="cuda")
    want = np.repeat(wv[0, :, 0], HEADS // KVH, 0)[None, None]
    v = torch.randn(400, KVH, HD, generator=g, device="cuda")
    pos = 390 - M - 50
    for e in [*range(12, 34), 60, 90]:
        q = (q0 * 2.0 ** e).to(torch.bfloat16 if bf16 else torch.float32)
        out = _values(same.attention(q, _ints([pos])))
        assert np.isfinite(out).all(), (e, np.argwhere(~np.isfinite(out))[:3])
        # (the scores' errors move probabilities, but here not the output)
        tol = R.attend_bound(want, np.abs(want), np.zeros(want.shape[:3]), HD, 400, bf16)
        assert (np.abs(out - want) <= tol).all(), e
    for sign in (1.0, -1.0):
        keys = torch.zeros(400, KVH, HD, device="cuda")
        keys[:, :, 0] = 1.0 if sign > 0 else -32.0
        peaks = [10, 70, 129, 150, pos + M // 2]
        for i, p in enumerate(peaks):
            keys[p, :, 0] = 2.0 ** (i + 1) if sign > 0 else -(2.0 ** (4 - i))
        c, vals = _appended(keys, v, seq)
        for e in (14, 18, 22, 24, 25, 26, 27, 28, 31, 40):
            out = _values(c.attention(_direction(M, dtype, 2.0 ** e), _ints([pos])))
            for m in range(M):
                at = peaks[-1] if pos + m >= peaks[-1] else peaks[-2]
                ref = np.repeat(vals[1][0, :, at], HEADS // KVH, 0)
                tol = R.attend_bound(ref, np.abs(ref), np.zeros(HEADS), HD, 400, bf16)
                assert (np.abs(out[0, m] - ref) <= tol).all(), (sign, e, m)


@pytest.mark.parametrize("dtype,M,seq", FORMS)
def test_a_factor_beyond_fp32_leaves_zero_scores_zero(dtype, M, seq):
    """Zero keys that share a block with huge ones behind a row, under huge queries: the row's
    scores are zeros, although scale times unit is past the largest number."""
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(47)
    x = torch.randn(320, 2 * KVH, HD, generator=g, device="cuda")
    last = 70 + M - 1
    k, v = x[:, :KVH] * 2.0 ** 60, x[:, KVH:]
    k[:last + 1] = 0
    assert last % 64 != 63
    c, vals = _appended(k, v, seq)
    q = (torch.randn(1, M, HEADS, HD, generator=g, device="cuda") * 2.0 ** 100).to(
        torch.float32 if dtype == "f32" else torch.bfloat16)
    _check(c, vals, q, 70)


def test_rows_rolled_back_leave_their_scale():
    """A rejected outlier raises its block's scale for good: the accepted codes in front are rounded
    to it, the next rows stand under it, and only a block written from its start has its own again."""
    torch = _torch()
    c = _cache(KVH, HD, 128)
    ref = [(np.zeros((1, KVH, 128, HD)), np.zeros((1, KVH, 2))) for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(53)
    x = torch.randn(1, 70, 2 * KVH, HD, generator=g, device="cuda")

    def append(rows, pos):
        c.append(rows[:, :, :KVH], rows[:, :, KVH:], _ints([pos]))
        for (codes, scale), y, t, s in zip(ref, (rows[:, :, :KVH], rows[:, :, KVH:]), (c.k, c.v),
                                           (c.k_scale, c.v_scale)):
            R.append(codes, scale, y.cpu().numpy(), [pos], [rows.shape[1]])
            assert np.array_equal(_values(t), codes)
            assert np.array_equal(s.cpu().numpy().astype(np.float64), scale)
        return c.k_scale[0, :, 0].clone(), _values(c.k)[0, :, :10].copy()

    first, codes0 = append(x[:, :10], 0)
    raised, codes1 = append(x[:, 10:13] * 2.0 ** 12, 10)       # drafted
    per = [t.cpu().numpy().astype(np.float64)[:, None, None] for t in (first, raised)]
    assert bool((raised > first).all())
    assert not np.array_equal(codes0 * per[0], codes1 * per[1])  # small values in front are coarser
    kept, codes2 = append(x[:, 10:12], 10)                      # rejected: others in their place
    assert torch.equal(kept, raised) and np.array_equal(codes1, codes2)
    anew, codes3 = append(x[:, :12], 0)
    assert bool((anew < raised).all()) and np.array_equal(
        codes3, R.e4m3_round(x[0, :10, :KVH].permute(1, 0, 2).cpu().numpy().astype(np.float64)
                             / anew.cpu().numpy()[:, None, None]))


@pytest.mark.parametrize("dtype,M,seq", FORMS)
def test_maxima_and_units_that_move(dtype, M, seq):
    """Value scales 2^20 apart both ways, blocks of zero values, and single keys that outweigh all
    others at places where the value scale falls or rises: the running maximum and the output's unit
    move together and apart."""
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(59)
    x = torch.randn(400, 2 * KVH, HD, generator=g, device="cuda")
    k, v = x[:, :KVH], x[:, KVH:]
    v[64:128] = 0
    v[128:192] *= 2.0 ** 20
    v[192:256] *= 2.0 ** -20
    q = torch.randn(1, M, HEADS, HD, generator=g, device="cuda").to(
        torch.float32 if dtype == "f32" else torch.bfloat16)
    unit = q[0].float() / q[0].float().norm(dim=-1, keepdim=True)
    for at, m, h, size in ((3, 0, 0, 40), (100, M - 1, 3, 30), (150, M // 2, 1, 50), (210, 0, 2, 60),
                           (257, M - 1, 0, 60)):
        k[at, h // (HEADS // KVH)] = size * unit[m, h]
    c, vals = _appended(k, v, seq)
    for pos in (62, 140, 255, 399 - M):
        for window in (0, 90):
            seen = c.v_scale[..., max(pos - window, 0) // 64 if window else 0:(pos + M - 1) // 64 + 1]
            _check(c, vals, q, pos, window, float(seen.max()))


@pytest.mark.parametrize("dtype,M,seq", FORMS)
@pytest.mark.parametrize("e", [90, 104, 118])
def test_values_near_the_largest(dtype, M, seq, e):
    """Values of 2^90 to the largest that a cache holds: sums over them stay in range, in the order
    that they are weighed and joined in."""
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(61)
    x = torch.randn(400, 2 * KVH, HD, generator=g, device="cuda")
    v = x[:, KVH:].clamp(-2, 2) * 2.0 ** e
    c, vals = _appended(x[:, :KVH], v, seq)
    q = torch.randn(1, M, HEADS, HD, generator=g, device="cuda").to(
        torch.float32 if dtype == "f32" else torch.bfloat16)
    for pos in (0, 140, 399 - M):
        _check(c, vals, q, pos)
