"""The 8-bit KV cache on the GPU against 64-bit references: appends bit for bit (codes and scales
have one right value each), attention within a bound derived from its roundings (kv8_ref)."""
import numpy as np
import pytest

import kv8_ref as R
from parity import has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a CUDA GPU")]

NAN_CODE = 0x7f


def _torch():
    import torch
    return torch


def _cache(heads, hd, seq, n=1, fill=None):
    from paper_2606_03113_gb300.runtime import KV8Cache
    torch = _torch()
    c = KV8Cache(heads, hd, seq, n_seq=n)
    if fill is not None:
        for t in (c.k, c.v):
            t.view(torch.uint8).fill_(fill)
        c.k_scale.fill_(float("nan"))
        c.v_scale.fill_(float("nan"))
    return c


def _ints(xs):
    torch = _torch()
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _values(t):
    return t.float().cpu().numpy().astype(np.float64)


def _same(a, b):
    return np.array_equal(a, b, equal_nan=True)


# ------------------------------------------------------------------ append

APPENDS = [  # dtype, heads, hd, n, M, seq, appends of (pos, rows)
    ("f32", 4, 64, 1, 5, 128, [([0], [5]), ([5], [5]), ([7], [3])]),
    ("bf16", 8, 128, 1, 1, 192, [([p], [1]) for p in (0, 1, 62, 63, 64, 65, 191)]),
    ("bf16", 2, 128, 3, 17, 256, [([0, 60, 239], [17, 9, 17]), ([3, 69, 200], [0, 17, 1])]),
    ("f32", 3, 128, 2, 200, 448, [([1, 63], [200, 130]), ([190, 0], [200, 1])]),
    ("bf16", 1, 64, 2, 65, 128, [([63, 0], [65, 64]), ([20, 64], [2, 64])]),
    ("bf16", 40, 128, 1, 129, 192, [([63], [129])]),
]


@pytest.mark.parametrize("dtype,heads,hd,n,M,seq,calls", APPENDS)
def test_append_is_exact(dtype, heads, hd, n, M, seq, calls):
    """Codes and scales equal the reference's, over a run of appends that roll back, start in the
    middle of blocks and raise their scales; everything else keeps its bytes."""
    torch = _torch()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    c = _cache(heads, hd, seq, n, fill=0x35)
    ref = [(_values(c.k), c.k_scale.cpu().numpy().astype(np.float64)),
           (_values(c.v), c.v_scale.cpu().numpy().astype(np.float64))]
    g = torch.Generator(device="cuda").manual_seed(M + heads)
    for i, (pos, rows) in enumerate(calls):
        qkv = torch.randn(n, M, 3 * heads, hd, generator=g, device="cuda") * 8.0 ** i
        qkv[:, ::3] *= 0.01
        qkv = qkv.to(dt)
        k, v = qkv[:, :, heads:2 * heads], qkv[:, :, 2 * heads:]
        c.append(k, v, _ints(pos), rows=_ints(rows))
        for (codes, scale), x, t, s in zip(ref, (k, v), (c.k, c.v), (c.k_scale, c.v_scale)):
            R.append(codes, scale, x.float().cpu().numpy(), pos, rows)
            assert _same(_values(t), codes), i
            assert _same(s.cpu().numpy().astype(np.float64), scale), i
    c.check()


def test_append_extremes():
    """Zeros, the type's largest and smallest values, NaN and infinities; a row of NaN alone."""
    torch = _torch()
    x = torch.zeros(1, 8, 2, 64, device="cuda")
    x[0, 1, 0, :4] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3.0])
    x[0, 2, 0] = float("nan")
    x[0, 3, 0, 5] = -448.0
    x[0, 4, 1, 6] = 3.0e38      # cut to 448 * 2^111
    x[0, 5, 1, 7] = -1.0e-30    # below half of the smallest code: a zero
    c = _cache(2, 64, 64, fill=0x11)
    c.append(x, x, _ints([3]))
    codes, scale = np.full((1, 2, 64, 64), _values(_cache(2, 64, 64, fill=0x11).k)), np.full((1, 2, 1), np.nan)
    R.append(codes, scale, x.cpu().numpy(), [3], [8])
    # (positions 0..2 were never appended: their scale is whatever stood there, here NaN)
    assert _same(_values(c.k), codes) and _same(_values(c.v), codes)
    y = torch.full((1, 2, 2, 64), 1e-42, device="cuda")  # all below 2^-126
    c2 = _cache(2, 64, 64)
    c2.append(y, y, _ints([0]))
    assert float(c2.k_scale.max()) == 2.0 ** -120
    assert _same(_values(c2.k)[0, :, :2], R.e4m3_round(np.full((2, 2, 64), float(np.float32(1e-42)) * 2.0 ** 120)))
    # without rows: all M, from the start of a block: nothing old takes part
    c3 = _cache(2, 64, 128, fill=0x7f)
    c3.append(x, x, _ints([64]))
    codes, scale = np.full((1, 2, 128, 64), np.nan), np.full((1, 2, 2), np.nan)
    R.append(codes, scale, x.cpu().numpy(), [64], [8])
    assert _same(_values(c3.k), codes)
    assert _same(c3.k_scale.cpu().numpy().astype(np.float64), scale)


def test_append_leaves_bad_sequences_alone():
    from paper_2606_03113_gb300 import ssd as S
    torch = _torch()
    c = _cache(2, 64, 128, n=6, fill=0x22)
    before = c.k.view(torch.uint8).clone()
    x = torch.ones(6, 4, 2, 64, device="cuda")
    c.append(x, x, _ints([-1, 125, 128, 2 ** 31 - 1, 0, 10]), rows=_ints([4, 4, 1, 4, 5, 4]))
    with pytest.raises(S.SsdError) as e:
        c.check()
    assert e.value.status == S.SSD_ERR_DEVICE_FLAG and "6" in str(e.value)  # both bits
    c.check()  # once
    after = c.k.view(torch.uint8)
    assert torch.equal(after[:5], before[:5])
    assert bool((c.k[5, :, 10:14].float() * c.k_scale[5, :, 0, None, None] == 1).all())
    c.append(x, x, _ints([124, 124, 0, 0, 0, 0]), rows=_ints([4, 0, 0, 0, 0, 0]))
    c.check()
    assert torch.equal(c.k.view(torch.uint8)[1:5], before[1:5])


# ------------------------------------------------------------------ attention

def _filled(c, pos, rows, first, window, seed):
    """Random codes and scales where rows can look, NaN codes and scales everywhere else.
    Returns K and V values in float64, NaN out of sight."""
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, heads, seq, hd = c.k.shape
    vals = []
    for codes, scales, spread in ((c.k, c.k_scale, 1.0), (c.v, c.v_scale, 4.0)):
        x = torch.randn(n, heads, seq, hd, generator=g, device="cuda") * 100
        codes.copy_(x.clamp(-448, 448).to(codes.dtype))
        e = torch.randint(-3, 4, scales.shape, generator=g, device="cuda") if spread > 1 else \
            torch.randint(-8, -5, scales.shape, generator=g, device="cuda")
        scales.copy_(torch.ldexp(torch.ones_like(scales), e))
        b = codes.view(torch.uint8)
        for i in range(n):
            lo = R.visible(pos[i], first[i], window)[0] if rows[i] else seq
            hi = pos[i] + rows[i]
            b[i, :, :min(lo, seq)] = NAN_CODE
            b[i, :, hi:] = 0xff
            scales[i, :, :min(lo, hi) // 64] = float("nan")
            scales[i, :, (hi + 63) // 64:] = float("inf")
        vals.append(_values(codes) * np.repeat(scales.cpu().numpy().astype(np.float64), 64, -1)[..., None])
    return vals


ATTEND = [  # dtype, heads, kv heads, hd, n, M, seq, pos, rows, first, window
    ("f32", 4, 4, 64, 1, 1, 64, [0], [1], [0], 0),
    ("f32", 4, 4, 64, 1, 5, 128, [40], [5], [0], 0),
    ("f32", 8, 2, 128, 2, 3, 320, [300, 17], [3, 2], [0, 5], 100),
    ("bf16", 8, 2, 128, 1, 1, 64, [0], [1], [0], 0),
    ("bf16", 8, 2, 128, 1, 1, 640, [639], [1], [0], 0),
    ("bf16", 8, 8, 128, 1, 2, 192, [62], [2], [0], 0),
    ("bf16", 4, 4, 64, 1, 17, 256, [63], [17], [0], 0),
    ("bf16", 32, 4, 128, 1, 17, 512, [495], [17], [0], 0),
    ("bf16", 8, 2, 128, 4, 5, 448, [443, 0, 64, 200], [5, 1, 3, 0], [0, 0, 65, 0], 0),
    ("bf16", 8, 2, 128, 4, 5, 448, [440, 9, 64, 127], [5, 5, 2, 4], [439, 12, 70, 500], 0),
    ("bf16", 6, 2, 128, 3, 4, 704, [700, 300, 33], [4, 4, 4], [0, 290, 0], 37),
    ("bf16", 4, 2, 128, 2, 9, 640, [600, 64], [9, 9], [0, 0], 1),
    ("bf16", 24, 1, 128, 1, 3, 256, [200], [3], [3], 64),
    ("bf16", 8, 4, 128, 1, 75, 384, [300], [75], [0], 0),
    ("bf16", 8, 1, 64, 2, 40, 256, [130, 0], [39, 40], [7, 0], 90),
    ("bf16", 5, 5, 128, 9, 1, 128, [127, 64, 63, 1, 0, 100, 90, 80, 70], [1] * 9, [0] * 9, 0),
    ("f32", 16, 2, 128, 1, 33, 192, [150], [33], [0], 0),
    ("bf16", 8, 8, 64, 3, 2, 1024, [1000, 5, 513], [2, 2, 1], [0, 0, 400], 0),
    ("f32", 6, 3, 64, 2, 4, 960, [950, 700], [4, 4], [10, 0], 300),
    ("bf16", 16, 2, 128, 2, 30, 1088, [1058, 3], [30, 7], [0, 0], 500),
    ("bf16", 4, 1, 128, 1, 160, 896, [730], [160], [729], 0),
    ("bf16", 4, 2, 128, 300, 1, 640, [(37 * i) % 640 for i in range(300)], [1] * 300,
     [(11 * i) % 90 for i in range(300)], 0),
    ("bf16", 32, 4, 128, 3, 40, 512, [100, 30, 400], [40, 33, 0], [120, 300, 0], 0),
    ("bf16", 16, 2, 128, 2, 64, 1152, [1000, 5], [64, 50], [0, 20], 100),
    ("bf16", 16, 2, 128, 5, 17, 832, [800, 1, 64, 127, 0], [17, 16, 1, 17, 17], [0, 0, 0, 5, 9], 0),
    ("bf16", 129, 1, 128, 1, 1, 320, [319], [1], [0], 0),
    ("bf16", 128, 1, 128, 2, 2, 192, [100, 63], [2, 1], [0, 0], 0),
]


def _attend(case, seed, out=None, c=None, q=None):
    torch = _torch()
    dtype, heads, kvh, hd, n, M, seq, pos, rows, first, window = case
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    c = c or _cache(kvh, hd, seq, n)
    vals = _filled(c, pos, rows, first, window, seed)
    if q is None:
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        q = torch.randn(n, M, heads + 2 * kvh, hd, generator=g, device="cuda").to(dt)[:, :, :heads]
    got = c.attention(q, _ints(pos), rows=_ints(rows), first=_ints(first), window=window, out=out)
    c.check()
    return c, q, vals, got


def _check(case, q, vals, got, before):
    dtype, heads, kvh, hd, n, M, seq, pos, rows, first, window = case
    ref = before.copy()
    mass, size = R.attend(_values(q), vals[0], vals[1], pos, rows, first, window, ref)
    keys = max(p + r for p, r in zip(pos, rows))
    tol = R.attend_bound(ref, mass, size, hd, keys, dtype == "bf16")
    out = _values(got)
    live = np.arange(M)[None] < np.asarray(rows)[:, None]
    assert np.array_equal(out[~live], before[~live])  # left as they were
    assert np.isfinite(out[live]).all()
    bad = np.abs(out - ref) > tol
    assert not bad[live].any(), (np.abs(out - ref)[live].max(), np.argwhere(bad)[:5])


@pytest.mark.parametrize("room", [0, 640, 2112])
@pytest.mark.parametrize("case", ATTEND, ids=lambda c: "-".join(str(x) for x in c[:7]))
def test_attention_against_64_bits(case, room):
    """Also in larger caches: items of several blocks, a cluster, and of blocks that share all
    items evenly, whose parts are joined behind them."""
    torch = _torch()
    case = case[:6] + (case[6] + room,) + case[7:]
    dtype, heads, kvh, hd, n, M, seq, pos, rows, first, window = case
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    out = torch.full((n, M, heads + 1, hd), 0.625, device="cuda", dtype=dt)[:, :, :heads]
    before = _values(out)
    c, q, vals, got = _attend(case, 11, out=out)
    assert got is out
    _check(case, q, vals, got, before)
    # equal calls, equal bits; without an output the same in a new tensor, zero from rows on
    again = c.attention(q, _ints(pos), rows=_ints(rows), first=_ints(first), window=window)
    live = torch.arange(M, device="cuda") < _ints(rows)[:, None]
    assert torch.equal(again[live], got[live]) and not bool(again[~live].any())


@pytest.mark.parametrize("M,window", [(4, 0), (4, 3), (17, 0), (70, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seq", [320, 1024, 2560])
def test_a_nan_value_reaches_the_rows_that_see_it(dtype, M, window, seq):
    """NaN codes of keys and values: rows that do not see the key are as if it were not there."""
    torch = _torch()
    case = (dtype, 8, 2, 128, 1, M, seq, [200], [M], [0], window)
    _, q, vals, clean = _attend(case, 5)
    c, _, _, _ = _attend(case, 5, q=q)
    at = 200 + M - 2  # the last row but one's own key
    cv = c.v.view(torch.uint8)
    cv[0, 1, at, 17] = NAN_CODE
    cv[0, 0, 200, 3] = 0xff
    got = c.attention(q, _ints([200]), window=window)
    seen = {m: [R.visible(200 + m, 0, window)[0] <= k <= 200 + m for k in (at, 200)] for m in range(M)}
    for m in range(M):
        want = clean[0, m].clone()
        if seen[m][0]:
            want[4:, 17] = float("nan")
        if seen[m][1]:
            want[:4, 3] = float("nan")
        assert torch.equal(got[0, m].isnan(), want.isnan()), m
        assert torch.equal(got[0, m].nan_to_num(7.0), want.nan_to_num(7.0)), m
    # a NaN key makes every output of the rows that see it NaN, of its heads alone
    cv[0, 1, at, 17] = 0x20
    cv[0, 0, 200, 3] = 0x20
    c.k.view(torch.uint8)[0, 0, at, 100] = NAN_CODE
    got = c.attention(q, _ints([200]), window=window)
    for m in range(M):
        assert bool(got[0, m, :4].isnan().all()) == seen[m][0] == bool(got[0, m, :4].isnan().any()), m
        assert not bool(got[0, m, 4:].isnan().any())


def test_infinite_and_nan_queries_stay_in_their_rows():
    torch = _torch()
    case = ("bf16", 8, 2, 128, 1, 5, 128, [100], [5], [0], 0)
    c, q, vals, clean = _attend(case, 8)
    q = q.clone()
    q[0, 1, 3, 5] = float("inf")
    q[0, 2, 6, 7] = float("nan")
    got = c.attention(q, _ints([100]))
    hit = torch.zeros(5, 8, dtype=torch.bool, device="cuda")
    hit[1, 3] = hit[2, 6] = True
    assert bool(got[0][hit].isnan().all())
    assert torch.equal(got[0][~hit], clean[0][~hit])


@pytest.mark.parametrize("M", [9, 40, 75])
@pytest.mark.parametrize("seq", [512, 2560])
def test_infinite_and_nan_queries_among_many_rows(M, seq):
    torch = _torch()
    case = ("bf16", 8, 2, 128, 1, M, seq, [300], [M], [0], 0)
    c, q, vals, clean = _attend(case, 12)
    q = q.clone()
    q[0, 1, 3, 5] = float("-inf")
    q[0, M - 1, 6, 7] = float("nan")
    got = c.attention(q, _ints([300]))
    hit = torch.zeros(M, 8, dtype=torch.bool, device="cuda")
    hit[1, 3] = hit[M - 1, 6] = True
    assert bool(got[0][hit].isnan().all())
    assert torch.equal(got[0][~hit], clean[0][~hit])


def test_scores_far_apart_and_scales_far_apart():
    """One key that outweighs all others by far, blocks of zeros at the smallest scale, value
    scales 2^40 apart: the running maximum and the output's unit move up and down."""
    torch = _torch()
    for dtype in ("bf16", "f32"):
        dt = torch.float32 if dtype == "f32" else torch.bfloat16
        c = _cache(2, 128, 512)
        g = torch.Generator(device="cuda").manual_seed(2)
        x = torch.randn(1, 512, 4, 128, generator=g, device="cuda")
        x[:, 64:128, 2:] = 0
        x[:, 128:192, 2:] *= 2.0 ** 20
        x[:, 192:256, 2:] *= 2.0 ** -20
        q = torch.randn(1, 2, 4, 128, generator=g, device="cuda").to(dt)
        x[0, 3, :2] = 40 * q[0, 0, ::2].float() / q[0, 0, ::2].float().norm(dim=-1, keepdim=True)
        x[0, 400, 0] = 60 * q[0, 1, 1].float() / q[0, 1, 1].float().norm()
        c.append(x[:, :, :2], x[:, :, 2:], _ints([0]))
        vals = [_values(t) * np.repeat(s.cpu().numpy().astype(np.float64), 64, -1)[..., None]
                for t, s in ((c.k, c.k_scale), (c.v, c.v_scale))]
        for pos in (62, 140, 260, 510):
            case = (dtype, 4, 2, 128, 1, 2, 512, [pos], [2], [0], 0)
            got = c.attention(q, _ints([pos]))
            ref = np.zeros(got.shape)
            mass, size = R.attend(_values(q), vals[0], vals[1], [pos], [2], [0], 0, ref)
            tol = R.attend_bound(ref, mass, size, 128, pos + 2, dtype == "bf16")
            assert (np.abs(_values(got) - ref) <= tol).all(), (dtype, pos)


@pytest.mark.parametrize("dtype,M,window", [("f32", 6, 50), ("bf16", 6, 50), ("bf16", 40, 50),
                                            ("bf16", 40, 130)])
@pytest.mark.parametrize("seq", [320, 1024, 2560])
def test_large_values_behind_the_window_cost_nothing(dtype, M, window, seq):
    """A block of values 2^40 above the others that only the first rows of a tile still see: the
    others keep all their bits."""
    torch = _torch()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    c = _cache(2, 128, seq)
    g = torch.Generator(device="cuda").manual_seed(31)
    x = torch.randn(1, 300, 4, 128, generator=g, device="cuda")
    x[:, 64:128, 2:] *= 2.0 ** 40
    c.append(x[:, :, :2], x[:, :, 2:], _ints([0]))
    vals = [_values(t) * np.repeat(s.cpu().numpy().astype(np.float64), 64, -1)[..., None]
            for t, s in ((c.k, c.k_scale), (c.v, c.v_scale))]
    q = torch.randn(1, M, 4, 128, generator=g, device="cuda").to(dt)
    pos = 125 + window  # row 0 sees keys 126 .., row 2 none below 128
    got = c.attention(q, _ints([pos]), window=window)
    ref = np.zeros(got.shape)
    mass, size = R.attend(_values(q), vals[0], vals[1], [pos], [M], [0], window, ref)
    tol = R.attend_bound(ref, mass, size, 128, window, dtype == "bf16")
    assert (np.abs(_values(got) - ref) <= tol).all()
    c.check()


@pytest.mark.parametrize("dtype,heads,hd,n,M,seq", [("bf16", 8, 128, 2, 3, 320), ("bf16", 8, 128, 2, 40, 640),
                                                    ("f32", 4, 64, 3, 7, 2048), ("bf16", 4, 128, 1, 5, 2560), ("bf16", 8, 128, 2, 40, 2560)])
def test_output_over_the_queries_of_fused_rows(dtype, heads, hd, n, M, seq):
    """q, k and v read in place from a product's rows, the output written over q; what
    stands behind it in the rows stays."""
    torch = _torch()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(5)
    c = _cache(2, hd, seq, n)
    old = torch.randn(n, 200, 4, hd, generator=g, device="cuda").to(dt)
    c.append(old[:, :, :2], old[:, :, 2:], _ints([0] * n))
    rows = torch.randn(n, M, heads + 4, hd, generator=g, device="cuda").to(dt)
    pos = _ints([200 - 31 * b for b in range(n)])
    c.append(rows[:, :, heads:heads + 2], rows[:, :, heads + 2:], pos)
    want = c.attention(rows[:, :, :heads], pos)
    kept = rows[:, :, heads:].clone()
    got = c.attention(rows[:, :, :heads], pos, out=rows[:, :, :heads])
    assert got.data_ptr() == rows.data_ptr() and torch.equal(got, want)
    assert torch.equal(rows[:, :, heads:], kept)
    c.check()


def test_a_padded_sequence_in_anothers_place():
    """Its pads are not appended; the scales of the sequence before it are zeroed."""
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(6)
    c, fresh = _cache(2, 64, 192, 2), _cache(2, 64, 192, 2)
    x = torch.randn(2, 150, 2, 64, generator=g, device="cuda")
    c.append(1e6 * x, 1e6 * x, _ints([0, 0]))
    for t in (c.k_scale, c.v_scale):
        t[1].zero_()
    y = x[:, :40].contiguous()
    q = torch.randn(2, 40, 4, 64, generator=g, device="cuda")
    for d in (c, fresh):
        d.append(y, y, _ints([0, 21]), rows=_ints([0, 40]))
    a, b = (d.attention(q, _ints([0, 21]), rows=_ints([0, 40]), first=_ints([0, 21])) for d in (c, fresh))
    assert torch.equal(a, b) and bool(a[1].isfinite().all()) and bool((a[1] != 0).any())
    assert torch.equal(c.v_scale[1, :, 0], fresh.v_scale[1, :, 0])


def test_attention_leaves_bad_sequences_alone():
    from paper_2606_03113_gb300 import ssd as S
    torch = _torch()
    for seq, M in ((128, 3), (1024, 3), (2560, 3), (2560, 40), (2560, 130)):
        _bad_sequences(S, torch, seq, M)


def _bad_sequences(S, torch, seq, M):
    c = _cache(2, 128, seq, n=5)
    out = torch.full((5, M, 4, 128), 5.0, device="cuda", dtype=torch.bfloat16)
    q = torch.ones_like(out)
    c.attention(q, _ints([-1, seq - 2, 0, 2 ** 31 - 1, 5]), rows=_ints([3, 3, M + 1, 1, M]), out=out)
    with pytest.raises(S.SsdError):
        c.check()
    assert bool((out[:4] == 5.0).all()) and not bool((out[4] == 5.0).any())


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes a side: the last head's last positions."""
    torch = _torch()
    heads, seq = 5, 7_340_032
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB")
    c = _cache(heads, 128, seq)
    g = torch.Generator(device="cuda").manual_seed(4)
    M, pos = 3, seq - 70
    vals = np.zeros((2, 1, heads, 128, 128))
    x = torch.randn(1, 67, 2 * heads, 128, generator=g, device="cuda").bfloat16()
    c.append(x[:, :, :heads], x[:, :, heads:], _ints([pos]))
    y = torch.randn(1, M, 2 * heads, 128, generator=g, device="cuda").bfloat16()
    c.append(y[:, :, :heads], y[:, :, heads:], _ints([seq - M]))
    for i, (t, s) in enumerate(((c.k, c.k_scale), (c.v, c.v_scale))):
        vals[i] = _values(t[:, :, seq - 128:]) * np.repeat(
            s[:, :, -2:].cpu().numpy().astype(np.float64), 64, -1)[..., None]
    q = torch.randn(1, M, heads, 128, generator=g, device="cuda").bfloat16()
    got = c.attention(q, _ints([seq - M]), window=60)
    ref = np.zeros(got.shape)
    mass, size = R.attend(_values(q), vals[0], vals[1], [128 - M], [M], [0], 60, ref)
    assert (np.abs(_values(got) - ref) <= R.attend_bound(ref, mass, size, 128, 60, True)).all()
    c.check()


# ------------------------------------------------------------------ how calls are made

def test_other_stream_and_captured_replays():
    """A captured append + attention replayed as the sequence grows; two graphs of one cache
    replayed on two streams; a call on a stream that is not the current one."""
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(9)
    kvh, heads, hd, seq = 2, 8, 128, 512
    x = torch.randn(1, seq, heads + 2 * kvh, hd, generator=g, device="cuda").bfloat16()
    plain = _cache(kvh, hd, seq)
    want = []
    for p in range(0, 300, 3):
        row = x[:, p:p + 3]
        plain.append(row[:, :, heads:heads + kvh], row[:, :, heads + kvh:], _ints([p]))
        want.append(plain.attention(row[:, :, :heads], _ints([p])))
    c = _cache(kvh, hd, seq)
    pos = _ints([0])
    buf = torch.zeros(1, 3, heads + 2 * kvh, hd, device="cuda", dtype=torch.bfloat16)
    out = torch.zeros(1, 3, heads, hd, device="cuda", dtype=torch.bfloat16)

    def step():
        c.append(buf[:, :, heads:heads + kvh], buf[:, :, heads + kvh:], pos)
        c.attention(buf[:, :, :heads], pos, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, p in enumerate(range(0, 300, 3)):
        buf.copy_(x[:, p:p + 3])
        pos.fill_(p)
        graph.replay()
        assert torch.equal(out, want[i]), p
    # two captured attentions over the same cache, at once
    q2 = x[:, 7:10, :heads].contiguous()
    outs = [torch.zeros_like(out) for _ in range(2)]
    graphs = []
    for o, q in zip(outs, (buf[:, :, :heads], q2)):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            c.attention(q, pos, out=o)
        graphs.append(gr)
    alone = []
    for gr, o in zip(graphs, outs):
        gr.replay()
        torch.cuda.synchronize()
        alone.append(o.clone())
        o.zero_()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for gr, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                gr.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))
    # a stream of the caller's, not the current one
    s = streams[0]
    s.wait_stream(torch.cuda.current_stream())
    got = c.attention(q2, pos, stream=s)
    s.synchronize()
    assert torch.equal(got, alone[1])
    c.check()


@pytest.mark.parametrize("M,seq", [(5, 4096), (12, 4096), (40, 1024), (40, 4096)])
def test_captured_calls_of_every_kind(M, seq):
    """Two captured attentions over two caches, replayed at once as their sequences grow, against
    plain calls; then two calls at once on streams of the caller's."""
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(15)
    kvh, heads, hd = 2, 8, 128
    caches, qs, poss, outs, graphs = [], [], [], [], []
    for i in range(2):
        c = _cache(kvh, hd, seq)
        x = torch.randn(1, seq, 2 * kvh, hd, generator=g, device="cuda").bfloat16()
        c.append(x[:, :, :kvh], x[:, :, kvh:], _ints([0]))
        caches.append(c)
        qs.append(torch.randn(1, M, heads, hd, generator=g, device="cuda").bfloat16())
        poss.append(_ints([0]))
        outs.append(torch.zeros_like(qs[i]))
        c.attention(qs[i], poss[i], out=outs[i])
    for c, q, p, o in zip(caches, qs, poss, outs):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            c.attention(q, p, out=o)
        graphs.append(gr)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for step in (0, 1, 63, 64, 500, seq - M):
        for i in range(2):
            poss[i].fill_(max(step - 40 * i, 0))
        want = [c.attention(q, p) for c, q, p in zip(caches, qs, poss)]
        torch.cuda.synchronize()
        for _ in range(3):
            for gr, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), step
        got = [c.attention(q, p, stream=s) for c, q, p, s in zip(caches, qs, poss, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), step
    for c in caches:
        c.check()


def test_a_verification_over_the_8_bit_cache():
    """The operators as a verification pass uses them: the rows' K and V appended, attention over
    the cache, the head's product, the log-probabilities of the drafted tokens and their
    alternatives; then a rollback, and the next rows over the shorter sequence."""
    torch = _torch()
    from paper_2606_03113_gb300 import ssd as S
    from paper_2606_03113_gb300.runtime import token_logprobs
    g = torch.Generator(device="cuda").manual_seed(21)
    kvh, heads, hd, V, ctx, M = 2, 4, 64, 1000, 90, 5
    c = _cache(kvh, hd, 192)
    head = torch.randn(V, heads * hd, generator=g, device="cuda")
    head *= 6.0 / head.norm(dim=-1, keepdim=True)
    kv = torch.randn(1, ctx, 2 * kvh, hd, generator=g, device="cuda")
    c.append(kv[:, :, :kvh], kv[:, :, kvh:], _ints([0]))
    codes = [[np.zeros((1, kvh, 192, hd)), np.zeros((1, kvh, 3))] for _ in range(2)]
    for s, x in zip(codes, (kv[:, :, :kvh], kv[:, :, kvh:])):
        R.append(s[0], s[1], x.cpu().numpy(), [0], [ctx])
    pos = ctx
    for accepted in (2, 4):
        rows = torch.randn(1, M, heads + 2 * kvh, hd, generator=g, device="cuda")
        tok = torch.randint(0, V, (M, 1), generator=g, device="cuda").int()
        tok[M - 1] = -1  # the last row has no draft
        c.append(rows[:, :, heads:heads + kvh], rows[:, :, heads + kvh:], _ints([pos]))
        o = c.attention(rows[:, :, :heads], _ints([pos]))
        z = torch.empty(M, V, device="cuda")
        S.ssd_gemv_noalloc(head.data_ptr(), S.SSD_DTYPE_F32, V, heads * hd, o.data_ptr(), M, z.data_ptr(),
                           0, torch.cuda.current_stream().cuda_stream)
        got = token_logprobs(z, tok, top_n=5, temperature=0.6)
        for s, x in zip(codes, (rows[:, :, heads:heads + kvh], rows[:, :, heads + kvh:])):
            R.append(s[0], s[1], x.cpu().numpy(), [pos], [M])
        vals = [s[0] * np.repeat(s[1], 64, -1)[..., None] for s in codes]
        ref = np.zeros((1, M, heads, hd))
        mass, size = R.attend(_values(rows[:, :, :heads]), vals[0], vals[1], [pos], [M], [0], 0, ref)
        tol = R.attend_bound(ref, mass, size, hd, pos + M, False)
        assert (np.abs(_values(o) - ref) <= tol).all()
        zr = ref.reshape(M, -1) @ _values(head).T
        lp, lse, ent, ids, tlp, _ = R.logprobs(zr, tok.cpu().numpy(), 0.6, 5)
        # logits off by at most |head row| |tol|, and the product's own sums; twice that, over the
        # temperature, in a log-probability
        off = 2 * (6.0 * np.linalg.norm(tol.reshape(M, -1), axis=-1).max()
                   + 300 * 2.0 ** -24 * 6.0 * np.linalg.norm(ref.reshape(M, -1), axis=-1).max()) / 0.6 + 1e-5
        assert np.abs(got.logprob.cpu().numpy() - lp).max() <= off
        assert np.abs(got.lse.cpu().numpy() - lse).max() <= off
        assert float(got.logprob[M - 1]) == 0.0
        gap = np.sort(zr, -1)[:, ::-1][:, :6]
        if (gap[:, :-1] - gap[:, 1:]).min() / 0.6 > off:
            assert np.array_equal(got.top_id.cpu().numpy(), ids)
        assert np.abs(got.top_logprob.cpu().numpy() - tlp).max() <= off
        pos += accepted  # roll back behind the accepted rows
    c.check()
