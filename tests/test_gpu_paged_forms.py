"""The attention over pages form by form (clusters, k_paged_rows and k_paged_stream on the line of units,
k_paged_wide with one accumulator and two): each case says which kernel its sizes have to reach, and
fails where they no longer do. Bounds count the bits that each form keeps of a probability: 16 for bf16,
24 for fp32."""
import numpy as np
import pytest

import paged_ref as R
from parity import has_gpu
from test_gpu_paged import _agree, _cache, _dtype, _err, _filled, _ints, _torch, _twin

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a CUDA GPU")]


def _forms(c, heads, M, window=0, longest=0):
    """The kernels that a call of these sizes can have taken, by the workspace that it asks for: parts of as
    many rows as a tile has, two for each block of a grid of two blocks an SM or one, or, where there is less
    work, for each of its units."""
    from paper_2606_03113_gb300 import ssd as S
    nbytes = S.ssd_paged_attention_bytes(c._c, heads, M, window, longest)
    if nbytes == 256:
        return {"cluster"}
    rows, hd, longest = M * heads // c.n_kv_heads, c.head_dim, longest or c.max_seq
    span = window + M if 0 < window < longest - M else longest

    def up(x):
        return (x + 255) // 256 * 256

    def work(most, tile, cost):
        units = c.n_seq * c.n_kv_heads * -(-rows // tile) * ((span + 126) // 64 + cost)
        blocks, part = min(most, units), min(rows, tile)
        return up(32 * blocks) + up(16 * blocks * part) + 8 * blocks * part * hd
    told = [("rows", 320, t, 3) for t in (8, 16, 32, 64) if t == 64 or rows <= t]
    told += [("stream", 160, 8 if rows <= 8 else 16, 3)] if rows <= 16 else \
        [("wide1", 160, 128, 3)] if rows <= 128 else [("wide2", 160, 256, 8)]
    if c.dtype == _torch().float32:
        told = [("rows", 320, 8 if rows <= 8 else 16, 3)]
    return {form for form, *sizes in told if work(*sizes) == nbytes}


def _held(c, layer, q, pos, rows, first=None, window=0, longest=0):
    """Runs the attention and holds it to the bound of its type's bits."""
    torch = _torch()
    got = c.attention(layer, q, _ints(pos), rows=_ints(rows), first=None if first is None else _ints(first),
                      window=window, longest=longest)
    f32 = q.dtype == torch.float32
    want, bound = R.attention(_twin(c), layer, q.float().cpu().numpy(), pos, rows,
                              first or [0] * len(pos), window, 24 if f32 else 16)
    have = got.float().cpu().numpy().astype(np.float64)
    half = 2.0 ** -24 if f32 else 2.0 ** -8
    for b, m in enumerate(rows):
        w, bd, h = want[b, :m], bound[b, :m], have[b, :m]
        assert np.isfinite(w).all() and np.isfinite(h).all()
        off = np.abs(h - w) - (bd + half * (np.abs(w) + bd) + 1e-37)
        assert off.size == 0 or off.max() <= 0, (b, off.max())
        assert not have[b, m:].any()
    return got


FORMS = [  # form, dtype, heads, kv heads, hd, page, sequences of (pos, rows), M, first, window
    ("stream", "bf16", 8, 2, 128, 16, [(3000, 1), (2500, 1), (100, 1)], 1, [0, 900, 0], 2100),
    ("stream", "bf16", 8, 2, 128, 64, [(2600, 3), (3100, 2), (40, 1)], 3, [10, 0, 0], 2100),
    ("stream", "bf16", 8, 2, 128, 64, [(2600, 4), (3100, 2), (40, 0)], 4, [2590, 0, 0], 0),
    ("stream", "bf16", 8, 2, 64, 32, [(2700, 2), (2300, 1), (1, 2)], 2, None, 2049),
    ("stream", "bf16", 8, 2, 64, 16, [(3000, 4), (2222, 3)], 4, [0, 2150], 2500),
    ("stream", "bf16", 10, 2, 64, 128, [(3000, 2), (2222, 1), (5, 0)], 2, [0, 2215, 0], 0),
    ("rows", "f32", 4, 2, 64, 16, [(2600, 2), (1500, 1)], 2, [700, 0], 1100),
    ("rows", "f32", 8, 1, 128, 32, [(1800, 1)], 1, None, 1025),
    ("rows", "f32", 8, 2, 64, 64, [(1500, 5), (700, 3)], 5, [0, 650], 600),
    ("rows", "f32", 6, 2, 128, 16, [(1300, 4), (1290, 1)], 4, None, 513),
    ("rows", "bf16", 8, 2, 64, 16, [(2600, 7), (2300, 3), (64, 2)], 7, [0, 2250, 0], 2100),
    ("rows", "bf16", 8, 2, 64, 16, [(2600, 7), (2300, 3), (33, 1)], 7, None, 0),
    ("rows", "bf16", 8, 2, 64, 32, [(2500, 13), (2200, 9), (3, 1)], 13, [5, 2190, 0], 2100),
    ("rows", "bf16", 8, 2, 64, 256, [(2500, 30), (2200, 9)], 30, [5, 2205], 0),
    ("wide1", "bf16", 8, 2, 128, 16, [(2600, 7), (2300, 3), (64, 2)], 7, [0, 2250, 0], 2100),
    ("wide1", "bf16", 8, 2, 128, 64, [(2500, 32), (2200, 9), (0, 5)], 32, [0, 2205, 3], 0),
    ("wide2", "bf16", 8, 1, 128, 16, [(2500, 40), (2200, 20)], 40, [0, 2210], 2100),
    ("wide2", "bf16", 16, 2, 128, 32, [(2300, 17), (77, 1)], 17, None, 0),
    ("cluster", "bf16", 8, 2, 64, 16, [(900, 7), (1500, 3)], 7, [0, 1450], 700),
    ("cluster", "bf16", 8, 2, 64, 16, [(900, 13), (1500, 9)], 13, [890, 0], 1000),
    ("cluster", "bf16", 8, 2, 128, 16, [(1900, 8), (1500, 3)], 8, [0, 1490], 1500),
    ("cluster", "f32", 4, 2, 128, 64, [(900, 2), (1500, 1)], 2, [890, 0], 700),
]


@pytest.mark.parametrize("form,dtype,heads,kvh,hd,page,seqs,M,first,window", FORMS)
def test_each_form_within_its_bits(form, dtype, heads, kvh, hd, page, seqs, M, first, window):
    """Sliding windows whose starts fall in the middle of items and stages, sequences padded in front, rows
    that see nothing, through the kernel that the case names."""
    torch = _torch()
    pos, rows = [p for p, _ in seqs], [m for _, m in seqs]
    width = (max(pos) + M) // page + 1
    c, g = _filled(dtype, 2, kvh, hd, page, len(seqs), width, seed=heads + page + M)
    assert _forms(c, heads, M, window) == {form}
    q = (1.5 * torch.randn(len(seqs), M, heads, hd, generator=g, device="cuda")).to(_dtype(dtype))
    a = _held(c, 1, q, pos, rows, first, window)
    assert torch.equal(a, _held(c, 1, q, pos, rows, first, window))
    c.check()


# form, dtype, heads, kv heads, hd, M, positions of the table
SHAPES = [("cluster", "bf16", 8, 2, 128, 1, 640), ("cluster", "bf16", 8, 2, 64, 10, 640),
          ("cluster", "bf16", 4, 1, 128, 8, 640), ("cluster", "f32", 8, 2, 128, 1, 640),
          ("stream", "bf16", 8, 2, 128, 1, 16384), ("stream", "bf16", 8, 2, 64, 4, 16384),
          ("rows", "bf16", 8, 2, 64, 6, 16384), ("rows", "bf16", 8, 2, 64, 15, 16384),
          ("rows", "f32", 8, 2, 64, 2, 16384), ("rows", "f32", 8, 2, 128, 5, 16384),
          ("wide1", "bf16", 8, 2, 128, 6, 16384), ("wide1", "bf16", 8, 2, 128, 32, 16384),
          ("wide2", "bf16", 8, 1, 128, 33, 16384)]


def _one_key_column(c, heads, M, keys, score):
    """Queries that look at a key's first column alone, and keys whose scores with them are score[j] (as near
    as the type has it) at positions below `keys` and 0 behind; the weights of the former among themselves
    in 64 bits."""
    torch = _torch()
    held, hd = c.table[0, :(keys + M - 1) // c.page + 1].long(), c.head_dim
    k0 = torch.zeros(len(held) * c.page, device="cuda", dtype=torch.float64)
    k0[:keys] = torch.as_tensor(score, device="cuda") * hd ** 0.5
    k0 = k0.to(c.dtype)
    at = torch.zeros(len(held), 1, c.n_kv_heads, c.page, hd, device="cuda", dtype=c.dtype)
    at[..., 0] = k0.view(len(held), 1, 1, c.page)
    c.pages[held, :, 0] = at
    q = torch.zeros(1, M, heads, hd, device="cuda", dtype=c.dtype)
    q[..., 0] = 1.0
    s = k0[:keys].double().cpu().numpy() / hd ** 0.5
    e = np.exp(s - s.max())
    return q, held, e / e.sum()


@pytest.mark.parametrize("form,dtype,heads,kvh,hd,M,cap", SHAPES)
def test_values_that_cancel_show_the_bits_of_a_probability(form, dtype, heads, kvh, hd, M, cap):
    """Values of magnitude one whose weighted mean is next to nothing: what is left is the error of the weights, and
    the output's own rounding hides none of it (the new rows' own values are zero). Weights rounded to 8 bits are
    ten times too far off."""
    torch = _torch()
    keys, page = 300, 32
    c, g = _filled(dtype, 1, kvh, hd, page, 1, (keys + M) // page + 1, seed=M,
                   room=cap // page - (keys + M) // page - 1)
    assert _forms(c, heads, M) == {form}
    rng = np.random.default_rng(hd + M)
    q, held, w = _one_key_column(c, heads, M, keys, rng.uniform(-3.0, 3.0, keys))

    def rounded(x):
        return torch.as_tensor(x).to(c.dtype).double().numpy()
    order = np.argsort(-w)
    v = np.zeros((keys, kvh, hd))
    run = np.zeros((kvh, hd))
    for n, j in enumerate(order):
        size = rounded(rng.uniform(0.75, 1.25, (kvh, hd)))
        # against what has come together so far; the last ones take what is left of it
        v[j] = np.where(run > 0, -size, size) if n < keys - 3 else rounded(-run / w[j])
        run += w[j] * v[j]
    assert np.abs(run).max() < 1e-6
    full = torch.zeros(len(held) * page, kvh, hd, dtype=torch.float64)
    full[:keys] = torch.as_tensor(v)
    c.pages[held, 0, 1] = full.view(len(held), page, kvh, hd).transpose(1, 2).to(c.dtype).cuda()
    _held(c, 0, q, [keys], [M])
    c.check()


@pytest.mark.parametrize("form,dtype,heads,kvh,hd,M,cap", SHAPES)
def test_large_values_stay_finite(form, dtype, heads, kvh, hd, M, cap):
    """A few hundred values of up to 2^119, all of one sign, their largest scores behind the first ones by a little
    less than what moves a running maximum's stand-in: the sums stay within fp32. So many sequences (all
    of the same pages) that a block walks whole items."""
    torch = _torch()
    keys, page, n = 300, 32, 48
    c, g = _filled(dtype, 1, kvh, hd, page, n, (keys + M) // page + 1, seed=M,
                   room=cap // page - (keys + M) // page - 1 if cap > 640 else 0)
    assert _forms(c, heads, M) == {form}
    c.table[:] = c.table[0]
    score = np.full(keys, 7.5 * np.log(2.0))
    score[:64] = 0.0
    q, held, _ = _one_key_column(c, heads, M, keys, score)
    v = (1.0 + torch.rand(len(held), kvh, page, hd, generator=g, device="cuda")) * 2.0 ** 118
    c.pages[held, 0, 1] = v.to(c.dtype)
    got = c.attention(0, q.expand(n, M, heads, hd).contiguous(), _ints([keys] * n)).double().cpu().numpy()
    bits, half = (24, 2.0 ** -24) if dtype == "f32" else (16, 2.0 ** -8)
    want, bound = R.attention(_twin(c), 0, q.float().cpu().numpy(), [keys], [M], [0], 0, bits)
    assert np.isfinite(want).all() and want.min() > 2.0 ** 118
    off = np.abs(got - want) - (bound + half * (want + bound))
    assert off.max() <= 0, off.max()
    c.check()


def test_what_is_no_number_slows_its_own_rows_alone():
    """An infinity that one sequence's last row sees, in one head: the others' rows keep their bits. Where the
    sequence is short, the call takes its time (each of the others' keys walked again by one thread a row took
    160 times as long), where it has 3000 keys, a few times that at most (they are looked through by 32 at a
    time, a round trip of a page's number and 64 bytes, for each quarter of the columns: 0.2 ms beside 0.15)."""
    torch = _torch()
    n, M, heads, kvh = 41, 17, 64, 8
    c, g = _filled("bf16", 1, kvh, 128, 64, n, 50, seed=3)
    assert _forms(c, heads, M) == {"wide2"}
    at = [0] + [3000 + 3 * b for b in range(n - 1)]
    pos = _ints(at)
    q = torch.randn(n, M, heads, 128, generator=g, device="cuda").bfloat16()

    def timed():
        took = []
        for _ in range(7):
            a, z = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            torch.cuda.synchronize()
            a.record()
            got = c.attention(0, q, pos)
            z.record()
            torch.cuda.synchronize()
            took.append(a.elapsed_time(z))
        return got, sorted(took)[3]
    want, before = timed()
    for b, times in ((0, 4), (20, 16)):
        p = at[b] + M - 1
        e = int(c.table[b, p // 64])
        was = c.pages[e, 0, 1, 0, p % 64, 5].clone()
        c.pages[e, 0, 1, 0, p % 64, 5] = float("inf")
        got, after = timed()
        hit = got[b, M - 1, :heads // kvh, 5]
        assert (hit == float("inf")).all()
        got[b, M - 1, :heads // kvh, 5] = want[b, M - 1, :heads // kvh, 5]
        assert torch.equal(got, want)
        assert after <= times * before, (b, before, after)
        c.pages[e, 0, 1, 0, p % 64, 5] = was
    c.check()


# ------------------------------------------------------------------ rows and pages beyond one pass

@pytest.mark.parametrize("dtype,heads,M", [("bf16", 41, 1), ("bf16", 64, 3), ("bf16", 80, 2), ("f32", 24, 2)])
def test_rows_of_more_chunks_than_threads_hold_at_once(dtype, heads, M):
    """Rows of more than 5 x 128 pieces of 16 bytes: a whole second batch of them, and a part of one."""
    torch = _torch()
    c = _cache(dtype, 2, heads, 128, 9, 16, 2, 4, fill=2.0)
    r = _twin(c)
    k, v = (torch.randn(2, M, heads, 128, device="cuda").to(_dtype(dtype)) for _ in range(2))
    pos, rows = [15, 30], [M, M - 1]
    for x in (c, r):
        x.reserve(*((_ints(pos), _ints(rows)) if x is c else (pos, rows)))
    c.append(1, k, v, _ints(pos), rows=_ints(rows))
    r.append(1, k.float().cpu().numpy(), v.float().cpu().numpy(), pos, rows)
    _agree(c, r)
    c.check()


@pytest.mark.parametrize("pool", [2399, 9000])
def test_too_few_pages_for_thousands_of_claims(pool):
    """More wanted entries than a reserve keeps in registers, shared and missing ones, in a pool that is one page
    short: claims are taken back, nothing changes, and what fits works."""
    torch = _torch()
    c = _cache("f32", 1, 1, 64, pool, 16, 3, 1300)
    r = _twin(c)
    taken = pool - 2399  # pages that nobody here names
    c.refs[:taken] = 1
    r.refs[:taken] = [1] * taken
    for x, ints in ((c, _ints), (r, list)):
        x.reserve(ints([0, 0, 0]), ints([16 * 1200, 0, 0]))
        x.fork(ints([0, 0, 2]))
    c.refs[:taken] = 1
    r.refs[:taken] = [1] * taken
    c.pages.copy_(torch.arange(pool, device="cuda").view(-1, 1, 1, 1, 1, 1).expand_as(c.pages))
    r.pages = c.pages.float().cpu().numpy()
    # 1100 pages that both ask for, of which the first sequence needs new ones, and 100 missing ones
    pos, rows = [7, 7, 0], [1100 * 16 - 7, 1100 * 16 - 7, 1600]
    for x, ints in ((c, _ints), (r, list)):
        x.reserve(ints(pos), ints(rows))
    assert _err(c) == r.err == R.PAGES
    _agree(c, r)
    r.err = 0
    rows[2] = 1584
    for x, ints in ((c, _ints), (r, list)):
        x.reserve(ints(pos), ints(rows))
    assert _err(c) == r.err == 0
    _agree(c, r)
