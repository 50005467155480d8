"""The paged KV cache on the GPU: pages, table and counts equal to a reference that moves them one by one,
attention within a bound derived from its roundings (paged_ref)."""
import numpy as np
import pytest

import paged_ref as R
from parity import has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a CUDA GPU")]


def _torch():
    import torch
    return torch


def _ints(xs):
    return _torch().tensor(xs, dtype=_torch().int32, device="cuda")


def _dtype(name):
    torch = _torch()
    return torch.float32 if name == "f32" else torch.bfloat16


def _cache(dtype, layers, heads, hd, pool, page, n, width, fill=0.0):
    from paper_2606_03113_gb300.runtime import PagedKVCache
    c = PagedKVCache(layers, heads, hd, pool, page=page, n_seq=n, max_seq=width * page,
                     dtype=_dtype(dtype))
    c.pages.fill_(fill)
    return c


def _twin(c):
    """The reference in the state of c."""
    r = R.Cache(c.n_layers, c.n_kv_heads, c.head_dim, c.n_pages, c.page, c.n_seq, c.max_pages)
    r.pages = c.pages.float().cpu().numpy()
    r.table = c.table.tolist()
    r.refs = c.refs.tolist()
    return r


def _agree(c, r, pages=True):
    assert c.refs.tolist() == r.refs
    assert c.table.tolist() == r.table
    if pages:
        assert np.array_equal(c.pages.float().cpu().numpy(), r.pages, equal_nan=True)


def _err(c):
    got = int(c.err.item())
    c.err.zero_()
    return got


# ------------------------------------------------------------------ pages

RUNS = [  # dtype, layers, heads, hd, page, sequences, entries, pool
    ("f32", 1, 1, 64, 16, 1, 4, 5),
    ("f32", 2, 4, 64, 16, 4, 5, 24),
    ("bf16", 3, 2, 128, 32, 7, 4, 33),
    ("bf16", 1, 3, 64, 64, 5, 3, 18),
    ("f32", 2, 1, 128, 256, 3, 2, 7),
    ("bf16", 2, 1, 64, 16, 33, 6, 250),
]


@pytest.mark.parametrize("dtype,layers,heads,hd,page,n,width,pool", RUNS)
def test_runs_of_calls_match_the_reference(dtype, layers, heads, hd, page, n, width, pool):
    """Sequences fork, are cut back, end, grow and are compacted: every table, count and byte."""
    torch = _torch()
    rng = np.random.default_rng(n * 100 + page)
    c = _cache(dtype, layers, heads, hd, pool, page, n, width, fill=7.0)
    r = _twin(c)
    g = torch.Generator(device="cuda").manual_seed(pool)
    length = [0] * n
    short = 0
    for step in range(40):
        kind = rng.integers(5)
        if kind == 0:
            parent = [int(x) for x in rng.integers(-1, n, n)]
            c.fork(_ints(parent))
            r.fork(parent)
            length = [length[p] if p >= 0 else 0 for p in parent]
        elif kind == 1:
            length = [int(rng.integers(0, x + 1)) if rng.random() < 0.4 else x for x in length]
            c.truncate(_ints(length))
            r.fork(None, length)
        elif kind == 2:
            used = c.compact()
            assert int(used.item()) == r.compact()
        elif kind == 3:
            parent = [int(x) for x in rng.integers(0, n, n)]
            keep = [int(rng.integers(0, width * page + 1)) for _ in range(n)]
            c.fork(_ints(parent), _ints(keep))
            r.fork(parent, keep)
            length = [min(length[p], k) for p, k in zip(parent, keep)]
        _agree(c, r)
        # some roll back into what they hold, some stay as they are
        pos = [int(rng.integers(0, x + 1)) if rng.random() < 0.2 else x for x in length]
        M = int(rng.choice([1, 3, page, page + 5]))
        rows = [int(min(rng.integers(0, M + 1), width * page - x)) for x in pos]
        r.err = 0
        c.reserve(_ints(pos), _ints(rows))
        r.reserve(pos, rows)
        assert _err(c) == r.err
        _agree(c, r)
        if r.err:
            short += 1
            continue
        layer = int(rng.integers(layers))
        k, v = (torch.randn(n, M, heads, hd, generator=g, device="cuda").to(_dtype(dtype))
                for _ in range(2))
        c.append(layer, k, v, _ints(pos), rows=_ints(rows))
        r.append(layer, k.float().cpu().numpy(), v.float().cpu().numpy(), pos, rows)
        _agree(c, r)
        assert _err(c) == r.err == 0
        length = [max(x, p + m) for x, p, m in zip(length, pos, rows)]
    assert short < 40


@pytest.mark.parametrize("n,width,pool", [(4096, 3, 9973), (1, 8000, 20011), (1025, 20, 24577), (3, 5000, 16384)])
def test_large_tables(n, width, pool):
    """More sequences, entries and pages than a pass of the planning block takes, among them odd
    numbers; all sequences share, and all but one copy."""
    c = _cache("f32", 1, 1, 64, pool, 16, n, width)
    rng = np.random.default_rng(n)
    r = _twin(c)
    first = [0] * n
    # the pool's first pages are in use in places, so that the free ones lie apart
    some = sorted(int(x) for x in rng.choice(pool // 2, pool // 5, replace=False))
    c.refs[_ints(some).long()] = 1
    for e in some:
        r.refs[e] = 1
    rows = [0] * n
    rows[n // 2] = min(width * 16 - 5, 16 * (pool // 8) + 3)
    c.reserve(_ints(first), _ints(rows))
    r.reserve(first, rows)
    _agree(c, r, pages=False)
    parent = [n // 2] * n
    cut = [int(rng.integers(0, 40)) for _ in range(n)]
    c.fork(_ints(parent), _ints(cut))
    r.fork(parent, cut)
    for e in some:
        r.refs[e] += 1
    _agree(c, r, pages=False)
    r.err = 0
    more = [int(x) for x in rng.integers(0, 3, n)]
    c.reserve(_ints(cut), _ints(more))
    r.reserve(cut, more)
    assert _err(c) == r.err
    _agree(c, r)
    assert int(c.compact().item()) == sum(x > 0 for x in r.refs)
    for e in some:  # (nobody names these: a compaction keeps their counts, not their names)
        pass
    refs = c.refs.tolist()
    low = sum(x > 0 for x in r.refs)
    assert all(refs[:low]) and not any(refs[low:])
    assert sorted(x for x in refs if x) == sorted(x for x in r.refs if x)


def test_two_long_sequences_that_share_everything_move_apart():
    """Claims on thousands of shared pages, over several passes of the planning block: where both ask, the second
    keeps the page; where one asks, it moves."""
    for both in (True, False):
        c = _cache("f32", 1, 1, 64, 6000, 16, 2, 2500)
        c.pages.copy_(_torch().arange(6000, device="cuda").view(-1, 1, 1, 1, 1, 1).expand_as(c.pages))
        c.reserve(_ints([0, 0]), _ints([40000, 0]))
        c.fork(_ints([0, 0]))
        r = _twin(c)
        pos, rows = [7, 7], [39993, 39000 if both else 0]
        c.reserve(_ints(pos), _ints(rows))
        r.reserve(pos, rows)
        _agree(c, r)
        assert _err(c) == r.err == 0 and max(r.refs) <= 2


def test_too_few_pages_change_nothing():
    """With shared pages claimed, missing ones asked for and one page too few: table, counts and contents stay,
    the next call that fits works."""
    c = _cache("bf16", 2, 2, 64, 9, 16, 4, 4, fill=3.0)
    c.reserve(_ints([0, 0, 0, 0]), _ints([20, 0, 0, 33]))    # 2 and 3 pages
    c.fork(_ints([0, 0, 0, 3]))
    r = _twin(c)
    before = c.pages.clone()
    # three sharers of the second page: two copies, one new page each for 33..47: 2 + 3 > 4 free
    pos, rows = [20, 20, 20, 40], [20, 20, 20, 0]
    c.reserve(_ints(pos), _ints(rows))
    r.reserve(pos, rows)
    assert _err(c) == r.err == R.PAGES
    _agree(c, r)
    assert _torch().equal(before, c.pages)
    with pytest.raises(Exception, match="free pages"):
        c.reserve(_ints(pos), _ints(rows))
        c.check()
    r.err = 0
    rows = [20, 2, 12, 0]                                    # 2 copies and one page
    c.reserve(_ints(pos), _ints(rows))
    r.reserve(pos, rows)
    assert _err(c) == r.err == 0
    _agree(c, r)


def test_bad_numbers_leave_their_sequence_alone():
    c = _cache("f32", 1, 2, 64, 40, 16, 6, 4)
    r = _twin(c)
    pos, rows = [0, -1, 60, 5, 64, 65], [3, 2, 5, -1, 0, 0]
    c.reserve(_ints(pos), _ints(rows))
    r.reserve(pos, rows)
    _agree(c, r)
    assert _err(c) == r.err == R.CAPACITY | R.CONTROL
    pos, rows = [0, 1, 2, 1 << 30, 2 ** 31 - 1, -2 ** 31], [2 ** 31 - 1, 1, 64, 1, 1, 1]
    c.reserve(_ints(pos), _ints(rows))
    r.err = 0
    r.reserve(pos, rows)
    _agree(c, r)
    assert _err(c) == r.err
    parent, keep = [6, 0, -2, 3, -1, 0], [9, -1, 9, 9, 9, 2 ** 31 - 1]
    c.fork(_ints(parent), _ints(keep))
    r.err = 0
    r.fork(parent, keep)
    _agree(c, r)
    assert _err(c) == r.err == R.CONTROL


def test_rows_are_not_written_to_missing_or_shared_pages():
    torch = _torch()
    c = _cache("bf16", 2, 2, 128, 12, 16, 3, 3)
    c.reserve(_ints([0, 0, 0]), _ints([20, 0, 0]))
    c.fork(_ints([0, 0, -1]))
    c.reserve(_ints([0, 20, 0]), _ints([0, 1, 0]))  # its second page is its own now, the first is shared
    c.table[2, 0] = 12                              # no page of the pool
    r = _twin(c)
    r.table[2][0] = -1
    x = torch.randn(3, 8, 2, 128, device="cuda").bfloat16()
    pos, rows = [14, 14, 0], [4, 8, 2]
    c.append(1, x, -x, _ints(pos), rows=_ints(rows))
    r.append(1, x.float().cpu().numpy(), -x.float().cpu().numpy(), pos, rows)
    assert _err(c) == r.err == R.TABLE
    assert np.array_equal(c.pages.float().cpu().numpy(), r.pages)
    pos, rows = [45, -1, 48], [4, 2, 1]
    c.append(1, x, x, _ints(pos), rows=_ints(rows))
    assert _err(c) == R.CAPACITY
    c.append(1, x, x, _ints([0, 0, 0]), rows=_ints([9, -1, 0]))
    assert _err(c) == R.CONTROL
    assert np.array_equal(c.pages.float().cpu().numpy(), r.pages)


def test_append_reads_rows_in_place():
    """K and V as parts of a product's rows, more heads than threads take at once, one row and many."""
    torch = _torch()
    for heads, M, n in ((40, 1, 3), (40, 70, 1), (3, 17, 2)):
        c = _cache("bf16", 1, heads, 128, 40, 32, n, 6)
        r = _twin(c)
        qkv = torch.randn(n, M, 3 * heads, 128, device="cuda").bfloat16()
        pos = [5 + 9 * b for b in range(n)]
        c.reserve(_ints(pos), M)
        r.reserve(pos, [M] * n)
        k, v = qkv[:, :, heads:2 * heads], qkv[:, :, 2 * heads:]
        c.append(0, k, v, _ints(pos))
        r.append(0, k.float().cpu().numpy(), v.float().cpu().numpy(), pos, [M] * n)
        _agree(c, r)
        c.check()


# ------------------------------------------------------------------ attention

def _filled(dtype, layers, heads, hd, page, n, width, seed, extra=3, room=0):
    """A cache whose sequences hold the first `width` pages' positions, in scattered pages of random
    contents, of `room` pages more that their tables have room for."""
    torch = _torch()
    pool = n * width + extra
    c = _cache(dtype, layers, heads, hd, pool, page, n, width + room)
    g = torch.Generator(device="cuda").manual_seed(seed)
    c.pages.normal_(generator=g)
    ids = torch.randperm(pool, generator=g, device="cuda")[:n * width].int()
    c.table[:, :width] = ids.view(n, width)
    c.refs[ids.long()] = 1
    return c, g


def _check_attention(c, layer, q, pos, rows, first=None, window=0, longest=0, out=None, **kw):
    torch = _torch()
    n, M, H, hd = q.shape
    before = None if out is None else out.clone()
    got = c.attention(layer, q, _ints(pos), rows=_ints(rows), first=None if first is None else _ints(first),
                      window=window, longest=longest, out=out, **kw)
    bits = 24 if q.dtype == torch.float32 else 8
    want, bound = R.attention(_twin(c), layer, q.float().cpu().numpy(), pos, rows, first or [0] * n, window,
                              bits)
    have = got.float().cpu().numpy().astype(np.float64)
    half = 2.0 ** -24 if bits == 24 else 2.0 ** -8
    for b in range(n):
        live = slice(0, max(rows[b], 0))
        w, bd, h = want[b, live], bound[b, live], have[b, live]
        assert np.array_equal(np.isnan(w), np.isnan(h))
        fine = ~np.isnan(w)
        off = np.abs(h - w)[fine] - (bd + half * (np.abs(w) + bd) + 1e-37)[fine]
        assert off.size == 0 or off.max() <= 0, (b, off.max())
        rest = got[b, max(rows[b], 0):]
        assert torch.equal(rest, torch.zeros_like(rest) if before is None else before[b, max(rows[b], 0):])
    return got


ATTEND = [  # dtype, layers, heads, kv heads, hd, page, sequences of (pos, rows), M, first, window, longest
    ("f32", 1, 4, 4, 64, 16, [(40, 5)], 5, None, 0, 0),
    ("f32", 2, 4, 2, 128, 32, [(0, 1)], 1, None, 0, 0),
    ("bf16", 2, 32, 8, 128, 16, [(1100, 1)], 1, None, 0, 1101),
    ("bf16", 1, 32, 8, 128, 64, [(0, 1), (1, 1), (15, 1), (16, 1), (63, 1), (64, 1), (65, 1)], 1, None, 0, 0),
    ("bf16", 1, 8, 8, 64, 16, [(127, 1), (128, 1), (129, 1), (500, 1)], 1, None, 0, 0),
    ("bf16", 1, 64, 8, 128, 64, [(777, 17)], 17, None, 0, 0),
    ("bf16", 1, 24, 8, 128, 128, [(300, 7), (20, 0), (1, 3)], 7, None, 0, 0),
    ("bf16", 2, 7, 1, 128, 16, [(200, 3), (90, 2)], 3, [150, 0], 0, 0),
    ("bf16", 1, 32, 32, 128, 16, [(400, 5), (63, 1), (250, 4)], 5, [0, 70, 100], 37, 0),
    ("f32", 1, 12, 3, 64, 64, [(100, 9), (0, 9), (64, 1)], 9, [0, 3, 200], 20, 0),
    ("bf16", 1, 16, 2, 64, 256, [(1000, 40)], 40, None, 100, 0),
    ("bf16", 1, 40, 5, 128, 32, [(333, 33), (10, 20)], 33, [12, 15], 0, 400),
    ("bf16", 1, 8, 1, 128, 16, [(2000, 2), (3, 2), (900, 1), (31, 2)], 2, None, 1, 0),
    ("f32", 1, 8, 2, 128, 16, [(4000, 2)], 2, None, 0, 0),
    ("bf16", 1, 8, 2, 128, 16, [(0, 300)], 300, None, 0, 0),
    ("f32", 1, 6, 2, 64, 16, [(3, 130)], 130, None, 50, 0),
    ("bf16", 1, 4, 4, 128, 16, [(5, 1)] * 61, 1, None, 0, 0),
    ("bf16", 1, 16, 1, 128, 64, [(150, 8), (64, 1), (0, 8)], 8, [0, 60, 0], 0, 0),
    ("bf16", 1, 64, 2, 128, 32, [(500, 6), (190, 5)], 6, [0, 300], 90, 0),
    ("bf16", 1, 12, 1, 128, 256, [(63, 65), (1, 64)], 65, None, 0, 0),
    ("bf16", 1, 16, 8, 128, 16, [(1, 140)], 140, None, 64, 0),
    ("bf16", 1, 8, 4, 128, 16, [(5000, 1), (4999, 1), (100, 1)], 1, None, 100, 0),
    ("bf16", 1, 8, 4, 64, 32, [(3000, 4), (2047, 1)], 4, [0, 2040], 0, 0),
    ("bf16", 1, 8, 2, 128, 16, [(3 * b % 70, 1 + b % 2) for b in range(150)], 2, None, 0, 0),
    ("f32", 1, 2, 1, 64, 16, [(5 * b % 90, 1) for b in range(70)], 1, None, 0, 0),
    ("f32", 1, 16, 2, 128, 64, [(700, 3), (1, 1)], 3, None, 0, 0),
    ("bf16", 1, 24, 8, 64, 64, [(150, 9), (600, 2)], 9, None, 0, 0),
]

# positions that the table has room for behind what a case needs: 0 deals short sequences out by clusters,
# more than 2048 by the line of units and, for many rows, to the tcgen05 tiles
ROOM = [0, 2100]


@pytest.mark.parametrize("room", ROOM)
@pytest.mark.parametrize("dtype,layers,heads,kvh,hd,page,seqs,M,first,window,longest", ATTEND)
def test_attention(dtype, layers, heads, kvh, hd, page, seqs, M, first, window, longest, room):
    torch = _torch()
    n = len(seqs)
    pos, rows = [p for p, _ in seqs], [m for _, m in seqs]
    width = max(p + M for p in pos) // page + 2
    c, g = _filled(dtype, layers, kvh, hd, page, n, width, seed=heads + page, room=room // page)
    q = (1.5 * torch.randn(n, M, heads, hd, generator=g, device="cuda")).to(_dtype(dtype))
    a = _check_attention(c, layers - 1, q, pos, rows, first, window, longest)
    assert torch.equal(a, _check_attention(c, layers - 1, q, pos, rows, first, window, longest))
    # rows in place of a product's, and an output with rows of its own
    qkv = torch.randn(n, M, heads + 5, hd, generator=g, device="cuda").to(q.dtype)
    qkv[:, :, :heads] = q
    out = torch.full((n, M, heads + 2, hd), 5.0, device="cuda", dtype=q.dtype)[:, :, :heads]
    b = _check_attention(c, layers - 1, qkv[:, :, :heads], pos, rows, first, window, longest, out=out)
    assert b.data_ptr() == out.data_ptr()
    # over the queries
    inplace = q.clone()
    _check_attention_inplace(c, layers - 1, inplace, a, pos, rows, first, window, longest)
    c.check()


def _check_attention_inplace(c, layer, q, want, pos, rows, first, window, longest):
    torch = _torch()
    was = q.clone()
    got = c.attention(layer, q, _ints(pos), rows=_ints(rows), first=None if first is None else _ints(first),
                      window=window, longest=longest, out=q)
    for b, m in enumerate(rows):
        assert torch.equal(got[b, :m], want[b, :m]) and torch.equal(got[b, m:], was[b, m:])


@pytest.mark.parametrize("dtype,hd,heads,kvh,M", [("bf16", 128, 8, 2, 1), ("bf16", 64, 8, 2, 6),
                                                 ("bf16", 128, 16, 1, 5), ("f32", 64, 4, 4, 5),
                                                 ("f32", 128, 4, 1, 2), ("bf16", 128, 64, 4, 9),
                                                 ("bf16", 128, 64, 8, 40)])
@pytest.mark.parametrize("room", ROOM)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_out_of_sight_does_not_matter(dtype, hd, heads, kvh, M, room, bad):
    """NaN and infinities in positions that no row sees, and in those that some rows see: in front of `first`,
    behind the window, behind the last row, in a row's future, in pages of others."""
    torch = _torch()
    n, page, width = 3, 16, 16
    c, g = _filled(dtype, 1, kvh, hd, page, n, width, seed=M, room=room // page)
    pos, rows, first, window = [100, 7, 180], [M, M, M - 1 if M > 1 else 1], [30, 0, 200], 60
    pages = c.pages.view(-1, 1, 2, kvh, page, hd)
    table = c.table.tolist()
    for e in set(range(c.n_pages)) - {e for line in table for e in line}:
        pages[e] = bad
    for b in range(n):
        for p in range(width * page):
            out_of_sight = p >= pos[b] + rows[b] or p < first[b] or p <= pos[b] - window
            if out_of_sight:
                pages[table[b][p // page], :, :, :, p % page] = bad
    q = torch.randn(n, M, heads, hd, generator=g, device="cuda").to(_dtype(dtype))
    a = _check_attention(c, 0, q, pos, rows, first, window)
    assert torch.isfinite(a.float()).all()
    # the last row's own value is seen by it alone
    if M > 2:
        side = 1
        at = pos[0] + rows[0] - 1
        pages[table[0][at // page], 0, side, 0, at % page, 3] = bad
        z = c.attention(0, q, _ints(pos), rows=_ints(rows), first=_ints(first), window=window)
        G = heads // kvh
        same = z == a
        assert same[1:].all() and same[0, :rows[0] - 1].all() and same[0, rows[0] - 1, G:].all()
        col = z[0, rows[0] - 1, :G, 3].float()
        assert (torch.isnan(col) if bad != bad else col == bad).all()
        keep = torch.ones(hd, dtype=torch.bool, device="cuda")
        keep[3] = False
        assert same[0, rows[0] - 1, :G][:, keep].all()
    # a value in the middle that every row sees, in a step that is seen whole
    at = 64
    pages[table[0][at // page], 0, 1, kvh - 1, at % page, 5] = bad
    z = c.attention(0, q, _ints(pos), rows=_ints(rows), first=_ints(first), window=window)
    col = z[0, :rows[0], heads - heads // kvh:, 5].float()
    live = torch.tensor([pos[0] + m - window < at for m in range(rows[0])], device="cuda")
    assert live[0] and (torch.isnan(col) if bad != bad else col == bad)[live].all()
    assert torch.isfinite(col[~live]).all() and torch.isfinite(z[1:].float()).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype,heads,kvh,M,cap", [("bf16", 8, 2, 1, 640), ("bf16", 8, 2, 1, 4096),
                                                  ("bf16", 64, 4, 10, 4096), ("f32", 4, 2, 3, 4096),
                                                  ("bf16", 8, 1, 4, 4096)])
def test_a_value_that_all_rows_see_reaches_them(dtype, heads, kvh, M, cap, bad):
    """NaN and infinity far from any mask's edge, with weights of many sizes, through every form."""
    torch = _torch()
    c, g = _filled(dtype, 1, kvh, 128, 64, 1, 9, seed=12, room=cap // 64 - 9)
    q = torch.randn(1, M, heads, 128, generator=g, device="cuda").to(_dtype(dtype))
    want = c.attention(0, q, _ints([500]))
    for at in (0, 70, 200, 499):
        e = int(c.table[0, at // 64])
        was = c.pages[e, 0, 1, 0, at % 64, 9].clone()
        c.pages[e, 0, 1, 0, at % 64, 9] = bad
        z = c.attention(0, q, _ints([500])).float()
        hit = z[0, :, :heads // kvh, 9]
        assert (torch.isnan(hit) if bad != bad else hit == bad).all(), at
        z[0, :, :heads // kvh, 9] = want[0, :, :heads // kvh, 9].float()
        assert torch.equal(z, want.float())
        c.pages[e, 0, 1, 0, at % 64, 9] = was
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_missing_page_is_told(dtype):
    torch = _torch()
    c, g = _filled(dtype, 1, 2, 128, 16, 2, 20, seed=1)
    q = torch.randn(2, 1, 4, 128, generator=g, device="cuda").to(_dtype(dtype))
    want = c.attention(0, q, _ints([300, 250]))
    c.table[0, 4] = -1
    got = c.attention(0, q, _ints([300, 250]))
    assert torch.equal(got[1], want[1]) and _err(c) == R.TABLE
    c.table[0, 4] = c.n_pages
    got = c.attention(0, q, _ints([300, 250]))
    assert torch.equal(got[1], want[1]) and _err(c) == R.TABLE
    # in front of what any row sees, and behind it, pages may be missing
    got = c.attention(0, q, _ints([300, 250]), window=300 - 80 + 1)
    c.table[0, 19] = -1
    again = c.attention(0, q, _ints([300, 250]), window=300 - 80 + 1)
    assert torch.equal(got, again)
    c.check()


@pytest.mark.parametrize("dtype,heads,room", [("bf16", 4, 0), ("bf16", 4, 2100), ("bf16", 64, 2100),
                                              ("f32", 4, 2100)])
def test_bad_positions_leave_the_output(dtype, heads, room):
    torch = _torch()
    c, g = _filled(dtype, 1, 2, 128, 16, 5, 4, seed=2, room=room // 16)
    q = torch.randn(5, 3, heads, 128, generator=g, device="cuda").to(_dtype(dtype))
    out = torch.full_like(q, 3.0)
    pos, rows = [c.max_seq - 2, -1, 5, 5, 30], [3, 1, 4, -1, 3]
    c.attention(0, q, _ints(pos), rows=_ints(rows), out=out)
    assert (out[:4] == 3.0).all() and (out[4] != 3.0).any() and _err(c) == R.CAPACITY | R.CONTROL
    out.fill_(3.0)
    pos, rows = [2 ** 31 - 1, -2 ** 31, 1 << 30, 0, 0], [1, 1, 1, 2 ** 31 - 1, -2 ** 31]
    c.attention(0, q, _ints(pos), rows=_ints(rows), out=out)
    assert (out == 3.0).all() and _err(c) == R.CAPACITY | R.CONTROL
    c.attention(0, q, _ints([30, 30, 30, 30, 30]), rows=_ints([3] * 5), out=out, longest=32)
    assert (out == 3.0).all() and _err(c) == R.CAPACITY


@pytest.mark.parametrize("dtype,hd,heads,room", [("f32", 64, 8, 0), ("f32", 128, 4, 2100), ("bf16", 64, 8, 0),
                                                 ("bf16", 128, 8, 2100), ("bf16", 128, 64, 2100)])
def test_scores_of_every_size(dtype, hd, heads, room):
    """Scores from zero to 1e4, where one key takes it all, and up to 1e32, where rounding decides which."""
    torch = _torch()
    c, g = _filled(dtype, 1, 2, hd, 32, 2, 10, seed=3, room=room // 32)
    q = torch.randn(2, 3, heads, hd, generator=g, device="cuda")
    q[0, 0] *= 1000.0
    q[0, 1] = 0.0
    q[1, 0] *= 1e-20
    q = q.to(_dtype(dtype))
    _check_attention(c, 0, q, [200, 290], [3, 3])
    for scale in (1e7, 1e30):  # rows with scores far apart in one tile
        mixed = q.clone()
        mixed[:, 1, ::3] = scale
        got = c.attention(0, mixed, _ints([200, 290]))
        want = c.attention(0, q, _ints([200, 290]))
        same = torch.ones(heads, dtype=torch.bool, device="cuda")
        same[::3] = False
        off = (got.float() - want.float()).abs()[:, 1][:, same]
        assert torch.isfinite(got.float()).all() and off.max() <= 2.0 ** -6 * want.float().abs().max()
    _check_attention(c, 0, mixed[:, ::2].contiguous(), [200, 290], [2, 2])
    held = c.table[0, :10].long()
    one, slot = c.table[0, 130 // 32].long(), 130 % 32
    for scale in (1e6, 1e9, 1e13, 1e30):
        # all keys alike but for one, whose score is twice as large: its value is the answer
        c.pages[held, 0, 0] = 0.5
        c.pages[one, 0, 0, :, slot] = 1.0
        big = torch.full_like(q, scale)
        got = c.attention(0, big, _ints([200, 290]))
        want = c.pages[one, 0, 1, :, slot]
        assert torch.equal(got[0], want.repeat_interleave(heads // 2, 0).expand(3, heads, hd))
        # all alike: the mean of 201 values. A sum of 201 terms in fp32, its parts' weights and the
        # division: below 2^-16 of the mean magnitude
        c.pages[one, 0, 0, :, slot] = 0.5
        got = c.attention(0, big, _ints([200, 290]))[0, 0].double()
        v = c.pages[held, 0, 1].double().permute(1, 0, 2, 3).reshape(2, -1, hd)[:, :201]
        mean, off = v.mean(1)[:, None], v.abs().mean(1)[:, None] * 2.0 ** -16
        half = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
        assert ((got.view(2, heads // 2, hd) - mean).abs() <= off + half * (mean.abs() + off)).all()
    c.check()


def test_long_cache_beyond_32_bits():
    """Pages behind 2^32 bytes and 2^31 elements, a long sequence whose pages lie there."""
    torch = _torch()
    page, heads, layers = 64, 8, 32
    c = _cache("bf16", layers, heads, 128, 640, page, 2, 320)  # 5.4 GB
    assert c.pages.numel() > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(4)
    high = torch.randperm(320, generator=g, device="cuda").int() + 320
    c.table[1] = high
    c.refs[high.long()] = 1
    c.pages[320:, 31] = torch.randn(320, 2, heads, page, 128, generator=g, device="cuda").bfloat16()
    M, pos = 2, 20000
    x = torch.randn(2, M, heads, 128, generator=g, device="cuda").bfloat16()
    q = torch.randn(2, M, 32, 128, generator=g, device="cuda").bfloat16()
    c.append(31, x, x, _ints([0, pos]), rows=_ints([0, M]))
    got = c.attention(31, q, _ints([0, pos]), rows=_ints([0, M]))
    c.check()
    at = high.long()
    kk, vv = (c.pages[at, 31, s].permute(1, 0, 2, 3).reshape(heads, -1, 128)[:, :pos + M].double()
              for s in (0, 1))
    assert torch.equal(kk[:, pos:], x[1].transpose(0, 1).double())
    for m in range(M):
        qq = q[1, m].double().view(heads, 4, 128)
        s = torch.einsum("ghd,gjd->ghj", qq, kk[:, :pos + m + 1]) / 128 ** 0.5
        w = torch.softmax(s, -1)
        o = torch.einsum("ghj,gjd->ghd", w, vv[:, :pos + m + 1])
        mag = torch.einsum("ghj,gjd->ghd", w, vv[:, :pos + m + 1].abs())
        off = (got[1, m].double().view(heads, 4, 128) - o).abs()
        # the roundings of paged_ref.attention: scores of at most 16 here, 8 bits of a probability
        rel = 2 * (18 * 2.0 ** -23 * 160 + 2.0 ** -22 * 17) + 2.0 ** -8 + (64 + pos / 64) * 2.0 ** -24
        assert (off <= rel * mag + 2.0 ** -8 * (o.abs() + rel * mag)).all()
    # copying and moving up there
    c.fork(_ints([1, 1]))
    c.reserve(_ints([pos + M, pos + M]), 1)
    r = c.table.tolist()
    e0, e1 = r[0][(pos + M) // page], r[1][(pos + M) // page]
    kept = (pos + M) % page
    assert e0 == 0 and e1 == int(high[(pos + M) // page])
    assert torch.equal(c.pages[e0, :, :, :, :kept], c.pages[e1, :, :, :, :kept])
    was = c.pages[at, 31].clone()
    assert int(c.compact().item()) == 321
    assert torch.equal(c.pages[c.table[1].long(), 31], was)
    assert torch.equal(got[1], c.attention(31, q, _ints([0, pos]), rows=_ints([0, M]))[1])
    c.check()


# ------------------------------------------------------------------ as they are used

def _step(c, layer_kv, q, parent, pos, rows):
    """A step of a search: fork, reserve, append and attend on both layers; positions move on the device."""
    outs = []
    c.fork(parent)
    c.reserve(pos, rows)
    for layer in range(c.n_layers):
        k, v = layer_kv[layer]
        c.append(layer, k, v, pos)
        outs.append(c.attention(layer, q, pos))
    pos += 1
    return outs


def test_a_search_in_a_graph():
    """Steps of a search over four continuations, captured once and replayed, against the same steps
    called one by one and against the reference."""
    torch = _torch()
    made = []
    for _ in range(2):
        c = _cache("bf16", 2, 2, 64, 40, 16, 4, 8)
        c.reserve(_ints([0] * 4), _ints([21, 0, 0, 0]))
        g = torch.Generator(device="cuda").manual_seed(5)
        x = torch.randn(4, 21, 2, 64, generator=g, device="cuda").bfloat16()
        for layer in range(2):
            c.append(layer, x, -x, _ints([0] * 4), rows=_ints([21, 0, 0, 0]))
        made.append(c)
    eager, captured = made
    ref = _twin(eager)
    parent = _ints([0, 0, 0, 0])
    q = torch.zeros(4, 1, 4, 64, device="cuda").bfloat16()
    kv = [tuple(torch.zeros(4, 1, 2, 64, device="cuda").bfloat16() for _ in range(2)) for _ in range(2)]
    pos = _ints([21] * 4)
    pos_g = pos.clone()
    one = _ints([1] * 4)
    warm = _cache("bf16", 2, 2, 64, 40, 16, 4, 8)
    _step(warm, kv, q, _ints([0] * 4), pos.clone(), one)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs_g = _step(captured, kv, q, parent, pos_g, one)
    rng = np.random.default_rng(6)
    at = 21
    for step in range(30):
        p = [0, 0, 0, 0] if step == 0 else [int(x) for x in rng.integers(0, 4, 4)]
        parent.copy_(_ints(p))
        q.normal_()
        for k, v in kv:
            k.normal_()
            v.normal_()
        outs = _step(eager, kv, q, parent, pos, one)
        graph.replay()
        ref.fork(p)
        ref.reserve([at] * 4, [1] * 4)
        for layer in range(2):
            ref.append(layer, kv[layer][0].float().cpu().numpy(), kv[layer][1].float().cpu().numpy(),
                       [at] * 4, [1] * 4)
            assert torch.equal(outs[layer], outs_g[layer])
            want, bound = R.attention(ref, layer, q.float().cpu().numpy(), [at] * 4, [1] * 4, [0] * 4, 0, 8)
            off = np.abs(outs[layer].float().cpu().numpy() - want)
            assert (off <= bound + 2.0 ** -8 * (np.abs(want) + bound)).all()
        at += 1
        _agree(eager, ref)
        _agree(captured, ref)
    eager.check()
    captured.check()


def test_calls_in_a_row_without_a_wait():
    """A call's first kernel is resident before the kernel in front of it has ended: steps whose positions, parents,
    rows and queries are made by kernels right in front of the calls that read them, against the same
    steps with a wait behind everything."""
    torch = _torch()

    def run(wait):
        c = _cache("bf16", 1, 2, 128, 60, 16, 6, 9)
        g = torch.Generator(device="cuda").manual_seed(21)
        pos = torch.zeros(6, dtype=torch.int32, device="cuda")
        parent = torch.arange(6, dtype=torch.int32, device="cuda")
        kv = torch.randn(6, 1, 4, 128, generator=g, device="cuda").bfloat16()
        q = torch.randn(6, 1, 8, 128, generator=g, device="cuda").bfloat16()
        mix = torch.randn(8, 8, generator=g, device="cuda").bfloat16()
        outs = []

        def then():
            if wait:
                torch.cuda.synchronize()
        for step in range(120):
            parent.add_(step % 3).remainder_(6)
            then()
            c.fork(parent)
            then()
            pos = pos[parent.long()]
            then()
            c.reserve(pos, 1)
            then()
            c.append(0, kv[:, :, :2], kv[:, :, 2:], pos)
            then()
            o = c.attention(0, q, pos, longest=144 if step % 2 else 0)
            then()
            q = torch.einsum("bmhd,hg->bmgd", o, mix).contiguous()
            kv = torch.tanh(o[:, :, :4] * 3).contiguous()
            then()
            pos = pos + 1
            if step % 40 == 39:
                used = c.compact()
                pos = pos // 2
                c.truncate(pos)
                outs.append(used)
            outs.append(o)
        torch.cuda.synchronize()
        c.check()
        return outs, c
    a, ca = run(True)
    for _ in range(3):
        b, cb = run(False)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        assert torch.equal(ca.table, cb.table) and torch.equal(ca.refs, cb.refs)
        assert torch.equal(ca.pages, cb.pages)


def test_calls_on_another_stream():
    """Every call given a stream of its own, while the current stream is busy with others' work."""
    torch = _torch()
    s = torch.cuda.Stream()
    c, g = _filled("bf16", 1, 2, 128, 16, 3, 6, seed=9, extra=20)
    d = _cache("bf16", 1, 2, 128, c.n_pages, 16, 3, 6)
    for t, u in ((d.pages, c.pages), (d.table, c.table), (d.refs, c.refs)):
        t.copy_(u)
    x = torch.randn(3, 2, 2, 128, generator=g, device="cuda").bfloat16()
    q = torch.randn(3, 2, 8, 128, generator=g, device="cuda").bfloat16()
    parent, pos, rows = _ints([1, 1, 2]), _ints([50, 50, 70]), _ints([2, 2, 2])
    torch.cuda.synchronize()

    def steps(c, **kw):
        c.fork(parent, **kw)
        c.reserve(pos, rows, **kw)
        c.append(0, x, x, pos, **kw)
        used = c.compact(**kw)
        return c.attention(0, q, pos, longest=96, **kw), used
    a, used_a = steps(c)
    torch.cuda.synchronize()
    busy = torch.randn(4096, 4096, device="cuda")
    for _ in range(20):
        busy = busy @ busy * 1e-3
    b, used_b = steps(d, stream=s)
    s.synchronize()
    assert torch.equal(a, b) and torch.equal(used_a, used_b) and torch.equal(c.table, d.table)
    assert torch.equal(c.pages, d.pages) and torch.equal(c.refs, d.refs)
    with pytest.raises(ValueError):
        c.fork(parent.cpu())
    c.check()


def test_two_attentions_at_once():
    """Two layers on two streams, eager and as two captured graphs: nothing is shared between the calls."""
    torch = _torch()
    c, g = _filled("bf16", 2, 4, 128, 32, 2, 100, seed=10)
    q = [torch.randn(2, 3, 16, 128, generator=g, device="cuda").bfloat16() for _ in range(2)]
    pos = _ints([3000, 1700])
    want = [c.attention(i, q[i], pos).clone() for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        got = [c.attention(i, q[i], pos, stream=streams[i]) for i in range(2)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs, outs = [], []
    for i in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(c.attention(i, q[i], pos))
        graphs.append(gr)
    for _ in range(10):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for gr, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    c.check()
