"""Operators over a paged KV cache, as cases that can be timed and compared.

The cache is a pool of pages. A page holds P positions of a sequence, K and V, all layers and heads;
a table names the pages of each sequence (-1: none), and `refs` counts for each page the entries
that name it (0: the page is free).

- "beam": a step of a search over several continuations: every sequence becomes a copy of its
  parent (fork: it shares the parent's pages), then gets a place for its next row (reserve: a shared
  page that is written next is copied first, and only the positions that are kept; a page that
  all of its sharers ask for stays with the last of them; new pages are the lowest free ones, in the
  order of sequences and positions).
- "admit": the oldest sequences end (their pages are free), the others move up, the last
  places get pages for new prompts and the running ones for their next row.
- "compact": the same with few, long sequences, and in between the pages in use move to the low end
  of the pool (the k-th page behind it to the k-th free one within it).
- "append": new K and V rows of every sequence go into the pages of a layer.
- "attend": attention of each sequence's new rows over the pages of a layer: row m sits at position
  pos + m and sees the keys up to its own position, from `first` on, and at most `window` of them. A
  row that sees none is zero; rows from `rows` on are left as they were.

Sizes are those of the decoder shapes in synth/workloads.py (layers, heads, head sizes, prompt
lengths, rows of a verification), the longer contexts and the batches are generic.
"""
from __future__ import annotations

import math

import torch

own = False

# layers, n_heads, n_kv_heads, head_dim, dtype of the decoder shapes
SHAPES = {"tiny": (4, 4, 4, 64, "f32"), "7b": (32, 32, 32, 128, "bf16"),
          "8b": (32, 32, 8, 128, "bf16"), "13b": (40, 40, 40, 128, "bf16"),
          "70b": (80, 64, 8, 128, "bf16")}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LAYERS = 2  # of the caches that an append or an attention works on, in the second of them


def listed():
    return [
        # four continuations of the fp32 decoder's prompt: nothing but latency
        dict(name="beam-tiny-4", kind="beam", shape="tiny", seqs=4, pos=40, page=16),
        # sixty-four answers sampled from one prompt of the 8B shape
        dict(name="beam-8b-64", kind="beam", shape="8b", seqs=64, pos=1064, page=64),
        # a server's step: 12 of 192 users leave, 12 prompts come, the others decode
        dict(name="admit-8b-192", kind="admit", shape="8b", seqs=192, ends=12, pos=2048, page=16),
        # two sequences of the fp32 decoder and their few pages
        dict(name="compact-tiny-2", kind="compact", shape="tiny", seqs=2, ends=1, pos=96, page=16),
        # one of four long sequences of the largest shape ends: bytes are everything
        dict(name="compact-70b-4", kind="compact", shape="70b", seqs=4, ends=1, pos=1600, page=16),
        # one decode step of sixteen users, each at a place of its own
        dict(name="append-8b-batch16", kind="append", shape="8b", seqs=16, rows=1, pos=1500,
             page=16, ragged=True),
        # a whole prompt behind a one-token prefix: every page of it starts in a tile's middle
        dict(name="append-13b-prompt2047", kind="append", shape="13b", seqs=1, rows=2047, pos=1,
             page=64, ragged=False),
        # the smallest attention there is: the fp32 decoder's verification of four drafts
        dict(name="attend-tiny-verify5", kind="attend", shape="tiny", seqs=1, rows=5, pos=40,
             page=16, ragged=False, window=0),
        # a draft (or autoregressive) step at the 8B shape's usual context
        dict(name="attend-8b-draft", kind="attend", shape="8b", seqs=1, rows=1, pos=1100, page=16,
             ragged=False, window=0),
        # the same step at the end of a long document: bytes are everything
        dict(name="attend-8b-long", kind="attend", shape="8b", seqs=1, rows=1, pos=131071, page=64,
             ragged=False, window=0),
        # the widest verification (16 drafts, 8 query heads to a KV head) over a long context
        dict(name="attend-70b-verify17", kind="attend", shape="70b", seqs=1, rows=17, pos=16000,
             page=64, ragged=False, window=0),
        # a padded batch: every sequence with a start, a length and a number of rows of its own,
        # under a sliding window
        dict(name="attend-7b-batch24", kind="attend", shape="7b", seqs=24, rows=5, pos=4000, page=16,
             ragged=True, window=2500),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _page_bytes(shape, page, layers):
    _, _, heads, hd, dtype = SHAPES[shape]
    return layers * 2 * heads * page * hd * (4 if dtype == "f32" else 2)


def draw(rng):
    kind = rng.choice(["beam", "admit", "compact", "append", "attend", "attend", "attend"])
    shape = rng.choice(list(SHAPES))
    layers, heads, kv_heads, hd, dtype = SHAPES[shape]
    page = rng.choice([16, 32, 64, 128])
    if kind == "beam":
        page = min(page, 64)
        per = _page_bytes(shape, page, layers)
        seqs = _log_uniform(rng, 2, max(3, min(64, (1 << 30) // (2 * per))))
        most = max(page, ((5 << 28) // per - 2 * seqs - 2) * page)
        return dict(kind=kind, shape=shape, seqs=seqs, pos=_log_uniform(rng, 8, min(most, 4000)),
                    page=page)
    if kind == "admit":
        seqs = _log_uniform(rng, 4, 192)
        return dict(kind=kind, shape=shape, seqs=seqs, ends=rng.randint(1, max(1, seqs // 8)),
                    pos=_log_uniform(rng, 16, 4000), page=page)
    if kind == "compact":
        page = 16 if shape != "tiny" else page
        seqs = rng.randint(2, 6)
        most = (2 << 30) // _page_bytes(shape, page, layers) // (seqs + 1) * page
        return dict(kind=kind, shape=shape, seqs=seqs, ends=rng.randint(1, max(1, seqs // 3)),
                    pos=_log_uniform(rng, 16, min(most, 4000)), page=page)
    seqs = rng.choice([1, 1, _log_uniform(rng, 2, 32)])
    if kind == "append":
        rows = _log_uniform(rng, 1, max(2, 2047 // seqs))
        return dict(kind=kind, shape=shape, seqs=seqs, rows=rows, pos=rng.randint(0, 4000),
                    page=page, ragged=seqs > 1 and rng.random() < 0.7)
    rows = rng.choice([1, 1, rng.randint(2, 17)])
    most = min(131000, 130000 * 8 // (seqs * kv_heads), (40 << 20) // (rows * seqs * heads // 4 + 1))
    pos = _log_uniform(rng, 1, max(64, most))
    window = rng.choice([0, 0, _log_uniform(rng, 16, 4096)])
    return dict(kind=kind, shape=shape, seqs=seqs, rows=rows, pos=pos, page=page,
                ragged=seqs > 1 and rng.random() < 0.7, window=window)


# ------------------------------------------------------------------ inputs

def _places(case, g, dev):
    """Positions of the first new rows, numbers of new rows, first visible positions."""
    n = case["seqs"]
    if not case["ragged"]:
        return (torch.full((n,), case["pos"], dtype=torch.int32, device=dev),
                torch.full((n,), case["rows"], dtype=torch.int32, device=dev),
                torch.zeros(n, dtype=torch.int32, device=dev))
    pos = torch.randint(case["pos"] // 8, case["pos"] + 1, (n,), generator=g, device=dev)
    rows = torch.randint(1, case["rows"] + 1, (n,), generator=g, device=dev)
    # half of the sequences are padded on the left
    first = torch.randint(0, 2, (n,), generator=g, device=dev) * (pos // 3)
    return pos.int(), rows.int(), first.int()


def _scattered(n, width, held, pool, g, dev):
    """A table whose sequence b holds held[b] pages of the pool, no two the same, in no order."""
    at = torch.arange(width, device=dev) < held[:, None]
    free = torch.randperm(pool, generator=g, device=dev)[:n * width].int().view(n, width)
    return torch.where(at, free, -1)


def _counts(table, n_pages):
    """How many entries name each page."""
    flat = table.flatten()
    return torch.zeros(n_pages, dtype=torch.int32, device=table.device).scatter_add_(
        0, flat.clamp_min(0).long(), (flat >= 0).int())


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    layers, heads, kv_heads, hd, dtype = SHAPES[case["shape"]]
    dt, n, P, kind = TYPES[dtype], case["seqs"], case["page"], case["kind"]
    st = dict(case=case)
    if kind in ("append", "attend"):
        layers = LAYERS
        pos, rows, first = _places(case, g, dev)
        width = (case["pos"] + case["rows"] + P - 1) // P
        pool = n * width + 8
        table = _scattered(n, width, (pos + rows + P - 1) // P, pool, g, dev)
        # q, k and v of the new rows as the QKV product leaves them: one row of all three
        M = case["rows"]
        qkv = torch.randn(n, M, heads + 2 * kv_heads, hd, generator=g, device=dev)
        qkv[:, :, heads:] *= torch.exp(0.3 * torch.randn(1, 1, 2 * kv_heads, 1, generator=g,
                                                         device=dev))
        if kind == "attend":
            # scores of a spread of about 1.5, in every head a little different
            qkv[:, :, :heads] *= 1.2 * torch.exp(0.2 * torch.randn(1, 1, heads, 1, generator=g,
                                                                   device=dev))
            st["out"] = torch.zeros(n, M, heads, hd, dtype=dt, device=dev)
        qkv = qkv.to(dt)
        st.update(q=qkv[:, :, :heads], new_k=qkv[:, :, heads:heads + kv_heads],
                  new_v=qkv[:, :, heads + kv_heads:], pos=pos, rows=rows, first=first)
    elif kind == "beam":
        # one prompt's whole pages are shared, the page that is being filled is each one's own
        whole = case["pos"] // P
        width, pool = whole + 2, whole + 2 * n + 2
        ids = torch.randperm(pool, generator=g, device=dev).int()
        table = torch.full((n, width), -1, dtype=torch.int32, device=dev)
        table[:, :whole] = ids[:whole]
        table[:, whole] = ids[whole:whole + n]
        st.update(parent=torch.randint(0, n, (n,), generator=g, device=dev).int(),
                  pos=torch.full((n,), case["pos"], dtype=torch.int32, device=dev),
                  rows=torch.ones(n, dtype=torch.int32, device=dev))
    else:
        # every sequence holds `pos` positions; the last `ends` places take prompts as long
        each = (case["pos"] + P - 1) // P
        width, ends = each + 1, case["ends"]
        pool = n * width + (n * width) // 4 + 1
        # the pages in use are the lowest ones, as a compacted pool's are, but in no order
        low = torch.randperm(n * each, generator=g, device=dev).int().view(n, each)
        table = torch.full((n, width), -1, dtype=torch.int32, device=dev)
        table[:, :each] = low
        parent = torch.arange(n, device=dev).int() + ends
        fresh = torch.arange(n, device=dev) >= n - ends
        st.update(parent=torch.where(fresh, -1, parent).int(),
                  pos=torch.where(fresh, 0, case["pos"]).int(),
                  rows=torch.where(fresh, case["pos"], 1).int())
        if kind == "admit":  # (the pages' contents are not touched)
            layers = 1
    shape = (pool, layers, 2, kv_heads, P, hd)
    if kind == "admit":
        pages = torch.zeros(shape, dtype=dt, device=dev)
    else:
        pages = torch.empty(shape, dtype=dt, device=dev)
        pages.normal_(generator=g)
        # channels differ in size, as those of K and V do
        pages *= torch.exp(0.4 * torch.randn(1, layers, 2, kv_heads, 1, hd, generator=g,
                                             device=dev)).to(dt)
    refs = _counts(table, pool)
    if own:
        from paper_2606_03113_gb300.runtime import PagedKVCache
        cache = PagedKVCache(layers, kv_heads, hd, pool, page=P, n_seq=n, max_seq=width * P, dtype=dt,
                             device=dev)
        cache.pages.copy_(pages)
        cache.table.copy_(table)
        cache.refs.copy_(refs)
        st["cache"] = cache
    else:
        st.update(pages=pages, table=table, refs=refs)
    return st


# ------------------------------------------------------------------ plain forms

def _fork_plain(st):
    table, refs, parent = st["table"], st["refs"], st["parent"].long()
    new = torch.where((parent >= 0)[:, None], table[parent.clamp_min(0)], -1)
    refs += _counts(new, refs.numel()) - _counts(table, refs.numel())
    table.copy_(new)


def _reserve_plain(st):
    table, refs, pages = st["table"], st["refs"], st["pages"]
    n, W = table.shape
    N, P = refs.numel(), st["case"]["page"]
    pos, rows = st["pos"].long()[:, None], st["rows"].long()[:, None]
    i = torch.arange(W, device=table.device)
    b = torch.arange(n, device=table.device)[:, None].expand(n, W)
    first = pos // P
    want = (i >= first) & (i <= (pos + rows - 1) // P) & (rows > 0)
    e = table.clamp_min(0).long()
    shared = want & (table >= 0) & (refs[e] > 1)
    zero = torch.zeros(N, dtype=torch.int32, device=table.device)
    claims = zero.scatter_add(0, e.flatten(), shared.flatten().int())
    last = zero.long().scatter_reduce(0, e.flatten(), torch.where(shared, b + 1, 0).flatten(), "amax")
    keep = shared & (claims == refs)[e] & (last[e] == b + 1)
    need = want & ((table < 0) | (shared & ~keep))
    need &= need.sum() <= (refs == 0).sum()  # all of them or none
    lowest = torch.argsort((refs > 0).int(), stable=True)  # the free ones first
    rank = need.flatten().int().cumsum(0).view(n, W) - 1
    new = lowest[rank.clamp_min(0)]
    # what is kept of the pages that a sequence no longer shares
    copied = need & shared & (i == first) & (pos % P > 0)
    at = torch.nonzero(copied)
    src, dst = e[at[:, 0], at[:, 1]], new[at[:, 0], at[:, 1]]
    kept = (torch.arange(P, device=table.device) < (pos % P)[at[:, 0]])[:, None, None, None, :, None]
    pages[dst] = torch.where(kept, pages[src], pages[dst])
    refs.scatter_add_(0, new.flatten(), need.flatten().int())
    refs.scatter_add_(0, e.flatten(), -(need & shared).flatten().int())
    table.copy_(torch.where(need, new.int(), table))


def _compact_plain(st):
    table, refs, pages = st["table"], st["refs"], st["pages"]
    ids = torch.arange(refs.numel(), device=refs.device)
    used = refs > 0
    low = used.sum()
    src = torch.nonzero(used & (ids >= low))[:, 0]
    dst = torch.nonzero(~used & (ids < low))[:, 0]
    pages[dst] = pages[src]
    ids[src] = dst
    table.copy_(torch.where(table >= 0, ids[table.clamp_min(0).long()].int(), -1))
    refs[dst] = refs[src]
    refs[src] = 0
    return low.int().view(1)


def _append_plain(st):
    pos, rows, pages = st["pos"].long(), st["rows"], st["pages"]
    n, M, heads, hd = st["new_k"].shape
    P = st["case"]["page"]
    m = torch.arange(M, device=pos.device)
    b, m = torch.nonzero(m < rows[:, None], as_tuple=True)
    p = pos[b] + m
    page = st["table"][b, p // P].long()
    h = torch.arange(heads, device=pos.device)
    pages[page[:, None], LAYERS - 1, 0, h, (p % P)[:, None]] = st["new_k"][b, m]
    pages[page[:, None], LAYERS - 1, 1, h, (p % P)[:, None]] = st["new_v"][b, m]


def _visible(pos, first, M, S, window):
    """(n, M, S): which keys each row sees."""
    dev = pos.device
    p = pos.long()[:, None] + torch.arange(M, device=dev)
    j = torch.arange(S, device=dev)
    lo = first.long()[:, None].expand_as(p)
    if window:
        lo = torch.maximum(lo, p - window + 1)
    return (j >= lo[..., None]) & (j <= p[..., None])


def _attend_plain(st):
    case, q = st["case"], st["q"]
    n, M, heads, hd = q.shape
    kvh = st["pages"].shape[3]
    S = case["pos"] + M
    held = st["table"].clamp_min(0).long()  # (a page that is not there is not seen)

    def values(side):
        x = st["pages"][:, LAYERS - 1, side][held]      # (n, W, kvh, P, hd)
        return x.permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :S].float()
    qf = q.float().view(n, M, kvh, heads // kvh, hd).permute(0, 2, 3, 1, 4)  # (n, kvh, G, M, hd)
    s = torch.matmul(qf.reshape(n, kvh, -1, hd), values(0).transpose(-1, -2))
    s = s.view(n, kvh, heads // kvh, M, S) * (1.0 / math.sqrt(hd))
    see = _visible(st["pos"], st["first"], M, S, case["window"])[:, None, None]
    s = torch.where(see, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.where(see, torch.exp(s - torch.where(m == -math.inf, 0.0, m)), 0.0)
    o = torch.matmul(e.view(n, kvh, -1, S), values(1)).view(n, kvh, heads // kvh, M, hd)
    o = torch.where(see.any(-1, keepdim=True), o / e.sum(-1, keepdim=True), 0.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(n, M, heads, hd).to(q.dtype)
    live = torch.arange(M, device=q.device) < st["rows"][:, None]
    return torch.where(live[:, :, None, None], o, st["out"])


def run(st):
    case = st["case"]
    kind = case["kind"]
    if own:
        c = st["cache"]
        if kind == "attend":
            return c.attention(LAYERS - 1, st["q"], st["pos"], rows=st["rows"], first=st["first"],
                               window=case["window"], longest=case["pos"] + case["rows"],
                               out=st["out"])
        if kind == "append":
            c.append(LAYERS - 1, st["new_k"], st["new_v"], st["pos"], rows=st["rows"])
            return c.pages
        c.fork(st["parent"])
        got = dict(used=c.compact()) if kind == "compact" else {}
        c.reserve(st["pos"], st["rows"])
        got.update(table=c.table, refs=c.refs)
        if kind != "admit":
            got["pages"] = c.pages
        return got
    if kind == "attend":
        return _attend_plain(st)
    if kind == "append":
        _append_plain(st)
        return st["pages"]
    _fork_plain(st)
    got = dict(used=_compact_plain(st)) if kind == "compact" else {}
    _reserve_plain(st)
    got.update(table=st["table"], refs=st["refs"])
    if kind != "admit":
        got["pages"] = st["pages"]
    return got


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    layers, heads, kvh, hd, dtype = SHAPES[case["shape"]]
    elt = 4 if dtype == "f32" else 2
    n, P, kind = case["seqs"], case["page"], case["kind"]
    if kind in ("beam", "admit", "compact"):
        # the table and the counts are read and written; `each`: pages of a sequence
        each = (case["pos"] + P - 1) // P
        per = _page_bytes(case["shape"], P, layers)
        if kind == "beam":
            # sequences that share their parent, but for the last of each parent's
            copies = n * (1 - 1 / n) ** n
            kept = case["pos"] % P / P
            pool = case["pos"] // P + 2 * n + 2
            return dict(bytes=2 * copies * kept * per + 8 * (n * (each + 1) + pool) + 12 * n, flops=0)
        pool = n * (each + 1) + n * (each + 1) // 4 + 1
        small = 8 * (n * (each + 1) + pool) + 12 * n
        if kind == "admit":
            return dict(bytes=small, flops=0)
        moved = case["ends"] * each * (1 - case["ends"] / n)
        return dict(bytes=2 * moved * per + small, flops=0)
    M = case["rows"]
    # ragged cases: the middle of the ranges that _places draws from
    pos = case["pos"] * (9 / 16 if case["ragged"] else 1)
    rows = (M + 1) / 2 if case["ragged"] else M
    first = pos / 6 if case["ragged"] else 0
    if kind == "append":
        return dict(bytes=4 * n * rows * kvh * hd * elt + 8 * n + 4 * n * (rows / P + 1), flops=0)
    w = case["window"] or 1 << 40
    keys = min(pos + rows - first, w + rows - 1)   # that some row sees
    pairs = rows * min(pos + (rows + 1) / 2 - first, w)
    kv = n * keys * (kvh * 2 * hd * elt + 4 / P)
    return dict(bytes=kv + 2 * n * rows * heads * hd * elt, flops=4 * hd * heads * n * pairs)


# ------------------------------------------------------------------ 64 bits, from the definitions

def _plain_state(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def _pages_by_hand(st):
    """What the page calls do to the pages' contents: sequence by sequence, entry by entry."""
    case, P = st["case"], st["case"]["page"]
    table, parent = st["table"].tolist(), st["parent"].tolist()
    pos, rows = st["pos"].tolist(), st["rows"].tolist()
    pages = st["pages"]
    table = [list(table[p]) if p >= 0 else [-1] * len(table[0]) for p in parent]

    def uses():
        count = [0] * pages.shape[0]
        for line in table:
            for e in line:
                if e >= 0:
                    count[e] += 1
        return count
    count = uses()
    if case["kind"] == "compact":
        held = [e for e in range(len(count)) if count[e]]
        holes = [e for e in range(len(held)) if not count[e]]
        to = dict(zip([e for e in held if e >= len(held)], holes))
        for a, z in to.items():
            pages[z] = pages[a]
        table = [[to.get(e, e) for e in line] for line in table]
        count = uses()
    free = [e for e in range(len(count)) if not count[e]]
    for b, line in enumerate(table):
        for i in range(pos[b] // P, (pos[b] + rows[b] - 1) // P + 1 if rows[b] else 0):
            e = line[i]
            if e >= 0 and count[e] == 1:
                continue
            line[i] = free.pop(0)
            count[line[i]] = 1
            if e >= 0:
                count[e] -= 1
                if i * P < pos[b]:
                    pages[line[i], ..., :pos[b] - i * P, :] = pages[e, ..., :pos[b] - i * P, :]
    return pages


def exact(case, seed):
    kind = case["kind"]
    if kind == "admit":
        return None
    st = _plain_state(case, seed)
    if kind in ("beam", "compact"):
        got = dict(table=None, refs=None, pages=_pages_by_hand(st))
        if kind == "compact":
            got["used"] = None
        return got
    _, heads, kvh, hd, _ = SHAPES[case["shape"]]
    n, M, P = case["seqs"], case["rows"], case["page"]
    pos, rows, first = (st[x].tolist() for x in ("pos", "rows", "first"))
    table = st["table"].tolist()
    pages = st["pages"]
    if kind == "append":
        for b in range(n):
            done = 0
            while done < rows[b]:
                at = pos[b] + done
                m = min(P - at % P, rows[b] - done)
                for side, name in ((0, "new_k"), (1, "new_v")):
                    pages[table[b][at // P], LAYERS - 1, side, :, at % P:at % P + m] = \
                        st[name][b, done:done + m].transpose(0, 1)
                done += m
        return pages
    out = torch.zeros(n, M, heads, hd, dtype=torch.float64, device=st["q"].device)
    for b in range(n):
        hi = pos[b] + rows[b]
        lo = max(0, first[b], pos[b] - case["window"] + 1 if case["window"] else 0)
        j = torch.arange(lo, hi, device=out.device)
        p = pos[b] + torch.arange(rows[b], device=out.device)
        bad = (j[None] > p[:, None]) | (j[None] < first[b])
        if case["window"]:
            bad |= j[None] <= p[:, None] - case["window"]
        at = st["table"][b].long()[j // P]
        for g in range(kvh):
            kk, vv = (pages[at, LAYERS - 1, side, g, j % P].double() for side in (0, 1))
            for h in range(g * heads // kvh, (g + 1) * heads // kvh):
                s = st["q"][b, :rows[b], h].double() @ kk.t() / hd ** 0.5
                s[bad] = -math.inf
                out[b, :rows[b], h] = torch.softmax(s, -1).nan_to_num(0.0) @ vv
    return out
