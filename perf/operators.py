"""Operators over an 8-bit KV cache and over logits, as cases that can be timed and compared.

- "append": new K and V rows of every sequence go into the 8-bit cache. A block of 64 positions of
  one KV head has one scale, the smallest power of two that brings the block's largest magnitude to
  448 or less; a row's codes are its values over that scale, rounded to e4m3. Where the new rows
  raise a block's scale, the codes of the rows before them in that block are rounded to the new one.
- "attend": attention of each sequence's new rows over its cache: row m sits at position pos + m and
  sees the keys up to its own position, from `first` on, and at most `window` of them. A row that
  sees none is zero; rows from `rows` on are left as they were.
- "logprobs": of every row of logits, at a temperature: the log-probabilities of given tokens, the
  log-sum-exp, the entropy and the most probable tokens (ties go to the lower id).

Sizes are those of the decoder shapes in synth/workloads.py (heads, head sizes, vocabularies, prompt
lengths, rows of a verification), the longer contexts and the batches are generic.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 64  # positions that share a scale
# n_heads, n_kv_heads, head_dim, vocab, dtype of the decoder shapes
SHAPES = {"tiny": (4, 4, 64, 1024, "f32"), "7b": (32, 32, 128, 32000, "bf16"),
          "8b": (32, 8, 128, 128256, "bf16"), "13b": (40, 40, 128, 32000, "bf16"),
          "70b": (64, 8, 128, 32000, "bf16")}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the rows of a verification pass of the fp32 decoder: nothing but latency
        dict(name="append-tiny-verify5", kind="append", shape="tiny", seqs=1, rows=5, pos=40,
             ragged=False, dtype="f32"),
        # one decode step of sixteen users, each at a place of its own
        dict(name="append-8b-batch16", kind="append", shape="8b", seqs=16, rows=1, pos=1500,
             ragged=True, dtype="bf16"),
        # a whole prompt behind a one-token prefix: every block of it starts in a tile's middle
        dict(name="append-13b-prompt2047", kind="append", shape="13b", seqs=1, rows=2047, pos=1,
             ragged=False, dtype="bf16"),
        # the smallest attention there is: the fp32 decoder's verification of four drafts
        dict(name="attend-tiny-verify5", kind="attend", shape="tiny", seqs=1, rows=5, pos=40,
             ragged=False, window=0, dtype="f32"),
        # a draft (or autoregressive) step at the 8B shape's usual context
        dict(name="attend-8b-draft", kind="attend", shape="8b", seqs=1, rows=1, pos=1100,
             ragged=False, window=0, dtype="bf16"),
        # the same step at the end of a long document: bytes are everything
        dict(name="attend-8b-long", kind="attend", shape="8b", seqs=1, rows=1, pos=131071,
             ragged=False, window=0, dtype="bf16"),
        # the widest verification (16 drafts, 8 query heads to a KV head) over a long context
        dict(name="attend-70b-verify17", kind="attend", shape="70b", seqs=1, rows=17, pos=16000,
             ragged=False, window=0, dtype="bf16"),
        # a padded batch: every sequence with a start, a length and a number of rows of its own,
        # under a sliding window
        dict(name="attend-7b-batch24", kind="attend", shape="7b", seqs=24, rows=5, pos=4000,
             ragged=True, window=2500, dtype="bf16"),
        # a chunk of a prompt behind the chunks before it
        dict(name="attend-8b-chunk512", kind="attend", shape="8b", seqs=1, rows=512, pos=7680,
             ragged=False, window=0, dtype="bf16"),
        # the rows of the fp32 decoder's verification
        dict(name="logprobs-tiny-verify5", kind="logprobs", rows=5, vocab=1024, tokens=1, top=5,
             temperature=1.0, dtype="f32", masked=False),
        # a verification of twelve drafts over the large vocabulary, fp32 logits as the exit head
        # leaves them, with twenty alternatives
        dict(name="logprobs-8b-verify13", kind="logprobs", rows=13, vocab=128256, tokens=1, top=20,
             temperature=0.6, dtype="f32", masked=False),
        # a prompt scored token by token, its logits in bf16, part of the vocabulary ruled out
        dict(name="logprobs-8b-prompt1023", kind="logprobs", rows=1023, vocab=128256, tokens=1,
             top=8, temperature=1.0, dtype="bf16", masked=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "logprobs"])
    if kind == "logprobs":
        vocab = rng.choice([1024, 32000, 128256, _log_uniform(rng, 300, 150000)])
        rows = _log_uniform(rng, 1, max(2, min(2047, 128256 * 1023 // vocab)))
        return dict(kind=kind, rows=rows, vocab=vocab, tokens=rng.randint(1, 4),
                    top=rng.randint(0, 20), temperature=round(rng.uniform(0.5, 1.5), 3),
                    dtype=rng.choice(["f32", "bf16"]), masked=rng.random() < 0.3)
    shape = rng.choice(list(SHAPES))
    heads, kv_heads, hd, _, dtype = SHAPES[shape]
    seqs = rng.choice([1, 1, _log_uniform(rng, 2, 32)])
    if kind == "append":
        rows = _log_uniform(rng, 1, max(2, 2047 // seqs))
        return dict(kind=kind, shape=shape, seqs=seqs, rows=rows, pos=rng.randint(0, 4000),
                    ragged=seqs > 1 and rng.random() < 0.7, dtype=dtype)
    rows = rng.choice([1, rng.randint(2, 17), _log_uniform(rng, 18, 500)])
    if seqs > 1:
        rows = min(rows, 17)
    most = min(131000, 130000 * 8 // (seqs * kv_heads), (40 << 20) // (rows * seqs * heads // 4 + 1))
    pos = _log_uniform(rng, 1, max(64, most))
    window = rng.choice([0, 0, _log_uniform(rng, 16, 4096)])
    return dict(kind=kind, shape=shape, seqs=seqs, rows=rows, pos=pos,
                ragged=seqs > 1 and rng.random() < 0.7, window=window, dtype=dtype)


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


def _scale_of(amax):
    """Smallest power of two s, from 2^-120 to 2^111, with amax <= 448 s."""
    m, e = torch.frexp(amax)  # amax = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    x = torch.where(m <= 0.875, e - 9, e - 8)
    x = torch.where(amax > 0, x, torch.full_like(x, -120)).clamp(-120, 111)
    return torch.ldexp(torch.ones_like(amax), x)


def _codes_of(x, scale):
    return (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _filled(n, heads, seq, hd, spread, g, dev):
    """A cache of values whose channels differ in size, as K and V of a decoder do."""
    size = torch.exp(spread * torch.randn(1, heads, 1, hd, generator=g, device=dev))
    codes = torch.empty((n, heads, seq, hd), dtype=torch.float8_e4m3fn, device=dev)
    scale = torch.empty((n, heads, seq // BLOCK), dtype=torch.float32, device=dev)
    for b in range(n):
        x = torch.randn(heads, seq, hd, generator=g, device=dev) * size[0]
        s = _scale_of(x.view(heads, seq // BLOCK, BLOCK * hd).abs().amax(-1))
        codes[b] = _codes_of(x, s.repeat_interleave(BLOCK, -1)[..., None])
        scale[b] = s
    return codes, scale


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = TYPES[case["dtype"]]
    st = dict(case=case)
    if case["kind"] == "logprobs":
        rows, vocab = case["rows"], case["vocab"]
        z = torch.randn(rows, vocab, generator=g, device=dev) * 2.0
        tok = torch.randint(0, vocab, (rows, case["tokens"]), generator=g, device=dev)
        # the model's own guess is right most of the time
        hit = torch.rand(rows, 1, generator=g, device=dev) < 0.7
        z.scatter_add_(1, tok[:, :1], 12.0 * hit.float())
        if case["masked"]:  # a grammar or a sampler has ruled out a fifth of the vocabulary
            z.masked_fill_(torch.rand(1, vocab, generator=g, device=dev) < 0.2, -math.inf)
        st.update(logits=z.to(dt), tokens=tok.int())
        return st
    heads, kv_heads, hd, _, _ = SHAPES[case["shape"]]
    n, rows = case["seqs"], case["rows"]
    seq = (case["pos"] + rows + BLOCK - 1) // BLOCK * BLOCK + BLOCK
    pos, new, first = _places(case, g, dev)
    k, ks = _filled(n, kv_heads, seq, hd, 0.5, g, dev)
    v, vs = _filled(n, kv_heads, seq, hd, 0.2, g, dev)
    # q, k and v of the new rows as the QKV product leaves them: one row of all three
    qkv = torch.randn(n, rows, heads + 2 * kv_heads, hd, generator=g, device=dev)
    qkv[:, :, heads:] *= torch.exp(0.3 * torch.randn(1, 1, 2 * kv_heads, 1, generator=g, device=dev))
    if case["kind"] == "attend":
        # scores of a spread of about 1.5, in every head a little different
        qkv[:, :, :heads] *= 1.2 * torch.exp(0.2 * torch.randn(1, 1, heads, 1, generator=g,
                                                               device=dev))
    qkv = qkv.to(dt)
    st.update(q=qkv[:, :, :heads], new_k=qkv[:, :, heads:heads + kv_heads],
              new_v=qkv[:, :, heads + kv_heads:], pos=pos, rows=new, first=first)
    if case["kind"] == "attend":
        st["out"] = torch.zeros(n, rows, heads, hd, dtype=dt, device=dev)
    if own:
        from paper_2606_03113_gb300.runtime import KV8Cache
        cache = KV8Cache(kv_heads, hd, seq, n_seq=n, device=dev)
        cache.k.copy_(k)
        cache.v.copy_(v)
        cache.k_scale.copy_(ks)
        cache.v_scale.copy_(vs)
        st["cache"] = cache
    else:
        st.update(k=k, v=v, k_scale=ks, v_scale=vs)
    return st


# ------------------------------------------------------------------ plain forms

def _append_plain(codes, scale, x, pos, rows):
    """Writes the first rows[b] of x[b] (n, M, heads, hd) at positions pos[b].. of the cache."""
    n, M, heads, hd = x.shape
    nb = (M + BLOCK - 2) // BLOCK + 1  # blocks that M rows can touch
    dev = x.device
    pos, rows = pos.long(), rows.long()
    blk = torch.minimum(pos[:, None] // BLOCK + torch.arange(nb, device=dev),
                        torch.full((1, 1), scale.shape[2] - 1, device=dev))
    p = blk[:, :, None] * BLOCK + torch.arange(BLOCK, device=dev)      # (n, nb, BLOCK)
    r = p - pos[:, None, None]
    is_new = (r >= 0) & (r < rows[:, None, None])
    # a block past the cache's last is the last one again: it has nothing new then
    again = torch.cat([torch.zeros(n, 1, dtype=torch.bool, device=dev), blk[:, 1:] == blk[:, :-1]], 1)
    is_new &= ~again[:, :, None]
    b = torch.arange(n, device=dev)
    h = torch.arange(heads, device=dev)
    at = (b[:, None, None], h[None, None, :], blk[:, :, None])         # (n, nb, heads)
    fresh = x[b[:, None, None], r.clamp(0, M - 1)].float()             # (n, nb, BLOCK, heads, hd)
    fresh = fresh.permute(0, 1, 3, 2, 4)                               # (n, nb, heads, BLOCK, hd)
    isn = is_new[:, :, None, :, None]
    old_codes = codes.view(n, heads, -1, BLOCK, hd)[at]                # (n, nb, heads, BLOCK, hd)
    old_scale = scale[at]
    amax = torch.where(isn, fresh, 0.0).abs().amax((-1, -2))
    has_old = (r[:, :, 0] < 0)[:, :, None]
    s = _scale_of(amax)
    s = torch.where(has_old, torch.maximum(s, old_scale), s)
    kept = old_codes.float() * (old_scale / s)[..., None, None]
    new = _codes_of(torch.where(isn, fresh / s[..., None, None], kept),
                    torch.ones((), device=dev))
    write = (isn | ((r < 0)[:, :, None, :, None])) & is_new.any(-1)[:, :, None, None, None]
    new = torch.where(write, new.float(), old_codes.float()).to(codes.dtype)
    s = torch.where(is_new.any(-1)[:, :, None], s, old_scale)
    codes.view(torch.uint8).view(n, heads, -1, BLOCK, hd)[at] = new.view(torch.uint8)
    scale[at] = s


def _visible(pos, rows, first, M, S, window):
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
    kvh = st["k"].shape[1]
    S = min(st["k"].shape[2], case["pos"] + M)
    def values(codes, scale):
        nb = (S + BLOCK - 1) // BLOCK
        x = codes[:, :, :nb * BLOCK].float() * scale[:, :, :nb].repeat_interleave(BLOCK, -1)[..., None]
        return x[:, :, :S]
    qf = q.float().view(n, M, kvh, heads // kvh, hd).permute(0, 2, 3, 1, 4)  # (n, kvh, G, M, hd)
    s = torch.matmul(qf.reshape(n, kvh, -1, hd), values(st["k"], st["k_scale"]).transpose(-1, -2))
    s = s.view(n, kvh, heads // kvh, M, S) * (1.0 / math.sqrt(hd))
    see = _visible(st["pos"], st["rows"], st["first"], M, S, case["window"])[:, None, None]
    s = torch.where(see, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.where(see, torch.exp(s - torch.where(m == -math.inf, 0.0, m)), 0.0)
    o = torch.matmul(e.view(n, kvh, -1, S), values(st["v"], st["v_scale"]))
    o = o.view(n, kvh, heads // kvh, M, hd)
    o = torch.where(see.any(-1, keepdim=True), o / e.sum(-1, keepdim=True), 0.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(n, M, heads, hd).to(q.dtype)
    live = torch.arange(M, device=q.device) < st["rows"][:, None]
    return torch.where(live[:, :, None, None], o, st["out"])


def _logprobs_plain(st):
    case = st["case"]
    raw = st["logits"].float()
    z = raw / case["temperature"]
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(-1, keepdim=True)
    lse = m + torch.log(total)
    p = e / total
    entropy = -torch.where(e > 0, p * (z - lse), 0.0).sum(-1)
    got = dict(logprob=z.gather(1, st["tokens"].long()) - lse, lse=lse[:, 0], entropy=entropy)
    if case["top"]:
        top = torch.sort(raw, dim=-1, descending=True, stable=True).indices[:, :case["top"]]
        got.update(top_id=top.int(), top_logprob=z.gather(1, top) - lse)
    return got


def run(st):
    case = st["case"]
    if case["kind"] == "append":
        if own:
            c = st["cache"]
            c.append(st["new_k"], st["new_v"], st["pos"], rows=st["rows"])
            return dict(k=c.k, v=c.v, k_scale=c.k_scale, v_scale=c.v_scale)
        _append_plain(st["k"], st["k_scale"], st["new_k"], st["pos"], st["rows"])
        _append_plain(st["v"], st["v_scale"], st["new_v"], st["pos"], st["rows"])
        return dict(k=st["k"], v=st["v"], k_scale=st["k_scale"], v_scale=st["v_scale"])
    if case["kind"] == "attend":
        if own:
            return st["cache"].attention(st["q"], st["pos"], rows=st["rows"], first=st["first"],
                                         window=case["window"], out=st["out"])
        return _attend_plain(st)
    if own:
        from paper_2606_03113_gb300.runtime import token_logprobs
        r = token_logprobs(st["logits"], st["tokens"], top_n=case["top"],
                           temperature=case["temperature"])
        got = dict(logprob=r.logprob, lse=r.lse, entropy=r.entropy)
        if case["top"]:
            got.update(top_id=r.top_id, top_logprob=r.top_logprob)
        return got
    return _logprobs_plain(st)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    elt = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "logprobs":
        n, v = case["rows"], case["vocab"]
        out = n * (4 * case["tokens"] * 2 + 8 + 8 * case["top"])
        # per logit: scale, subtract, exponential, two sums
        return dict(bytes=n * v * elt + out, flops=6 * n * v)
    heads, kvh, hd, _, _ = SHAPES[case["shape"]]
    n, M = case["seqs"], case["rows"]
    # ragged cases: the middle of the ranges that _places draws from
    pos = case["pos"] * (9 / 16 if case["ragged"] else 1)
    rows = (M + 1) / 2 if case["ragged"] else M
    first = pos / 6 if case["ragged"] else 0
    if case["kind"] == "append":
        vals = 2 * n * rows * kvh * hd
        blocks = 2 * n * kvh * (rows / BLOCK + 1)
        return dict(bytes=vals * (elt + 1) + blocks * 4 + 8 * n, flops=3 * vals)
    w = case["window"] or 1 << 40
    keys = min(pos + rows - first, w + rows - 1)   # that some row sees
    pairs = rows * min(pos + (rows + 1) / 2 - first, w)
    kv = n * keys * kvh * (2 * hd + 8 / BLOCK)
    return dict(bytes=kv + 2 * n * rows * heads * hd * elt, flops=4 * hd * heads * n * pairs)


# ------------------------------------------------------------------ 64 bits, from the definitions

def _plain_state(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def exact(case, seed):
    st = _plain_state(case, seed)
    if case["kind"] == "logprobs":
        cols = dict(logprob=[], lse=[], entropy=[], top_logprob=[])
        for r0 in range(0, case["rows"], 64):
            z = st["logits"][r0:r0 + 64].double() / case["temperature"]
            lse = torch.logsumexp(z, -1)
            lp = z - lse[:, None]
            cols["lse"].append(lse)
            cols["entropy"].append(-(torch.special.xlogy(lp.exp(), lp.exp())).sum(-1))
            cols["logprob"].append(torch.gather(lp, 1, st["tokens"][r0:r0 + 64].long()))
            if case["top"]:
                cols["top_logprob"].append(torch.topk(lp, case["top"], -1).values)
        got = {k: torch.cat(v) for k, v in cols.items() if v}
        if case["top"]:
            got["top_id"] = None
        return got
    heads, kvh, hd, _, _ = SHAPES[case["shape"]]
    n, M = case["seqs"], case["rows"]
    pos, rows, first = (st[x].tolist() for x in ("pos", "rows", "first"))
    if case["kind"] == "append":
        # the scales have one value each, the codes are rounded by choice: block by block from the
        # rows' magnitudes
        got = {}
        for name in ("k", "v"):
            scale = st[name + "_scale"].double()
            x = st["new_" + name].double().abs().amax(-1)  # (n, M, heads)
            for b in range(n):
                for j in range(pos[b] // BLOCK, (pos[b] + rows[b] - 1) // BLOCK + 1):
                    lo, hi = max(pos[b], j * BLOCK), min(pos[b] + rows[b], (j + 1) * BLOCK)
                    top = x[b, lo - pos[b]:hi - pos[b]].amax(0)
                    # (a magnitude of 448 2^k itself takes 2^k: log2 may be a bit above k there)
                    s = torch.exp2(torch.ceil(torch.log2(top / 448.0) - 1e-12))
                    scale[b, :, j] = torch.maximum(s, scale[b, :, j]) if lo > j * BLOCK else s
            got[name + "_scale"] = scale
        return dict(k=None, v=None, **got)
    out = torch.zeros(n, M, heads, hd, dtype=torch.float64, device=st["q"].device)
    for b in range(n):
        hi = pos[b] + rows[b]
        lo = max(0, first[b], pos[b] - case["window"] + 1 if case["window"] else 0)
        j = torch.arange(lo, hi, device=out.device)
        p = pos[b] + torch.arange(rows[b], device=out.device)
        bad = (j[None] > p[:, None]) | (j[None] < first[b])
        if case["window"]:
            bad |= j[None] <= p[:, None] - case["window"]
        for g in range(kvh):
            kk, vv = ((st[x][b, g, lo:hi].double().t() * st[x + "_scale"][b, g].double()[j // BLOCK]).t()
                      for x in ("k", "v"))
            for h in range(g * heads // kvh, (g + 1) * heads // kvh):
                s = st["q"][b, :rows[b], h].double() @ kk.t() / hd ** 0.5
                s[bad] = -math.inf
                out[b, :rows[b], h] = torch.softmax(s, -1).nan_to_num(0.0) @ vv
    return out
