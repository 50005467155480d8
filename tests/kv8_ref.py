"""64-bit references of the 8-bit KV cache, its attention and the token log-probabilities, in
numpy, from their definitions: loops over sequences, heads and blocks, no code of the package."""
import math

import numpy as np

BLOCK = 64


def e4m3_round(x):
    """Nearest e4m3 number (ties to even, cut at 448, NaN kept) of float64 values."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.floor(np.log2(np.where(a > 0, a, 1.0)))
    # log2 can be off at powers of two
    e = np.where(2.0 ** e > np.where(a > 0, a, 1.0), e - 1, e)
    e = np.where(2.0 ** (e + 1) <= np.where(a > 0, a, 1.0), e + 1, e)
    step = 2.0 ** (np.maximum(e, -6) - 3)
    y = np.minimum(np.rint(a / step) * step, 448.0)
    return np.where(np.isnan(x), np.nan, np.copysign(y, x))


def scale_of(amax):
    """Smallest power of two in 2^-120 .. 2^111 with amax <= 448 times it."""
    if not amax > 0:
        return 2.0 ** -120
    e = math.ceil(math.log2(amax / 448.0))
    while amax <= 448.0 * 2.0 ** (e - 1):
        e -= 1
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** min(max(e, -120), 111)


def append(codes, scale, x, pos, rows):
    """codes [n][heads][seq][hd] (values of the codes), scale [n][heads][seq/64], in place."""
    n, M, heads, hd = x.shape
    for b in range(n):
        p0, m = int(pos[b]), int(rows[b])
        if p0 < 0 or m < 0 or m > M or p0 + m > codes.shape[2]:
            continue
        for h in range(heads):
            for j in range(p0 // BLOCK, (p0 + m - 1) // BLOCK + 1 if m else 0):
                lo, hi = max(p0, j * BLOCK), min(p0 + m, (j + 1) * BLOCK)
                new = x[b, lo - p0:hi - p0, h].astype(np.float64)
                new = np.where(np.isfinite(new), new, np.nan)
                amax = np.nanmax(np.abs(new), initial=0.0)
                s = scale_of(amax)
                if lo > j * BLOCK:
                    old = float(scale[b, h, j])
                    s = max(s, old)
                    if s > old:
                        c = codes[b, h, j * BLOCK:lo]
                        codes[b, h, j * BLOCK:lo] = e4m3_round(c * (old / s))
                codes[b, h, lo:hi] = e4m3_round(new / s)
                scale[b, h, j] = s


def visible(p, first, window):
    """(lo, hi): the keys that a row at position p sees; lo > hi: none."""
    lo = max(int(first), 0)
    if window > 0:
        lo = max(lo, p - window + 1)
    return lo, p


def attend(q, k, v, pos, rows, first, window, out):
    """q [n][M][heads][hd], k, v [n][kv][seq][hd] values, float64; out in place.  Returns the
    sums sum p |v| / sum p beside each output and the rows' largest sum |q k| / sqrt(hd)."""
    n, M, heads, hd = q.shape
    kv = k.shape[1]
    mass, size = np.zeros(out.shape), np.zeros(out.shape[:3])
    for b in range(n):
        for m in range(int(rows[b])):
            lo, hi = visible(int(pos[b]) + m, first[b], window)
            for h in range(heads):
                g = h // (heads // kv)
                if lo > hi:
                    out[b, m, h] = 0.0
                    continue
                kk, vv, qq = k[b, g, lo:hi + 1], v[b, g, lo:hi + 1], q[b, m, h]
                with np.errstate(invalid="ignore"):
                    s = kk @ qq / math.sqrt(hd)
                    p = np.exp(s - np.max(s))
                    p /= p.sum()
                    out[b, m, h] = p @ vv
                    mass[b, m, h] = p @ np.abs(vv)
                    size[b, m, h] = np.max(np.abs(kk) @ np.abs(qq)) / math.sqrt(hd)
    return mass, size


def attend_bound(ref, mass, size, hd, keys, bf16):
    """How far a right kernel's outputs may be from ref.  u = 2^-24.
    - scores: hd products and sums in fp32 (a tensor core cuts: 2u each), then two scalings and a
      subtraction: off by d <= (2 hd + 8) u size, and e^d moves a probability by that much;
    - the exponential: 4u, the probability's own rounding: f16 (2^-11) or two f16 parts (2^-21);
      queries in two f16 parts: 2^-21 of size, in the scores of fp32 rows;
    - sums over the keys, cut at each 16-key step, and their joins: (keys / 8 + 64) u, numerator and
      denominator; then the output's own rounding."""
    u = 2.0 ** -24
    d = (2 * hd + 8) * u * size + (0 if bf16 else 2.0 ** -21 * size)
    rel = 2 * d + 8 * u + (2.0 ** -11 if bf16 else 2.0 ** -21) + 2 * (keys / 8 + 64) * u
    return rel[..., None] * mass * 1.01 + (2.0 ** -8 if bf16 else 2 * u) * np.abs(ref) + 1e-30


def logprobs(z, tokens, t, top):
    """float64 rows z [n][V]; tokens [n][k]: (logprob, lse, entropy, ids, top_logprob, spread),
    spread = sum p |z/t - max|."""
    n, V = z.shape
    lp = np.full(tokens.shape, np.nan)
    lse, ent, spread = np.zeros(n), np.zeros(n), np.zeros(n)
    ids, tlp = np.full((n, top), -1, np.int32), np.full((n, top), -np.inf)
    for r in range(n):
        x = z[r] / t
        with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
            if np.isnan(x).any() or np.isposinf(x).any():
                lse[r] = ent[r] = np.nan
            elif not (x > -np.inf).any():
                lse[r], ent[r] = -np.inf, np.nan
            else:
                mx = x.max()
                lse[r] = mx + math.log(np.exp(x - mx).sum())
                p = np.exp(x - lse[r])
                live = p > 0
                ent[r] = -(p[live] * (x[live] - lse[r])).sum()
                spread[r] = (p[live] * np.abs(x[live] - mx)).sum()
            for j, v in enumerate(tokens[r]):
                if v == -1:
                    lp[r, j] = 0.0
                elif 0 <= v < V:
                    lp[r, j] = x[v] - lse[r]
            order = sorted((i for i in range(V) if z[r, i] > -np.inf),
                           key=lambda i: (-z[r, i], i))[:top] if V <= 4096 else [
                i for i in np.lexsort((np.arange(V), -np.where(np.isnan(z[r]), -np.inf, z[r])))[:top]
                if z[r, i] > -np.inf]
            for j, i in enumerate(order):
                ids[r, j], tlp[r, j] = i, x[i] - lse[r]
    return lp, lse, ent, ids, tlp, spread
