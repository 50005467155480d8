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


def _check(c, vals, q, pos, window=0):
    M = q.shape[1]
    got = c.attention(q, _ints([pos]), window=window)
    c.check()
    ref = np.zeros(got.shape)
    mass, size = R.attend(_values(q), vals[0], vals[1], [pos], [M], [0], window, ref)
    tol = R.attend_bound(ref, mass, size, HD, pos + M, got.dtype == _torch().bfloat16)
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
