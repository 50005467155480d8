"""Token log-probabilities on the GPU against a 64-bit reference, with a bound from the roundings of
a one-pass sum: ids exactly, values within it."""
import numpy as np
import pytest

import kv8_ref as R
from parity import has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a CUDA GPU")]

U = 2.0 ** -24


def _run(z, tokens=None, **kw):
    from paper_2606_03113_gb300.runtime import token_logprobs
    return token_logprobs(z, tokens, **kw)


def _check(z, tok, t, top, got):
    """S is a sum of terms 2^d, d = z c - m, each off by the rounding of d (u |d|, and u |z c| for
    c's own), the exponential (4 u) and the additions: a thread adds at most V / 256 + 64 terms,
    then joins of parts (64).  So ln S is off by add + arg with add = (V/256 + 136) u and arg =
    3 u spread (probability-weighted |d|); lse adds the product m ln 2 (3 u |lse| and |max|).
    The entropy ln S - T / S: T's terms are weighted by |d|, its error twice that and one more
    rounding of each |d|."""
    zz = z.float().cpu().numpy().astype(np.float64)
    n, V = zz.shape
    tk = tok.cpu().numpy().reshape(n, -1)
    lp, lse, ent, ids, tlp, spread = R.logprobs(zz, tk, t, top)
    fin = np.where(np.isfinite(zz), zz, 0.0)
    big = np.abs(fin).max(-1) / t
    add = (V / 256 + 136) * U
    tol = add + 3 * U * spread + 6 * U * (big + np.abs(np.nan_to_num(lse, neginf=0.0))) + 8 * U
    g = lambda x: x.cpu().numpy().astype(np.float64)  # noqa: E731

    def near(x, y, tol):
        with np.errstate(invalid="ignore"):
            ok = (np.abs(x - y) <= tol) | (x == y) | (np.isnan(x) & np.isnan(y))
        assert ok.all(), (np.nanmax(np.abs(x - y)), np.argwhere(~ok)[:4], x[~ok][:4], y[~ok][:4])

    near(g(got.lse), lse, tol)
    near(g(got.entropy), ent, 3 * tol * (1 + spread))
    near(g(got.logprob).reshape(n, -1), lp, tol[:, None] * 2)
    if top:
        assert np.array_equal(got.top_id.cpu().numpy(), ids)
        near(g(got.top_logprob), tlp, tol[:, None] * 2)
    else:
        assert got.top_id is None and got.top_logprob is None


SIZES = [  # rows, vocab, dtype, tokens, top, temperature, offset (elements), gap between rows
    (1, 1, "f32", 1, 1, 1.0, 0, 0), (1, 2, "bf16", 2, 2, 0.5, 1, 0), (3, 31, "f32", 1, 31, 1.0, 1, 2),
    (5, 1024, "f32", 1, 5, 1.0, 0, 0), (7, 1000, "bf16", 3, 20, 0.7, 3, 5),
    (2, 8191, "bf16", 1, 32, 1.3, 0, 1), (2, 8193, "f32", 4, 32, 2.0, 2, 1),
    (13, 32000, "f32", 1, 8, 0.6, 0, 0), (3, 32001, "bf16", 1, 20, 1.0, 5, 0),
    (1, 128256, "f32", 1, 20, 1.0, 0, 0), (2, 128256, "bf16", 1, 0, 1.0, 0, 0),
    (700, 1500, "bf16", 1, 4, 1.0, 0, 1), (640, 2000, "f32", 1, 32, 1.0, 1, 3),
]


@pytest.mark.parametrize("rows,V,dtype,ntok,top,t,off,gap", SIZES)
def test_against_64_bits(rows, V, dtype, ntok, top, t, off, gap):
    import torch
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(V)
    flat = (torch.randn(rows * (V + gap) + off, generator=g, device="cuda") * 4).to(dt)
    z = flat[off:].view(rows, V + gap)[:, :V]
    tok = torch.randint(0, V, (rows, ntok), generator=g, device="cuda").int()
    tok[0, 0] = -1
    got = _run(z, tok, top_n=top, temperature=t)
    _check(z, tok, t, top, got)
    again = _run(z, tok, top_n=top, temperature=t)
    for a, b in zip(got[:5], again[:5]):
        assert a is b is None or torch.equal(a.view(torch.int32), b.view(torch.int32))


@pytest.mark.parametrize("V", [40, 1024, 5000, 128256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_and_masks(V, dtype):
    """Equal logits, two values, few finite ones, runs in order, a period that puts all large ones
    into a few threads, masks of the type's lowest value, signed zeros."""
    import torch
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    inf = float("inf")
    ar = torch.arange(V, device="cuda")
    low = torch.finfo(dt).min
    rows = [torch.zeros(V, device="cuda"), torch.full((V,), -3.5, device="cuda"),
            (ar % 7 == 3).float(), torch.where(ar % (V // 11 + 1) == 1, ar * 1e-3, -inf),
            ar * 1e-3, -ar * 1e-3, torch.where(ar // 8 % 256 < 3, 5.0 + (ar // 8192) * 0.5, 0.0),
            torch.where(ar % 3 == 0, ar.float() % 50, low), torch.where(ar == V - 1, 2.0, -inf),
            torch.where(ar % 2 == 0, 0.0, -0.0), torch.full((V,), low, device="cuda"),
            torch.where(ar // 8 % 256 == 200, 3.0 + (ar % 8) * 0.25, -1.0)]
    z = torch.stack([r.float() for r in rows]).to(dt)
    tok = torch.full((len(rows), 2), V - 1, dtype=torch.int32, device="cuda")
    tok[:, 1] = 3
    top = min(32, V)
    if V > 20000:  # few rows are cut into chunks, many are not: both ways
        many = z.repeat(60, 1)
        got = _run(many, tok.repeat(60, 1), top_n=top)
        n = len(rows)
        for i in (0, 59):
            part = type(got)(*[x[i * n:(i + 1) * n] if x is not None else None for x in got])
            _check(z, tok, 1.0, top, part)
    _check(z, tok, 1.0, top, _run(z, tok, top_n=top))


def test_rows_without_a_distribution():
    import torch
    inf, nan = float("inf"), float("nan")
    for V in (300, 40000):
        z = torch.randn(6, V, device="cuda")
        z[0] = -inf
        z[1, V // 2] = nan
        z[2, 3] = inf
        z[3, 1:] = -inf
        z[4, V - 1] = nan
        z[4, :V - 1] = -inf
        tok = torch.tensor([0, 1, 3, 0, V - 1, 2], dtype=torch.int32, device="cuda")
        got = _run(z, tok, top_n=4)
        _check(z, tok, 1.0, 4, got)
        assert float(got.lse[0]) == -inf and bool(got.entropy[0].isnan())
        assert got.top_id[0].tolist() == [-1] * 4
        assert float(got.entropy[3]) == 0.0 and float(got.logprob[3]) == 0.0


def test_bad_tokens_set_the_bit():
    import torch
    from paper_2606_03113_gb300 import ssd as S
    z = torch.randn(4, 50, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = _run(z, torch.tensor([-1, 0, 49, -1], dtype=torch.int32, device="cuda"), err=err)
    assert int(err) == 0 and float(got.logprob[0]) == 0.0
    got = _run(z, torch.tensor([50, -2, 2 ** 31 - 1, 7], dtype=torch.int32, device="cuda"), err=err)
    assert int(err) == S.DEV_ERR_TOKEN
    assert got.logprob.isnan().tolist() == [True, True, True, False]
    got = _run(z, top_n=3)
    assert got.logprob is None and got.top_id.shape == (4, 3)
    assert _run(z, torch.zeros(4, 0, dtype=torch.int32, device="cuda")).logprob.shape == (4, 0)


def test_exit_statistics_agree():
    """The same logits through the exit head's statistics and through this operator."""
    import torch
    import synth
    from paper_2606_03113_gb300.runtime import DeviceModel, Engine
    from synth.workloads import TINY
    eng = Engine(DeviceModel(TINY.shape), TINY.max_seq)
    eng.set_ar()
    ids = synth.prompt_ids(TINY.prompt_len, TINY.shape.vocab)
    eng.prefill(ids[:-4])
    z, st = eng.forward_exit(ids[-4:], TINY.prompt_len - 4, 4, topk=5)
    got = _run(torch.from_numpy(z).cuda(), top_n=8)
    for i, s in enumerate(st):
        assert got.top_id[i].tolist() == s["top_idx"]
        assert abs(float(got.lse[i]) - s["lse"]) <= 1e-5 * max(1, abs(s["lse"]))
        assert abs(float(got.entropy[i]) - s["entropy"]) <= 2e-5 * s["entropy"]
        assert abs(-float(got.top_logprob[i, :5].mean()) - s["conf_k"]) <= 2e-5 * s["conf_k"]
    eng.close()


def test_captured_and_on_another_stream():
    import torch
    z = torch.randn(3, 32000, device="cuda")
    tok = torch.randint(0, 32000, (3, 1), device="cuda").int()
    want = _run(z, tok, top_n=6)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _run(z, tok, top_n=6)
    z.copy_(z.flip(0))
    tok.copy_(tok.flip(0))
    graph.replay()
    for a, b in zip(want[:5], got[:5]):
        assert torch.equal(a.flip(0), b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    there = _run(z, tok, top_n=6, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(there[:5], got[:5]))


def test_rows_past_32_bits():
    """The last rows of logits that span more than 2^32 bytes."""
    import torch
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB")
    n, V = 17500, 128256
    z = torch.zeros(n, V, dtype=torch.bfloat16, device="cuda")
    last = torch.randn(3, V, device="cuda").bfloat16()
    z[-3:] = last
    tok = torch.full((n, 1), 5, dtype=torch.int32, device="cuda")
    got = _run(z, tok, top_n=2)
    part = type(got)(*[x[-3:] if x is not None else None for x in got])
    _check(last, tok[-3:], 1.0, 2, part)
    assert abs(float(got.lse[0]) - np.log(V)) < 1e-5 and got.top_id[0].tolist() == [0, 1]


def test_many_rows_of_fp32_and_parts_of_steps():
    """A block a row with a step in advance: rows that end within a step, at odd places."""
    import torch
    for V in (1023, 4096, 4100, 9001, 12288):
        g = torch.Generator(device="cuda").manual_seed(V)
        flat = torch.randn(700 * (V + 3), generator=g, device="cuda") * 3
        z = flat.view(700, V + 3)[:, 1:V + 1]
        tok = torch.randint(0, V, (700, 1), generator=g, device="cuda").int()
        _check(z[:50], tok[:50], 0.8, 9, type(_run(z[:1]))(*[
            x[:50] if x is not None else None for x in _run(z, tok, top_n=9, temperature=0.8)]))
