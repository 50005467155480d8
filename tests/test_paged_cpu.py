"""The paged cache's host side: struct layout, refusals of the C entry points and of the Python ones
(nothing here needs a GPU or reaches one), and the reference that the GPU tests compare with."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import paged_ref as R
from paper_2606_03113_gb300 import ssd as S
from paper_2606_03113_gb300.runtime import PagedKVCache

BUF = 0x7f0000000000  # an address that is only looked at


def cache(**kw):
    base = dict(n_layers=2, n_seq=2, n_kv_heads=4, head_dim=128, page=16, n_pages=32, max_pages=64,
                dtype=S.SSD_DTYPE_BF16, pages=BUF, table=BUF, refs=BUF)
    base.update(kw)
    return S.ssd_paged_cache(**base)


def test_cache_struct_matches_the_c_compiler(tmp_path):
    src = tmp_path / "l.c"
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "ssd_ops.h"', "int main(void) {",
             'printf("%zu %d %d\\n", sizeof(ssd_paged_cache), SSD_PAGED_ERR_PAGES, SSD_PAGED_ERR_TABLE);']
    for f, _ in S.ssd_paged_cache._fields_:
        lines.append(f'printf("%zu\\n", offsetof(ssd_paged_cache, {f}));')
    src.write_text("\n".join(lines + ["return 0; }"]))
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.check_call(["gcc", "-std=c11", "-I", inc, str(src), "-o", str(tmp_path / "l")])
    got = subprocess.check_output([str(tmp_path / "l")], text=True).split()
    assert [int(x) for x in got[:3]] == [C.sizeof(S.ssd_paged_cache), S.PAGED_ERR_PAGES, S.PAGED_ERR_TABLE]
    assert [int(x) for x in got[3:]] == [getattr(S.ssd_paged_cache, f).offset
                                         for f, _ in S.ssd_paged_cache._fields_]


INVALID, UNSUPPORTED, CAPACITY = S.SSD_ERR_INVALID_ARG, S.SSD_ERR_UNSUPPORTED, S.SSD_ERR_CAPACITY
BAD_CACHES = [(dict(head_dim=96), UNSUPPORTED), (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED),
              (dict(page=512), UNSUPPORTED), (dict(page=0), UNSUPPORTED), (dict(page=-16), UNSUPPORTED),
              (dict(n_seq=0), INVALID), (dict(n_seq=4097), INVALID), (dict(n_layers=0), INVALID),
              (dict(n_layers=1025), INVALID), (dict(n_kv_heads=0), INVALID),
              (dict(n_kv_heads=1025), INVALID), (dict(dtype=2), INVALID), (dict(n_pages=0), INVALID),
              (dict(n_pages=(1 << 24) + 1), INVALID), (dict(max_pages=0), INVALID),
              (dict(max_pages=(1 << 26) + 1), INVALID),
              (dict(n_seq=4096, max_pages=1 << 20), INVALID),
              (dict(pages=None), INVALID), (dict(pages=BUF + 8), INVALID), (dict(table=None), INVALID),
              (dict(table=BUF + 2), INVALID), (dict(refs=None), INVALID), (dict(refs=BUF + 4), INVALID)]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_bad_caches_are_refused(bad, status):
    c = cache(**bad)
    for call in (lambda: S.ssd_paged_reserve(c, BUF, 0, 1, BUF, 1 << 30),
                 lambda: S.ssd_paged_fork(c, BUF), lambda: S.ssd_paged_compact(c, BUF, BUF, 1 << 30),
                 lambda: S.ssd_paged_append(c, 0, BUF, BUF, 512, 1, BUF),
                 lambda: S.ssd_paged_attention(c, 0, BUF, 4, 512, 1, BUF, 0, 0, 0, 0, BUF, 512, BUF,
                                               1 << 30)):
        with pytest.raises(S.SsdError) as e:
            call()
        assert e.value.status == status and "cache" in str(e.value)
    assert S.ssd_paged_workspace_bytes(c) == 0
    assert S.ssd_paged_attention_bytes(c, 4, 1) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(pos=0), INVALID), (dict(M=0), INVALID), (dict(M=-1), INVALID), (dict(M=1025), CAPACITY),
    (dict(work=0), INVALID), (dict(work=BUF + 128), INVALID), (dict(nbytes=100), CAPACITY)])
def test_reserve_refuses(kw, status):
    a = dict(pos=BUF, M=1, work=BUF, nbytes=1 << 20)
    a.update(kw)
    with pytest.raises(S.SsdError) as e:
        S.ssd_paged_reserve(cache(), a["pos"], 0, a["M"], a["work"], a["nbytes"])
    assert e.value.status == status


def test_fork_and_compact_refuse():
    with pytest.raises(S.SsdError) as e:
        S.ssd_paged_fork(cache(), 0, 0)
    assert e.value.status == INVALID
    for work, nbytes, status in ((0, 1 << 20, INVALID), (BUF + 16, 1 << 20, INVALID), (BUF, 64, CAPACITY)):
        with pytest.raises(S.SsdError) as e:
            S.ssd_paged_compact(cache(), BUF, work, nbytes)
        assert e.value.status == status
    assert S.lib().ssd_paged_fork(None, BUF, None, None, None) == INVALID


@pytest.mark.parametrize("kw,status", [
    (dict(layer=-1), INVALID), (dict(layer=2), INVALID), (dict(k=0), INVALID), (dict(v=BUF + 4), INVALID),
    (dict(stride=511), INVALID), (dict(stride=516), INVALID), (dict(stride=-512), INVALID),
    (dict(M=0), INVALID), (dict(M=1025), CAPACITY), (dict(pos=0), INVALID)])
def test_append_refuses(kw, status):
    a = dict(layer=0, k=BUF, v=BUF, stride=512, M=1, pos=BUF)
    a.update(kw)
    with pytest.raises(S.SsdError) as e:
        S.ssd_paged_append(cache(), a["layer"], a["k"], a["v"], a["stride"], a["M"], a["pos"])
    assert e.value.status == status


@pytest.mark.parametrize("kw,status", [
    (dict(layer=-1), INVALID), (dict(layer=2), INVALID), (dict(q=0), INVALID), (dict(q=BUF + 4), INVALID),
    (dict(heads=3), INVALID), (dict(heads=6), INVALID), (dict(heads=0), INVALID),
    (dict(q_stride=511), INVALID), (dict(q_stride=516), INVALID), (dict(out=0), INVALID),
    (dict(out=BUF + 8), INVALID), (dict(out_stride=100), INVALID),
    (dict(out=BUF, q=BUF, out_stride=1024), INVALID), (dict(pos=0), INVALID), (dict(window=-1), INVALID),
    (dict(M=0), INVALID), (dict(M=1025), CAPACITY), (dict(longest=-1), INVALID),
    (dict(longest=1025), CAPACITY)])
def test_attention_refuses(kw, status):
    a = dict(layer=0, q=BUF, heads=4, q_stride=512, M=1, pos=BUF, window=0, longest=0, out=BUF + 4096,
             out_stride=512, work=BUF, nbytes=1 << 30)
    a.update(kw)
    with pytest.raises(S.SsdError) as e:
        S.ssd_paged_attention(cache(), a["layer"], a["q"], a["heads"], a["q_stride"], a["M"], a["pos"],
                              0, 0, a["window"], a["longest"], a["out"], a["out_stride"], a["work"],
                              a["nbytes"])
    assert e.value.status == status


def test_attention_counts_rows_in_31_bits():
    """Rows of a KV head are numbered in 31 bits, by tiles of up to 256: more are refused, also where `longest`
    keeps the work itself small."""
    c = cache(n_seq=1, n_kv_heads=1, head_dim=64, max_pages=1 << 20)
    assert S.ssd_paged_attention_bytes(c, 65536, (1 << 15) - 1, 0, 1) > 0
    for M in (1 << 15, 40000, 1 << 24):
        assert S.ssd_paged_attention_bytes(c, 65536, M, 0, 1) == 0
        with pytest.raises(S.SsdError) as e:
            S.ssd_paged_attention(c, 0, BUF, 65536, 65536 * 64, M, BUF, 0, 0, 0, 1, BUF, 65536 * 64, BUF,
                                  1 << 40)
        assert e.value.status == CAPACITY and "rows" in str(e.value)


# ------------------------------------------------------------- the Python entry points

def py_cache(**kw):
    a = dict(n_layers=2, n_kv_heads=4, head_dim=64, n_pages=8, page=16, n_seq=3, max_seq=64,
             dtype=torch.float32, device="cpu")
    a.update(kw)
    return PagedKVCache(**a)


@pytest.mark.parametrize("kw", [
    dict(head_dim=96), dict(page=8), dict(page=24), dict(dtype=torch.float16), dict(n_layers=0),
    dict(n_kv_heads=0), dict(n_pages=0), dict(n_seq=0), dict(n_seq=4097), dict(max_seq=0),
    dict(max_seq=(1 << 30) + 1)])
def test_python_cache_refuses(kw):
    with pytest.raises(ValueError):
        py_cache(**kw)


def test_python_cache_layout():
    c = py_cache(max_seq=50)
    assert c.max_seq == 64 and c.max_pages == 4 and c.pages.shape == (8, 2, 2, 4, 16, 64)
    assert (c.table == -1).all() and c.table.shape == (3, 4) and not c.refs.any()
    with pytest.raises(AttributeError):
        c.table = torch.zeros(3, 4)


def test_python_calls_refuse():
    c = py_cache()
    pos = torch.zeros(3, dtype=torch.int32)
    k = torch.zeros(3, 2, 4, 64)
    q = torch.zeros(3, 2, 8, 64)
    bad = [
        lambda: c.reserve(None), lambda: c.reserve(pos.long()), lambda: c.reserve(pos[:2]),
        lambda: c.reserve(pos, 0), lambda: c.reserve(pos, 65), lambda: c.reserve(pos, None),
        lambda: c.reserve(pos, torch.zeros(2, dtype=torch.int32)),
        lambda: c.fork(None), lambda: c.fork(pos.float()), lambda: c.fork(pos, pos[:1]),
        lambda: c.truncate(None), lambda: c.truncate(torch.zeros(6, dtype=torch.int32)[::2]),
        lambda: c.append(2, k, k, pos), lambda: c.append(-1, k, k, pos),
        lambda: c.append(0, k.bfloat16(), k.bfloat16(), pos), lambda: c.append(0, k, k[:, :1], pos),
        lambda: c.append(0, k, k, None), lambda: c.append(0, k[:2], k[:2], pos),
        lambda: c.append(0, k.transpose(1, 2).contiguous().transpose(1, 2), k, pos),
        lambda: c.append(0, k.clone().requires_grad_(), k, pos),
        lambda: c.attention(2, q, pos), lambda: c.attention(0, q[:, :, :6], pos),
        lambda: c.attention(0, q.bfloat16(), pos), lambda: c.attention(0, q, None),
        lambda: c.attention(0, q, pos, window=-1), lambda: c.attention(0, q, pos, longest=65),
        lambda: c.attention(0, q, pos, longest=-1), lambda: c.attention(0, q[0], pos),
        lambda: c.attention(0, q, pos, out=q[:, :1]), lambda: c.attention(0, q, pos, out=q.bfloat16()),
        lambda: c.attention(0, q, pos, first=pos.long()),
        # everything is in order, but there is no GPU here
        lambda: c.reserve(pos), lambda: c.fork(pos), lambda: c.compact(), lambda: c.append(0, k, k, pos),
        lambda: c.attention(0, q, pos)]
    for call in bad:
        with pytest.raises(ValueError):
            call()


def test_tangents_are_refused():
    """No entry point has a forward-mode derivative: a dual tensor's tangent would be lost."""
    from torch.autograd import forward_ad
    from paper_2606_03113_gb300.runtime import KV8Cache, token_logprobs
    c, c8 = py_cache(), KV8Cache(4, 64, 64, n_seq=3, device="cpu")
    pos = torch.zeros(3, dtype=torch.int32)
    k, q, z = torch.zeros(3, 2, 4, 64), torch.zeros(3, 2, 8, 64), torch.zeros(2, 9)
    with forward_ad.dual_level():
        dk, dq, dz = (forward_ad.make_dual(x, torch.ones_like(x)) for x in (k, q, z))
        for call in (lambda: c.append(0, dk, k, pos), lambda: c.append(0, k, dk, pos),
                     lambda: c.attention(0, dq, pos), lambda: c.attention(0, q, pos, out=dq),
                     lambda: c8.append(dk, k, pos), lambda: c8.attention(dq, pos),
                     lambda: token_logprobs(dz)):
            with pytest.raises(ValueError, match="tangent"):
                call()
        with pytest.raises(ValueError, match="CUDA"):  # others are as ever
            c.append(0, k, k, pos)


def test_every_error_bit_of_the_kernels_is_named():
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    csrc = os.path.join(root, "paper_2606_03113_gb300", "csrc")
    header = open(os.path.join(root, "include", "ssd_ops.h")).read()
    named = {k: int(v) for k, v in re.findall(r"#define SSD_(?:DEV|PAGED)_ERR_(\w+) (\d+)", header)}
    enum = dict(re.findall(r"kErr(\w+) = (\d+)", open(os.path.join(csrc, "common.cuh")).read()))
    used = set()
    for f in ("paged_pages.cu", "paged_attention.cu", "kv8_plan.cuh"):
        used |= set(re.findall(r"kErr([A-Z]\w+)", open(os.path.join(csrc, f)).read()))
    assert used >= {"Capacity", "Control", "Pages", "Table"}
    names = S.DEV_ERR_NAMES | S.PAGED_ERR_NAMES
    for u in used:
        assert named[u.upper()] == int(enum[u]) and int(enum[u]) in names
    assert "free pages" in S.dev_err_text(34) and "positions" in S.dev_err_text(34)


# ------------------------------------------------------------- the reference itself

def test_reference_keeps_what_sequences_hold():
    """Random forks, truncations, ends, rows and compactions: a sequence's rows are those of a plain
    list of its own, whatever pages hold them."""
    rng = np.random.default_rng(0)
    n, W, P = 5, 6, 16
    c = R.Cache(1, 1, 1, 40, P, n, W)
    told = [[] for _ in range(n)]
    for step in range(300):
        kind = rng.integers(4)
        if kind == 0:
            parent = [int(x) for x in rng.integers(-1, n, n)]
            c.fork(parent)
            told = [list(told[p]) if p >= 0 else [] for p in parent]
        elif kind == 1:
            told = [t[:int(rng.integers(0, len(t) + 1))] if rng.random() < 0.3 else t for t in told]
            c.fork(None, [len(t) for t in told])
        elif kind == 2:
            low = c.compact()
            assert all(c.refs[:low]) and not any(c.refs[low:])
        pos = [len(t) for t in told]
        rows = [int(min(rng.integers(0, 20), W * P - x)) for x in pos]
        err = c.err
        c.reserve(pos, rows)
        assert c.err == err
        x = rng.normal(size=(n, 20, 1, 1)).astype(np.float32)
        c.append(0, x, -x, pos, rows)
        told = [t + [float(v) for v in x[b, :rows[b], 0, 0]] for b, t in enumerate(told)]
        for b, t in enumerate(told):
            assert np.array_equal(c.rows(0, 0, b, 0, len(t))[0, :, 0], t) if t else True
        assert sum(c.refs) == sum(e >= 0 for line in c.table for e in line)
    assert c.err == 0


def test_reference_last_sharer_keeps_the_page():
    c = R.Cache(1, 1, 1, 8, 16, 3, 2)
    c.reserve([0, 0, 0], [5, 0, 0])
    c.fork([0, 0, 0])
    assert c.table == [[0, -1]] * 3 and c.refs[0] == 3
    c.reserve([5, 5, 5], [1, 1, 1])
    assert c.table == [[1, -1], [2, -1], [0, -1]] and c.refs[:3] == [1, 1, 1]
    c.fork([0, 0, 0])
    c.reserve([5, 5, 5], [1, 0, 1])       # one who shares does not ask: both others move
    assert c.table == [[0, -1], [1, -1], [2, -1]]
