"""The 8-bit cache's and the token scores' host side: struct layout, refusals of the C entry
points and of the Python ones (nothing here needs a GPU or reaches one), and the references that
the GPU tests compare with, pinned against torch's own e4m3 type."""
import ctypes as C
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import kv8_ref as R
from paper_2606_03113_gb300 import ssd as S
from paper_2606_03113_gb300.runtime import KV8Cache, token_logprobs

BUF = 0x7f0000000000  # an address that is only looked at


def cache(**kw):
    base = dict(n_seq=2, n_kv_heads=4, head_dim=128, max_seq=1024, k=BUF, v=BUF, k_scale=BUF,
                v_scale=BUF)
    base.update(kw)
    return S.ssd_kv8_cache(**base)


def test_cache_struct_matches_the_c_compiler(tmp_path):
    src = tmp_path / "l.c"
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "ssd_ops.h"', "int main(void) {",
             'printf("%zu %d %d %d\\n", sizeof(ssd_kv8_cache), SSD_KV8_BLOCK, SSD_KV8_MAX_SEQS, SSD_MAX_TOP);']
    for f, _ in S.ssd_kv8_cache._fields_:
        lines.append(f'printf("%zu\\n", offsetof(ssd_kv8_cache, {f}));')
    src.write_text("\n".join(lines + ["return 0; }"]))
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.check_call(["gcc", "-std=c11", "-I", inc, str(src), "-o", str(tmp_path / "l")])
    got = subprocess.check_output([str(tmp_path / "l")], text=True).split()
    assert [int(x) for x in got[:4]] == [C.sizeof(S.ssd_kv8_cache), S.KV8_BLOCK, S.KV8_MAX_SEQS,
                                         S.MAX_TOP]
    assert [int(x) for x in got[4:]] == [getattr(S.ssd_kv8_cache, f).offset
                                         for f, _ in S.ssd_kv8_cache._fields_]


BAD_CACHES = [(dict(head_dim=96), S.SSD_ERR_UNSUPPORTED), (dict(head_dim=0), S.SSD_ERR_UNSUPPORTED),
              (dict(max_seq=100), S.SSD_ERR_INVALID_ARG), (dict(max_seq=0), S.SSD_ERR_INVALID_ARG),
              (dict(max_seq=-64), S.SSD_ERR_INVALID_ARG), (dict(n_seq=0), S.SSD_ERR_INVALID_ARG),
              (dict(n_seq=4097), S.SSD_ERR_INVALID_ARG),
              (dict(n_kv_heads=0), S.SSD_ERR_INVALID_ARG), (dict(k=None), S.SSD_ERR_INVALID_ARG),
              (dict(v=BUF + 8), S.SSD_ERR_INVALID_ARG), (dict(k_scale=None), S.SSD_ERR_INVALID_ARG),
              (dict(v_scale=BUF + 2), S.SSD_ERR_INVALID_ARG)]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_bad_caches_are_refused(bad, status):
    c = cache(**bad)
    with pytest.raises(S.SsdError) as e:
        S.ssd_kv8_append(c, BUF, BUF, S.SSD_DTYPE_BF16, 512, 1, BUF)
    assert e.value.status == status and "cache" in str(e.value)
    with pytest.raises(S.SsdError) as e:
        S.ssd_kv8_attention(c, BUF, S.SSD_DTYPE_BF16, 4, 512, 1, BUF, 0, 0, 0, BUF, 512, BUF, 1 << 30)
    assert e.value.status == status
    assert S.ssd_kv8_attention_bytes(c, S.SSD_DTYPE_BF16, 4, 1) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), S.SSD_ERR_INVALID_ARG), (dict(v=BUF + 4), S.SSD_ERR_INVALID_ARG),
    (dict(dtype=2), S.SSD_ERR_INVALID_ARG), (dict(stride=511), S.SSD_ERR_INVALID_ARG),
    (dict(stride=516), S.SSD_ERR_INVALID_ARG), (dict(stride=-512), S.SSD_ERR_INVALID_ARG),
    (dict(M=0), S.SSD_ERR_INVALID_ARG), (dict(M=1025), S.SSD_ERR_CAPACITY),
    (dict(pos=0), S.SSD_ERR_INVALID_ARG)])
def test_append_refuses(kw, status):
    a = dict(k=BUF, v=BUF, dtype=S.SSD_DTYPE_BF16, stride=512, M=1, pos=BUF)
    a.update(kw)
    with pytest.raises(S.SsdError) as e:
        S.ssd_kv8_append(cache(), a["k"], a["v"], a["dtype"], a["stride"], a["M"], a["pos"])
    assert e.value.status == status
    assert S.lib().ssd_kv8_append(None, BUF, BUF, 1, 512, 1, BUF, None, None, None) == \
        S.SSD_ERR_INVALID_ARG


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), S.SSD_ERR_INVALID_ARG), (dict(q=BUF + 2), S.SSD_ERR_INVALID_ARG),
    (dict(out=0), S.SSD_ERR_INVALID_ARG), (dict(dtype=5), S.SSD_ERR_INVALID_ARG),
    (dict(heads=6), S.SSD_ERR_INVALID_ARG), (dict(heads=0), S.SSD_ERR_INVALID_ARG),
    (dict(heads=2), S.SSD_ERR_INVALID_ARG), (dict(qs=1020), S.SSD_ERR_INVALID_ARG),
    (dict(os=1028), S.SSD_ERR_INVALID_ARG), (dict(M=0), S.SSD_ERR_INVALID_ARG),
    (dict(M=1030), S.SSD_ERR_CAPACITY), (dict(window=-1), S.SSD_ERR_INVALID_ARG),
    (dict(pos=0), S.SSD_ERR_INVALID_ARG), (dict(seq=4096, ws=0), S.SSD_ERR_INVALID_ARG),
    (dict(seq=4096, ws=BUF + 16), S.SSD_ERR_INVALID_ARG),
    (dict(seq=4096, wb=1000), S.SSD_ERR_CAPACITY)])
def test_attention_refuses(kw, status):
    a = dict(q=BUF, out=BUF, dtype=S.SSD_DTYPE_BF16, heads=8, qs=1024, os=1024, M=3, window=0, pos=BUF,
             ws=BUF, wb=1 << 30, seq=1024)
    a.update(kw)
    with pytest.raises(S.SsdError) as e:
        S.ssd_kv8_attention(cache(max_seq=a["seq"]), a["q"], a["dtype"], a["heads"], a["qs"], a["M"], a["pos"], 0, 0,
                            a["window"], a["out"], a["os"], a["ws"], a["wb"])
    assert e.value.status == status
    with pytest.raises(S.SsdError) as e:  # more than 2^31 units of work
        S.ssd_kv8_attention(cache(max_seq=1 << 30, n_seq=4096), BUF, S.SSD_DTYPE_BF16, 8, 1024, 64, BUF,
                            0, 0, 0, BUF, 1024, BUF, 1 << 40)
    assert e.value.status == S.SSD_ERR_CAPACITY


def test_attention_workspace_sizes():
    """Small caches need none, others what their parts take, the same for every length."""
    assert S.ssd_kv8_attention_bytes(cache(max_seq=512), S.SSD_DTYPE_BF16, 8, 1) == 256
    assert S.ssd_kv8_attention_bytes(cache(max_seq=2048), S.SSD_DTYPE_BF16, 8, 1) == 256
    few = S.ssd_kv8_attention_bytes(cache(max_seq=2112), S.SSD_DTYPE_BF16, 8, 1)
    more = S.ssd_kv8_attention_bytes(cache(max_seq=1 << 14), S.SSD_DTYPE_BF16, 8, 8)
    assert 256 < few < more == S.ssd_kv8_attention_bytes(cache(max_seq=1 << 20), S.SSD_DTYPE_BF16, 8, 8)
    assert S.ssd_kv8_attention_bytes(cache(max_seq=1 << 14), S.SSD_DTYPE_BF16, 8, 9) > more
    for ws, nbytes, status in ((BUF, few - 1, S.SSD_ERR_CAPACITY), (0, few, S.SSD_ERR_INVALID_ARG)):
        with pytest.raises(S.SsdError) as e:
            S.ssd_kv8_attention(cache(max_seq=2112), BUF, S.SSD_DTYPE_BF16, 8, 1024, 1, BUF, 0, 0, 0, BUF,
                                1024, ws, nbytes)
        assert e.value.status == status


@pytest.mark.parametrize("kw,status", [
    (dict(z=0), S.SSD_ERR_INVALID_ARG), (dict(z=BUF + 1), S.SSD_ERR_INVALID_ARG),
    (dict(dtype=9), S.SSD_ERR_INVALID_ARG), (dict(rows=0), S.SSD_ERR_INVALID_ARG),
    (dict(vocab=0), S.SSD_ERR_INVALID_ARG), (dict(stride=999), S.SSD_ERR_INVALID_ARG),
    (dict(tok=0), S.SSD_ERR_INVALID_ARG), (dict(lp=0), S.SSD_ERR_INVALID_ARG),
    (dict(ntok=-1), S.SSD_ERR_INVALID_ARG), (dict(t=0.0), S.SSD_ERR_INVALID_ARG),
    (dict(t=float("nan")), S.SSD_ERR_INVALID_ARG), (dict(t=-1.0), S.SSD_ERR_INVALID_ARG),
    (dict(t=float("inf")), S.SSD_ERR_INVALID_ARG), (dict(top=33), S.SSD_ERR_INVALID_ARG),
    (dict(top=-1), S.SSD_ERR_INVALID_ARG), (dict(top=4, vocab=3, stride=3), S.SSD_ERR_INVALID_ARG),
    (dict(ids=0), S.SSD_ERR_INVALID_ARG), (dict(tops=0), S.SSD_ERR_INVALID_ARG)])
def test_token_logprobs_refuses(kw, status):
    a = dict(z=BUF, dtype=S.SSD_DTYPE_F32, rows=2, vocab=1000, stride=1000, tok=BUF, ntok=1, t=1.0,
             top=4, lp=BUF, ids=BUF, tops=BUF)
    a.update(kw)
    with pytest.raises(S.SsdError) as e:
        S.ssd_token_logprobs(a["z"], a["dtype"], a["rows"], a["vocab"], a["stride"], a["tok"],
                             a["ntok"], a["t"], a["top"], a["lp"], BUF, BUF, a["ids"], a["tops"])
    assert e.value.status == status


def test_python_entry_points_refuse_wrong_tensors():
    c = KV8Cache(2, 64, 100, n_seq=2, device="cpu")
    assert c.max_seq == 128 and c.k_scale.shape == (2, 2, 2)
    pos = torch.zeros(2, dtype=torch.int32)
    kv = torch.zeros(2, 3, 2, 64)
    for bad in (kv[:1], kv[..., :32], kv.double(), kv[0], kv.transpose(1, 2), torch.zeros(2, 3, 4, 64),
                torch.zeros(2, 5, 2, 64)[:, :3], torch.zeros(2, 3, 2, 128)[..., ::2]):
        with pytest.raises(ValueError):
            c.append(bad, bad, pos)
    for args in ((kv, kv.bfloat16(), pos), (kv, torch.zeros(2, 3, 4, 64)[:, :, :2], pos),
                 (kv, kv, pos.long()), (kv, kv, pos[:1]), (kv, kv, None),
                 (kv, kv, pos, torch.zeros(2)), (kv, kv, torch.zeros(4, dtype=torch.int32)[::2]),
                 (kv.requires_grad_(), kv, pos)):
        with pytest.raises(ValueError):
            c.append(*args)
    kv = kv.detach()
    with pytest.raises(ValueError, match="CUDA"):  # right in all but the device
        c.append(kv, kv, pos)
    q = torch.zeros(2, 3, 4, 64)
    for args, kw in (((q[:, :, :3], pos), {}), ((q.half(), pos), {}), ((q, pos), dict(window=-1)),
                     ((q, pos), dict(window=1 << 31)), ((q, pos), dict(out=q.bfloat16())),
                     ((q, pos), dict(out=q[:, :2])), ((q, pos), dict(first=pos.long())),
                     ((q, None), {}), ((q[0], pos), {})):
        with pytest.raises(ValueError):
            c.attention(*args, **kw)
    with pytest.raises(ValueError, match="CUDA"):
        c.attention(q, pos)
    for args in ((2, 96, 64), (0, 64, 64), (2, 64, 0), (2, 64, 64, 0), (2, 64, 64, 5000)):
        with pytest.raises(ValueError):
            KV8Cache(*args, device="cpu")
    z = torch.zeros(3, 50)
    t = torch.zeros(3, dtype=torch.int32)
    for args, kw in (((z[0],), {}), ((z.half(),), {}), ((z.t(),), {}), ((z, t.long()), {}),
                     ((z, t[:2]), {}), ((z, t), dict(top_n=33)), ((z, t), dict(top_n=-1)),
                     ((z[:, :4], t), dict(top_n=5)), ((z.expand(3, 50)[:1].expand(3, 50), t), {}),
                     ((z, t), dict(err=torch.zeros(1)))):
        with pytest.raises(ValueError):
            token_logprobs(*args, **kw)
    with pytest.raises(ValueError, match="CUDA"):
        token_logprobs(z, t)


def test_an_output_over_its_queries_has_their_stride():
    with pytest.raises(S.SsdError, match="strides differ"):
        S.ssd_kv8_attention(cache(), BUF, S.SSD_DTYPE_BF16, 8, 1024, 3, BUF, 0, 0, 0, BUF, 2048, BUF, 1 << 30)
    c = KV8Cache(2, 64, 64, device="cpu")
    pos = torch.zeros(1, dtype=torch.int32)
    buf = torch.zeros(1, 4, 4, 64)
    with pytest.raises(ValueError, match="strides differ"):
        c.attention(buf[:, ::2], pos, out=buf[:, :2])
    with pytest.raises(ValueError, match="CUDA"):
        c.attention(buf[:, ::2], pos, out=buf[:, ::2])


def test_the_caches_tensors_are_written_not_replaced():
    c = KV8Cache(2, 64, 64, device="cpu")
    for name in ("k", "v", "k_scale", "v_scale", "err"):
        with pytest.raises(AttributeError):
            setattr(c, name, torch.zeros(1))
    c.k_scale.fill_(2.0)
    assert bool((c.k_scale == 2.0).all())


def test_row_strides_that_are_read_in_place():
    """Slices of a fused q | k | v row, single rows and single sequences."""
    c = KV8Cache(2, 64, 64, n_seq=3, device="cpu")
    qkv = torch.zeros(3, 5, 8, 64)
    assert c._rows(qkv[:, :, 4:6], 2, "k") == (5, 512)
    assert c._rows(qkv[:, 2:3, 4:6], 2, "k") == (1, 2560)
    with pytest.raises(ValueError):
        c._rows(qkv[:, 1:, 4:6], 2, "k")  # the sequences' rows are not at one distance
    c1 = KV8Cache(2, 64, 64, device="cpu")
    assert c1._rows(qkv[:1, 1:4, 6:], 2, "k") == (3, 512)
    assert c1._rows(qkv[1:2, 2:3, 6:], 2, "k") == (1, 128)


def test_reference_rounding_is_the_type_s():
    g = torch.Generator().manual_seed(3)
    x = torch.cat([torch.randn(20000, generator=g) * 2.0 ** torch.randint(-14, 9, (20000,), generator=g),
                   torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float(),
                   torch.linspace(-448, 448, 30001), torch.tensor([0.0, -0.0, 448.0, 464.0 - 1e-3])])
    x = x[~x.isnan()].clamp(-448, 448)
    want = x.to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(R.e4m3_round(x.double().numpy()), want)


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.0 * 2 ** 20, 20), (449.0, 1), (1.0, -8), (1.75, -8),
                                    (1.7500001, -7), (2.0 ** -130, -120), (0.0, -120),
                                    (3.3e38, 111)])
def test_reference_scale(amax, e):
    assert R.scale_of(amax) == 2.0 ** e


def test_every_error_bit_of_the_kernels_is_named():
    """The bits that the kernels set are those of the header and of the binding, each with words."""
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    csrc = os.path.join(root, "paper_2606_03113_gb300", "csrc")
    header = open(os.path.join(root, "include", "ssd_ops.h")).read()
    named = {k: int(v) for k, v in re.findall(r"#define SSD_DEV_ERR_(\w+) (\d+)", header)}
    enum = dict(re.findall(r"kErr(\w+) = (\d+)", open(os.path.join(csrc, "common.cuh")).read()))
    used = set()
    for f in ("kv8_append.cu", "kv8_attention.cu", "kv8_plan.cuh", "kv8_wide.cuh", "logprobs.cu"):
        used |= set(re.findall(r"kErr([A-Z]\w+)", open(os.path.join(csrc, f)).read()))
    assert used == {"Token", "Capacity", "Control", "Timeout"}
    assert named == {u.upper(): int(enum[u]) for u in used}
    assert named == {k[8:]: v for k, v in vars(S).items() if k.startswith("DEV_ERR_") and k != "DEV_ERR_NAMES"}
    assert set(S.DEV_ERR_NAMES) == set(named.values())
    assert "gave up" in S.dev_err_text(16) and "positions" not in S.dev_err_text(16)
    both = S.dev_err_text(S.DEV_ERR_CAPACITY | S.DEV_ERR_CONTROL)
    assert "6" in both and "positions" in both and "rows" in both


@pytest.mark.parametrize("kw,M", [(dict(max_seq=64), 65), (dict(max_seq=1024), 1 << 30),
                                  (dict(max_seq=1 << 30, n_seq=4096), 64)])
def test_sizes_that_attention_refuses_have_no_workspace(kw, M):
    """The size query says 0, with the message of the call itself."""
    c = cache(**kw)
    with pytest.raises(S.SsdError) as e:
        S.ssd_kv8_attention(c, BUF, S.SSD_DTYPE_BF16, 8, 1024, M, BUF, 0, 0, 0, BUF, 1024, BUF, 1 << 40)
    assert e.value.status == S.SSD_ERR_CAPACITY
    why = S.lib().ssd_last_error(None)
    with pytest.raises(S.SsdError):  # another message in between
        S.ssd_kv8_append(cache(n_seq=0), BUF, BUF, S.SSD_DTYPE_BF16, 512, 1, BUF)
    assert S.ssd_kv8_attention_bytes(c, S.SSD_DTYPE_BF16, 8, M) == 0
    assert S.lib().ssd_last_error(None) == why
    assert S.ssd_kv8_attention_bytes(cache(max_seq=64), S.SSD_DTYPE_BF16, 8, 64) > 0


def test_the_module_imports_with_a_torch_without_cuda():
    """A PyTorch that lacks CUDA's own calls: the module, its checks and its refusals are there."""
    code = """
import torch
if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    del torch._C._cuda_getCurrentRawStream
from paper_2606_03113_gb300 import runtime
c = runtime.KV8Cache(2, 64, 64, device="cpu")
try:
    c.append(torch.zeros(1, 1, 2, 64), torch.zeros(1, 1, 2, 64), torch.zeros(1, dtype=torch.int32))
except ValueError as e:
    assert "CUDA" in str(e), e
else:
    raise SystemExit("not refused")
class Stream:
    cuda_stream = 77
torch.cuda.current_stream = lambda index: Stream()
assert runtime._current_stream(0) == 77
print("fine")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    got = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True)
    assert got.returncode == 0 and got.stdout.strip() == "fine", got.stderr
