"""Device model and engine on top of the C ABI.

`DeviceModel` allocates a Llama-shaped decoder's weights with PyTorch on one
GPU and fills them with the library's seeded synthetic-weight fixture (the
same generator the CPU oracle reads).  `Engine` owns one ssd_ctx: workspace
(KV cache, activations, control block) from PyTorch, work on a PyTorch stream.
`KV8Cache` is a layer's KV cache held in 8 bits, with its append and attention;
`PagedKVCache` a decoder's KV cache in pages that sequences share; `token_logprobs`
scores given tokens over rows of logits.
"""
from __future__ import annotations

import ctypes as C
import operator
from typing import NamedTuple

import numpy as np
import torch
from torch.autograd import forward_ad

import synth
from synth.workloads import ModelShape, Workload

from . import ssd as S


def _dt(shape: ModelShape):
    return (torch.bfloat16, S.SSD_DTYPE_BF16) if shape.dtype == "bf16" else (torch.float32,
                                                                            S.SSD_DTYPE_F32)


class DeviceModel:
    """Synthetic weights of `shape` on `device`: N(0, sigma^2)-like matrices
    (synth.h), out/down projections of the second half of the layers scaled by
    late_scale, unit norm weights."""

    def __init__(self, shape: ModelShape, device: str = "cuda:0", seed: int = synth.SEED_WEIGHTS):
        self.shape = shape
        self.device = torch.device(device)
        dt, code = _dt(shape)
        self.dtype_code = code
        s = shape
        stream = torch.cuda.current_stream(self.device).cuda_stream

        def mat(rows, cols, tid, sigma):
            t = torch.empty((rows, cols), dtype=dt, device=self.device)
            S.ssd_synth_fill(t.data_ptr(), code, t.numel(), seed, tid, sigma, stream)
            return t

        def ones(n):
            return torch.ones(n, dtype=dt, device=self.device)

        self.embed = mat(s.vocab, s.d_model, synth.TID_EMBED, s.sigma)
        self.lm_head = mat(s.vocab, s.d_model, synth.TID_LMHEAD, s.sigma)
        self.final_norm = ones(s.d_model)
        self.layers = []
        qd = s.n_heads * s.head_dim
        for l in range(s.n_layers):
            late = s.late_scale if l >= s.n_layers // 2 else 1.0
            base = synth.layer_tid(l, 0)
            self.layers.append(dict(
                attn_norm=ones(s.d_model),
                wqkv=mat(s.qkv_rows, s.d_model, base + 0, s.sigma),
                wo=mat(s.d_model, qd, base + 1, s.sigma * late),
                ffn_norm=ones(s.d_model),
                w_gate_up=mat(2 * s.ffn_dim, s.d_model, base + 2, s.sigma),
                w_down=mat(s.d_model, s.ffn_dim, base + 3, s.sigma * late)))
        torch.cuda.current_stream(self.device).synchronize()

    def weight_bytes(self) -> int:
        n = self.embed.numel() + self.lm_head.numel()
        for L in self.layers:
            n += sum(t.numel() for t in L.values())
        return n * self.embed.element_size()


class Engine:
    def __init__(self, model: DeviceModel, max_seq: int, stream: torch.cuda.Stream | None = None):
        s = model.shape
        self.model = model
        self.shape = s
        self.max_seq = max_seq
        self.stream = stream or torch.cuda.current_stream(model.device)
        cfg = S.ssd_model_cfg(s.n_layers, s.d_model, s.n_heads, s.n_kv_heads, s.head_dim, s.ffn_dim,
                              s.vocab, max_seq, s.rms_eps, s.rope_theta, model.dtype_code)
        self.cfg = cfg
        nbytes = S.ssd_workspace_bytes(cfg)
        if nbytes == 0:
            raise S.SsdError(S.SSD_ERR_INVALID_ARG, "ssd_workspace_bytes", "invalid configuration")
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=model.device)
        base = self.workspace.data_ptr()
        ptr = (base + 255) // 256 * 256
        L = s.n_layers
        arrs = {}
        for key in ("attn_norm", "wqkv", "wo", "ffn_norm", "w_gate_up", "w_down"):
            a = (C.c_void_p * L)(*[lw[key].data_ptr() for lw in model.layers])
            arrs[key] = a
        self._arrs = arrs
        w = S.ssd_weights(model.embed.data_ptr(), model.lm_head.data_ptr(),
                          model.final_norm.data_ptr(),
                          *[C.cast(arrs[k], C.POINTER(C.c_void_p))
                            for k in ("attn_norm", "wqkv", "wo", "ffn_norm", "w_gate_up", "w_down")])
        self.ctx = S.ssd_init_model(cfg, w, ptr, nbytes, self.stream.cuda_stream)
        self.policy_kind = None
        self.kmax = 0

    # ----------------------------------------------------------- policies
    def set_policy(self, kind: int, cand=(), kmax: int = 0, static_l: int = 0, static_k: int = 0,
                   qnet_params: np.ndarray | None = None, qnet_hidden: int = 0, trace_T: int = 20,
                   topk: int = 5, fixed_k: int = 0, conf_threshold: float = 0.0,
                   temperature: float = 0.0, sample_seed: int = 0, qnet_in: int = 3,
                   discard_on_continue: bool = False):
        """temperature > 0 turns on speculative sampling at that temperature
        (drafts drawn from the exit distribution, emitted tokens distributed
        as the full model's), with uniforms keyed by sample_seed."""
        cand_arr = (C.c_int32 * max(1, len(cand)))(*cand)
        qp = None
        if qnet_params is not None:
            arr = np.ascontiguousarray(qnet_params, dtype=np.float32).ravel()
            # the library copies W1[hidden][in], b1, W2[2][hidden], b2 from this pointer
            need = qnet_hidden * (qnet_in + 3) + 2
            if kind == S.SSD_POLICY_LEDE and arr.size != need:
                raise ValueError(f"qnet_params holds {arr.size} floats; a network with "
                                 f"{qnet_in} inputs and {qnet_hidden} hidden units needs {need}")
            self._qp = arr
            qp = self._qp.ctypes.data_as(C.POINTER(C.c_float))
        p = S.ssd_policy(kind, len(cand), C.cast(cand_arr, C.POINTER(C.c_int32)), kmax, static_l,
                         static_k, qnet_in, qnet_hidden, qp, trace_T, topk, fixed_k, conf_threshold,
                         temperature, sample_seed, 1 if discard_on_continue else 0)
        S.ssd_set_policy(self.ctx, p)
        self.policy_kind = kind
        self.kmax = 0 if kind == S.SSD_POLICY_AR else kmax

    # Each setter takes temperature= and sample_seed= (sampled decoding).
    def set_ar(self, **sampling):
        self.set_policy(S.SSD_POLICY_AR, **sampling)

    def set_static(self, l: int, k: int, kmax: int | None = None, **sampling):
        self.set_policy(S.SSD_POLICY_STATIC, kmax=kmax or k, static_l=l, static_k=k, **sampling)

    def set_lede(self, w: Workload, qnet_params: np.ndarray | None = None, kmax: int | None = None,
                 cand=None, fixed_k: int = 0, state: str = "paper",
                 discard_on_continue: bool = False, **sampling):
        """LEDE (§3.3); one candidate is the ablation without dynamic exit,
        fixed_k > 0 the one without adaptive drafting (Table 3).  state
        "paper": the network reads (C_5, H, C_trace); "pooled": the mean
        final-normed exit state of the round's rows and the max-probability
        (d_model + 1 inputs)."""
        if state not in ("paper", "pooled"):
            raise ValueError(f"unknown state {state!r}")
        q_in = 3 if state == "paper" else w.shape.d_model + 1
        qp = (qnet_params if qnet_params is not None
              else synth.qnet_hidden_params(q_in, w.qnet_hidden))
        self.set_policy(S.SSD_POLICY_LEDE, cand=tuple(cand or w.candidates), kmax=kmax or w.kmax,
                        qnet_params=qp, qnet_hidden=w.qnet_hidden, fixed_k=fixed_k,
                        qnet_in=q_in, discard_on_continue=discard_on_continue, **sampling)

    def set_threshold(self, l: int, tau: float, kmax: int, **sampling):
        """Fixed exit layer l; drafting goes on while a draft's max-probability
        is >= tau (a Draft & Verify-style rule, §4.1 baselines)."""
        self.set_policy(S.SSD_POLICY_THRESHOLD, kmax=kmax, static_l=l, conf_threshold=tau,
                        **sampling)

    # ------------------------------------------------------------ running
    def prefill(self, ids) -> int:
        return S.ssd_prefill(self.ctx, ids)

    def resume(self, ids):
        S.ssd_resume(self.ctx, ids)

    def step(self, cap: int):
        return S.ssd_step(self.ctx, cap)

    def generate(self, n: int, rounds: bool = False):
        out, nr, infos = S.ssd_generate(self.ctx, n, rounds_cap=n if rounds else 0)
        return out, nr, infos

    def generate_async(self, n: int, out: torch.Tensor | None = None):
        S.ssd_generate_async(self.ctx, n, out.data_ptr() if out is not None else 0)

    def generate_result(self, traces: bool = False, cap: int = 4096):
        return S.ssd_generate_result(self.ctx, cap if traces else 0)

    def traces(self, cap: int = 4096):
        return S.ssd_read_traces(self.ctx, cap)

    def forward_exit(self, ids, pos0: int, l_exit: int, topk: int = 5, logits: bool = True):
        return S.ssd_forward_exit(self.ctx, ids, pos0, l_exit, topk, logits, self.shape.vocab)

    def qnet_eval(self, states):
        return S.ssd_qnet_eval(self.ctx, states)

    def read_kv(self, layer, kind, head, p0, n):
        return S.ssd_read_kv(self.ctx, layer, kind, head, p0, n, self.shape.head_dim)

    def read_state(self):
        return S.ssd_read_state(self.ctx)

    def op_gemv(self, which: int, layer: int, x: torch.Tensor, y: torch.Tensor, stream=None):
        M = x.shape[0]
        st = (stream or self.stream).cuda_stream
        S.ssd_op_gemv(self.ctx, which, layer, M, x.data_ptr(), y.data_ptr(), st)

    def op_layer(self, kernel: int, layer: int, M: int, pos0: int, stream=None):
        st = (stream or self.stream).cuda_stream
        S.ssd_op_layer(self.ctx, kernel, layer, M, pos0, st)

    def close(self):
        if getattr(self, "ctx", None):
            S.ssd_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def pass_launches(n_layers: int, bf16: bool = True) -> int:
    """Kernel launches of a pass over n layers: bf16 runs the first QKV, then
    per layer attention and one chained launch (O, gate/up, down, next QKV);
    fp32 launches the five layer kernels per layer."""
    if n_layers <= 0:
        return 0
    return 2 * n_layers + 1 if bf16 else S.KERNELS_PER_LAYER * n_layers


def kernels_per_round(trace: dict, n_layers: int, kind: int, bf16: bool = True) -> int:
    """Kernel launches of one round of the round graph, from its record:
    round_begin, walk (embed; per visited segment its layers, head, decide),
    draft_begin, drafts (embed, layers 1..l*, head, decide), verify (embed,
    all layers, head), accept.  A head counts once (its product, the
    statistics and, in sampled decoding, the weight sums behind it), and so
    does attention (its splits and their merge)."""
    n = 1  # round_begin
    if trace["kcap"] > 0:
        prev = 0
        n += 1  # embed
        for c in trace["visited"]:
            n += pass_launches(c - prev, bf16) + 2
            prev = c
        n += 1  # draft_begin
        n += (trace["k"] - 1) * (1 + pass_launches(trace["lstar"], bf16) + 2)
    n += 1 + pass_launches(n_layers, bf16) + 1 + 1
    return n


# ------------------------------------------- 8-bit KV cache, token scores

_CODES = {torch.float32: S.SSD_DTYPE_F32, torch.bfloat16: S.SSD_DTYPE_BF16}


def _dtype_code(t: torch.Tensor, what: str) -> int:
    code = _CODES.get(t.dtype)
    if code is None:
        raise ValueError(f"{what} must be float32 or bfloat16, not {t.dtype}")
    return code


def _on(t, device: torch.device, what: str) -> int:
    """The device address of t, or 0 for None."""
    if t is None:
        return 0
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, not on {device}")
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what} requires a gradient: there is no backward pass")
    if forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError(f"{what} has a tangent: there is no forward-mode derivative")
    return t.data_ptr()


def _per_seq(t, n_seq: int, device: torch.device, what: str) -> int:
    """The address of an int32 [n_seq] tensor, or 0 for None."""
    if t is None:
        return 0
    if t.dtype is not torch.int32 or t.shape != (n_seq,) or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous int32 tensor of {n_seq} elements")
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, not on {device}")
    return t.data_ptr()


# The address of a device's current stream (its index given), without a Stream object where this
# PyTorch has that call: one built without CUDA has not, and imports this module all the same.
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _elsewhere(device: torch.device, stream):
    """None where a call's work belongs on the current stream of the current device; else a
    context that makes it so (`stream`'s, or `device`'s current one)."""
    if device.type != "cuda":
        raise ValueError(f"a CUDA device is needed, not {device}")
    if stream is not None:
        if stream.device != device:
            raise ValueError(f"the stream is on {stream.device}, not on {device}")
        return torch.cuda.stream(stream)
    return None if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _rows_of(x: torch.Tensor, n: int, heads: int, hd: int, what: str) -> tuple[int, int]:
    """(M, elements between rows) of x [n, M, heads, hd]."""
    shape, strides = x.shape, x.stride()
    if len(shape) != 4 or shape[0] != n or shape[2] != heads or shape[3] != hd or shape[1] < 1:
        raise ValueError(f"{what} must be [{n}, M, {heads}, {hd}], not {list(shape)}")
    s0, s1, s2, s3 = strides
    M = shape[1]
    row = s1 if M > 1 else (s0 if n > 1 else heads * hd)
    if s3 != 1 or (s2 != hd and heads > 1) or (n > 1 and s0 != M * row):
        raise ValueError(f"{what}: a row's heads must lie one behind the other, and the rows "
                         f"of all sequences at one distance; strides are {strides}")
    return M, row


class KV8Cache:
    """The KV cache of one layer in 8 bits (ssd_kv8_cache, include/ssd_ops.h): e4m3 codes `k`, `v`
    [n_seq, n_kv_heads, max_seq, head_dim], one scale per 64 positions and KV head in `k_scale`,
    `v_scale` [n_seq, n_kv_heads, max_seq / 64].  `max_seq` is rounded up to a multiple of 64.

    Calls enqueue on `stream`, or on the current stream of the cache's device, and do not
    synchronise; the caller orders streams, and keeps tensors that another stream made alive
    (`Tensor.record_stream`).  They can be captured into CUDA graphs after a first call outside
    of a capture.  What only the device can see sets a bit in `err`, which `check` reads: positions
    outside the cache and bad row numbers leave the sequence alone, a kernel whose wait gave up
    after some seconds leaves the call's outputs undefined.

    A sequence that takes over another's place and begins inside of a block of 64 positions (a
    padded batch whose pads are not appended) has its `k_scale[b]` and `v_scale[b]` zeroed first:
    the scale that stands there counts as that of the positions in front."""

    # the tensors can be written, but not replaced: calls have their addresses
    k, v = (property(operator.attrgetter(x)) for x in ("_k", "_v"))
    k_scale, v_scale = (property(operator.attrgetter(x)) for x in ("_k_scale", "_v_scale"))
    err = property(operator.attrgetter("_err"))

    def __init__(self, n_kv_heads: int, head_dim: int, max_seq: int, n_seq: int = 1,
                 device: str | torch.device = "cuda:0"):
        device = torch.device(device)
        if device.type == "cuda" and device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        if head_dim not in (64, 128):
            raise ValueError(f"head_dim must be 64 or 128, not {head_dim}")
        if n_kv_heads < 1 or max_seq < 1 or not 1 <= n_seq <= S.KV8_MAX_SEQS:
            raise ValueError("n_kv_heads, max_seq and n_seq must be positive, "
                             f"n_seq at most {S.KV8_MAX_SEQS}")
        self.device, self.n_seq, self.n_kv_heads, self.head_dim = device, n_seq, n_kv_heads, head_dim
        self.max_seq = (max_seq + S.KV8_BLOCK - 1) // S.KV8_BLOCK * S.KV8_BLOCK
        shape = (n_seq, n_kv_heads, self.max_seq, head_dim)
        scales = (n_seq, n_kv_heads, self.max_seq // S.KV8_BLOCK)
        # zeros where nothing was appended, for whoever looks at the tensors
        self._k = torch.zeros(shape, dtype=torch.float8_e4m3fn, device=device)
        self._v = torch.zeros(shape, dtype=torch.float8_e4m3fn, device=device)
        self._k_scale = torch.zeros(scales, dtype=torch.float32, device=device)
        self._v_scale = torch.zeros(scales, dtype=torch.float32, device=device)
        self._err = torch.zeros(1, dtype=torch.int32, device=device)
        self._c = S.ssd_kv8_cache(n_seq, n_kv_heads, head_dim, self.max_seq, self.k.data_ptr(),
                                  self.v.data_ptr(), self.k_scale.data_ptr(),
                                  self.v_scale.data_ptr())
        self._err_at = self._err.data_ptr()
        self._work = {}  # (dtype code, n_heads, M) -> workspace bytes

    def _rows(self, x: torch.Tensor, heads: int, what: str) -> tuple[int, int]:
        """(M, elements between rows) of x [n_seq, M, heads, head_dim]."""
        return _rows_of(x, self.n_seq, heads, self.head_dim, what)

    def append(self, k: torch.Tensor, v: torch.Tensor, pos: torch.Tensor,
               rows: torch.Tensor | None = None, stream=None):
        """Writes k[b, m], v[b, m] ([n_seq, M, n_kv_heads, head_dim]) for m < rows[b] (all M
        without `rows`) to positions pos[b] + m.  Positions from pos[b] on count as free; a scale
        that rows rolled back have raised stays until its block is written from the start."""
        code = _dtype_code(k, "k")
        if v.dtype != k.dtype:
            raise ValueError("k and v must have one type")
        M, row = self._rows(k, self.n_kv_heads, "k")
        if self._rows(v, self.n_kv_heads, "v") != (M, row):
            raise ValueError("k and v must have the same rows and strides")
        if pos is None:
            raise ValueError("pos is missing")
        kp, vp = _on(k, self.device, "k"), _on(v, self.device, "v")
        pp = _per_seq(pos, self.n_seq, self.device, "pos")
        rp = _per_seq(rows, self.n_seq, self.device, "rows")
        there = _elsewhere(self.device, stream)
        if there is not None:
            with there:
                return self.append(k, v, pos, rows)
        S.ssd_kv8_append(self._c, kp, vp, code, row, M, pp, rp, self._err_at,
                         _current_stream(self.device.index))

    def attention(self, q: torch.Tensor, pos: torch.Tensor, rows: torch.Tensor | None = None,
                  first: torch.Tensor | None = None, window: int = 0,
                  out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """softmax(q k^T / sqrt(head_dim)) v for q [n_seq, M, n_heads, head_dim]: row m < rows[b]
        of sequence b sits at position pos[b] + m, whose key has been appended, and sees the keys
        up to its own from first[b] on, at most `window` of them (0: all).  A row that sees
        none is zero.  Returns `out`, which keeps its rows from rows[b] on; without it a new
        tensor, where those are zero (a sequence with bad positions leaves its own unset)."""
        code = _dtype_code(q, "q")
        heads = q.shape[2] if q.dim() == 4 else 0
        M, row = self._rows(q, heads, "q")
        if heads < 1 or heads % self.n_kv_heads:
            raise ValueError(f"q has {heads} heads: not a multiple of {self.n_kv_heads}")
        if pos is None:
            raise ValueError("pos is missing")
        qp = _on(q, self.device, "q")
        pp = _per_seq(pos, self.n_seq, self.device, "pos")
        rp = _per_seq(rows, self.n_seq, self.device, "rows")
        fp = _per_seq(first, self.n_seq, self.device, "first")
        if out is not None:
            if out.dtype != q.dtype:
                raise ValueError("out must have q's type")
            Mo, orow = self._rows(out, heads, "out")
            if Mo != M:
                raise ValueError("out must have q's rows")
            if _on(out, self.device, "out") == qp and orow != row:
                raise ValueError("out is q, but their strides differ")
        if not 0 <= window < 1 << 31:
            raise ValueError(f"window must be 0 (none) or a positive int32, not {window}")
        key = (code, heads, M)
        nbytes = self._work.get(key)
        if nbytes is None:
            nbytes = S.ssd_kv8_attention_bytes(self._c, code, heads, M)
            self._work[key] = nbytes
        there = _elsewhere(self.device, stream)
        if there is not None:
            with there:
                return self.attention(q, pos, rows, first, window, out)
        if out is None:
            make = torch.empty if rows is None else torch.zeros
            out = make((self.n_seq, M, heads, self.head_dim), dtype=q.dtype, device=self.device)
            orow = heads * self.head_dim
        # (256: none is used; others stay this call's until the launches)
        work = torch.empty(nbytes, dtype=torch.uint8, device=self.device) if nbytes > 256 else None
        S.ssd_kv8_attention(self._c, qp, code, heads, row, M, pp, rp, fp, window, out.data_ptr(), orow,
                            work.data_ptr() if work is not None else 0, nbytes, self._err_at,
                            _current_stream(self.device.index))
        return out

    def check(self):
        """Waits for the device and raises SsdError, with what it was, if a call since the last
        check set an error bit there."""
        torch.cuda.synchronize(self.device)
        bits = int(self.err.item())
        if bits:
            self.err.zero_()
            raise S.SsdError(S.SSD_ERR_DEVICE_FLAG, "KV8Cache", S.dev_err_text(bits))


class PagedKVCache:
    """A decoder's KV cache in pages that sequences share and give back (ssd_paged_cache,
    include/ssd_ops.h): `pages` [n_pages, n_layers, 2 (K, V), n_kv_heads, page, head_dim] (a view: in
    memory the heads stand in front of K and V), the pages of each sequence in `table`
    [n_seq, max_seq / page] (-1: none), how many entries name each page in `refs` [n_pages] (0: free).
    `max_seq` is rounded up to a multiple of `page` (a power of two from 16 to 256).

    A step of decoding: `fork` where sequences branch, are cut back or end; `reserve` the places of the new
    rows (a shared page is copied before it is written); for each layer `append` their K and V and
    `attention` of their queries.  `compact` moves what is in use to the low end of the pool.

    Calls enqueue on `stream`, or on the current stream of the cache's device, and do not
    synchronise; the caller orders streams (`fork`, `reserve` and `compact` against every other
    call on the cache), and keeps tensors that another stream made alive
    (`Tensor.record_stream`).  They can be captured into CUDA graphs after a first call outside
    of a capture.  What only the device can see sets a bit in `err`, which `check` reads: positions
    outside the cache, bad row numbers and parents leave the sequence alone; a `reserve` for which the
    free pages do not suffice changes nothing; rows whose page is missing or shared are not appended,
    and a sequence that sees a missing page has undefined attention."""

    # the tensors can be written, but not replaced: calls have their addresses
    pages, table, refs, err = (property(operator.attrgetter(x))
                               for x in ("_pages", "_table", "_refs", "_err"))

    def __init__(self, n_layers: int, n_kv_heads: int, head_dim: int, n_pages: int, page: int = 64,
                 n_seq: int = 1, max_seq: int | None = None, dtype: torch.dtype = torch.bfloat16,
                 device: str | torch.device = "cuda:0"):
        device = torch.device(device)
        if device.type == "cuda" and device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        if head_dim not in (64, 128):
            raise ValueError(f"head_dim must be 64 or 128, not {head_dim}")
        if page not in S.PAGE_SIZES:
            raise ValueError(f"page must be one of {S.PAGE_SIZES}, not {page}")
        if dtype not in _CODES:
            raise ValueError(f"dtype must be float32 or bfloat16, not {dtype}")
        if n_layers < 1 or n_kv_heads < 1 or n_pages < 1 or not 1 <= n_seq <= S.KV8_MAX_SEQS:
            raise ValueError("n_layers, n_kv_heads, n_pages and n_seq must be positive, "
                             f"n_seq at most {S.KV8_MAX_SEQS}")
        max_seq = n_pages * page if max_seq is None else max_seq
        if not 1 <= max_seq <= 1 << 30:
            raise ValueError(f"max_seq must be in 1..2^30, not {max_seq}")
        self.device, self.dtype, self.page = device, dtype, page
        self.n_layers, self.n_kv_heads, self.head_dim = n_layers, n_kv_heads, head_dim
        self.n_seq, self.n_pages = n_seq, n_pages
        self.max_pages = (max_seq + page - 1) // page
        self.max_seq = self.max_pages * page
        # a head's keys and values in a page lie side by side
        self._pages = torch.zeros((n_pages, n_layers, n_kv_heads, 2, page, head_dim), dtype=dtype,
                                  device=device).transpose(2, 3)
        self._table = torch.full((n_seq, self.max_pages), -1, dtype=torch.int32, device=device)
        self._refs = torch.zeros(n_pages, dtype=torch.int32, device=device)
        self._err = torch.zeros(1, dtype=torch.int32, device=device)
        self._c = S.ssd_paged_cache(n_layers, n_seq, n_kv_heads, head_dim, page, n_pages,
                                    self.max_pages, _CODES[dtype], self._pages.data_ptr(),
                                    self._table.data_ptr(), self._refs.data_ptr())
        self._err_at = self._err.data_ptr()
        # of the calls that change pages, which run one after the other
        self._plan_bytes = S.ssd_paged_workspace_bytes(self._c) if device.type == "cuda" else 0
        self._plan = torch.empty(self._plan_bytes, dtype=torch.uint8, device=device)
        self._plan_at = self._plan.data_ptr()
        self._work = {}  # (n_heads, M, window, longest) -> workspace bytes
        # what every call looks at (the calls of a decode step are as short as their launches: they
        # look at each tensor once, and leave the words of a refusal to the slower checks)
        self._at = C.addressof(self._c)
        self._lib = S.lib()
        self._seqs = torch.Size((n_seq,))
        self._index = device.index if device.type == "cuda" else -1

    def _ints(self, t, what: str) -> int:
        """The address of an int32 [n_seq] tensor, or 0 for None."""
        if t is None:
            return 0
        if t.dtype is not torch.int32 or t.shape != self._seqs or not t.is_contiguous() or \
                t.get_device() != self._index:
            return _per_seq(t, self.n_seq, self.device, what)
        return t.data_ptr()

    def _rows(self, x: torch.Tensor, heads: int, what: str) -> tuple[int, int, int]:
        """(address, M, elements between rows) of x [n_seq, M, heads, head_dim]."""
        if x.dtype is not self.dtype:
            raise ValueError(f"{what} must be {self.dtype}, as the cache, not {x.dtype}")
        M, row = _rows_of(x, self.n_seq, heads, self.head_dim, what)
        at = x.data_ptr() if x.get_device() == self._index and not x.requires_grad and \
            forward_ad._current_level < 0 else _on(x, self.device, what)
        return at, M, row

    def _here(self, stream) -> bool:
        """Whether a call's work belongs on the current stream of the current device."""
        return stream is None and self._index >= 0 and _current_device() == self._index

    def _layer(self, layer: int) -> int:
        if not 0 <= layer < self.n_layers:
            raise ValueError(f"layer must be in 0..{self.n_layers - 1}, not {layer}")
        return layer

    def reserve(self, pos: torch.Tensor, rows: torch.Tensor | int = 1, stream=None):
        """Pages for rows[b] new rows (or `rows` of each sequence) at positions pos[b] and up: missing
        ones, and copies of shared ones up to pos[b] (what stood from there on in such a page is left
        behind), are taken lowest first.  Changes nothing where too few pages are free (`check` raises)."""
        if pos is None:
            raise ValueError("pos is missing")
        pp = self._ints(pos, "pos")
        rp, M = 0, self.max_seq
        if isinstance(rows, int):
            M = rows
            if not 1 <= M <= self.max_seq:
                raise ValueError(f"rows must be in 1..{self.max_seq}, not {M}")
        else:
            rp = self._ints(rows, "rows")
            if not rp:
                raise ValueError("rows is missing")
        if not self._here(stream):
            there = _elsewhere(self.device, stream)
            if there is not None:
                with there:
                    return self.reserve(pos, rows)
        st = self._lib.ssd_paged_reserve(self._at, pp, rp, M, self._plan_at, self._plan_bytes,
                                         self._err_at, _current_stream(self._index))
        if st:
            S._check(st, "ssd_paged_reserve")

    def fork(self, parent: torch.Tensor | None, length: torch.Tensor | None = None, stream=None):
        """Sequence b becomes the first length[b] positions (all without `length`) of what sequence
        parent[b] was (-1: empty; without `parent`: of itself), sharing its pages."""
        if parent is None and length is None:
            raise ValueError("neither parent nor length")
        pp, lp = self._ints(parent, "parent"), self._ints(length, "length")
        if not self._here(stream):
            there = _elsewhere(self.device, stream)
            if there is not None:
                with there:
                    return self.fork(parent, length)
        st = self._lib.ssd_paged_fork(self._at, pp, lp, self._err_at, _current_stream(self._index))
        if st:
            S._check(st, "ssd_paged_fork")

    def truncate(self, length: torch.Tensor, stream=None):
        """Sequence b keeps its first length[b] positions and gives the pages behind them back."""
        if length is None:
            raise ValueError("length is missing")
        self.fork(None, length, stream)

    def compact(self, stream=None) -> torch.Tensor:
        """Moves the pages in use to the low end of the pool; the free ones are its tail then.
        Returns how many are in use (int32 [1] on the device)."""
        if not self._here(stream):
            there = _elsewhere(self.device, stream)
            if there is not None:
                with there:
                    return self.compact()
        used = torch.empty(1, dtype=torch.int32, device=self.device)
        st = self._lib.ssd_paged_compact(self._at, used.data_ptr(), self._plan_at, self._plan_bytes,
                                         self._err_at, _current_stream(self._index))
        if st:
            S._check(st, "ssd_paged_compact")
        return used

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, pos: torch.Tensor,
               rows: torch.Tensor | None = None, stream=None):
        """Writes k[b, m], v[b, m] ([n_seq, M, n_kv_heads, head_dim]) for m < rows[b] (all M
        without `rows`) to positions pos[b] + m of a layer, which have been reserved."""
        layer = self._layer(layer)
        kp, M, row = self._rows(k, self.n_kv_heads, "k")
        vp, Mv, vrow = self._rows(v, self.n_kv_heads, "v")
        if Mv != M or vrow != row:
            raise ValueError("k and v must have the same rows and strides")
        if pos is None:
            raise ValueError("pos is missing")
        pp, rp = self._ints(pos, "pos"), self._ints(rows, "rows")
        if not self._here(stream):
            there = _elsewhere(self.device, stream)
            if there is not None:
                with there:
                    return self.append(layer, k, v, pos, rows)
        st = self._lib.ssd_paged_append(self._at, layer, kp, vp, row, M, pp, rp, self._err_at,
                                        _current_stream(self._index))
        if st:
            S._check(st, "ssd_paged_append")

    def attention(self, layer: int, q: torch.Tensor, pos: torch.Tensor,
                  rows: torch.Tensor | None = None, first: torch.Tensor | None = None,
                  window: int = 0, longest: int = 0, out: torch.Tensor | None = None,
                  stream=None) -> torch.Tensor:
        """softmax(q k^T / sqrt(head_dim)) v over a layer's pages for q [n_seq, M, n_heads,
        head_dim]: row m < rows[b] of sequence b sits at position pos[b] + m, whose key has been
        appended, and sees the keys up to its own from first[b] on, at most `window` of them
        (0: all).  A row that sees none is zero.  Scores and sums are fp32, probabilities too, or of
        16 bits in a bf16 cache.  `longest`: no sequence's pos[b] + rows[b] exceeds
        it (0: max_seq), which short sequences in a large table gain by.  Returns `out`, which keeps
        its rows from rows[b] on; without it a new tensor, where those are zero (a sequence with
        bad positions leaves its own unset)."""
        layer = self._layer(layer)
        shape = q.shape
        heads = shape[2] if len(shape) == 4 else 0
        qp, M, row = self._rows(q, heads, "q")
        if heads < 1 or heads % self.n_kv_heads:
            raise ValueError(f"q has {heads} heads: not a multiple of {self.n_kv_heads}")
        if pos is None:
            raise ValueError("pos is missing")
        pp, rp, fp = self._ints(pos, "pos"), self._ints(rows, "rows"), self._ints(first, "first")
        if out is not None:
            op, Mo, orow = self._rows(out, heads, "out")
            if Mo != M:
                raise ValueError("out must have q's rows")
            if op == qp and orow != row:
                raise ValueError("out is q, but their strides differ")
        if not 0 <= window < 1 << 31:
            raise ValueError(f"window must be 0 (none) or a positive int32, not {window}")
        if not 0 <= longest <= self.max_seq:
            raise ValueError(f"longest must be in 0..{self.max_seq}, not {longest}")
        key = (heads, M, window, longest)
        nbytes = self._work.get(key)
        if nbytes is None:
            nbytes = S.ssd_paged_attention_bytes(self._c, heads, M, window, longest)
            if len(self._work) < 4096:  # (a caller may pass another `longest` every step)
                self._work[key] = nbytes
        if not self._here(stream):
            there = _elsewhere(self.device, stream)
            if there is not None:
                with there:
                    return self.attention(layer, q, pos, rows, first, window, longest, out)
        if out is None:
            make = torch.empty if rows is None else torch.zeros
            out = make((self.n_seq, M, heads, self.head_dim), dtype=q.dtype, device=self.device)
            op, orow = out.data_ptr(), heads * self.head_dim
        # (256: none is used; others stay this call's until the launches)
        work = torch.empty(nbytes, dtype=torch.uint8, device=self.device) if nbytes > 256 else None
        st = self._lib.ssd_paged_attention(self._at, layer, qp, heads, row, M, pp, rp, fp, window, longest,
                                           op, orow, work.data_ptr() if work is not None else 0, nbytes,
                                           self._err_at, _current_stream(self._index))
        if st:
            S._check(st, "ssd_paged_attention")
        return out

    def check(self):
        """Waits for the device and raises SsdError, with what it was, if a call since the last
        check set an error bit there."""
        torch.cuda.synchronize(self.device)
        bits = int(self.err.item())
        if bits:
            self.err.zero_()
            raise S.SsdError(S.SSD_ERR_DEVICE_FLAG, "PagedKVCache", S.dev_err_text(bits))


class TokenLogprobs(NamedTuple):
    """Per row of logits: log-probabilities of the given tokens [rows, n] (None without tokens),
    log-sum-exp and entropy [rows], ids and log-probabilities of the most probable tokens
    [rows, top_n] (None for top_n 0), and the device word of error bits [1]."""
    logprob: torch.Tensor | None
    lse: torch.Tensor
    entropy: torch.Tensor
    top_id: torch.Tensor | None
    top_logprob: torch.Tensor | None
    err: torch.Tensor | None


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor | None = None, top_n: int = 0,
                   temperature: float = 1.0, err: torch.Tensor | None = None,
                   stream=None) -> TokenLogprobs:
    """ssd_token_logprobs on logits [rows, vocab] (float32 or bfloat16, rows at any distance) and
    tokens [rows, n] or [rows] (int32; -1: no token here, its result is 0).  Other ids outside the
    vocabulary give NaN and set a bit in `err` (device int32 [1]) where one is given.  Enqueues on
    `stream`, or on the current stream of the logits' device; does not synchronise."""
    code = _dtype_code(logits, "logits")
    shape = logits.shape
    if len(shape) != 2 or shape[0] < 1 or shape[1] < 1:
        raise ValueError(f"logits must be [rows, vocab], not {list(shape)}")
    n, vocab = shape
    row, one = logits.stride()
    if vocab > 1 and one != 1:
        raise ValueError("a row's logits must be consecutive")
    if n == 1:
        row = vocab
    elif row < vocab:
        raise ValueError("rows of logits must not overlap")
    if not 0 <= top_n <= S.MAX_TOP or top_n > vocab:
        raise ValueError(f"top_n must be in 0..{S.MAX_TOP} and at most the vocabulary, not {top_n}")
    dev = logits.device
    zp = _on(logits, dev, "logits")
    ntok, tp = 0, 0
    if tokens is not None:
        tshape = tokens.shape
        if tokens.dtype is not torch.int32 or len(tshape) not in (1, 2) or tshape[0] != n or \
                not tokens.is_contiguous():
            raise ValueError(f"tokens must be a contiguous int32 tensor [{n}, n] or [{n}]")
        ntok = 1 if len(tshape) == 1 else tshape[1]
        tp = _on(tokens, dev, "tokens")
    if err is not None and (err.dtype != torch.int32 or err.numel() < 1):
        raise ValueError("err must be an int32 tensor")
    ep = _on(err, dev, "err")
    there = _elsewhere(dev, stream)
    if there is not None:
        with there:
            return token_logprobs(logits, tokens, top_n, temperature, err)
    empty, f32 = torch.empty, torch.float32
    lp = ids = top = None
    lpp = ip = lp_top = 0
    if tokens is not None:
        lp = empty(tshape, dtype=f32, device=dev)
        lpp = lp.data_ptr()
    lse = empty(n, dtype=f32, device=dev)
    entropy = empty(n, dtype=f32, device=dev)
    if top_n > 0:
        ids = empty((n, top_n), dtype=torch.int32, device=dev)
        top = empty((n, top_n), dtype=f32, device=dev)
        ip, lp_top = ids.data_ptr(), top.data_ptr()
    S.ssd_token_logprobs(zp, code, n, vocab, row, tp, ntok, temperature, top_n, lpp, lse.data_ptr(),
                         entropy.data_ptr(), ip, lp_top, ep, _current_stream(dev.index))
    return TokenLogprobs(lp, lse, entropy, ids, top, err)
