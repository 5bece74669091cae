"""A small convenience layer over the C-ABI binding: owns a context and the
result tensors, so a caller writes ``eng.lookup_inject(tokens, h)``.

Nothing is computed here -- every call goes straight to libtfe.so.
"""
from __future__ import annotations

import contextlib
from dataclasses import dataclass

import numpy as np
import torch

from . import binding as tfe


@dataclass
class LookupOutput:
    out: torch.Tensor          # [Q, d] hidden dtype
    sel_phrase: torch.Tensor   # uint32 bit patterns in an int32 tensor, [Q] or [Q, n_orders]
    sel_slot: torch.Tensor     # int32
    flags: torch.Tensor        # uint8


class Engram:
    """GPU-resident phrase index + GPU-tier row store for one table."""

    def __init__(self, phrase_tokens, phrase_len, init_slot, gpu_rows: torch.Tensor, *, vocab, orders,
                 load_factor=0.7, hidden_dtype=tfe.HIDDEN_BF16, max_kicks=0, stream=None, device_build=False):
        assert gpu_rows.is_cuda and gpu_rows.dtype == torch.bfloat16 and gpu_rows.is_contiguous()
        self.rows = gpu_rows
        self.C, self.d = gpu_rows.shape
        self.orders = tuple(int(o) for o in orders)
        self.hidden_dtype = hidden_dtype
        self.torch_hidden = torch.bfloat16 if hidden_dtype == tfe.HIDDEN_BF16 else torch.float32
        self.cfg = tfe.make_config(d=self.d, vocab=vocab, orders=self.orders, n_phrases=len(phrase_len),
                                   gpu_slots=self.C, load_factor=load_factor, hidden_dtype=hidden_dtype,
                                   max_kicks=max_kicks)
        self.ctx = 0
        if device_build:        # the phrase arrays go to (or already are on) the device; the index is built there
            dev = gpu_rows.device
            as_dev = lambda a, dt: a.to(dev, dt).contiguous() if torch.is_tensor(a) else \
                torch.from_numpy(np.ascontiguousarray(a)).to(dev, dt)
            pt = as_dev(phrase_tokens, torch.int32).reshape(-1, 4)
            pl = as_dev(phrase_len, torch.uint8)
            sl = as_dev(init_slot, torch.int32)
            self.ctx = tfe.tfe_index_build_device(self.cfg, pt, pl, sl, gpu_rows, stream)
        else:
            self.ctx = tfe.tfe_index_build(self.cfg, phrase_tokens, phrase_len, init_slot, gpu_rows, stream)

    def close(self):
        if getattr(self, "ctx", 0):
            tfe.tfe_destroy(self.ctx)
            self.ctx = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def lookup_inject(self, tokens: torch.Tensor, h: torch.Tensor, out: torch.Tensor | None = None, *,
                      q_start=0, policy=tfe.POLICY_LONGEST, gate=tfe.GATE_CONST, lam=1.0, want_sel=True,
                      stream=None) -> LookupOutput:
        B, T = tokens.shape
        Q = B * (T - q_start)
        assert tokens.dtype == torch.int32 and tokens.is_cuda
        assert h.shape == (Q, self.d) and h.dtype == self.torch_hidden
        if out is None:
            out = torch.empty_like(h)
        shape = (Q,) if policy == tfe.POLICY_LONGEST else (Q, len(self.orders))
        sp = ss = fl = None
        if want_sel:
            sp = torch.empty(shape, dtype=torch.int32, device=h.device)
            ss = torch.empty(shape, dtype=torch.int32, device=h.device)
            fl = torch.empty(shape, dtype=torch.uint8, device=h.device)
        tfe.tfe_lookup_inject(self.ctx, tokens, B, T, q_start, h, out, policy=policy, gate=gate, lam=lam,
                              sel_phrase=sp, sel_slot=ss, flags=fl, stream=stream)
        return LookupOutput(out, sp, ss, fl)

    def miss_list(self, cap: int | None = None, stream=None, allow_overflow=False):
        if cap is None:
            cap = 1 << 20
        return tfe.tfe_miss_list(self.ctx, cap, stream, allow_overflow)

    def prefetch_candidates(self, history: torch.Tensor, cand_tokens: torch.Tensor, cand_prob: torch.Tensor, *,
                            usefulness: torch.Tensor | None = None, benefit_host=1.0, benefit_ssd=2.0, budget=4096,
                            stream=None):
        """(phrase, tier, score, src, [written, found]) device tensors of the `budget` best candidates."""
        B, H = history.shape
        K = cand_tokens.shape[1]
        dev = cand_tokens.device
        ph = torch.empty(max(budget, 1), dtype=torch.int32, device=dev)
        tr = torch.empty(max(budget, 1), dtype=torch.uint8, device=dev)
        sc = torch.empty(max(budget, 1), dtype=torch.float32, device=dev)
        sr = torch.empty(max(budget, 1), dtype=torch.int32, device=dev)
        cnt = torch.zeros(2, dtype=torch.int32, device=dev)
        tfe.tfe_prefetch_candidates(self.ctx, history, B, H, cand_tokens, cand_prob, K, out_phrase=ph, out_tier=tr,
                                    out_score=sc, out_src=sr, out_count=cnt, usefulness=usefulness,
                                    benefit_host=benefit_host, benefit_ssd=benefit_ssd, budget=budget, stream=stream)
        return ph, tr, sc, sr, cnt

    def cache_install(self, phrase_ids, src_rows, dst_slots, stream=None):
        tfe.tfe_cache_install(self.ctx, phrase_ids, src_rows, dst_slots, stream)

    def cache_install_device(self, phrase_ids: torch.Tensor, src_rows: torch.Tensor, dst_slots: torch.Tensor, stream=None):
        """Device tensors in, (applied uint8 [n], count int32 [1]) device tensors out; nothing synchronises."""
        n = int(phrase_ids.shape[0])
        applied = torch.empty(max(n, 1), dtype=torch.uint8, device=phrase_ids.device)
        count = torch.zeros(1, dtype=torch.int32, device=phrase_ids.device)
        tfe.tfe_cache_install_device(self.ctx, n, phrase_ids, src_rows, dst_slots, applied, count, stream)
        return applied[:n], count

    def cache_policy_enable(self, stream=None):
        tfe.tfe_cache_policy_enable(self.ctx, stream)

    def cache_select_victims(self, n, half_life=0, stream=None):
        return tfe.tfe_cache_select_victims(self.ctx, n, half_life, stream)

    def cache_stats(self, stream=None):
        return tfe.tfe_cache_stats(self.ctx, self.C, stream)


def bf16_tensor_from_bits(bits: np.ndarray, device) -> torch.Tensor:
    """uint16 bit patterns -> torch.bfloat16 tensor on ``device`` (no conversion)."""
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(device).view(torch.bfloat16)


def bits_from_bf16_tensor(t: torch.Tensor) -> np.ndarray:
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class EarlyExitHead:
    """softmax(W_pref h) + top-K on the GPU.  ``w_pref``: bf16 CUDA tensor [V, d], kept alive here."""

    def __init__(self, w_pref: torch.Tensor, max_batch: int = 256):
        assert w_pref.is_cuda and w_pref.dtype == torch.bfloat16 and w_pref.is_contiguous()
        self.w = w_pref
        self.V, self.d = w_pref.shape
        self.max_batch = max_batch
        self.handle = tfe.tfe_head_create(w_pref, self.V, self.d, max_batch)

    def close(self):
        if getattr(self, "handle", 0):
            tfe.tfe_head_destroy(self.handle)
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:       # interpreter shutdown: the binding may be gone already
            pass

    def topk(self, hidden: torch.Tensor, K: int, stream=None):
        """(tokens int32 [B, K], prob float32 [B, K]) on the device."""
        assert hidden.is_cuda and hidden.dtype == torch.bfloat16 and hidden.is_contiguous()
        B = hidden.shape[0]
        tokens = torch.empty((B, K), dtype=torch.int32, device=hidden.device)
        prob = torch.empty((B, K), dtype=torch.float32, device=hidden.device)
        tfe.tfe_head_topk(self.handle, hidden, B, K, tokens, prob, stream)
        return tokens, prob

    def logits(self, B: int) -> torch.Tensor:
        """fp32 [B, V] copy of the logits of the most recent call (synchronises)."""
        addr, ld, _ = tfe.tfe_head_buffers(self.handle)
        torch.cuda.synchronize()
        return _device_view(addr, (B, ld), "<f4", self.w.device)[:, :self.V].clone()

    def lse(self, B: int) -> torch.Tensor:
        _, _, addr = tfe.tfe_head_buffers(self.handle)
        torch.cuda.synchronize()
        return _device_view(addr, (B,), "<f4", self.w.device).clone()

    def status(self) -> int:
        return tfe.tfe_head_status(self.handle)


class _DevicePointer:
    def __init__(self, ptr, shape, typestr):
        self.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": typestr, "data": (ptr, False), "version": 2}


def _device_view(ptr: int, shape, typestr: str, device) -> torch.Tensor:
    """A tensor over library-owned device memory (no copy, no ownership)."""
    return torch.as_tensor(_DevicePointer(ptr, shape, typestr), device=device)


class MinedPhrases:
    """Result of mine_ngrams: device tensors cut to the entries written, plus the host-side totals."""

    def __init__(self, tokens, length, count, n_found, distinct, hist):
        self.phrase_tokens, self.phrase_len, self.count = tokens, length, count
        self.n_found, self.distinct, self.hist = n_found, distinct, hist

    def __len__(self):
        return self.phrase_len.numel()


def mine_ngrams(corpus: torch.Tensor, *, vocab: int, orders, min_count: int = 2, cap: int, want_hist: bool = True,
                workspace: torch.Tensor | None = None, stream=None) -> MinedPhrases:
    """Every n-gram of `corpus` (device int32 [L]) that occurs at least `min_count` times, in order of first
    occurrence; `count` holds uint32 values in an int32 tensor.  The result feeds Engram(device_build=True).
    `workspace`: a device uint8 tensor of tfe_mine_workspace_bytes(L, n_orders) bytes kept by the caller across
    calls (None: the library allocates and frees its own)."""
    assert corpus.is_cuda and corpus.dtype == torch.int32 and corpus.is_contiguous()
    dev = corpus.device
    pt = torch.empty((max(cap, 1), 4), dtype=torch.int32, device=dev)
    pl = torch.empty(max(cap, 1), dtype=torch.uint8, device=dev)
    pc = torch.empty(max(cap, 1), dtype=torch.int32, device=dev)
    n_found, distinct, hist = tfe.tfe_mine_ngrams(corpus, corpus.numel(), vocab, orders, min_count, cap, pt, pl, pc,
                                                  want_hist=want_hist, workspace=workspace,
                                                  workspace_bytes=0 if workspace is None else workspace.numel(),
                                                  stream=stream)
    n = min(n_found, cap)
    return MinedPhrases(pt[:n], pl[:n], pc[:n], n_found, distinct, hist)


def assign_residency(count: torch.Tensor, gpu_slots: int, host_min_count: int = 2, stream=None):
    """(init_slot int32 [N] on the device, (n_gpu, n_host, n_ssd)): the gpu_slots most frequent phrases start in
    the GPU tier (equal counts: smaller id first; slots in id order), the rest is tagged host or SSD by count."""
    assert count.is_cuda and count.dtype == torch.int32 and count.is_contiguous()
    init_slot = torch.empty(max(count.numel(), 1), dtype=torch.int32, device=count.device)
    tiers = tfe.tfe_assign_residency(count, count.numel(), gpu_slots, host_min_count, init_slot, stream)
    return init_slot[:count.numel()], tiers


# ---- rows of logits ----------------------------------------------------------------------------

_ROW_DTYPES = {torch.bfloat16: tfe.DTYPE_BF16, torch.float32: tfe.DTYPE_F32}
_SIZE_MAX = (1 << 31) - 1           # ctypes cuts a larger size to its low 32 bits


def _require(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


@contextlib.contextmanager
def _elsewhere(device: torch.device, stream):
    """The operands' device made current and, with a stream given, results allocated for that stream."""
    with torch.cuda.device(device):
        if stream is None:
            yield
        else:
            with torch.cuda.stream(torch.cuda.ExternalStream(stream, device) if isinstance(stream, int) else stream):
                yield


# A decode step makes the calls below by the thousand: checks build their messages only when they fail, and the common case
# of the current device and stream goes without a context.


def _here(device: torch.device, stream) -> bool:
    return stream is None and device.index == torch.cuda.current_device()


def _where(device: torch.device, stream) -> int:
    return tfe.current_stream_address(device.index) if stream is None else tfe._stream(stream)


def _row_matrix(t: torch.Tensor, what: str):
    """(rows, columns, elements between rows, the library's type number) of a 2-D CUDA matrix with contiguous rows."""
    kind = _ROW_DTYPES.get(t.dtype)
    if kind is None or not t.is_cuda or t.dim() != 2:
        raise ValueError(f"{what}: a 2-D bf16 or fp32 CUDA tensor is needed")
    n, v = t.shape
    if (n | v) > _SIZE_MAX:
        raise ValueError(f"{what}: more than 2^31 - 1 rows or columns")
    ld, step = t.stride()
    if v < 1 or (step != 1 and v != 1):
        raise ValueError(f"{what}: rows must be contiguous and not empty")
    if n <= 1:
        ld = v
    elif ld < v:
        raise ValueError(f"{what}: rows must not overlap")
    return n, v, ld, kind


def _vector(t: torch.Tensor, shape, dtype, device, what: str) -> int:
    """The address of a contiguous tensor of this shape, type and device."""
    if t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous {dtype} tensor of shape {tuple(shape)} on {device} is needed")
    return t.data_ptr()


def _written(out: torch.Tensor):
    """Tells autograd that the caller's tensor has new contents, as torch's own in-place operations do."""
    if not out.is_inference():
        torch.autograd.graph.increment_version(out)


def quantize_fp8(x: torch.Tensor, block_rows: int = 1, *, stream=None):
    """(q float8_e4m3fn [R, C], scale float32): `x` [R, C] in 8 bits with a scale for every `block_rows` x 128 values -- 1
    for activations, 128 for weights (see tfe_quantize_fp8).  q's rows start on 16-byte boundaries, as matmul_fp8 takes them: where
    C is not a multiple of 16 they lie that much further apart."""
    if not _here(x.device, stream):
        with _elsewhere(x.device, stream):
            return _quantize_fp8(x, block_rows, stream)
    return _quantize_fp8(x, block_rows, None)


def _quantize_fp8(x, block_rows, stream):
    r, c, ld, kind = _row_matrix(x, "x")
    if block_rows != 1 and block_rows != 128:
        raise ValueError("block_rows: 1 or 128")
    dev = x.device
    pitch = (c + 15) & ~15
    q = torch.empty_strided((r, c), (pitch, 1), dtype=torch.float8_e4m3fn, device=dev)
    scale = torch.empty(-(-r // block_rows), -(-c // 128), dtype=torch.float32, device=dev)
    tfe.tfe_quantize_fp8_ld(x.data_ptr(), kind, r, c, ld, block_rows, q.data_ptr(), pitch, scale.data_ptr(), _where(dev, stream))
    return q, scale


def _fp8_matrix(t: torch.Tensor, what: str):
    if not t.is_cuda or t.dim() != 2 or t.dtype != torch.float8_e4m3fn:
        raise ValueError(f"{what}: a 2-D float8_e4m3fn CUDA tensor is needed")
    n, k = t.shape
    if (n | k) > _SIZE_MAX:
        raise ValueError(f"{what}: more than 2^31 - 1 rows or columns")
    ld, step = t.stride()
    if n <= 1:
        ld = -(-k // 16) * 16
    if k < 1 or (step != 1 and k != 1) or ld < k or ld % 16 != 0 or t.data_ptr() % 16 != 0:
        raise ValueError(f"{what}: contiguous rows that start on 16-byte boundaries are needed")
    return n, k, ld


def matmul_fp8(a: torch.Tensor, a_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, *,
               out_dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """a [M, K] times the transpose of w [N, K], both as quantize_fp8 makes them (block_rows 1 and 128): [M, N] in fp32 or
    bf16 (see tfe_matmul_fp8).  `out`: where it goes instead of a new tensor.  A product that fails on the device leaves NaN in
    what it did not finish; matmul_fp8_status() tells."""
    if not _here(a.device, stream):
        with _elsewhere(a.device, stream):
            return _matmul_fp8(a, a_scale, w, w_scale, out_dtype, out, stream)
    return _matmul_fp8(a, a_scale, w, w_scale, out_dtype, out, None)


def _matmul_fp8(a, a_scale, w, w_scale, out_dtype, out, stream):
    m, k, lda = _fp8_matrix(a, "a")
    n, kw, ldw = _fp8_matrix(w, "w")
    dev = a.device
    if n < 1 or kw != k or w.device != dev:
        raise ValueError("w: the width and device of a are needed")
    kb = -(-k // 128)
    a_s = _vector(a_scale, (m, kb), torch.float32, dev, "a_scale")
    w_s = _vector(w_scale, (-(-n // 128), kb), torch.float32, dev, "w_scale")
    given = out
    if given is None:
        if out_dtype not in _ROW_DTYPES:
            raise ValueError("out_dtype: bfloat16 or float32")
        out = torch.empty(m, n, dtype=out_dtype, device=dev)
        ldo, kind = n, _ROW_DTYPES[out_dtype]
    else:
        om, on, ldo, kind = _row_matrix(out, "out")
        if om != m or on != n or out.device != dev:
            raise ValueError("out: [M, N] on the operands' device is needed")
        at, end = out.data_ptr(), out.data_ptr() + ((m - 1) * ldo + n) * out.element_size()
        for start, size in ((a.data_ptr(), (m - 1) * lda + k), (w.data_ptr(), (n - 1) * ldw + k), (a_s, 4 * m * kb), (w_s, 4 * w_scale.numel())):
            if m and at < start + size and start < end:
                raise ValueError("out: must not touch the operands")
    tfe.tfe_matmul_fp8(a.data_ptr(), lda, a_s, m, w.data_ptr(), ldw, w_s, n, k, out.data_ptr(), kind, ldo, _where(dev, stream))
    if given is not None:
        _written(out)
    return out


def matmul_fp8_status(stream=None) -> int:
    """0, or the device's status word if a product on it failed since the last report, which clears it (see
    tfe_matmul_fp8_status).  Synchronises."""
    return tfe.tfe_matmul_fp8_status(stream)


class QuantizedHead:
    """The vocabulary projection in 8 bits: half the bytes of EarlyExitHead's weights to read per call, logits instead of a
    top-K.  ``w``: bf16 or fp32 [V, d], d a multiple of 16; it is converted once and not kept."""

    def __init__(self, w: torch.Tensor):
        _require(w.dim() == 2 and w.shape[1] % 16 == 0, "w: [V, d] with d a multiple of 16 is needed")
        self.V, self.d = w.shape
        self.w, self.w_scale = quantize_fp8(w, block_rows=128)

    def logits(self, hidden: torch.Tensor, out_dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None, *,
               stream=None) -> torch.Tensor:
        """[B, V] logits of `hidden` [B, d], whose rows are converted within the call."""
        if hidden.dim() != 2 or hidden.shape[1] != self.d:
            raise ValueError(f"hidden: [B, {self.d}] is needed")
        if not _here(hidden.device, stream):
            with _elsewhere(hidden.device, stream):
                return self.logits(hidden, out_dtype, out)
        q, scale = quantize_fp8(hidden, 1)
        return matmul_fp8(q, scale, self.w, self.w_scale, out_dtype=out_dtype, out=out)

    def sample(self, hidden: torch.Tensor, u: torch.Tensor, *, stream=None, **settings):
        """(token, prob) of one draw per row of `hidden` by `u` (see sample_tokens for the settings)."""
        if not _here(hidden.device, stream):
            with _elsewhere(hidden.device, stream):
                return self.sample(hidden, u, **settings)
        return sample_tokens(self.logits(hidden), u, **settings)

    def status(self) -> int:
        """matmul_fp8_status on the weights' device."""
        with torch.cuda.device(self.w.device):
            return matmul_fp8_status()


def sample_tokens(logits: torch.Tensor, u: torch.Tensor, *, temperature: torch.Tensor | None = None,
                  top_k: torch.Tensor | None = None, top_p: torch.Tensor | None = None, min_p: torch.Tensor | None = None,
                  stream=None):
    """(token int32 [B], prob float32 [B]): one draw per row of `logits` [B, V] by the numbers `u` [B] in [0, 1), after
    temperature, min-p, top-k and top-p (see tfe_sample_tokens).  The settings are device tensors of B values
    (top_k int32, the others fp32) or None."""
    if not _here(logits.device, stream):
        with _elsewhere(logits.device, stream):
            return _sample_tokens(logits, u, temperature, top_k, top_p, min_p, stream)
    return _sample_tokens(logits, u, temperature, top_k, top_p, min_p, None)


def _sample_tokens(logits, u, temperature, top_k, top_p, min_p, stream):
    b, v, ld, kind = _row_matrix(logits, "logits")
    dev = logits.device
    shape, f32 = (b,), torch.float32
    ua = _vector(u, shape, f32, dev, "u")
    t = None if temperature is None else _vector(temperature, shape, f32, dev, "temperature")
    k = None if top_k is None else _vector(top_k, shape, torch.int32, dev, "top_k")
    p = None if top_p is None else _vector(top_p, shape, f32, dev, "top_p")
    m = None if min_p is None else _vector(min_p, shape, f32, dev, "min_p")
    token = torch.empty(b, dtype=torch.int32, device=dev)
    prob = u.new_empty(b)
    tfe.tfe_sample_tokens(logits.data_ptr(), kind, b, v, ld, ua, token.data_ptr(), prob.data_ptr(),
                          temperature=t, top_k=k, top_p=p, min_p=m, stream=_where(dev, stream))
    return token, prob


def _teacher(logits, teacher_ids, teacher_logits):
    n, v, ld, kind = _row_matrix(logits, "logits")
    _require(teacher_ids.dim() == 2, "teacher_ids: [rows, K] is needed")
    shape = (n, teacher_ids.shape[1])
    ids = _vector(teacher_ids, shape, torch.int32, logits.device, "teacher_ids")
    t = _vector(teacher_logits, shape, torch.float32, logits.device, "teacher_logits")
    return (logits.data_ptr(), kind, n, v, ld, ids, t, shape[1])


def distill_forward(logits: torch.Tensor, teacher_ids: torch.Tensor, teacher_logits: torch.Tensor, tau: float = 1.0, *,
                    stream=None):
    """(loss, lse), fp32 [N] each: the divergence from the teacher's top logits to the rows of `logits` [N, V] (see
    tfe_distill_forward), and the log-sum-exp of logits / tau that the gradient needs."""
    if not _here(logits.device, stream):
        with _elsewhere(logits.device, stream):
            return _distill_forward(logits, teacher_ids, teacher_logits, tau, stream)
    return _distill_forward(logits, teacher_ids, teacher_logits, tau, None)


def _distill_forward(logits, teacher_ids, teacher_logits, tau, stream):
    rows = _teacher(logits, teacher_ids, teacher_logits)
    dev, n = logits.device, rows[2]
    loss, lse = teacher_logits.new_empty(n), teacher_logits.new_empty(n)
    tfe.tfe_distill_forward(*rows, tau, loss.data_ptr(), lse.data_ptr(), _where(dev, stream))
    return loss, lse


def distill_backward(grad_loss: torch.Tensor, logits: torch.Tensor, teacher_ids: torch.Tensor,
                     teacher_logits: torch.Tensor, lse: torch.Tensor, tau: float = 1.0, *,
                     out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The gradient [N, V] of sum(grad_loss * loss) with respect to the logits.  `out`: where it goes, of the logits'
    shape and type; `out=logits` overwrites them."""
    if not _here(logits.device, stream):
        with _elsewhere(logits.device, stream):
            return _distill_backward(grad_loss, logits, teacher_ids, teacher_logits, lse, tau, out, stream)
    return _distill_backward(grad_loss, logits, teacher_ids, teacher_logits, lse, tau, out, None)


def _distill_backward(grad_loss, logits, teacher_ids, teacher_logits, lse, tau, out, stream):
    rows = _teacher(logits, teacher_ids, teacher_logits)
    dev, kind, n, v = logits.device, rows[1], rows[2], rows[3]
    g = _vector(grad_loss, (n,), torch.float32, dev, "grad_loss")
    norm = _vector(lse, (n,), torch.float32, dev, "lse")
    given = out
    if given is None:
        out, ld_out = logits.new_empty(n, v), v
    else:
        on, ov, ld_out, out_kind = _row_matrix(out, "out")
        if on != n or ov != v or out_kind != kind or out.device != dev:
            raise ValueError("out: the logits' shape, type and device are needed")
    tfe.tfe_distill_backward(*rows, tau, norm, g, out.data_ptr(), ld_out, _where(dev, stream))
    if given is not None:
        _written(out)
    return out


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, teacher_ids, teacher_logits, tau):
        loss, lse = distill_forward(logits, teacher_ids, teacher_logits, tau)
        ctx.save_for_backward(logits, teacher_ids, teacher_logits, lse)
        ctx.tau = tau
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss):
        logits, ids, t, lse = ctx.saved_tensors
        return distill_backward(grad_loss.contiguous(), logits, ids, t, lse, ctx.tau), None, None, None


def distill_loss(logits: torch.Tensor, teacher_ids: torch.Tensor, teacher_logits: torch.Tensor, tau: float = 1.0) -> torch.Tensor:
    """distill_forward's loss [N] as a node of autograd: the gradient goes to the logits, none to the teacher.  Reduce it
    as the training wants, e.g. ``(distill_loss(z, ids, t) * weight).sum()``."""
    return _DistillLoss.apply(logits, teacher_ids, teacher_logits, tau)
