"""The operators around the MoE layer (second part of include/moev.h) on torch tensors.

Like the rest of the package these functions check and marshal arguments; every step runs in the
library's kernels, asynchronously on torch's current stream.  A call whose tensors do not fit raises
:class:`MoevError` (``MOEV_EINVAL``) before anything is launched.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import (ACT_BF16, ACT_FP32, ACTQ_NONE, W_INT4, W_MXFP4, MoevError, _DraftBatch, _KvCache, _Linear, _Norm, lib)

_AFMT = {torch.bfloat16: ACT_BF16, torch.float32: ACT_FP32}
_EINVAL = 1
_raw_stream = torch._C._cuda_getCurrentRawStream


def _bad(text: str):
    raise MoevError(_EINVAL, text)


def _stream(t: torch.Tensor) -> int:
    """Raw handle of the current stream; the kernels run on the current device."""
    dev = t.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        _bad(f"tensors must be on the current CUDA device, got {t.device}")
    return _raw_stream(dev)


def _same_device(first: torch.Tensor, *others):
    dev = first.get_device()
    for t in others:
        if t is not None and t.get_device() != dev:
            _bad(f"tensors on different devices: {first.device} and {t.device}")


def _rows(t: torch.Tensor, name: str, n: int, width: int, dtype) -> int:
    """Row stride of a tensor whose first dimension is rows and whose others are contiguous (``width`` elements)."""
    if t.dtype != dtype or t.dim() < 2 or t.shape[0] != n or t.numel() != n * width:
        _bad(f"{name}: expected {n} rows of {width} {dtype}, got {tuple(t.shape)} {t.dtype}")
    step = 1
    for size, stride in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if size != 1 and stride != step:
            _bad(f"{name}: everything behind the first dimension must be contiguous, got strides {t.stride()}")
        step *= size
    return t.stride(0) if n > 1 else width


def add_rmsnorm(x: torch.Tensor, weight: torch.Tensor, out: dict, residual: torch.Tensor = None, eps: float = 1e-6,
                act_quant: int = ACTQ_NONE) -> dict:
    """moev_add_rmsnorm: ``out`` maps "y" / "residual" / "codes" / "scales" to the tensors that are wanted
    (codes uint8 or float8_e4m3fn [n, H] and scales float32 [n, ceil(H / 128)] exactly with ``act_quant``)."""
    if x.dim() != 2 or x.dtype not in _AFMT:
        _bad(f"x: expected a bfloat16 or float32 matrix, got {tuple(x.shape)} {x.dtype}")
    n, H = x.shape
    y, ro, codes, scales = out.get("y"), out.get("residual"), out.get("codes"), out.get("scales")
    _same_device(x, weight, residual, y, ro, codes, scales)
    if weight.dtype not in _AFMT or weight.shape != (H,) or not weight.is_contiguous():
        _bad(f"weight: expected {H} contiguous bfloat16 or float32 values")
    p = _Norm(n=n, H=H, afmt=_AFMT[x.dtype], wfmt=_AFMT[weight.dtype], eps=eps, act_quant=act_quant, x=x.data_ptr(), w=weight.data_ptr(),
              x_stride=_rows(x, "x", n, H, x.dtype))
    if residual is not None:
        p.residual, p.residual_stride = residual.data_ptr(), _rows(residual, "residual", n, H, x.dtype)
    if y is not None:
        p.y, p.y_stride = y.data_ptr(), _rows(y, "y", n, H, x.dtype)
    if ro is not None:
        p.residual_out, p.residual_out_stride = ro.data_ptr(), _rows(ro, "out residual", n, H, x.dtype)
    if codes is not None:
        if codes.dtype not in (torch.uint8, torch.float8_e4m3fn):
            _bad(f"codes: expected uint8 or float8_e4m3fn, got {codes.dtype}")
        p.codes, p.codes_stride = codes.data_ptr(), _rows(codes, "codes", n, H, codes.dtype)
    if scales is not None:
        if scales.dtype != torch.float32 or scales.shape != (n, (H + 127) // 128) or not scales.is_contiguous():
            _bad(f"scales: expected contiguous float32 [{n}, {(H + 127) // 128}]")
        p.scales = scales.data_ptr()
    st = lib().moev_add_rmsnorm(C.byref(p), _stream(x))
    if st != 0:
        raise MoevError(st, "moev_add_rmsnorm rejected the call")
    return out


class W4Linear:
    """A 4-bit weight laid out for the kernel, once: ``codes`` uint8 [N, K / 2]; ``scales`` bfloat16 [N, K / group]
    (``W_INT4``) or uint8 [N, K / 32] (``W_MXFP4``); ``bias`` float32 [N] or None.  ``codes`` and ``scales`` are not kept."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, wfmt: int = W_INT4, group: int = 32, bias: torch.Tensor = None):
        if codes.dtype != torch.uint8 or codes.dim() != 2 or not codes.is_contiguous():
            _bad(f"codes: expected contiguous uint8 [N, K / 2], got {tuple(codes.shape)} {codes.dtype}")
        N, K = codes.shape[0], codes.shape[1] * 2
        self.N, self.K, self.wfmt, self.group = N, K, wfmt, group
        self._c = _Linear(N, K, wfmt, group)
        size = lib().moev_w4_packed_bytes(C.byref(self._c))
        if size == 0:
            _bad(f"no 4-bit linear layer of N={N}, K={K}, wfmt={wfmt}, group={group}")
        want = torch.uint8 if wfmt == W_MXFP4 else torch.bfloat16
        if scales.dtype != want or scales.shape != (N, K // group) or not scales.is_contiguous():
            _bad(f"scales: expected contiguous {want} [{N}, {K // group}], got {tuple(scales.shape)} {scales.dtype}")
        if bias is not None and (bias.dtype != torch.float32 or bias.shape != (N,) or not bias.is_contiguous()):
            _bad(f"bias: expected contiguous float32 [{N}]")
        _same_device(codes, scales, bias)
        self.bias = bias
        stream = _stream(codes)
        self.packed = torch.empty(size, dtype=torch.uint8, device=codes.device)
        st = lib().moev_w4_pack(C.byref(self._c), codes.data_ptr(), scales.data_ptr(), self.packed.data_ptr(), stream)
        if st != 0:
            raise MoevError(st, "moev_w4_pack rejected the weight")
        self._ref = C.byref(self._c)
        self._packed_ptr = self.packed.data_ptr()
        self._bias_ptr = None if bias is None else bias.data_ptr()
        self._dev = codes.get_device()

    def __call__(self, x: torch.Tensor, y: torch.Tensor = None) -> torch.Tensor:
        """moev_linear_w4: x bfloat16 [n, K] -> y bfloat16 or float32 [n, N] (allocated as bfloat16 when not given)."""
        n = x.shape[0]
        if y is None:
            y = torch.empty(n, self.N, dtype=torch.bfloat16, device=x.device)
        if y.dtype not in _AFMT:
            _bad(f"y: expected bfloat16 or float32, got {y.dtype}")
        if x.get_device() != self._dev or y.get_device() != self._dev:
            _bad(f"x and y must be on the weight's device cuda:{self._dev}")
        st = lib().moev_linear_w4(self._ref, self._packed_ptr, self._bias_ptr, x.data_ptr(), _rows(x, "x", n, self.K, torch.bfloat16), n,
                                  y.data_ptr(), _rows(y, "y", n, self.N, y.dtype), _AFMT[y.dtype], _stream(x))
        if st != 0:
            raise MoevError(st, "moev_linear_w4 rejected the call")
        return y


class KvCache:
    """Paged 8-bit cache over the caller's tensors: k [pages, heads, page, D] and v [pages, heads, D, page] in uint8
    or float8_e4m3fn, k_scale and v_scale float32 [pages, heads]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        if k.dim() != 4 or v.dim() != 4 or k.shape[:2] != v.shape[:2] or k.shape[2:] != (v.shape[3], v.shape[2]):
            _bad(f"k and v: expected [pages, heads, page, D] and [pages, heads, D, page], got {tuple(k.shape)} and {tuple(v.shape)}")
        for name, t in (("k", k), ("v", v)):
            if t.dtype not in (torch.uint8, torch.float8_e4m3fn) or not t.is_contiguous():
                _bad(f"{name}: expected contiguous uint8 or float8_e4m3fn, got {t.dtype}")
        n, heads, page, D = k.shape
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            if t.dtype != torch.float32 or t.shape != (n, heads) or not t.is_contiguous():
                _bad(f"{name}: expected contiguous float32 [{n}, {heads}]")
        _same_device(k, v, k_scale, v_scale)
        if page not in (16, 32, 64, 128) or D not in (64, 128):
            _bad(f"pages of {page} tokens and heads of {D} dimensions are not served (16, 32, 64, 128; 64, 128)")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.n_kv_heads, self.page, self.head_dim = n, heads, page, D
        self._c = _KvCache(n, page, heads, D, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())
        self._ref = C.byref(self._c)

    @classmethod
    def empty(cls, n_pages: int, page: int, n_kv_heads: int, head_dim: int, device="cuda") -> "KvCache":
        k = torch.zeros(n_pages, n_kv_heads, page, head_dim, dtype=torch.uint8, device=device)
        v = torch.zeros(n_pages, n_kv_heads, head_dim, page, dtype=torch.uint8, device=device)
        return cls(k, v, torch.ones(n_pages, n_kv_heads, device=device), torch.ones(n_pages, n_kv_heads, device=device))


class DraftBatch:
    """The drafts of one call (moev_draft_batch): int32 tensors cu [n_seq + 1], ctx_len [n_seq], page_table [n_seq, cols],
    parent [n_tokens] or None for chains; max_drafts and max_len bound every sequence.  The tensors are the caller's and
    may be rewritten between calls.  ``status`` (int32 [1], optional) collects what the kernels reject."""

    def __init__(self, cu: torch.Tensor, ctx_len: torch.Tensor, page_table: torch.Tensor, max_drafts: int, max_len: int,
                 parent: torch.Tensor = None, status: torch.Tensor = None):
        n = ctx_len.numel()
        if page_table.dim() != 2 or page_table.shape[0] != n or cu.numel() != n + 1:
            _bad(f"cu, ctx_len and page_table disagree about the number of sequences: {cu.numel()}, {n}, {tuple(page_table.shape)}")
        for name, t in (("cu", cu), ("ctx_len", ctx_len), ("page_table", page_table), ("parent", parent), ("status", status)):
            if t is not None and (t.dtype != torch.int32 or not t.is_contiguous()):
                _bad(f"{name}: expected a contiguous int32 tensor")
        _same_device(cu, ctx_len, page_table, parent, status)
        self.cu, self.ctx_len, self.page_table, self.parent, self.status = cu, ctx_len, page_table, parent, status
        self.max_drafts, self.max_len = max_drafts, max_len
        self._c = _DraftBatch(n, 0, max_drafts, max_len, page_table.shape[1], cu.data_ptr(), ctx_len.data_ptr(), page_table.data_ptr(),
                              None if parent is None else parent.data_ptr(), None if status is None else status.data_ptr())
        self._ref = C.byref(self._c)

    def _for(self, n_tokens: int):
        if self.parent is not None and self.parent.numel() < n_tokens:
            _bad(f"parent has {self.parent.numel()} entries for {n_tokens} token rows")
        self._c.n_tokens = n_tokens
        return self._ref


def cache_append(cache: KvCache, batch: DraftBatch, k: torch.Tensor, v: torch.Tensor, rope: torch.Tensor = None, q: torch.Tensor = None,
                 q_out: torch.Tensor = None):
    """moev_cache_append: k, v bfloat16 [n_tokens, heads, D]; rope float32 [positions, D] (cosines, sines); q bfloat16
    [n_tokens, query heads, D], rotated into q_out (default: in place).  Returns q_out."""
    T, D, heads = k.shape[0], cache.head_dim, cache.n_kv_heads
    bf16 = torch.bfloat16
    n_heads, q_ptr, q_stride, o_ptr, o_stride = 0, None, 0, None, 0
    if q is not None:
        q_out = q if q_out is None else q_out
        n_heads = q.numel() // (T * D) if T else heads
        q_ptr, q_stride = q.data_ptr(), _rows(q, "q", T, n_heads * D, bf16)
        o_ptr, o_stride = q_out.data_ptr(), _rows(q_out, "q_out", T, n_heads * D, bf16)
    if rope is not None and (rope.dtype != torch.float32 or rope.dim() != 2 or rope.shape[1] != D or not rope.is_contiguous()):
        _bad(f"rope: expected contiguous float32 [positions, {D}]")
    _same_device(k, v, cache.k, batch.cu, rope, q, q_out)
    st = lib().moev_cache_append(cache._ref, batch._for(T), k.data_ptr(), _rows(k, "k", T, heads * D, bf16), v.data_ptr(),
                                 _rows(v, "v", T, heads * D, bf16), None if rope is None else rope.data_ptr(),
                                 0 if rope is None else rope.shape[0], q_ptr, q_stride, n_heads, o_ptr, o_stride, _stream(k))
    if st != 0:
        raise MoevError(st, "moev_cache_append rejected the call (alignment, strides, head counts or bounds)")
    return q_out


def cache_attend_workspace(cache: KvCache, batch: DraftBatch, n_heads: int, window: int = 0, n_tokens: int = None) -> torch.Tensor:
    """A workspace for cache_attend calls of this size (``n_tokens`` rows; by default one full tree per sequence)."""
    n = batch.ctx_len.numel() * batch.max_drafts if n_tokens is None else n_tokens
    batch._c.n_tokens = n
    size = lib().moev_cache_attend_workspace(cache._ref, batch._ref, n_heads, window)
    return torch.empty(size, dtype=torch.uint8, device=cache.k.device)


def cache_attend(cache: KvCache, batch: DraftBatch, q: torch.Tensor, out: torch.Tensor = None, lse: torch.Tensor = None, scale: float = None,
                 window: int = 0, sinks: torch.Tensor = None, workspace: torch.Tensor = None) -> torch.Tensor:
    """moev_cache_attend: q, out bfloat16 [n_tokens, query heads, D]; lse float32 [n_tokens, query heads]; sinks float32
    [query heads].  Without a workspace that is large enough, one is taken from torch's allocator for the call."""
    T, D = q.shape[0], cache.head_dim
    n_heads = q.numel() // (T * D) if T else cache.n_kv_heads
    if out is None:
        out = torch.zeros_like(q)
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != (T, n_heads) or not lse.is_contiguous()):
        _bad(f"lse: expected contiguous float32 [{T}, {n_heads}]")
    if sinks is not None and (sinks.dtype != torch.float32 or sinks.shape != (n_heads,) or not sinks.is_contiguous()):
        _bad(f"sinks: expected contiguous float32 [{n_heads}]")
    _same_device(q, cache.k, batch.cu, out, lse, sinks, workspace)
    b = batch._for(T)
    q_stride, o_stride = _rows(q, "q", T, n_heads * D, torch.bfloat16), _rows(out, "out", T, n_heads * D, torch.bfloat16)
    L = lib()
    size = L.moev_cache_attend_workspace(cache._ref, b, n_heads, window)
    if size and (workspace is None or workspace.numel() * workspace.element_size() < size):
        workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
    st = L.moev_cache_attend(cache._ref, b, q.data_ptr(), q_stride, n_heads, D ** -0.5 if scale is None else scale, window,
                             None if sinks is None else sinks.data_ptr(), out.data_ptr(), o_stride, None if lse is None else lse.data_ptr(),
                             workspace.data_ptr() if size else None, size, _stream(q))
    if st != 0:
        raise MoevError(st, "moev_cache_attend rejected the call (alignment, strides, head counts, scale or bounds)")
    return out
