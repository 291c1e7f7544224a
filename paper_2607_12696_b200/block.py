"""The operators around the MoE layer (second part of include/moev.h) on torch tensors.

Like the rest of the package these functions check and marshal arguments; every step runs in the
library's kernels, asynchronously on torch's current stream.  The checks are compiled
(``csrc/block_py.cpp``): a small call's kernels take less time than the same checks in Python.  A call
whose tensors do not fit raises :class:`MoevError` (``MOEV_EINVAL``) before anything is launched.
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass

import torch

from .binding import (_OUT_FIELDS, ACTQ_NONE, W_INT4, W_MXFP4, MoevError, _Block, _BlockOptions, _DraftBatch, _KvCache, _Layer, _Linear, _Out, _ptr,
                      lib)

_EINVAL = 1
_ext = None


def _fast():
    """The compiled checks (``_block``); like the library itself they have no fallback."""
    global _ext
    if _ext is None:
        lib()
        from . import _block
        _ext = _block
    return _ext


def _bad(text: str):
    raise MoevError(_EINVAL, text)


def _int32(**named):
    for name, v in named.items():
        if not -2 ** 31 <= v < 2 ** 31:
            _bad(f"{name}: {v} does not fit in 32 bits")


def _same_device(first: torch.Tensor, *others):
    for t in others:
        if t is not None and t.device != first.device:
            _bad(f"tensors on different devices: {first.device} and {t.device}")


def add_rmsnorm(x: torch.Tensor, weight: torch.Tensor, out: dict, residual: torch.Tensor = None, eps: float = 1e-6,
                act_quant: int = ACTQ_NONE) -> dict:
    """moev_add_rmsnorm: ``out`` maps "y" / "residual" / "codes" / "scales" to the tensors that are wanted
    (codes uint8 or float8_e4m3fn [n, H] and scales float32 [n, ceil(H / 128)] exactly with ``act_quant``)."""
    get = out.get
    (_ext or _fast()).add_rmsnorm(x, weight, residual, get("y"), get("residual"), get("codes"), get("scales"), eps, act_quant)
    return out


class W4Linear:
    """A 4-bit weight laid out for the kernel, once: ``codes`` uint8 [N, K / 2]; ``scales`` bfloat16 [N, K / group]
    (``W_INT4``) or uint8 [N, K / 32] (``W_MXFP4``); ``bias`` float32 [N] or None.  ``codes`` and ``scales`` are not kept."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, wfmt: int = W_INT4, group: int = 32, bias: torch.Tensor = None):
        if codes.dtype != torch.uint8 or codes.dim() != 2 or not codes.is_contiguous():
            _bad(f"codes: expected contiguous uint8 [N, K / 2], got {tuple(codes.shape)} {codes.dtype}")
        N, K = codes.shape[0], codes.shape[1] * 2
        self.N, self.K, self.wfmt, self.group = N, K, wfmt, group
        _int32(N=N, K=K, wfmt=wfmt, group=group)
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
        dev = codes.get_device()
        if dev < 0 or dev != torch.cuda.current_device():
            _bad(f"tensors must be on the current CUDA device, got {codes.device}")
        self.bias = bias
        self.packed = torch.empty(size, dtype=torch.uint8, device=codes.device)
        st = lib().moev_w4_pack(C.byref(self._c), codes.data_ptr(), scales.data_ptr(), self.packed.data_ptr(),
                                C.c_void_p(torch.cuda.current_stream().cuda_stream))
        if st != 0:
            raise MoevError(st, "moev_w4_pack rejected the weight")
        self._address()

    def _address(self):
        self._args = (C.addressof(self._c), self.packed.data_ptr(), 0 if self.bias is None else self.bias.data_ptr(), self.packed.get_device())

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k not in ("_c", "_args")}

    def __setstate__(self, state):  # a copy has addresses of its own
        self.__dict__.update(state)
        self._c = _Linear(self.N, self.K, self.wfmt, self.group)
        self._address()

    def __call__(self, x: torch.Tensor, y: torch.Tensor = None) -> torch.Tensor:
        """moev_linear_w4: x bfloat16 [n, K] -> y bfloat16 or float32 [n, N] (allocated as bfloat16 when not given)."""
        return (_ext or _fast()).linear_w4(*self._args, x, y)


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
        _int32(pages=n, heads=heads)
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            if t.dtype != torch.float32 or t.shape != (n, heads) or not t.is_contiguous():
                _bad(f"{name}: expected contiguous float32 [{n}, {heads}]")
        _same_device(k, v, k_scale, v_scale)
        if page not in (16, 32, 64, 128) or D not in (64, 128):
            _bad(f"pages of {page} tokens and heads of {D} dimensions are not served (16, 32, 64, 128; 64, 128)")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.n_kv_heads, self.page, self.head_dim = n, heads, page, D
        self._c = _KvCache(n, page, heads, D, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())
        self._at = C.addressof(self._c)
        self._dev = k.get_device()

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
        _int32(sequences=n, max_drafts=max_drafts, max_len=max_len, columns=page_table.shape[1])
        self._c = _DraftBatch(n, 0, max_drafts, max_len, page_table.shape[1], cu.data_ptr(), ctx_len.data_ptr(), page_table.data_ptr(),
                              None if parent is None else parent.data_ptr(), None if status is None else status.data_ptr())
        self._at = C.addressof(self._c)
        self._parents = 0 if parent is None else parent.numel()
        self._dev = cu.get_device()


def _together(cache: KvCache, batch: DraftBatch):
    if cache._dev != batch._dev:
        _bad(f"cache and batch on different devices: {cache.k.device} and {batch.cu.device}")


def cache_append(cache: KvCache, batch: DraftBatch, k: torch.Tensor, v: torch.Tensor, rope: torch.Tensor = None, q: torch.Tensor = None,
                 q_out: torch.Tensor = None):
    """moev_cache_append: k, v bfloat16 [n_tokens, heads, D]; rope float32 [positions, D] (cosines, sines); q bfloat16
    [n_tokens, query heads, D], rotated into q_out (default: in place).  Returns q_out."""
    if cache._dev != batch._dev:
        _together(cache, batch)
    return (_ext or _fast()).cache_append(cache._at, batch._at, batch._parents, cache._dev, k, v, rope, q, q_out)


def cache_attend_workspace(cache: KvCache, batch: DraftBatch, n_heads: int, window: int = 0) -> torch.Tensor:
    """A workspace for cache_attend calls with these bounds (it does not depend on the number of token rows)."""
    _int32(n_heads=n_heads, window=window)
    size = lib().moev_cache_attend_workspace(C.byref(cache._c), C.byref(batch._c), n_heads, window)
    return torch.empty(size, dtype=torch.uint8, device=cache.k.device)


def cache_attend(cache: KvCache, batch: DraftBatch, q: torch.Tensor, out: torch.Tensor = None, lse: torch.Tensor = None, scale: float = None,
                 window: int = 0, sinks: torch.Tensor = None, workspace: torch.Tensor = None) -> torch.Tensor:
    """moev_cache_attend: q, out bfloat16 [n_tokens, query heads, D]; lse float32 [n_tokens, query heads]; sinks float32
    [query heads]; scale defaults to D ** -0.5.  Without a workspace that is large enough, one is taken from torch's
    allocator for the call."""
    if cache._dev != batch._dev:
        _together(cache, batch)
    if scale is None:
        scale = 0.0
    elif scale == 0.0:
        _bad("scale: expected a positive number")
    return (_ext or _fast()).cache_attend(cache._at, batch._at, batch._parents, cache._dev, q, out, lse, scale, window, sinks, workspace)


@dataclass
class Block:
    """One decoder block for :meth:`MoeVerifier.verify_blocks`: norm weights bfloat16 [H], the fused query / key / value
    projection and the output projection, the block's cache, its MoE layer (``binding.make_layer``)."""
    attn_norm: torch.Tensor
    qkv: W4Linear
    o: W4Linear
    cache: KvCache
    ffn_norm: torch.Tensor
    layer: _Layer
    window: int = 0
    sinks: torch.Tensor = None

    def _c(self, H: int, n_heads: int) -> _Block:
        for name, t in (("attn_norm", self.attn_norm), ("ffn_norm", self.ffn_norm)):
            if t.dtype != torch.bfloat16 or t.shape != (H,) or not t.is_contiguous():
                _bad(f"{name}: expected {H} contiguous bfloat16 values")
        if self.sinks is not None and (self.sinks.dtype != torch.float32 or self.sinks.shape != (n_heads,) or not self.sinks.is_contiguous()):
            _bad(f"sinks: expected contiguous float32 [{n_heads}]")
        _int32(window=self.window)
        return _Block(self.attn_norm.data_ptr(), self.ffn_norm.data_ptr(), self.qkv._c, self.o._c, self.qkv._args[1], self.o._args[1],
                      self.qkv._args[2], self.o._args[2], _ptr(self.sinks), self.window, self.cache._c, self.layer)


# outputs of the MoE layers beside y: type and least size for T token rows
_DIAGNOSTICS = (("n_active", lambda c, T: 1, torch.int32), ("topk_ids", lambda c, T: T * c.top_k, torch.int32),
                ("topk_w", lambda c, T: T * c.top_k, torch.float32), ("union_ids", lambda c, T: c.E, torch.int32),
                ("offsets", lambda c, T: c.E + 1, torch.int32), ("perm", lambda c, T: T * c.top_k, torch.int32))


def verify_blocks(verifier, blocks: list, batch: DraftBatch, hidden: torch.Tensor, n_heads: int, outs: list, rope: torch.Tensor = None,
                  eps: float = 1e-6, scale: float = None, final_norm: torch.Tensor = None, final_out: torch.Tensor = None,
                  workspace: torch.Tensor = None):
    """moev_verify_blocks: ``hidden`` bfloat16 [n_tokens, H] is the residual stream before the first block and becomes the one
    after the last; ``outs[l]`` (``MoeVerifier.alloc_out``) receives block l's MoE outputs; with ``final_norm`` the normed
    stream goes to ``final_out``.  Returns the workspace, which a next call of the same size may be given."""
    H = verifier.cfg.H
    if hidden.dtype != torch.bfloat16 or hidden.dim() != 2 or hidden.shape[1] != H or not hidden.is_contiguous():
        _bad(f"hidden: expected contiguous bfloat16 [n_tokens, {H}], got {tuple(hidden.shape)} {hidden.dtype}")
    T, n = hidden.shape[0], len(blocks)
    _int32(token_rows=T, n_heads=n_heads, positions=0 if rope is None else rope.shape[0])
    if len(outs) != n or not n:
        _bad(f"{n} blocks and {len(outs)} outputs")
    if batch.parent is not None and batch._parents < T:
        _bad(f"parent has {batch._parents} entries for {T} token rows")
    D = blocks[0].cache.head_dim
    if rope is not None and (rope.dtype != torch.float32 or rope.dim() != 2 or rope.shape[1] != D or not rope.is_contiguous()):
        _bad(f"rope: expected contiguous float32 [positions, {D}]")
    if any(b.cache.head_dim != D for b in blocks):
        _bad("blocks with heads of different sizes need a call each")
    if scale is not None and scale == 0.0:  # to the C entry point: no scale given
        _bad("scale: expected a positive number")
    if (final_norm is None) != (final_out is None):
        _bad("final_norm and final_out go together")
    if final_norm is not None and (final_norm.dtype != torch.bfloat16 or final_norm.shape != (H,) or not final_norm.is_contiguous()
                                   or final_out.dtype != torch.bfloat16 or final_out.shape != (T, H) or not final_out.is_contiguous()):
        _bad(f"final_norm, final_out: expected contiguous bfloat16 [{H}] and [{T}, {H}]")
    _same_device(hidden, batch.cu, rope, final_norm, final_out, workspace, *[o.get(f) for o in outs for f in _OUT_FIELDS],
                 *[t for b in blocks for t in (b.cache.k, b.attn_norm, b.ffn_norm, b.sinks, b.qkv.packed, b.o.packed)])
    for o in outs:
        for f, size, dtype in _DIAGNOSTICS:
            t = o.get(f)
            if t is not None and (t.dtype != dtype or t.numel() < size(verifier.cfg, T) or not t.is_contiguous()):
                _bad(f"outs: {f} must be contiguous {dtype} of {size(verifier.cfg, T)} elements or more, got {tuple(t.shape)} {t.dtype}")
    if not hidden.is_cuda or hidden.get_device() != torch.cuda.current_device():
        _bad(f"tensors must be on the current CUDA device, got {hidden.device}")
    for o in outs:
        if o["y"].dtype != torch.bfloat16 or o["y"].shape[0] < T or o["y"].shape[1:] != (H,) or not o["y"].is_contiguous():
            _bad(f"outs: y must be contiguous bfloat16 [{T}, {H}]")
    BA = (_Block * n)(*[b._c(H, n_heads) for b in blocks])
    OA = (_Out * n)()
    for i, out in enumerate(outs):
        for f in _OUT_FIELDS:
            setattr(OA[i], f, _ptr(out.get(f)))
    d = _DraftBatch.from_buffer_copy(batch._c)
    d.n_tokens = T
    opt = _BlockOptions(n_heads, eps, 0.0 if scale is None else scale, _ptr(rope), 0 if rope is None else rope.shape[0], _ptr(final_norm), _ptr(final_out))
    size = lib().moev_verify_blocks_workspace(verifier._h, n, BA, C.byref(d), C.byref(opt))
    if size and (workspace is None or not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < size):
        workspace = torch.empty(size, dtype=torch.uint8, device=hidden.device)
    verifier._check(lib().moev_verify_blocks(verifier._h, n, BA, C.byref(d), C.byref(opt), hidden.data_ptr(), OA, _ptr(workspace), size, verifier._stream()))
    return workspace
