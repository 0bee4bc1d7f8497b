"""Thin ctypes binding of ``libhook_attn.so`` (declared in ``include/hook_attn.h``).

Argument marshalling only: every step of the path runs in the CUDA kernels.  PyTorch is used
for device memory and streams.  There is no CPU fallback -- if the compiled library is missing
the import of this module's entry points fails loudly.  The short calls around the attention are
marshalled by the compiled module ``_marshal`` (``csrc/marshal.cpp``), which calls the same library.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libhook_attn.so")

HOOK_ATTN_OK = 0
HOOK_ATTN_ERR_INVALID_ARG = -1
HOOK_ATTN_ERR_UNSUPPORTED = -2
HOOK_ATTN_ERR_WORKSPACE = -3
HOOK_ATTN_ERR_CUDA = -4
HOOK_ATTN_ERR_TIMEOUT = -5
HOOK_ATTN_ERR_BOUNDS = -6
HOOK_ATTN_ERR_NO_PAGES = -7
HOOK_PROBE_ROWS_ALL = 0
HOOK_PROBE_ROWS_LAST = 1

EXPORTS = ("hook_attn_create", "hook_attn_destroy", "hook_attn_workspace_bytes",
           "hook_attn_prefill", "hook_attn_decode", "hook_attn_mixed", "hook_attn_decode_static_scratch",
           "hook_attn_score", "hook_steer_residual", "hook_capture_qk", "hook_rope_append", "hook_adjust_logits",
           "hook_cache_fork", "hook_cache_extend", "hook_cache_free", "hook_cache_compact", "hook_cache_copy_pages",
           "hook_q4_slab_bytes", "hook_rope_append_q4", "hook_attn_decode_q4", "hook_cache_read_q4", "hook_cache_copy_pages_q4",
           "hook_sample_tokens", "hook_attn_selftest_wait_limit", "hook_attn_strerror")
HOOK_SCORE_MEAN = 0
HOOK_SCORE_SUM_NORMALIZE = 1
STATIC_SCRATCH_BYTES = 16 << 20   # HOOK_ATTN_STATIC_SCRATCH_BYTES
HOOK_DTYPE_BF16, HOOK_DTYPE_F16, HOOK_DTYPE_F32 = 0, 1, 2
HOOK_ROPE_AXES_BLOCKED, HOOK_ROPE_AXES_CYCLIC = 0, 1
HOOK_ROPE_PAIR_HALVES, HOOK_ROPE_PAIR_ADJACENT = 0, 1
HOOK_ROPE_MAX_AXES = 4
# Arguments between the handle and the stream: p an address, i an int32.
_AROUND = {"hook_rope_append": "p", "hook_adjust_logits": "p", "hook_cache_fork": "pppi", "hook_cache_extend": "ppp",
           "hook_cache_free": "pppi", "hook_cache_compact": "pppppp", "hook_cache_copy_pages": "p", "hook_rope_append_q4": "pp",
           "hook_attn_decode_q4": "pp", "hook_cache_read_q4": "pp", "hook_cache_copy_pages_q4": "p", "hook_sample_tokens": "p"}


class HookAttnParams(ctypes.Structure):
    """Mirror of ``hook_attn_params``."""
    _fields_ = [
        ("num_seqs", ctypes.c_int32), ("total_q", ctypes.c_int32),
        ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
        ("num_blocks", ctypes.c_int32), ("max_blocks_per_seq", ctypes.c_int32),
        ("num_spans", ctypes.c_int32), ("probe_rows", ctypes.c_int32),
        ("scale", ctypes.c_float), ("max_seq_len", ctypes.c_int32),
        ("q", ctypes.c_void_p), ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p),
        ("kv_block_stride", ctypes.c_int64), ("kv_token_stride", ctypes.c_int64),
        ("kv_head_stride", ctypes.c_int64),
        ("block_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p),
        ("cu_q_lens", ctypes.c_void_p), ("spans", ctypes.c_void_p),
        ("steer_vec", ctypes.c_void_p), ("out", ctypes.c_void_p),
        ("span_mass", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t), ("status", ctypes.c_void_p),
        ("head_mask", ctypes.c_void_p), ("alpha", ctypes.c_void_p),
    ]


def _fields(text: str, ctype) -> list:
    return [(name, ctype) for name in text.split()]


class HookRopeParams(ctypes.Structure):
    """Mirror of ``hook_rope_params``."""
    _fields_ = (
        _fields("num_seqs total_q num_q_heads num_kv_heads head_dim page_size num_blocks max_blocks_per_seq dtype rotary_dim num_axes",
                ctypes.c_int32)
        + [("axis_pairs", ctypes.c_int32 * HOOK_ROPE_MAX_AXES), ("axis_order", ctypes.c_int32), ("pairing", ctypes.c_int32),
           ("factor", ctypes.c_float)]
        + _fields("q k v", ctypes.c_void_p)
        + _fields("q_row_stride q_head_stride k_row_stride k_head_stride v_row_stride v_head_stride", ctypes.c_int64)
        + _fields("inv_freq positions", ctypes.c_void_p) + [("position_axis_stride", ctypes.c_int64)]
        + _fields("q_out k_cache v_cache", ctypes.c_void_p)
        + _fields("kv_block_stride kv_token_stride kv_head_stride", ctypes.c_int64)
        + _fields("block_table seq_lens cu_q_lens status", ctypes.c_void_p))


class HookLogitsParams(ctypes.Structure):
    """Mirror of ``hook_logits_params``."""
    _fields_ = (
        _fields("num_rows vocab_size max_tokens num_bias num_masks dtype out_dtype", ctypes.c_int32)
        + _fields("logits out", ctypes.c_void_p) + _fields("logits_row_stride out_row_stride", ctypes.c_int64)
        + [("tokens", ctypes.c_void_p), ("tokens_row_stride", ctypes.c_int64)]
        + _fields("prompt_lens total_lens repetition presence frequency bias_offsets bias_tokens bias_values mask", ctypes.c_void_p)
        + [("mask_row_stride", ctypes.c_int64)] + _fields("mask_rows status", ctypes.c_void_p))


class HookCachePool(ctypes.Structure):
    """Mirror of ``hook_cache_pool``."""
    _fields_ = (_fields("num_seqs max_blocks_per_seq num_blocks page_size", ctypes.c_int32)
                + _fields("block_table seq_lens page_refs status", ctypes.c_void_p))


class HookCacheCopyParams(ctypes.Structure):
    """Mirror of ``hook_cache_copy_params``."""
    _fields_ = (_fields("num_layers num_blocks page_size num_kv_heads head_dim max_pairs", ctypes.c_int32)
                + _fields("kv_block_stride kv_token_stride kv_head_stride", ctypes.c_int64)
                + _fields("k_caches v_caches pairs num_pairs status", ctypes.c_void_p))


class HookQ4Cache(ctypes.Structure):
    """Mirror of ``hook_q4_cache``."""
    _fields_ = [("pages", ctypes.c_void_p)] + _fields("block_stride head_stride", ctypes.c_int64) + [("group", ctypes.c_int32)]


class HookQ4ReadParams(ctypes.Structure):
    """Mirror of ``hook_q4_read_params``."""
    _fields_ = (_fields("num_seqs num_kv_heads head_dim page_size num_blocks max_blocks_per_seq to_num_blocks to_max_blocks_per_seq", ctypes.c_int32)
                + _fields("block_table seq_lens first k_cache v_cache", ctypes.c_void_p)
                + _fields("kv_block_stride kv_token_stride kv_head_stride", ctypes.c_int64) + _fields("to_table status", ctypes.c_void_p))


class HookQ4CopyParams(ctypes.Structure):
    """Mirror of ``hook_q4_copy_params``."""
    _fields_ = (_fields("num_layers num_blocks page_size num_kv_heads head_dim group max_pairs", ctypes.c_int32)
                + _fields("block_stride head_stride", ctypes.c_int64) + _fields("pages pairs num_pairs status", ctypes.c_void_p))


class HookSampleParams(ctypes.Structure):
    """Mirror of ``hook_sample_params``."""
    _fields_ = (_fields("num_rows vocab_size dtype", ctypes.c_int32) + [("logits", ctypes.c_void_p), ("logits_row_stride", ctypes.c_int64)]
                + _fields("uniform temperature top_k top_p min_p tokens status", ctypes.c_void_p))


class HookAttnError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} (code {code})")


_lib = _compiled = None


class _Missing:
    """In the place of the compiled part where that cannot be loaded: the short calls raise, the others do not need it."""

    def __init__(self, why: ImportError):
        self.why = why

    def __getattr__(self, name):
        raise ImportError("the binding's compiled part (_marshal.so) is missing or was built for another torch or Python: build it with "
                          "`python -m paper_2603_06588_b200.csrc.build`") from self.why


def load_library() -> ctypes.CDLL:
    """Load the compiled CUDA library; raises if it has not been built.  The compiled part of the binding is loaded beside it; where it
    is missing, the calls that it marshals raise."""
    global _lib, _compiled
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2603_06588_b200.csrc.build` "
                "(there is no fallback path)")
        lib = ctypes.CDLL(LIB_PATH)
        lib.hook_attn_create.restype = ctypes.c_int
        lib.hook_attn_create.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int]
        lib.hook_attn_destroy.restype = ctypes.c_int
        lib.hook_attn_destroy.argtypes = [ctypes.c_void_p]
        lib.hook_attn_workspace_bytes.restype = ctypes.c_size_t
        lib.hook_attn_workspace_bytes.argtypes = [ctypes.POINTER(HookAttnParams), ctypes.c_int]
        for name in ("hook_attn_prefill", "hook_attn_decode", "hook_attn_decode_static_scratch"):
            fn = getattr(lib, name)
            fn.restype = ctypes.c_int
            fn.argtypes = [ctypes.c_void_p, ctypes.POINTER(HookAttnParams), ctypes.c_void_p]
        lib.hook_attn_mixed.restype = ctypes.c_int
        lib.hook_attn_mixed.argtypes = [ctypes.c_void_p, ctypes.POINTER(HookAttnParams), ctypes.POINTER(HookAttnParams),
                                        ctypes.c_void_p]
        lib.hook_attn_score.restype = ctypes.c_int
        lib.hook_attn_score.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                        ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
        lib.hook_steer_residual.restype = ctypes.c_int
        lib.hook_steer_residual.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float,
                                            ctypes.c_int64, ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p]
        lib.hook_capture_qk.restype = ctypes.c_int
        lib.hook_capture_qk.argtypes = [ctypes.c_void_p, ctypes.POINTER(HookAttnParams), ctypes.c_int, ctypes.c_void_p,
                                        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        void_p, i32 = ctypes.c_void_p, ctypes.c_int32              # structs are passed by address
        for name, args in _AROUND.items():
            fn = getattr(lib, name)
            fn.restype = ctypes.c_int
            fn.argtypes = [void_p] + [i32 if a == "i" else void_p for a in args] + [void_p]
        lib.hook_q4_slab_bytes.restype = ctypes.c_size_t
        lib.hook_q4_slab_bytes.argtypes = [i32, i32]
        lib.hook_attn_selftest_wait_limit.restype = ctypes.c_int
        lib.hook_attn_selftest_wait_limit.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_uint64, ctypes.c_void_p,
                                                      ctypes.c_void_p]
        lib.hook_attn_strerror.restype = ctypes.c_char_p
        lib.hook_attn_strerror.argtypes = [ctypes.c_int]
        try:
            from . import _marshal
        except ImportError as e:
            _marshal = _Missing(e)
        _lib, _compiled = lib, _marshal
    return _lib


def strerror(code: int) -> str:
    return load_library().hook_attn_strerror(int(code)).decode()


def q4_slab_bytes(head_dim: int, group: int) -> int:
    """Bytes that a page of a 4-bit cache takes for one KV head: the last dimension of its uint8 ``pages [num_blocks, Hkv, bytes]``, from which
    the calls tell the group.  A fresh cache may hold anything."""
    nbytes = int(load_library().hook_q4_slab_bytes(int(head_dim), int(group)))
    if nbytes == 0:
        raise HookAttnError(HOOK_ATTN_ERR_UNSUPPORTED, "hook_q4_slab_bytes")
    return nbytes


def _dptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def make_params(*, q, k_cache, v_cache, block_table, seq_lens, cu_q_lens=None, spans=None,
                head_mask=None, alpha=None, steer_vec=None, scale: float = 0.0,
                probe_rows: int = HOOK_PROBE_ROWS_ALL, out=None, span_mass=None, workspace=None,
                status=None, max_seq_len: int = 0) -> Tuple[HookAttnParams, list]:
    """Marshal tensors into a ``hook_attn_params``.  ``head_mask`` / ``alpha`` are HOST tensors
    (uint8 / float32); everything else lives on the device.  Returns the struct and a list of
    objects that must stay alive until the call has been issued."""
    keep = []
    p = HookAttnParams()
    total_q, hq, d = q.shape
    nb, page, hkv, d2 = k_cache.shape
    assert d2 == d and v_cache.shape == k_cache.shape and v_cache.stride() == k_cache.stride()
    assert k_cache.stride(3) == 1 and q.is_contiguous()
    p.num_seqs = int(seq_lens.shape[0])
    p.total_q = int(total_q)
    p.num_q_heads, p.num_kv_heads, p.head_dim, p.page_size = int(hq), int(hkv), int(d), int(page)
    p.num_blocks = int(nb)
    p.max_blocks_per_seq = int(block_table.shape[1]) if block_table.dim() == 2 else 0
    p.num_spans = 0 if spans is None else int(spans.shape[1])
    p.probe_rows = int(probe_rows)
    p.scale = float(scale)
    p.max_seq_len = int(max_seq_len)
    p.q, p.k_cache, p.v_cache = q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr()
    p.kv_block_stride, p.kv_token_stride, p.kv_head_stride = (int(k_cache.stride(0)),
                                                               int(k_cache.stride(1)),
                                                               int(k_cache.stride(2)))
    p.block_table, p.seq_lens = block_table.data_ptr(), seq_lens.data_ptr()
    p.cu_q_lens = _dptr(cu_q_lens)
    p.spans = _dptr(spans)
    p.steer_vec = _dptr(steer_vec)
    p.out = _dptr(out)
    p.span_mass = _dptr(span_mass)
    p.workspace = _dptr(workspace)
    p.workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    p.status = _dptr(status)
    if head_mask is not None:
        hm = head_mask.detach().to("cpu", torch.uint8).contiguous()
        keep.append(hm)
        p.head_mask = hm.data_ptr()
    if alpha is not None:
        al = alpha.detach().to("cpu", torch.float32).contiguous()
        keep.append(al)
        p.alpha = al.data_ptr()
    return p, keep


class HookAttn:
    """Per-device handle plus the entry points, taking torch CUDA tensors."""

    def __init__(self, device: int = 0):
        lib = load_library()
        h = ctypes.c_void_p()
        rc = lib.hook_attn_create(ctypes.byref(h), int(device))
        if rc != HOOK_ATTN_OK:
            raise HookAttnError(rc, "hook_attn_create")
        self._lib = lib
        self._h = h
        self._index = int(device)
        self._marshal = _compiled
        self._calls = {name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _AROUND}
        self._workspace_bytes = ctypes.cast(lib.hook_attn_workspace_bytes, ctypes.c_void_p).value
        self.device = torch.device("cuda", int(device))

    def close(self):
        if getattr(self, "_h", None):
            self._lib.hook_attn_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- raw calls -----------------------------------------------------------------------
    def workspace_bytes(self, params: HookAttnParams, is_decode) -> int:
        """``is_decode``: False / True, 2 for the decode half of a mixed step, or 3 for the decode over a 4-bit cache."""
        return int(self._lib.hook_attn_workspace_bytes(ctypes.byref(params), int(is_decode)))

    def call(self, params: HookAttnParams, is_decode: bool, stream: Optional[int] = None) -> int:
        """Issue the call described by ``params``; returns the library's return code."""
        if stream is None:
            stream = torch.cuda.current_stream(self.device).cuda_stream
        fn = self._lib.hook_attn_decode if is_decode else self._lib.hook_attn_prefill
        return int(fn(self._h, ctypes.byref(params), ctypes.c_void_p(stream)))

    def call_decode_static_scratch(self, params: HookAttnParams, stream: Optional[int] = None) -> int:
        """``hook_attn_decode_static_scratch``: decode for callers that cannot allocate or pass
        scratch; the partials go into the library's fixed array (``STATIC_SCRATCH_BYTES``).
        Returns the library's return code."""
        if stream is None:
            stream = torch.cuda.current_stream(self.device).cuda_stream
        return int(self._lib.hook_attn_decode_static_scratch(self._h, ctypes.byref(params),
                                                             ctypes.c_void_p(stream)))

    def selftest_wait_limit(self, limit_ns: int = 200_000_000, stream=None):
        """Run the bounded-wait self-test; returns ``(status_code, waited_ns)`` read back from the device."""
        status = torch.zeros(1, dtype=torch.int32, device=self.device)
        waited = torch.zeros(1, dtype=torch.int64, device=self.device)
        rc = int(self._lib.hook_attn_selftest_wait_limit(self._h, status.data_ptr(), int(limit_ns), waited.data_ptr(),
                                                         self._stream(stream)))
        if rc != HOOK_ATTN_OK:
            raise HookAttnError(rc, "hook_attn_selftest_wait_limit")
        torch.cuda.synchronize(self.device)
        return int(status.item()), int(waited.item())

    def _stream(self, stream):
        return ctypes.c_void_p(torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream)

    def hook_attn_score(self, span_mass: torch.Tensor, mode: int = HOOK_SCORE_SUM_NORMALIZE, scores=None, stream=None):
        """Analyzer reduction: ``span_mass`` fp32 ``[R, P, S]`` (device) -> ``scores`` fp32 ``[R, S]``."""
        rows, nprobed, nspans = span_mass.shape
        assert span_mass.dtype == torch.float32 and span_mass.is_contiguous()
        if scores is None:
            scores = torch.empty((rows, nspans), dtype=torch.float32, device=span_mass.device)
        rc = int(self._lib.hook_attn_score(self._h, span_mass.data_ptr(), rows, nprobed, nspans, int(mode),
                                           scores.data_ptr(), self._stream(stream)))
        if rc != HOOK_ATTN_OK:
            raise HookAttnError(rc, "hook_attn_score")
        return scores

    def hook_steer_residual(self, hidden: torch.Tensor, steer_vec: torch.Tensor, alpha: float, stream=None):
        """Residual-stream steering in place: ``hidden`` bf16 ``[T, H]`` (device, rows may be strided),
        ``steer_vec`` fp32 ``[H]``."""
        assert hidden.dtype == torch.bfloat16 and hidden.dim() == 2 and hidden.stride(1) == 1
        assert steer_vec.dtype == torch.float32 and steer_vec.is_contiguous()
        rc = int(self._lib.hook_steer_residual(self._h, hidden.data_ptr(), steer_vec.data_ptr(), float(alpha),
                                               hidden.shape[0], hidden.shape[1], hidden.stride(0), self._stream(stream)))
        if rc != HOOK_ATTN_OK:
            raise HookAttnError(rc, "hook_steer_residual")
        return hidden

    def hook_capture_qk(self, is_decode: bool, *, q, k_cache, v_cache, block_table, seq_lens, cu_q_lens=None,
                        head_mask=None, probe_rows=HOOK_PROBE_ROWS_ALL, status=None, stream=None,
                        q_out=None, k_out=None, cu_k_lens=None, max_seq_len: int = 0, **_ignored):
        """Raw q/k capture of the probed heads.  Returns ``(q_out [rows, P, D], k_out [sum L, P, D], cu_k_lens)``.
        The three outputs are allocated (and the prefix sums computed, with one host sync for the total)
        unless the caller passes them."""
        nprobed = 0 if head_mask is None else int((head_mask != 0).sum())
        total_q, hq, d = q.shape
        last_only = is_decode or probe_rows == HOOK_PROBE_ROWS_LAST
        rows = int(seq_lens.shape[0]) if last_only else int(total_q)
        cu_k = cu_k_lens
        if cu_k is None:
            cu_k = torch.zeros(seq_lens.shape[0] + 1, dtype=torch.int32, device=q.device)
            cu_k[1:] = torch.cumsum(seq_lens, 0)
        if q_out is None:
            q_out = torch.zeros((rows, nprobed, d), dtype=torch.bfloat16, device=q.device)
        if k_out is None:
            k_out = torch.zeros((int(cu_k[-1].item()), nprobed, d), dtype=torch.bfloat16, device=q.device)
        p, keep = make_params(q=q, k_cache=k_cache, v_cache=v_cache, block_table=block_table, seq_lens=seq_lens,
                              cu_q_lens=cu_q_lens, head_mask=head_mask, probe_rows=probe_rows, status=status,
                              max_seq_len=max_seq_len)
        rc = int(self._lib.hook_capture_qk(self._h, ctypes.byref(p), int(bool(is_decode)), q_out.data_ptr(),
                                           k_out.data_ptr(), cu_k.data_ptr(), self._stream(stream)))
        del keep
        if rc != HOOK_ATTN_OK:
            raise HookAttnError(rc, "hook_capture_qk")
        return q_out, k_out, cu_k

    # -- what a decode step needs around the attention --------------------------------------
    # These calls are short: a compiled module checks the tensors (AssertionError), fills the C structs, allocates the results and calls
    # the library (one row of hook_rope_append: 11.7 us a call with the same done here, 5.4 us with it, of which the launch is 2.9).
    def _short(self, name: str, call, stream, *args):
        got = call(self._calls[name], self._h.value if self._h else 0, self._index, stream, *args)
        if type(got) is int:
            if got != HOOK_ATTN_OK:
                raise HookAttnError(got, name)
            return None
        return got

    def hook_rope_append(self, *, q, k, v, k_cache, v_cache, block_table, seq_lens, inv_freq, cu_q_lens=None, positions=None,
                         axis_pairs=None, axis_order: int = HOOK_ROPE_AXES_BLOCKED, pairing: int = HOOK_ROPE_PAIR_HALVES,
                         factor: float = 1.0, q_out=None, status=None, stream=None) -> torch.Tensor:
        """Rotates ``q [T, Hq, D]`` and ``k [T, Hkv, D]`` and appends k and ``v`` to the pages of the rows' sequences.
        ``inv_freq`` fp32 ``[R / 2]`` gives the frequencies of the pairs and R; ``axis_pairs`` how many pairs each axis has (default:
        one axis); ``positions`` int32 ``[axes, T]`` (default: the rows' places in their sequences).  bf16, fp16 or fp32 in, the
        rotated queries out as bf16, contiguous, like the attention reads them."""
        return self._short("hook_rope_append", self._marshal.rope_append, stream, q, k, v, k_cache, v_cache, block_table, seq_lens, inv_freq,
                           cu_q_lens, positions, axis_pairs, axis_order, pairing, factor, q_out, status)

    def hook_adjust_logits(self, logits, *, out=None, tokens=None, prompt_lens=None, total_lens=None, repetition=None, presence=None,
                           frequency=None, bias_offsets=None, bias_tokens=None, bias_values=None, mask=None, mask_rows=None,
                           status=None, stream=None) -> torch.Tensor:
        """Penalties, biases and grammar masks on ``logits [rows, vocab]`` (bf16, fp16 or fp32; rows may be strided), in place or into
        ``out`` (the same type, or fp32).  ``tokens`` int32 ``[rows, max_tokens]`` holds each row's prompt and what was generated;
        the biases are lists in rows (``bias_offsets [rows + 1]``); ``mask`` int32 ``[masks, ceil(vocab / 32)]`` has a bit for each allowed
        token and ``mask_rows`` says which of them a row has (negative: none)."""
        return self._short("hook_adjust_logits", self._marshal.adjust_logits, stream, logits, out, tokens, prompt_lens, total_lens, repetition,
                           presence, frequency, bias_offsets, bias_tokens, bias_values, mask, mask_rows, status)

    def hook_cache_fork(self, block_table, seq_lens, page_refs, parents, children, status=None, stream=None) -> None:
        """Sequence ``children[i]`` (empty) becomes a copy of ``parents[i]`` that shares its pages."""
        self._short("hook_cache_fork", self._marshal.cache_fork, stream, block_table, seq_lens, page_refs, status, parents, children)

    def hook_cache_extend(self, block_table, seq_lens, page_refs, new_rows, pairs=None, status=None, stream=None) -> torch.Tensor:
        """Room for ``new_rows[s]`` more tokens in every sequence; returns ``pairs`` int32 ``[seqs, 2]``, the pages to copy before
        anything is appended (-1: none)."""
        return self._short("hook_cache_extend", self._marshal.cache_extend, stream, block_table, seq_lens, page_refs, status, new_rows, pairs)

    def hook_cache_free(self, block_table, seq_lens, page_refs, seqs, keep_lens=None, status=None, stream=None) -> None:
        """Cuts the sequences ``seqs`` to their first ``keep_lens`` tokens (default: to nothing)."""
        self._short("hook_cache_free", self._marshal.cache_free, stream, block_table, seq_lens, page_refs, status, seqs, keep_lens)

    def hook_cache_compact(self, block_table, seq_lens, page_refs, status=None, stream=None):
        """Plans how the used pages move together at the low end of the pool.  Returns ``(block_table, page_refs, page_map, pairs,
        num_pairs)`` as they are once the pairs are copied; the old ones stay as they are."""
        return self._short("hook_cache_compact", self._marshal.cache_compact, stream, block_table, seq_lens, page_refs, status)

    def hook_cache_copy_pages(self, caches, pairs, num_pairs=None, status=None, stream=None) -> None:
        """Copies pages ``pairs[i] = (source, destination)`` in the ``caches``, a list of ``(k_cache, v_cache)`` of the layers (one
        shape, one set of strides).  ``num_pairs``: int32 ``[1]`` on the device, how many of the pairs count (2^22 at most)."""
        self._short("hook_cache_copy_pages", self._marshal.cache_copy_pages, stream, caches, pairs, num_pairs, status)

    # -- a cache held in 4 bits --------------------------------------------------------------
    def hook_rope_append_q4(self, *, q, k, v, pages, block_table, seq_lens, inv_freq, cu_q_lens=None, positions=None, axis_pairs=None,
                            axis_order: int = HOOK_ROPE_AXES_BLOCKED, pairing: int = HOOK_ROPE_PAIR_HALVES, factor: float = 1.0, q_out=None,
                            status=None, stream=None) -> torch.Tensor:
        """:meth:`hook_rope_append` into a 4-bit cache, ``pages`` uint8 ``[num_blocks, Hkv, q4_slab_bytes(D, group)]``: keys and values are
        quantised as they are written.  Returns the rotated queries."""
        return self._short("hook_rope_append_q4", self._marshal.rope_append_q4, stream, q, k, v, pages, block_table, seq_lens, inv_freq,
                           cu_q_lens, positions, axis_pairs, axis_order, pairing, factor, q_out, status)

    def hook_attn_decode_q4(self, *, q, pages, block_table, seq_lens, spans=None, head_mask=None, alpha=None, steer_vec=None, scale: float = 0.0,
                            out=None, span_mass=None, workspace=None, status=None, max_seq_len: int = 0, stream=None):
        """:meth:`hook_attn_decode` over a 4-bit cache: ``q`` bf16 ``[seqs, Hq, D]``, ``head_mask`` and ``alpha`` on the host.  Returns
        ``(out, span_mass)``; ``span_mass`` is None without probes.  ``workspace``: uint8 of
        ``workspace_bytes(params, 3)``, 256-byte aligned; allocated if not given."""
        return self._short("hook_attn_decode_q4", self._marshal.attn_decode_q4, stream, q, pages, block_table, seq_lens, spans, head_mask, alpha,
                           steer_vec, scale, out, span_mass, workspace, status, max_seq_len, self._workspace_bytes)

    def hook_cache_read_q4(self, pages, block_table, seq_lens, *, k_cache, v_cache, to_table, first=None, status=None, stream=None) -> None:
        """Reads positions ``first[s]`` (default 0) to ``seq_lens[s]`` of every sequence back to the pages ``to_table`` of a bf16 cache, where
        :meth:`hook_attn_prefill` and :meth:`hook_capture_qk` find them."""
        self._short("hook_cache_read_q4", self._marshal.cache_read_q4, stream, pages, block_table, seq_lens, k_cache, v_cache, to_table, first, status)

    def hook_cache_copy_pages_q4(self, caches, pairs, num_pairs=None, status=None, stream=None) -> None:
        """:meth:`hook_cache_copy_pages` for 4-bit caches, a list of the layers' ``pages``."""
        self._short("hook_cache_copy_pages_q4", self._marshal.cache_copy_pages_q4, stream, caches, pairs, num_pairs, status)

    # -- the choice of a token ---------------------------------------------------------------
    def hook_sample_tokens(self, logits, uniform, *, temperature=None, top_k=None, top_p=None, min_p=None, tokens=None, status=None,
                           stream=None) -> torch.Tensor:
        """A token for each row of ``logits [rows, vocab]`` (bf16, fp16 or fp32; rows may be strided) from one random number in [0, 1) each:
        ``uniform``, ``temperature``, ``top_p``, ``min_p`` fp32 and ``top_k`` int32, all ``[rows]``.  Temperature 0 takes the largest logit.
        Returns int32 ``[rows]``; -1 for a row that has nothing to choose from or a parameter out of range."""
        return self._short("hook_sample_tokens", self._marshal.sample_tokens, stream, logits, uniform, temperature, top_k, top_p, min_p, tokens, status)

    # -- convenience ---------------------------------------------------------------------
    def plan(self, is_decode: bool, *, q, k_cache, v_cache, block_table, seq_lens, cu_q_lens=None,
             spans=None, head_mask=None, alpha=None, steer_vec=None, scale=0.0,
             probe_rows=HOOK_PROBE_ROWS_ALL, out=None, span_mass=None, status=None,
             max_seq_len: int = 0, mixed_half: bool = False) -> "HookAttnPlan":
        """Marshal the arguments once (allocating `out`, `span_mass` and scratch when they are not
        given); the returned plan re-issues the same call with one C call per step."""
        total_q, hq, d = q.shape
        if out is None:
            out = torch.empty_like(q)
        nprobed = 0 if head_mask is None else int((head_mask != 0).sum())
        nspans = 0 if spans is None else int(spans.shape[1])
        if span_mass is None and nprobed and nspans:
            rows = seq_lens.shape[0] if (is_decode or probe_rows == HOOK_PROBE_ROWS_LAST) else total_q
            span_mass = torch.zeros((rows, nprobed, nspans), dtype=torch.float32, device=q.device)
        p, keep = make_params(q=q, k_cache=k_cache, v_cache=v_cache, block_table=block_table,
                              seq_lens=seq_lens, cu_q_lens=cu_q_lens, spans=spans,
                              head_mask=head_mask, alpha=alpha, steer_vec=steer_vec, scale=scale,
                              probe_rows=probe_rows, out=out, span_mass=span_mass, status=status,
                              max_seq_len=max_seq_len)
        nbytes = self.workspace_bytes(p, 2 if (is_decode and mixed_half) else is_decode)
        ws = None
        if nbytes:
            ws = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
            p.workspace = ws.data_ptr()
            p.workspace_bytes = nbytes
        keep += [q, k_cache, v_cache, block_table, seq_lens, cu_q_lens, spans, steer_vec, status, ws]
        return HookAttnPlan(self, is_decode, p, out, span_mass, keep)

    def mixed_plan(self, prefill_kw: dict, decode_kw: dict) -> "HookAttnMixedPlan":
        """A step with a decode batch and prefill chunks (``hook_attn_mixed``): marshals both halves once."""
        return HookAttnMixedPlan(self, self.plan(False, **prefill_kw), self.plan(True, mixed_half=True, **decode_kw))

    def hook_attn_mixed(self, prefill_kw: dict, decode_kw: dict):
        """Returns ``((out, span_mass) of the prefill half, (out, span_mass) of the decode half)``."""
        pl = self.mixed_plan(prefill_kw, decode_kw)
        pl.run()
        return (pl.prefill.out, pl.prefill.span_mass), (pl.decode.out, pl.decode.span_mass)

    def hook_attn_prefill(self, **kw):
        """Prefill / chunked prefill.  Returns ``(out, span_mass)``."""
        pl = self.plan(False, **kw)
        pl.run()
        return pl.out, pl.span_mass

    def hook_attn_decode(self, **kw):
        """Decode (one query row per sequence).  Returns ``(out, span_mass)``."""
        pl = self.plan(True, **kw)
        pl.run()
        return pl.out, pl.span_mass


class HookAttnPlan:
    """A marshalled call: ``run()`` enqueues it on the current (or given) CUDA stream."""

    def __init__(self, eng: HookAttn, is_decode: bool, params: HookAttnParams, out, span_mass, keep):
        self.eng, self.is_decode, self.params = eng, is_decode, params
        self.out, self.span_mass, self._keep = out, span_mass, keep
        self._fn = eng._lib.hook_attn_decode if is_decode else eng._lib.hook_attn_prefill
        self._ref = ctypes.byref(params)

    def run(self, stream: Optional[int] = None) -> None:
        if stream is None:
            stream = torch.cuda.current_stream(self.eng.device).cuda_stream
        rc = int(self._fn(self.eng._h, self._ref, ctypes.c_void_p(stream)))
        if rc != HOOK_ATTN_OK:
            raise HookAttnError(rc, "hook_attn_decode" if self.is_decode else "hook_attn_prefill")


class HookAttnMixedPlan:
    """The two marshalled halves of a mixed step; ``run()`` issues them with one ``hook_attn_mixed`` call."""

    def __init__(self, eng: HookAttn, prefill: HookAttnPlan, decode: HookAttnPlan):
        self.eng, self.prefill, self.decode = eng, prefill, decode

    def run(self, stream: Optional[int] = None) -> None:
        if stream is None:
            stream = torch.cuda.current_stream(self.eng.device).cuda_stream
        rc = int(self.eng._lib.hook_attn_mixed(self.eng._h, self.prefill._ref, self.decode._ref, ctypes.c_void_p(stream)))
        if rc != HOOK_ATTN_OK:
            raise HookAttnError(rc, "hook_attn_mixed")


def case_to_device(case, device="cuda") -> dict:
    """Keyword arguments for :meth:`HookAttn.hook_attn_prefill` / ``hook_attn_decode`` from an
    input-generator case (device copies of the tensors; host copies of head_mask / alpha)."""
    dev = torch.device(device)
    kw = dict(q=case.q.to(dev), k_cache=case.k_cache.to(dev), v_cache=case.v_cache.to(dev),
              block_table=case.block_table.to(dev), seq_lens=case.seq_lens.to(dev),
              scale=case.scale, probe_rows=case.probe_rows)
    if not case.is_decode:
        kw["cu_q_lens"] = case.cu_q_lens.to(dev)
    if case.spans is not None:
        kw["spans"] = case.spans.to(dev)
    if case.steer_vec is not None:
        kw["steer_vec"] = case.steer_vec.to(dev)
    if case.head_mask is not None:
        kw["head_mask"] = case.head_mask
    if case.alpha is not None:
        kw["alpha"] = case.alpha
    return kw
