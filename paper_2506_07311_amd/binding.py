"""ctypes binding of libpagedattn.so -- argument marshalling only.

Every function has the name and argument meaning of its C entry point in
``include/pagedattn.h``; torch tensors supply device pointers and the current
HIP stream, nothing else.  There is no CPU fallback: if the HIP library has not
been built, loading raises.

A call that is given ``stream=`` runs there, and what it allocates is that stream's
memory; ordering its tensors' other uses around it is the caller's, as for any
work on another stream.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libpagedattn.so"
_lib = None

PA_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

EXPORTS = (
    "paged_kv_append", "paged_kv_gather", "paged_attention_workspace_bytes", "paged_attention_decode",
    "paged_attention_prefill", "paged_attention_decode_mod", "paged_attention_prefill_mod", "paged_decode_step",
    "paged_attention_decode_static", "paged_plan_step", "paged_release_blocks", "pa_rope_frequencies", "paged_rope_append",
    "paged_attention_tree_workspace_bytes", "paged_attention_tree", "paged_tree_accept", "paged_norm_rope_append",
    "pa_mx4_record_bytes", "paged_norm_rope_append_mx4", "paged_kv_append_mx4", "paged_kv_gather_mx4",
    "paged_attention_mx4_workspace_bytes", "paged_attention_mx4", "pa_debug_check",
    "pa_status_string", "pa_set_option", "pa_stream_read", "pa_profile_enable", "pa_profile_reset",
    "pa_profile_read",
    "pa_pool_create", "pa_pool_destroy", "pa_pool_set_growth", "pa_pool_reserve", "pa_pool_release", "pa_pool_share_prefix",
    "pa_pool_make_writable", "pa_pool_make_writable_mx4", "pa_pool_num_free", "pa_pool_num_blocks", "pa_pool_get_row", "pa_pool_refcount",
)


class PagedAttnError(RuntimeError):
    pass


class _Desc(ctypes.Structure):
    _fields_ = [("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p),
                ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64),
                ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


def library_path() -> str:
    return os.path.join(_HERE, _LIB_NAME)


def load_library():
    """Load the HIP library built in-tree (``python -m paper_2506_07311_amd.build``)."""
    global _lib
    if _lib is None:
        path = library_path()
        if not os.path.exists(path):
            raise PagedAttnError(
                f"{path} is missing: build the HIP library first (python -m paper_2506_07311_amd.build). "
                "There is no CPU fallback.")
        lib = ctypes.CDLL(path)
        sizes = ("paged_attention_workspace_bytes", "paged_attention_tree_workspace_bytes", "paged_attention_mx4_workspace_bytes",
                 "pa_mx4_record_bytes")
        for name in sizes:
            getattr(lib, name).restype = ctypes.c_size_t
        lib.pa_status_string.restype = ctypes.c_char_p
        for name in EXPORTS:
            if name not in sizes and name != "pa_status_string":
                getattr(lib, name).restype = ctypes.c_int
        _lib = lib
    return _lib


def _check(status: int, what: str):
    if status != 0:
        msg = load_library().pa_status_string(status).decode()
        raise PagedAttnError(f"{what}: {msg} (status {status})")


def _p(t: Optional[torch.Tensor]):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _new(shape, dtype, device, stream) -> torch.Tensor:
    """Memory that a call on ``stream`` writes.  Of another stream than the current one it comes from that stream's part of
    the allocator: whatever used it before and whoever gets it afterwards is then ordered by that stream, on which the
    call may still be running when the tensor is dropped.  The current stream, whose work may read a result, is told as
    well."""
    here = torch.cuda.current_stream(device)
    if stream is None or stream.cuda_stream == here.cuda_stream:
        return torch.empty(shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(here)
    return t


def _i32(t: torch.Tensor, what: str) -> torch.Tensor:
    if t.dtype != torch.int32 or not t.is_contiguous() or not t.is_cuda:
        raise PagedAttnError(f"{what} must be a contiguous int32 device tensor")
    return t


def cache_desc(k_cache: torch.Tensor, v_cache: torch.Tensor, head_major: bool = False) -> _Desc:
    """Descriptor of the pools.  Token-major ``[NP, P, Hkv, d]`` unless head_major (``[NP, Hkv, P, d]``).
    Either may be a strided view as long as head_dim is contiguous and K and V share strides."""
    if k_cache.dtype not in PA_DTYPE or v_cache.dtype != k_cache.dtype:
        raise PagedAttnError(f"unsupported cache dtype {k_cache.dtype}")
    if k_cache.dim() != 4 or k_cache.shape != v_cache.shape or k_cache.stride() != v_cache.stride():
        raise PagedAttnError("k_cache and v_cache must be 4-d with equal shapes and strides")
    if not (k_cache.is_cuda and v_cache.is_cuda) or k_cache.stride(3) != 1:
        raise PagedAttnError("caches must be device tensors with a contiguous head_dim")
    if head_major:
        NP, Hkv, P, d = k_cache.shape
        sp, sh, st, _ = k_cache.stride()
    else:
        NP, P, Hkv, d = k_cache.shape
        sp, st, sh, _ = k_cache.stride()
    return _Desc(k_cache.data_ptr(), v_cache.data_ptr(), sp, st, sh, NP, P, Hkv, d, PA_DTYPE[k_cache.dtype])


def _dense(t: torch.Tensor, what: str, dtype) -> torch.Tensor:
    if t.dtype != dtype or not t.is_contiguous() or not t.is_cuda:
        raise PagedAttnError(f"{what} must be a contiguous device tensor of dtype {dtype}")
    return t


class PreparedCall:
    """One entry point with its arguments already marshalled (pointers, sizes and the stream as of preparation).
    Calling it repeats exactly that call: for steady-state loops over the same buffers, where checking and
    converting the arguments again would cost more host time than the step takes on the GPU.  The tensors are kept
    alive by the object; their contents may change between calls, their addresses and shapes may not."""

    __slots__ = ("_fn", "_args", "_keep", "_what", "result")

    def __init__(self, fn, args, keep, what, result=None):
        self._fn, self._args, self._keep, self._what, self.result = fn, args, keep, what, result

    def __call__(self):
        st = self._fn(*self._args)
        if st:
            _check(st, self._what)
        return self.result


def prepare_kv_append(k_cache, v_cache, k_new, v_new, seq_ids, positions, block_table, *, head_major=False,
                      stream=None) -> PreparedCall:
    lib = load_library()
    d = cache_desc(k_cache, v_cache, head_major)
    T = int(seq_ids.shape[0])
    _dense(k_new, "k_new", k_cache.dtype), _dense(v_new, "v_new", k_cache.dtype)
    if tuple(k_new.shape) != (T, d.num_kv_heads, d.head_dim) or k_new.shape != v_new.shape:
        raise PagedAttnError("k_new/v_new must be [T, Hkv, d]")
    _i32(seq_ids, "seq_ids"), _i32(positions, "positions"), _i32(block_table, "block_table")
    args = (ctypes.byref(d), _p(k_new), _p(v_new), _p(seq_ids), _p(positions), ctypes.c_int32(T), _p(block_table),
            ctypes.c_int32(block_table.shape[0]), ctypes.c_int32(block_table.shape[1]), _stream(stream))
    return PreparedCall(lib.paged_kv_append, args, (d, k_cache, v_cache, k_new, v_new, seq_ids, positions, block_table),
                        "paged_kv_append")


def paged_kv_append(k_cache, v_cache, k_new, v_new, seq_ids, positions, block_table, *, head_major=False,
                    stream=None) -> None:
    prepare_kv_append(k_cache, v_cache, k_new, v_new, seq_ids, positions, block_table, head_major=head_major,
                      stream=stream)()


def paged_kv_gather(k_cache, v_cache, block_table, seq_lens, cu_seq_lens, total_tokens: int, max_seq_len: int, *,
                    head_major=False, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    lib = load_library()
    d = cache_desc(k_cache, v_cache, head_major)
    _i32(block_table, "block_table"), _i32(seq_lens, "seq_lens"), _i32(cu_seq_lens, "cu_seq_lens")
    out_k, out_v = (_new((total_tokens, d.num_kv_heads, d.head_dim), k_cache.dtype, k_cache.device, stream) for _ in range(2))
    st = lib.paged_kv_gather(ctypes.byref(d), _p(out_k), _p(out_v), _p(block_table), _p(seq_lens), _p(cu_seq_lens),
                             ctypes.c_int32(seq_lens.shape[0]), ctypes.c_int32(block_table.shape[1]),
                             ctypes.c_int32(max_seq_len), _stream(stream))
    _check(st, "paged_kv_gather")
    return out_k, out_v


def paged_attention_workspace_bytes(batch: int, num_q_heads: int, head_dim: int, total_q: int,
                                    max_seq_len: int) -> int:
    return int(load_library().paged_attention_workspace_bytes(
        ctypes.c_int32(batch), ctypes.c_int32(num_q_heads), ctypes.c_int32(head_dim), ctypes.c_int32(total_q),
        ctypes.c_int32(max_seq_len)))


def _workspace(workspace, nbytes, device, stream):
    return _new(nbytes, torch.uint8, device, stream) if workspace is None else workspace


def paged_attention_decode(k_cache, v_cache, q, block_table, seq_lens, max_seq_len: int, scale: float, *,
                           out=None, lse=None, workspace=None, head_major=False, stream=None):
    """Returns ``out`` ([B, Hq, d], dtype of q).  ``lse`` (float32 [B, Hq]) is filled when given."""
    return prepare_decode(k_cache, v_cache, q, block_table, seq_lens, max_seq_len, scale, out=out, lse=lse,
                          workspace=workspace, head_major=head_major, stream=stream)()


def prepare_decode(k_cache, v_cache, q, block_table, seq_lens, max_seq_len: int, scale: float, *,
                   out=None, lse=None, workspace=None, head_major=False, stream=None) -> PreparedCall:
    """paged_attention_decode with its arguments marshalled once; the call returns ``out``."""
    lib = load_library()
    d = cache_desc(k_cache, v_cache, head_major)
    _dense(q, "q", k_cache.dtype)
    B, Hq, hd = q.shape
    if hd != d.head_dim or seq_lens.shape[0] != B or block_table.shape[0] != B:
        raise PagedAttnError("q must be [B, Hq, d] with B matching seq_lens and block_table")
    _i32(block_table, "block_table"), _i32(seq_lens, "seq_lens")
    out = _new(q.shape, q.dtype, q.device, stream) if out is None else _dense(out, "out", q.dtype)
    if lse is not None:
        _dense(lse, "lse", torch.float32)
    if workspace is None:   # (a workspace that is passed in is checked by the library itself)
        workspace = _workspace(None, paged_attention_workspace_bytes(B, Hq, hd, B, max_seq_len), q.device, stream)
    args = (ctypes.byref(d), _p(q), _p(out), _p(lse), _p(block_table), _p(seq_lens), ctypes.c_int32(B),
            ctypes.c_int32(Hq), ctypes.c_int32(block_table.shape[1]), ctypes.c_int32(max_seq_len),
            ctypes.c_float(scale), _p(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()),
            _stream(stream))
    return PreparedCall(lib.paged_attention_decode, args,
                        (d, k_cache, v_cache, q, out, lse, block_table, seq_lens, workspace), "paged_attention_decode",
                        out)


def paged_attention_decode_static(k_cache, v_cache, q, block_table, seq_lens, max_seq_len: int, scale: float, *,
                                  out, lse=None, head_major=False, stream=None):
    """paged_attention_decode without a workspace: the split-KV partials go to the library's static scratch array.
    Nothing is allocated here either: ``out`` ([B, Hq, d], dtype of q) must be passed in and is returned."""
    lib = load_library()
    d = cache_desc(k_cache, v_cache, head_major)
    _dense(q, "q", k_cache.dtype)
    B, Hq, hd = q.shape
    if hd != d.head_dim or seq_lens.shape[0] != B or block_table.shape[0] != B:
        raise PagedAttnError("q must be [B, Hq, d] with B matching seq_lens and block_table")
    _i32(block_table, "block_table"), _i32(seq_lens, "seq_lens")
    _dense(out, "out", q.dtype)
    if lse is not None:
        _dense(lse, "lse", torch.float32)
    st = lib.paged_attention_decode_static(ctypes.byref(d), _p(q), _p(out), _p(lse), _p(block_table), _p(seq_lens),
                                           ctypes.c_int32(B), ctypes.c_int32(Hq), ctypes.c_int32(block_table.shape[1]),
                                           ctypes.c_int32(max_seq_len), ctypes.c_float(scale), _stream(stream))
    _check(st, "paged_attention_decode_static")
    return out


def paged_attention_prefill(k_cache, v_cache, q, cu_q_lens, max_q_len: int, block_table, seq_lens,
                            max_seq_len: int, scale: float, causal: bool, *, out=None, lse=None, workspace=None,
                            head_major=False, stream=None):
    """Returns ``out`` ([total_q, Hq, d], dtype of q).  ``lse`` (float32 [total_q, Hq]) is filled when given."""
    return prepare_prefill(k_cache, v_cache, q, cu_q_lens, max_q_len, block_table, seq_lens, max_seq_len, scale,
                           causal, out=out, lse=lse, workspace=workspace, head_major=head_major, stream=stream)()


def prepare_prefill(k_cache, v_cache, q, cu_q_lens, max_q_len: int, block_table, seq_lens, max_seq_len: int,
                    scale: float, causal: bool, *, out=None, lse=None, workspace=None, head_major=False,
                    stream=None) -> PreparedCall:
    """paged_attention_prefill with its arguments marshalled once; the call returns ``out``."""
    lib = load_library()
    d = cache_desc(k_cache, v_cache, head_major)
    _dense(q, "q", k_cache.dtype)
    total_q, Hq, hd = q.shape
    B = int(seq_lens.shape[0])
    if hd != d.head_dim or block_table.shape[0] != B or cu_q_lens.shape[0] != B + 1:
        raise PagedAttnError("q must be [total_q, Hq, d]; cu_q_lens int32[B+1]")
    _i32(block_table, "block_table"), _i32(seq_lens, "seq_lens"), _i32(cu_q_lens, "cu_q_lens")
    out = _new(q.shape, q.dtype, q.device, stream) if out is None else _dense(out, "out", q.dtype)
    if lse is not None:
        _dense(lse, "lse", torch.float32)
    if workspace is None:
        workspace = _workspace(None, paged_attention_workspace_bytes(B, Hq, hd, total_q, max_seq_len), q.device, stream)
    args = (ctypes.byref(d), _p(q), _p(out), _p(lse), _p(cu_q_lens), ctypes.c_int32(total_q),
            ctypes.c_int32(max_q_len), _p(block_table), _p(seq_lens), ctypes.c_int32(B), ctypes.c_int32(Hq),
            ctypes.c_int32(block_table.shape[1]), ctypes.c_int32(max_seq_len), ctypes.c_float(scale),
            ctypes.c_int32(1 if causal else 0), _p(workspace),
            ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream))
    return PreparedCall(lib.paged_attention_prefill, args,
                        (d, k_cache, v_cache, q, out, lse, cu_q_lens, block_table, seq_lens, workspace),
                        "paged_attention_prefill", out)


class _Mods(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int32), ("softcap", ctypes.c_float), ("alibi_slopes", ctypes.c_void_p),
                ("doc_ids", ctypes.c_void_p), ("doc_stride", ctypes.c_int64), ("user_mod", ctypes.c_int32),
                ("user_data", ctypes.c_void_p)]


PA_MOD_PREFIX_LM = 1   # kId of pa_mod_prefix_lm in include/pagedattn_mods.h


def prefix_lm_data(prefix_len: torch.Tensor, prefix_bias: float = 0.0) -> torch.Tensor:
    """A pa_prefix_lm_data struct in device memory (pointer to int32[batch] prefix lengths, then the bias), to pass as
    ``user_data`` with ``user_mod=PA_MOD_PREFIX_LM``.  The caller keeps ``prefix_len`` alive while the struct is in use."""
    import struct
    _i32(prefix_len, "prefix_len")
    raw = struct.pack("<Qfi", prefix_len.data_ptr(), float(prefix_bias), 0)
    return torch.tensor(list(raw), dtype=torch.uint8).to(prefix_len.device)


def _mods(window, softcap, alibi_slopes, doc_ids, Hq, B, user_mod=0, user_data=None):
    if alibi_slopes is not None:
        _dense(alibi_slopes, "alibi_slopes", torch.float32)
        if tuple(alibi_slopes.shape) != (Hq,):
            raise PagedAttnError("alibi_slopes must be float32[Hq]")
    if doc_ids is not None:
        _i32(doc_ids, "doc_ids")
        if doc_ids.dim() != 2 or doc_ids.shape[0] != B:
            raise PagedAttnError("doc_ids must be int32[batch, doc_stride]")
    if user_mod and (user_data is None or not user_data.is_cuda):
        raise PagedAttnError("a user modification needs its user_data in device memory")
    return _Mods(int(window), float(softcap), None if alibi_slopes is None else alibi_slopes.data_ptr(),
                 None if doc_ids is None else doc_ids.data_ptr(), 0 if doc_ids is None else doc_ids.shape[1],
                 int(user_mod), None if user_data is None else user_data.data_ptr())


def paged_attention_decode_mod(k_cache, v_cache, q, block_table, seq_lens, max_seq_len: int, scale: float, *,
                               window: int = 0, softcap: float = 0.0, alibi_slopes=None, doc_ids=None,
                               user_mod: int = 0, user_data=None,
                               out=None, lse=None, workspace=None, head_major=False, stream=None):
    """paged_attention_decode with mask / score modifications (see pa_attn_mods in the header)."""
    lib = load_library()
    d = cache_desc(k_cache, v_cache, head_major)
    _dense(q, "q", k_cache.dtype)
    B, Hq, hd = q.shape
    if hd != d.head_dim or seq_lens.shape[0] != B or block_table.shape[0] != B:
        raise PagedAttnError("q must be [B, Hq, d] with B matching seq_lens and block_table")
    _i32(block_table, "block_table"), _i32(seq_lens, "seq_lens")
    out = _new(q.shape, q.dtype, q.device, stream) if out is None else _dense(out, "out", q.dtype)
    if lse is not None:
        _dense(lse, "lse", torch.float32)
    mods = _mods(window, softcap, alibi_slopes, doc_ids, Hq, B, user_mod, user_data)
    workspace = _workspace(workspace, paged_attention_workspace_bytes(B, Hq, hd, B, max_seq_len), q.device, stream)
    st = lib.paged_attention_decode_mod(ctypes.byref(d), _p(q), _p(out), _p(lse), _p(block_table), _p(seq_lens),
                                        ctypes.c_int32(B), ctypes.c_int32(Hq), ctypes.c_int32(block_table.shape[1]),
                                        ctypes.c_int32(max_seq_len), ctypes.c_float(scale), ctypes.byref(mods),
                                        _p(workspace),
                                        ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream))
    _check(st, "paged_attention_decode_mod")
    return out


def prepare_decode_step(k_cache, v_cache, k_new, v_new, q, block_table, seq_lens, max_seq_len: int, scale: float, *,
                        window: int = 0, softcap: float = 0.0, alibi_slopes=None, doc_ids=None, user_mod: int = 0,
                        user_data=None, out=None, lse=None, workspace=None, head_major=False,
                        stream=None) -> PreparedCall:
    """paged_decode_step (append of one new token per sequence + decode, one call) with its arguments marshalled once;
    the call returns ``out``."""
    lib = load_library()
    d = cache_desc(k_cache, v_cache, head_major)
    _dense(q, "q", k_cache.dtype)
    B, Hq, hd = q.shape
    if hd != d.head_dim or seq_lens.shape[0] != B or block_table.shape[0] != B:
        raise PagedAttnError("q must be [B, Hq, d] with B matching seq_lens and block_table")
    _dense(k_new, "k_new", k_cache.dtype), _dense(v_new, "v_new", k_cache.dtype)
    if tuple(k_new.shape) != (B, d.num_kv_heads, hd) or tuple(v_new.shape) != (B, d.num_kv_heads, hd):
        raise PagedAttnError("k_new / v_new must be [B, Hkv, d]")
    _i32(block_table, "block_table"), _i32(seq_lens, "seq_lens")
    out = _new(q.shape, q.dtype, q.device, stream) if out is None else _dense(out, "out", q.dtype)
    if lse is not None:
        _dense(lse, "lse", torch.float32)
    if workspace is None:
        workspace = _workspace(None, paged_attention_workspace_bytes(B, Hq, hd, B, max_seq_len), q.device, stream)
    m = _mods(window, softcap, alibi_slopes, doc_ids, Hq, B, user_mod, user_data)
    args = (ctypes.byref(d), _p(k_new), _p(v_new), _p(q), _p(out), _p(lse), _p(block_table), _p(seq_lens),
            ctypes.c_int32(B), ctypes.c_int32(Hq), ctypes.c_int32(block_table.shape[1]), ctypes.c_int32(max_seq_len),
            ctypes.c_float(scale), ctypes.byref(m), _p(workspace),
            ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream))
    return PreparedCall(lib.paged_decode_step, args,
                        (d, m, k_cache, v_cache, k_new, v_new, q, out, lse, block_table, seq_lens, workspace,
                         alibi_slopes, doc_ids, user_data), "paged_decode_step", out)


def paged_decode_step(k_cache, v_cache, k_new, v_new, q, block_table, seq_lens, max_seq_len: int, scale: float,
                      **kw):
    """Appends token s of ``k_new`` / ``v_new`` ([B, Hkv, d]) at position seq_lens[s] - 1 and decodes, in one call.
    Returns ``out``; keyword arguments as for prepare_decode_step."""
    return prepare_decode_step(k_cache, v_cache, k_new, v_new, q, block_table, seq_lens, max_seq_len, scale, **kw)()


def paged_attention_prefill_mod(k_cache, v_cache, q, cu_q_lens, max_q_len: int, block_table, seq_lens,
                                max_seq_len: int, scale: float, causal: bool, *, window: int = 0,
                                softcap: float = 0.0, alibi_slopes=None, doc_ids=None, user_mod: int = 0,
                                user_data=None, out=None, lse=None, workspace=None, head_major=False, stream=None):
    """paged_attention_prefill with mask / score modifications (see pa_attn_mods in the header)."""
    lib = load_library()
    d = cache_desc(k_cache, v_cache, head_major)
    _dense(q, "q", k_cache.dtype)
    total_q, Hq, hd = q.shape
    B = int(seq_lens.shape[0])
    if hd != d.head_dim or block_table.shape[0] != B or cu_q_lens.shape[0] != B + 1:
        raise PagedAttnError("q must be [total_q, Hq, d]; cu_q_lens int32[B+1]")
    _i32(block_table, "block_table"), _i32(seq_lens, "seq_lens"), _i32(cu_q_lens, "cu_q_lens")
    out = _new(q.shape, q.dtype, q.device, stream) if out is None else _dense(out, "out", q.dtype)
    if lse is not None:
        _dense(lse, "lse", torch.float32)
    mods = _mods(window, softcap, alibi_slopes, doc_ids, Hq, B, user_mod, user_data)
    workspace = _workspace(workspace, paged_attention_workspace_bytes(B, Hq, hd, total_q, max_seq_len), q.device, stream)
    st = lib.paged_attention_prefill_mod(ctypes.byref(d), _p(q), _p(out), _p(lse), _p(cu_q_lens),
                                         ctypes.c_int32(total_q), ctypes.c_int32(max_q_len), _p(block_table),
                                         _p(seq_lens), ctypes.c_int32(B), ctypes.c_int32(Hq),
                                         ctypes.c_int32(block_table.shape[1]), ctypes.c_int32(max_seq_len),
                                         ctypes.c_float(scale), ctypes.c_int32(1 if causal else 0),
                                         ctypes.byref(mods), _p(workspace),
                                         ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                                         _stream(stream))
    _check(st, "paged_attention_prefill_mod")
    return out


# ---- a step of drafted tokens (see the block of that name in include/pagedattn.h) -----------------------------------

def _together(what: str, *tensors) -> torch.device:
    """All tensors on the current device, whose stream the call goes to."""
    dev = None
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise PagedAttnError(f"{what}: every tensor must be a device tensor")
        if dev is not None and t.device != dev:
            raise PagedAttnError(f"{what}: tensors on {dev} and {t.device}")
        dev = t.device
    if dev is not None and dev.index != torch.cuda.current_device():
        raise PagedAttnError(f"{what}: tensors on {dev}, but the current device is cuda:{torch.cuda.current_device()}")
    return dev


def _shaped(t: torch.Tensor, what: str, shape, dtype=torch.int32) -> torch.Tensor:
    if t.dtype != dtype or not t.is_contiguous() or not t.is_cuda or tuple(t.shape) != tuple(shape):
        raise PagedAttnError(f"{what} must be a contiguous {dtype} device tensor of shape {list(shape)}, "
                             f"got {t.dtype} {list(t.shape)}")
    return t


def _or_new(t, what, shape, device, stream, dtype=torch.int32):
    return _new(shape, dtype, device, stream) if t is None else _shaped(t, what, shape, dtype)


class StepPlan(NamedTuple):
    """What paged_plan_step leaves: the arguments of the calls that follow."""
    seq_lens: torch.Tensor
    cu_q_lens: torch.Tensor
    seq_ids: torch.Tensor
    positions: torch.Tensor
    rope_positions: torch.Tensor
    tree_mask: Optional[torch.Tensor]    # None: left out
    shortage: torch.Tensor


def prepare_plan_step(ctx_lens, new_lens, block_table, num_blocks, free_pages, free_count, page_size: int, max_rows: int, *,
                      parents=None, mask_words: int = 1, seq_lens=None, cu_q_lens=None, seq_ids=None, positions=None,
                      rope_positions=None, tree_mask=None, shortage=None, stream=None) -> PreparedCall:
    """paged_plan_step with its arguments marshalled once; the call returns a StepPlan.  Outputs are allocated unless
    given (tree_mask: int64 [max_rows, mask_words], the bits of the header's uint64; mask_words=0 leaves the masks out, as for
    a prompt, whose tokens may then be more than masks have bits)."""
    lib = load_library()
    dev = _together("paged_plan_step", ctx_lens, new_lens, block_table, num_blocks, free_pages, free_count, parents, seq_lens,
                    cu_q_lens, seq_ids, positions, rope_positions, tree_mask, shortage)
    B = int(ctx_lens.shape[0])
    _i32(block_table, "block_table"), _i32(free_pages, "free_pages")
    if block_table.dim() != 2 or block_table.shape[0] != B or free_pages.dim() != 1:
        raise PagedAttnError("block_table must be [batch, max_blocks], free_pages one-dimensional")
    _shaped(ctx_lens, "ctx_lens", (B,)), _shaped(new_lens, "new_lens", (B,)), _shaped(num_blocks, "num_blocks", (B,))
    _shaped(free_count, "free_count", (1,))
    if parents is not None:
        _shaped(parents, "parents", (max_rows,))
    if tree_mask is not None:
        mask_words = int(tree_mask.shape[-1])
    plan = StepPlan(_or_new(seq_lens, "seq_lens", (B,), dev, stream), _or_new(cu_q_lens, "cu_q_lens", (B + 1,), dev, stream),
                    _or_new(seq_ids, "seq_ids", (max_rows,), dev, stream), _or_new(positions, "positions", (max_rows,), dev, stream),
                    _or_new(rope_positions, "rope_positions", (max_rows,), dev, stream),
                    _or_new(tree_mask, "tree_mask", (max_rows, mask_words), dev, stream, torch.int64) if mask_words else None,
                    _or_new(shortage, "shortage", (2,), dev, stream))
    args = (_p(ctx_lens), _p(new_lens), ctypes.c_int32(B), _p(parents), ctypes.c_int32(page_size), _p(block_table),
            ctypes.c_int32(block_table.shape[1]), _p(num_blocks), _p(free_pages), _p(free_count), ctypes.c_int32(max_rows),
            _p(plan.seq_lens), _p(plan.cu_q_lens), _p(plan.seq_ids), _p(plan.positions), _p(plan.rope_positions),
            _p(plan.tree_mask), ctypes.c_int32(mask_words), _p(plan.shortage), _stream(stream))
    return PreparedCall(lib.paged_plan_step, args, (ctx_lens, new_lens, parents, block_table, num_blocks, free_pages,
                                                    free_count, plan), "paged_plan_step", plan)


def paged_plan_step(ctx_lens, new_lens, block_table, num_blocks, free_pages, free_count, page_size: int, max_rows: int,
                    **kw) -> StepPlan:
    """Slots, positions, ancestor masks and pages of a step from the requests' lengths; block_table, num_blocks and
    free_count are updated in place.  Keyword arguments as for prepare_plan_step."""
    return prepare_plan_step(ctx_lens, new_lens, block_table, num_blocks, free_pages, free_count, page_size, max_rows,
                             **kw)()


def prepare_release_blocks(keep_lens, block_table, num_blocks, free_pages, free_count, page_size: int, *,
                           stream=None) -> PreparedCall:
    lib = load_library()
    _together("paged_release_blocks", keep_lens, block_table, num_blocks, free_pages, free_count)
    B = int(keep_lens.shape[0])
    _i32(block_table, "block_table"), _i32(free_pages, "free_pages")
    if block_table.dim() != 2 or block_table.shape[0] != B or free_pages.dim() != 1:
        raise PagedAttnError("block_table must be [batch, max_blocks], free_pages one-dimensional")
    _shaped(keep_lens, "keep_lens", (B,)), _shaped(num_blocks, "num_blocks", (B,)), _shaped(free_count, "free_count", (1,))
    args = (_p(keep_lens), ctypes.c_int32(B), ctypes.c_int32(page_size), _p(block_table), ctypes.c_int32(block_table.shape[1]),
            _p(num_blocks), _p(free_pages), _p(free_count), ctypes.c_int32(free_pages.shape[0]), _stream(stream))
    return PreparedCall(lib.paged_release_blocks, args, (keep_lens, block_table, num_blocks, free_pages, free_count),
                        "paged_release_blocks")


def paged_release_blocks(keep_lens, block_table, num_blocks, free_pages, free_count, page_size: int, *, stream=None) -> None:
    """Gives the pages behind the first keep_lens[s] tokens of each sequence back to the free list, in place.  Pages that the
    list has no room for stay mapped."""
    prepare_release_blocks(keep_lens, block_table, num_blocks, free_pages, free_count, page_size, stream=stream)()


PA_ROPE_SCALING = {"none": 0, "linear": 1, "base": 2, "parts": 3, "ramp": 4}


def pa_rope_frequencies(rotary_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                        context: float = 8192.0, slow: float = 1.0, fast: Optional[float] = None) -> Tuple[torch.Tensor, float]:
    """(float64 [rotary_dim / 2] on the host, radians a position; factor on the turned coordinates).  ``fast`` defaults to 4
    turns for "parts" and 32 for "ramp"."""
    if scaling not in PA_ROPE_SCALING:
        raise PagedAttnError(f"scaling must be one of {sorted(PA_ROPE_SCALING)}")
    out = torch.empty(max(int(rotary_dim) // 2, 1), dtype=torch.float64)
    mscale = ctypes.c_float(0.0)
    fast = (32.0 if scaling == "ramp" else 4.0) if fast is None else fast
    _check(load_library().pa_rope_frequencies(ctypes.c_void_p(out.data_ptr()), ctypes.byref(mscale), ctypes.c_int32(rotary_dim),
                                              ctypes.c_double(base), ctypes.c_int(PA_ROPE_SCALING[scaling]),
                                              ctypes.c_double(factor), ctypes.c_double(context), ctypes.c_double(slow),
                                              ctypes.c_double(fast)), "pa_rope_frequencies")
    return out, mscale.value


def _rows(t: torch.Tensor, what: str, shape, dtype) -> torch.Tensor:
    """[T, heads, d] whose tokens may lie apart (a part of one projection) but whose heads are contiguous."""
    if t.dtype != dtype or not t.is_cuda or tuple(t.shape) != tuple(shape) or \
            (t.numel() and (t.stride(2) != 1 or (t.shape[1] > 1 and t.stride(1) != t.shape[2]) or
                            (t.shape[0] > 1 and t.stride(0) < t.shape[1] * t.shape[2]))):
        raise PagedAttnError(f"{what} must be a {dtype} device tensor {list(shape)} with contiguous heads, tokens apart")
    return t


def _token_stride(t) -> ctypes.c_int64:
    return ctypes.c_int64(0 if t is None or t.shape[0] < 2 else t.stride(0))


def prepare_rope_append(k_cache, v_cache, q, k_new, v_new, rope_positions, seq_ids, positions, block_table, inv_freq, *,
                        interleaved: bool = False, mscale: float = 1.0, q_out=None, head_major=False,
                        stream=None) -> PreparedCall:
    """paged_rope_append with its arguments marshalled once; the call returns ``q_out`` (allocated unless given; may be q).
    q, or k_new and v_new with seq_ids, positions and block_table, may be None.  inv_freq: float64 [rotary_dim / 2] on the device."""
    lib = load_library()
    d = cache_desc(k_cache, v_cache, head_major)
    dev = _together("paged_rope_append", k_cache, v_cache, q, k_new, v_new, rope_positions, seq_ids, positions, block_table,
                    inv_freq, q_out)
    T = int(rope_positions.shape[0])
    _shaped(rope_positions, "rope_positions", (T,))
    if inv_freq.dim() != 1:
        raise PagedAttnError("inv_freq must be float64[rotary_dim / 2]")
    _shaped(inv_freq, "inv_freq", inv_freq.shape, torch.float64)
    Hq = 0
    if q is not None:
        Hq = int(q.shape[1]) if q.dim() == 3 else 0
        _rows(q, "q", (T, Hq, d.head_dim), k_cache.dtype)
        q_out = _new((T, Hq, d.head_dim), q.dtype, dev, stream) if q_out is None else \
            _rows(q_out, "q_out", (T, Hq, d.head_dim), q.dtype)
    elif q_out is not None:
        raise PagedAttnError("q_out without q")
    B = MB = 0
    if k_new is not None:
        if v_new is None or seq_ids is None or positions is None or block_table is None:
            raise PagedAttnError("k_new needs v_new, seq_ids, positions and block_table")
        _rows(k_new, "k_new", (T, d.num_kv_heads, d.head_dim), k_cache.dtype)
        _rows(v_new, "v_new", (T, d.num_kv_heads, d.head_dim), k_cache.dtype)
        _shaped(seq_ids, "seq_ids", (T,)), _shaped(positions, "positions", (T,)), _i32(block_table, "block_table")
        if block_table.dim() != 2:
            raise PagedAttnError("block_table must be [batch, max_blocks]")
        B, MB = block_table.shape
    elif v_new is not None:
        raise PagedAttnError("v_new without k_new")
    args = (ctypes.byref(d), _p(q), _token_stride(q), _p(q_out), _token_stride(q_out), ctypes.c_int32(Hq), _p(k_new),
            _token_stride(k_new), _p(v_new), _token_stride(v_new), _p(rope_positions), _p(seq_ids), _p(positions),
            ctypes.c_int32(T), _p(block_table), ctypes.c_int32(B), ctypes.c_int32(MB), _p(inv_freq),
            ctypes.c_int32(2 * inv_freq.shape[0]), ctypes.c_int32(1 if interleaved else 0), ctypes.c_float(mscale),
            _stream(stream))
    return PreparedCall(lib.paged_rope_append, args, (d, k_cache, v_cache, q, q_out, k_new, v_new, rope_positions, seq_ids,
                                                      positions, block_table, inv_freq), "paged_rope_append", q_out)


def paged_rope_append(k_cache, v_cache, q, k_new, v_new, rope_positions, seq_ids, positions, block_table, inv_freq, **kw):
    """Turns q and k_new by their positions, K and V into their pages.  Returns ``q_out``; keyword arguments as for
    prepare_rope_append."""
    return prepare_rope_append(k_cache, v_cache, q, k_new, v_new, rope_positions, seq_ids, positions, block_table, inv_freq,
                               **kw)()


def paged_attention_tree_workspace_bytes(batch: int, num_q_heads: int, num_kv_heads: int, head_dim: int, total_q: int,
                                         max_q_len: int, max_seq_len: int) -> int:
    return int(load_library().paged_attention_tree_workspace_bytes(
        ctypes.c_int32(batch), ctypes.c_int32(num_q_heads), ctypes.c_int32(num_kv_heads), ctypes.c_int32(head_dim),
        ctypes.c_int32(total_q), ctypes.c_int32(max_q_len), ctypes.c_int32(max_seq_len)))


def prepare_attention_tree(k_cache, v_cache, q, cu_q_lens, max_q_len: int, tree_mask, block_table, seq_lens, max_seq_len: int,
                           scale: float, *, out=None, lse=None, workspace=None, head_major=False,
                           stream=None) -> PreparedCall:
    """paged_attention_tree with its arguments marshalled once; the call returns ``out``.  tree_mask: int64 [total_q, words]."""
    lib = load_library()
    d = cache_desc(k_cache, v_cache, head_major)
    dev = _together("paged_attention_tree", k_cache, v_cache, q, cu_q_lens, tree_mask, block_table, seq_lens, out, lse, workspace)
    _dense(q, "q", k_cache.dtype)
    if q.dim() != 3 or q.shape[2] != d.head_dim:
        raise PagedAttnError("q must be [total_q, Hq, d]")
    total_q, Hq, hd = q.shape
    B = int(seq_lens.shape[0])
    _shaped(seq_lens, "seq_lens", (B,)), _shaped(cu_q_lens, "cu_q_lens", (B + 1,)), _i32(block_table, "block_table")
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise PagedAttnError("block_table must be [batch, max_blocks]")
    if tree_mask.dim() != 2:
        raise PagedAttnError("tree_mask must be int64[total_q, words]")
    words = int(tree_mask.shape[1])
    _shaped(tree_mask, "tree_mask", (total_q, words), torch.int64)
    out = _new(q.shape, q.dtype, q.device, stream) if out is None else _shaped(out, "out", q.shape, q.dtype)
    if lse is not None:
        _shaped(lse, "lse", (total_q, Hq), torch.float32)
    if workspace is None:
        workspace = _workspace(None, paged_attention_tree_workspace_bytes(B, Hq, d.num_kv_heads, hd, total_q, max_q_len,
                                                                          max_seq_len), dev, stream)
    args = (ctypes.byref(d), _p(q), _p(out), _p(lse), _p(cu_q_lens), ctypes.c_int32(total_q), ctypes.c_int32(max_q_len),
            _p(tree_mask), ctypes.c_int32(words), _p(block_table), _p(seq_lens), ctypes.c_int32(B), ctypes.c_int32(Hq),
            ctypes.c_int32(block_table.shape[1]), ctypes.c_int32(max_seq_len), ctypes.c_float(scale), _p(workspace),
            ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream))
    return PreparedCall(lib.paged_attention_tree, args,
                        (d, k_cache, v_cache, q, out, lse, cu_q_lens, tree_mask, block_table, seq_lens, workspace),
                        "paged_attention_tree", out)


def paged_attention_tree(k_cache, v_cache, q, cu_q_lens, max_q_len: int, tree_mask, block_table, seq_lens, max_seq_len: int,
                         scale: float, **kw):
    """Attention of trees of drafted tokens.  Returns ``out`` ([total_q, Hq, d], dtype of q); keyword arguments as for
    prepare_attention_tree."""
    return prepare_attention_tree(k_cache, v_cache, q, cu_q_lens, max_q_len, tree_mask, block_table, seq_lens, max_seq_len,
                                  scale, **kw)()


def prepare_tree_accept(k_cache, v_cache, cu_q_lens, seq_lens, max_q_len: int, block_table, path, path_lens, *, parents=None,
                        tokens=None, targets=None, next_tokens=None, kept_lens=None, head_major=False,
                        stream=None) -> PreparedCall:
    """paged_tree_accept with its arguments marshalled once; the call returns (path, path_lens, next_tokens, kept_lens), the last
    two allocated unless given.  path: int32 [batch, max_path].  Without parents, tokens and targets path and path_lens are read."""
    lib = load_library()
    d = cache_desc(k_cache, v_cache, head_major)
    dev = _together("paged_tree_accept", k_cache, v_cache, cu_q_lens, seq_lens, block_table, path, path_lens, parents, tokens,
                    targets, next_tokens, kept_lens)
    B = int(seq_lens.shape[0])
    _shaped(seq_lens, "seq_lens", (B,)), _shaped(cu_q_lens, "cu_q_lens", (B + 1,)), _i32(block_table, "block_table")
    if path.dim() != 2 or block_table.dim() != 2 or block_table.shape[0] != B:
        raise PagedAttnError("path must be [batch, max_path], block_table [batch, max_blocks]")
    _shaped(path, "path", (B, path.shape[1])), _shaped(path_lens, "path_lens", (B,))
    given = tokens is None
    if (targets is None) != given or (parents is None) != given or (given and next_tokens is not None):
        raise PagedAttnError("parents, tokens and targets come together, next_tokens with them")
    if not given:
        for t, what in ((parents, "parents"), (tokens, "tokens"), (targets, "targets")):
            if _i32(t, what).dim() != 1 or t.shape != tokens.shape:
                raise PagedAttnError("parents, tokens and targets must be int32[rows], equally long")
        next_tokens = _or_new(next_tokens, "next_tokens", (B,), dev, stream)
    kept_lens = _or_new(kept_lens, "kept_lens", (B,), dev, stream)
    args = (ctypes.byref(d), _p(cu_q_lens), _p(seq_lens), ctypes.c_int32(B), ctypes.c_int32(max_q_len), _p(parents), _p(tokens),
            _p(targets), _p(path), ctypes.c_int32(path.shape[1]), _p(path_lens), _p(next_tokens), _p(kept_lens),
            _p(block_table), ctypes.c_int32(block_table.shape[1]), _stream(stream))
    return PreparedCall(lib.paged_tree_accept, args, (d, k_cache, v_cache, cu_q_lens, seq_lens, block_table, path, path_lens,
                                                      parents, tokens, targets, next_tokens, kept_lens), "paged_tree_accept",
                        (path, path_lens, next_tokens, kept_lens))


def paged_tree_accept(k_cache, v_cache, cu_q_lens, seq_lens, max_q_len: int, block_table, path, path_lens, **kw):
    """Finds what stays of a verified tree and moves its K and V rows together.  Returns (path, path_lens, next_tokens,
    kept_lens); keyword arguments as for prepare_tree_accept."""
    return prepare_tree_accept(k_cache, v_cache, cu_q_lens, seq_lens, max_q_len, block_table, path, path_lens, **kw)()


# ---- normalised heads, positions of several numbers, the 4-bit cache (see the block of that name in include/pagedattn.h) -------

class _NormRope(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "q_out", "k_new", "v_new")] + \
        [(n, ctypes.c_int64) for n in ("q_stride", "q_out_stride", "k_stride", "v_stride")] + \
        [(n, ctypes.c_void_p) for n in ("rope_positions", "pair_axes", "inv_freq", "q_weight", "k_weight", "seq_ids", "positions",
                                        "block_table")] + \
        [(n, ctypes.c_int32) for n in ("num_q_heads", "T", "batch", "max_blocks", "axes", "rotary_dim", "interleaved", "norm_q", "norm_k",
                                       "q_weight_heads", "k_weight_heads", "weight_dtype")] + \
        [(n, ctypes.c_float) for n in ("eps", "weight_offset", "mscale")]


class _Mx4Desc(ctypes.Structure):
    _fields_ = [("records", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


def pa_mx4_record_bytes(page_size: int, head_dim: int) -> int:
    return int(load_library().pa_mx4_record_bytes(ctypes.c_int32(page_size), ctypes.c_int32(head_dim)))


def pa_mx4_cache(num_pages: int, page_size: int, num_kv_heads: int, head_dim: int, device="cuda") -> torch.Tensor:
    """An empty 4-bit cache: uint8 [num_pages, num_kv_heads, page_size, 17/16 head_dim], a page's record of a KV head in the last two
    dimensions (not token by token: the layout is the header's).  A shape that calls check against their tensors'."""
    size = pa_mx4_record_bytes(page_size, head_dim)
    if size == 0:
        raise PagedAttnError("a 4-bit cache has pages of 16 tokens or more, a power of two, and head_dim 64, 128 or 256; "
                             f"got {page_size} and {head_dim}")
    return torch.empty((num_pages, num_kv_heads, page_size, size // page_size), dtype=torch.uint8, device=device)


def mx4_desc(cache: torch.Tensor, head_dim: int) -> _Mx4Desc:
    """Descriptor of a 4-bit cache: uint8 [num_pages, Hkv, page_size, 17/16 head_dim] as of pa_mx4_cache, or [num_pages, Hkv, record],
    whose record's size gives the tokens of a page once the head_dim is known."""
    if cache.dtype != torch.uint8 or cache.dim() not in (3, 4) or not cache.is_cuda or cache.stride(-1) != 1 or \
            (cache.dim() == 4 and cache.stride(2) != cache.shape[3]):
        raise PagedAttnError("a 4-bit cache is a uint8 device tensor [num_pages, Hkv, page_size, 17/16 head_dim] or "
                             "[num_pages, Hkv, record] with contiguous records")
    NP, Hkv = cache.shape[:2]
    size = cache.shape[2] if cache.dim() == 3 else cache.shape[2] * cache.shape[3]
    page = (size * 16 // (17 * head_dim) if head_dim > 0 else 0) if cache.dim() == 3 else cache.shape[2]
    if size == 0 or pa_mx4_record_bytes(page, head_dim) != size:
        raise PagedAttnError(f"records of {size} bytes, {list(cache.shape)}, hold no page of heads of {head_dim}")
    return _Mx4Desc(cache.data_ptr(), cache.stride(0) if NP > 1 else Hkv * size, cache.stride(1) if Hkv > 1 else size, NP, page, Hkv,
                    head_dim)


def _weights(w, what, heads, d, dtype):
    """(pointer, [heads, d] and not [d])"""
    if w is None:
        return 0, 0
    if w.dtype not in (dtype, torch.float32) or not w.is_contiguous() or tuple(w.shape) not in ((d,), (heads, d)):
        raise PagedAttnError(f"{what} must be a contiguous {dtype} or float32 tensor [{d}] or [{heads}, {d}], got {w.dtype} {list(w.shape)}")
    return w.data_ptr(), int(w.dim() == 2)


def _norm_rope(what, caches, Hkv, d, dtype, q, k_new, v_new, rope_positions, seq_ids, positions, block_table, inv_freq, q_weight, k_weight, eps,
               weight_offset, norm_q, norm_k, pair_axes, interleaved, mscale, q_out, stream):
    dev = _together(what, *caches, q, k_new, v_new, rope_positions, seq_ids, positions, block_table, inv_freq, q_weight, k_weight, pair_axes,
                    q_out)
    if rope_positions.dim() not in (1, 2):
        raise PagedAttnError("rope_positions must be int32[T] or [axes, T]")
    T = int(rope_positions.shape[-1])
    axes = int(rope_positions.shape[0]) if rope_positions.dim() == 2 else 1
    _shaped(rope_positions, "rope_positions", rope_positions.shape)
    if inv_freq.dim() != 1:
        raise PagedAttnError("inv_freq must be float64[rotary_dim / 2]")
    _shaped(inv_freq, "inv_freq", inv_freq.shape, torch.float64)
    if pair_axes is not None:
        _shaped(pair_axes, "pair_axes", inv_freq.shape)
    elif axes > 1:
        raise PagedAttnError("positions of several numbers need pair_axes")
    Hq = 0
    if q is not None:
        Hq = int(q.shape[1]) if q.dim() == 3 else 0
        _rows(q, "q", (T, Hq, d), dtype)
        q_out = _new((T, Hq, d), dtype, dev, stream) if q_out is None else _rows(q_out, "q_out", (T, Hq, d), dtype)
    elif q_out is not None:
        raise PagedAttnError("q_out without q")
    B = MB = 0
    if k_new is not None:
        if v_new is None or seq_ids is None or positions is None or block_table is None:
            raise PagedAttnError("k_new needs v_new, seq_ids, positions and block_table")
        _rows(k_new, "k_new", (T, Hkv, d), dtype)
        _rows(v_new, "v_new", (T, Hkv, d), dtype)
        _shaped(seq_ids, "seq_ids", (T,)), _shaped(positions, "positions", (T,)), _i32(block_table, "block_table")
        if block_table.dim() != 2:
            raise PagedAttnError("block_table must be [batch, max_blocks]")
        B, MB = block_table.shape
    elif v_new is not None:
        raise PagedAttnError("v_new without k_new")
    qw, qw_heads = _weights(q_weight, "q_weight", Hq, d, dtype)
    kw, kw_heads = _weights(k_weight, "k_weight", Hkv, d, dtype)
    kinds = {w.dtype for w in (q_weight, k_weight) if w is not None}
    if len(kinds) > 1:
        raise PagedAttnError("q_weight and k_weight must be of one type")

    def ptr(t):
        return 0 if t is None else t.data_ptr()

    def apart(t):
        return 0 if t is None or t.shape[0] < 2 else t.stride(0)

    r = _NormRope(ptr(q), ptr(q_out), ptr(k_new), ptr(v_new), apart(q), apart(q_out), apart(k_new), apart(v_new), ptr(rope_positions),
                  ptr(pair_axes), ptr(inv_freq), qw, kw, ptr(seq_ids), ptr(positions), ptr(block_table), Hq, T, B, MB, axes,
                  2 * inv_freq.shape[0], int(bool(interleaved)), int(bool(norm_q)), int(bool(norm_k)), qw_heads, kw_heads,
                  PA_DTYPE[kinds.pop() if kinds else dtype], eps, weight_offset, mscale)
    keep = (r, caches, q, q_out, k_new, v_new, rope_positions, pair_axes, inv_freq, q_weight, k_weight, seq_ids, positions, block_table)
    return r, keep, q_out


def prepare_norm_rope_append(k_cache, v_cache, q, k_new, v_new, rope_positions, seq_ids, positions, block_table, inv_freq, *, q_weight=None,
                             k_weight=None, eps: float = 1e-6, weight_offset: float = 0.0, norm_q: bool = True, norm_k: bool = True,
                             pair_axes=None, interleaved: bool = False, mscale: float = 1.0, q_out=None, head_major=False,
                             stream=None) -> PreparedCall:
    """paged_norm_rope_append with its arguments marshalled once; the call returns ``q_out`` (allocated unless given; may be q).
    rope_positions: int32 [T], or [axes, T] with pair_axes int32 [rotary_dim / 2].  q_weight, k_weight: [d] or [heads, d].  The rest as
    for prepare_rope_append."""
    lib = load_library()
    d = cache_desc(k_cache, v_cache, head_major)
    r, keep, q_out = _norm_rope("paged_norm_rope_append", (k_cache, v_cache), d.num_kv_heads, d.head_dim, k_cache.dtype, q, k_new, v_new,
                                rope_positions, seq_ids, positions, block_table, inv_freq, q_weight, k_weight, eps, weight_offset, norm_q,
                                norm_k, pair_axes, interleaved, mscale, q_out, stream)
    return PreparedCall(lib.paged_norm_rope_append, (ctypes.byref(d), ctypes.byref(r), _stream(stream)), (d, keep),
                        "paged_norm_rope_append", q_out)


def paged_norm_rope_append(k_cache, v_cache, q, k_new, v_new, rope_positions, seq_ids, positions, block_table, inv_freq, **kw):
    """Norms of the heads of q and k_new, their rotary positions, K and V into their pages.  Returns ``q_out``; keyword arguments as
    for prepare_norm_rope_append."""
    return prepare_norm_rope_append(k_cache, v_cache, q, k_new, v_new, rope_positions, seq_ids, positions, block_table, inv_freq, **kw)()


def prepare_norm_rope_append_mx4(cache, q, k_new, v_new, rope_positions, seq_ids, positions, block_table, inv_freq, *, q_weight=None,
                                 k_weight=None, eps: float = 1e-6, weight_offset: float = 0.0, norm_q: bool = True, norm_k: bool = True,
                                 pair_axes=None, interleaved: bool = False, mscale: float = 1.0, q_out=None,
                                 stream=None) -> PreparedCall:
    """prepare_norm_rope_append into a 4-bit cache (pa_mx4_cache)."""
    lib = load_library()
    x = q if q is not None else k_new
    if x is None or x.dim() != 3 or x.dtype not in PA_DTYPE:
        raise PagedAttnError("q or k_new must be a float32, bfloat16 or float16 tensor [T, heads, d]")
    d = mx4_desc(cache, int(x.shape[2]))
    r, keep, q_out = _norm_rope("paged_norm_rope_append_mx4", (cache,), d.num_kv_heads, d.head_dim, x.dtype, q, k_new, v_new, rope_positions,
                                seq_ids, positions, block_table, inv_freq, q_weight, k_weight, eps, weight_offset, norm_q, norm_k, pair_axes,
                                interleaved, mscale, q_out, stream)
    return PreparedCall(lib.paged_norm_rope_append_mx4, (ctypes.byref(d), ctypes.c_int32(PA_DTYPE[x.dtype]), ctypes.byref(r), _stream(stream)),
                        (d, keep), "paged_norm_rope_append_mx4", q_out)


def paged_norm_rope_append_mx4(cache, q, k_new, v_new, rope_positions, seq_ids, positions, block_table, inv_freq, **kw):
    """paged_norm_rope_append into a 4-bit cache.  Returns ``q_out``; keyword arguments as for prepare_norm_rope_append_mx4."""
    return prepare_norm_rope_append_mx4(cache, q, k_new, v_new, rope_positions, seq_ids, positions, block_table, inv_freq, **kw)()


def prepare_kv_append_mx4(cache, k_new, v_new, seq_ids, positions, block_table, *, stream=None) -> PreparedCall:
    """paged_kv_append_mx4 with its arguments marshalled once.  k_new, v_new: [T, Hkv, d], contiguous."""
    lib = load_library()
    _together("paged_kv_append_mx4", cache, k_new, v_new, seq_ids, positions, block_table)
    if k_new.dim() != 3 or k_new.dtype not in PA_DTYPE:
        raise PagedAttnError("k_new must be a float32, bfloat16 or float16 tensor [T, Hkv, d]")
    d = mx4_desc(cache, int(k_new.shape[2]))
    _dense(k_new, "k_new", k_new.dtype), _dense(v_new, "v_new", k_new.dtype)
    T = int(k_new.shape[0])
    if k_new.shape[1] != d.num_kv_heads or k_new.shape != v_new.shape:
        raise PagedAttnError("k_new/v_new must be [T, Hkv, d]")
    _shaped(seq_ids, "seq_ids", (T,)), _shaped(positions, "positions", (T,)), _i32(block_table, "block_table")
    if block_table.dim() != 2:
        raise PagedAttnError("block_table must be [batch, max_blocks]")
    args = (ctypes.byref(d), ctypes.c_int32(PA_DTYPE[k_new.dtype]), _p(k_new), _p(v_new), _p(seq_ids), _p(positions), ctypes.c_int32(T),
            _p(block_table), ctypes.c_int32(block_table.shape[0]), ctypes.c_int32(block_table.shape[1]), _stream(stream))
    return PreparedCall(lib.paged_kv_append_mx4, args, (d, cache, k_new, v_new, seq_ids, positions, block_table), "paged_kv_append_mx4")


def paged_kv_append_mx4(cache, k_new, v_new, seq_ids, positions, block_table, *, stream=None) -> None:
    """K and V rows into their pages of a 4-bit cache."""
    prepare_kv_append_mx4(cache, k_new, v_new, seq_ids, positions, block_table, stream=stream)()


def prepare_kv_gather_mx4(cache, block_table, seq_lens, *, cu_lens, max_seq_len: int, out_k, out_v, first_lens=None,
                          stream=None) -> PreparedCall:
    """paged_kv_gather_mx4 with its arguments marshalled once; the call returns (out_k, out_v), [rows, Hkv, d] of a type of the caller's."""
    lib = load_library()
    _together("paged_kv_gather_mx4", cache, block_table, first_lens, seq_lens, cu_lens, out_k, out_v)
    if out_k.dim() != 3 or out_k.dtype not in PA_DTYPE:
        raise PagedAttnError("out_k must be a float32, bfloat16 or float16 tensor [rows, Hkv, d]")
    d = mx4_desc(cache, int(out_k.shape[2]))
    _dense(out_k, "out_k", out_k.dtype), _dense(out_v, "out_v", out_k.dtype)
    if out_k.shape[1] != d.num_kv_heads or out_k.shape != out_v.shape:
        raise PagedAttnError("out_k/out_v must be [rows, Hkv, d]")
    B = int(seq_lens.shape[0])
    _shaped(seq_lens, "seq_lens", (B,)), _shaped(cu_lens, "cu_lens", (B + 1,)), _i32(block_table, "block_table")
    if first_lens is not None:
        _shaped(first_lens, "first_lens", (B,))
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise PagedAttnError("block_table must be [batch, max_blocks]")
    args = (ctypes.byref(d), ctypes.c_int32(PA_DTYPE[out_k.dtype]), _p(out_k), _p(out_v),
            ctypes.c_int32(out_k.shape[0]), _p(block_table), _p(first_lens), _p(seq_lens), _p(cu_lens), ctypes.c_int32(B),
            ctypes.c_int32(block_table.shape[1]), ctypes.c_int32(max_seq_len), _stream(stream))
    return PreparedCall(lib.paged_kv_gather_mx4, args, (d, cache, block_table, first_lens, seq_lens, cu_lens, out_k, out_v),
                        "paged_kv_gather_mx4", (out_k, out_v))


def paged_kv_gather_mx4(cache, block_table, seq_lens, *, cu_lens, max_seq_len: int, out_k, out_v, first_lens=None, stream=None):
    """What a 4-bit cache holds of the sequences (from token first_lens[s] on).  Returns (out_k, out_v)."""
    return prepare_kv_gather_mx4(cache, block_table, seq_lens, cu_lens=cu_lens, max_seq_len=max_seq_len, out_k=out_k, out_v=out_v,
                                 first_lens=first_lens, stream=stream)()


def paged_attention_mx4_workspace_bytes(batch: int, num_q_heads: int, num_kv_heads: int, head_dim: int, total_q: int, max_q_len: int,
                                        max_seq_len: int) -> int:
    return int(load_library().paged_attention_mx4_workspace_bytes(
        ctypes.c_int32(batch), ctypes.c_int32(num_q_heads), ctypes.c_int32(num_kv_heads), ctypes.c_int32(head_dim),
        ctypes.c_int32(total_q), ctypes.c_int32(max_q_len), ctypes.c_int32(max_seq_len)))


def prepare_attention_mx4(cache, q, cu_q_lens, max_q_len: int, block_table, seq_lens, max_seq_len: int, scale: float, *, out=None, lse=None,
                          workspace=None, stream=None) -> PreparedCall:
    """paged_attention_mx4 with its arguments marshalled once; the call returns ``out``."""
    lib = load_library()
    dev = _together("paged_attention_mx4", cache, q, cu_q_lens, block_table, seq_lens, out, lse, workspace)
    if q.dim() != 3 or q.dtype not in PA_DTYPE:
        raise PagedAttnError("q must be a float32, bfloat16 or float16 tensor [total_q, Hq, d]")
    _dense(q, "q", q.dtype)
    d = mx4_desc(cache, int(q.shape[2]))
    total_q, Hq, hd = q.shape
    B = int(seq_lens.shape[0])
    _shaped(seq_lens, "seq_lens", (B,)), _shaped(cu_q_lens, "cu_q_lens", (B + 1,)), _i32(block_table, "block_table")
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise PagedAttnError("block_table must be [batch, max_blocks]")
    out = _new(q.shape, q.dtype, q.device, stream) if out is None else _shaped(out, "out", q.shape, q.dtype)
    if lse is not None:
        _shaped(lse, "lse", (total_q, Hq), torch.float32)
    if workspace is None:
        workspace = _workspace(None, paged_attention_mx4_workspace_bytes(B, Hq, d.num_kv_heads, hd, total_q, max_q_len, max_seq_len), dev,
                               stream)
    args = (ctypes.byref(d), ctypes.c_int32(PA_DTYPE[q.dtype]), _p(q), _p(out), _p(lse), _p(cu_q_lens), ctypes.c_int32(total_q),
            ctypes.c_int32(max_q_len), _p(block_table), _p(seq_lens), ctypes.c_int32(B), ctypes.c_int32(Hq),
            ctypes.c_int32(block_table.shape[1]), ctypes.c_int32(max_seq_len), ctypes.c_float(scale), _p(workspace),
            ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream))
    return PreparedCall(lib.paged_attention_mx4, args, (d, cache, q, out, lse, cu_q_lens, block_table, seq_lens, workspace),
                        "paged_attention_mx4", out)


def paged_attention_mx4(cache, q, cu_q_lens, max_q_len: int, block_table, seq_lens, max_seq_len: int, scale: float, **kw):
    """Attention of the sequences' last tokens over a 4-bit cache.  Returns ``out`` ([total_q, Hq, d], dtype of q); keyword arguments as
    for prepare_attention_mx4."""
    return prepare_attention_mx4(cache, q, cu_q_lens, max_q_len, block_table, seq_lens, max_seq_len, scale, **kw)()


def pa_debug_check(k_cache, v_cache, block_table, seq_lens, seq_ids=None, positions=None, *, head_major=False,
                   stream=None) -> Tuple[int, int, int]:
    """Counts of violated device-side preconditions: (page ids out of range, lengths out of range, appended tokens
    out of range).  Synchronises the stream."""
    d = cache_desc(k_cache, v_cache, head_major)
    _i32(block_table, "block_table"), _i32(seq_lens, "seq_lens")
    T = 0
    if seq_ids is not None:
        _i32(seq_ids, "seq_ids"), _i32(positions, "positions")
        T = int(seq_ids.shape[0])
    scratch = _new(4, torch.int64, k_cache.device, stream)
    counts = (ctypes.c_int64 * 3)()
    st = load_library().pa_debug_check(ctypes.byref(d), _p(block_table), _p(seq_lens),
                                       ctypes.c_int32(block_table.shape[0]), ctypes.c_int32(block_table.shape[1]),
                                       _p(seq_ids), _p(positions), ctypes.c_int32(T), _p(scratch), counts,
                                       _stream(stream))
    _check(st, "pa_debug_check")
    return int(counts[0]), int(counts[1]), int(counts[2])


def pa_set_option(name: str, value: int) -> None:
    _check(load_library().pa_set_option(name.encode(), ctypes.c_int64(value)), f"pa_set_option({name})")


def pa_stream_read(a: torch.Tensor, b: torch.Tensor, bytes_each: int, sink: torch.Tensor, *, stream=None) -> None:
    """Plain contiguous read of the first ``bytes_each`` bytes of two device tensors (bandwidth yardstick)."""
    if a.numel() * a.element_size() < bytes_each or b.numel() * b.element_size() < bytes_each:
        raise PagedAttnError("pa_stream_read: buffers shorter than bytes_each")
    _check(load_library().pa_stream_read(_p(a), _p(b), ctypes.c_size_t(bytes_each), _p(sink), _stream(stream)),
           "pa_stream_read")


def pa_profile_enable(on: bool) -> None:
    _check(load_library().pa_profile_enable(ctypes.c_int32(1 if on else 0)), "pa_profile_enable")


def pa_profile_reset() -> None:
    _check(load_library().pa_profile_reset(), "pa_profile_reset")


def pa_profile_read(kernel_prefix: str) -> Tuple[int, float]:
    n = ctypes.c_int32(0)
    ms = ctypes.c_double(0.0)
    _check(load_library().pa_profile_read(kernel_prefix.encode(), ctypes.byref(n), ctypes.byref(ms)),
           "pa_profile_read")
    return n.value, ms.value


# ---- KV page manager (host object; see the pa_pool_* block of include/pagedattn.h) ----------------------------

class PoolHandle(ctypes.c_void_p):
    """Opaque pa_pool*; remembers whether a device table is attached (then calls take the current stream)."""
    on_device = False


def pa_pool_create(num_pages: int, page_size: int, max_seqs: int, max_blocks: int,
                   device_table: Optional[torch.Tensor] = None) -> PoolHandle:
    """Returns the pool handle.  device_table: int32 [max_seqs, max_blocks] device tensor kept current by the pool,
    or None for a host-only pool (no GPU needed)."""
    if device_table is not None:
        _i32(device_table, "device_table")
        if tuple(device_table.shape) != (max_seqs, max_blocks):
            raise PagedAttnError("device_table must have shape [max_seqs, max_blocks]")
    handle = PoolHandle(0)
    handle.on_device = device_table is not None
    _check(load_library().pa_pool_create(ctypes.byref(handle), ctypes.c_int32(num_pages), ctypes.c_int32(page_size),
                                         ctypes.c_int32(max_seqs), ctypes.c_int32(max_blocks), _p(device_table)),
           "pa_pool_create")
    return handle


def pa_pool_destroy(pool) -> None:
    _check(load_library().pa_pool_destroy(pool), "pa_pool_destroy")


PA_GROW_EXACT, PA_GROW_POW2 = 0, 1


def pa_pool_set_growth(pool, policy: int) -> None:
    _check(load_library().pa_pool_set_growth(pool, ctypes.c_int32(policy)), "pa_pool_set_growth")


def _pool_stream(pool, stream) -> ctypes.c_void_p:
    return _stream(stream) if pool.on_device else ctypes.c_void_p(0)


def pa_pool_reserve(pool, seq: int, length: int, *, stream=None) -> None:
    _check(load_library().pa_pool_reserve(pool, ctypes.c_int32(seq), ctypes.c_int32(length),
                                          _pool_stream(pool, stream)), "pa_pool_reserve")


def pa_pool_release(pool, seq: int, *, stream=None) -> None:
    _check(load_library().pa_pool_release(pool, ctypes.c_int32(seq), _pool_stream(pool, stream)),
           "pa_pool_release")


def pa_pool_share_prefix(pool, dst_seq: int, src_seq: int, prefix_tokens: int, *, stream=None) -> None:
    _check(load_library().pa_pool_share_prefix(pool, ctypes.c_int32(dst_seq), ctypes.c_int32(src_seq),
                                               ctypes.c_int32(prefix_tokens), _pool_stream(pool, stream)),
           "pa_pool_share_prefix")


def pa_pool_make_writable(pool, k_cache, v_cache, seq: int, position: int, *, head_major=False, stream=None) -> None:
    desc = cache_desc(k_cache, v_cache, head_major)
    _check(load_library().pa_pool_make_writable(pool, ctypes.byref(desc), ctypes.c_int32(seq),
                                                ctypes.c_int32(position), _stream(stream)), "pa_pool_make_writable")


def pa_pool_make_writable_mx4(pool, cache, seq: int, position: int, *, head_dim: Optional[int] = None, stream=None) -> None:
    """head_dim: of a cache [num_pages, Hkv, record], whose shape does not say it."""
    if head_dim is None:
        if cache.dim() != 4:
            raise PagedAttnError("pa_pool_make_writable_mx4: a cache [num_pages, Hkv, record] needs head_dim")
        head_dim = cache.shape[3] * 16 // 17
    desc = mx4_desc(cache, head_dim)
    _check(load_library().pa_pool_make_writable_mx4(pool, ctypes.byref(desc), ctypes.c_int32(seq), ctypes.c_int32(position),
                                                    _stream(stream)), "pa_pool_make_writable_mx4")


def pa_pool_num_free(pool) -> int:
    return load_library().pa_pool_num_free(pool)


def pa_pool_num_blocks(pool, seq: int) -> int:
    return load_library().pa_pool_num_blocks(pool, ctypes.c_int32(seq))


def pa_pool_get_row(pool, seq: int):
    """The sequence's mapped pages, in block order, as a list of ints."""
    n = pa_pool_num_blocks(pool, seq)
    if n < 0:
        raise PagedAttnError("pa_pool_get_row: invalid sequence")
    row = (ctypes.c_int32 * max(n, 1))()
    _check(load_library().pa_pool_get_row(pool, ctypes.c_int32(seq), row, ctypes.c_int32(n)), "pa_pool_get_row")
    return list(row[:n])


def pa_pool_refcount(pool, page: int) -> int:
    return load_library().pa_pool_refcount(pool, ctypes.c_int32(page))
