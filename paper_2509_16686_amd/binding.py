"""Thin ctypes binding of libegmla.so.

Argument marshalling only: every step of append / decode / prefill runs in
the library's HIP kernels.  Tensors are torch tensors on the GPU (torch is
used for device memory and streams); bf16 storage is ``torch.bfloat16``.
The functions carry the C entry points' names without the ``eg_mla_``
prefix.  If the library is missing this module raises; there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libegmla.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = range(5)
FP32, BF16 = 0, 1
PATH_AUTO, PATH_VALU, PATH_MFMA = 0, 1, 2

# Every symbol include/eg_mla.h declares.
EXPORTS = ["eg_mla_status_string", "eg_mla_check_dims", "eg_mla_append", "eg_mla_decode_workspace_size",
           "eg_mla_decode", "eg_mla_decode_planned", "eg_mla_gate_rows", "eg_mla_prefill_workspace_size",
           "eg_mla_prefill_ref", "eg_mla_prefill_varlen_workspace_size", "eg_mla_prefill_varlen",
           "eg_mla_decode_literal_workspace_size", "eg_mla_decode_literal", "eg_mla_decode_noalloc",
           "eg_mla_append_workspace_size", "eg_mla_append_ws", "eg_mla_gate_table_marks_size",
           "eg_mla_gate_table", "eg_mla_page_plan", "eg_mla_page_release", "eg_mla_qk_norm_rope",
           "eg_mla_decode_shared_workspace_size", "eg_mla_decode_shared", "eg_mla_page_means",
           "eg_mla_page_scores_workspace_size", "eg_mla_page_scores", "eg_mla_select_pages",
           "eg_mla_rope_frequencies", "eg_mla_rope_rows", "eg_mla_quant_row_bytes", "eg_mla_quant_write", "eg_mla_quant_read",
           "eg_mla_quant_attend_workspace_size", "eg_mla_quant_attend"]
NOALLOC_SCRATCH_BYTES = 32 << 20  # EG_MLA_NOALLOC_SCRATCH_BYTES
LITERAL_NO_LN, LITERAL_ADD = 1, 2
ROPE_PAIRS, ROPE_HALF = 0, 1


class Dims(ctypes.Structure):
    _fields_ = [("num_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("v_head_dim", ctypes.c_int32),
                ("latent_dim", ctypes.c_int32), ("rope_dim", ctypes.c_int32), ("gate_dim", ctypes.c_int32),
                ("vocab_size", ctypes.c_int32), ("page_size", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
                ("dtype", ctypes.c_int32)]


class Plan(ctypes.Structure):
    _fields_ = [("path", ctypes.c_int32), ("split_tokens", ctypes.c_int32),
                ("split_start_event", ctypes.c_void_p), ("split_stop_event", ctypes.c_void_p),
                ("id_slices", ctypes.c_int32)]


class Rope(ctypes.Structure):
    """eg_mla_rope; `frequencies` points into an array that make_rope keeps beside it."""
    _fields_ = [("layout", ctypes.c_int32), ("theta", ctypes.c_float),
                ("frequencies", ctypes.POINTER(ctypes.c_double)), ("magnitude", ctypes.c_float)]


class EgMlaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libegmla.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2509_16686_amd.build`")
    # torch first: its HIP runtime carries the same SONAME, so the library binds to that one instance
    import torch  # noqa: F401
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    pd, pp = ctypes.POINTER(Dims), ctypes.POINTER(Plan)
    L.eg_mla_status_string.restype = ctypes.c_char_p
    L.eg_mla_status_string.argtypes = [ctypes.c_int]
    L.eg_mla_check_dims.restype = ctypes.c_int
    L.eg_mla_check_dims.argtypes = [pd]
    L.eg_mla_append.restype = ctypes.c_int
    L.eg_mla_append.argtypes = [pd, i32, i32, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, i64, vp]
    L.eg_mla_append_workspace_size.restype = sz
    L.eg_mla_append_workspace_size.argtypes = [pd, i32, i32]
    L.eg_mla_append_ws.restype = ctypes.c_int
    L.eg_mla_append_ws.argtypes = [pd, i32, i32, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, i64, vp, sz, vp]
    L.eg_mla_decode_workspace_size.restype = sz
    L.eg_mla_decode_workspace_size.argtypes = [pd, i32, i32, pp]
    L.eg_mla_decode.restype = ctypes.c_int
    L.eg_mla_decode.argtypes = [pd, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, i64, vp, sz, vp, vp]
    L.eg_mla_decode_planned.restype = ctypes.c_int
    L.eg_mla_decode_planned.argtypes = [pd, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, i64, vp, sz, vp, vp, pp]
    L.eg_mla_decode_noalloc.restype = ctypes.c_int
    L.eg_mla_decode_noalloc.argtypes = [pd, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, i64, vp, vp]
    L.eg_mla_gate_rows.restype = ctypes.c_int
    L.eg_mla_gate_rows.argtypes = [pd, i32, i32, i64, vp, vp, vp, vp, vp]
    L.eg_mla_gate_table_marks_size.restype = sz
    L.eg_mla_gate_table_marks_size.argtypes = [pd, i32, i32]
    L.eg_mla_gate_table.restype = ctypes.c_int
    L.eg_mla_gate_table.argtypes = [pd, i32, i32, i64, vp, vp, vp, vp, vp, sz, ctypes.c_uint32, vp]
    L.eg_mla_prefill_workspace_size.restype = sz
    L.eg_mla_prefill_workspace_size.argtypes = [pd, i32]
    L.eg_mla_prefill_ref.restype = ctypes.c_int
    L.eg_mla_prefill_ref.argtypes = [pd, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    L.eg_mla_prefill_varlen_workspace_size.restype = sz
    L.eg_mla_prefill_varlen_workspace_size.argtypes = [pd, i32]
    L.eg_mla_prefill_varlen.restype = ctypes.c_int
    L.eg_mla_prefill_varlen.argtypes = [pd, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    L.eg_mla_decode_literal_workspace_size.restype = sz
    L.eg_mla_decode_literal_workspace_size.argtypes = [pd, i32, i32]
    L.eg_mla_decode_literal.restype = ctypes.c_int
    L.eg_mla_decode_literal.argtypes = [pd, i32, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_uint32, vp, vp, i32, i64,
                                        vp, sz, vp, vp]
    L.eg_mla_page_plan.restype = ctypes.c_int
    L.eg_mla_page_plan.argtypes = [i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp]
    L.eg_mla_page_release.restype = ctypes.c_int
    L.eg_mla_page_release.argtypes = [i32, i32, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp]
    L.eg_mla_qk_norm_rope.restype = ctypes.c_int
    L.eg_mla_qk_norm_rope.argtypes = [pd, i32, vp, i64, vp, vp, vp, i64, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, i64,
                                      vp]
    L.eg_mla_decode_shared_workspace_size.restype = sz
    L.eg_mla_decode_shared_workspace_size.argtypes = [pd, i32, i32, i32]
    L.eg_mla_decode_shared.restype = ctypes.c_int
    L.eg_mla_decode_shared.argtypes = [pd, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, i32, i64, vp, sz, vp, vp]
    L.eg_mla_page_means.restype = ctypes.c_int
    L.eg_mla_page_means.argtypes = [pd, i32, vp, vp, vp, vp, vp, vp, i32, i64, vp, vp]
    L.eg_mla_page_scores_workspace_size.restype = sz
    L.eg_mla_page_scores_workspace_size.argtypes = [pd, i32]
    L.eg_mla_page_scores.restype = ctypes.c_int
    L.eg_mla_page_scores.argtypes = [pd, i32, vp, vp, vp, vp, vp, i32, i64, vp, sz, vp, vp]
    L.eg_mla_select_pages.restype = ctypes.c_int
    L.eg_mla_select_pages.argtypes = [pd, i32, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp]
    pr, f32 = ctypes.POINTER(Rope), ctypes.c_float
    L.eg_mla_rope_frequencies.restype = ctypes.c_int
    L.eg_mla_rope_frequencies.argtypes = [i32, f32, f32, i32, f32, f32, ctypes.POINTER(ctypes.c_double)]
    L.eg_mla_rope_rows.restype = ctypes.c_int
    L.eg_mla_rope_rows.argtypes = [pr, i32, i32, i32, i32, i32, i32, vp, i64, i64, vp, i32, vp, i64, i64, vp]
    L.eg_mla_quant_row_bytes.restype = i64
    L.eg_mla_quant_row_bytes.argtypes = [pd]
    L.eg_mla_quant_write.restype = ctypes.c_int
    L.eg_mla_quant_write.argtypes = [pd, pr, i32, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
    L.eg_mla_quant_read.restype = ctypes.c_int
    L.eg_mla_quant_read.argtypes = [pd, i32, i32, vp, vp, vp, vp, vp, i32, i64, vp, vp]
    L.eg_mla_quant_attend_workspace_size.restype = sz
    L.eg_mla_quant_attend_workspace_size.argtypes = [pd, i32, i32, i32]
    L.eg_mla_quant_attend.restype = ctypes.c_int
    L.eg_mla_quant_attend.argtypes = [pd, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, i64, vp, sz, vp, vp]
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().eg_mla_status_string(status).decode()


def make_dims(*, num_heads, head_dim, v_head_dim, latent_dim, rope_dim, vocab_size, page_size=64,
              gate_dim=None, softmax_scale=0.0, dtype=BF16) -> Dims:
    return Dims(num_heads, head_dim, v_head_dim, latent_dim, rope_dim,
                latent_dim if gate_dim is None else gate_dim, vocab_size, page_size, softmax_scale, dtype)


def make_plan(path: int = PATH_AUTO, split_tokens: int = 0, start_event=None, stop_event=None,
              id_slices: int = 0) -> Plan:
    return Plan(path, split_tokens, start_event, stop_event, id_slices)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        try:  # the handle alone: 0.3 us instead of 2.8 for a Stream object
            return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
        except AttributeError:
            return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(st: int, where: str):
    if st != OK:
        raise EgMlaError(st, where)


def check_dims(dims: Dims) -> int:
    return lib().eg_mla_check_dims(ctypes.byref(dims))


def decode_workspace_size(dims: Dims, batch: int, max_pages_per_seq: int, plan: Optional[Plan] = None) -> int:
    return lib().eg_mla_decode_workspace_size(ctypes.byref(dims), batch, max_pages_per_seq,
                                               None if plan is None else ctypes.byref(plan))


def prefill_workspace_size(dims: Dims, seq_len: int) -> int:
    return lib().eg_mla_prefill_workspace_size(ctypes.byref(dims), seq_len)


def decode(dims: Dims, q, latent_cache, token_id_cache, gate_table, w_uk, w_uv, seq_lens, page_table,
           max_pages_per_seq: int, workspace, out, plan: Optional[Plan] = None, stream=None) -> None:
    """eg_mla_decode / eg_mla_decode_planned over device tensors."""
    L = lib()
    batch = int(q.shape[0])
    num_slots = int(latent_cache.shape[0])
    ws_bytes = workspace.numel() * workspace.element_size()
    args = (ctypes.byref(dims), batch, _ptr(q), _ptr(latent_cache), _ptr(token_id_cache), _ptr(gate_table),
            _ptr(w_uk), _ptr(w_uv), _ptr(seq_lens), _ptr(page_table), max_pages_per_seq, num_slots,
            _ptr(workspace), ws_bytes, _ptr(out), _stream(stream))
    if plan is None:
        _check(L.eg_mla_decode(*args), "eg_mla_decode")
    else:
        _check(L.eg_mla_decode_planned(*args, ctypes.byref(plan)), "eg_mla_decode_planned")


def decode_noalloc(dims: Dims, q, latent_cache, token_id_cache, gate_table, w_uk, w_uv, seq_lens, page_table,
                   max_pages_per_seq: int, out, stream=None) -> None:
    """eg_mla_decode_noalloc over device tensors (no workspace: the library's scratch array)."""
    _check(lib().eg_mla_decode_noalloc(ctypes.byref(dims), int(q.shape[0]), _ptr(q), _ptr(latent_cache),
                                       _ptr(token_id_cache), _ptr(gate_table), _ptr(w_uk), _ptr(w_uv), _ptr(seq_lens),
                                       _ptr(page_table), max_pages_per_seq, int(latent_cache.shape[0]), _ptr(out),
                                       _stream(stream)), "eg_mla_decode_noalloc")


def append(dims: Dims, x, token_ids, positions, slots, w_dkv, kv_norm_w, latent_cache, token_id_cache,
           rope_theta: float = 10000.0, stream=None) -> None:
    """eg_mla_append over device tensors."""
    n, hidden = int(x.shape[0]), int(x.shape[1])
    _check(lib().eg_mla_append(ctypes.byref(dims), n, hidden, _ptr(x), _ptr(token_ids), _ptr(positions),
                               _ptr(slots), _ptr(w_dkv), _ptr(kv_norm_w), rope_theta, _ptr(latent_cache),
                               _ptr(token_id_cache), int(latent_cache.shape[0]), _stream(stream)), "eg_mla_append")


def append_workspace_size(dims: Dims, n_tokens: int, hidden: int) -> int:
    return lib().eg_mla_append_workspace_size(ctypes.byref(dims), n_tokens, hidden)


def append_ws(dims: Dims, x, token_ids, positions, slots, w_dkv, kv_norm_w, latent_cache, token_id_cache, workspace,
              rope_theta: float = 10000.0, stream=None) -> None:
    """eg_mla_append_ws over device tensors (workspace: a uint8 device tensor)."""
    n, hidden = int(x.shape[0]), int(x.shape[1])
    _check(lib().eg_mla_append_ws(ctypes.byref(dims), n, hidden, _ptr(x), _ptr(token_ids), _ptr(positions),
                                  _ptr(slots), _ptr(w_dkv), _ptr(kv_norm_w), rope_theta, _ptr(latent_cache),
                                  _ptr(token_id_cache), int(latent_cache.shape[0]), _ptr(workspace),
                                  int(workspace.numel()) if workspace is not None else 0, _stream(stream)),
           "eg_mla_append_ws")


def gate_rows(dims: Dims, ids, emb, w_ue, out, stream=None) -> None:
    """eg_mla_gate_rows over device tensors: out[i] = W_UE Emb[ids[i]]."""
    n = int(ids.shape[0])
    emb_vocab, emb_dim = int(emb.shape[0]), int(emb.shape[1])
    _check(lib().eg_mla_gate_rows(ctypes.byref(dims), emb_dim, emb_vocab, n, _ptr(ids), _ptr(emb), _ptr(w_ue),
                                  _ptr(out), _stream(stream)), "eg_mla_gate_rows")


def gate_table_marks_size(dims: Dims, emb_dim: int, emb_vocab: int) -> int:
    return int(lib().eg_mla_gate_table_marks_size(ctypes.byref(dims), emb_dim, emb_vocab))


def gate_table(dims: Dims, ids, emb, w_ue, table, marks, stamp: int, stream=None) -> None:
    """eg_mla_gate_table over device tensors: table[id] = W_UE Emb[id] for the distinct ids."""
    n = int(ids.shape[0])
    emb_vocab, emb_dim = int(emb.shape[0]), int(emb.shape[1])
    _check(lib().eg_mla_gate_table(ctypes.byref(dims), emb_dim, emb_vocab, n, _ptr(ids), _ptr(emb), _ptr(w_ue),
                                   _ptr(table), _ptr(marks), int(marks.numel() * marks.element_size()), stamp,
                                   _stream(stream)), "eg_mla_gate_table")


def decode_literal_workspace_size(dims: Dims, batch: int, max_pages: int) -> int:
    return lib().eg_mla_decode_literal_workspace_size(ctypes.byref(dims), batch, max_pages)


def decode_literal(dd, gate_full, ln_w, ln_b, flags: int, workspace, stream=None) -> None:
    """eg_mla_decode_literal over a staged DeviceDecode (its gate table is not used)."""
    _check(lib().eg_mla_decode_literal(ctypes.byref(dd.dims), int(dd.q.shape[0]), _ptr(dd.q), _ptr(dd.cache),
                                       _ptr(dd.ids), _ptr(gate_full), _ptr(dd.w_uk), _ptr(dd.w_uv), _ptr(ln_w),
                                       _ptr(ln_b), flags, _ptr(dd.seq_lens), _ptr(dd.page_table), dd.max_pages,
                                       int(dd.cache.shape[0]), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _ptr(dd.out), _stream(stream)),
           "eg_mla_decode_literal")


def prefill_varlen_workspace_size(dims: Dims, total_tokens: int) -> int:
    return lib().eg_mla_prefill_varlen_workspace_size(ctypes.byref(dims), total_tokens)


def prefill_varlen(dims: Dims, cu_seqlens, q, latent, token_ids, gate_table, w_uk, w_uv, workspace, out,
                   stream=None) -> None:
    """eg_mla_prefill_varlen over device tensors (sequences packed back to back)."""
    batch = int(cu_seqlens.shape[0]) - 1
    T = int(q.shape[0])
    _check(lib().eg_mla_prefill_varlen(ctypes.byref(dims), batch, T, _ptr(cu_seqlens), _ptr(q), _ptr(latent),
                                       _ptr(token_ids), _ptr(gate_table), _ptr(w_uk), _ptr(w_uv), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _ptr(out), _stream(stream)),
           "eg_mla_prefill_varlen")


def prefill_ref(dims: Dims, q, latent, token_ids, gate_table, w_uk, w_uv, workspace, out, stream=None) -> None:
    """eg_mla_prefill_ref over device tensors."""
    T = int(q.shape[0])
    _check(lib().eg_mla_prefill_ref(ctypes.byref(dims), T, _ptr(q), _ptr(latent), _ptr(token_ids),
                                    _ptr(gate_table), _ptr(w_uk), _ptr(w_uv), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _ptr(out), _stream(stream)),
           "eg_mla_prefill_ref")


# ---------------------------------------------------------------------------
# around the decode of a paged server: page tables, query and key rows, a
# shared prefix, sparse attention over pages
# ---------------------------------------------------------------------------
def _expect(name: str, *specs) -> None:
    """Refuses tensors that the C entry would misread.  A spec is (key, tensor or None, type or None, shape or None);
    every tensor has that type and shape, is contiguous and lies on the current GPU."""
    import torch
    here = None
    for key, t, dtype, shape in specs:
        if t is None:
            continue
        dev = t.get_device()
        if here is None:
            here = torch.cuda.current_device() if dev >= 0 else 0
        if (dtype is None or t.dtype is dtype) and dev == here and t.is_contiguous() and (shape is None or t.shape == shape):
            continue
        raise ValueError(f"{name}: {key} is {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}; expected "
                         f"contiguous{'' if dtype is None else f' {dtype}'}{'' if shape is None else f' {tuple(shape)}'} "
                         "on the current GPU")


def _storage(dims: Dims):
    import torch
    return torch.bfloat16 if dims.dtype == BF16 else torch.float32


def _bytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def page_plan(page_size: int, cached_lens, new_lens, page_table, free_pages, free_count, seq_lens, cu_seqlens, positions,
              slots, free_count_out, position_base=None, stream=None) -> None:
    """eg_mla_page_plan over int32 device tensors: page_table [B, max_pages] is updated, seq_lens, cu_seqlens,
    positions, slots and free_count_out are written."""
    from torch import int32 as i
    b, width, n, free = cached_lens.shape[0], page_table.shape[1], slots.shape[0], free_pages.shape[0]
    name = "eg_mla_page_plan"
    _expect(name, ("cached_lens", cached_lens, i, (b,)), ("new_lens", new_lens, i, (b,)),
            ("page_table", page_table, i, (b, width)), ("free_pages", free_pages, i, (free,)),
            ("free_count", free_count, i, (1,)), ("seq_lens", seq_lens, i, (b,)), ("cu_seqlens", cu_seqlens, i, (b + 1,)),
            ("positions", positions, i, (n,)), ("slots", slots, i, (n,)), ("free_count_out", free_count_out, i, (1,)),
            ("position_base", position_base, i, (b,)))
    _check(lib().eg_mla_page_plan(b, page_size, width, n, cached_lens.data_ptr(), new_lens.data_ptr(), _ptr(position_base),
                                  page_table.data_ptr(), free_pages.data_ptr(), free_count.data_ptr(), free, seq_lens.data_ptr(),
                                  cu_seqlens.data_ptr(), positions.data_ptr(), slots.data_ptr(), free_count_out.data_ptr(),
                                  _stream(stream)), name)


def page_release(page_size: int, seq_lens, ended, page_table, free_pages, free_count, seq_lens_out, free_count_out,
                 stream=None) -> None:
    """eg_mla_page_release over int32 device tensors: free_pages is updated, seq_lens_out and free_count_out written."""
    from torch import int32 as i
    b, width, free = seq_lens.shape[0], page_table.shape[1], free_pages.shape[0]
    name = "eg_mla_page_release"
    _expect(name, ("seq_lens", seq_lens, i, (b,)), ("ended", ended, i, (b,)), ("page_table", page_table, i, (b, width)),
            ("free_pages", free_pages, i, (free,)), ("free_count", free_count, i, (1,)),
            ("seq_lens_out", seq_lens_out, i, (b,)), ("free_count_out", free_count_out, i, (1,)))
    _check(lib().eg_mla_page_release(b, page_size, width, seq_lens.data_ptr(), ended.data_ptr(), page_table.data_ptr(),
                                     free_pages.data_ptr(), free_count.data_ptr(), free, seq_lens_out.data_ptr(),
                                     free_count_out.data_ptr(), _stream(stream)), name)


def _row_stride(name: str, key: str, t, n: int, row: int, dtype) -> int:
    """Elements between the rows of a [n, row] or [n, heads, d] tensor, or a view, whose rows are contiguous."""
    import torch
    shape, strides = t.shape, t.stride()
    inner = 1
    for size, step in zip(shape[:0:-1], strides[:0:-1]):
        if size != 1 and step != inner:
            inner = -1
            break
        inner *= size
    if shape[0] != n or (n and inner != row):
        raise ValueError(f"{name}: {key} is {tuple(shape)} with strides {strides}, not {n} contiguous rows of {row}")
    dev = t.get_device()
    if t.dtype is not dtype or dev < 0 or dev != torch.cuda.current_device():
        raise ValueError(f"{name}: {key} is {t.dtype} on {t.device}; expected {dtype} on the current GPU")
    return strides[0] if n > 1 else row


def qk_norm_rope(dims: Dims, q, q_out, kv, latent_cache, token_id_cache, token_ids, positions, slots, q_norm_w=None,
                 kv_norm_w=None, k_norm_w=None, rope_theta: float = 10000.0, stream=None) -> None:
    """eg_mla_qk_norm_rope over device tensors: q [n, H, d_h + d_r] or [n, H (d_h + d_r)] and kv [n, d_c + d_r], or
    views with a stride between their rows; q (with q_out) or kv (with the cache arguments) may be None."""
    from torch import int32 as i
    name, dt = "eg_mla_qk_norm_rope", _storage(dims)
    if q is None and kv is None:
        raise ValueError(f"{name}: neither q nor kv")
    n = (kv if q is None else q).shape[0]
    dq, row = dims.head_dim + dims.rope_dim, dims.latent_dim + dims.rope_dim
    specs = [("positions", positions, i, (n,))]
    qs = ks = num_slots = 0
    if q is not None:
        if q_out is None or q_out.shape[0] != n or q_out.numel() != n * dims.num_heads * dq:
            raise ValueError(f"{name}: q_out does not hold {n} rows of {dims.num_heads} heads of {dq} values")
        qs = _row_stride(name, "q", q, n, dims.num_heads * dq, dt)
        specs += (("q_out", q_out, dt, None), ("q_norm_w", q_norm_w, dt, (dq,)))
    if kv is not None:
        ks = _row_stride(name, "kv", kv, n, row, dt)
        num_slots = latent_cache.shape[0]
        specs += (("latent_cache", latent_cache, dt, (num_slots, row)),
                  ("token_id_cache", token_id_cache, i, (num_slots,)), ("token_ids", token_ids, i, (n,)),
                  ("slots", slots, i, (n,)), ("kv_norm_w", kv_norm_w, dt, (dims.latent_dim,)),
                  ("k_norm_w", k_norm_w, dt, (dims.rope_dim,)))
    _expect(name, *specs)
    _check(lib().eg_mla_qk_norm_rope(ctypes.byref(dims), n, _ptr(q), qs, _ptr(q_norm_w), _ptr(q_out), _ptr(kv), ks,
                                     _ptr(kv_norm_w), _ptr(k_norm_w), _ptr(token_ids), _ptr(positions), _ptr(slots),
                                     rope_theta, _ptr(latent_cache), _ptr(token_id_cache), num_slots, _stream(stream)),
           name)


def decode_shared_workspace_size(dims: Dims, batch: int, max_pages_per_seq: int, max_prefix_pages: int) -> int:
    return lib().eg_mla_decode_shared_workspace_size(ctypes.byref(dims), batch, max_pages_per_seq, max_prefix_pages)


def decode_shared(dims: Dims, q, latent_cache, token_id_cache, gate_table, w_uk, w_uv, prefix_len, prefix_table,
                  seq_lens, page_table, max_pages_per_seq: int, workspace, out, stream=None) -> None:
    """eg_mla_decode_shared over device tensors: prefix_len [1] and prefix_table [pages] (or None: no prefix) name the
    shared tokens, seq_lens and page_table each sequence's own."""
    from torch import int32 as i
    name, dt = "eg_mla_decode_shared", _storage(dims)
    b, slots, h = q.shape[0], latent_cache.shape[0], dims.num_heads
    dh, dv, dc, dr = dims.head_dim, dims.v_head_dim, dims.latent_dim, dims.rope_dim
    pages = 0 if prefix_table is None else prefix_table.shape[0]
    _expect(name, ("q", q, dt, (b, h, dh + dr)), ("latent_cache", latent_cache, dt, (slots, dc + dr)),
            ("token_id_cache", token_id_cache, i, (slots,)), ("gate_table", gate_table, dt, (dims.vocab_size, dc)),
            ("w_uk", w_uk, dt, (h, dh, dc)), ("w_uv", w_uv, dt, (h, dv, dc)), ("prefix_len", prefix_len, i, (1,)),
            ("prefix_table", prefix_table, i, (pages,)), ("seq_lens", seq_lens, i, (b,)),
            ("page_table", page_table, i, (b, max_pages_per_seq)), ("out", out, dt, (b, h, dv)),
            ("workspace", workspace, None, None))
    _check(lib().eg_mla_decode_shared(ctypes.byref(dims), b, _ptr(q), _ptr(latent_cache), _ptr(token_id_cache),
                                      gate_table.data_ptr(), w_uk.data_ptr(), w_uv.data_ptr(), _ptr(prefix_len), _ptr(prefix_table),
                                      pages, _ptr(seq_lens), _ptr(page_table), max_pages_per_seq, slots,
                                      _ptr(workspace), _bytes(workspace), out.data_ptr(), _stream(stream)), name)


def page_means(dims: Dims, latent_cache, token_id_cache, gate_table, first_tokens, seq_lens, page_table,
               max_pages_per_seq: int, means, stream=None) -> None:
    """eg_mla_page_means over device tensors: means [num_slots / P, d_c + d_r] is updated."""
    from torch import int32 as i
    name, dt = "eg_mla_page_means", _storage(dims)
    b, slots, row = seq_lens.shape[0], latent_cache.shape[0], dims.latent_dim + dims.rope_dim
    _expect(name, ("latent_cache", latent_cache, dt, (slots, row)), ("token_id_cache", token_id_cache, i, (slots,)),
            ("gate_table", gate_table, dt, (dims.vocab_size, dims.latent_dim)),
            ("first_tokens", first_tokens, i, (b,)), ("seq_lens", seq_lens, i, (b,)),
            ("page_table", page_table, i, (b, max_pages_per_seq)), ("means", means, dt, (slots // dims.page_size, row)))
    _check(lib().eg_mla_page_means(ctypes.byref(dims), b, _ptr(latent_cache), _ptr(token_id_cache), gate_table.data_ptr(),
                                   _ptr(first_tokens), _ptr(seq_lens), _ptr(page_table), max_pages_per_seq, slots,
                                   means.data_ptr(), _stream(stream)), name)


def page_scores_workspace_size(dims: Dims, batch: int) -> int:
    return lib().eg_mla_page_scores_workspace_size(ctypes.byref(dims), batch)


def page_scores(dims: Dims, q, w_uk, means, seq_lens, page_table, max_pages_per_seq: int, workspace, scores,
                stream=None) -> None:
    """eg_mla_page_scores over device tensors: scores [B, max_pages_per_seq] fp32 is written."""
    from torch import float32, int32 as i
    name, dt = "eg_mla_page_scores", _storage(dims)
    b, pages, dr = q.shape[0], means.shape[0], dims.rope_dim
    _expect(name, ("q", q, dt, (b, dims.num_heads, dims.head_dim + dr)),
            ("w_uk", w_uk, dt, (dims.num_heads, dims.head_dim, dims.latent_dim)),
            ("means", means, dt, (pages, dims.latent_dim + dr)), ("seq_lens", seq_lens, i, (b,)),
            ("page_table", page_table, i, (b, max_pages_per_seq)), ("scores", scores, float32, (b, max_pages_per_seq)),
            ("workspace", workspace, None, None))
    _check(lib().eg_mla_page_scores(ctypes.byref(dims), b, _ptr(q), w_uk.data_ptr(), means.data_ptr(), _ptr(seq_lens),
                                    _ptr(page_table), max_pages_per_seq, pages * dims.page_size, _ptr(workspace),
                                    _bytes(workspace), scores.data_ptr(), _stream(stream)), name)


def select_pages(dims: Dims, scores, seq_lens, page_table, max_pages_per_seq: int, sel_pages, sel_lens,
                 keep_first: int = 0, keep_last: int = 1, sel_index=None, stream=None) -> None:
    """eg_mla_select_pages over device tensors: sel_pages [B, keep], sel_lens [B] and sel_index [B, keep] (or None) are
    written; decode(..., sel_lens, sel_pages, keep, ...) attends to the chosen pages."""
    from torch import float32, int32 as i
    name = "eg_mla_select_pages"
    b, keep = sel_pages.shape
    _expect(name, ("scores", scores, float32, (b, max_pages_per_seq)), ("seq_lens", seq_lens, i, (b,)),
            ("page_table", page_table, i, (b, max_pages_per_seq)), ("sel_pages", sel_pages, i, (b, keep)),
            ("sel_lens", sel_lens, i, (b,)), ("sel_index", sel_index, i, (b, keep)))
    _check(lib().eg_mla_select_pages(ctypes.byref(dims), b, scores.data_ptr(), _ptr(seq_lens), _ptr(page_table),
                                     max_pages_per_seq, keep, keep_first, keep_last, sel_pages.data_ptr(), sel_lens.data_ptr(),
                                     _ptr(sel_index), _stream(stream)), name)


# ---------------------------------------------------------------------------
# rotation of rows, and the 8-bit latent cache
# ---------------------------------------------------------------------------
def rope_frequencies(rope_dim: int, factor: float, trained_positions: int, theta: float = 10000.0,
                     slow_turns: float = 1.0, fast_turns: float = 32.0) -> list:
    """eg_mla_rope_frequencies: radians a position of each pair of a layer whose context is stretched."""
    f = (ctypes.c_double * max(rope_dim // 2, 1))()
    _check(lib().eg_mla_rope_frequencies(rope_dim, theta, factor, trained_positions, slow_turns, fast_turns, f),
           "eg_mla_rope_frequencies")
    return list(f)


def make_rope(layout: int = ROPE_PAIRS, theta: float = 10000.0, frequencies=None, magnitude: float = 1.0) -> Rope:
    """A rotation; `frequencies` (d_r / 2 numbers, radians a position) take the place of theta's."""
    r = Rope(layout, theta, None, magnitude)
    if frequencies is not None:
        r.values = (ctypes.c_double * len(frequencies))(*frequencies)
        r.frequencies = r.values
    return r


def _rope_of(name: str, rope: Optional[Rope], rope_dim: int):
    """The rotation's pointer; its frequencies have to be those of rope_dim / 2 pairs."""
    if rope is None:
        return None
    values = getattr(rope, "values", None)
    if values is not None and len(values) != rope_dim // 2:
        raise ValueError(f"{name}: {len(values)} frequencies for {rope_dim // 2} pairs")
    return ctypes.byref(rope)


def rope_rows(rope: Rope, x, positions, out, rope_dim: int, rope_offset: Optional[int] = None, inverse: bool = False,
              stream=None) -> None:
    """eg_mla_rope_rows over device tensors: x and out [n, heads, head_dim] of one type, or views whose last dimension
    is contiguous; out may be x.  The part starts at rope_offset (the row's last rope_dim values unless given)."""
    import torch
    name = "eg_mla_rope_rows"
    n, heads, dim = x.shape
    here = torch.cuda.current_device() if x.get_device() >= 0 else 0
    for key, t in (("x", x), ("out", out)):
        if (t.dtype not in (torch.bfloat16, torch.float32) or t.dtype is not x.dtype or t.shape != x.shape
                or (t.stride(2) != 1 and dim > 1) or t.get_device() != here):
            raise ValueError(f"{name}: {key} is {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}; expected "
                             f"bfloat16 or float32 {tuple(x.shape)}, alike in x and out, with a contiguous last dimension "
                             "on the current GPU")
    _expect(name, ("positions", positions, torch.int32, (n,)))
    _check(lib().eg_mla_rope_rows(_rope_of(name, rope, rope_dim), BF16 if x.dtype is torch.bfloat16 else FP32, n, heads,
                                  dim, dim - rope_dim if rope_offset is None else rope_offset, rope_dim, x.data_ptr(),
                                  x.stride(0), x.stride(1), positions.data_ptr(), int(inverse), out.data_ptr(),
                                  out.stride(0), out.stride(1), _stream(stream)), name)


def quant_row_bytes(dims: Dims) -> int:
    return lib().eg_mla_quant_row_bytes(ctypes.byref(dims))


def _quant_cache(dims: Dims, codes, scales) -> list:
    import torch
    n = codes.shape[0]
    return [("codes", codes, torch.uint8, (n, dims.latent_dim + 2 * dims.rope_dim)), ("scales", scales, torch.uint8, (n,))]


def quant_write(dims: Dims, rope: Optional[Rope], kv, positions, slots, codes, scales, gate_table=None, token_ids=None,
             kv_norm_w=None, k_norm_w=None, stream=None) -> None:
    """eg_mla_quant_write over device tensors: kv [n, d_c + d_r], or a view with a stride between its rows, into rows of
    codes [num_slots, d_c + 2 d_r] and scales [num_slots] (uint8)."""
    from torch import bfloat16, int32 as i
    name, n = "eg_mla_quant_write", kv.shape[0]
    stride = _row_stride(name, "kv", kv, n, dims.latent_dim + dims.rope_dim, bfloat16)
    _expect(name, ("slots", slots, i, (n,)), ("positions", positions, i, (n,)), ("token_ids", token_ids, i, (n,)),
            ("gate_table", gate_table, bfloat16, (dims.vocab_size, dims.latent_dim)),
            ("kv_norm_w", kv_norm_w, bfloat16, (dims.latent_dim,)), ("k_norm_w", k_norm_w, bfloat16, (dims.rope_dim,)),
            *_quant_cache(dims, codes, scales))
    _check(lib().eg_mla_quant_write(ctypes.byref(dims), _rope_of(name, rope, dims.rope_dim), n, kv.data_ptr(), stride,
                                 _ptr(kv_norm_w), _ptr(k_norm_w), _ptr(gate_table), _ptr(token_ids), _ptr(positions),
                                 slots.data_ptr(), codes.data_ptr(), scales.data_ptr(), codes.shape[0], _stream(stream)), name)


def quant_read(dims: Dims, codes, scales, first_tokens, cu_seqlens, page_table, out, max_pages_per_seq: Optional[int] = None,
            stream=None) -> None:
    """eg_mla_quant_read over device tensors: out [total, d_c + d_r] (bf16), packed by cu_seqlens [B + 1]; max_pages_per_seq
    is page_table's width where there is one."""
    from torch import bfloat16, int32 as i
    name, b = "eg_mla_quant_read", cu_seqlens.shape[0] - 1
    width = page_table.shape[1] if page_table is not None else max_pages_per_seq
    if width is None:
        raise ValueError(f"{name}: neither page_table nor max_pages_per_seq")
    _expect(name, ("cu_seqlens", cu_seqlens, i, (b + 1,)), ("first_tokens", first_tokens, i, (b,)),
            ("page_table", page_table, i, (b, width)), ("out", out, bfloat16, (out.shape[0], dims.latent_dim + dims.rope_dim)),
            *_quant_cache(dims, codes, scales))
    _check(lib().eg_mla_quant_read(ctypes.byref(dims), b, out.shape[0], codes.data_ptr(), scales.data_ptr(), _ptr(first_tokens),
                                cu_seqlens.data_ptr(), _ptr(page_table), width, codes.shape[0], out.data_ptr(),
                                _stream(stream)), name)


def quant_attend_workspace_size(dims: Dims, batch: int, n_queries: int, max_pages_per_seq: int) -> int:
    return lib().eg_mla_quant_attend_workspace_size(ctypes.byref(dims), batch, n_queries, max_pages_per_seq)


def quant_attend(dims: Dims, q, cu_seqlens, codes, scales, w_uk, w_uv, seq_lens, page_table, max_pages_per_seq: int,
              workspace, out, stream=None) -> None:
    """eg_mla_quant_attend over device tensors: q [n, H, d_h + d_r] packed by cu_seqlens [B + 1], or (None) one new token a
    sequence; out [n, H, d_v]."""
    from torch import bfloat16 as bf, int32 as i, uint8
    name, n, b, h = "eg_mla_quant_attend", q.shape[0], seq_lens.shape[0], dims.num_heads
    _expect(name, ("q", q, bf, (n, h, dims.head_dim + dims.rope_dim)), ("cu_seqlens", cu_seqlens, i, (b + 1,)),
            ("w_uk", w_uk, bf, (h, dims.head_dim, dims.latent_dim)), ("w_uv", w_uv, bf, (h, dims.v_head_dim, dims.latent_dim)),
            ("seq_lens", seq_lens, i, (b,)), ("page_table", page_table, i, (b, max_pages_per_seq)),
            ("out", out, bf, (n, h, dims.v_head_dim)), ("workspace", workspace, uint8, None), *_quant_cache(dims, codes, scales))
    _check(lib().eg_mla_quant_attend(ctypes.byref(dims), b, n, q.data_ptr(), _ptr(cu_seqlens), codes.data_ptr(),
                                  scales.data_ptr(), w_uk.data_ptr(), w_uv.data_ptr(), seq_lens.data_ptr(), _ptr(page_table),
                                  max_pages_per_seq, codes.shape[0], workspace.data_ptr(), workspace.numel(), out.data_ptr(),
                                  _stream(stream)), name)


# ---------------------------------------------------------------------------
# device-side staging of generated workloads (plain copies, no arithmetic)
# ---------------------------------------------------------------------------
@dataclass
class DeviceDecode:
    dims: Dims
    q: object
    cache: object
    ids: object
    gate: object
    w_uk: object
    w_uv: object
    seq_lens: object
    page_table: object
    max_pages: int
    out: object


def dims_for(wl) -> Dims:
    return make_dims(num_heads=wl.heads, head_dim=wl.head_dim, v_head_dim=wl.v_head_dim, latent_dim=wl.latent_dim,
                     rope_dim=wl.rope_dim, vocab_size=wl.vocab, page_size=wl.page_size,
                     gate_dim=wl.gate_dim, dtype=BF16 if wl.dtype == "bf16" else FP32)


def to_device_tensor(a, storage: str, device="cuda"):
    """Host array (bf16 as uint16 bits) -> device tensor of the storage type."""
    import numpy as np
    import torch
    if storage == "bf16" and a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(a)).to(device)


def stage_decode(inp, device="cuda") -> DeviceDecode:
    """Copies a generated DecodeInputs to the device and allocates `out`."""
    import torch
    wl = inp.wl
    st = wl.dtype
    dt = torch.bfloat16 if st == "bf16" else torch.float32
    return DeviceDecode(
        dims=dims_for(wl), q=to_device_tensor(inp.q, st, device), cache=to_device_tensor(inp.latent_cache, st, device),
        ids=to_device_tensor(inp.token_ids, "int", device), gate=to_device_tensor(inp.gate_table, st, device),
        w_uk=to_device_tensor(inp.w_uk, st, device), w_uv=to_device_tensor(inp.w_uv, st, device),
        seq_lens=to_device_tensor(inp.seq_lens, "int", device),
        page_table=None if inp.page_table is None else to_device_tensor(inp.page_table, "int", device),
        max_pages=inp.max_pages, out=torch.empty((wl.batch, wl.heads, wl.v_head_dim), dtype=dt, device=device))


def alloc_workspace(nbytes: int, device="cuda"):
    import torch
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def run_decode(dd: DeviceDecode, plan: Optional[Plan] = None, workspace=None, stream=None):
    """Sizes a workspace (unless given) and runs one decode; returns dd.out."""
    if workspace is None:
        workspace = alloc_workspace(decode_workspace_size(dd.dims, int(dd.q.shape[0]), dd.max_pages, plan))
    decode(dd.dims, dd.q, dd.cache, dd.ids, dd.gate, dd.w_uk, dd.w_uv, dd.seq_lens, dd.page_table, dd.max_pages,
           workspace, dd.out, plan=plan, stream=stream)
    return dd.out


def out_to_f64(t):
    """Device output -> float64 numpy (exact widening)."""
    import torch
    return t.detach().to(torch.float64).cpu().numpy()
