"""ctypes binding of libspdecode.so: argument marshalling only.

Every function here has the name and argument order of the C entry point it
calls (see include/spdecode.h).  Tensors are torch tensors on the GPU; the
binding passes their device pointers and the current torch stream.  There is no
fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspdecode.so")

SPD_OK = 0
SPD_F32, SPD_BF16 = 0, 1
SPD_MAX_COMPACT_ROWS = 65536
STAGE_PREFIX, STAGE_SUFFIX, STAGE_MERGE = 1, 2, 4

_lib = None


class SpdError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class AttnDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("num_prompts", ctypes.c_int32), ("num_samples", ctypes.c_int32),
                ("max_samples_per_prompt", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("sm_scale", ctypes.c_float), ("stages", ctypes.c_uint32)]


class PrefixLevel(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("lens", ctypes.c_void_p),
                ("indptr", ctypes.c_void_p), ("page_indices", ctypes.c_void_p),
                ("sample_indptr", ctypes.c_void_p), ("num_groups", ctypes.c_int32),
                ("max_samples_per_group", ctypes.c_int32), ("max_len", ctypes.c_int64)]


class RowCopy(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("row_bytes", ctypes.c_int64)]


class PromptDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("num_prompts", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("sm_scale", ctypes.c_float), ("q_stride", ctypes.c_int64),
                ("kv_stride", ctypes.c_int64)]


class Penalties(ctypes.Structure):
    _fields_ = [("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p), ("presence", ctypes.c_void_p),
                ("prompt_bits", ctypes.c_void_p), ("prompt_bits_stride", ctypes.c_int64),
                ("prompt_of_row", ctypes.c_void_p), ("tokens", ctypes.c_void_p), ("token_row_stride", ctypes.c_int64),
                ("token_step_stride", ctypes.c_int64), ("token_lens", ctypes.c_void_p), ("max_tokens", ctypes.c_int64),
                ("bias_indptr", ctypes.c_void_p), ("bias_tokens", ctypes.c_void_p), ("bias_values", ctypes.c_void_p),
                ("allowed_bits", ctypes.c_void_p), ("allowed_stride", ctypes.c_int64),
                ("allowed_of_row", ctypes.c_void_p)]


def load() -> ctypes.CDLL:
    """Load the HIP library.  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it first (paper_2502_02534_amd/csrc/build.sh "
                           "or __graft_entry__.build()); there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
    dp = ctypes.POINTER(AttnDesc)
    lib.spd_status_string.restype = ctypes.c_char_p
    lib.spd_status_string.argtypes = [ctypes.c_int]
    lib.spd_attn_plan.restype = ctypes.c_int
    lib.spd_attn_plan.argtypes = [dp, i64, i64] + [ctypes.POINTER(ctypes.c_int32)] * 4
    lib.shared_prefix_decode_attn_workspace_size.restype = sz
    lib.shared_prefix_decode_attn_workspace_size.argtypes = [dp, i64, i64]
    lib.shared_prefix_decode_attn.restype = ctypes.c_int
    lib.shared_prefix_decode_attn.argtypes = [dp] + [vp] * 12 + [i64, i64, vp, vp, vp, sz, vp]
    lib.sample_tokens_workspace_size.restype = sz
    lib.sample_tokens_workspace_size.argtypes = [i64, i64]
    lib.sample_tokens.restype = ctypes.c_int
    lib.sample_tokens.argtypes = [vp, ctypes.c_int32, i64, i64, i64, vp, vp, vp, vp, vp, sz, vp]
    lib.sample_tokens_static.restype = ctypes.c_int
    lib.sample_tokens_static.argtypes = [vp, ctypes.c_int32, i64, i64, i64, vp, vp, vp, vp, vp]
    lib.sample_tokens_filtered.restype = ctypes.c_int
    lib.sample_tokens_filtered.argtypes = [vp, ctypes.c_int32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lp = ctypes.POINTER(PrefixLevel)
    lib.shared_prefix_decode_attn_levels_workspace_size.restype = sz
    lib.shared_prefix_decode_attn_levels_workspace_size.argtypes = [dp, ctypes.c_int32, lp, i64]
    lib.shared_prefix_decode_attn_levels.restype = ctypes.c_int
    lib.shared_prefix_decode_attn_levels.argtypes = [dp, vp, ctypes.c_int32, lp] + [vp] * 5 + [i64, vp, vp, vp, sz, vp]
    lib.append_suffix_kv.restype = ctypes.c_int
    lib.append_suffix_kv.argtypes = [dp] + [vp] * 7 + [i64, vp, ctypes.c_int32, vp, vp]
    for fn in (lib.decode_step_select, lib.decode_step_record):
        fn.restype = ctypes.c_int
        fn.argtypes = [vp, i64, ctypes.c_int32, ctypes.POINTER(RowCopy), vp]
    lib.decode_step_advance.restype = ctypes.c_int
    lib.decode_step_advance.argtypes = ([vp, i64, ctypes.c_int32, ctypes.POINTER(RowCopy), ctypes.c_int32,
                                         ctypes.POINTER(RowCopy), dp] + [vp] * 7 +
                                        [i64, vp, ctypes.c_int32, vp, vp, vp])
    pp = ctypes.POINTER(PromptDesc)
    lib.prompt_attn_workspace_size.restype = sz
    lib.prompt_attn_workspace_size.argtypes = [pp, i64, i64, i64]
    lib.prompt_attn.restype = ctypes.c_int
    lib.prompt_attn.argtypes = [pp] + [vp] * 7 + [i64, i64, i64, vp, vp, vp, sz, vp]
    lib.build_page_tables_workspace_size.restype = sz
    lib.build_page_tables_workspace_size.argtypes = [i64]
    lib.build_page_tables.restype = ctypes.c_int
    lib.build_page_tables.argtypes = ([i64, ctypes.c_int32] + [vp] * 5 + [i64, vp, i64, i64] + [vp] * 7 + [sz, vp])
    lib.build_page_tables_packed.restype = ctypes.c_int
    lib.build_page_tables_packed.argtypes = ([i64, ctypes.c_int32] + [vp] * 5 + [i64, vp, i64, i64] + [vp] * 9 + [sz, vp])
    lib.write_prompt_kv.restype = ctypes.c_int
    lib.write_prompt_kv.argtypes = [pp, vp, vp, vp, i64, i64, vp, vp, vp]
    lib.mark_prompt_tokens.restype = ctypes.c_int
    lib.mark_prompt_tokens.argtypes = [vp, vp, i64, i64, vp, i64, ctypes.c_int32, vp]
    lib.penalize_logits.restype = ctypes.c_int
    lib.penalize_logits.argtypes = [vp, ctypes.c_int32, i64, i64, i64, ctypes.POINTER(Penalties), vp, i64, vp]
    lib.token_logprobs_workspace_size.restype = sz
    lib.token_logprobs_workspace_size.argtypes = [i64, i64, ctypes.c_int32]
    lib.token_logprobs.restype = ctypes.c_int
    lib.token_logprobs.argtypes = [vp, ctypes.c_int32, i64, i64, i64, vp, vp, ctypes.c_int32] + [vp] * 7 + [sz, vp]
    lib.accumulate_kv_weights_workspace_size.restype = sz
    lib.accumulate_kv_weights_workspace_size.argtypes = [pp, i64, i64, i64]
    lib.accumulate_kv_weights.restype = ctypes.c_int
    lib.accumulate_kv_weights.argtypes = [pp] + [vp] * 7 + [i64, i64, i64, ctypes.c_float, vp, vp, i64, vp, sz, vp]
    lib.select_kv_tokens_workspace_size.restype = sz
    lib.select_kv_tokens_workspace_size.argtypes = [i64, ctypes.c_int32, i64]
    lib.select_kv_tokens.restype = ctypes.c_int
    lib.select_kv_tokens.argtypes = [vp, i64, i64, ctypes.c_int32, vp, i64, vp, i64, ctypes.c_int32, ctypes.c_int32, vp, i64, vp, vp, sz, vp]
    lib.compact_kv.restype = ctypes.c_int
    lib.compact_kv.argtypes = [pp, vp, i64, i64, vp, i64] + [vp] * 10 + [i64, vp, vp]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().spd_status_string(status).decode()


# What a call passes is plain integers (the prototypes turn them into pointers): a ctypes object per
# argument, and a stream object per call, cost more host time than the smallest calls take on the GPU.
def _ptr(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def _bytes(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.numel() * t.element_size()


_cuda_ready = False


def _forget_cuda() -> None:
    global _cuda_ready
    _cuda_ready = False


os.register_at_fork(after_in_child=_forget_cuda)  # torch refuses a forked child that its parent's GPU state went into


def _stream(stream) -> int:
    if stream is None:
        global _cuda_ready
        if not _cuda_ready:
            torch.cuda.init()
            _cuda_ready = True
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def make_desc(*, dtype: int, num_q_heads: int, num_kv_heads: int, head_dim: int, num_prompts: int,
              num_samples: int, max_samples_per_prompt: int = 0, page_size: int = 0,
              sm_scale: float = 0.0, stages: int = 0) -> AttnDesc:
    return AttnDesc(dtype, num_q_heads, num_kv_heads, head_dim, num_prompts, num_samples,
                    max_samples_per_prompt, page_size, sm_scale, stages)


def spd_attn_plan(desc: AttnDesc, max_prefix_len: int, max_suffix_len: int):
    vals = [ctypes.c_int32() for _ in range(4)]
    rc = load().spd_attn_plan(ctypes.byref(desc), max_prefix_len, max_suffix_len,
                              *[ctypes.byref(v) for v in vals])
    if rc != SPD_OK:
        raise SpdError(rc, "spd_attn_plan")
    return tuple(v.value for v in vals)


def shared_prefix_decode_attn_workspace_size(desc: AttnDesc, max_prefix_len: int, max_suffix_len: int) -> int:
    return int(load().shared_prefix_decode_attn_workspace_size(ctypes.byref(desc), max_prefix_len, max_suffix_len))


def shared_prefix_decode_attn(desc: AttnDesc, q, k_prefix, v_prefix, prefix_lens, prefix_indptr,
                              prefix_page_indices, sample_indptr, k_suffix, v_suffix, suffix_lens,
                              suffix_page_indptr, suffix_page_indices, max_prefix_len: int,
                              max_suffix_len: int, out, lse_out, workspace, stream=None) -> None:
    rc = load().shared_prefix_decode_attn(
        ctypes.byref(desc), _ptr(q), _ptr(k_prefix), _ptr(v_prefix), _ptr(prefix_lens),
        _ptr(prefix_indptr), _ptr(prefix_page_indices), _ptr(sample_indptr), _ptr(k_suffix),
        _ptr(v_suffix), _ptr(suffix_lens), _ptr(suffix_page_indptr), _ptr(suffix_page_indices),
        int(max_prefix_len), int(max_suffix_len), _ptr(out), _ptr(lse_out), _ptr(workspace),
        _bytes(workspace), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "shared_prefix_decode_attn")


def sample_tokens_workspace_size(rows: int, vocab: int) -> int:
    return int(load().sample_tokens_workspace_size(rows, vocab))


def sample_tokens(logits, logits_dtype: int, rows: int, vocab: int, row_stride: int, temperature,
                  top_p, uniforms, tokens_out, workspace, stream=None) -> None:
    rc = load().sample_tokens(
        _ptr(logits), logits_dtype, int(rows), int(vocab), int(row_stride), _ptr(temperature),
        _ptr(top_p), _ptr(uniforms), _ptr(tokens_out), _ptr(workspace),
        _bytes(workspace), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "sample_tokens")


def sample_tokens_static(logits, logits_dtype: int, rows: int, vocab: int, row_stride: int, temperature,
                         top_p, uniforms, tokens_out, stream=None) -> None:
    rc = load().sample_tokens_static(
        _ptr(logits), logits_dtype, int(rows), int(vocab), int(row_stride), _ptr(temperature),
        _ptr(top_p), _ptr(uniforms), _ptr(tokens_out), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "sample_tokens_static")


def append_suffix_kv(desc: AttnDesc, k_new, v_new, k_suffix, v_suffix, suffix_lens, suffix_page_indptr,
                     suffix_page_indices, max_suffix_len: int, last_tokens=None, end_token: int = -1,
                     finished=None, stream=None) -> None:
    rc = load().append_suffix_kv(
        ctypes.byref(desc), _ptr(k_new), _ptr(v_new), _ptr(k_suffix), _ptr(v_suffix), _ptr(suffix_lens),
        _ptr(suffix_page_indptr), _ptr(suffix_page_indices), int(max_suffix_len), _ptr(last_tokens),
        int(end_token), _ptr(finished), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "append_suffix_kv")


def make_row_copies(pairs):
    """ctypes array of RowCopy from (src tensor, dst tensor, bytes per row) triples."""
    arr = (RowCopy * len(pairs))()
    for i, (src, dst, row_bytes) in enumerate(pairs):
        arr[i] = RowCopy(src.data_ptr(), dst.data_ptr(), int(row_bytes))
    return arr


def decode_step_select(step_state, num_steps: int, copies, stream=None) -> None:
    rc = load().decode_step_select(_ptr(step_state), int(num_steps), len(copies), copies, _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "decode_step_select")


def decode_step_record(step_state, num_steps: int, copies, stream=None) -> None:
    rc = load().decode_step_record(_ptr(step_state), int(num_steps), len(copies), copies, _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "decode_step_record")


def decode_step_advance(step_state, num_steps: int, record, select, desc: AttnDesc, k_steps, v_steps, k_suffix,
                        v_suffix, suffix_lens, suffix_page_indptr, suffix_page_indices, max_suffix_len: int,
                        last_tokens=None, end_token: int = -1, finished=None, lens_record=None, stream=None) -> None:
    """`record` / `select`: ctypes arrays from make_row_copies, or None for no copies of that kind."""
    rc = load().decode_step_advance(
        _ptr(step_state), int(num_steps), 0 if record is None else len(record), record,
        0 if select is None else len(select), select, ctypes.byref(desc), _ptr(k_steps), _ptr(v_steps),
        _ptr(k_suffix), _ptr(v_suffix), _ptr(suffix_lens), _ptr(suffix_page_indptr), _ptr(suffix_page_indices),
        int(max_suffix_len), _ptr(last_tokens), int(end_token), _ptr(finished), _ptr(lens_record), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "decode_step_advance")


def make_levels(levels):
    """ctypes array of PrefixLevel from records with tensor fields k, v, lens, indptr, sample_indptr
    (and optionally page_indices) plus max_samples_per_group and max_len."""
    arr = (PrefixLevel * len(levels))()
    for i, lv in enumerate(levels):
        pages = getattr(lv, "page_indices", None)
        arr[i] = PrefixLevel(lv.k.data_ptr(), lv.v.data_ptr(), lv.lens.data_ptr(), lv.indptr.data_ptr(),
                             0 if pages is None else pages.data_ptr(), lv.sample_indptr.data_ptr(),
                             int(lv.lens.numel()), int(lv.max_samples_per_group), int(lv.max_len))
    return arr


def shared_prefix_decode_attn_levels_workspace_size(desc: AttnDesc, levels, max_suffix_len: int) -> int:
    return int(load().shared_prefix_decode_attn_levels_workspace_size(ctypes.byref(desc), len(levels), levels,
                                                                      int(max_suffix_len)))


def shared_prefix_decode_attn_levels(desc: AttnDesc, q, levels, k_suffix, v_suffix, suffix_lens,
                                     suffix_page_indptr, suffix_page_indices, max_suffix_len: int, out, lse_out,
                                     workspace, stream=None) -> None:
    rc = load().shared_prefix_decode_attn_levels(
        ctypes.byref(desc), _ptr(q), len(levels), levels, _ptr(k_suffix), _ptr(v_suffix), _ptr(suffix_lens),
        _ptr(suffix_page_indptr), _ptr(suffix_page_indices), int(max_suffix_len), _ptr(out), _ptr(lse_out),
        _ptr(workspace), _bytes(workspace),
        _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "shared_prefix_decode_attn_levels")


def sample_tokens_filtered(logits, logits_dtype: int, rows: int, vocab: int, row_stride: int, temperature,
                           top_p, top_k, min_p, uniforms, tokens_out, workspace, stream=None) -> None:
    rc = load().sample_tokens_filtered(
        _ptr(logits), logits_dtype, int(rows), int(vocab), int(row_stride), _ptr(temperature), _ptr(top_p),
        _ptr(top_k), _ptr(min_p), _ptr(uniforms), _ptr(tokens_out), _ptr(workspace),
        _bytes(workspace), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "sample_tokens_filtered")


def make_prompt_desc(*, dtype: int, num_q_heads: int, num_kv_heads: int, head_dim: int, num_prompts: int,
                     page_size: int = 0, causal: bool = True, sm_scale: float = 0.0, q_stride: int = 0,
                     kv_stride: int = 0) -> PromptDesc:
    return PromptDesc(dtype, num_q_heads, num_kv_heads, head_dim, num_prompts, page_size, 1 if causal else 0, sm_scale,
                      q_stride, kv_stride)


def prompt_attn_workspace_size(desc: PromptDesc, total_queries: int, max_query_len: int, max_kv_len: int) -> int:
    return int(load().prompt_attn_workspace_size(ctypes.byref(desc), int(total_queries), int(max_query_len),
                                                 int(max_kv_len)))


def prompt_attn(desc: PromptDesc, q, k, v, query_indptr, kv_lens, kv_indptr, kv_page_indices, total_queries: int,
                max_query_len: int, max_kv_len: int, out, lse_out, workspace, stream=None) -> None:
    rc = load().prompt_attn(
        ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(query_indptr), _ptr(kv_lens), _ptr(kv_indptr),
        _ptr(kv_page_indices), int(total_queries), int(max_query_len), int(max_kv_len), _ptr(out), _ptr(lse_out),
        _ptr(workspace), _bytes(workspace), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "prompt_attn")


def build_page_tables_workspace_size(num_requests: int) -> int:
    return int(load().build_page_tables_workspace_size(int(num_requests)))


def build_page_tables(num_requests: int, page_size: int, lens, held_lens, held_indptr, held_pages, free_pages,
                      num_free: int, free_begin, max_pages: int, max_tokens: int, page_indptr, page_indices, lens_out,
                      new_indptr, slot_map, free_end, workspace, stream=None) -> None:
    rc = load().build_page_tables(  # (pointers taken in place: the call is short, and fourteen helper calls are half a microsecond of it)
        int(num_requests), int(page_size),
        0 if lens is None else lens.data_ptr(),
        0 if held_lens is None else held_lens.data_ptr(),
        0 if held_indptr is None else held_indptr.data_ptr(),
        0 if held_pages is None else held_pages.data_ptr(),
        0 if free_pages is None else free_pages.data_ptr(),
        int(num_free),
        0 if free_begin is None else free_begin.data_ptr(),
        int(max_pages), int(max_tokens),
        0 if page_indptr is None else page_indptr.data_ptr(),
        0 if page_indices is None else page_indices.data_ptr(),
        0 if lens_out is None else lens_out.data_ptr(),
        0 if new_indptr is None else new_indptr.data_ptr(),
        0 if slot_map is None else slot_map.data_ptr(),
        0 if free_end is None else free_end.data_ptr(),
        0 if workspace is None else workspace.data_ptr(),
        0 if workspace is None else workspace.nbytes, _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "build_page_tables")


def build_page_tables_packed(num_requests: int, page_size: int, lens, held_lens, held_indptr, held_pages, free_pages,
                             num_free: int, free_begin, max_pages: int, max_tokens: int, page_indptr, page_indices, lens_out,
                             new_indptr, slot_map, free_end, packed_indptr, packed_lens, workspace, stream=None) -> None:
    rc = load().build_page_tables_packed(
        int(num_requests), int(page_size), _ptr(lens), _ptr(held_lens), _ptr(held_indptr), _ptr(held_pages), _ptr(free_pages),
        int(num_free), _ptr(free_begin), int(max_pages), int(max_tokens), _ptr(page_indptr), _ptr(page_indices), _ptr(lens_out),
        _ptr(new_indptr), _ptr(slot_map), _ptr(free_end), _ptr(packed_indptr), _ptr(packed_lens), _ptr(workspace),
        _bytes(workspace), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "build_page_tables_packed")


def write_prompt_kv(desc: PromptDesc, k, v, slot_map, num_tokens: int, num_pages: int, k_pool, v_pool,
                    stream=None) -> None:
    rc = load().write_prompt_kv(ctypes.byref(desc), _ptr(k), _ptr(v), _ptr(slot_map), int(num_tokens), int(num_pages),
                                _ptr(k_pool), _ptr(v_pool), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "write_prompt_kv")


def mark_prompt_tokens(tokens, indptr, num_prompts: int, vocab: int, bits, bits_stride: int, accumulate: bool = False,
                       stream=None) -> None:
    rc = load().mark_prompt_tokens(_ptr(tokens), _ptr(indptr), int(num_prompts), int(vocab), _ptr(bits),
                                   int(bits_stride), 1 if accumulate else 0, _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "mark_prompt_tokens")


def make_penalties(*, repetition=None, frequency=None, presence=None, prompt_bits=None, prompt_of_row=None,
                   tokens=None, token_lens=None, bias_indptr=None, bias_tokens=None, bias_values=None,
                   allowed_bits=None, allowed_of_row=None) -> Penalties:
    """Penalties from tensors, strides included: `tokens` is [rows, steps] with any strides (a loop's
    [steps, rows] record is passed as its transposed view).  The tensors have to outlive the record."""
    row = lambda t: 0 if t is None else t.stride(0)
    return Penalties(_ptr(repetition), _ptr(frequency), _ptr(presence), _ptr(prompt_bits), row(prompt_bits),
                     _ptr(prompt_of_row), _ptr(tokens), row(tokens), 0 if tokens is None else tokens.stride(1),
                     _ptr(token_lens), 0 if tokens is None else tokens.shape[1], _ptr(bias_indptr), _ptr(bias_tokens),
                     _ptr(bias_values), _ptr(allowed_bits), row(allowed_bits), _ptr(allowed_of_row))


def penalize_logits(logits, logits_dtype: int, rows: int, vocab: int, row_stride: int, penalties: Penalties, out,
                    out_stride: int, stream=None) -> None:
    rc = load().penalize_logits(_ptr(logits), int(logits_dtype), int(rows), int(vocab), int(row_stride),
                                ctypes.byref(penalties), _ptr(out), int(out_stride), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "penalize_logits")


def token_logprobs_workspace_size(rows: int, vocab: int, num_top: int) -> int:
    return int(load().token_logprobs_workspace_size(int(rows), int(vocab), int(num_top)))


def token_logprobs(logits, logits_dtype: int, rows: int, vocab: int, row_stride: int, temperature, tokens, num_top: int, logprobs,
                   ranks, entropy, lse, top_tokens, top_logprobs, workspace, stream=None) -> None:
    rc = load().token_logprobs(_ptr(logits), int(logits_dtype), int(rows), int(vocab), int(row_stride), _ptr(temperature), _ptr(tokens),
                               int(num_top), _ptr(logprobs), _ptr(ranks), _ptr(entropy), _ptr(lse), _ptr(top_tokens),
                               _ptr(top_logprobs), _ptr(workspace), _bytes(workspace), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "token_logprobs")


def accumulate_kv_weights_workspace_size(desc: PromptDesc, total_queries: int, max_query_len: int, max_kv_len: int) -> int:
    return int(load().accumulate_kv_weights_workspace_size(ctypes.byref(desc), int(total_queries), int(max_query_len), int(max_kv_len)))


def accumulate_kv_weights(desc: PromptDesc, q, k, query_indptr, kv_lens, kv_indptr, kv_page_indices, lse, total_queries: int,
                          max_query_len: int, max_kv_len: int, decay: float, weights, weights_out, weights_stride: int, workspace,
                          stream=None) -> None:
    rc = load().accumulate_kv_weights(
        ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(query_indptr), _ptr(kv_lens), _ptr(kv_indptr), _ptr(kv_page_indices), _ptr(lse),
        int(total_queries), int(max_query_len), int(max_kv_len), float(decay), _ptr(weights), _ptr(weights_out), int(weights_stride),
        _ptr(workspace), _bytes(workspace), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "accumulate_kv_weights")


def select_kv_tokens_workspace_size(num_seqs: int, num_heads: int, max_kv_len: int) -> int:
    return int(load().select_kv_tokens_workspace_size(int(num_seqs), int(num_heads), int(max_kv_len)))


def select_kv_tokens(weights, weights_stride: int, num_seqs: int, num_heads: int, kv_lens, max_kv_len: int, budgets, max_new_len: int,
                     sinks: int, recent: int, source, source_stride: int, new_lens, workspace, stream=None) -> None:
    rc = load().select_kv_tokens(_ptr(weights), int(weights_stride), int(num_seqs), int(num_heads), _ptr(kv_lens), int(max_kv_len),
                                 _ptr(budgets), int(max_new_len), int(sinks), int(recent), _ptr(source), int(source_stride),
                                 _ptr(new_lens), _ptr(workspace), _bytes(workspace), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "select_kv_tokens")


def compact_kv(desc: PromptDesc, source, source_seq_stride: int, source_head_stride: int, new_lens, max_new_len: int, kv_indptr,
               kv_page_indices, k, v, out_indptr, out_page_indices, k_out, v_out, weights, weights_out, weights_stride: int, lens_out,
               stream=None) -> None:
    rc = load().compact_kv(
        ctypes.byref(desc), _ptr(source), int(source_seq_stride), int(source_head_stride), _ptr(new_lens), int(max_new_len),
        _ptr(kv_indptr), _ptr(kv_page_indices), _ptr(k), _ptr(v), _ptr(out_indptr), _ptr(out_page_indices), _ptr(k_out), _ptr(v_out),
        _ptr(weights), _ptr(weights_out), int(weights_stride), _ptr(lens_out), _stream(stream))
    if rc != SPD_OK:
        raise SpdError(rc, "compact_kv")
