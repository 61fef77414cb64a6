"""Python binding of libptd.so, the MI355X (gfx950) Progressive Tree Drafting
hot path.

The functions named ``ptd_*`` mirror the C entry points of ``include/ptd.h``
one to one: they marshal arguments (torch tensors or raw integer device
addresses, a HIP stream) and raise :class:`PTDError` on a non-zero status.
Every step of the path runs in the library's HIP kernels; torch only provides
device memory and the stream.  There is no CPU fallback: without a built
``libptd.so`` the import fails.

The lower-case helpers (``tree_mask``, ``tree_attention``, ``topk_argmax``,
``verify``, ``expand``, ``verify_expand``, ``tree_rope``, ``kv_commit``,
``verify_sample``, ``step_prune``, ``prompt_attention``, ``qk_norm_rope``,
``token_logprobs``, ``page_copy``, the ``Pool``, ``PageTables`` and ``BlockKV`` classes)
allocate outputs with torch and call the entry points.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch  # loads the HIP runtime that libptd.so then shares

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libptd.so")

PTD_F32, PTD_BF16 = 0, 1
PTD_ROPE_HALF, PTD_ROPE_INTERLEAVED = 0, 1
PTD_MAX_T, PTD_MAX_K, PTD_MAX_DEPTH = 1024, 16, 64
STATUS = {0: "PTD_OK", 1: "PTD_ERR_NULL", 2: "PTD_ERR_SHAPE", 3: "PTD_ERR_DTYPE",
          4: "PTD_ERR_ALIGN", 5: "PTD_ERR_WORKSPACE", 6: "PTD_ERR_HIP",
          7: "PTD_ERR_BAD_TREE", 8: "PTD_ERR_KV_LEN", 9: "PTD_ERR_BAD_PATH",
          10: "PTD_ERR_PAGE", 11: "PTD_ERR_SCRATCH", 12: "PTD_ERR_NO_PAGES",
          13: "PTD_ERR_ROWS", 14: "PTD_ERR_VALUE"}
PTD_NOALLOC_SCRATCH_BYTES = 64 << 20


class PTDError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)} "
                         f"({_lib.ptd_status_string(status).decode()})")


class AttnShape(ctypes.Structure):
    """ptd_attn_shape"""
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32),
                ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("L_cap", ctypes.c_int32), ("in_dtype", ctypes.c_int),
                ("out_dtype", ctypes.c_int), ("scale", ctypes.c_float)]


class KVPages(ctypes.Structure):
    """ptd_kv_pages"""
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p),
                ("page_table", ctypes.c_void_p), ("page_size", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("num_pages", ctypes.c_int32)]


class KVPagesFp8Blk(ctypes.Structure):
    """ptd_kv_pages_fp8blk"""
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p),
                ("scales", ctypes.c_void_p), ("page_table", ctypes.c_void_p),
                ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("scale_rows", ctypes.c_int32)]


class PageState(ctypes.Structure):
    """ptd_page_state"""
    _fields_ = [("page_table", ctypes.c_void_p), ("num_held", ctypes.c_void_p),
                ("free_pages", ctypes.c_void_p), ("num_free", ctypes.c_void_p),
                ("B", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("num_pages", ctypes.c_int32)]


class PromptShape(ctypes.Structure):
    """ptd_prompt_shape"""
    _fields_ = [("B", ctypes.c_int32), ("N", ctypes.c_int32), ("Hq", ctypes.c_int32),
                ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32), ("ldq", ctypes.c_int64),
                ("ldk", ctypes.c_int64), ("ldv", ctypes.c_int64), ("in_dtype", ctypes.c_int),
                ("out_dtype", ctypes.c_int), ("scale", ctypes.c_float)]


class QKShape(ctypes.Structure):
    """ptd_qk_shape"""
    _fields_ = [("N", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("D", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("pairing", ctypes.c_int32),
                ("norm", ctypes.c_int32), ("dtype", ctypes.c_int), ("w_dtype", ctypes.c_int),
                ("ldq", ctypes.c_int64), ("ldk", ctypes.c_int64), ("ldv", ctypes.c_int64),
                ("ldqo", ctypes.c_int64), ("ldko", ctypes.c_int64), ("eps", ctypes.c_double),
                ("theta", ctypes.c_double)]


class KVStore(ctypes.Structure):
    """ptd_kv_store"""
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p),
                ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32)]


class PageArray(ctypes.Structure):
    """ptd_page_array"""
    _fields_ = [("base", ctypes.c_void_p), ("heads", ctypes.c_int32), ("units", ctypes.c_int32),
                ("unit_rows", ctypes.c_int32), ("unit_bytes", ctypes.c_int32)]


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                      "(hipcc --offload-arch=gfx950)")
_lib = ctypes.CDLL(LIB_PATH)

_vp, _i32, _i64, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
_SIGS = {
    "ptd_status_string": ([ctypes.c_int], ctypes.c_char_p),
    "ptd_version": ([], ctypes.c_int),
    "ptd_build_tree_mask": ([_vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp], ctypes.c_int),
    "ptd_tree_attention_workspace_bytes": ([ctypes.POINTER(AttnShape), _i32], _sz),
    "ptd_tree_attention": ([_vp, _vp, _vp, _vp, _vp, _i32, _vp, ctypes.POINTER(AttnShape),
                            _vp, _vp, _sz, _vp, _vp], ctypes.c_int),
    "ptd_tree_attention_ragged": ([_vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp,
                                   ctypes.POINTER(AttnShape), _vp, _vp, _sz, _vp, _vp],
                                  ctypes.c_int),
    "ptd_tree_attention_noalloc": ([_vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp,
                                    ctypes.POINTER(AttnShape), _vp, _vp, _vp], ctypes.c_int),
    "ptd_tree_attention_fp8kv": ([_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp,
                                  ctypes.POINTER(AttnShape), _vp, _sz, _vp, _vp], ctypes.c_int),
    "ptd_tree_attention_paged_fp8kv": ([_vp, ctypes.POINTER(KVPages), _vp, _vp, _vp, _vp, _vp,
                                        _i32, _vp, ctypes.POINTER(AttnShape), _vp, _sz, _vp,
                                        _vp], ctypes.c_int),
    "ptd_tree_attention_paged": ([_vp, ctypes.POINTER(KVPages), _vp, _vp, _vp, _i32, _vp,
                                  ctypes.POINTER(AttnShape), _vp, _vp, _sz, _vp, _vp],
                                 ctypes.c_int),
    "ptd_topk_workspace_bytes": ([_i32, _i32, _i32], _sz),
    "ptd_topk_argmax": ([_vp, ctypes.c_int, _i32, _i32, _i64, _i32, _vp, _vp, _vp, _vp,
                         _sz, _vp], ctypes.c_int),
    "ptd_verify": ([_vp, _vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp], ctypes.c_int),
    "ptd_expand": ([_vp, _vp, _vp, _i32, _i32, _vp, _i32, _vp, _i32, _i32, _vp, _vp, _vp,
                    _vp, _vp], ctypes.c_int),
    "ptd_verify_expand": ([_vp, _vp, _vp, _vp, _i32, _i32, _vp, _i32, _vp, _i32, _i32, _vp,
                           _vp, _vp, _vp, _vp, _vp, _vp, _vp], ctypes.c_int),
    "ptd_tree_rope": ([_vp, _vp, _vp, _vp, _i32, ctypes.POINTER(AttnShape), ctypes.c_double,
                       _vp, _i32, _vp, _vp, _vp], ctypes.c_int),
    "ptd_kv_commit": ([_vp, _vp, _vp, _vp, _vp, _i32, ctypes.POINTER(AttnShape), _vp, _vp,
                       _vp], ctypes.c_int),
    "ptd_verify_sample_workspace_bytes": ([_i32, _i32, _i32], _sz),
    "ptd_step_prune": ([_vp, _vp, _vp, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp],
                       ctypes.c_int),
    "ptd_pool_bytes": ([_i32, _i32, _i32], _sz),
    "ptd_pool_init": ([_vp, _sz, _i32, _i32, _i32, _vp], ctypes.c_int),
    "ptd_pool_merge": ([_vp, _sz, _i32, _i32, _i32, _vp, _vp, _vp, _i32, _vp, _vp],
                       ctypes.c_int),
    "ptd_pool_retrieve": ([_vp, _sz, _i32, _i32, _i32, _vp, _i32, _vp, _vp, _vp, _vp],
                          ctypes.c_int),
    "ptd_tree_attention_paged_fp8blk": ([_vp, ctypes.POINTER(KVPagesFp8Blk), _vp, _vp, _vp, _i32,
                                         _vp, ctypes.POINTER(AttnShape), _vp, _sz, _vp, _vp],
                                        ctypes.c_int),
    "ptd_kv_write_fp8blk": ([_vp, _vp, ctypes.c_int, _i64, _i64, _i32, _vp, _vp, _i32,
                             ctypes.POINTER(KVPagesFp8Blk), _i32, _i32, _vp, _vp], ctypes.c_int),
    "ptd_page_init": ([ctypes.POINTER(PageState), _vp], ctypes.c_int),
    "ptd_page_plan": ([ctypes.POINTER(PageState), _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp,
                       _vp], ctypes.c_int),
    "ptd_page_plan_shared": ([ctypes.POINTER(PageState), _vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp,
                              _vp, _vp], ctypes.c_int),
    "ptd_page_fork": ([ctypes.POINTER(PageState)] + [_vp] * 10, ctypes.c_int),
    "ptd_page_compact": ([ctypes.POINTER(PageState), _vp, _vp, _vp, _vp, _vp], ctypes.c_int),
    "ptd_page_copy": ([ctypes.POINTER(PageArray), _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp],
                      ctypes.c_int),
    "ptd_qk_norm_rope": ([_vp] * 9 + [ctypes.POINTER(KVStore), ctypes.POINTER(QKShape), _vp, _vp,
                                      _vp], ctypes.c_int),
    "ptd_token_logprobs_workspace_bytes": ([_i32, _i32, _i32], _sz),
    "ptd_token_logprobs": ([_vp, ctypes.c_int, _i32, _i32, _i64, _vp, _vp, _i32, ctypes.c_double,
                            _i32, _vp, _vp, _vp, _vp, _vp, _sz, _vp, _vp], ctypes.c_int),
    "ptd_prompt_attention": ([_vp, _vp, _vp, _vp, _vp, ctypes.POINTER(PromptShape), _vp, _vp],
                             ctypes.c_int),
    "ptd_verify_sample": ([_vp, ctypes.c_int, _i32, _i64, _vp, _vp, _vp, _i32, _i32,
                           ctypes.c_double, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp, _vp],
                          ctypes.c_int),
}
for _name, (_args, _res) in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.argtypes = _args
    _f.restype = _res


_Tensor = torch.Tensor


def _ptr(x):
    if type(x) is _Tensor:
        return x.data_ptr()
    if x is None:
        return None
    if isinstance(x, _Tensor):
        return x.data_ptr()
    return int(x)


def _stream(s):
    if s is None:
        if not torch.cuda.is_initialized():
            return torch.cuda.current_stream().cuda_stream
        # the handle alone: building the Stream object took 2.8 of a call's 7-10 us
        # of host time, this 0.3
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    if isinstance(s, torch.cuda.Stream):
        return s.cuda_stream
    return int(s)


def _check(st: int, where: str):
    if st != 0:
        raise PTDError(st, where)


# ---------------------------------------------------------------------------
# entry points (same names and argument order as include/ptd.h)
# ---------------------------------------------------------------------------
def ptd_status_string(status: int) -> str:
    return _lib.ptd_status_string(status).decode()


def ptd_version() -> int:
    return _lib.ptd_version()


def ptd_build_tree_mask(parent, tree_len, B, T, mask, depth, dev_status=None, stream=None):
    _check(_lib.ptd_build_tree_mask(_ptr(parent), _ptr(tree_len), B, T, _ptr(mask),
                                    _ptr(depth), _ptr(dev_status), _stream(stream)),
           "ptd_build_tree_mask")


def ptd_tree_attention_workspace_bytes(shape: AttnShape, T: int) -> int:
    return _lib.ptd_tree_attention_workspace_bytes(ctypes.byref(shape), T)


def ptd_tree_attention(q, k_cache, v_cache, kv_len, parent, T, out, shape: AttnShape,
                       mask=None, workspace=None, workspace_bytes=0, dev_status=None,
                       stream=None):
    _check(_lib.ptd_tree_attention(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(kv_len),
                                   _ptr(parent), T, _ptr(out), ctypes.byref(shape),
                                   _ptr(mask), _ptr(workspace), workspace_bytes,
                                   _ptr(dev_status), _stream(stream)),
           "ptd_tree_attention")


def ptd_tree_attention_ragged(q, k_cache, v_cache, kv_len, tree_len, parent, T, out,
                              shape: AttnShape, mask=None, workspace=None, workspace_bytes=0,
                              dev_status=None, stream=None):
    _check(_lib.ptd_tree_attention_ragged(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(kv_len),
                                          _ptr(tree_len), _ptr(parent), T, _ptr(out),
                                          ctypes.byref(shape), _ptr(mask), _ptr(workspace),
                                          workspace_bytes, _ptr(dev_status), _stream(stream)),
           "ptd_tree_attention_ragged")


def ptd_tree_attention_noalloc(q, k_cache, v_cache, kv_len, tree_len, parent, T, out,
                               shape: AttnShape, mask=None, dev_status=None, stream=None):
    _check(_lib.ptd_tree_attention_noalloc(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(kv_len),
                                           _ptr(tree_len), _ptr(parent), T, _ptr(out),
                                           ctypes.byref(shape), _ptr(mask), _ptr(dev_status),
                                           _stream(stream)),
           "ptd_tree_attention_noalloc")


def ptd_tree_attention_fp8kv(q, k_cache, v_cache, k_scale, v_scale, kv_len, tree_len, parent, T,
                             out, shape: AttnShape, workspace=None, workspace_bytes=0,
                             dev_status=None, stream=None):
    _check(_lib.ptd_tree_attention_fp8kv(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(k_scale),
                                         _ptr(v_scale), _ptr(kv_len), _ptr(tree_len),
                                         _ptr(parent), T, _ptr(out), ctypes.byref(shape),
                                         _ptr(workspace), workspace_bytes, _ptr(dev_status),
                                         _stream(stream)),
           "ptd_tree_attention_fp8kv")


def ptd_tree_attention_paged_fp8kv(q, kv: KVPages, k_scale, v_scale, kv_len, tree_len, parent, T,
                                   out, shape: AttnShape, workspace=None, workspace_bytes=0,
                                   dev_status=None, stream=None):
    _check(_lib.ptd_tree_attention_paged_fp8kv(_ptr(q), ctypes.byref(kv), _ptr(k_scale),
                                               _ptr(v_scale), _ptr(kv_len), _ptr(tree_len),
                                               _ptr(parent), T, _ptr(out), ctypes.byref(shape),
                                               _ptr(workspace), workspace_bytes, _ptr(dev_status),
                                               _stream(stream)),
           "ptd_tree_attention_paged_fp8kv")


def ptd_tree_attention_paged(q, kv: KVPages, kv_len, tree_len, parent, T, out, shape: AttnShape,
                             mask=None, workspace=None, workspace_bytes=0, dev_status=None,
                             stream=None):
    _check(_lib.ptd_tree_attention_paged(_ptr(q), ctypes.byref(kv), _ptr(kv_len), _ptr(tree_len),
                                         _ptr(parent), T, _ptr(out), ctypes.byref(shape),
                                         _ptr(mask), _ptr(workspace), workspace_bytes,
                                         _ptr(dev_status), _stream(stream)),
           "ptd_tree_attention_paged")


def ptd_tree_attention_paged_fp8blk(q, kv: KVPagesFp8Blk, kv_len, tree_len, parent, T, out,
                                    shape: AttnShape, workspace=None, workspace_bytes=0,
                                    dev_status=None, stream=None):
    _check(_lib.ptd_tree_attention_paged_fp8blk(_ptr(q), ctypes.byref(kv), _ptr(kv_len),
                                                _ptr(tree_len), _ptr(parent), T, _ptr(out),
                                                ctypes.byref(shape), _ptr(workspace),
                                                workspace_bytes, _ptr(dev_status),
                                                _stream(stream)),
           "ptd_tree_attention_paged_fp8blk")


def ptd_kv_write_fp8blk(k, v, dtype, ldk, ldv, N, slots, src, rows_per_seq, kv: KVPagesFp8Blk,
                        Hkv, D, dev_status=None, stream=None):
    _check(_lib.ptd_kv_write_fp8blk(_ptr(k), _ptr(v), dtype, ldk, ldv, N, _ptr(slots), _ptr(src),
                                    rows_per_seq, ctypes.byref(kv), Hkv, D, _ptr(dev_status),
                                    _stream(stream)),
           "ptd_kv_write_fp8blk")


def ptd_page_init(state: PageState, stream=None):
    _check(_lib.ptd_page_init(ctypes.byref(state), _stream(stream)), "ptd_page_init")


def ptd_page_plan(state: PageState, kv_len, new_len, N, rows_per_seq, row_start, slots,
                  positions=None, dev_status=None, stream=None):
    _check(_lib.ptd_page_plan(ctypes.byref(state), _ptr(kv_len), _ptr(new_len), N, rows_per_seq,
                              _ptr(row_start), _ptr(slots), _ptr(positions), _ptr(dev_status),
                              _stream(stream)),
           "ptd_page_plan")


def ptd_prompt_attention(q, k, v, row_start, out, shape: PromptShape, dev_status=None,
                         stream=None):
    _check(_lib.ptd_prompt_attention(_ptr(q), _ptr(k), _ptr(v), _ptr(row_start), _ptr(out),
                                     ctypes.byref(shape), _ptr(dev_status), _stream(stream)),
           "ptd_prompt_attention")


def ptd_page_plan_shared(state: PageState, refs, kv_len, new_len, N, rows_per_seq, row_start, slots,
                         positions=None, dev_status=None, stream=None):
    _check(_lib.ptd_page_plan_shared(ctypes.byref(state), _ptr(refs), _ptr(kv_len), _ptr(new_len), N,
                                     rows_per_seq, _ptr(row_start), _ptr(slots), _ptr(positions),
                                     _ptr(dev_status), _stream(stream)),
           "ptd_page_plan_shared")


def ptd_page_fork(state: PageState, refs, from_, len_, table_next, held_next, copy_src, copy_dst,
                  copy_rows, dev_status=None, stream=None):
    _check(_lib.ptd_page_fork(ctypes.byref(state), _ptr(refs), _ptr(from_), _ptr(len_),
                              _ptr(table_next), _ptr(held_next), _ptr(copy_src), _ptr(copy_dst),
                              _ptr(copy_rows), _ptr(dev_status), _stream(stream)),
           "ptd_page_fork")


def ptd_page_compact(state: PageState, refs, move_src, move_dst, dev_status=None, stream=None):
    _check(_lib.ptd_page_compact(ctypes.byref(state), _ptr(refs), _ptr(move_src), _ptr(move_dst),
                                 _ptr(dev_status), _stream(stream)),
           "ptd_page_compact")


def ptd_page_copy(arrays, num_pages, n, src, dst, rows=None, dev_status=None, stream=None):
    """arrays: a ctypes array of PageArray (which a program makes once), or a sequence."""
    if not isinstance(arrays, ctypes.Array):
        arrays = (PageArray * len(arrays))(*arrays)
    _check(_lib.ptd_page_copy(arrays, len(arrays), num_pages, n, _ptr(src), _ptr(dst), _ptr(rows),
                              _ptr(dev_status), _stream(stream)),
           "ptd_page_copy")


def ptd_qk_norm_rope(q, k, v, q_weight, k_weight, positions, slots, q_out, k_out,
                     store: Optional[KVStore], shape: QKShape,
                     inv_freq: Optional[Sequence[float]] = None, dev_status=None, stream=None):
    """inv_freq: host sequence of rot_dim/2 floats, or None for theta^(-2p/rot_dim)."""
    f = None
    if inv_freq is not None:
        if len(inv_freq) != shape.rot_dim // 2:
            raise ValueError("inv_freq needs rot_dim/2 entries")
        f = (ctypes.c_double * max(1, len(inv_freq)))(*[float(x) for x in inv_freq])
    _check(_lib.ptd_qk_norm_rope(_ptr(q), _ptr(k), _ptr(v), _ptr(q_weight), _ptr(k_weight),
                                 _ptr(positions), _ptr(slots), _ptr(q_out), _ptr(k_out),
                                 None if store is None else ctypes.byref(store),
                                 ctypes.byref(shape), None if f is None else ctypes.cast(f, _vp),
                                 _ptr(dev_status), _stream(stream)),
           "ptd_qk_norm_rope")


def ptd_token_logprobs_workspace_bytes(R: int, V: int, k: int) -> int:
    return _lib.ptd_token_logprobs_workspace_bytes(R, V, k)


def ptd_token_logprobs(logits, dtype, R, V, ld, tokens, nodes, T, temperature, k, logprob,
                       entropy=None, topk_idx=None, topk_logprob=None, workspace=None,
                       workspace_bytes=0, dev_status=None, stream=None):
    _check(_lib.ptd_token_logprobs(_ptr(logits), dtype, R, V, ld, _ptr(tokens), _ptr(nodes), T,
                                   float(temperature), k, _ptr(logprob), _ptr(entropy),
                                   _ptr(topk_idx), _ptr(topk_logprob), _ptr(workspace),
                                   workspace_bytes, _ptr(dev_status), _stream(stream)),
           "ptd_token_logprobs")


def ptd_topk_workspace_bytes(R: int, V: int, k: int) -> int:
    return _lib.ptd_topk_workspace_bytes(R, V, k)


def ptd_topk_argmax(logits, dtype, R, V, ld, k, argmax, topk_idx=None, topk_val=None,
                    workspace=None, workspace_bytes=0, stream=None):
    _check(_lib.ptd_topk_argmax(_ptr(logits), dtype, R, V, ld, k, _ptr(argmax),
                                _ptr(topk_idx), _ptr(topk_val), _ptr(workspace),
                                workspace_bytes, _stream(stream)),
           "ptd_topk_argmax")


def ptd_verify(argmax, draft_tokens, parent, tree_len, B, T, accept_len, accept_nodes,
               out_tokens, dev_status=None, stream=None):
    _check(_lib.ptd_verify(_ptr(argmax), _ptr(draft_tokens), _ptr(parent), _ptr(tree_len),
                           B, T, _ptr(accept_len), _ptr(accept_nodes), _ptr(out_tokens),
                           _ptr(dev_status), _stream(stream)),
           "ptd_verify")


def ptd_expand(parent, tokens, tree_len, B, T, topk_idx, k, width_sched, d_max, T_max,
               parent_next, tokens_next, tree_len_next, dev_status=None, stream=None):
    ws = (ctypes.c_int32 * max(1, len(width_sched)))(*[int(x) for x in width_sched])
    if len(width_sched) < d_max:
        raise ValueError("width_sched needs d_max entries")
    _check(_lib.ptd_expand(_ptr(parent), _ptr(tokens), _ptr(tree_len), B, T, _ptr(topk_idx),
                           k, ctypes.cast(ws, _vp), d_max, T_max, _ptr(parent_next),
                           _ptr(tokens_next), _ptr(tree_len_next), _ptr(dev_status),
                           _stream(stream)),
           "ptd_expand")


def ptd_verify_expand(argmax, draft_tokens, parent, tree_len, B, T, topk_idx, k, width_sched,
                      d_max, T_max, accept_len, accept_nodes, out_tokens, parent_next,
                      tokens_next, tree_len_next, dev_status=None, stream=None):
    if len(width_sched) < d_max:
        raise ValueError("width_sched needs d_max entries")
    ws = (ctypes.c_int32 * max(1, len(width_sched)))(*[int(x) for x in width_sched])
    _check(_lib.ptd_verify_expand(_ptr(argmax), _ptr(draft_tokens), _ptr(parent),
                                  _ptr(tree_len), B, T, _ptr(topk_idx), k,
                                  ctypes.cast(ws, _vp), d_max, T_max, _ptr(accept_len),
                                  _ptr(accept_nodes), _ptr(out_tokens), _ptr(parent_next),
                                  _ptr(tokens_next), _ptr(tree_len_next), _ptr(dev_status),
                                  _stream(stream)),
           "ptd_verify_expand")


def ptd_tree_rope(q, k_cache, kv_len, parent, T, shape: AttnShape, theta=10000.0,
                  inv_freq: Optional[Sequence[float]] = None, pairing=PTD_ROPE_HALF,
                  pos_out=None, dev_status=None, stream=None):
    """inv_freq: host sequence of D/2 floats, or None for theta^(-2p/D)."""
    f = None
    if inv_freq is not None:
        if len(inv_freq) != shape.D // 2:
            raise ValueError("inv_freq needs D/2 entries")
        f = (ctypes.c_double * len(inv_freq))(*[float(x) for x in inv_freq])
    _check(_lib.ptd_tree_rope(_ptr(q), _ptr(k_cache), _ptr(kv_len), _ptr(parent), T,
                              ctypes.byref(shape), float(theta),
                              None if f is None else ctypes.cast(f, _vp), pairing,
                              _ptr(pos_out), _ptr(dev_status), _stream(stream)),
           "ptd_tree_rope")


def ptd_kv_commit(k_cache, v_cache, kv_len, accept_len, accept_nodes, T, shape: AttnShape,
                  kv_len_next, dev_status=None, stream=None):
    _check(_lib.ptd_kv_commit(_ptr(k_cache), _ptr(v_cache), _ptr(kv_len), _ptr(accept_len),
                              _ptr(accept_nodes), T, ctypes.byref(shape), _ptr(kv_len_next),
                              _ptr(dev_status), _stream(stream)),
           "ptd_kv_commit")


def ptd_verify_sample_workspace_bytes(B: int, T: int, V: int) -> int:
    return _lib.ptd_verify_sample_workspace_bytes(B, T, V)


def ptd_verify_sample(logits, dtype, V, ld, draft_tokens, parent, tree_len, B, T, temperature,
                      u_node, u_bonus, accept_len, accept_nodes, out_tokens, workspace=None,
                      workspace_bytes=0, dev_status=None, stream=None):
    _check(_lib.ptd_verify_sample(_ptr(logits), dtype, V, ld, _ptr(draft_tokens), _ptr(parent),
                                  _ptr(tree_len), B, T, float(temperature), _ptr(u_node),
                                  _ptr(u_bonus), _ptr(accept_len), _ptr(accept_nodes),
                                  _ptr(out_tokens), _ptr(workspace), workspace_bytes,
                                  _ptr(dev_status), _stream(stream)),
           "ptd_verify_sample")


def ptd_step_prune(parent, tokens, tree_len, B, T, d_max, T_max, parent_next, tokens_next,
                   tree_len_next, dev_status=None, stream=None):
    _check(_lib.ptd_step_prune(_ptr(parent), _ptr(tokens), _ptr(tree_len), B, T, d_max, T_max,
                               _ptr(parent_next), _ptr(tokens_next), _ptr(tree_len_next),
                               _ptr(dev_status), _stream(stream)),
           "ptd_step_prune")


def ptd_pool_bytes(B: int, e_max: int, n_cap: int) -> int:
    return _lib.ptd_pool_bytes(B, e_max, n_cap)


def ptd_pool_init(pool, pool_bytes, B, e_max, n_cap, stream=None):
    _check(_lib.ptd_pool_init(_ptr(pool), pool_bytes, B, e_max, n_cap, _stream(stream)),
           "ptd_pool_init")


def ptd_pool_merge(pool, pool_bytes, B, e_max, n_cap, parent, tokens, tree_len, T,
                   dev_status=None, stream=None):
    _check(_lib.ptd_pool_merge(_ptr(pool), pool_bytes, B, e_max, n_cap, _ptr(parent),
                               _ptr(tokens), _ptr(tree_len), T, _ptr(dev_status),
                               _stream(stream)),
           "ptd_pool_merge")


def ptd_pool_retrieve(pool, pool_bytes, B, e_max, n_cap, last_token, T_max, parent_out,
                      tokens_out, tree_len_out, stream=None):
    _check(_lib.ptd_pool_retrieve(_ptr(pool), pool_bytes, B, e_max, n_cap, _ptr(last_token),
                                  T_max, _ptr(parent_out), _ptr(tokens_out),
                                  _ptr(tree_len_out), _stream(stream)),
           "ptd_pool_retrieve")


# ---------------------------------------------------------------------------
# tensor helpers: allocate outputs, check device/dtype/contiguity, call
# ---------------------------------------------------------------------------
def _need_gpu(*ts):
    for t in ts:
        if t is not None and (not isinstance(t, torch.Tensor) or not t.is_cuda
                              or not t.is_contiguous()):
            raise ValueError("expected contiguous GPU tensors")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return PTD_BF16
    if t.dtype == torch.float32:
        return PTD_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def attn_shape(q: torch.Tensor, k_cache: torch.Tensor, out_dtype=None,
               scale: float = 0.0) -> AttnShape:
    B, T, Hq, D = q.shape
    _, Hkv, L_cap, _ = k_cache.shape
    od = _dtype_code(q) if out_dtype is None else (
        PTD_BF16 if out_dtype == torch.bfloat16 else PTD_F32)
    return AttnShape(B, Hq, Hkv, D, L_cap, _dtype_code(q), od, float(scale))


def tree_mask(parent: torch.Tensor, tree_len: Optional[torch.Tensor] = None,
              dev_status: Optional[torch.Tensor] = None):
    _need_gpu(parent, tree_len)
    B, T = parent.shape
    mask = torch.empty((B, T, (T + 63) // 64), dtype=torch.int64, device=parent.device)
    depth = torch.empty((B, T), dtype=torch.int32, device=parent.device)
    ptd_build_tree_mask(parent, tree_len, B, T, mask, depth, dev_status)
    return mask, depth


def tree_attention(q, k_cache, v_cache, kv_len, parent, mask=None, out=None,
                   out_dtype=None, scale: float = 0.0, workspace=None,
                   dev_status=None, tree_len=None):
    """tree_len int32 [B] (optional): a padded batch of trees of different
    sizes (ptd_tree_attention_ragged); nodes >= tree_len[b] get zero rows."""
    _need_gpu(q, k_cache, v_cache, kv_len, parent, mask, tree_len)
    B, T, Hq, D = q.shape
    shape = attn_shape(q, k_cache, out_dtype, scale)
    if out is None:
        od = torch.bfloat16 if shape.out_dtype == PTD_BF16 else torch.float32
        out = torch.empty((B, T, Hq, D), dtype=od, device=q.device)
    nbytes = ptd_tree_attention_workspace_bytes(shape, T)
    if workspace is None and nbytes:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    wsb = 0 if workspace is None else workspace.numel()
    if tree_len is None:
        ptd_tree_attention(q, k_cache, v_cache, kv_len, parent, T, out, shape, mask,
                           workspace, wsb, dev_status)
    else:
        ptd_tree_attention_ragged(q, k_cache, v_cache, kv_len, tree_len, parent, T, out, shape,
                                  mask, workspace, wsb, dev_status)
    return out


def tree_attention_fp8kv(q, k_cache, v_cache, k_scale, v_scale, kv_len, parent, out=None,
                         out_dtype=None, scale: float = 0.0, workspace=None, dev_status=None,
                         tree_len=None):
    """k_cache, v_cache uint8 [B][Hkv][L_cap][D] E4M3 codes; k_scale, v_scale
    float32 [Hkv] (or None); q bf16; otherwise as tree_attention."""
    _need_gpu(q, k_cache, v_cache, k_scale, v_scale, kv_len, parent, tree_len)
    if k_cache.dtype != torch.uint8 or v_cache.dtype != torch.uint8:
        raise ValueError("expected uint8 E4M3 caches")
    B, T, Hq, D = q.shape
    _, Hkv, L, _ = k_cache.shape
    shape = AttnShape(B, Hq, Hkv, D, L, _dtype_code(q),
                      _dtype_code(q) if out_dtype is None else
                      (PTD_BF16 if out_dtype == torch.bfloat16 else PTD_F32), float(scale))
    if out is None:
        od = torch.bfloat16 if shape.out_dtype == PTD_BF16 else torch.float32
        out = torch.empty((B, T, Hq, D), dtype=od, device=q.device)
    nbytes = ptd_tree_attention_workspace_bytes(shape, T)
    if workspace is None and nbytes:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    ptd_tree_attention_fp8kv(q, k_cache, v_cache, k_scale, v_scale, kv_len, tree_len, parent, T,
                             out, shape, workspace, 0 if workspace is None else workspace.numel(),
                             dev_status)
    return out


def tree_attention_paged(q, k_pages, v_pages, page_table, kv_len, parent, out=None,
                         out_dtype=None, scale: float = 0.0, workspace=None, dev_status=None,
                         tree_len=None, k_scale=None, v_scale=None):
    """k_pages, v_pages [num_pages][Hkv][page_size][D] (bf16, or uint8 E4M3
    codes with optional k_scale / v_scale [Hkv]), page_table int32
    [B][max_pages]; otherwise as tree_attention."""
    _need_gpu(q, k_pages, v_pages, page_table, kv_len, parent, tree_len, k_scale, v_scale)
    B, T, Hq, D = q.shape
    num_pages, Hkv, ps, _ = k_pages.shape
    max_pages = page_table.shape[1]
    shape = AttnShape(B, Hq, Hkv, D, max_pages * ps, _dtype_code(q),
                      _dtype_code(q) if out_dtype is None else
                      (PTD_BF16 if out_dtype == torch.bfloat16 else PTD_F32), float(scale))
    if out is None:
        od = torch.bfloat16 if shape.out_dtype == PTD_BF16 else torch.float32
        out = torch.empty((B, T, Hq, D), dtype=od, device=q.device)
    nbytes = ptd_tree_attention_workspace_bytes(shape, T)
    if workspace is None and nbytes:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    kv = KVPages(k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(), ps, max_pages,
                 num_pages)
    wsb = 0 if workspace is None else workspace.numel()
    if k_pages.dtype == torch.uint8:
        ptd_tree_attention_paged_fp8kv(q, kv, k_scale, v_scale, kv_len, tree_len, parent, T, out,
                                       shape, workspace, wsb, dev_status)
    else:
        ptd_tree_attention_paged(q, kv, kv_len, tree_len, parent, T, out, shape, None, workspace,
                                 wsb, dev_status)
    return out


def topk_argmax(logits: torch.Tensor, k: int, with_values: bool = True, workspace=None):
    """logits [R][V] with unit stride along V (a row stride ld >= V is allowed),
    or any contiguous [..][V]; returns (argmax [R], idx [R][k], val [R][k])."""
    if not logits.is_cuda:
        raise ValueError("expected GPU logits")
    if logits.dim() != 2:
        logits = logits.reshape(-1, logits.shape[-1])
    if logits.stride(1) != 1:
        raise ValueError("logits need unit stride along the vocabulary")
    R, V = logits.shape
    ld = logits.stride(0)
    dev = logits.device
    am = torch.empty(R, dtype=torch.int32, device=dev)
    idx = torch.empty((R, k), dtype=torch.int32, device=dev)
    val = torch.empty((R, k), dtype=torch.float32, device=dev) if with_values else None
    nbytes = ptd_topk_workspace_bytes(R, V, k)
    if workspace is None and nbytes:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    ptd_topk_argmax(logits, _dtype_code(logits), R, V, ld, k, am, idx, val, workspace,
                    0 if workspace is None else workspace.numel())
    return am, idx, val


def verify(argmax, draft_tokens, parent, tree_len=None, dev_status=None):
    _need_gpu(argmax, draft_tokens, parent, tree_len)
    B, T = parent.shape
    dev = parent.device
    al = torch.empty(B, dtype=torch.int32, device=dev)
    an = torch.empty((B, T), dtype=torch.int32, device=dev)
    ot = torch.empty((B, T + 1), dtype=torch.int32, device=dev)
    ptd_verify(argmax, draft_tokens, parent, tree_len, B, T, al, an, ot, dev_status)
    return al, an, ot


def expand(parent, tokens, topk_idx, width_sched: Sequence[int], d_max: int, T_max: int,
           tree_len=None, dev_status=None):
    _need_gpu(parent, tokens, topk_idx, tree_len)
    B, T = parent.shape
    k = topk_idx.shape[-1]
    dev = parent.device
    pn = torch.empty((B, T_max), dtype=torch.int32, device=dev)
    tn = torch.empty((B, T_max), dtype=torch.int32, device=dev)
    ln = torch.empty(B, dtype=torch.int32, device=dev)
    ptd_expand(parent, tokens, tree_len, B, T, topk_idx, k, width_sched, d_max, T_max,
               pn, tn, ln, dev_status)
    return pn, tn, ln


def verify_expand(argmax, draft_tokens, parent, topk_idx, width_sched: Sequence[int],
                  d_max: int, T_max: int, tree_len=None, dev_status=None):
    """Returns (accept_len, accept_nodes, out_tokens, parent_next, tokens_next,
    tree_len_next)."""
    _need_gpu(argmax, draft_tokens, parent, topk_idx, tree_len)
    B, T = parent.shape
    k = topk_idx.shape[-1]
    dev = parent.device
    al = torch.empty(B, dtype=torch.int32, device=dev)
    an = torch.empty((B, T), dtype=torch.int32, device=dev)
    ot = torch.empty((B, T + 1), dtype=torch.int32, device=dev)
    pn = torch.empty((B, T_max), dtype=torch.int32, device=dev)
    tn = torch.empty((B, T_max), dtype=torch.int32, device=dev)
    ln = torch.empty(B, dtype=torch.int32, device=dev)
    ptd_verify_expand(argmax, draft_tokens, parent, tree_len, B, T, topk_idx, k, width_sched,
                      d_max, T_max, al, an, ot, pn, tn, ln, dev_status)
    return al, an, ot, pn, tn, ln


def tree_rope(q, k_cache, kv_len, parent, theta: float = 10000.0, inv_freq=None,
              pairing: int = PTD_ROPE_HALF, dev_status=None):
    """Turns q [B][T][Hq][D] and the tree rows kv_len + i of k_cache
    [B][Hkv][L_cap][D] in place (either may be None); returns the positions
    int32 [B][T]."""
    _need_gpu(q, k_cache, kv_len, parent)
    B, T = parent.shape
    ref = q if q is not None else k_cache
    Hq, D = (q.shape[2], q.shape[3]) if q is not None else (1, k_cache.shape[3])
    Hkv, L_cap = (k_cache.shape[1], k_cache.shape[2]) if k_cache is not None else (1, T)
    dt = _dtype_code(ref)
    shape = AttnShape(B, Hq, Hkv, D, L_cap, dt, dt, 0.0)
    pos = torch.empty((B, T), dtype=torch.int32, device=parent.device)
    ptd_tree_rope(q, k_cache, kv_len, parent, T, shape, theta, inv_freq, pairing, pos,
                  dev_status)
    return pos


def kv_commit(k_cache, v_cache, kv_len, accept_len, accept_nodes, dev_status=None):
    """Moves the accepted nodes' rows in place; returns kv_len_next int32 [B]."""
    _need_gpu(k_cache, v_cache, kv_len, accept_len, accept_nodes)
    B, Hkv, L_cap, D = k_cache.shape
    T = accept_nodes.shape[-1]
    dt = _dtype_code(k_cache)
    shape = AttnShape(B, Hkv, Hkv, D, L_cap, dt, dt, 0.0)
    nxt = torch.empty(B, dtype=torch.int32, device=k_cache.device)
    ptd_kv_commit(k_cache, v_cache, kv_len, accept_len, accept_nodes, T, shape, nxt,
                  dev_status)
    return nxt


def verify_sample(logits, draft_tokens, parent, temperature: float, u_node, u_bonus,
                  tree_len=None, workspace=None, dev_status=None):
    """logits [B][T+1][V] or [B*(T+1)][V] (unit stride along V); uniforms
    u_node float64 [B][T], u_bonus float64 [B][T+1].
    Returns (accept_len, accept_nodes, out_tokens)."""
    _need_gpu(draft_tokens, parent, tree_len, u_node, u_bonus)
    if not logits.is_cuda:
        raise ValueError("expected GPU logits")
    B, T = parent.shape
    lg = logits.reshape(B * (T + 1), logits.shape[-1]) if logits.dim() != 2 else logits
    if lg.stride(1) != 1:
        raise ValueError("logits need unit stride along the vocabulary")
    if u_node.dtype != torch.float64 or u_bonus.dtype != torch.float64:
        raise TypeError("uniforms are float64")
    V, ld = lg.shape[1], lg.stride(0)
    dev = parent.device
    al = torch.empty(B, dtype=torch.int32, device=dev)
    an = torch.empty((B, T), dtype=torch.int32, device=dev)
    ot = torch.empty((B, T + 1), dtype=torch.int32, device=dev)
    nbytes = ptd_verify_sample_workspace_bytes(B, T, V)
    if workspace is None:
        workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
    ptd_verify_sample(lg, _dtype_code(lg), V, ld, draft_tokens, parent, tree_len, B, T,
                      temperature, u_node, u_bonus, al, an, ot, workspace, workspace.numel(),
                      dev_status)
    return al, an, ot


def step_prune(parent, tokens, d_max: int, T_max: int, tree_len=None, dev_status=None):
    """Returns (parent_next, tokens_next, tree_len_next)."""
    _need_gpu(parent, tokens, tree_len)
    B, T = parent.shape
    dev = parent.device
    pn = torch.empty((B, T_max), dtype=torch.int32, device=dev)
    tn = torch.empty((B, T_max), dtype=torch.int32, device=dev)
    ln = torch.empty(B, dtype=torch.int32, device=dev)
    ptd_step_prune(parent, tokens, tree_len, B, T, d_max, T_max, pn, tn, ln, dev_status)
    return pn, tn, ln


class Pool:
    """A device candidate pool of B sequences (at most e_max trees of at
    most n_cap nodes per sequence), set up on construction."""

    def __init__(self, B: int, e_max: int, n_cap: int, device="cuda"):
        self.B, self.e_max, self.n_cap = B, e_max, n_cap
        self.nbytes = ptd_pool_bytes(B, e_max, n_cap)
        if not self.nbytes:
            raise ValueError("invalid pool sizes")
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        ptd_pool_init(self.buf, self.nbytes, B, e_max, n_cap)

    def merge(self, parent, tokens, tree_len=None, dev_status=None):
        _need_gpu(parent, tokens, tree_len)
        ptd_pool_merge(self.buf, self.nbytes, self.B, self.e_max, self.n_cap, parent, tokens,
                       tree_len, parent.shape[1], dev_status)

    def retrieve(self, last_token, T_max: int):
        """Returns (parent, tokens, tree_len) of the candidate trees."""
        _need_gpu(last_token)
        dev = self.buf.device
        po = torch.empty((self.B, T_max), dtype=torch.int32, device=dev)
        to = torch.empty((self.B, T_max), dtype=torch.int32, device=dev)
        ln = torch.empty(self.B, dtype=torch.int32, device=dev)
        ptd_pool_retrieve(self.buf, self.nbytes, self.B, self.e_max, self.n_cap, last_token,
                          T_max, po, to, ln)
        return po, to, ln


# ---------------------------------------------------------------------------
# prompts, page tables and 8-bit pages with block scales
# ---------------------------------------------------------------------------
def _need_here(*ts):
    """Tensors on the current device: the calls run on its current stream."""
    for t in ts:
        if t is not None and (not isinstance(t, torch.Tensor) or not t.is_cuda
                              or t.device.index != torch.cuda.current_device()):
            raise ValueError("expected tensors on the current GPU")


def _need_i32(*ts):
    _need_here(*ts)
    for t in ts:
        if t is not None and (t.dtype != torch.int32 or not t.is_contiguous()):
            raise ValueError("expected contiguous int32 tensors")


def _rows(t, heads=None):
    """Row stride of [N][heads][D] rows whose heads are dense."""
    if t.dim() != 3 or (t.shape[0] and (t.stride(2) != 1 or
                                        (t.shape[1] > 1 and t.stride(1) != t.shape[2]))):
        raise ValueError("expected [N][heads][D] rows with dense heads")
    if t.shape[0] > 1 and t.stride(0) < t.shape[1] * t.shape[2]:
        raise ValueError("expected rows that do not overlap")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2]


def prompt_attention(q, k, v, row_start, out=None, out_dtype=None, scale: float = 0.0,
                     dev_status=None):
    """Causal attention over packed prompts: q [N][Hq][D], k, v [N][Hkv][D] (views of
    a wider projection are taken as they are), row_start int32 [B + 1].  Returns
    out [N][Hq][D]; rows outside the sequences are left as they are (a new out:
    zero, which is a pass over it: 10 of 509 us for 8192 rows of 32 heads; an out that
    is passed in spares it)."""
    _need_here(q, k, v)
    _need_i32(row_start, dev_status)
    N, Hq, D = q.shape
    if k.shape != v.shape or k.shape[0] != N or k.shape[2] != D or k.dtype != q.dtype \
            or v.dtype != q.dtype or row_start.dim() != 1 or row_start.numel() < 2:
        raise ValueError("expected q [N][Hq][D], k and v [N][Hkv][D] of one dtype, row_start [B+1]")
    code = _dtype_code(q)
    if out is None:
        out = torch.zeros((N, Hq, D), dtype=out_dtype or q.dtype, device=q.device)
    elif out.shape != q.shape or not out.is_contiguous():
        raise ValueError("expected contiguous out of q's shape")
    _need_here(out)
    shape = PromptShape(row_start.numel() - 1, N, Hq, k.shape[1], D, _rows(q), _rows(k), _rows(v),
                        code, _dtype_code(out), float(scale))
    ptd_prompt_attention(q, k, v, row_start, out, shape, dev_status)
    return out


def qk_norm_rope(q, k, positions, q_weight=None, k_weight=None, eps: Optional[float] = 1e-6,
                 rot_dim: Optional[int] = None, theta: float = 10000.0, inv_freq=None,
                 pairing: int = PTD_ROPE_HALF, v=None, slots=None, k_pages=None, v_pages=None,
                 q_out=None, k_out=None, dev_status=None):
    """Norm of every head of q [N][Hq][D] and k [N][Hkv][D] (views of a wider projection are
    taken as they are; eps None: no norm), rotation of their first rot_dim dimensions
    (None: all) by positions int32 [N], and with slots int32 [N] the rows of k and v into k_pages,
    v_pages [pages][Hkv][page_size][D] (a contiguous cache [B][Hkv][L_cap][D] is B pages of L_cap
    rows).  Returns (q_out, k_out), new ones where not given (then rows at a negative position
    hold nothing); q and k themselves are turned in place."""
    _need_here(q, k, v, q_weight, k_weight, k_pages, v_pages, q_out, k_out)
    _need_i32(positions, slots, dev_status)
    if q.dim() != 3 or k.dim() != 3 or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2] or k.dtype != q.dtype:
        raise ValueError("expected q [N][Hq][D] and k [N][Hkv][D] of one dtype")
    N, Hq, D = q.shape
    Hkv, code = k.shape[1], _dtype_code(q)
    rot = D if rot_dim is None else rot_dim
    if (positions is not None and positions.numel() != N) or (slots is not None and slots.numel() != N):
        raise ValueError("expected a position and a slot per row")
    if eps is None and (q_weight is not None or k_weight is not None):
        raise ValueError("weights belong to the norm")
    w = [x for x in (q_weight, k_weight) if x is not None]
    if any(x.shape != (D,) or not x.is_contiguous() or x.dtype != w[0].dtype for x in w):
        raise ValueError("expected weights [D] of one dtype")
    store = None
    if slots is not None:
        if v is None or k_pages is None or v_pages is None or v.shape != k.shape or v.dtype != k.dtype:
            raise ValueError("expected v [N][Hkv][D], k_pages and v_pages with slots")
        for x in (k_pages, v_pages):
            if x.dim() != 4 or x.shape != k_pages.shape or x.shape[1] != Hkv or x.shape[3] != D \
                    or x.dtype != k.dtype or not x.is_contiguous():
                raise ValueError("expected contiguous pages [pages][Hkv][page_size][D] of k's dtype")
        store = KVStore(k_pages.data_ptr(), v_pages.data_ptr(), k_pages.shape[2], k_pages.shape[0])
    elif v is not None or k_pages is not None or v_pages is not None:
        raise ValueError("rows into pages need slots")
    if q_out is None:
        q_out = torch.empty((N, Hq, D), dtype=q.dtype, device=q.device)
    if k_out is None:
        k_out = torch.empty((N, Hkv, D), dtype=q.dtype, device=q.device)
    if q_out.shape != q.shape or k_out.shape != k.shape or q_out.dtype != q.dtype or k_out.dtype != k.dtype:
        raise ValueError("expected outputs of q's and k's shape and dtype")
    shape = QKShape(N, Hq, Hkv, D, rot, pairing, 0 if eps is None else 1, code,
                    _dtype_code(w[0]) if w else code, _rows(q), _rows(k), 0 if v is None else _rows(v),
                    _rows(q_out), _rows(k_out), 0.0 if eps is None else float(eps), float(theta))
    ptd_qk_norm_rope(q, k, v if store else None, q_weight, k_weight, positions, slots, q_out, k_out,
                     store, shape, inv_freq, dev_status)
    return q_out, k_out


def token_logprobs(logits, tokens=None, k: int = 0, nodes=None, temperature: float = 1.0,
                   with_entropy: bool = True, workspace=None, dev_status=None):
    """logits [R][V] or [B][T+1][V] with unit stride along V (rows may lie further apart),
    tokens int32 of R elements (-1: none) or None; with nodes int32 [B][T] (accept_nodes of
    verify) tokens are its out_tokens [B][T+1], and each is scored in the row that emitted it.
    Returns (logprob [R] or None, entropy [R] or None, idx [R][k], logprobs of idx [R][k]; None
    without k)."""
    _need_here(logits, workspace)
    _need_i32(tokens, nodes, dev_status)
    if logits.dim() != 2:
        logits = logits.reshape(-1, logits.shape[-1])
    R, V = logits.shape
    if V > 1 and logits.stride(1) != 1 or R > 1 and logits.stride(0) < V:
        raise ValueError("logits need unit stride along the vocabulary, and rows that do not overlap")
    T = 0
    if tokens is not None and tokens.numel() != R:
        raise ValueError("expected a token per row")
    if nodes is not None:
        if tokens is None or nodes.dim() != 2 or nodes.shape[0] * (nodes.shape[1] + 1) != R:
            raise ValueError("expected tokens [B][T+1] and nodes [B][T]")
        T = nodes.shape[1]
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("expected a contiguous workspace")
    dev = logits.device
    lp = torch.empty(R, dtype=torch.float32, device=dev) if tokens is not None else None
    ent = torch.empty(R, dtype=torch.float32, device=dev) if with_entropy else None
    idx = torch.empty((R, k), dtype=torch.int32, device=dev) if k else None
    val = torch.empty((R, k), dtype=torch.float32, device=dev) if k else None
    nbytes = ptd_token_logprobs_workspace_bytes(R, V, k)
    if workspace is None and nbytes:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    ptd_token_logprobs(logits, _dtype_code(logits), R, V, logits.stride(0) if R > 1 else V, tokens,
                       nodes, T, temperature, k, lp, ent, idx, val, workspace,
                       0 if workspace is None else workspace.numel() * workspace.element_size(), dev_status)
    return lp, ent, idx, val


def page_arrays(*caches):
    """The page arrays of caches for page_copy: BlockKV objects, or tensors of pages
    [num_pages][Hkv][page_size][D] of any dtype.  A program makes them once."""
    got = []
    for x in caches:
        if isinstance(x, BlockKV):
            got += [(y, 1) for y in (x.k_pages, x.v_pages)] + [(x.scales, x.scale_rows)]
        else:
            got.append((x, 1))
    pages = {x.shape[0] for x, _ in got}
    if len(pages) != 1 or any(x.dim() != 4 or not x.is_contiguous() for x, _ in got):
        raise ValueError("expected contiguous pages [num_pages][Hkv][page_size][D], as many in each cache")
    rows = [PageArray(x.data_ptr(), x.shape[1], x.shape[2], n, x.shape[3] * x.element_size()) for x, n in got]
    arrays = (PageArray * len(rows))(*rows)
    arrays.tensors = [x for x, _ in got]
    return arrays


def page_copy(arrays, src, dst, rows=None, dev_status=None):
    """Pages src[i] to dst[i] (int32 [n], -1: none) in every array of page_arrays(), the first
    rows[i] rows of them or (None) all."""
    _need_here(*arrays.tensors)
    _need_i32(src, dst, rows, dev_status)
    n = src.numel()
    if dst.numel() != n or (rows is not None and rows.numel() != n):
        raise ValueError("expected as many destinations and rows as sources")
    ptd_page_copy(arrays, arrays.tensors[0].shape[0], n, src, dst, rows, dev_status)


class PageTables:
    """Page tables of B sequences over num_pages pages of page_size rows, on the
    GPU: plan() gives every sequence the pages its lengths ask for.  With shared=True
    sequences may hold pages together: fork() and compact()."""

    def __init__(self, B: int, page_size: int, max_pages: int, num_pages: int, device="cuda",
                 shared: bool = False):
        def i32(*shape):
            return torch.empty(shape, dtype=torch.int32, device=device)

        self.page_table, self.num_held = i32(B, max_pages), i32(B)
        self.free_pages, self.num_free = i32(num_pages), i32(1)
        self.refs = torch.zeros(num_pages, dtype=torch.int32, device=device) if shared else None
        self.B, self.page_size = B, page_size
        self.max_pages, self.num_pages = max_pages, num_pages
        _need_here(self.page_table)
        ptd_page_init(self.state())

    def state(self) -> PageState:
        return PageState(self.page_table.data_ptr(), self.num_held.data_ptr(),
                         self.free_pages.data_ptr(), self.num_free.data_ptr(), self.B,
                         self.page_size, self.max_pages, self.num_pages)

    def plan(self, kv_len, new_len, N: int, rows_per_seq: int = 0, dev_status=None):
        """Returns (row_start [B + 1], or None with rows_per_seq; slots [N];
        positions [N])."""
        _need_i32(kv_len, new_len, dev_status, self.page_table)
        if kv_len.numel() != self.B or new_len.numel() != self.B:
            raise ValueError("expected lengths of B sequences")
        dev = self.page_table.device
        start = None if rows_per_seq else torch.empty(self.B + 1, dtype=torch.int32, device=dev)
        slots, pos = (torch.empty(N, dtype=torch.int32, device=dev) for _ in range(2))
        if self.refs is None:
            ptd_page_plan(self.state(), kv_len, new_len, N, rows_per_seq, start, slots, pos, dev_status)
        else:
            ptd_page_plan_shared(self.state(), self.refs, kv_len, new_len, N, rows_per_seq, start,
                                 slots, pos, dev_status)
        return start, slots, pos

    def _need_shared(self):
        if self.refs is None:
            raise ValueError("tables of one holder per page: make them with shared=True")

    def fork(self, from_, len_, dev_status=None):
        """Sequence b goes on from the first len_[b] rows of sequence from_[b] (-1: it ends);
        returns (copy_src, copy_dst, copy_rows) int32 [B] for page_copy, which has to follow before
        rows are written.  page_table and num_held are new tensors afterwards (so a captured fork goes
        on from the tables of its capture: a graph that is replayed calls ptd_page_fork with two
        tables of its own)."""
        self._need_shared()
        _need_i32(from_, len_, dev_status, self.page_table)
        if from_.numel() != self.B or len_.numel() != self.B:
            raise ValueError("expected sources and lengths of B sequences")
        dev = self.page_table.device
        table, held = torch.full_like(self.page_table, -1), torch.empty_like(self.num_held)
        src, dst, rows = (torch.empty(self.B, dtype=torch.int32, device=dev) for _ in range(3))
        ptd_page_fork(self.state(), self.refs, from_, len_, table, held, src, dst, rows, dev_status)
        self.page_table, self.num_held = table, held
        return src, dst, rows

    def compact(self, dev_status=None):
        """Moves the held pages to the lowest ids; returns (move_src, move_dst) int32
        [num_pages / 2] for page_copy, which has to follow."""
        self._need_shared()
        _need_i32(dev_status, self.page_table)
        dev = self.page_table.device
        src, dst = (torch.empty(self.num_pages // 2, dtype=torch.int32, device=dev) for _ in range(2))
        ptd_page_compact(self.state(), self.refs, src, dst, dev_status)
        return src, dst


class BlockKV:
    """One layer's keys and values in 8-bit pages with a scale per scale_rows rows
    and head (head dimension 128)."""

    def __init__(self, num_pages: int, Hkv: int, page_size: int, scale_rows: int = 32,
                 device="cuda"):
        if scale_rows not in (32, 64, 128) or page_size % scale_rows:
            raise ValueError("scale_rows is 32, 64 or 128 and divides page_size")
        shape = (num_pages, Hkv, page_size, 128)
        self.k_pages = torch.zeros(shape, dtype=torch.uint8, device=device)
        self.v_pages = torch.zeros(shape, dtype=torch.uint8, device=device)
        blocks = page_size // scale_rows
        n = num_pages * Hkv * blocks * 2
        # (the kernels read the exponents in 4-byte words)
        self._words = torch.full(((n + 3) // 4 * 4,), 127, dtype=torch.uint8, device=device)
        self.scales = self._words[:n].view(num_pages, Hkv, blocks, 2)
        self.num_pages, self.Hkv, self.page_size, self.scale_rows = num_pages, Hkv, page_size, scale_rows

    def pages(self, page_table=None) -> KVPagesFp8Blk:
        return KVPagesFp8Blk(self.k_pages.data_ptr(), self.v_pages.data_ptr(),
                             self.scales.data_ptr(),
                             None if page_table is None else page_table.data_ptr(),
                             self.page_size, 0 if page_table is None else page_table.shape[1],
                             self.num_pages, self.scale_rows)

    def write(self, k, v, slots, src=None, rows_per_seq: int = 0, dev_status=None):
        """Rows of k, v [N][Hkv][128] (bf16 or fp32) to the slots int32 [N] (any shape
        of N elements); src: rows within each sequence's rows_per_seq.  The rows of a
        block in front of the first new one keep their values, coded under the block's new
        scale: rejected tree rows can cost them places for good, unless a commit writes the
        sequence's last block anew from its first row (ptd_kv_write_fp8blk)."""
        _need_here(k, v, self.k_pages)
        _need_i32(slots, src, dev_status)
        N = slots.numel()
        if k.shape != v.shape or k.shape[0] != N or k.shape[1:] != (self.Hkv, 128) \
                or k.dtype != v.dtype or (src is not None and src.numel() != N):
            raise ValueError("expected k and v [N][Hkv][128] and N slots")
        ptd_kv_write_fp8blk(k, v, _dtype_code(k), _rows(k), _rows(v), N, slots, src, rows_per_seq,
                            self.pages(), self.Hkv, 128, dev_status)

    def tree_attention(self, q, page_table, kv_len, parent, out=None, out_dtype=None,
                       scale: float = 0.0, workspace=None, dev_status=None, tree_len=None):
        """q bf16 [B][T][Hq][128], page_table int32 [B][max_pages]; otherwise as
        tree_attention_paged."""
        _need_gpu(q, page_table, kv_len, parent, tree_len)
        _need_here(q, self.k_pages)
        _need_i32(page_table, kv_len, parent, tree_len, dev_status)
        B, T, Hq, D = q.shape
        if page_table.dim() != 2 or page_table.shape[0] != B or kv_len.numel() != B \
                or parent.shape != (B, T) or (tree_len is not None and tree_len.numel() != B):
            raise ValueError("expected page_table [B][max_pages], kv_len and tree_len [B], "
                             "parent [B][T]")
        if workspace is not None and not workspace.is_contiguous():
            raise ValueError("expected a contiguous workspace")
        if out is None:
            out = torch.empty((B, T, Hq, D), dtype=out_dtype or q.dtype, device=q.device)
        elif out.shape != q.shape or not out.is_contiguous():
            raise ValueError("expected contiguous out of q's shape")
        _need_here(out, workspace)
        shape = AttnShape(B, Hq, self.Hkv, D, page_table.shape[1] * self.page_size, _dtype_code(q),
                          _dtype_code(out), float(scale))
        nbytes = ptd_tree_attention_workspace_bytes(shape, T)
        if workspace is None and nbytes:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
        ptd_tree_attention_paged_fp8blk(q, self.pages(page_table), kv_len, tree_len, parent, T, out,
                                        shape, workspace,
                                        0 if workspace is None else workspace.numel(), dev_status)
        return out
