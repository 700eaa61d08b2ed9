"""Same-name Python bindings of include/prism_ops.h (argument marshalling only; device tensors in,
device tensors out; work is enqueued on torch's current stream)."""
from __future__ import annotations

import ctypes as C

import torch

from .binding import PRISM_BF16, PRISM_IMPL_AUTO, PrismError, lib, _ProbeRecord

_proto_done = False


class _KvCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_stride", C.c_int64), ("num_pages", C.c_int32),
                ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32)]


def _L():
    global _proto_done
    L = lib()
    if not _proto_done:
        vp, i32, f32, f64 = C.c_void_p, C.c_int32, C.c_float, C.c_double
        L.prism_op_pack.argtypes = [vp, i32, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp]
        L.prism_op_embed.argtypes = [vp, i32, vp, i32, i32, vp, vp]
        L.prism_op_rmsnorm.argtypes = [vp, vp, i32, i32, i32, f32, vp, vp]
        L.prism_op_qknorm_rope.argtypes = [vp, i32, vp, i32, i32, i32, i32, i32, vp, vp, f32, f32, i32, vp]
        L.prism_op_gemm.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp]
        L.prism_op_gemm_qkv_rope.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, f32, vp, f32, i32, vp, vp]
        L.prism_op_gemm_qkv_rope.restype = C.c_int
        L.prism_op_attention.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, i32, vp, vp]
        L.prism_op_probe.argtypes = [vp, vp, i32, i32, vp, vp, i32, f32, vp, vp]
        L.prism_op_route.argtypes = [vp, vp, vp, i32, i32, i32, f64, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.prism_op_route_static.argtypes = L.prism_op_route.argtypes
        L.prism_op_route_static.restype = C.c_int
        L.prism_op_wait_selftest.argtypes = [C.c_uint64, vp, vp]
        L.prism_op_wait_selftest.restype = C.c_int
        L.prism_op_compact.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, vp]
        L.prism_op_gemm_bias.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp]
        L.prism_op_layernorm.argtypes = [vp, vp, vp, i32, i32, i32, f32, vp, vp]
        L.prism_op_embed_encoder.argtypes = [vp, vp, vp, i32, vp, vp, i32, i32, i32, vp, vp]
        L.prism_op_probe_encoder.argtypes = [vp, vp, i32, i32, vp, vp, f32, vp, i32, vp, vp, vp, vp, vp]
        L.prism_op_dequant_w4.argtypes = [vp, i32, i32, i32, vp, vp]
        i64, pkv = C.c_int64, C.POINTER(_KvCache)
        L.prism_op_page_append.argtypes = [vp, vp, vp, i32, i32, i32, i32, i64, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp]
        L.prism_op_page_release.argtypes = [vp, i32, vp, vp, i32, i32, i32, i32, i32, i64, vp, i64, vp, vp, vp, vp, vp, vp]
        L.prism_op_qknorm_rope_paged.argtypes = [vp, i64, vp, vp, i32, i32, i32, vp, vp, f32, f32, vp, i64, pkv, vp, vp]
        L.prism_op_attention_paged_bytes.argtypes = [i32] * 8 + [C.POINTER(i64), C.POINTER(i64)]
        L.prism_op_attention_paged_plan.argtypes = [vp, vp] + [i32] * 9 + [vp, i64, vp, vp]
        L.prism_op_attention_paged.argtypes = [vp, i64, pkv, vp, i64, i32, vp, i64, i32, i32, i32, i32, i32, vp, i64, vp, i64,
                                               vp, vp]
        for n in ("page_append", "page_release", "qknorm_rope_paged", "attention_paged_bytes", "attention_paged_plan",
                  "attention_paged"):
            getattr(L, "prism_op_" + n).restype = C.c_int
        for n in ("gemm_bias", "layernorm", "embed_encoder", "probe_encoder", "dequant_w4"):
            getattr(L, "prism_op_" + n).restype = C.c_int
        for n in ("pack", "embed", "rmsnorm", "qknorm_rope", "gemm", "attention", "probe", "route", "compact"):
            getattr(L, "prism_op_" + n).restype = C.c_int
        _proto_done = True
    return L


def _p(t):
    return None if t is None else t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _check(rc, what):
    if rc != 0:
        raise PrismError(rc, what)


def prism_op_pack(query, cand_tokens, cand_offsets, total, vocab, tokens, pos, cu, seq2orig, err_word):
    _check(_L().prism_op_pack(_p(query), query.numel(), _p(cand_tokens), _p(cand_offsets), cand_offsets.numel() - 1,
                              total, vocab, _p(tokens), _p(pos), _p(cu), _p(seq2orig), _p(err_word), _stream()), "pack")


def prism_op_embed(table, dtype, tokens, x):
    _check(_L().prism_op_embed(_p(table), dtype, _p(tokens), tokens.numel(), x.shape[1], _p(x), _stream()), "embed")


def prism_op_rmsnorm(x, gain, dtype, eps, out):
    _check(_L().prism_op_rmsnorm(_p(x), _p(gain), dtype, x.shape[0], x.shape[1], eps, _p(out), _stream()), "rmsnorm")


def prism_op_qknorm_rope(qkv, dtype, pos, n_q_heads, n_kv_heads, head_dim, qk_norm, g_q, g_k, eps, theta, max_pos):
    _check(_L().prism_op_qknorm_rope(_p(qkv), dtype, _p(pos), qkv.shape[0], n_q_heads, n_kv_heads, head_dim, qk_norm,
                                     _p(g_q), _p(g_k), eps, theta, max_pos, _stream()), "qknorm_rope")


def prism_op_gemm(a, b, b2, out, resid, m, n, k, dtype, epilogue, impl, err_word):
    _check(_L().prism_op_gemm(_p(a), _p(b), _p(b2), _p(out), _p(resid), m, n, k, dtype, epilogue, impl, _p(err_word),
                              _stream()), "gemm")


def prism_op_dequant_w4(blob, n, k, group, out):
    _check(_L().prism_op_dequant_w4(_p(blob), n, k, group, _p(out), _stream()), "dequant_w4")


def prism_op_gemm_bias(a, b, bias, out, resid, m, n, k, dtype, epilogue, impl, err_word):
    _check(_L().prism_op_gemm_bias(_p(a), _p(b), _p(bias), _p(out), _p(resid), m, n, k, dtype, epilogue, impl, _p(err_word),
                                   _stream()), "gemm_bias")


def prism_op_layernorm(x, gain, shift, dtype, eps, out):
    _check(_L().prism_op_layernorm(_p(x), _p(gain), _p(shift), dtype, x.shape[0], x.shape[1], eps, _p(out), _stream()),
           "layernorm")


def prism_op_embed_encoder(table, pos_table, type_row, dtype, tokens, pos, pos_offset, x):
    _check(_L().prism_op_embed_encoder(_p(table), _p(pos_table), _p(type_row), dtype, _p(tokens), _p(pos), pos_offset,
                                       tokens.numel(), x.shape[1], _p(x), _stream()), "embed_encoder")


def prism_op_probe_encoder(x, cu, n, gain, shift, eps, dense_w, dtype, dense_b, out_w, out_b, scores):
    _check(_L().prism_op_probe_encoder(_p(x), _p(cu), n, x.shape[1], _p(gain), _p(shift), eps, _p(dense_w), dtype, _p(dense_b),
                                       _p(out_w), _p(out_b), _p(scores), _stream()), "probe_encoder")


def prism_op_gemm_qkv_rope(a, w_qkv, out, m, k, n_q_heads, n_kv_heads, qk_norm, g_q, g_k, eps, pos, theta, max_pos, err_word):
    _check(_L().prism_op_gemm_qkv_rope(_p(a), _p(w_qkv), _p(out), m, k, n_q_heads, n_kv_heads, qk_norm, _p(g_q), _p(g_k),
                                       eps, _p(pos), theta, max_pos, _p(err_word), _stream()), "gemm_qkv_rope")


def prism_op_attention(qkv, out, cu, n_seq, max_len, n_q_heads, n_kv_heads, head_dim, causal, dtype, impl, err_word=None):
    _check(_L().prism_op_attention(_p(qkv), _p(out), _p(cu), n_seq, qkv.shape[0], max_len, n_q_heads, n_kv_heads, head_dim,
                                   causal, dtype, impl, _p(err_word), _stream()), "attention")


def prism_op_probe(x, cu, n, g_final, score_head, dtype, eps, scores):
    _check(_L().prism_op_probe(_p(x), _p(cu), n, x.shape[1], _p(g_final), _p(score_head), dtype, eps, _p(scores),
                               _stream()), "probe")


def prism_op_route(scores, cu_old, seq2orig_old, n, mode, keep_count, cv_threshold, n_clusters, std_ddof, select_winners,
                   is_final, layer, cu_new, seq2orig_new, old_of_new, state, res_idx, res_score, rec):
    _check(_L().prism_op_route(_p(scores), _p(cu_old), _p(seq2orig_old), n, mode, keep_count, cv_threshold, n_clusters,
                               std_ddof, select_winners, is_final, layer, _p(cu_new), _p(seq2orig_new), _p(old_of_new),
                               _p(state), _p(res_idx), _p(res_score), _p(rec), _stream()), "route")


def prism_op_route_static(scores, cu_old, seq2orig_old, n, mode, keep_count, cv_threshold, n_clusters, std_ddof,
                          select_winners, is_final, layer, cu_new, seq2orig_new, old_of_new, state, res_idx, res_score, rec):
    """prism_op_route without any device allocation (scratch built into the library; n <= 1024)."""
    _check(_L().prism_op_route_static(_p(scores), _p(cu_old), _p(seq2orig_old), n, mode, keep_count, cv_threshold,
                                      n_clusters, std_ddof, select_winners, is_final, layer, _p(cu_new), _p(seq2orig_new),
                                      _p(old_of_new), _p(state), _p(res_idx), _p(res_score), _p(rec), _stream()),
           "route_static")


def prism_op_compact(x_old, x_new, cu_old, cu_new, old_of_new, n_new, total_new):
    _check(_L().prism_op_compact(_p(x_old), _p(x_new), _p(cu_old), _p(cu_new), _p(old_of_new), n_new, total_new,
                                 x_old.shape[1], _stream()), "compact")


# ---- paged key/value cache.  Block tables are int32 [n_seq, max_pages] (rows may be strided), caches
# [num_pages, n_kv_heads, page_size, head_dim] (pages may be strided, what lies inside a page may not), matrices [rows, width]
# (rows may be strided).  A tensor of another element type or layout, or on another device than the current one, is refused:
# the kernels would read past it.
def _refuse_unless(ok, what):
    if not ok:
        raise PrismError(-1, what)


def _here(what, *tensors):
    devices = {t.get_device() for t in tensors if t is not None}  # -1: host memory
    _refuse_unless(len(devices) == 1 and -1 not in devices and torch.cuda.current_device() in devices,
                   what + ": a tensor is not on the current device")


def _ints(what, *pairs):
    for t, n in pairs:
        _refuse_unless(t.dtype == torch.int32 and t.is_contiguous() and t.numel() >= n, what + ": int32, contiguous, long enough")


def _rows(what, t, dtype, width=None):
    _refuse_unless(t.dim() == 2 and t.dtype == (torch.bfloat16 if dtype == PRISM_BF16 else torch.float32) and
                   (t.shape[1] == width or width is None) and (t.stride(1) == 1 or t.numel() <= 1),
                   what + ": matrix of the stated element type and width, rows without gaps inside")
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], t.stride(0))


def _table(what, t, n):
    _refuse_unless(t.dim() == 2 and t.dtype == torch.int32 and t.shape[0] >= n and (t.stride(1) == 1 or t.shape[1] <= 1 or t.numel() == 0),
                   what + ": int32 block table with a row per sequence")
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], t.stride(0))


def _cache(what, k, v, dtype):
    _refuse_unless(k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype ==
                   (torch.bfloat16 if dtype == PRISM_BF16 else torch.float32), what + ": k and v caches of one layout")
    pages, heads, page, dh = k.shape
    _refuse_unless(k[:1].is_contiguous(), what + ": a page of the cache has gaps inside")
    stride = k.stride(0) if pages > 1 else heads * page * dh
    return _KvCache(_p(k), _p(v), stride, pages, page, heads, dh, dtype)


def prism_op_page_append(len_new, kv_len_in, kv_len_out, page_size, num_pages, block_table, free_pages, n_free_in, n_free_out,
                         cu_q, pos, slot_map, err_word):
    n, total = len_new.numel(), slot_map.numel()
    _here("page_append", len_new, kv_len_in, kv_len_out, block_table, free_pages, n_free_in, n_free_out, cu_q, pos, slot_map,
          err_word)
    _ints("page_append", (len_new, n), (kv_len_in, n), (kv_len_out, n), (free_pages, num_pages), (n_free_in, 1), (n_free_out, 1),
          (cu_q, n + 1), (pos, total), (slot_map, total), (err_word, 1))
    stride = _table("page_append", block_table, n)
    _check(_L().prism_op_page_append(_p(len_new), _p(kv_len_in), _p(kv_len_out), n, page_size, num_pages, block_table.shape[1],
                                     stride, _p(block_table), _p(free_pages), _p(n_free_in), _p(n_free_out), total, _p(cu_q),
                                     _p(pos), _p(slot_map), _p(err_word), _stream()), "page_append")


def prism_op_page_release(old_of_new, kv_len_in, kv_len_out, page_size, num_pages, shared_pages, table_in, table_out, free_pages,
                          n_free_in, n_free_out, err_word, n_new=None):
    """n_new: survivors (default: all of old_of_new, which may be a longer buffer)."""
    n, n_new = kv_len_in.numel(), old_of_new.numel() if n_new is None else n_new
    _here("page_release", old_of_new, kv_len_in, kv_len_out, table_in, table_out, free_pages, n_free_in, n_free_out, err_word)
    _ints("page_release", (old_of_new, n_new), (kv_len_in, n), (kv_len_out, n), (free_pages, num_pages), (n_free_in, 1),
          (n_free_out, 1), (err_word, 1))
    s_in, s_out = _table("page_release", table_in, n), _table("page_release", table_out, n)
    _refuse_unless(table_out.shape[1] == table_in.shape[1], "page_release: tables of one width")
    _check(_L().prism_op_page_release(_p(old_of_new), n_new, _p(kv_len_in), _p(kv_len_out), n, page_size, num_pages, shared_pages,
                                      table_in.shape[1], s_in, _p(table_in), s_out, _p(table_out), _p(free_pages),
                                      _p(n_free_in), _p(n_free_out), _p(err_word), _stream()), "page_release")


def prism_op_qknorm_rope_paged(qkv, dtype, pos, slot_map, n_q_heads, qk_norm, g_q, g_k, eps, theta, q_out, k_cache, v_cache,
                               err_word):
    what = "qknorm_rope_paged"
    _here(what, qkv, pos, slot_map, g_q, g_k, q_out, k_cache, v_cache, err_word)
    c = _cache(what, k_cache, v_cache, dtype)
    rows = qkv.shape[0]
    s_in = _rows(what, qkv, dtype, (n_q_heads + 2 * c.n_kv_heads) * c.head_dim)
    s_out = _rows(what, q_out, dtype, n_q_heads * c.head_dim)
    _refuse_unless(q_out.shape[0] >= rows, what + ": a row of q_out for every row of qkv")
    _ints(what, (pos, rows), (slot_map, rows), (err_word, 1))
    for g in (g_q, g_k) if qk_norm else ():
        _refuse_unless(g is not None and g.dtype == qkv.dtype and g.is_contiguous() and g.numel() == c.head_dim, what + ": gains")
    _check(_L().prism_op_qknorm_rope_paged(_p(qkv), s_in, _p(pos), _p(slot_map), rows, n_q_heads, qk_norm, _p(g_q), _p(g_k), eps,
                                           theta, _p(q_out), s_out, C.byref(c), _p(err_word), _stream()), what)


def prism_op_attention_paged_bytes(n_seq, total_q, max_q_len, n_q_heads, n_kv_heads, head_dim, dtype, impl=PRISM_IMPL_AUTO):
    """(bytes of the plan, bytes of the workspace); needs no device."""
    plan, ws = C.c_int64(), C.c_int64()
    _check(_L().prism_op_attention_paged_bytes(n_seq, total_q, max_q_len, n_q_heads, n_kv_heads, head_dim, dtype, impl,
                                               C.byref(plan), C.byref(ws)), "attention_paged_bytes")
    return plan.value, ws.value


def prism_op_attention_paged_plan(cu_q, kv_len, total_q, max_q_len, n_q_heads, n_kv_heads, head_dim, dtype, causal, plan, err_word,
                                  impl=PRISM_IMPL_AUTO):
    n = kv_len.numel()
    _here("attention_paged_plan", cu_q, kv_len, plan, err_word)
    _ints("attention_paged_plan", (cu_q, n + 1), (kv_len, n), (err_word, 1))
    _refuse_unless(plan.is_contiguous(), "attention_paged_plan: plan")
    _check(_L().prism_op_attention_paged_plan(_p(cu_q), _p(kv_len), n, total_q, max_q_len, n_q_heads, n_kv_heads, head_dim, dtype,
                                              causal, impl, _p(plan), plan.numel() * plan.element_size(), _p(err_word),
                                              _stream()), "attention_paged_plan")


def prism_op_attention_paged(q, k_cache, v_cache, block_table, plan, n_seq, max_q_len, n_q_heads, dtype, out, workspace, err_word,
                             impl=PRISM_IMPL_AUTO):
    what = "attention_paged"
    _here(what, q, k_cache, v_cache, block_table, plan, out, workspace, err_word)
    c = _cache(what, k_cache, v_cache, dtype)
    s_q = _rows(what, q, dtype, n_q_heads * c.head_dim)
    s_out = _rows(what, out, dtype, n_q_heads * c.head_dim)
    _refuse_unless(out.shape[0] >= q.shape[0], what + ": a row of out for every row of q")
    _ints(what, (err_word, 1))
    stride = _table(what, block_table, n_seq)
    _refuse_unless(plan.is_contiguous() and (workspace is None or workspace.is_contiguous()), what + ": plan and workspace")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_L().prism_op_attention_paged(_p(q), s_q, C.byref(c), _p(block_table), stride, block_table.shape[1], _p(plan),
                                         plan.numel() * plan.element_size(), n_seq, q.shape[0], max_q_len, n_q_heads, impl,
                                         _p(out), s_out, _p(workspace), ws_bytes, _p(err_word), _stream()), what)


def prism_op_wait_selftest(limit_cycles, err_word):
    _check(_L().prism_op_wait_selftest(int(limit_cycles), _p(err_word), _stream()), "wait_selftest")


RECORD_BYTES = C.sizeof(_ProbeRecord)


def decode_record(buf: torch.Tensor) -> _ProbeRecord:
    """A uint8 tensor holding one prism_probe_record (copied from the device) -> ctypes struct."""
    raw = bytes(buf.cpu().numpy().tobytes())
    return _ProbeRecord.from_buffer_copy(raw)
