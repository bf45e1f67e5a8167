"""Thin Python binding of liblethe.so (include/lethe.h): argument marshalling
only.  Every step of the decode/prune path runs in the library's HIP kernels;
torch provides device memory and the current HIP stream.

There is no fallback: if the library is missing, importing this module's
functions raises.
"""
import ctypes
import math
import os

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "liblethe.so")

OK, ERR_INVALID, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = 0, -1, -2, -3, -4
BF16, F32, F16 = 0, 1, 2
MAX_AXES = 4
DEV_APPEND_OVERFLOW, DEV_INFEASIBLE, DEV_BAD_LAYOUT, DEV_HEAD_MISMATCH, DEV_WAIT_TIMEOUT = 1, 2, 4, 8, 16
OP_DECODE, OP_SPARSITY, OP_SELECT, OP_COMPACT, OP_DECODE_FINAL, OP_COMPACT_PLAN = 0, 1, 2, 3, 4, 5

SHRINK_NO_BREAKPOINT, SHRINK_NOT_TRIGGERED = -1, -2

EXPORTED = ("lethe_workspace_bytes", "lethe_state_bytes", "lethe_decode_attn_score", "lethe_decode_attn_score_final",
            "lethe_decode_attn_score_noalloc", "lethe_kv_compact_plan", "lethe_decode_attn_score_compact",
            "lethe_layer_sparsity", "lethe_rasr_select", "lethe_rasr_select_shared",
            "lethe_segmented_shrink", "lethe_kv_compact", "lethe_kv_compact_layers", "lethe_score_flush",
            "lethe_prefill_attn_score", "lethe_prefill_workspace_bytes", "lethe_paged_append",
            "lethe_paged_attn_score", "lethe_paged_attn_workspace_bytes", "lethe_paged_evict",
            "lethe_paged_evict_workspace_bytes", "lethe_status_string")


class CCache(ctypes.Structure):
    """Mirror of ``lethe_cache``."""
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("score", ctypes.c_void_p),
        ("len", ctypes.c_void_p), ("seq_base", ctypes.c_void_p), ("cap", ctypes.c_void_p),
        ("rows_per_layer", ctypes.c_int64), ("num_layers", ctypes.c_int32),
        ("num_seqs", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("dev_status", ctypes.c_void_p), ("state", ctypes.c_void_p),
    ]


class CPagedCache(ctypes.Structure):
    """Mirror of ``lethe_paged_cache``."""
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("score", ctypes.c_void_p), ("pos", ctypes.c_void_p),
        ("len", ctypes.c_void_p), ("seen", ctypes.c_void_p), ("page_table", ctypes.c_void_p),
        ("num_pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
        ("num_layers", ctypes.c_int32), ("num_seqs", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("dev_status", ctypes.c_void_p),
    ]


class CRotary(ctypes.Structure):
    """Mirror of ``lethe_rotary``."""
    _fields_ = [
        ("inv_freq", ctypes.c_void_p), ("axis_pos", ctypes.c_void_p), ("rot_dim", ctypes.c_int32),
        ("num_axes", ctypes.c_int32), ("sections", ctypes.c_int32 * MAX_AXES), ("adjacent", ctypes.c_int32),
    ]


class LetheError(RuntimeError):
    def __init__(self, fn, status):
        super().__init__("%s: %s (%d)" % (fn, status_string(status), status))
        self.status = status


_lib = None


def load():
    """Load liblethe.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("liblethe.so is not built; run `python -m paper_2511_06029_amd.build` "
                              "(the HIP library is required: there is no CPU fallback)")
        lib = ctypes.CDLL(LIB_PATH)
        vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
        pc = ctypes.POINTER(CCache)
        lib.lethe_workspace_bytes.argtypes = [pc, ctypes.c_int]
        lib.lethe_workspace_bytes.restype = sz
        lib.lethe_state_bytes.argtypes = [pc]
        lib.lethe_state_bytes.restype = sz
        lib.lethe_score_flush.argtypes = [pc, vp]
        lib.lethe_score_flush.restype = ctypes.c_int
        lib.lethe_decode_attn_score.argtypes = [pc, i32, vp, vp, vp, ctypes.c_float, ctypes.c_float, vp, vp, sz, vp]
        lib.lethe_decode_attn_score.restype = ctypes.c_int
        lib.lethe_decode_attn_score_final.argtypes = lib.lethe_decode_attn_score.argtypes
        lib.lethe_decode_attn_score_final.restype = ctypes.c_int
        lib.lethe_decode_attn_score_noalloc.argtypes = [pc, i32, vp, vp, vp, ctypes.c_float, ctypes.c_float, vp, vp]
        lib.lethe_decode_attn_score_noalloc.restype = ctypes.c_int
        lib.lethe_layer_sparsity.argtypes = [pc, vp, i32, i32, vp, vp, vp, vp, sz, vp]
        lib.lethe_layer_sparsity.restype = ctypes.c_int
        lib.lethe_rasr_select.argtypes = [pc, vp, i32, i32, vp, vp, sz, vp]
        lib.lethe_rasr_select.restype = ctypes.c_int
        lib.lethe_rasr_select_shared.argtypes = [pc, vp, i32, i32, vp, vp, sz, vp]
        lib.lethe_rasr_select_shared.restype = ctypes.c_int
        lib.lethe_segmented_shrink.argtypes = [pc, i32, ctypes.c_float, i32, i32, vp, vp, vp, vp, sz, vp]
        lib.lethe_segmented_shrink.restype = ctypes.c_int
        lib.lethe_prefill_attn_score.argtypes = [pc, i32, vp, vp, vp, ctypes.c_int64, i32, i32, ctypes.c_float,
                                                 vp, vp, sz, vp]
        lib.lethe_prefill_attn_score.restype = ctypes.c_int
        lib.lethe_prefill_workspace_bytes.argtypes = [pc, ctypes.c_int64]
        lib.lethe_prefill_workspace_bytes.restype = sz
        lib.lethe_kv_compact.argtypes = [pc, vp, vp, sz, vp]
        lib.lethe_kv_compact.restype = ctypes.c_int
        lib.lethe_kv_compact_layers.argtypes = [pc, i32, i32, vp, vp, sz, vp]
        lib.lethe_kv_compact_layers.restype = ctypes.c_int
        lib.lethe_kv_compact_plan.argtypes = [pc, vp, vp, sz, vp]
        lib.lethe_kv_compact_plan.restype = ctypes.c_int
        lib.lethe_decode_attn_score_compact.argtypes = [pc, i32, vp, vp, vp, ctypes.c_float, ctypes.c_float, vp,
                                                        vp, sz, vp, sz, vp]
        lib.lethe_decode_attn_score_compact.restype = ctypes.c_int
        i64, pp = ctypes.c_int64, ctypes.POINTER(CPagedCache)
        lib.lethe_paged_append.argtypes = [pp, i32, vp, i64, vp, i64, vp, i64, vp, vp, i64, i32,
                                           ctypes.POINTER(CRotary), vp, vp]
        lib.lethe_paged_append.restype = ctypes.c_int
        lib.lethe_paged_attn_score.argtypes = [pp, i32, vp, vp, vp, i64, i32, i32, ctypes.c_float, ctypes.c_float,
                                               ctypes.c_float, vp, vp, sz, vp]
        lib.lethe_paged_attn_score.restype = ctypes.c_int
        lib.lethe_paged_attn_workspace_bytes.argtypes = [pp, i64, i32, i32]
        lib.lethe_paged_attn_workspace_bytes.restype = sz
        lib.lethe_paged_evict.argtypes = [pp, vp, i32, i32, i32, vp, sz, vp]
        lib.lethe_paged_evict.restype = ctypes.c_int
        lib.lethe_paged_evict_workspace_bytes.argtypes = [pp]
        lib.lethe_paged_evict_workspace_bytes.restype = sz
        lib.lethe_status_string.argtypes = [ctypes.c_int]
        lib.lethe_status_string.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def status_string(status):
    return load().lethe_status_string(int(status)).decode()


DEV_STATUS_NAMES = ((DEV_APPEND_OVERFLOW, "append overflow"), (DEV_INFEASIBLE, "infeasible budget"),
                    (DEV_BAD_LAYOUT, "bad layout"), (DEV_HEAD_MISMATCH, "head mismatch"),
                    (DEV_WAIT_TIMEOUT, "wait timeout (results of that call unspecified)"))


def dev_status_names(bits):
    """The names of the device status bits set in `bits` (include/lethe.h)."""
    names = [name for bit, name in DEV_STATUS_NAMES if int(bits) & bit]
    rest = int(bits) & ~sum(bit for bit, _ in DEV_STATUS_NAMES)
    if rest:
        names.append("unknown bits %#x" % rest)
    return names


def _p(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        import torch
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _check(fn, st):
    if st != OK:
        raise LetheError(fn, st)


def workspace_bytes(cache, op):
    return int(load().lethe_workspace_bytes(ctypes.byref(cache.c_struct()), int(op)))


def state_bytes(cache):
    return int(load().lethe_state_bytes(ctypes.byref(cache.c_struct())))


def score_flush(cache, stream=None):
    """lethe_score_flush: apply the pending decode step of every (layer, sequence)."""
    _check("lethe_score_flush", load().lethe_score_flush(ctypes.byref(cache.c_struct()), _stream(stream)))


def decode_attn_score(cache, layer, q, k_new, v_new, gamma, softmax_scale, out, ws, stream=None):
    """lethe_decode_attn_score: append (k_new/v_new may be None), attend; the
    score update of this step stays pending until the next call on the layer,
    score_flush or a prune call."""
    st = load().lethe_decode_attn_score(ctypes.byref(cache.c_struct()), int(layer), _p(q), _p(k_new),
                                        _p(v_new), float(gamma), float(softmax_scale), _p(out), _p(ws),
                                        ws.numel() * ws.element_size(), _stream(stream))
    _check("lethe_decode_attn_score", st)


def decode_attn_score_final(cache, layer, q, k_new, v_new, gamma, softmax_scale, out, ws, stream=None):
    """lethe_decode_attn_score_final: the same step with its own score update
    applied within the call (nothing left pending); ws sized for
    OP_DECODE_FINAL."""
    st = load().lethe_decode_attn_score_final(ctypes.byref(cache.c_struct()), int(layer), _p(q), _p(k_new),
                                              _p(v_new), float(gamma), float(softmax_scale), _p(out), _p(ws),
                                              ws.numel() * ws.element_size(), _stream(stream))
    _check("lethe_decode_attn_score_final", st)


def decode_attn_score_noalloc(cache, layer, q, k_new, v_new, gamma, softmax_scale, out, stream=None):
    """lethe_decode_attn_score_noalloc: the decode step without a workspace
    (the chunk partials use the library's static device scratch)."""
    st = load().lethe_decode_attn_score_noalloc(ctypes.byref(cache.c_struct()), int(layer), _p(q), _p(k_new),
                                                _p(v_new), float(gamma), float(softmax_scale), _p(out),
                                                _stream(stream))
    _check("lethe_decode_attn_score_noalloc", st)


def layer_sparsity(cache, global_budget, recent, sink, sparsity_in, sparsity_out, budget_out,
                   ws=None, stream=None):
    """lethe_layer_sparsity: Hoyer sparsity per (sequence, layer) and budgets."""
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    st = load().lethe_layer_sparsity(ctypes.byref(cache.c_struct()), _p(global_budget), int(recent), int(sink),
                                     _p(sparsity_in), _p(sparsity_out), _p(budget_out), _p(ws), nbytes,
                                     _stream(stream))
    _check("lethe_layer_sparsity", st)


def rasr_select(cache, budget, recent, sink, keep, ws=None, stream=None):
    """lethe_rasr_select: keep mask of every segment."""
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    st = load().lethe_rasr_select(ctypes.byref(cache.c_struct()), _p(budget), int(recent), int(sink), _p(keep),
                                  _p(ws), nbytes, _stream(stream))
    _check("lethe_rasr_select", st)


def prefill_attn_score(cache, layer, q, q_start, q_len, max_q_len, max_kv_len, softmax_scale, out, ws,
                       stream=None):
    """lethe_prefill_attn_score: causal prefill attention over the q_len newest
    rows of every sequence, seeding their scores (Eq. 2).  q: bf16 [rows][H_Q][D];
    q_start int64 [B], q_len int32 [B] (device); out fp32 like q."""
    rows = q.shape[0]
    st = load().lethe_prefill_attn_score(ctypes.byref(cache.c_struct()), int(layer), _p(q), _p(q_start), _p(q_len),
                                         int(rows), int(max_q_len), int(max_kv_len), float(softmax_scale), _p(out),
                                         _p(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                         _stream(stream))
    _check("lethe_prefill_attn_score", st)


def rasr_select_shared(cache, budget, recent, sink, keep, ws=None, stream=None):
    """lethe_rasr_select_shared: one keep mask per (layer, sequence) from the
    head-summed score, written for every KV head."""
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    st = load().lethe_rasr_select_shared(ctypes.byref(cache.c_struct()), _p(budget), int(recent), int(sink),
                                         _p(keep), _p(ws), nbytes, _stream(stream))
    _check("lethe_rasr_select_shared", st)


def segmented_shrink(cache, segments, tau, recent, sink, evict_threshold, breakpoint, keep, ws=None,
                     stream=None):
    """lethe_segmented_shrink: Algorithm 1 with the size trigger; updates
    evict_threshold (int32 [L][B]) in place, fills breakpoint (or None)."""
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    st = load().lethe_segmented_shrink(ctypes.byref(cache.c_struct()), int(segments), float(tau), int(recent),
                                       int(sink), _p(evict_threshold), _p(breakpoint), _p(keep), _p(ws), nbytes,
                                       _stream(stream))
    _check("lethe_segmented_shrink", st)


def kv_compact(cache, keep, ws, stream=None):
    """lethe_kv_compact: in-place order-preserving compaction; updates len."""
    st = load().lethe_kv_compact(ctypes.byref(cache.c_struct()), _p(keep), _p(ws),
                                 ws.numel() * ws.element_size(), _stream(stream))
    _check("lethe_kv_compact", st)


def kv_compact_layers(cache, layer_begin, layer_count, keep, ws, stream=None):
    """lethe_kv_compact_layers: the compaction of layers layer_begin ..
    layer_begin + layer_count - 1 only."""
    st = load().lethe_kv_compact_layers(ctypes.byref(cache.c_struct()), int(layer_begin), int(layer_count), _p(keep),
                                        _p(ws), ws.numel() * ws.element_size(), _stream(stream))
    _check("lethe_kv_compact_layers", st)


def kv_compact_plan(cache, keep, plan, stream=None):
    """lethe_kv_compact_plan: record the compaction the next decode step of
    each layer carries out (nothing in the cache changes)."""
    st = load().lethe_kv_compact_plan(ctypes.byref(cache.c_struct()), _p(keep), _p(plan),
                                      plan.numel() * plan.element_size(), _stream(stream))
    _check("lethe_kv_compact_plan", st)


def decode_attn_score_compact(cache, layer, q, k_new, v_new, gamma, softmax_scale, out, plan, ws, stream=None):
    """lethe_decode_attn_score_compact: the layer's planned compaction, then
    its decode step, in one call."""
    st = load().lethe_decode_attn_score_compact(ctypes.byref(cache.c_struct()), int(layer), _p(q), _p(k_new),
                                                _p(v_new), float(gamma), float(softmax_scale), _p(out), _p(plan),
                                                plan.numel() * plan.element_size(), _p(ws),
                                                ws.numel() * ws.element_size(), _stream(stream))
    _check("lethe_decode_attn_score_compact", st)


def _row_stride(fn, t, heads, dim, dtype):
    """Elements between the rows of a [rows][heads][dim] tensor whose heads lie side by side."""
    rows, h, d = t.shape if t.dim() == 3 else (0, -1, -1)
    if h != heads or d != dim or t.dtype != dtype:
        raise LetheError(fn, ERR_INVALID)
    row, head, elem = t.stride()
    if rows and (elem != 1 or (heads > 1 and head != dim)):
        raise LetheError(fn, ERR_INVALID)
    return row if rows > 1 else heads * dim


def _check_place(fn, cache, *tensors):
    """Every tensor (None: not given) lies on the cache's device."""
    for t in tensors:
        if t is not None and t.device != cache.device:
            raise LetheError(fn, ERR_INVALID)


def _check_batch(fn, cache, q_start, q_len):
    _check_place(fn, cache, q_start, q_len)
    if (q_start.dtype != cache.torch.int64 or q_len.dtype != cache.torch.int32 or q_start.numel() != cache.B or
            q_len.numel() != cache.B or not q_start.is_contiguous() or not q_len.is_contiguous()):
        raise LetheError(fn, ERR_INVALID)


def _paged_call(fn, cache, stream, *args):
    """A call of the library on the cache's device and, by default, its current stream."""
    cuda = cache.torch.cuda
    if cuda.current_device() != cache.device.index:
        with cuda.device(cache.device):
            return _paged_call(fn, cache, stream, *args)
    if stream is None:  # the raw handle: a Stream object costs 2.8 us of the 12 that a one-token call takes
        stream = cache.torch._C._cuda_getCurrentRawStream(cache.device.index)
    elif not isinstance(stream, int):
        stream = stream.cuda_stream
    st = getattr(load(), fn)(cache.ref, *args, stream)
    if st != OK:
        raise LetheError(fn, st)


def paged_append(cache, layer, q, k_new, v_new, q_start, q_len, max_q_len, rotary, q_out, stream=None):
    """lethe_paged_append: rotate the new tokens' queries into q_out and their keys into the pages, with their
    values; rows of q, k_new and v_new may be strided (parts of one projection).  q and q_out may both be None;
    rotary None rotates nothing."""
    fn = "lethe_paged_append"
    rows = k_new.shape[0]
    kd = _row_stride(fn, k_new, cache.HK, cache.D, cache.tdtype)
    vd = _row_stride(fn, v_new, cache.HK, cache.D, cache.tdtype)
    qd, qp, op = 0, None, None
    if q is not None:
        qd, qp = _row_stride(fn, q, cache.HQ, cache.D, cache.tdtype), q.data_ptr()
    if v_new.shape[0] != rows or (q is not None and q.shape[0] != rows):
        raise LetheError(fn, ERR_INVALID)
    if q_out is not None:
        if q_out.dtype != cache.tdtype or not q_out.is_contiguous() or q_out.shape != (rows, cache.HQ, cache.D):
            raise LetheError(fn, ERR_INVALID)
        op = q_out.data_ptr()
    if rotary is not None and rotary.rows != rows:
        raise LetheError(fn, ERR_INVALID)
    _check_place(fn, cache, q, k_new, v_new, q_out, *(() if rotary is None else (rotary.inv_freq, rotary.axis_pos)))
    _check_batch(fn, cache, q_start, q_len)
    _paged_call(fn, cache, stream, layer, qp, qd, k_new.data_ptr(), kd, v_new.data_ptr(), vd, q_start.data_ptr(),
                q_len.data_ptr(), rows, max_q_len, None if rotary is None else rotary.ref, op)


def paged_attn_score(cache, layer, q, q_start, q_len, max_q_len, max_kv_len, gamma, softmax_scale, softcap, out, ws,
                     stream=None):
    """lethe_paged_attn_score: causal attention of the q_len newest rows of every sequence over its paged rows, with
    the score update where gamma > 0; scores capped by softcap * tanh(x / softcap) where softcap > 0.  q and out:
    [rows][H_Q][D] in the cache's type, contiguous; ws from cache.attn_workspace."""
    fn = "lethe_paged_attn_score"
    rows = q.shape[0]
    for t in (q, out):
        if t.dtype != cache.tdtype or not t.is_contiguous() or t.shape != (rows, cache.HQ, cache.D):
            raise LetheError(fn, ERR_INVALID)
    _check_place(fn, cache, q, out, ws)
    if not ws.is_contiguous():
        raise LetheError(fn, ERR_INVALID)
    _check_batch(fn, cache, q_start, q_len)
    _paged_call(fn, cache, stream, layer, q.data_ptr(), q_start.data_ptr(), q_len.data_ptr(), rows, max_q_len,
                max_kv_len, gamma, softmax_scale, softcap, out.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size())


def paged_evict(cache, budget, recent, sink, ws, max_kv_len=None, stream=None):
    """lethe_paged_evict: bring every segment to its budget (int32 [num_seqs][num_layers]); updates len.  ws from
    cache.evict_workspace; max_kv_len: an upper bound of the lengths (default: the tables' room)."""
    fn = "lethe_paged_evict"
    if budget.dtype != cache.torch.int32 or not budget.is_contiguous() or budget.shape != (cache.B, cache.L):
        raise LetheError(fn, ERR_INVALID)
    _check_place(fn, cache, budget, ws)
    if not ws.is_contiguous():
        raise LetheError(fn, ERR_INVALID)
    _paged_call(fn, cache, stream, budget.data_ptr(), recent, sink, 0x7fffffff if max_kv_len is None else max_kv_len,
                ws.data_ptr(), ws.numel() * ws.element_size())


class Rotary:
    """Rotary positions of a call of paged_append (``lethe_rotary``): inv_freq fp32 [rot_dim / 2], axis_pos int32
    [axes][rows], sections the number of pairs of each axis; adjacent pairs elements 2j and 2j + 1 instead of j and
    j + rot_dim / 2."""

    def __init__(self, inv_freq, axis_pos, sections, adjacent=False):
        if str(inv_freq.dtype) != "torch.float32" or not inv_freq.is_contiguous():
            raise LetheError("Rotary", ERR_INVALID)
        if str(axis_pos.dtype) != "torch.int32" or not axis_pos.is_contiguous() or axis_pos.dim() != 2:
            raise LetheError("Rotary", ERR_INVALID)
        if not 1 <= len(sections) <= MAX_AXES or axis_pos.shape[0] != len(sections):
            raise LetheError("Rotary", ERR_INVALID)
        self.inv_freq, self.axis_pos, self.rows = inv_freq, axis_pos, axis_pos.shape[1]
        full = [int(x) for x in sections] + [0] * (MAX_AXES - len(sections))
        self._c = CRotary(inv_freq.data_ptr(), axis_pos.data_ptr(), 2 * inv_freq.numel(), len(sections),
                          (ctypes.c_int32 * MAX_AXES)(*full), int(bool(adjacent)))

        self.ref = ctypes.byref(self._c)


class LethePagedCache:
    """A paged KV cache in the layout of include/lethe.h over tensors that the caller holds: k, v
    [pages][H_KV][page_size][D], score fp32 and pos int32 [pages][H_KV][page_size], len and seen int32 [layers][seqs],
    page_table int32 [layers][seqs][max_pages].  ``allocate`` makes them."""

    def __init__(self, k, v, score, pos, len_, seen, page_table, num_q_heads):
        import torch
        self.torch = torch
        self.num_pages, self.HK, self.page_size, self.D = (int(x) for x in k.shape)
        self.L, self.B, self.max_pages = (int(x) for x in page_table.shape)
        self.HQ = int(num_q_heads)
        self.tdtype = k.dtype
        codes = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}
        rows = (self.num_pages, self.HK, self.page_size)
        for t, dtype, shape in ((k, k.dtype, rows + (self.D,)), (v, k.dtype, rows + (self.D,)),
                                (score, torch.float32, rows), (pos, torch.int32, rows),
                                (len_, torch.int32, (self.L, self.B)), (seen, torch.int32, (self.L, self.B)),
                                (page_table, torch.int32, (self.L, self.B, self.max_pages))):
            if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.device != k.device:
                raise LetheError("LethePagedCache", ERR_INVALID)
        if k.dtype not in codes:
            raise LetheError("LethePagedCache", ERR_INVALID)
        self.k, self.v, self.score, self.pos = k, v, score, pos
        self.len, self.seen, self.page_table = len_, seen, page_table
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self._c = CPagedCache(k.data_ptr(), v.data_ptr(), score.data_ptr(), pos.data_ptr(), len_.data_ptr(),
                              seen.data_ptr(), page_table.data_ptr(), self.num_pages, self.page_size, self.max_pages,
                              self.L, self.B, self.HQ, self.HK, self.D, codes[k.dtype], self.dev_status.data_ptr())
        self.device, self.ref = k.device, ctypes.byref(self._c)
        if self.evict_workspace_bytes() == 0:
            raise LetheError("LethePagedCache", ERR_UNSUPPORTED)

    @classmethod
    def allocate(cls, num_layers, num_seqs, num_pages, page_size, max_pages, num_q_heads, num_kv_heads, head_dim,
                 dtype="bf16", device="cuda"):
        """An empty cache: no rows, no pages in any table (-1)."""
        import torch
        t = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
        rows = (num_pages, num_kv_heads, page_size)
        make = lambda shape, d: torch.zeros(shape, dtype=d, device=device)  # noqa: E731
        return cls(make(rows + (head_dim,), t), make(rows + (head_dim,), t), make(rows, torch.float32),
                   make(rows, torch.int32), make((num_layers, num_seqs), torch.int32),
                   make((num_layers, num_seqs), torch.int32),
                   torch.full((num_layers, num_seqs, max_pages), -1, dtype=torch.int32, device=device), num_q_heads)

    def evict_workspace_bytes(self):
        return int(load().lethe_paged_evict_workspace_bytes(self.ref))

    def evict_workspace(self):
        return self.torch.empty(self.evict_workspace_bytes(), dtype=self.torch.uint8, device=self.device)

    def attn_workspace(self, q_rows, max_q_len, max_kv_len):
        """Workspace of paged_attn_score for calls within these bounds."""
        n = int(load().lethe_paged_attn_workspace_bytes(self.ref, int(q_rows), int(max_q_len),
                                                        int(max_kv_len)))
        if n == 0:
            raise LetheError("lethe_paged_attn_workspace_bytes", ERR_UNSUPPORTED)
        return self.torch.empty(n, dtype=self.torch.uint8, device=self.device)


class LetheCache:
    """A ragged KV cache in the layout of include/lethe.h, allocated with torch.

    ``caps[b]`` rows per (layer, sequence, KV head) segment; segment (l, b, h)
    starts at row ``l * rows_per_layer + seq_base[b] + h * caps[b]``."""

    def __init__(self, num_layers, caps, num_q_heads, num_kv_heads, head_dim, dtype="bf16", device="cuda"):
        import torch
        self.torch = torch
        self.L = int(num_layers)
        self.caps = [int(c) for c in caps]
        self.B = len(self.caps)
        self.HQ, self.HK, self.D = int(num_q_heads), int(num_kv_heads), int(head_dim)
        self.G = self.HQ // self.HK
        self.dtype_code = BF16 if dtype == "bf16" else F32
        self.tdtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        bases, acc = [], 0
        for c in self.caps:
            bases.append(acc)
            acc += self.HK * c
        self.seq_base_host = bases
        self.rows_per_layer = max(acc, 1)
        R = self.rows_per_layer
        self.k = torch.zeros((self.L, R, self.D), dtype=self.tdtype, device=device)
        self.v = torch.zeros((self.L, R, self.D), dtype=self.tdtype, device=device)
        self.score = torch.zeros((self.L, R), dtype=torch.float32, device=device)
        self.len = torch.zeros((self.L, self.B), dtype=torch.int32, device=device)
        self.seq_base = torch.tensor(bases, dtype=torch.int64, device=device)
        self.cap = torch.tensor(self.caps, dtype=torch.int32, device=device)
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=device)
        self._c = None
        desc = self._struct(0)
        nstate = int(load().lethe_state_bytes(ctypes.byref(desc)))
        if nstate == 0:
            raise LetheError("lethe_state_bytes", ERR_UNSUPPORTED)
        self.state = torch.zeros(nstate, dtype=torch.uint8, device=device)

    def _struct(self, state_ptr):
        return CCache(self.k.data_ptr(), self.v.data_ptr(), self.score.data_ptr(), self.len.data_ptr(),
                      self.seq_base.data_ptr(), self.cap.data_ptr(), self.rows_per_layer, self.L, self.B,
                      self.HQ, self.HK, self.D, self.dtype_code, self.dev_status.data_ptr(), state_ptr)

    def c_struct(self):
        if self._c is None:
            self._c = self._struct(self.state.data_ptr())
        return self._c

    def flush(self, stream=None):
        """Make ``score`` current (apply the pending decode step)."""
        score_flush(self, stream)

    def reset_state(self):
        """Drop any pending decode step (after editing len / scores directly)."""
        self.state.zero_()

    def seg_rows(self, b, h):
        """Row range of segment (., b, h) within a layer."""
        start = self.seq_base_host[b] + h * self.caps[b]
        return start, start + self.caps[b]

    def workspace(self, op):
        n = workspace_bytes(self, op)
        return self.torch.zeros(max(n, 1), dtype=self.torch.uint8, device=self.k.device)

    def prefill_workspace(self, q_rows):
        n = int(load().lethe_prefill_workspace_bytes(ctypes.byref(self.c_struct()), int(q_rows)))
        return self.torch.zeros(max(n, 1), dtype=self.torch.uint8, device=self.k.device)

    def default_scale(self):
        return 1.0 / math.sqrt(self.D)
