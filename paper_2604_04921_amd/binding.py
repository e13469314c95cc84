"""ctypes binding of libtri.so: same entry points as include/tri.h, argument marshalling only.

torch owns the device memory and the stream; every step of the path runs inside the library.
"""
import ctypes
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtri.so")

TRI_OK = 0
TRI_ERR_INVALID_ARG, TRI_ERR_UNSUPPORTED, TRI_ERR_WORKSPACE, TRI_ERR_HIP = -1, -2, -3, -4
TRI_F32, TRI_BF16, TRI_FP4 = 0, 1, 2
TRI_PAIR_INTERLEAVED, TRI_PAIR_HALF = 0, 1
TRI_SCORE_FULL, TRI_SCORE_TRIG_ONLY, TRI_SCORE_NORM_ONLY, TRI_SCORE_NORM_UNWEIGHTED = 0, 1, 2, 3

EXPORTS = ["tri_last_error", "tri_build_centers", "tri_centers_accumulate", "tri_centers_finalize", "tri_band_diagnostics", "tri_workspace_size", "tri_score", "tri_select_topk",
           "tri_compact", "tri_compact_fill", "tri_compress_step", "tri_static_scratch_size", "tri_compress_step_static",
           "tri_append", "tri_attend", "tri_attend_shared", "tri_attend_workspace_size", "tri_append4", "tri_pack4", "tri_unpack4", "tri_attend4", "tri_attend4_shared",
           "tri_attend4_workspace_size", "tri_timing_attach", "tri_timing_detach"]


class TriModel(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("rope_theta", ctypes.c_double), ("pairs", ctypes.c_int32),
                ("n_offsets", ctypes.c_int32), ("offsets", ctypes.c_void_p), ("score_variant", ctypes.c_int32),
                ("head_budgets", ctypes.c_void_p)]


class TriCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("dtype", ctypes.c_int32), ("n_seqs", ctypes.c_int32),
                ("seq_len", ctypes.c_void_p), ("cur_pos", ctypes.c_void_p),
                ("max_seq_len", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("block_table", ctypes.c_void_p), ("max_blocks_per_seq", ctypes.c_int32),
                ("stride_layer", ctypes.c_int64), ("stride_seq_or_block", ctypes.c_int64),
                ("stride_head", ctypes.c_int64), ("stride_slot", ctypes.c_int64),
                ("pos_stride_layer", ctypes.c_int64), ("pos_stride_seq_or_block", ctypes.c_int64),
                ("pos_stride_head", ctypes.c_int64), ("k_rotated", ctypes.c_int32), ("n_blocks", ctypes.c_int32)]


class TriCache4(ctypes.Structure):
    _fields_ = [("c", TriCache), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("rows", ctypes.c_int32)]


class TriTokens(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("max_tokens", ctypes.c_int32), ("start", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("head_len", ctypes.c_void_p), ("rotated", ctypes.c_int32)]


class TriAttention(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("out", ctypes.c_void_p), ("q_stride_token", ctypes.c_int64), ("q_stride_head", ctypes.c_int64),
                ("out_stride_token", ctypes.c_int64), ("out_stride_head", ctypes.c_int64), ("scale", ctypes.c_float),
                ("causal", ctypes.c_int32)]


class TriError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__("tri status %d: %s" % (status, msg))
        self.status = status


_lib = None


def lib():
    """Load libtri.so.  torch is imported first so that the HIP runtime it ships is the one in use."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libtri.so is not built (run paper_2604_04921_amd/build.py); there is no fallback")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        L.tri_last_error.restype = ctypes.c_char_p
        L.tri_last_error.argtypes = []
        L.tri_build_centers.restype = i32
        L.tri_build_centers.argtypes = [ctypes.POINTER(TriModel), vp, i32, i64, vp, vp]
        L.tri_centers_accumulate.restype = i32
        L.tri_centers_accumulate.argtypes = [ctypes.POINTER(TriModel), vp, i32, i64, vp, i32, vp]
        L.tri_centers_finalize.restype = i32
        L.tri_centers_finalize.argtypes = [ctypes.POINTER(TriModel), vp, i64, vp, vp]
        L.tri_band_diagnostics.restype = i32
        L.tri_band_diagnostics.argtypes = [ctypes.POINTER(TriModel), vp, vp, vp, vp, i32, vp, vp]
        L.tri_workspace_size.restype = ctypes.c_size_t
        L.tri_workspace_size.argtypes = [ctypes.POINTER(TriModel), ctypes.POINTER(TriCache), i32]
        L.tri_score.restype = i32
        L.tri_score.argtypes = [ctypes.POINTER(TriModel), vp, ctypes.POINTER(TriCache), vp, vp, vp, ctypes.c_size_t, vp]
        L.tri_select_topk.restype = i32
        L.tri_select_topk.argtypes = [ctypes.POINTER(TriModel), vp, ctypes.POINTER(TriCache), i32, vp, vp, vp,
                                      ctypes.c_size_t, vp]
        L.tri_compact.restype = i32
        L.tri_compact.argtypes = [ctypes.POINTER(TriModel), ctypes.POINTER(TriCache), ctypes.POINTER(TriCache), i32,
                                  vp, vp, vp, vp]
        L.tri_compact_fill.restype = i32
        L.tri_compact_fill.argtypes = [ctypes.POINTER(TriModel), ctypes.POINTER(TriCache), i32, vp, vp, vp, vp]
        L.tri_compress_step.restype = i32
        L.tri_compress_step.argtypes = [ctypes.POINTER(TriModel), vp, ctypes.POINTER(TriCache),
                                        ctypes.POINTER(TriCache), i32, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.tri_static_scratch_size.restype = ctypes.c_size_t
        L.tri_static_scratch_size.argtypes = []
        L.tri_compress_step_static.restype = i32
        L.tri_compress_step_static.argtypes = [ctypes.POINTER(TriModel), vp, ctypes.POINTER(TriCache),
                                               ctypes.POINTER(TriCache), i32, vp, vp, vp, vp]
        L.tri_append.restype = i32
        L.tri_append.argtypes = [ctypes.POINTER(TriModel), ctypes.POINTER(TriCache), i32, ctypes.POINTER(TriTokens), vp, vp, i64, i64, vp, vp]
        L.tri_attend.restype = i32
        L.tri_attend.argtypes = [ctypes.POINTER(TriModel), ctypes.POINTER(TriCache), i32, ctypes.POINTER(TriTokens),
                                 ctypes.POINTER(TriAttention), vp, ctypes.c_size_t, vp]
        L.tri_attend_shared.restype = i32
        L.tri_attend_shared.argtypes = [ctypes.POINTER(TriModel), ctypes.POINTER(TriCache), vp, ctypes.POINTER(TriCache), i32,
                                        ctypes.POINTER(TriTokens), ctypes.POINTER(TriAttention), vp, ctypes.c_size_t, vp]
        L.tri_attend_workspace_size.restype = ctypes.c_size_t
        L.tri_attend_workspace_size.argtypes = [ctypes.POINTER(TriModel), ctypes.POINTER(TriCache), ctypes.POINTER(TriCache),
                                                ctypes.POINTER(TriTokens)]
        c4 = ctypes.POINTER(TriCache4)
        L.tri_append4.restype = i32
        L.tri_append4.argtypes = [ctypes.POINTER(TriModel), c4, i32, ctypes.POINTER(TriTokens), vp, vp, i64, i64, vp, vp]
        L.tri_pack4.restype = i32
        L.tri_pack4.argtypes = [ctypes.POINTER(TriModel), ctypes.POINTER(TriCache), c4, i32, vp, vp, vp, vp]
        L.tri_unpack4.restype = i32
        L.tri_unpack4.argtypes = [ctypes.POINTER(TriModel), c4, ctypes.POINTER(TriCache), i32, vp, vp, vp, vp]
        L.tri_attend4.restype = i32
        L.tri_attend4.argtypes = [ctypes.POINTER(TriModel), c4, i32, ctypes.POINTER(TriTokens), ctypes.POINTER(TriAttention), vp, ctypes.c_size_t, vp]
        L.tri_attend4_shared.restype = i32
        L.tri_attend4_shared.argtypes = [ctypes.POINTER(TriModel), c4, vp, ctypes.POINTER(TriCache), i32, ctypes.POINTER(TriTokens), ctypes.POINTER(TriAttention), vp,
                                         ctypes.c_size_t, vp]
        L.tri_attend4_workspace_size.restype = ctypes.c_size_t
        L.tri_attend4_workspace_size.argtypes = [ctypes.POINTER(TriModel), c4, ctypes.POINTER(TriCache), ctypes.POINTER(TriTokens)]
        L.tri_timing_attach.restype = i32
        L.tri_timing_attach.argtypes = [vp, i32]
        L.tri_timing_detach.restype = i32
        L.tri_timing_detach.argtypes = []
        _lib = L
    return _lib


def _check(rc):
    if rc != TRI_OK:
        raise TriError(rc, lib().tri_last_error().decode())


def _p(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None:
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # (the current stream's handle without an object around it: 1 us of a call)
        return raw(-1) if raw is not None else torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream


def _dtype(t):
    if t.dtype == torch.bfloat16:
        return TRI_BF16
    if t.dtype == torch.float32:
        return TRI_F32
    raise TypeError("float32 or bfloat16 tensors only, got %s" % t.dtype)


class Model:
    """Host-side tri_model; keeps the offsets array alive."""

    def __init__(self, n_layers, n_q_heads, n_kv_heads, head_dim, rope_theta, offsets, pairs=TRI_PAIR_INTERLEAVED,
                 score_variant=TRI_SCORE_FULL, head_budgets=None):
        self._offsets = np.ascontiguousarray(offsets, dtype=np.int64)
        self._head_budgets = head_budgets   # device int32 [n_layers][n_kv_heads] or None; kept alive here
        if head_budgets is not None:
            assert head_budgets.dtype == torch.int32 and head_budgets.is_contiguous()
            assert tuple(head_budgets.shape) == (n_layers, n_kv_heads)
        self.c = TriModel(n_layers, n_q_heads, n_kv_heads, head_dim, float(rope_theta), pairs, len(self._offsets),
                          self._offsets.ctypes.data_as(ctypes.c_void_p), int(score_variant),
                          None if head_budgets is None else head_budgets.data_ptr())
        self.n_layers, self.n_q_heads, self.n_kv_heads, self.head_dim = n_layers, n_q_heads, n_kv_heads, head_dim   # (a field of the struct costs a call 0.1 us)
        self.ref = ctypes.byref(self.c)


class Cache:
    """tri_cache over torch tensors.

    contiguous: k, v [L][S][Hkv][N][d], pos [L][S][Hkv][N]
    paged:      k, v [L][n_blocks][Hkv][block][d], pos [L][n_blocks][Hkv][block], block_table [S][max_blocks]
    Strides are taken from the tensors; the last dimension must be dense."""

    def __init__(self, k, v, pos, seq_len, cur_pos, max_seq_len, block_table=None, k_rotated=False):
        assert k.dim() == 5 and pos.dim() == 4 and k.stride(4) == 1 and pos.stride(3) == 1
        assert v is None or (v.stride() == k.stride() and v.dtype == k.dtype)
        assert pos.dtype == torch.int32 and seq_len.dtype == torch.int32 and cur_pos.dtype == torch.int32
        self.tensors = (k, v, pos, seq_len, cur_pos, block_table)
        self.n_seqs, self.dtype, self.device = seq_len.numel(), k.dtype, k.device
        self.sizes = tuple(min(n) for n in zip(k.shape[:4], pos.shape, (k if v is None else v).shape))
        self.layers, self.heads = self.sizes[0], self.sizes[2]
        bs = 0 if block_table is None else k.shape[3]
        self.c = TriCache(k.data_ptr(), 0 if v is None else v.data_ptr(), pos.data_ptr(), _dtype(k),
                          seq_len.numel(), seq_len.data_ptr(), cur_pos.data_ptr(), int(max_seq_len), bs,
                          0 if block_table is None else block_table.data_ptr(),
                          0 if block_table is None else block_table.shape[1],
                          k.stride(0), k.stride(1), k.stride(2), k.stride(3),
                          pos.stride(0), pos.stride(1), pos.stride(2), int(bool(k_rotated)),
                          0 if block_table is None else k.shape[1])
        if block_table is not None:
            assert block_table.dtype == torch.int32 and block_table.is_contiguous()
        self.ref = ctypes.byref(self.c)


class Cache4:
    """tri_cache4 over torch tensors: keys (post-RoPE) and values in 4 bits.

    contiguous: k, v uint8 [L][S][Hkv][N][64], k_scale, v_scale uint8 [L][S][Hkv][N][4], pos int32 [L][S][Hkv][N]
    paged:      the same over blocks, as Cache
    Strides are taken from the tensors (k_scale's and v_scale's are four times those of pos); the last dimensions must be dense.  rows: the type of k_new, v_new, q and out (None: bfloat16)."""

    def __init__(self, k, v, k_scale, v_scale, pos, seq_len, cur_pos, max_seq_len, block_table=None, rows=None):
        for t in (k, v, k_scale, v_scale):
            if t.dtype != torch.uint8 or t.dim() != 5 or t.stride(4) != 1 or t.device != k.device:
                raise ValueError("k, v, k_scale, v_scale: uint8 of five dimensions with dense rows, on one device")
        if k.shape[4] != 64 or v.shape != k.shape or v.stride() != k.stride():
            raise ValueError("k, v: rows of 64 bytes, of the same shape and strides, got %s and %s" % (tuple(k.shape), tuple(v.shape)))
        if pos.dtype != torch.int32 or pos.shape != k.shape[:4] or pos.stride(3) != 1 or pos.device != k.device:
            raise ValueError("pos: int32 %s with dense rows, where k is" % (tuple(k.shape[:4]),))
        for t in (k_scale, v_scale):
            if t.shape != pos.shape + (4,) or t.stride()[:4] != tuple(4 * n for n in pos.stride()):
                raise ValueError("k_scale, v_scale: %s with four times the strides of pos" % (tuple(pos.shape) + (4,),))
        for t in (seq_len, cur_pos, block_table):
            if t is not None and (t.dtype != torch.int32 or not t.is_contiguous() or t.device != k.device):
                raise ValueError("seq_len, cur_pos, block_table: int32, contiguous, where k is")
        if cur_pos.numel() != seq_len.numel():
            raise ValueError("cur_pos: as many as seq_len's %d, got %d" % (seq_len.numel(), cur_pos.numel()))
        if block_table is None and (k.shape[1] < seq_len.numel() or k.shape[3] < max_seq_len):
            raise ValueError("k, v: %d sequences of %d slots, got %s" % (seq_len.numel(), max_seq_len, tuple(k.shape)))
        if block_table is not None and (block_table.dim() != 2 or block_table.shape[0] < seq_len.numel()):
            raise ValueError("block_table: two dimensions, %d sequences, got %s" % (seq_len.numel(), tuple(block_table.shape)))
        rows = torch.bfloat16 if rows is None else rows
        if rows not in (torch.bfloat16, torch.float32):
            raise TypeError("rows: float32 or bfloat16, got %s" % rows)
        self.tensors = (k, v, k_scale, v_scale, pos, seq_len, cur_pos, block_table)
        self.n_seqs, self.dtype, self.device = seq_len.numel(), rows, k.device
        self.sizes = tuple(k.shape[:4])
        self.layers, self.heads = self.sizes[0], self.sizes[2]
        table = (0, 0, 0, 0) if block_table is None else (k.shape[3], block_table.data_ptr(), block_table.shape[1], k.shape[1])
        c = TriCache(k.data_ptr(), v.data_ptr(), pos.data_ptr(), TRI_FP4, seq_len.numel(), seq_len.data_ptr(), cur_pos.data_ptr(), int(max_seq_len), table[0], table[1], table[2],
                     *(2 * k.stride(i) for i in range(4)), pos.stride(0), pos.stride(1), pos.stride(2), 1, table[3])
        self.c = TriCache4(c, k_scale.data_ptr(), v_scale.data_ptr(), TRI_BF16 if rows == torch.bfloat16 else TRI_F32)
        self.ref = ctypes.byref(self.c)


class Tokens:
    """tri_tokens over torch tensors: a step's new tokens, sequence by sequence.

    pos int32 [T]; start int32 [S + 1] (None: one token per sequence); max_tokens bounds the tokens of one sequence (default T);
    head_len int32 [L][S][Hkv] or None; rotated: the q and k rows given are post-RoPE already."""

    def __init__(self, pos, start=None, max_tokens=None, head_len=None, rotated=False):
        for t in (pos, start, head_len):
            assert t is None or (t.dtype == torch.int32 and t.is_contiguous())
        self.tensors = (pos, start, head_len)
        self.n_tokens = n = pos.numel()
        self.starts, self.head_shape, self.device = None if start is None else start.numel(), None if head_len is None else tuple(head_len.shape), pos.device
        for t in (start, head_len):
            if t is not None and t.device != pos.device:
                raise ValueError("start and head_len must lie where pos does, on %s" % pos.device)
        self.c = TriTokens(n, n if max_tokens is None else int(max_tokens), None if start is None else start.data_ptr(), pos.data_ptr(),
                           None if head_len is None else head_len.data_ptr(), int(bool(rotated)))
        self.ref = ctypes.byref(self.c)


def _here(t, cache, name):
    if t.device != cache.device:
        raise ValueError("%s: on %s, the cache on %s" % (name, t.device, cache.device))


def _rows(t, heads, tokens, cache, name):
    """Strides of rows [T][heads][d] of the cache's type and device, d dense; any strides of the other two (0 where there is one token, or head)."""
    n, strides = tokens.n_tokens, t.stride()
    if t.shape != (n, heads, 128) or strides[2] != 1:
        raise ValueError("%s: [%d][%d][128] with dense rows, got %s" % (name, n, heads, tuple(t.shape)))
    if t.dtype != cache.dtype:
        raise TypeError("%s: %s, the cache holds %s" % (name, t.dtype, cache.dtype))
    if t.device != cache.device:
        _here(t, cache, name)
    if n == 1 or heads == 1:
        return strides[0] if n > 1 else 0, strides[1] if heads > 1 else 0
    return strides


def _covers(model, cache, layer, name="the cache"):
    """That a layer's call stays inside the cache's arrays."""
    if cache.layers <= layer or cache.heads < model.n_kv_heads:
        raise ValueError("%s: %d layers of %d heads, not layer %d of %d heads" % (name, cache.layers, cache.heads, layer, model.n_kv_heads))


def _room(model, cache, seqs, slots, name):
    """That the cache's arrays have all layers and heads of the model, and `slots` slots of `seqs` sequences; paged, that a table has these sequences, and the arrays all blocks that ids can name."""
    layers, many, heads, most = cache.sizes
    k, table = cache.tensors[0], cache.tensors[-1]
    if layers < model.n_layers or heads < model.n_kv_heads:
        raise ValueError("%s: %d layers of %d heads, the model's %d of %d" % (name, layers, heads, model.n_layers, model.n_kv_heads))
    if table is None and (many < seqs or most < slots):
        raise ValueError("%s: room for %d sequences of %d slots, not %d of %d" % (name, many, most, seqs, slots))
    if table is not None and (table.dim() != 2 or table.shape[0] < seqs or (many, most) != (k.shape[1], k.shape[3])):
        raise ValueError("%s: a table %s of %d blocks of %d for %d sequences, k's blocks being %d of %d" % (name, tuple(table.shape), many, most, seqs, k.shape[1], k.shape[3]))


def _fits(model, cache, tokens):
    """What the kernels take on trust of the step's arrays: their sizes, and that they lie where the cache does."""
    if tokens.starts is not None and tokens.starts <= cache.n_seqs:
        raise ValueError("start: %d entries, not n_seqs + 1 = %d" % (tokens.starts, cache.n_seqs + 1))
    if tokens.head_shape is not None:
        got, shape = tokens.head_shape, (model.n_layers, cache.n_seqs, model.n_kv_heads)
        if got != shape and got != (shape[0] * shape[1] * shape[2],):
            raise ValueError("head_len: %s, not %s" % (got, shape))
    if tokens.device != cache.device:
        _here(tokens, cache, "the step's tokens")


def _bytes(workspace, cache):
    if workspace is None:
        return 0
    _here(workspace, cache, "workspace")
    if not workspace.is_contiguous():
        raise ValueError("workspace: must be contiguous")
    return workspace.numel() * workspace.element_size()


def _append(entry, model, cache, layer, tokens, k_new, v_new, new_seq_len, stream):
    strides = _rows(k_new, model.n_kv_heads, tokens, cache, "k_new")
    if _rows(v_new, model.n_kv_heads, tokens, cache, "v_new") != strides:
        raise ValueError("k_new and v_new must have the same strides")
    _covers(model, cache, layer)
    _fits(model, cache, tokens)
    _lengths(new_seq_len, cache)
    _check(entry(model.ref, cache.ref, layer, tokens.ref, k_new.data_ptr(), v_new.data_ptr(), strides[0], strides[1],
                 _p(new_seq_len), _stream(stream)))


def _lengths(new_seq_len, cache):
    if new_seq_len is not None:
        _here(new_seq_len, cache, "new_seq_len")
        if new_seq_len.dtype != torch.int32:
            raise TypeError("new_seq_len: int32, got %s" % new_seq_len.dtype)
        if new_seq_len.numel() < cache.n_seqs or not new_seq_len.is_contiguous():
            raise ValueError("new_seq_len: %d entries side by side, got %s" % (cache.n_seqs, tuple(new_seq_len.shape)))


def tri_append(model, cache, layer, tokens, k_new, v_new, new_seq_len=None, stream=None):
    """k_new, v_new [T][Hkv][d], with the same strides, to the end of every sequence of layer `layer`.  new_seq_len int32 [S] or None."""
    _append(lib().tri_append, model, cache, layer, tokens, k_new, v_new, new_seq_len, stream)


def tri_append4(model, cache, layer, tokens, k_new, v_new, new_seq_len=None, stream=None):
    """tri_append for a Cache4: rows of its `rows` type, rotated on the way where the step's are pre-RoPE, and rounded to 4 bits."""
    _append(lib().tri_append4, model, cache, layer, tokens, k_new, v_new, new_seq_len, stream)


def _move(entry, model, src, dst, budget, kept_idx, kept_cnt, new_seq_len, stream):
    _here(dst, src, "dst")
    most = (src.c.c if isinstance(src, Cache4) else src.c).max_seq_len
    _room(model, src, src.n_seqs, most, "src")
    _room(model, dst, src.n_seqs, min(int(budget), most), "dst")
    inst = model.n_layers * src.n_seqs * model.n_kv_heads
    for t, n, name in ((kept_idx, inst * int(budget), "kept_idx"), (kept_cnt, inst, "kept_cnt")):
        if t is not None:
            _here(t, src, name)
            if t.dtype != torch.int32 or not t.is_contiguous() or t.numel() < n:
                raise ValueError("%s: int32, %d entries side by side, got %s %s" % (name, n, t.dtype, tuple(t.shape)))
    _lengths(new_seq_len, src)
    _check(entry(model.ref, src.ref, dst.ref, int(budget), _p(kept_idx), _p(kept_cnt), _p(new_seq_len), _stream(stream)))


def tri_pack4(model, src, dst, budget, kept_idx=None, kept_cnt=None, new_seq_len=None, stream=None):
    """Slots of a Cache into a Cache4, all layers: those that kept_idx [L][S][Hkv][budget] and kept_cnt [L][S][Hkv] name, or the first min(length, budget).  dst has arrays for src's
    sequences and min(budget, src's max_seq_len) slots of each; its own lengths and max_seq_len are not read."""
    _move(lib().tri_pack4, model, src, dst, budget, kept_idx, kept_cnt, new_seq_len, stream)


def tri_unpack4(model, src, dst, budget, kept_idx=None, kept_cnt=None, new_seq_len=None, stream=None):
    """Slots of a Cache4 into a Cache (k_rotated), as tri_pack4."""
    _move(lib().tri_unpack4, model, src, dst, budget, kept_idx, kept_cnt, new_seq_len, stream)


def _attention(model, cache, layer, tokens, q, out, scale, causal):
    _covers(model, cache, layer)
    _fits(model, cache, tokens)
    heads = model.n_q_heads
    qs, os_ = _rows(q, heads, tokens, cache, "q"), _rows(out, heads, tokens, cache, "out")
    return TriAttention(q.data_ptr(), out.data_ptr(), qs[0], qs[1], os_[0], os_[1], model.head_dim ** -0.5 if scale is None else scale,
                        1 if causal else 0)


def tri_attend(model, cache, layer, tokens, q, out, scale=None, causal=True, workspace=None, stream=None):
    """out [T][Hq][d] <- attention of q [T][Hq][d] over layer `layer` of the cache.  scale None: 1 / sqrt(d)."""
    at = _attention(model, cache, layer, tokens, q, out, scale, causal)
    _check(lib().tri_attend(model.ref, cache.ref, layer, tokens.ref, ctypes.byref(at), _p(workspace), _bytes(workspace, cache), _stream(stream)))


def tri_attend_shared(model, prefix, group, cache, layer, tokens, q, out, scale=None, causal=True, workspace=None, stream=None):
    """tri_attend with the keys of shared prefixes: group int32 [P + 1] (first sequence of every prefix's), None for one prefix."""
    assert group is None or (group.dtype == torch.int32 and group.is_contiguous() and group.numel() == prefix.c.n_seqs + 1)
    at = _attention(model, cache, layer, tokens, q, out, scale, causal)
    _here(prefix, cache, "prefix")
    _covers(model, prefix, layer, "prefix")
    if group is not None:
        _here(group, cache, "group")
    _check(lib().tri_attend_shared(model.ref, prefix.ref, _p(group), cache.ref, layer, tokens.ref, ctypes.byref(at), _p(workspace),
                                   _bytes(workspace, cache), _stream(stream)))


def tri_attend_workspace_size(model, cache, tokens, prefix=None):
    n = int(lib().tri_attend_workspace_size(model.ref, None if prefix is None else prefix.ref, cache.ref, tokens.ref))
    if n == ctypes.c_size_t(-1).value:
        raise TriError(TRI_ERR_INVALID_ARG, lib().tri_last_error().decode())
    return n


def tri_attend4(model, cache, layer, tokens, q, out, scale=None, causal=True, workspace=None, stream=None):
    """tri_attend over a Cache4; q and out of its `rows` type."""
    at = _attention(model, cache, layer, tokens, q, out, scale, causal)
    _check(lib().tri_attend4(model.ref, cache.ref, layer, tokens.ref, ctypes.byref(at), _p(workspace), _bytes(workspace, cache), _stream(stream)))


def tri_attend4_shared(model, prefix, group, cache, layer, tokens, q, out, scale=None, causal=True, workspace=None, stream=None):
    """tri_attend_shared with the prefixes in a Cache4, the sequences' own keys in a Cache of the prefix's `rows` type."""
    if group is not None and (group.dtype != torch.int32 or not group.is_contiguous() or group.numel() != prefix.n_seqs + 1):
        raise ValueError("group: int32, %d entries side by side" % (prefix.n_seqs + 1))
    at = _attention(model, cache, layer, tokens, q, out, scale, causal)
    _here(prefix, cache, "prefix")
    _covers(model, prefix, layer, "prefix")
    if group is not None:
        _here(group, cache, "group")
    _check(lib().tri_attend4_shared(model.ref, prefix.ref, _p(group), cache.ref, layer, tokens.ref, ctypes.byref(at), _p(workspace),
                                    _bytes(workspace, cache), _stream(stream)))


def tri_attend4_workspace_size(model, cache, tokens, own=None):
    """Bytes for tri_attend4, or (own: the sequences' Cache, `cache` being the prefixes') for tri_attend4_shared."""
    n = int(lib().tri_attend4_workspace_size(model.ref, cache.ref, None if own is None else own.ref, tokens.ref))
    if n == ctypes.c_size_t(-1).value:
        raise TriError(TRI_ERR_INVALID_ARG, lib().tri_last_error().decode())
    return n


def tri_build_centers(model, q_samples, centers_out, stream=None):
    """q_samples [T][L][Hq][d] (contiguous) -> centers_out [L][Hq][F][3] float32."""
    assert q_samples.is_contiguous() and centers_out.is_contiguous() and centers_out.dtype == torch.float32
    _check(lib().tri_build_centers(model.ref, _p(q_samples), _dtype(q_samples), q_samples.shape[0], _p(centers_out),
                                   _stream(stream)))


def tri_centers_accumulate(model, q_samples, sums, first, stream=None):
    """Adds the sums of one chunk q_samples [T][L][Hq][d] to sums [L][Hq][F][3] float64 (first: overwrite)."""
    assert q_samples.is_contiguous() and sums.is_contiguous() and sums.dtype == torch.float64
    _check(lib().tri_centers_accumulate(model.ref, _p(q_samples), _dtype(q_samples), q_samples.shape[0], _p(sums),
                                        int(bool(first)), _stream(stream)))


def tri_centers_finalize(model, sums, total_tokens, centers_out, stream=None):
    assert sums.is_contiguous() and sums.dtype == torch.float64 and centers_out.dtype == torch.float32
    _check(lib().tri_centers_finalize(model.ref, _p(sums), int(total_tokens), _p(centers_out), _stream(stream)))


def tri_band_diagnostics(model, q_centers, k_centers, mrl_out, contrib_out=None, top_k=0, top_bands_out=None, stream=None):
    _check(lib().tri_band_diagnostics(model.ref, _p(q_centers), _p(k_centers), _p(mrl_out), _p(contrib_out), int(top_k),
                                      _p(top_bands_out), _stream(stream)))


def tri_workspace_size(model, cache, budget):
    return int(lib().tri_workspace_size(model.ref, cache.ref, int(budget)))


def tri_score(model, centers, cache, final_out, raw_out, workspace, stream=None):
    _check(lib().tri_score(model.ref, _p(centers), cache.ref, _p(final_out), _p(raw_out), _p(workspace),
                           workspace.numel() * workspace.element_size(), _stream(stream)))


def tri_select_topk(model, final_scores, cache, budget, kept_idx, kept_cnt, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().tri_select_topk(model.ref, _p(final_scores), cache.ref, int(budget), _p(kept_idx), _p(kept_cnt),
                                 _p(workspace), ws_bytes, _stream(stream)))


def tri_compact(model, src, dst, budget, kept_idx, kept_cnt, new_seq_len=None, stream=None):
    _check(lib().tri_compact(model.ref, src.ref, dst.ref, int(budget), _p(kept_idx), _p(kept_cnt), _p(new_seq_len),
                             _stream(stream)))


def tri_compact_fill(model, cache, budget, kept_idx, kept_cnt, new_seq_len=None, stream=None):
    _check(lib().tri_compact_fill(model.ref, cache.ref, int(budget), _p(kept_idx), _p(kept_cnt), _p(new_seq_len),
                                  _stream(stream)))


def tri_compress_step(model, centers, src, dst, budget, kept_idx, kept_cnt, new_seq_len, workspace, stream=None):
    _check(lib().tri_compress_step(model.ref, _p(centers), src.ref, dst.ref if dst is not None else None, int(budget), _p(kept_idx), _p(kept_cnt),
                                   _p(new_seq_len), _p(workspace), workspace.numel() * workspace.element_size(),
                                   _stream(stream)))


def tri_static_scratch_size():
    return int(lib().tri_static_scratch_size())


def tri_compress_step_static(model, centers, src, dst, budget, kept_idx, kept_cnt, new_seq_len, stream=None):
    """tri_compress_step on the library's own scratch array: no workspace argument, no allocation."""
    _check(lib().tri_compress_step_static(model.ref, _p(centers), src.ref, dst.ref if dst is not None else None, int(budget),
                                          _p(kept_idx), _p(kept_cnt), _p(new_seq_len), _stream(stream)))


def tri_timing_attach(events):
    """events: list of torch.cuda.Event (timing enabled, each recorded once before so that its handle exists),
    laid out start0, stop0, start1, stop1, ...  Returns the ctypes array that must be kept alive until detach."""
    arr = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
    _check(lib().tri_timing_attach(arr, len(events) // 2))
    return arr


def tri_timing_detach():
    return int(lib().tri_timing_detach())
