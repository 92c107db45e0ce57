"""Convenience layer over binding.py: uploads host arrays, allocates outputs and
workspace with torch, calls the library.  No arithmetic of the method lives here."""

import contextlib

import numpy as np
import torch

from . import binding as B


# name -> (slkv_dtype, torch dtype of the queries, torch dtype of keys and values)
DTYPES = {"f32": (B.SLKV_F32, torch.float32, torch.float32), "bf16": (B.SLKV_BF16, torch.bfloat16, torch.bfloat16),
          "f16": (B.SLKV_F16, torch.float16, torch.float16),
          "bf16_kv8": (B.SLKV_BF16_KV_FP8, torch.bfloat16, torch.uint8)}   # E4M3 bytes travel as uint8
# types of a cache (Cache): these, and 4 bits, whose bytes hold two E2M1 values each, with an exponent byte for every 32 of them
CACHE_DTYPES = dict(DTYPES, bf16_kv4=(B.SLKV_BF16_KV_MXFP4, torch.bfloat16, torch.uint8))
_NOTHING = torch.empty((0,), dtype=torch.uint8)


def to_device(arr, dtype, device="cuda"):
    """numpy fp32 / fp16 array, uint16 array of bfloat16 bit patterns or uint8 array of E4M3 bytes -> device tensor."""
    if dtype == "bf16_kv8":
        arr = np.ascontiguousarray(arr)
        if arr.dtype == np.uint8:
            return torch.from_numpy(arr).to(device)
        dtype = "bf16"
    if dtype == "bf16":
        t = torch.from_numpy(np.ascontiguousarray(arr).view(np.int16)).to(device)
        return t.view(torch.bfloat16)
    if dtype == "f16":
        return torch.from_numpy(np.ascontiguousarray(arr, dtype=np.float16)).to(device)
    return torch.from_numpy(np.ascontiguousarray(arr, dtype=np.float32)).to(device)


def to_host(t):
    """device tensor -> numpy (bfloat16 comes back as uint16 bit patterns)."""
    if t.dtype == torch.bfloat16:
        return t.view(torch.int16).cpu().numpy().view(np.uint16)
    return t.cpu().numpy()


class _Buffers:
    """What the two kinds of call share.  The constructor allocates and zero-fills on the stream that is current there; run() on another stream
    asks, as for the inputs, that this stream has waited for that one.  Calls of one object use the same buffers: each has to wait for the one before it."""

    def _failed(self, error, stream):
        if error.status == B.SLKV_ERR_HIP:      # some of its launches may have run: the next call finds the workspace's header clear all the same
            try:
                with torch.cuda.stream(stream):
                    self.workspace[:B.SLKV_WORKSPACE_HEADER_BYTES].zero_()
            except RuntimeError:                # (a device that takes no launch at all: the call's own error is the one to report)
                pass


class LayerCall(_Buffers):
    """Device buffers + descriptor for repeated calls on one layer's shapes."""

    def __init__(self, dtype, B_, Hq, Hkv, d, w, cu_seqlens, budgets, pool_kernel=7, pool=B.SLKV_POOL_MAX,
                 device="cuda", debug_scores=False, k_strides=None, v_strides=None):
        """k_strides / v_strides: (token stride, head stride) in elements; default = head-major
        contiguous [Hkv][T][d]."""
        T = int(cu_seqlens[-1])
        self.dtype = dtype
        self.layer = B.Layer(DTYPES[dtype][0], B_, Hq, Hkv, d, w, cu_seqlens,
                             budgets, k_strides or (d, T * d), v_strides or (d, T * d), pool_kernel, pool)
        self.offsets, self.total_kept = B.slkv_compacted_sizes(self.layer)
        tdt = DTYPES[dtype][2]
        rows = max(self.total_kept, 1)
        self.k_out = torch.empty((rows, d), dtype=tdt, device=device)
        self.v_out = torch.empty((rows, d), dtype=tdt, device=device)
        self.kept_idx = torch.empty((rows,), dtype=torch.int32, device=device)
        self.out_offsets = torch.empty((B_ * Hkv + 1,), dtype=torch.int64, device=device)
        self.workspace = torch.zeros((B.slkv_workspace_bytes(self.layer),), dtype=torch.uint8, device=device)   # zero-filled once
        self.importance = self.pooled = None
        if debug_scores:
            self.importance = torch.zeros((max(Hkv * T, 1),), dtype=torch.float32, device=device)
            self.pooled = torch.zeros((max(Hkv * T, 1),), dtype=torch.float32, device=device)

    def run(self, qwin, k, v, stream=None):
        try:
            B.slkv_compress_layer(self.layer, qwin, k, v, self.k_out, self.v_out, self.kept_idx, self.workspace,
                                  self.out_offsets, self.importance, self.pooled, stream)
        except B.SlkvError as e:
            self._failed(e, stream)
            raise


class RaggedCall(_Buffers):
    """Device buffers + descriptor for repeated re-compression calls on one ragged cache shape."""

    def __init__(self, dtype, B_, Hq, Hkv, d, w, in_offsets, budgets, pool_kernel=7, pool=B.SLKV_POOL_MAX,
                 device="cuda", debug_scores=False, positions=True):
        rows_in = int(in_offsets[-1])
        self.rag = B.Ragged(DTYPES[dtype][0], B_, Hq, Hkv, d, w, in_offsets, budgets,
                            pool_kernel, pool)
        self.offsets, self.total_kept = B.slkv_recompress_sizes(self.rag)
        tdt = DTYPES[dtype][2]
        rows = max(self.total_kept, 1)
        self.k_out = torch.empty((rows, d), dtype=tdt, device=device)
        self.v_out = torch.empty((rows, d), dtype=tdt, device=device)
        self.kept_idx = torch.empty((rows,), dtype=torch.int32, device=device)
        self.pos_out = torch.empty((rows,), dtype=torch.int32, device=device) if positions else None
        self.out_offsets = torch.empty((B_ * Hkv + 1,), dtype=torch.int64, device=device)
        self.workspace = torch.zeros((B.slkv_recompress_workspace_bytes(self.rag),), dtype=torch.uint8, device=device)
        self.importance = self.pooled = None
        if debug_scores:
            self.importance = torch.zeros((max(rows_in, 1),), dtype=torch.float32, device=device)
            self.pooled = torch.zeros((max(rows_in, 1),), dtype=torch.float32, device=device)

    def run(self, qwin, k_in, v_in, pos_in=None, stream=None):
        try:
            B.slkv_recompress_layer(self.rag, qwin, k_in, v_in, self.k_out, self.v_out, self.kept_idx, self.workspace,
                                    pos_in, self.pos_out if pos_in is not None else None, self.out_offsets,
                                    self.importance, self.pooled, stream)
        except B.SlkvError as e:
            self._failed(e, stream)
            raise


def score_heads(rows, needle_start, needle_len, topk, acc=None, stream=None):
    """rows: [L,H,T,n] fp32 device tensor.  Returns (acc [L,H,5], scores [L,H,3]) float64 device tensors."""
    L, H, T, n = rows.shape
    first = acc is None
    if first:
        acc = torch.empty((L, H, 5), dtype=torch.float64, device=rows.device)
    scores = torch.empty((L, H, 3), dtype=torch.float64, device=rows.device)
    ws = torch.empty((max(B.slkv_score_heads_workspace_bytes(L, H, T, n), 16),), dtype=torch.uint8, device=rows.device)
    B.slkv_score_heads(rows, needle_start, needle_len, topk, acc, scores, ws, stream, first)
    return acc, scores


def score_heads_ex(rows, needle_start, needle_len, topk, aggregation=B.SLKV_AGG_MICRO, components=(True, True, True),
                   acc=None, stream=None):
    """As score_heads through slkv_score_heads_ex: acc is [L,H,8]."""
    L, H, T, n = rows.shape
    first = acc is None
    if first:
        acc = torch.empty((L, H, 8), dtype=torch.float64, device=rows.device)
    scores = torch.empty((L, H, 3), dtype=torch.float64, device=rows.device)
    ws = torch.empty((max(B.slkv_score_heads_workspace_bytes(L, H, T, n), 16),), dtype=torch.uint8, device=rows.device)
    B.slkv_score_heads_ex(rows, needle_start, needle_len, topk, acc, scores, ws, aggregation, components, stream, first)
    return acc, scores


def score_heads_qk(q, k, needle_start, needle_len, topk, acc=None, stream=None):
    """q [L,Hq,T,d], k [L,Hkv,n,d] bf16 device tensors.  Returns (acc [L,Hq,5], scores [L,Hq,3]) float64 device tensors."""
    L, Hq, T, d = q.shape
    n = k.shape[2]
    first = acc is None
    if first:
        acc = torch.empty((L, Hq, 5), dtype=torch.float64, device=q.device)
    scores = torch.empty((L, Hq, 3), dtype=torch.float64, device=q.device)
    ws = torch.empty((B.slkv_score_heads_qk_workspace_bytes(L, Hq, T, n),), dtype=torch.uint8, device=q.device)
    B.slkv_score_heads_qk(q, k, needle_start, needle_len, topk, acc, scores, ws, stream, first)
    return acc, scores


class Cache:
    """One layer's cache for decoding: packed K and V rows in a room per segment (sequence b, KV head h: b * Hkv + h), of which the first
    lengths[s] are in use.

    `offsets` [B * Hkv + 1]: the rooms.  The arrays are allocated unless they are given (k, v [rows, d], "bf16_kv4": [rows, d / 2] uint8 and
    k_scale, v_scale [rows, d / 32] uint8; lengths [B * Hkv], pos [rows] int32; weight [rows] fp32); given keys without lengths fill their
    rooms.  positions, weights = False: a cache without these arrays.  Calls run on `stream`, or the current stream of the cache's device; the caller orders those that
    read or write the same arrays on several streams (attend() writes the weights where it has to add to them), and the object outlives the graphs that
    captured them.  attend() has scratch of its own on every stream and in every graph that torch captures."""

    def __init__(self, dtype, B_, Hq, Hkv, d, offsets, k=None, v=None, k_scale=None, v_scale=None, lengths=None, pos=None, weight=None,
                 device="cuda", positions=True, weights=True):
        code, self.query_dtype, self.row_dtype = CACHE_DTYPES[dtype]
        self.dtype, self.B, self.Hq, self.Hkv, self.d = dtype, B_, Hq, Hkv, d
        self.layout = B.CacheLayout(code, B_, Hq, Hkv, d, offsets)
        offsets = self.layout.offsets
        rows, S = int(offsets[-1]), B_ * Hkv
        four = dtype == "bf16_kv4"
        if (k is None) != (v is None) or (k is not None and four and (k_scale is None or v_scale is None)):
            raise ValueError("keys, values and their scales are given together")
        if k is not None:
            device = k.device
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._here = contextlib.nullcontext()
        if lengths is None:
            lengths = torch.zeros((S,), dtype=torch.int32, device=self.device) if k is None else torch.from_numpy(np.diff(offsets).astype(np.int32)).to(self.device)
        width = d // 2 if four else d

        def array(t, shape, tdt, name, make):
            if t is None:
                return make(shape, dtype=tdt, device=self.device)
            return self._tensor(t, shape, tdt, name)

        self.k = array(k, (rows, width), self.row_dtype, "k", torch.empty)
        self.v = array(v, (rows, width), self.row_dtype, "v", torch.empty)
        self.k_scale = array(k_scale, (rows, d // 32), torch.uint8, "k_scale", torch.empty) if four else None
        self.v_scale = array(v_scale, (rows, d // 32), torch.uint8, "v_scale", torch.empty) if four else None
        self.lengths = self._tensor(lengths, (S,), torch.int32, "lengths")
        self.pos = array(pos, (rows,), torch.int32, "pos", torch.zeros) if positions or pos is not None else None
        self.weight = array(weight, (rows,), torch.float32, "weight", torch.zeros) if weights or weight is not None else None
        self.rows_in_all = rows
        self._arrays = B.CacheTensors(self.k, self.v, self.k_scale, self.v_scale, self.lengths, self.pos, self.weight)
        self._workspaces, self._attend_like = {}, {}

    def _tensor(self, t, shape, tdt, name, contiguous=True):
        if t.dtype != tdt or t.shape != shape:
            raise ValueError("%s: %s of shape %s wanted, got %s of shape %s" % (name, tdt, shape, t.dtype, tuple(t.shape)))
        if t.device != self.device:
            raise ValueError("%s is on %s, the cache on %s" % (name, t.device, self.device))
        if contiguous and not t.is_contiguous():
            raise ValueError("%s is not contiguous" % name)
        return t

    def _on(self, stream):
        """The call's stream as the current one, so that what it allocates belongs to it; without one, the cache's device, where it is not current."""
        if stream is not None:
            if stream.device != self.device:
                raise ValueError("stream is of %s, the cache on %s" % (stream.device, self.device))
            return torch.cuda.stream(stream)
        return self._here if torch.cuda.current_device() == self.device.index else torch.cuda.device(self.device)

    def _attend_buffers(self, T, weights, stream):
        """A workspace for a call on the stream of this handle, and a tensor in the shape of its lse.  Calls that follow each other on a stream share one, which grows with
        the largest of them; a captured call has its own, which stays with its graph: the graph may be replayed anywhere.  (0.2 to 0.4 us of the host; a tensor for every call 0.9.)"""
        like = self._attend_like.get((T, weights))
        if like is None:
            like = B.slkv_attend_workspace_bytes(self.layout, T, weights), torch.empty((self.B, self.Hq, T), dtype=torch.float32, device=self.device)
            self._attend_like[T, weights] = like
        ws = None if torch.cuda.is_current_stream_capturing() else self._workspaces.get(stream, _NOTHING)
        if ws is None:
            ws = torch.empty((like[0],), dtype=torch.uint8, device=self.device)
        elif ws.nbytes < like[0]:
            ws = self._workspaces[stream] = torch.empty((like[0],), dtype=torch.uint8, device=self.device)
        return ws, like[1]

    def fill(self, k_rows, v_rows, src_offsets, pos=None, stream=None):
        """The rows that a prefill kept (LayerCall's k_out, v_out, offsets, kept_idx) become the cache."""
        rows = int(src_offsets[-1])
        for t, name in ((k_rows, "k_rows"), (v_rows, "v_rows")):
            if t.dim() != 2 or t.shape[0] < rows:
                raise ValueError("%s: at least %d rows wanted, got shape %s" % (name, rows, tuple(t.shape)))
            self._tensor(t, (t.shape[0], self.d), self.query_dtype, name)
        if pos is not None:
            self._tensor(pos, (max(pos.shape[0], rows),), torch.int32, "pos")
        with self._on(stream):
            B.slkv_fill_cache(self.layout, self._arrays, src_offsets, k_rows, v_rows, pos)

    def append(self, k, v, pos=None, at=None, stream=None):
        """k, v [B, Hkv, T, d] (strides of multiples of 16 bytes, 0 among them, rows contiguous), pos [B, T]: the next T tokens enter behind the rows in use, or behind the first at[s]
        of them (drafted tokens that were not accepted are overwritten this way)."""
        shape = (self.B, self.Hkv, k.shape[2] if k.dim() == 4 else 0, self.d)
        for t, name in ((k, "k"), (v, "v")):
            if self._tensor(t, shape, self.query_dtype, name, contiguous=False).stride(3) != 1:
                raise ValueError("%s: rows are not contiguous" % name)
        if pos is not None:
            self._tensor(pos, (self.B, shape[2]), torch.int32, "pos")
        if at is not None:
            self._tensor(at, (self.B * self.Hkv,), torch.int32, "at")
        with self._on(stream):
            B.slkv_append_cache(self.layout, self._arrays, k, v, pos, at)

    def attend(self, q, out=None, lse=None, weight=None, stream=None):
        """q [B, Hq, T, d]: the queries of the T latest tokens, whose rows are in the cache.  Returns (out [B, Hq, T, d], lse [B, Hq, T] fp32).
        weight: where the cache's weights plus this call's go; None: the cache's own array, if it has one; False: nowhere."""
        if q.dim() != 4:
            raise ValueError("q: four dimensions wanted, got shape %s" % (tuple(q.shape),))
        T = q.shape[2]
        shape = (self.B, self.Hq, T, self.d)
        self._tensor(q, shape, self.query_dtype, "q")
        if weight is None:
            weight = self.weight
        elif weight is False:
            weight = None
        else:
            self._tensor(weight, (self.rows_in_all,), torch.float32, "weight")
        with self._on(stream):
            handle = B._stream(None)
            ws, lse_like = self._attend_buffers(T, weight is not None, handle)
            out = torch.empty_like(q) if out is None else self._tensor(out, shape, self.query_dtype, "out")
            lse = torch.empty_like(lse_like) if lse is None else self._tensor(lse, shape[:3], torch.float32, "lse")
            B.slkv_attend_cache(self.layout, self._arrays, q, out, ws, lse, weight, handle)
        return out, lse

    def rows(self, out_offsets, stream=None):
        """Every segment's latest out_offsets[s + 1] - out_offsets[s] rows as values: (k, v [rows, d], pos [rows] or None).  Output rows that have no
        row in the cache hold nothing in particular."""
        rows = int(out_offsets[-1])
        with self._on(stream):
            k, v = self.k.new_empty((2, rows, self.d), dtype=self.query_dtype).unbind(0)
            pos = self.pos.new_empty((rows,)) if self.pos is not None else None
            B.slkv_cache_rows(self.layout, self._arrays, out_offsets, k, v, pos)
        return k, v, pos

    def evict(self, budgets, keep_last, out, kept_idx=None, stream=None):
        """The rows that stay within the capacities `budgets` [Hkv], by accumulated weight and the latest keep_last always, go to the Cache `out`.
        kept_idx [rows of out] int32, may be None: their numbers inside their segments."""
        if kept_idx is not None:
            self._tensor(kept_idx, (out.rows_in_all,), torch.int32, "kept_idx")
        if out.device != self.device:
            raise ValueError("out is on %s, the cache on %s" % (out.device, self.device))
        with self._on(stream):
            B.slkv_evict_cache(self.layout, self._arrays, out.layout, out._arrays, keep_last, budgets, kept_idx)
