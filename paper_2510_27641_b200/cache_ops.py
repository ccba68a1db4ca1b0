"""Python binding of the cache's operators: rows held in 4 bits (``specattn_kv4_*``) and eviction by accumulated
attention weight (``specattn_accumulate``, ``specattn_evict``, ``specattn_move_rows``); see
``include/specattn.h`` for what each computes.

Argument marshalling only.  Every call runs on the device of its tensors (all of them CUDA tensors of one
device), on ``stream`` or that device's current stream.  A ``status`` that is not given is not reported."""
from __future__ import annotations

import ctypes as C
from typing import Sequence

import torch

from . import (AccumulateArgs, EvictArgs, Kv4RowsArgs, Kv4VerifyArgs, MoveArgs, SpecAttnError, _Calls, _raw_device, _stream_ptr, lib)

__all__ = ["kv4_cache", "kv4_append", "kv4_read", "kv4_verify", "kv4_verify_workspace_bytes", "accumulate_attention", "evict",
           "move_rows"]

_DTYPES = {torch.bfloat16: 0, torch.float16: 1}
_I32, _F32 = torch.int32, torch.float32
_calls = _Calls()


def _device(first: torch.Tensor, *others: torch.Tensor | None) -> int:
    """The index of the device that all tensors of a call are on."""
    index = first.get_device()
    if index < 0:
        raise ValueError("CUDA tensors expected")
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError("all tensors of a call have to be on one device")
    return index


def _call(name: str, ref, index: int, stream):
    """The entry point, on the device that the tensors are on."""
    entry = getattr(lib(), name)
    if index == _raw_device():
        rc = entry(ref, _stream_ptr(stream))
    else:
        with torch.cuda.device(index):
            rc = entry(ref, _stream_ptr(stream))
    if rc != 0:
        raise SpecAttnError(rc, name)


def _strides(t: torch.Tensor, first: int, last: int):
    """Strides of the dimensions first ... last - 1; of one that has a single entry it says nothing."""
    return [s if n > 1 else 0 for s, n in zip(t.stride()[first:last], t.shape[first:last])]


def _behind(stream, made, device):
    """What was allocated on the current stream is used on the caller's: whoever had the memory before is done by then, and
    nobody gets it earlier than that stream is done."""
    if made and stream != torch.cuda.current_stream(device):
        stream.wait_stream(torch.cuda.current_stream(device))
        for t in made:
            t.record_stream(stream)


def _apart(*tensors):
    """Tensors that a call writes: no two elements in one place."""
    for t in tensors:
        assert t.numel() == 0 or all(s > 0 for s, n in zip(t.stride(), t.shape) if n > 1), "a tensor that is written may not be expanded"


def _ints(t: torch.Tensor | None, n: int, what: str):
    """A vector of n 32-bit integers (or None), by address."""
    if t is None:
        return None
    assert t.dtype is _I32 and t.numel() == n and t.is_contiguous(), f"{what}: {n} contiguous int32 values expected"
    return t.data_ptr()


def kv4_cache(n_pages: int, page_size: int, n_kv_heads: int, *, dtype: torch.dtype = torch.bfloat16, device=None):
    """An empty paged 4-bit cache of one layer: (codes uint8 [n_pages, 2, page_size, n_kv_heads, 64], params ``dtype``
    [n_pages, 2, page_size, n_kv_heads, 2]), the slots of a page and head side by side in memory."""
    dev = torch.device("cuda") if device is None else device
    shape = (n_pages, 2, n_kv_heads, page_size)
    assert dtype in _DTYPES
    return (torch.zeros(*shape, 64, dtype=torch.uint8, device=dev).transpose(2, 3),
            torch.zeros(*shape, 2, dtype=dtype, device=dev).transpose(2, 3))


def _cache_key(codes, params, block_table, pages_per_seq):
    """What the fixed part of a cache's description depends on."""
    key = codes.shape, codes.stride(), codes.dtype, params.shape, params.stride(), params.dtype
    return key + ((pages_per_seq,) if block_table is None else (block_table.shape, block_table.stride(), block_table.dtype))


def _fill_cache(c, codes, params, block_table, pages_per_seq, batch):
    n_pages, two, page, heads, row = codes.shape
    assert two == 2 and row == 64 and codes.dtype is torch.uint8 and codes.stride(4) == 1, \
        "codes: uint8 [n_pages, 2, page_size, n_kv_heads, 64] expected"
    assert params.dtype in _DTYPES and params.shape == (n_pages, 2, page, heads, 2) and params.stride(4) == 1, \
        "params: bf16 or fp16 [n_pages, 2, page_size, n_kv_heads, 2] expected"
    c.n_pages, c.page_size, c.dtype = n_pages, page, _DTYPES[params.dtype]
    c.stride_page, c.stride_kv, c.stride_slot, c.stride_head = _strides(codes, 0, 4)
    c.pstride_page, c.pstride_kv, c.pstride_slot, c.pstride_head = _strides(params, 0, 4)
    c.block_table_stride = _pages_per_seq(block_table, pages_per_seq, batch)


def _pages_per_seq(table, pages_per_seq, batch) -> int:
    """Pages that may be looked up for a sequence: with a block table, its entries from one sequence to the next."""
    if table is None:
        assert pages_per_seq is not None, "without a block table: pages_per_seq"
        return int(pages_per_seq)
    assert table.dtype is _I32 and table.dim() == 2 and table.shape[0] == batch and table.is_contiguous(), \
        "block_table: contiguous int32 [batch, pages] expected"
    return table.shape[1]


def _rows(name, k, v, codes, params, start, n, block_table, pages_per_seq, status, stream):
    index = _device(k, v, codes, params, start, n, block_table, status)
    key = (name, k.shape, k.stride(), k.dtype, v.shape, v.stride(), v.dtype) + _cache_key(codes, params, block_table, pages_per_seq)

    def make():
        b, t, h, d = k.shape
        assert v.shape == k.shape and h == codes.shape[3] and k.stride(3) == 1 and v.stride(3) == 1
        a = Kv4RowsArgs()
        a.struct_size = C.sizeof(Kv4RowsArgs)
        a.batch, a.n_tokens, a.n_kv_heads, a.head_dim = b, t, h, d
        _fill_cache(a.cache, codes, params, block_table, pages_per_seq, b)
        assert k.dtype is params.dtype and v.dtype is params.dtype, "k, v: of the type of params"
        _apart(*((codes, params) if name.endswith("append") else (k, v)))
        a.k_stride_batch, a.k_stride_token, a.k_stride_head = _strides(k, 0, 3)
        a.v_stride_batch, a.v_stride_token, a.v_stride_head = _strides(v, 0, 3)
        return a, a.cache, C.byref(a), b

    a, c, ref, b = _calls.get(key, make)
    c.codes, c.params = codes.data_ptr(), params.data_ptr()
    if block_table is not None:
        assert block_table.is_contiguous()
        c.block_table = block_table.data_ptr()
    a.k, a.v = k.data_ptr(), v.data_ptr()
    a.start, a.n_new, a.status = _ints(start, b, "start"), _ints(n, b, "n"), _ints(status, b, "status")
    _call(name, ref, index, stream)


def kv4_append(k: torch.Tensor, v: torch.Tensor, codes: torch.Tensor, params: torch.Tensor, start: torch.Tensor, *,
               n_new: torch.Tensor | None = None, block_table: torch.Tensor | None = None, pages_per_seq: int | None = None,
               status: torch.Tensor | None = None, stream=None):
    """specattn_kv4_append: rows of k, v [B, T, n_kv_heads, 128] (bf16 or fp16 as ``params``, unit innermost stride) go
    to positions start[b] + t, t < n_new[b] (None: all T).  Returns ``status`` ([B] int32, written where given)."""
    _rows("specattn_kv4_append", k, v, codes, params, start, n_new, block_table, pages_per_seq, status, stream)
    return status


def kv4_read(codes: torch.Tensor, params: torch.Tensor, start: torch.Tensor, *, n: torch.Tensor | None = None,
             n_tokens: int | None = None, k: torch.Tensor | None = None, v: torch.Tensor | None = None,
             block_table: torch.Tensor | None = None, pages_per_seq: int | None = None, status: torch.Tensor | None = None,
             stream=None):
    """specattn_kv4_read: rows start[b] + t, t < n[b] (None: all), as values of the type of ``params``.  Returns (k, v
    [B, T, n_kv_heads, 128], status).  k and v are made (T = n_tokens, rows that are not read zero) where not given."""
    if k is None or v is None:
        shape = (start.shape[0], int(n_tokens), codes.shape[3], 128) if k is None and v is None else (v if k is None else k).shape
        made = [torch.zeros(shape, dtype=params.dtype, device=params.device) for x in (k, v) if x is None]
        if stream is not None:
            _behind(stream, made, params.device)   # (filled on the current stream, too)
        v = made.pop() if v is None else v
        k = made.pop() if k is None else k
    _rows("specattn_kv4_read", k, v, codes, params, start, n, block_table, pages_per_seq, status, stream)
    return k, v, status


def kv4_verify_workspace_bytes(q: torch.Tensor, codes: torch.Tensor) -> int:
    """Bytes of workspace that kv4_verify wants for queries and a cache of these shapes."""
    a = Kv4VerifyArgs()
    a.struct_size = C.sizeof(Kv4VerifyArgs)
    a.batch, a.n_q, a.n_q_heads, a.head_dim = q.shape
    a.n_kv_heads, a.n_groups, a.cache.n_pages, a.cache.page_size = codes.shape[3], 1, codes.shape[0], codes.shape[2]
    with torch.cuda.device(_device(q)):
        n = int(lib().specattn_kv4_verify_workspace_bytes(C.byref(a)))
    if n == 0:
        raise SpecAttnError(-6, "specattn_kv4_verify_workspace_bytes")
    return n


def kv4_verify(q: torch.Tensor, codes: torch.Tensor, params: torch.Tensor, kv_len: torch.Tensor, *,
               block_table: torch.Tensor | None = None, pages_per_seq: int | None = None, idx: torch.Tensor | None = None,
               counts: torch.Tensor | None = None, n_groups: int = 1, dense: bool = False, sm_scale: float = 0.0,
               tail_len: int = 0, out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
               status: torch.Tensor | None = None, workspace: torch.Tensor | None = None, flags: int = 0, stream=None):
    """specattn_kv4_verify for one target layer: attention of q [B, T, H_q, 128] (of the type of ``params``) over the listed
    positions (idx [B, n_groups, stride], counts [B, n_groups]; all positions where ``dense``) and the tail of a 4-bit
    cache.  Returns (out [B, T, H_q, 128] of q's type, or float32 where ``out`` is, lse f32 [B, T, H_q], status).
    A step over such a cache is select_topp and one call per target layer; VerifyStep and verify_step_host take 16-bit pools."""
    index = _device(q, codes, params, kv_len, block_table, None if dense else idx, None if dense else counts, out, lse, status, workspace)
    assert dense or (idx is not None and counts is not None), "idx and counts expected, or dense"
    shape = q.shape
    # (out, lse and the workspace are made here or looked at by every call)
    key = (shape, q.dtype, n_groups, dense, sm_scale, tail_len, flags, out is not None and out.dtype is _F32, index,
           None if dense else idx.shape) + _cache_key(codes, params, block_table, pages_per_seq)

    def make():
        b, t, hq, d = shape
        a = Kv4VerifyArgs()
        a.struct_size = C.sizeof(Kv4VerifyArgs)
        a.batch, a.n_q, a.n_q_heads, a.n_kv_heads, a.head_dim = b, t, hq, codes.shape[3], d
        a.n_groups, a.dense, a.out_f32 = n_groups, int(bool(dense)), int(out is not None and out.dtype is _F32)
        _fill_cache(a.cache, codes, params, block_table, pages_per_seq, b)
        assert q.dtype is params.dtype, "q: of the type of params"
        if not dense:
            assert idx.dim() == 3 and idx.shape[0] == b and idx.shape[1] == n_groups, "idx: [B, n_groups, stride] expected"
            a.idx_stride = idx.shape[2]
        a.sm_scale, a.tail_len, a.flags = float(sm_scale), int(tail_len), int(flags)
        return a, a.cache, C.byref(a), kv4_verify_workspace_bytes(q, codes) if b > 0 else 256, (b, t, hq)

    a, c, ref, need, rows = _calls.get(key, make)
    assert q.is_contiguous()
    made = []
    if out is None:
        out = torch.empty_like(q)
        made.append(out)
    else:
        assert (out.dtype is _F32 or out.dtype is q.dtype) and out.shape == shape and out.is_contiguous(), \
            "out: contiguous, of q's shape, of q's type or float32"
    if lse is None:
        lse = q.new_empty(rows, dtype=_F32)
        made.append(lse)
    else:
        assert lse.dtype is _F32 and lse.shape == rows and lse.is_contiguous()
    if workspace is None:
        workspace = q.new_empty(need // 2)   # (in the queries' 16-bit type)
        made.append(workspace)
        a.workspace_bytes = need
    else:
        assert workspace.is_contiguous()
        a.workspace_bytes = workspace.numel() * workspace.element_size()
    c.codes, c.params = codes.data_ptr(), params.data_ptr()
    if block_table is not None:
        assert block_table.is_contiguous()
        c.block_table = block_table.data_ptr()
    a.q, a.kv_len = q.data_ptr(), _ints(kv_len, rows[0], "kv_len")
    if not dense:
        assert idx.dtype is _I32 and idx.is_contiguous()
        a.idx, a.counts = idx.data_ptr(), _ints(counts, rows[0] * n_groups, "counts")
    a.out, a.lse, a.workspace = out.data_ptr(), lse.data_ptr(), workspace.data_ptr()
    a.status = _ints(status, rows[0], "status")
    if stream is not None:
        _behind(stream, made, index)
    _call("specattn_kv4_verify", ref, index, stream)
    return out, lse, status


def accumulate_attention(draft_probs: Sequence[torch.Tensor | None], kv_len: torch.Tensor, scores: torch.Tensor | None = None, *,
                         n_groups: int = 1, head_group: Sequence[int] | None = None, decay: float = 1.0,
                         out: torch.Tensor | None = None, row_status: torch.Tensor | None = None, stream=None):
    """specattn_accumulate: out = decay * scores + the attention that each position got in ``draft_probs`` (per draft
    layer a float32 tensor [B, H_d, gamma, L_stride], or None to leave the layer's entries of out alone).  scores, out: float32
    [n_layers, B, n_groups, L]; out None: in place; scores None: zeros.  Returns (out, row_status).

    Column i counts for slot i.  After an eviction slots are no longer tokens in order: the maps of a draft that keeps its whole
    cache are first gathered by ``positions``, each head's by those of the group that it feeds."""
    n = len(draft_probs)
    probs = next((t for t in draft_probs if t is not None), None)
    assert probs is not None, "draft_probs: a layer's at least"
    if out is None:
        assert scores is not None, "scores or out expected"
        out = scores
    index = _device(probs, kv_len, scores, out, row_status, *draft_probs)
    shape, out_shape = probs.shape, out.shape
    key = (n, shape, out_shape, n_groups, None if head_group is None else tuple(head_group), decay)

    def make():
        b, heads, gamma, width = shape
        assert out_shape == (n, b, n_groups, out_shape[3])
        a = AccumulateArgs()
        a.struct_size = C.sizeof(AccumulateArgs)
        a.n_layers, a.batch, a.n_draft_heads, a.gamma, a.n_groups = n, b, heads, gamma, n_groups
        a.L_stride, a.score_stride, a.decay = width, out_shape[3], float(decay)
        ptrs = (C.c_void_p * n)()
        a.draft_probs = ptrs
        groups = None
        if head_group is not None:
            assert len(head_group) == heads
            groups = (C.c_int32 * heads)(*[int(x) for x in head_group])
            a.head_group = groups
        return a, C.byref(a), ptrs, groups, b

    a, ref, ptrs, _, b = _calls.get(key, make)
    for u, t in enumerate(draft_probs):
        assert t is None or (t.dtype is _F32 and t.is_contiguous() and (t is probs or t.shape == shape))
        ptrs[u] = None if t is None else t.data_ptr()
    assert out.dtype is _F32 and out.is_contiguous()
    assert scores is None or scores is out or (scores.dtype is _F32 and scores.is_contiguous() and scores.shape == out_shape)
    a.kv_len = _ints(kv_len, b, "kv_len")
    a.scores_in, a.scores_out = None if scores is None else scores.data_ptr(), out.data_ptr()
    a.row_status = _ints(row_status, n * b * n_groups, "row_status")
    _call("specattn_accumulate", ref, index, stream)
    return out, row_status


def _like_scores(t, scores, dtype, what):
    """A tensor of the scores' shape (or None), by address."""
    if t is None:
        return None
    assert t.dtype is dtype and t.shape == scores.shape and t.is_contiguous(), f"{what}: contiguous {dtype} of the scores' shape expected"
    return t.data_ptr()


def evict(scores: torch.Tensor, kv_len: torch.Tensor, budget: int, *, n_sink: int = 0, n_recent: int = 0,
          positions: torch.Tensor | None = None, seq_len: torch.Tensor | None = None, src: torch.Tensor | None = None,
          dst: torch.Tensor | None = None, n_moves: torch.Tensor | None = None, new_len: torch.Tensor | None = None,
          scores_out: torch.Tensor | None = None, positions_out: torch.Tensor | None = None, stream=None):
    """specattn_evict: which ``budget`` slots of every sequence stay, by scores [n_layers, B, G, L] (float32), and the moves
    that close the gaps.  Returns (src, dst [n_layers, B, G, moves at most], n_moves [n_layers, B, G], new_len [B]),
    int32.  ``scores_out`` / ``positions_out`` (may be ``scores`` / ``positions``) receive scores and positions as they lie
    after the moves."""
    index = _device(scores, kv_len, positions, seq_len, src, dst, n_moves, new_len, scores_out, positions_out)
    stride = None if src is None else src.shape[3]
    key = (scores.shape, scores.dtype, stride, budget, n_sink, n_recent)

    def make():
        n, b, g, width = scores.shape
        assert scores.dtype is _F32
        a = EvictArgs()
        a.struct_size = C.sizeof(EvictArgs)
        a.n_layers, a.batch, a.n_groups, a.L = n, b, g, width
        a.budget, a.n_sink, a.n_recent = int(budget), int(n_sink), int(n_recent)
        a.move_stride = max(0, min(a.budget, width - a.budget)) if stride is None else stride
        return a, C.byref(a), (n, b, g, a.move_stride), b

    a, ref, moves, b = _calls.get(key, make)
    assert scores.is_contiguous()
    made = []

    def new(shape):
        made.append(scores.new_empty(shape, dtype=_I32))
        return made[-1]

    if src is None:
        src = new(moves)
    if dst is None:
        dst = new(moves)
    assert src.dtype is _I32 and src.shape == moves and src.is_contiguous(), "src: contiguous int32 [n_layers, B, G, moves]"
    assert dst.dtype is _I32 and dst.shape == moves and dst.is_contiguous(), "dst: like src"
    if n_moves is None:
        n_moves = new(moves[:3])
    if new_len is None:
        new_len = new((b,))
    a.scores, a.kv_len = scores.data_ptr(), _ints(kv_len, b, "kv_len")
    a.src, a.dst = src.data_ptr(), dst.data_ptr()
    a.seq_len = None if seq_len is None else _ints(seq_len, b, "seq_len")
    a.n_moves = _ints(n_moves, moves[0] * b * moves[2], "n_moves")
    a.new_len = _ints(new_len, b, "new_len")
    a.positions = None if positions is None else _like_scores(positions, scores, _I32, "positions")
    a.positions_out = None if positions_out is None else _like_scores(positions_out, scores, _I32, "positions_out")
    a.scores_out = None if scores_out is None else _like_scores(scores_out, scores, _F32, "scores_out")
    if stream is not None:
        _behind(stream, made, index)
    _call("specattn_evict", ref, index, stream)
    return src, dst, n_moves, new_len


def move_rows(pools: Sequence[torch.Tensor], src: torch.Tensor, dst: torch.Tensor, n_moves: torch.Tensor, *,
              params: Sequence[torch.Tensor] | None = None, block_table: torch.Tensor | None = None,
              pages_per_seq: int | None = None, status: torch.Tensor | None = None, stream=None):
    """specattn_move_rows: the moves of one draft layer's lists (src, dst [B, G, stride], n_moves [B, G] as ``evict`` gives
    them), in place, in the pools [n_pages, 2, page_size, n_kv_heads, X] of the layers that follow it: all of one
    shape, type and strides, with ``params`` beside them where the cache is held in 4 bits.  Returns ``status``."""
    n = len(pools)
    if n == 0:
        if status is not None:
            with torch.cuda.stream(stream):
                status.zero_()
        return status
    assert params is None or len(params) == n
    index = _device(src, dst, n_moves, block_table, status, *pools, *(params or ()))
    pool, par = pools[0], None if params is None else params[0]
    shape, strides, par_strides = pool.shape, pool.stride(), None if par is None else par.stride()
    key = ("move", n, shape, strides, pool.dtype, src.shape, pages_per_seq, None if block_table is None else block_table.shape,
           None if par is None else (par.shape, par_strides, par.dtype))

    def make():
        n_pages, two, page, heads, width = pool.shape
        b, g, stride = src.shape
        assert two == 2 and pool.stride(4) == 1
        _apart(pool, *(() if par is None else (par,)))
        a = MoveArgs()
        a.struct_size = C.sizeof(MoveArgs)
        a.n_pools, a.batch, a.n_groups, a.n_kv_heads, a.page_size, a.n_pages = n, b, g, heads, page, n_pages
        size = pool.element_size()
        a.row_bytes = width * size
        a.stride_page, a.stride_kv, a.stride_slot, a.stride_head = [x * size for x in _strides(pool, 0, 4)]
        if par is not None:
            assert par.shape[:4] == pool.shape[:4] and par.stride(4) == 1
            size = par.element_size()
            a.param_bytes = par.shape[4] * size
            a.pstride_page, a.pstride_kv, a.pstride_slot, a.pstride_head = [x * size for x in _strides(par, 0, 4)]
        a.block_table_stride, a.move_stride = _pages_per_seq(block_table, pages_per_seq, b), stride
        ptrs, par_ptrs = (C.c_void_p * n)(), None if par is None else (C.c_void_p * n)()
        a.pools, a.params = ptrs, par_ptrs
        return a, C.byref(a), b, b * g, ptrs, par_ptrs

    a, ref, b, lists, ptrs, par_ptrs = _calls.get(key, make)
    for i, t in enumerate(pools):
        assert t is pool or (t.dtype is pool.dtype and t.shape == shape and t.stride() == strides), "pools of one shape, type and strides expected"
        ptrs[i] = t.data_ptr()
    if par is not None:
        for i, t in enumerate(params):
            assert t is par or (t.dtype is par.dtype and t.shape == par.shape and t.stride() == par_strides), "params of one shape, type and strides expected"
            par_ptrs[i] = t.data_ptr()
    assert src.dtype is _I32 and src.is_contiguous()
    assert dst.dtype is _I32 and dst.is_contiguous() and dst.shape == src.shape
    if block_table is not None:
        assert block_table.dtype is _I32 and block_table.is_contiguous()
        a.block_table = block_table.data_ptr()
    a.src, a.dst, a.n_moves = src.data_ptr(), dst.data_ptr(), _ints(n_moves, lists, "n_moves")
    a.status = _ints(status, b, "status")
    _call("specattn_move_rows", ref, index, stream)
    return status
