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
    entry = getattr(lib(), "specattn_" + name)
    if index == _raw_device():
        rc = entry(ref, _stream_ptr(stream))
    else:
        with torch.cuda.device(index):
            rc = entry(ref, _stream_ptr(stream))
    if rc != 0:
        raise SpecAttnError(rc, "specattn_" + name)


def _strides(t: torch.Tensor, first: int, last: int):
    """Strides of the dimensions first ... last - 1; of one that has a single entry it says nothing."""
    return [s if n > 1 else 0 for s, n in zip(t.stride()[first:last], t.shape[first:last])]


def _ints(t: torch.Tensor | None, n: int, what: str):
    """A vector of n 32-bit integers (or None), by address."""
    if t is None:
        return None
    assert t.dtype is torch.int32 and t.is_contiguous() and t.numel() == n, f"{what}: {n} contiguous int32 values expected"
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
    return (codes.shape, codes.stride(), params.shape, params.stride(), params.dtype,
            None if block_table is None else (block_table.shape, block_table.stride()), pages_per_seq)


def _fill_cache(c, codes, params, block_table, pages_per_seq):
    """What does not change from call to call of one shape."""
    n_pages, two, page, heads, row = codes.shape
    assert two == 2 and row == 64 and codes.dtype is torch.uint8 and codes.stride(4) == 1, \
        "codes: uint8 [n_pages, 2, page_size, n_kv_heads, 64] expected"
    assert params.dtype in _DTYPES and params.shape == (n_pages, 2, page, heads, 2) and params.stride(4) == 1, \
        "params: bf16 or fp16 [n_pages, 2, page_size, n_kv_heads, 2] expected"
    c.n_pages, c.page_size, c.dtype = n_pages, page, _DTYPES[params.dtype]
    c.stride_page, c.stride_kv, c.stride_slot, c.stride_head = _strides(codes, 0, 4)
    c.pstride_page, c.pstride_kv, c.pstride_slot, c.pstride_head = _strides(params, 0, 4)
    if block_table is not None:
        assert block_table.dim() == 2 and (block_table.shape[1] <= 1 or block_table.stride(1) == 1)
        c.block_table_stride = _table_stride(block_table)
    else:
        assert pages_per_seq is not None, "without a block table: pages_per_seq"
        c.block_table_stride = int(pages_per_seq)


def _table_stride(table: torch.Tensor) -> int:
    """Entries from one sequence to the next, which the library takes for the number of pages that it may look up."""
    assert table.shape[0] <= 1 or table.stride(0) == table.shape[1], "block_table: contiguous [batch, pages] expected"
    return table.shape[1]


def _set_cache(c, codes, params, block_table):
    assert codes.dtype is torch.uint8
    c.codes, c.params = codes.data_ptr(), params.data_ptr()
    if block_table is not None:
        assert block_table.dtype is torch.int32
        c.block_table = block_table.data_ptr()


def _rows(name, k, v, codes, params, start, n, block_table, pages_per_seq, status, stream):
    index = _device(k, v, codes, params, start, n, block_table, status)
    key = ("rows", k.shape, k.stride(), v.shape, v.stride(), _cache_key(codes, params, block_table, pages_per_seq))

    def make():
        b, t, h, d = k.shape
        assert v.shape == k.shape and h == codes.shape[3] and k.stride(3) == 1 and v.stride(3) == 1
        assert block_table is None or block_table.shape[0] == b
        a = Kv4RowsArgs()
        a.struct_size = C.sizeof(Kv4RowsArgs)
        a.batch, a.n_tokens, a.n_kv_heads, a.head_dim = b, t, h, d
        _fill_cache(a.cache, codes, params, block_table, pages_per_seq)
        a.k_stride_batch, a.k_stride_token, a.k_stride_head = _strides(k, 0, 3)
        a.v_stride_batch, a.v_stride_token, a.v_stride_head = _strides(v, 0, 3)
        return a, C.byref(a)

    a, ref = _calls.get(key, make)
    assert k.dtype is params.dtype and v.dtype is params.dtype, "k, v: of the type of params"
    _set_cache(a.cache, codes, params, block_table)
    a.k, a.v = k.data_ptr(), v.data_ptr()
    a.start, a.n_new, a.status = _ints(start, a.batch, "start"), _ints(n, a.batch, "n"), _ints(status, a.batch, "status")
    _call(name, ref, index, stream)


def kv4_append(k: torch.Tensor, v: torch.Tensor, codes: torch.Tensor, params: torch.Tensor, start: torch.Tensor, *,
               n_new: torch.Tensor | None = None, block_table: torch.Tensor | None = None, pages_per_seq: int | None = None,
               status: torch.Tensor | None = None, stream=None):
    """specattn_kv4_append: rows of k, v [B, T, n_kv_heads, 128] (bf16 or fp16 as ``params``, unit innermost stride) go
    to positions start[b] + t, t < n_new[b] (None: all T).  Returns ``status`` ([B] int32, written where given)."""
    _rows("kv4_append", k, v, codes, params, start, n_new, block_table, pages_per_seq, status, stream)
    return status


def kv4_read(codes: torch.Tensor, params: torch.Tensor, start: torch.Tensor, *, n: torch.Tensor | None = None,
             n_tokens: int | None = None, k: torch.Tensor | None = None, v: torch.Tensor | None = None,
             block_table: torch.Tensor | None = None, pages_per_seq: int | None = None, status: torch.Tensor | None = None,
             stream=None):
    """specattn_kv4_read: rows start[b] + t, t < n[b] (None: all), as values of the type of ``params``.  Returns (k, v
    [B, T, n_kv_heads, 128], status).  k and v are made (T = n_tokens, rows behind n[b] zero) where not given."""
    if k is None or v is None:
        shape = (start.shape[0], int(n_tokens), codes.shape[3], 128) if k is None and v is None else (v if k is None else k).shape
        new = torch.empty if n is None and status is None else torch.zeros
        made = [new(shape, dtype=params.dtype, device=params.device) for x in (k, v) if x is None]
        if stream is not None:   # made on the current stream, written on the caller's
            _hand_over(made, stream)
        v = made.pop() if v is None else v
        k = made.pop() if k is None else k
    _rows("kv4_read", k, v, codes, params, start, n, block_table, pages_per_seq, status, stream)
    return k, v, status


def _hand_over(made, stream):
    """Tensors that the current stream has filled, used on another one."""
    stream.wait_stream(torch.cuda.current_stream(made[0].device))
    for t in made:
        t.record_stream(stream)


def _make_verify(q, codes, params, kv_len, block_table, pages_per_seq, idx, n_groups, dense, sm_scale, tail_len, out_f32):
    b, t, hq, d = q.shape
    a = Kv4VerifyArgs()
    a.struct_size = C.sizeof(Kv4VerifyArgs)
    a.batch, a.n_q, a.n_q_heads, a.n_kv_heads, a.head_dim = b, t, hq, codes.shape[3], d
    a.n_groups, a.dense, a.out_f32 = n_groups, int(bool(dense)), int(out_f32)
    _fill_cache(a.cache, codes, params, block_table, pages_per_seq)
    assert block_table is None or block_table.shape[0] == b
    if not dense:
        assert idx.dim() == 3 and idx.shape[0] == b and idx.shape[1] == n_groups and idx.is_contiguous()
        a.idx_stride = idx.shape[2]
    a.sm_scale, a.tail_len = float(sm_scale), int(tail_len)
    return a, C.byref(a)


def kv4_verify_workspace_bytes(q: torch.Tensor, codes: torch.Tensor) -> int:
    """Bytes of workspace that kv4_verify wants for queries and a cache of these shapes."""
    a = Kv4VerifyArgs()
    a.struct_size = C.sizeof(Kv4VerifyArgs)
    a.batch, a.n_q, a.n_q_heads, a.head_dim = q.shape
    a.n_kv_heads, a.n_groups, a.cache.n_pages, a.cache.page_size = codes.shape[3], 1, codes.shape[0], codes.shape[2]
    with torch.cuda.device(_device(q)):
        n = int(lib().specattn_kv4_verify_workspace_bytes(C.byref(a)))
    if n == 0 and a.batch > 0:
        raise SpecAttnError(-6, "specattn_kv4_verify_workspace_bytes")
    return n


def kv4_verify(q: torch.Tensor, codes: torch.Tensor, params: torch.Tensor, kv_len: torch.Tensor, *,
               block_table: torch.Tensor | None = None, pages_per_seq: int | None = None, idx: torch.Tensor | None = None,
               counts: torch.Tensor | None = None, n_groups: int = 1, dense: bool = False, sm_scale: float = 0.0,
               tail_len: int = 0, out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
               status: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """specattn_kv4_verify for one target layer: attention of q [B, T, H_q, 128] (of the type of ``params``) over the listed
    positions (idx [B, n_groups, stride], counts [B, n_groups]; all positions where ``dense``) and the tail of a 4-bit
    cache.  Returns (out [B, T, H_q, 128] of q's type, or float32 where ``out`` is, lse f32 [B, T, H_q], status)."""
    shape = q.shape
    index = _device(q, codes, params, kv_len, block_table, idx, counts, out, lse, status, workspace)
    made = []
    if out is None:
        out = torch.empty(shape, dtype=q.dtype, device=q.device)
        made.append(out)
    if lse is None:
        lse = torch.empty(shape[:3], dtype=torch.float32, device=q.device)
        made.append(lse)
    dense = bool(dense)
    f32 = out.dtype is torch.float32
    key = ("verify", shape, _cache_key(codes, params, block_table, pages_per_seq), None if dense else (idx.shape, idx.stride()),
           n_groups, dense, sm_scale, tail_len, f32)
    a, ref = _calls.get(key, _make_verify, q, codes, params, kv_len, block_table, pages_per_seq, idx, n_groups, dense, sm_scale,
                        tail_len, f32)
    assert q.dtype is params.dtype and q.is_contiguous(), "q: contiguous, of the type of params"
    assert (f32 or out.dtype is q.dtype) and out.shape == shape and out.is_contiguous(), "out: contiguous, of q's type or float32"
    assert lse.dtype is torch.float32 and lse.shape == shape[:3] and lse.is_contiguous()
    if workspace is None:
        need = _calls.get(("workspace", shape, codes.shape[2:4], index), kv4_verify_workspace_bytes, q, codes)
        workspace = torch.empty((need,), dtype=torch.uint8, device=q.device)
        made.append(workspace)
    else:
        assert workspace.is_contiguous()
    _set_cache(a.cache, codes, params, block_table)
    a.q, a.kv_len = q.data_ptr(), _ints(kv_len, shape[0], "kv_len")
    if not dense:
        assert idx.dtype is torch.int32
        a.idx, a.counts = idx.data_ptr(), _ints(counts, shape[0] * n_groups, "counts")
    a.out, a.lse, a.status = out.data_ptr(), lse.data_ptr(), _ints(status, shape[0], "status")
    a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _call("kv4_verify", ref, index, stream)
    if stream is not None:
        for t in made:
            t.record_stream(stream)   # allocated here, used on the caller's stream
    return out, lse, status


def accumulate_attention(draft_probs: Sequence[torch.Tensor | None], kv_len: torch.Tensor, scores: torch.Tensor | None = None, *,
                         n_groups: int = 1, head_group: Sequence[int] | None = None, decay: float = 1.0,
                         out: torch.Tensor | None = None, row_status: torch.Tensor | None = None, stream=None):
    """specattn_accumulate: out = decay * scores + the attention that each position got in ``draft_probs`` (per draft
    layer a float32 tensor [B, H_d, gamma, L_stride], or None to leave the layer's scores alone).  scores, out: float32
    [n_layers, B, n_groups, L]; out None: in place; scores None: zeros.  Returns (out, row_status)."""
    n = len(draft_probs)
    probs = next(t for t in draft_probs if t is not None)
    if out is None:
        assert scores is not None, "scores or out expected"
        out = scores
    index = _device(probs, kv_len, scores, out, row_status, *draft_probs)
    b, heads, gamma, width = shape = probs.shape
    key = ("accumulate", n, shape, out.shape, n_groups, None if head_group is None else tuple(head_group), float(decay))

    def make():
        assert out.shape == (n, b, n_groups, out.shape[3])
        a = AccumulateArgs()
        a.struct_size = C.sizeof(AccumulateArgs)
        a.n_layers, a.batch, a.n_draft_heads, a.gamma, a.n_groups = n, b, heads, gamma, n_groups
        a.L_stride, a.score_stride, a.decay = width, out.shape[3], float(decay)
        ptrs = (C.c_void_p * n)()
        a.draft_probs = ptrs
        groups = None
        if head_group is not None:
            assert len(head_group) == heads
            groups = (C.c_int32 * heads)(*[int(x) for x in head_group])
            a.head_group = groups
        return a, C.byref(a), ptrs, groups

    a, ref, ptrs, _ = _calls.get(key, make)
    for u, t in enumerate(draft_probs):
        assert t is None or (t.dtype is torch.float32 and t.is_contiguous() and t.shape == shape)
        ptrs[u] = None if t is None else t.data_ptr()
    assert out.dtype is torch.float32 and out.is_contiguous()
    assert scores is None or (scores.dtype is torch.float32 and scores.is_contiguous() and scores.shape == out.shape)
    a.kv_len = _ints(kv_len, b, "kv_len")
    a.scores_in, a.scores_out = None if scores is None else scores.data_ptr(), out.data_ptr()
    a.row_status = _ints(row_status, n * b * n_groups, "row_status")
    _call("accumulate", ref, index, stream)
    return out, row_status


def evict(scores: torch.Tensor, kv_len: torch.Tensor, budget: int, *, n_sink: int = 0, n_recent: int = 0,
          positions: torch.Tensor | None = None, seq_len: torch.Tensor | None = None, src: torch.Tensor | None = None,
          dst: torch.Tensor | None = None, n_moves: torch.Tensor | None = None, new_len: torch.Tensor | None = None,
          scores_out: torch.Tensor | None = None, positions_out: torch.Tensor | None = None, stream=None):
    """specattn_evict: which ``budget`` slots of every sequence stay, by scores [n_layers, B, G, L] (float32), and the moves
    that close the gaps.  Returns (src, dst [n_layers, B, G, moves at most], n_moves [n_layers, B, G], new_len [B]),
    int32.  ``scores_out`` / ``positions_out`` (may be ``scores`` / ``positions``) receive scores and positions as they lie
    after the moves."""
    n, b, g, width = scores.shape
    index = _device(scores, kv_len, positions, seq_len, src, dst, n_moves, new_len, scores_out, positions_out)
    assert scores.dtype is torch.float32 and scores.is_contiguous()
    budget = int(budget)
    room = max(0, min(budget, width - budget))
    made = []

    def new(*shape):
        made.append(torch.empty(shape, dtype=torch.int32, device=scores.device))
        return made[-1]

    src = new(n, b, g, room) if src is None else src
    dst = new(n, b, g, room) if dst is None else dst
    n_moves = new(n, b, g) if n_moves is None else n_moves
    new_len = new(b) if new_len is None else new_len
    stride = src.shape[3]
    for t in (src, dst):
        assert t.dtype is torch.int32 and t.is_contiguous() and t.shape == (n, b, g, stride), "src, dst: int32 [n_layers, B, G, moves]"
    for t in (scores_out, positions, positions_out):
        assert t is None or (t.is_contiguous() and t.shape == scores.shape)
    assert scores_out is None or scores_out.dtype is torch.float32
    assert (positions is None or positions.dtype is torch.int32) and (positions_out is None or positions_out.dtype is torch.int32)

    def make():
        a = EvictArgs()
        a.struct_size = C.sizeof(EvictArgs)
        a.n_layers, a.batch, a.n_groups, a.L, a.move_stride = n, b, g, width, stride
        a.budget, a.n_sink, a.n_recent = budget, int(n_sink), int(n_recent)
        return a, C.byref(a)

    a, ref = _calls.get(("evict", scores.shape, stride, budget, n_sink, n_recent), make)
    a.scores, a.kv_len, a.seq_len = scores.data_ptr(), _ints(kv_len, b, "kv_len"), _ints(seq_len, b, "seq_len")
    a.positions = None if positions is None else positions.data_ptr()
    a.src, a.dst = src.data_ptr(), dst.data_ptr()
    a.n_moves, a.new_len = _ints(n_moves, n * b * g, "n_moves"), _ints(new_len, b, "new_len")
    a.scores_out = None if scores_out is None else scores_out.data_ptr()
    a.positions_out = None if positions_out is None else positions_out.data_ptr()
    _call("evict", ref, index, stream)
    if stream is not None:
        for t in made:
            t.record_stream(stream)
    return src, dst, n_moves, new_len


def move_rows(pools: Sequence[torch.Tensor], src: torch.Tensor, dst: torch.Tensor, n_moves: torch.Tensor, *,
              params: Sequence[torch.Tensor] | None = None, block_table: torch.Tensor | None = None,
              pages_per_seq: int | None = None, status: torch.Tensor | None = None, stream=None):
    """specattn_move_rows: the moves of one draft layer's lists (src, dst [B, G, stride], n_moves [B, G] as ``evict`` gives
    them), in place, in the pools [n_pages, 2, page_size, n_kv_heads, X] of the layers that follow it: all of one
    shape, type and strides, with ``params`` beside them where the cache is held in 4 bits.  Returns ``status``."""
    if len(pools) == 0:
        if status is not None:
            status.zero_()
        return status
    pool = pools[0]
    par = None if params is None else params[0]
    index = _device(pool, src, dst, n_moves, block_table, status, *pools[1:], *(params or ()))
    key = ("move", len(pools), pool.shape, pool.stride(), pool.dtype, None if par is None else (par.shape, par.stride(), par.dtype),
           src.shape, None if block_table is None else (block_table.shape, block_table.stride()), pages_per_seq)

    def make():
        n_pages, two, page, heads, width = pool.shape
        b, g, stride = src.shape
        assert two == 2 and pool.stride(4) == 1
        a = MoveArgs()
        a.struct_size = C.sizeof(MoveArgs)
        a.n_pools, a.batch, a.n_groups, a.n_kv_heads, a.page_size, a.n_pages = len(pools), b, g, heads, page, n_pages
        size = pool.element_size()
        a.row_bytes = width * size
        a.stride_page, a.stride_kv, a.stride_slot, a.stride_head = [x * size for x in _strides(pool, 0, 4)]
        ptrs, par_ptrs = (C.c_void_p * len(pools))(), None
        a.pools = ptrs
        if par is not None:
            assert len(params) == len(pools) and par.shape[:4] == pool.shape[:4] and par.stride(4) == 1
            size = par.element_size()
            a.param_bytes = par.shape[4] * size
            a.pstride_page, a.pstride_kv, a.pstride_slot, a.pstride_head = [x * size for x in _strides(par, 0, 4)]
            par_ptrs = (C.c_void_p * len(pools))()
            a.params = par_ptrs
        if block_table is not None:
            assert block_table.dim() == 2 and block_table.shape[0] == b and (block_table.shape[1] <= 1 or block_table.stride(1) == 1)
            a.block_table_stride = _table_stride(block_table)
        else:
            assert pages_per_seq is not None, "without a block table: pages_per_seq"
            a.block_table_stride = int(pages_per_seq)
        a.move_stride = stride
        return a, C.byref(a), ptrs, par_ptrs

    a, ref, ptrs, par_ptrs = _calls.get(key, make)
    for i, t in enumerate(pools):
        assert t is pool or (t.shape == pool.shape and t.stride() == pool.stride() and t.dtype is pool.dtype)
        ptrs[i] = t.data_ptr()
    if par is not None:
        for i, t in enumerate(params):
            assert t is par or (t.shape == par.shape and t.stride() == par.stride() and t.dtype is par.dtype)
            par_ptrs[i] = t.data_ptr()
    for t in (src, dst):
        assert t.dtype is torch.int32 and t.is_contiguous() and t.shape == src.shape
    if block_table is not None:
        assert block_table.dtype is torch.int32
        a.block_table = block_table.data_ptr()
    a.src, a.dst, a.n_moves = src.data_ptr(), dst.data_ptr(), _ints(n_moves, a.batch * a.n_groups, "n_moves")
    a.status = _ints(status, a.batch, "status")
    _call("move_rows", ref, index, stream)
    return status
