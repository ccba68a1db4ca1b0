"""The cache's operators without a GPU: structs, refusals, and what four bits keep of a row."""
import ctypes as C
import re
import subprocess
from pathlib import Path

import pytest
import torch

import paper_2510_27641_b200 as sa
from kv4_util import quantise, values
from paper_2510_27641_b200 import cache_ops

ROOT = Path(__file__).resolve().parent.parent
STRUCTS = {"specattn_kv4_cache": sa.Kv4Cache, "specattn_kv4_rows_args": sa.Kv4RowsArgs, "specattn_kv4_verify_args": sa.Kv4VerifyArgs,
           "specattn_accumulate_args": sa.AccumulateArgs, "specattn_evict_args": sa.EvictArgs, "specattn_move_args": sa.MoveArgs}
POINTER = 1 << 20     # aligned, never followed: every call below is refused before it would be


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2510_27641_b200 import build
    build.build()


def test_every_field_lies_where_the_header_puts_it(tmp_path):
    text = ['#include <stdio.h>\n#include <stddef.h>\n#include "specattn.h"\nint main(){']
    for name, s in STRUCTS.items():
        text.append(f'printf("%zu", sizeof({name}));')
        text += [f'printf(" %zu", offsetof({name}, {f[0]}));' for f in s._fields_]
        text.append('printf("\\n");')
    (tmp_path / "sz.c").write_text("\n".join(text) + "return 0;}\n")
    subprocess.run(["gcc", "-I", str(ROOT / "include"), str(tmp_path / "sz.c"), "-o", str(tmp_path / "sz")], check=True)
    got = subprocess.run([str(tmp_path / "sz")], check=True, capture_output=True, text=True).stdout.splitlines()
    for line, s in zip(got, STRUCTS.values()):
        assert [int(x) for x in line.split()] == [C.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_], s


def test_the_declared_entry_points_are_exported():
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "specattn.h").read_text(), flags=re.S)
    names = set(re.findall(r"\b(specattn_[a-z0-9_]+)\s*\(", text))
    assert {"specattn_kv4_append", "specattn_kv4_read", "specattn_kv4_verify", "specattn_kv4_verify_workspace_bytes", "specattn_accumulate",
            "specattn_evict", "specattn_move_rows"} <= names
    for n in names:
        assert hasattr(sa.lib(), n), n


def _cache(c):
    c.codes = c.params = POINTER
    c.n_pages, c.page_size, c.block_table_stride, c.dtype = 8, 16, 4, 0
    c.stride_page, c.stride_kv, c.stride_slot, c.stride_head = 4096, 2048, 64, 1024
    c.pstride_page, c.pstride_kv, c.pstride_slot, c.pstride_head = 128, 64, 2, 32


def _rows():
    a = sa.Kv4RowsArgs()
    a.struct_size = C.sizeof(sa.Kv4RowsArgs)
    a.batch, a.n_tokens, a.n_kv_heads, a.head_dim = 2, 3, 2, 128
    _cache(a.cache)
    a.k = a.v = a.start = POINTER
    for side in "kv":
        for what, x in (("batch", 768), ("token", 256), ("head", 128)):
            setattr(a, f"{side}_stride_{what}", x)
    return a


def _verify():
    a = sa.Kv4VerifyArgs()
    a.struct_size = C.sizeof(sa.Kv4VerifyArgs)
    a.batch, a.n_q, a.n_q_heads, a.n_kv_heads, a.head_dim, a.n_groups = 2, 3, 8, 2, 128, 1
    _cache(a.cache)
    a.q = a.kv_len = a.idx = a.counts = a.out = a.lse = a.workspace = POINTER
    a.idx_stride, a.workspace_bytes = 64, 1 << 30
    return a


def _accumulate():
    a = sa.AccumulateArgs()
    a.struct_size = C.sizeof(sa.AccumulateArgs)
    a.n_layers, a.batch, a.n_draft_heads, a.gamma, a.n_groups, a.L_stride, a.score_stride, a.decay = 1, 2, 4, 3, 2, 64, 64, 1.0
    a.draft_probs = (C.c_void_p * 1)(POINTER)
    a.kv_len = a.scores_out = POINTER
    a.head_group = (C.c_int32 * 4)(0, 0, 1, 1)
    return a


def _evict():
    a = sa.EvictArgs()
    a.struct_size = C.sizeof(sa.EvictArgs)
    a.n_layers, a.batch, a.n_groups, a.L, a.budget, a.n_sink, a.n_recent, a.move_stride = 1, 2, 2, 100, 60, 4, 8, 40
    a.scores = a.src = a.dst = a.n_moves = POINTER
    a.kv_len, a.new_len = POINTER, POINTER + 4096
    return a


def _move():
    a = sa.MoveArgs()
    a.struct_size = C.sizeof(sa.MoveArgs)
    a.n_pools, a.batch, a.n_groups, a.n_kv_heads, a.page_size, a.n_pages = 1, 2, 1, 2, 16, 8
    a.pools = (C.c_void_p * 1)(POINTER)
    a.row_bytes, a.stride_page, a.stride_kv, a.stride_slot, a.stride_head = 256, 16384, 8192, 512, 256
    a.src = a.dst = a.n_moves = POINTER
    a.block_table_stride, a.move_stride = 4, 10
    return a


NULL, SIZE, RANGE, ALIGN, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4, -5, -6
REFUSALS = [
    ("kv4_append", _rows, [("struct_size", 8, SIZE), ("batch", -1, RANGE), ("batch", 1 << 17, RANGE), ("n_tokens", -1, RANGE), ("n_kv_heads", 0, RANGE),
                           ("head_dim", 64, UNSUPPORTED), ("reserved", 1, RANGE), ("k", None, NULL), ("v", None, NULL), ("start", None, NULL),
                           ("cache.codes", None, NULL), ("cache.params", None, NULL), ("cache.n_pages", 0, RANGE), ("cache.page_size", 0, RANGE),
                           ("cache.dtype", 2, RANGE), ("cache.block_table_stride", -1, RANGE), ("cache.codes", POINTER + 8, ALIGN),
                           ("cache.params", POINTER + 2, ALIGN), ("cache.stride_slot", 72, ALIGN), ("cache.pstride_head", 3, ALIGN),
                           ("k", POINTER + 2, ALIGN), ("v_stride_head", 132, ALIGN), ("k_stride_token", 4, ALIGN)]),
    ("kv4_read", _rows, [("struct_size", 0, SIZE), ("head_dim", 129, UNSUPPORTED), ("v", None, NULL)]),
    ("kv4_verify", _verify, [("struct_size", 0, SIZE), ("batch", -1, RANGE), ("n_q", 0, RANGE), ("n_q_heads", 7, RANGE), ("n_groups", 3, RANGE),
                             ("sm_scale", -1.0, RANGE), ("sm_scale", float("nan"), RANGE), ("tail_len", 65, RANGE), ("tail_len", -1, RANGE),
                             ("flags", 1, RANGE), ("flags", 6, RANGE), ("flags", 4, UNSUPPORTED), ("head_dim", 64, UNSUPPORTED), ("n_q", 17, UNSUPPORTED), ("n_q", 1 << 30, UNSUPPORTED),
                             ("batch", 1025, UNSUPPORTED), ("idx_stride", -1, RANGE), ("idx_stride", (1 << 23) + 1, UNSUPPORTED),
                             ("q", None, NULL), ("kv_len", None, NULL), ("idx", None, NULL), ("counts", None, NULL), ("out", None, NULL),
                             ("lse", None, NULL), ("workspace", None, NULL), ("q", POINTER + 8, ALIGN), ("out", POINTER + 8, ALIGN),
                             ("workspace", POINTER + 128, ALIGN), ("cache.codes", None, NULL), ("cache.dtype", -1, RANGE),
                             ("cache.n_pages", 1 << 31, RANGE), ("cache.stride_head", 8, ALIGN), ("n_q_heads", 1 << 30, UNSUPPORTED),
                             ("cache.stride_page", -1024, UNSUPPORTED), ("cache.stride_kv", -1024, UNSUPPORTED),
                             ("cache.stride_slot", -64, UNSUPPORTED), ("cache.stride_head", -64, UNSUPPORTED),
                             ("cache.pstride_page", -2, UNSUPPORTED), ("cache.pstride_kv", -2, UNSUPPORTED),
                             ("cache.pstride_slot", -2, UNSUPPORTED), ("cache.pstride_head", -2, UNSUPPORTED),
                             ("cache.stride_page", 1 << 36, UNSUPPORTED), ("cache.stride_slot", 1 << 36, UNSUPPORTED),
                             ("cache.stride_kv", 1 << 36, UNSUPPORTED), ("cache.pstride_page", 1 << 33, UNSUPPORTED),
                             ("cache.block_table_stride", 1 << 31, UNSUPPORTED)]),
    ("accumulate", _accumulate, [("struct_size", 0, SIZE), ("n_layers", 0, RANGE), ("n_layers", 65, RANGE), ("batch", -1, RANGE), ("gamma", 0, RANGE),
                                 ("gamma", 1025, UNSUPPORTED), ("n_groups", 0, RANGE), ("n_draft_heads", 257, RANGE), ("L_stride", 0, RANGE),
                                 ("L_stride", 196612, RANGE), ("L_stride", 63, ALIGN), ("score_stride", 0, RANGE), ("decay", -0.5, RANGE),
                                 ("decay", float("nan"), RANGE), ("decay", float("inf"), RANGE), ("kv_len", None, NULL), ("scores_out", None, NULL),
                                 ("draft_probs", None, NULL), ("draft_probs", (C.c_void_p * 1)(POINTER + 4), ALIGN),
                                 ("head_group", (C.c_int32 * 4)(0, 0, 2, 1), RANGE), ("head_group", (C.c_int32 * 4)(0, -1, 1, 1), RANGE)]),
    ("evict", _evict, [("struct_size", 0, SIZE), ("n_layers", 0, RANGE), ("batch", -1, RANGE), ("L", 0, RANGE), ("L", 196609, RANGE), ("budget", 0, RANGE),
                       ("n_sink", -1, RANGE), ("n_recent", -1, RANGE), ("n_recent", 57, RANGE), ("n_recent", (1 << 31) - 1, RANGE),
                       ("move_stride", 39, RANGE), ("reserved", 1, RANGE), ("scores", None, NULL), ("kv_len", None, NULL), ("src", None, NULL),
                       ("dst", None, NULL), ("n_moves", None, NULL), ("new_len", None, NULL), ("positions_out", POINTER, NULL),
                       ("new_len", POINTER, RANGE), ("seq_len", POINTER + 4096, RANGE)]),
    ("move_rows", _move, [("struct_size", 0, SIZE), ("n_pools", -1, RANGE), ("batch", -1, RANGE), ("n_groups", 3, RANGE), ("page_size", 0, RANGE),
                          ("n_pages", 0, RANGE), ("row_bytes", 24, ALIGN), ("row_bytes", 8192, RANGE), ("row_bytes", 0, RANGE), ("stride_slot", 8, ALIGN),
                          ("param_bytes", 4, NULL), ("params", (C.c_void_p * 1)(POINTER), NULL), ("pools", None, NULL),
                          ("pools", (C.c_void_p * 1)(None), NULL), ("pools", (C.c_void_p * 1)(POINTER + 8), ALIGN), ("src", None, NULL),
                          ("dst", None, NULL), ("n_moves", None, NULL), ("block_table_stride", -1, RANGE), ("move_stride", -1, RANGE),
                          ("batch", 70000, UNSUPPORTED), ("stride_page", -16, RANGE), ("stride_kv", -16, RANGE), ("stride_slot", -16, RANGE),
                          ("stride_head", -16, RANGE), ("pstride_page", -4, RANGE), ("pstride_kv", -4, RANGE),
                          ("pstride_slot", -4, RANGE), ("pstride_head", -4, RANGE)]),
]


@pytest.mark.parametrize("name,make,field,value,code", [(n, m, *r) for n, m, rs in REFUSALS for r in rs])
def test_refusals(name, make, field, value, code):
    a = make()
    at = a
    *outer, last = field.split(".")
    for o in outer:
        at = getattr(at, o)
    setattr(at, last, value)
    before = sa.kernel_launch_count()
    assert getattr(sa.lib(), "specattn_" + name)(C.byref(a), None) == code
    assert sa.kernel_launch_count() == before
    if name == "kv4_verify" and field in ("n_q", "tail_len", "head_dim", "n_groups"):
        assert sa.lib().specattn_kv4_verify_workspace_bytes(C.byref(a)) == 0


@pytest.mark.parametrize("name,make", [(n, m) for n, m, _ in REFUSALS])
def test_nothing_to_do_and_no_arguments(name, make):
    entry = getattr(sa.lib(), "specattn_" + name)
    assert entry(None, None) == NULL
    a = make()
    a.batch = 0
    assert entry(C.byref(a), None) == 0
    if name in ("kv4_append", "kv4_read"):   # no token: no rows to look at
        a = make()
        a.n_tokens, a.k, a.v, a.status = 0, None, None, None
        assert entry(C.byref(a), None) == 0
    if name == "move_rows":
        a = make()
        a.move_stride, a.src, a.dst, a.status = 0, None, None, None
        assert entry(C.byref(a), None) == 0


def test_tensors_that_no_call_takes():
    codes, params = torch.zeros(4, 2, 16, 2, 64, dtype=torch.uint8), torch.zeros(4, 2, 16, 2, 2, dtype=torch.bfloat16)
    k, n = torch.zeros(1, 3, 2, 128, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        sa.kv4_append(k, k, codes, params, n, pages_per_seq=4)
    with pytest.raises(ValueError, match="CUDA"):
        sa.kv4_verify(k, codes, params, n, pages_per_seq=4, dense=True)
    with pytest.raises(ValueError, match="CUDA"):
        sa.accumulate_attention([torch.zeros(1, 1, 1, 8)], n, torch.zeros(1, 1, 1, 8))
    with pytest.raises(ValueError, match="CUDA"):
        sa.evict(torch.zeros(1, 1, 1, 8), n, 4)
    with pytest.raises(ValueError, match="CUDA"):
        sa.move_rows([codes], n, n, n)


class _Recorder:
    """Stands in for the shared library: keeps what it was called with."""

    def __init__(self):
        self.seen = []

    def __getattr__(self, name):
        def entry(ref, stream=None):
            self.seen.append((name, ref._obj))
            return 4096
        def call(ref, stream):
            self.seen.append((name, ref._obj))
            return 0
        return entry if name.endswith("bytes") else call


@pytest.fixture
def recorder(monkeypatch):
    r = _Recorder()
    monkeypatch.setattr(cache_ops, "lib", lambda: r)
    monkeypatch.setattr(cache_ops, "_stream_ptr", lambda stream: 0)
    monkeypatch.setattr(cache_ops, "_raw_device", lambda: 0)
    monkeypatch.setattr(cache_ops, "_device", lambda *t: 0)
    monkeypatch.setattr(cache_ops, "kv4_verify_workspace_bytes", lambda q, codes: 4096)
    monkeypatch.setattr(cache_ops, "_calls", sa._Calls())
    return r


def test_types_and_shapes_that_are_refused(recorder):
    codes, params = torch.zeros(4, 2, 16, 2, 64, dtype=torch.uint8), torch.zeros(4, 2, 16, 2, 2, dtype=torch.bfloat16)
    k, n = torch.zeros(2, 3, 2, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    table = torch.zeros(2, 2, dtype=torch.int32)
    append = lambda k=k, v=k, codes=codes, params=params, n=n, **kw: sa.kv4_append(k, v, codes, params, n, **kw)
    append(block_table=table)
    for bad in (dict(k=k.half()), dict(v=k.float()), dict(n=n.long()), dict(n=n[:1]), dict(codes=codes.to(torch.int8)), dict(params=params.float()),
                dict(params=params[:3]), dict(k=k[..., :64]), dict(k=k[:, :, :1], v=k[:, :, :1]), dict(block_table=table.long()),
                dict(block_table=table[:1]), dict(block_table=torch.zeros(2, 4, dtype=torch.int32)[:, :2]), dict(status=n.float()), {}):
        with pytest.raises(AssertionError):
            append(**({"block_table": table} | bad if bad else {}))
    idx, cnt = torch.zeros(2, 1, 8, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32)
    q = torch.zeros(2, 3, 8, 128, dtype=torch.bfloat16)
    sa.kv4_verify(q, codes, params, n, block_table=table, idx=idx, counts=cnt)
    for bad in (dict(q=q.half()), dict(q=q.transpose(1, 2)), dict(idx=idx.long()), dict(idx=idx[:, 0]), dict(counts=cnt.long()),
                dict(counts=cnt[:1]), dict(out=q.half()), dict(out=q[:1]), dict(lse=q[..., 0]), dict(n_groups=2)):
        with pytest.raises(AssertionError):
            kw = dict(q=q, idx=idx, counts=cnt) | bad
            sa.kv4_verify(kw.pop("q"), codes, params, n, block_table=table, **kw)
    with pytest.raises(AssertionError):
        sa.evict(torch.zeros(1, 2, 1, 8), n, 4, src=torch.zeros(1, 2, 1, 4, dtype=torch.int64))
    with pytest.raises(AssertionError):
        sa.evict(torch.zeros(1, 2, 1, 8, dtype=torch.float64), n, 4)
    with pytest.raises(AssertionError):
        sa.accumulate_attention([torch.zeros(2, 1, 1, 8)], n, torch.zeros(2, 2, 1, 8))
    with pytest.raises(AssertionError):
        sa.accumulate_attention([torch.zeros(2, 1, 1, 8)], n)
    with pytest.raises(AssertionError):
        sa.accumulate_attention([None, None], n, torch.zeros(2, 2, 1, 8))
    with pytest.raises(AssertionError):
        sa.kv4_verify(q, codes, params, n, block_table=table, idx=idx)
    # what is written twice in one place
    same = k[:, :1].expand(2, 3, 2, 128)
    append(k=same, v=same, block_table=table)
    for bad in (dict(k=same), dict(v=same)):
        with pytest.raises(AssertionError):
            sa.kv4_read(codes, params, n, block_table=table, **({"k": k, "v": k} | bad))
    with pytest.raises(AssertionError):
        append(codes=codes[:1].expand(4, 2, 16, 2, 64), block_table=table)
    moves = torch.zeros(2, 1, 8, dtype=torch.int32)
    with pytest.raises(AssertionError):
        sa.move_rows([codes[:, :1].expand(4, 2, 16, 2, 64)], moves, moves, cnt, block_table=table)


def test_kept_structs_follow_every_value_of_a_call(recorder):
    codes, params = torch.zeros(4, 2, 16, 2, 64, dtype=torch.uint8), torch.zeros(4, 2, 16, 2, 2, dtype=torch.bfloat16)
    n, q = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 3, 8, 128, dtype=torch.bfloat16)
    table = torch.zeros(2, 2, dtype=torch.int32)
    got = []
    for kw in (dict(sm_scale=0.5), dict(sm_scale=0.25), dict(tail_len=3), dict(out=torch.zeros(q.shape)), dict(pages_per_seq=2)):
        sa.kv4_verify(q, codes, params, n, dense=True, **({"block_table": table} if "pages_per_seq" not in kw else {}), **kw)
        a = recorder.seen[-1][1]
        got.append((a.sm_scale, a.tail_len, a.out_f32, a.cache.block_table is None, a.dense, a.idx is None, a.n_q_heads))
    assert got == [(0.5, 0, 0, False, 1, True, 8), (0.25, 0, 0, False, 1, True, 8), (0.0, 3, 0, False, 1, True, 8),
                   (0.0, 0, 1, False, 1, True, 8), (0.0, 0, 0, True, 1, True, 8)]
    w = torch.zeros(1, 2, 1, 100)
    for budget, sink in ((60, 0), (60, 4), (50, 4)):
        sa.evict(w, n, budget, n_sink=sink)
        a = recorder.seen[-1][1]
        assert (a.budget, a.n_sink, a.move_stride, a.positions) == (budget, sink, min(budget, 100 - budget), None)
    probs = [torch.zeros(2, 4, 3, 64), None]
    for decay, groups in ((1.0, None), (0.5, None), (0.5, [0, 0, 0, 0])):
        sa.accumulate_attention(probs, n, torch.zeros(2, 2, 1, 64), decay=decay, head_group=groups)
        a = recorder.seen[-1][1]
        assert (a.decay, bool(a.head_group), a.draft_probs[0], a.draft_probs[1]) == (decay, groups is not None, probs[0].data_ptr(), None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_what_four_bits_keep_of_a_row(dtype):
    """Half a step of the scale, and what the scale's own rounding adds at the far end of the codes."""
    gen = torch.Generator().manual_seed(1)
    x = (torch.randn(500, 128, generator=gen) * torch.exp(3 * torch.randn(500, 1, generator=gen)) + torch.randn(500, 1, generator=gen)).to(dtype)
    got, (codes, params) = values(*quantise(x)), quantise(x)
    s = params[:, :1].double()
    half = torch.finfo(dtype).eps / 2
    assert torch.all((got - x.double()).abs() <= s * (0.5 + 15 * half) * (1 + 2.0 ** -20))
    assert torch.equal(params[:, 1], x.amin(-1))
