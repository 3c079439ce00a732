"""What the calls of a block-scaled cache and of its pages refuse before anything is enqueued: host checks, over a context that is made up
here and addresses that nobody follows.  No GPU call."""
import ctypes as C

import pytest
import torch

from paper_2603_08899_b200 import binding as cb
from paper_2603_08899_b200 import build

ARG, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4, -5
AT = 1 << 20                                         # an aligned address


class Ctx(C.Structure):
    """The context as csrc/common.cuh declares it."""
    _fields_ = [("device", C.c_int), ("sm_count", C.c_int), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
                ("block_table", C.c_void_p), ("max_pages", C.c_int32), ("last_error", C.c_int), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("attention_path", C.c_int), ("wait_ns", C.c_ulonglong),
                ("k_block", C.c_void_p), ("v_block", C.c_void_p), ("k_soft", C.c_void_p), ("v_soft", C.c_void_p), ("block", C.c_int),
                ("k_layers", C.c_void_p), ("v_layers", C.c_void_p), ("layer_block", C.c_int)]


class Stream:
    cuda_stream = 0


@pytest.fixture()
def ctx():
    build.build()
    return Ctx(sm_count=148)


def handle(ctx):
    return C.c_void_p(C.addressof(ctx)) if ctx is not None else None


def refused(code, call, *a, **kw):
    with pytest.raises(cb.ConfuError) as e:
        call(*a, **kw)
    assert e.value.code == code


def dims(**kw):
    d = dict(B=2, Hq=8, Hkv=2, D=128, T=4, Cn=2, S=0, dtype=cb.FP8_BLOCK)
    d.update(kw)
    return cb.make_dims(**d)


def scales(ctx, *a):
    return cb.confu_set_kv_block_scales(handle(ctx), *a)


def test_settings(ctx):
    for block in (0, 1, 16, 33, 96, 256, -32):
        refused(ARG, scales, ctx, AT, AT, None, None, block)
        refused(ARG, cb.confu_set_kv_block_scale_layers, handle(ctx), AT, AT, block)
    refused(ARG, scales, ctx, AT, None, None, None, 32)
    refused(ARG, scales, ctx, AT, AT, AT, None, 32)
    refused(ARG, scales, ctx, None, None, AT, AT, 32)
    refused(ARG, cb.confu_set_kv_block_scale_layers, handle(ctx), AT, None, 32)
    refused(ARG, scales, None, AT, AT, None, None, 32)
    scales(ctx, AT, 2 * AT, 3 * AT, 4 * AT, 64)
    cb.confu_set_kv_block_scale_layers(handle(ctx), 5 * AT, 6 * AT, 128)
    assert (ctx.k_block, ctx.v_block, ctx.k_soft, ctx.v_soft, ctx.block) == (AT, 2 * AT, 3 * AT, 4 * AT, 64)
    assert (ctx.k_layers, ctx.v_layers, ctx.layer_block) == (5 * AT, 6 * AT, 128)
    scales(ctx, None, None)
    cb.confu_set_kv_block_scale_layers(handle(ctx), None, None)
    assert (ctx.k_block, ctx.k_soft, ctx.block, ctx.k_layers, ctx.layer_block) == (None, None, 0, None, 0)


def test_dims_and_paths(ctx):
    path = lambda **kw: cb.lib().confu_attention_path(C.byref(ctx), C.byref(dims(**kw)))  # noqa: E731
    for kw in (dict(D=96), dict(D=256), dict(Hq=9)):
        assert path(**kw) == SHAPE
    for kw in (dict(Hq=66), dict(S=129), dict(T=65)):
        assert path(**kw) == UNSUPPORTED
    assert path(dtype=4) == ARG and path(dtype=-1) == ARG
    for kw in (dict(), dict(D=64), dict(Hq=64), dict(S=128), dict(T=64, Cn=64), dict(T=1, Cn=0)):
        assert path(**kw) >= 0
        assert cb.lib().confu_plan_bytes(C.byref(ctx), C.byref(dims(**kw))) > 0
    ctx.attention_path = cb.ATTENTION_TENSOR_PAIR
    assert path() == UNSUPPORTED
    # 16 rows x heads of a kv head (32 at head dim 64), 20 (one M tile), 256 of few and of many (sequence, kv head) pairs
    few, one, whole, batch = dict(T=4, Cn=0), dict(T=5, Cn=0), dict(T=60, Cn=4), dict(T=60, Cn=4, B=100)
    G, N, T = cb.ATTENTION_GENERIC, cb.ATTENTION_TENSOR_NARROW, cb.ATTENTION_TENSOR
    for option, want in ((cb.ATTENTION_AUTO, (G, N, N, T)), (cb.ATTENTION_GENERIC, (G,) + 3 * (UNSUPPORTED,)), (cb.ATTENTION_TENSOR, (N, N, N, T))):
        ctx.attention_path = option
        assert tuple(path(**kw) for kw in (few, one, whole, batch)) == want
        assert tuple(path(D=64, **kw) for kw in (dict(T=8, Cn=0), dict(T=9, Cn=0), whole, batch)) == want
    ctx.attention_path, ctx.sm_count = cb.ATTENTION_AUTO, 1          # a share is walked by a CTA per group of query rows
    assert path(T=64, Cn=64) == UNSUPPORTED and path(**whole) == T and path(**one) == N


def attention(ctx, d, table=True, soft=None, ws=1 << 40, n_slots=1280, q=AT):
    ctx.workspace, ctx.workspace_bytes = AT, ws
    ctx.block_table, ctx.max_pages = (AT, 4) if table else (None, 0)
    cb.confu_tree_attention(handle(ctx), d, q, AT, AT, n_slots, AT, AT, soft, soft, AT, AT, None, AT, None, AT, Stream())


def test_attention_append_and_compaction(ctx):
    scales(ctx, AT, AT, None, None, 32)
    cb.confu_set_kv_block_scale_layers(handle(ctx), AT, AT, 32)
    refused(UNSUPPORTED, attention, ctx, dims(), table=False)
    refused(SHAPE, attention, ctx, dims(), n_slots=1281)
    refused(ALIGN, attention, ctx, dims(), q=AT + 2)
    refused(WORKSPACE, attention, ctx, dims(), ws=1000)
    refused(ARG, attention, ctx, dims(S=4))
    refused(UNSUPPORTED, attention, ctx, dims(S=4), soft=AT)         # soft prompts without scales
    append = lambda d: cb.confu_kv_append(handle(ctx), d, AT, AT, AT, AT, AT, AT, Stream())  # noqa: E731
    compact = lambda d, n=2: cb.confu_kv_compact(handle(ctx), d, n, AT, AT, AT, AT, AT, AT, AT, AT, Stream())  # noqa: E731
    ctx.block_table = None
    refused(UNSUPPORTED, append, dims())
    refused(UNSUPPORTED, compact, dims())
    ctx.block_table, ctx.max_pages = AT, 4
    scales(ctx, None, None)
    cb.confu_set_kv_block_scale_layers(handle(ctx), None, None)
    refused(UNSUPPORTED, attention, ctx, dims())
    refused(UNSUPPORTED, append, dims())
    refused(UNSUPPORTED, compact, dims())
    refused(ARG, compact, dims(), -1)
    append(dims(B=0))
    compact(dims(B=0))


def test_pages(ctx):
    pages = lambda n=10, rows=4, width=3, ref=AT, table=AT: cb.ConfuPages(n, rows, width, ref, table)  # noqa: E731
    L = cb.lib()
    st = C.c_void_p(0)
    at = C.c_void_p(AT)
    p = C.byref

    def fork(pg=pages(), d=None, layers=2, k=at, n=3, ws=at, ws_bytes=1 << 30, src=at):
        return L.confu_pages_fork(p(ctx), p(d or dims(dtype=torch.bfloat16)), layers, k, at, p(pg) if pg else None, n, src, at, at, ws, C.c_size_t(ws_bytes), st, st)

    def compact(pg=pages(), d=None, layers=2, used=at, ws=at, ws_bytes=1 << 30):
        return L.confu_pages_compact(p(ctx), p(d or dims(dtype=torch.bfloat16)), layers, at, at, p(pg) if pg else None, st, used, ws, C.c_size_t(ws_bytes), st)

    def copy(n_pages=10, n=3, d=None, src=at):
        return L.confu_pages_copy(p(ctx), p(d or dims(dtype=torch.bfloat16)), 2, at, at, n_pages, n, src, at, st, st)
    reserve = lambda pg=pages(), n=3, rows=at: L.confu_pages_reserve(p(ctx), p(pg) if pg else None, n, rows, at, st, st)  # noqa: E731
    free = lambda pg=pages(), n=3, rows=at: L.confu_pages_free(p(ctx), p(pg) if pg else None, n, rows, st, st)  # noqa: E731
    for call in (fork, compact, reserve, free):
        assert call(None) == ARG
        assert call(pages(ref=None)) == ARG and call(pages(table=None)) == ARG
        for bad in (pages(n=0), pages(rows=0), pages(width=-1)):
            assert call(bad) == SHAPE
        assert call(pages(ref=AT + 4)) == ALIGN
        assert call(pages(n=(1 << 24))) == UNSUPPORTED and call(pages(width=1 << 24)) == UNSUPPORTED      # 2^31 slots
    for call in (fork, reserve, free):
        assert call(n=-1) == ARG and call(n=1025) == UNSUPPORTED and call(n=0) == 0
    assert reserve(rows=st) == ARG and free(rows=st) == ARG and fork(src=st) == ARG and copy(src=st) == ARG
    assert fork(layers=-1) == ARG and fork(k=st) == ARG and copy(n=-1) == ARG and copy(n_pages=0) == ARG and copy(n_pages=1 << 24) == UNSUPPORTED and copy(n=0) == 0
    assert fork(ws=st) == WORKSPACE and fork(ws_bytes=100) == WORKSPACE and fork(ws=C.c_void_p(AT + 8)) == ALIGN
    assert compact(used=st) == ARG and compact(ws_bytes=100) == WORKSPACE
    block = dims()
    assert fork(d=block) == compact(d=block) == copy(d=block) == UNSUPPORTED          # no scales to copy along
    assert fork(d=dims(D=80)) == SHAPE
    assert L.confu_pages_reserve(None, p(pages()), 3, at, at, st, st) == ARG
    assert cb.confu_pages_workspace_bytes(0) == 0 and cb.confu_pages_workspace_bytes(5) >= 8 * 1024
    assert cb.confu_pages_workspace_bytes(1 << 20) >= 12 << 20
    assert b"free pages" in L.confu_status_string(cb.ST_NO_PAGES) and b"page" in L.confu_status_string(cb.ST_BAD_PAGES)
