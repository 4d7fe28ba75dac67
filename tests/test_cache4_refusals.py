"""Arguments that the calls of the 4-bit cache and of the page tables refuse, before any launch.

No GPU: every call here is answered by the host's checks.  The addresses are never followed."""
import ctypes

import pytest
import torch

from paper_2407_07304_b200 import binding as slim
from paper_2407_07304_b200 import harness

A = 1 << 20        # an aligned address that nothing reads
C, E = 1 << 21, 1 << 22
INVALID, UNSUPPORTED, WORKSPACE, OK = (slim.SLIM_ERR_INVALID_ARG, slim.SLIM_ERR_UNSUPPORTED, slim.SLIM_ERR_WORKSPACE, slim.SLIM_OK)


def cache(**kw):
    f = dict(codes=A, scales=A, block_table=A, num_pages=8, page_tokens=128, num_kv_heads=2, head_dim=128, max_pages_per_seq=4)
    f.update(kw)
    return slim.SlimCacheStruct(*[f[n] for n, _ in slim.SlimCacheStruct._fields_])


CACHES = [(dict(c=cache(codes=None)), INVALID), (dict(c=cache(scales=None)), INVALID), (dict(c=cache(block_table=None)), INVALID),
          (dict(c=cache(codes=A + 8)), INVALID), (dict(c=cache(scales=A + 4)), INVALID), (dict(c=cache(num_pages=0)), INVALID),
          (dict(c=cache(num_kv_heads=0)), INVALID), (dict(c=cache(max_pages_per_seq=0)), INVALID), (dict(c=cache(page_tokens=64)), UNSUPPORTED),
          (dict(c=cache(head_dim=64)), UNSUPPORTED), (dict(B=-1), INVALID), (dict(B=65536), UNSUPPORTED), (dict(B=0), OK)]


@pytest.mark.parametrize("name", ["slim_kv4_append", "slim_kv4_read"])
@pytest.mark.parametrize("kw,want", CACHES + [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=A + 8), INVALID), (dict(v=A + 2), INVALID), (dict(cu=None), INVALID),
    (dict(start=None), INVALID), (dict(n=-1), INVALID), (dict(n=0, k=None), OK), (dict(n=1 << 30), UNSUPPORTED),
])
def test_rows_are_refused(name, kw, want):
    f = dict(c=cache(), k=A, v=A, cu=A, start=A, B=2, n=3)
    f.update(kw)
    assert getattr(slim.lib(), name)(ctypes.byref(f["c"]), f["k"], f["v"], f["cu"], f["start"], f["B"], f["n"], None) == want


@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("kw,want", CACHES + [
    (dict(q=None), INVALID), (dict(q=A + 8), INVALID), (dict(out=None), INVALID), (dict(out=A + 8), INVALID), (dict(cu=None), INVALID),
    (dict(kv=None), INVALID), (dict(mq=-1), INVALID), (dict(mk=-1), INVALID), (dict(mk=513), INVALID), (dict(hq=0), INVALID), (dict(hq=5), UNSUPPORTED),
    (dict(ws=None), WORKSPACE), (dict(n=8), WORKSPACE), (dict(ws=A + 2), INVALID), (dict(mq=0, q=None), OK),
])
def test_prefill_refuses(step, kw, want):
    f = dict(c=cache(), q=A, out=A, cu=A, kv=A, B=2, mq=3, mk=512, hq=4, ws=A, n=64)
    f.update(kw)
    new = (A, A) if step else ()
    fn = slim.lib().slim_prefill4_step if step else slim.lib().slim_attn4_prefill
    assert fn(ctypes.byref(f["c"]), f["q"], *new, f["out"], f["cu"], f["kv"], f["B"], f["mq"], f["mk"], f["hq"], 0.1, f["ws"], f["n"], None) == want


@pytest.mark.parametrize("k,v", [(None, A), (A, None), (A + 8, A), (A, A + 8)])
def test_prefill_step_refuses_rows(k, v):
    assert slim.lib().slim_prefill4_step(ctypes.byref(cache()), A, k, v, A, A, A, 2, 3, 512, 4, 0.1, A, 64, None) == INVALID


@pytest.mark.parametrize("kw,want", CACHES + [
    (dict(q=None), INVALID), (dict(q=A + 8), INVALID), (dict(out=None), INVALID), (dict(out=A + 8), INVALID), (dict(kv=None), INVALID),
    (dict(k=A), INVALID), (dict(v=A), INVALID), (dict(k=A, v=A + 8), INVALID), (dict(mk=-1), INVALID), (dict(mk=513), INVALID), (dict(hq=0), INVALID),
    (dict(hq=5), UNSUPPORTED), (dict(hq=34), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(n=1000), WORKSPACE), (dict(ws=A + 8), INVALID),
    (dict(B=65535, hq=1 << 17, c=cache(num_kv_heads=1 << 16)), UNSUPPORTED),
])
def test_decode_refuses(kw, want):
    f = dict(c=cache(), q=A, k=None, v=None, out=A, kv=A, B=2, mk=512, hq=4, ws=A, n=1 << 30)
    f.update(kw)
    assert slim.lib().slim_attn4_decode(ctypes.byref(f["c"]), f["q"], f["k"], f["v"], f["out"], f["kv"], f["B"], f["mk"], f["hq"], 0.1, f["ws"], f["n"],
                                        None) == want


def test_sizes():
    L = slim.lib()
    assert L.slim_cache4_code_bytes(7, 5) == 7 * 5 * 2 * 128 * 64 and L.slim_cache4_scale_bytes(7, 5) == 7 * 5 * 2 * 128 * 4
    assert L.slim_cache4_code_bytes(0, 5) == 0 and L.slim_cache4_scale_bytes(7, -1) == 0
    assert L.slim_attn4_workspace_bytes(32, 32) > slim.WORKSPACE_HEADER_BYTES and L.slim_attn4_workspace_bytes(5, 2) == 0
    assert L.slim_attn4_workspace_bytes(34, 2) == 0 and L.slim_attn4_workspace_bytes(32, 2) > L.slim_attn4_workspace_bytes(16, 2)
    assert L.slim_pages_workspace_bytes(0, 4) == 0 and L.slim_pages_workspace_bytes(9, -1) == 0
    sizes = [[L.slim_pages_workspace_bytes(n, r) for r in (0, 1, 50)] for n in (1, 100, 1000)]
    assert all(a < b for row in sizes for a, b in zip(row, row[1:])) and all(a < b for x, y in zip(sizes, sizes[1:]) for a, b in zip(x, y))


def pages(**kw):
    f = dict(refs=A, table=A, held=A, num_pages=8, rows=3, stride=4)
    f.update(kw)
    return slim.SlimPagesStruct(*[f[n] for n, _ in slim.SlimPagesStruct._fields_])


def layer(**kw):
    f = dict(codes=A, scales=A, num_kv_heads=2, row_bytes=64)
    f.update(kw)
    return (slim.SlimLayerStruct * 1)(slim.SlimLayerStruct(*[f[n] for n, _ in slim.SlimLayerStruct._fields_]))


BAD_PAGES = [(dict(refs=None), INVALID), (dict(refs=A + 2), INVALID), (dict(table=None), INVALID), (dict(table=A + 1), INVALID), (dict(held=None), INVALID),
             (dict(num_pages=0), INVALID), (dict(rows=-1), INVALID), (dict(stride=0), INVALID), (dict(num_pages=(1 << 23) + 1), UNSUPPORTED),
             (dict(rows=(1 << 23) + 1), UNSUPPORTED)]
BAD_LAYERS = [(dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(codes=A + 8), INVALID), (dict(num_kv_heads=0), INVALID),
              (dict(num_kv_heads=65536), UNSUPPORTED), (dict(row_bytes=96), UNSUPPORTED), (dict(row_bytes=0), UNSUPPORTED)]


def call_fork(**kw):
    f = dict(src=pages(), dst=pages(table=C, held=C), parent=A, kv=A, len=C, layers=layer(), nl=1, result=A, ws=A, n=1 << 30)
    f.update(kw)
    return slim.lib().slim_pages_fork(ctypes.byref(f["src"]), ctypes.byref(f["dst"]), f["parent"], f["kv"], f["len"], f["layers"], f["nl"], f["result"],
                                      f["ws"], f["n"], None)


def call_grow(**kw):
    f = dict(src=pages(), kv=A, room=1, result=A, ws=A, n=1 << 30)
    f.update(kw)
    return slim.lib().slim_pages_grow(ctypes.byref(f["src"]), f["kv"], f["room"], f["result"], f["ws"], f["n"], None)


def call_compact(**kw):
    f = dict(src=pages(), dst=pages(), layers=layer(), nl=1, result=A, ws=A, n=1 << 30)
    f.update(kw)
    return slim.lib().slim_pages_compact(ctypes.byref(f["src"]), ctypes.byref(f["dst"]), f["layers"], f["nl"], f["result"], f["ws"], f["n"], None)


@pytest.mark.parametrize("call", [call_fork, call_grow, call_compact])
@pytest.mark.parametrize("fields,want", BAD_PAGES)
def test_page_tables_are_refused(call, fields, want):
    assert call(src=pages(**fields)) == want


@pytest.mark.parametrize("call", [call_fork, call_compact])
@pytest.mark.parametrize("fields,want", BAD_LAYERS)
def test_layers_are_refused(call, fields, want):
    assert call(layers=layer(**fields)) == want


@pytest.mark.parametrize("call,kw,want", [
    (call_fork, dict(parent=None), INVALID), (call_fork, dict(kv=None), INVALID), (call_fork, dict(len=None), INVALID), (call_fork, dict(len=A), INVALID),
    (call_fork, dict(result=None), INVALID), (call_fork, dict(nl=-1), INVALID), (call_fork, dict(layers=None), INVALID),
    (call_fork, dict(dst=pages(held=C)), INVALID), (call_fork, dict(dst=pages(table=C)), INVALID), (call_fork, dict(dst=pages(table=C, held=C, num_pages=7)), INVALID),
    (call_fork, dict(dst=pages(table=C, held=C, stride=5)), INVALID), (call_fork, dict(dst=pages(table=C, held=C, rows=-2)), INVALID),
    (call_fork, dict(ws=None), WORKSPACE), (call_fork, dict(n=64), WORKSPACE), (call_fork, dict(ws=A + 8), INVALID),
    (call_grow, dict(kv=None), INVALID), (call_grow, dict(room=-1), INVALID), (call_grow, dict(result=None), INVALID), (call_grow, dict(ws=None), WORKSPACE),
    (call_compact, dict(dst=pages(rows=2)), INVALID), (call_compact, dict(dst=pages(num_pages=9)), INVALID), (call_compact, dict(result=None), INVALID),
    (call_compact, dict(n=64), WORKSPACE),
])
def test_page_calls_refuse(call, kw, want):
    assert call(**kw) == want


@pytest.mark.parametrize("call,kw", [
    # a table of 48 bytes, counts of 12: the second one begins inside the first, or the first inside the second
    (call_fork, dict(dst=pages(table=A + 16, held=C))), (call_fork, dict(src=pages(table=A + 44), dst=pages(table=A, held=C))),
    (call_fork, dict(dst=pages(table=C, held=A + 8))), (call_fork, dict(src=pages(refs=A + 28), dst=pages(table=C, held=C))),
    (call_fork, dict(len=A + 8)), (call_fork, dict(parent=C)), (call_fork, dict(parent=C + 8)),
    (call_fork, dict(src=pages(rows=1), dst=pages(table=A - 32, held=C))),
    (call_compact, dict(dst=pages(table=A + 16))), (call_compact, dict(dst=pages(table=A - 16))), (call_compact, dict(dst=pages(held=A + 4))),
    (call_compact, dict(dst=pages(refs=A + 4))),
])
def test_tables_that_overlap_in_part_are_refused(call, kw):
    # (too small a workspace: a call that passes this check never launches)
    assert call(n=0, **kw) == INVALID


def test_tables_side_by_side_are_not():
    assert call_fork(n=0, dst=pages(table=A + 48, held=A + 12), len=A + 12) == WORKSPACE
    assert call_compact(n=0) == call_compact(n=0, dst=pages(table=A - 48, held=A + 12, refs=A + 32)) == WORKSPACE


def test_binding_refuses():
    make = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype)  # noqa: E731
    with pytest.raises(TypeError):
        slim.SlimPages(make(4, dtype=torch.int64), make(2, 3), make(2))
    with pytest.raises(TypeError):
        slim.SlimPages(make(4), make(2, 3), make(3))
    with pytest.raises(TypeError):
        slim.SlimPages(make(4), make(3, 2).T, make(2))
    with pytest.raises(ValueError):
        slim.PageLayers([slim.SlimCache4(1, 1, 1, device="cpu"), slim.SlimCache(1, 1, 2, device="cpu")])
    p, o = slim.SlimPages.empty(4, 2, 3, "cpu"), slim.SlimPages.empty(4, 2, 3, "cpu")
    layers = slim.PageLayers([slim.SlimCache4(1, 1, 5, device="cpu")])
    ws = slim.pages_workspace(4, 2, "cpu")
    with pytest.raises(slim.SlimError):      # a pool of another size
        slim.slim_pages_fork(layers, p, o, make(2), make(2), make(2), make(2), ws)
    with pytest.raises(slim.SlimError):      # one parent too few
        slim.slim_pages_fork(None, p, o, make(1), make(2), make(2), make(2), ws)
    with pytest.raises(slim.SlimError):
        slim.slim_pages_grow(p, make(2, dtype=torch.int64), 1, make(2), ws)
    int8, int4 = slim.SlimCache(1, 2, 1, device="cpu"), slim.SlimCache4(1, 2, 1, device="cpu")
    rows = torch.zeros((1, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(slim.SlimError):      # the other cache's codes would be read as this one's
        slim.slim_kv4_append(int8, rows, rows, make(2), make(1), 1, 1)
    with pytest.raises(slim.SlimError):
        slim.slim_kv_append(int4, rows, rows, make(2), make(1), 1, 1)
    with pytest.raises(slim.SlimError):
        slim.slim_attn_decode(int4, rows, rows, make(1), 1, 1, 2, 0.1, ws)
    with pytest.raises(slim.SlimError):      # rows that do not lie one behind the other
        slim.slim_attn4_decode(int4, torch.zeros((1, 4, 128), dtype=torch.bfloat16)[:, ::2], rows, make(1), 1, 1, 2, 0.1, ws)
    with pytest.raises(slim.SlimError):
        slim.slim_attn4_decode(int4, rows.float(), rows, make(1), 1, 1, 2, 0.1, ws)
    with pytest.raises(slim.SlimError):
        slim.slim_kv4_append(int4, rows[:, :1], rows, make(2), make(1), 1, 1)
    with pytest.raises(slim.SlimError):
        slim.slim_kv4_read(int4, rows.float(), rows, make(2), make(1), 1, 1)
    with pytest.raises(TypeError):
        int4.set_block_table(make(2, 3, dtype=torch.int64))


def test_sampled_run_refuses():
    run = harness.SampledRun(1, 4, 2, num_pages=4, rows=3, max_tokens=256, device="cpu")
    for counts in ([1, 1], [1, -1, 1], [257, 0, 0]):
        with pytest.raises(ValueError):
            run.advance(counts)
    for parents in ([0, 1], [0, 1, 3], [0, 1, -2]):
        with pytest.raises(ValueError):
            run.fork(parents)
    assert run.lens == [-1, -1, -1]
