"""What the binding of the 4-bit cache refuses because a kernel would read or write past it.

No GPU: the refusals come before any launch, and so do those of tensors that lie in host memory."""
import pytest
import torch

from paper_2407_07304_b200 import binding as slim


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def rows(*shape):
    return torch.zeros((*shape, 128), dtype=torch.bfloat16)


B, HQ, HKV, TOKENS = 3, 4, 2, 5
GOOD = dict(k=(TOKENS, HKV), v=(TOKENS, HKV), q=(TOKENS, HQ), out=(TOKENS, HQ), cu=B + 1, lens=B, dtype=torch.int32, rows=B, B=B)


def call(name, **kw):
    f = dict(GOOD)
    f.update(kw)
    cache = slim.SlimCache4(f["rows"], HKV, 2, device="cpu")
    k, v, q, out = (rows(*f[n]) for n in ("k", "v", "q", "out"))
    cu, lens = i32(f["cu"]).to(f["dtype"]), i32(f["lens"]).to(f["dtype"])
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    if name in ("slim_kv4_append", "slim_kv4_read"):
        getattr(slim, name)(cache, k, v, cu, lens, f["B"], 2)
    elif name == "slim_attn4_prefill":
        slim.slim_attn4_prefill(cache, q, out, cu, lens, f["B"], 2, 256, HQ, 0.1, ws)
    elif name == "slim_prefill4_step":
        slim.slim_prefill4_step(cache, q, k, v, out, cu, lens, f["B"], 2, 256, HQ, 0.1, ws)
    elif name == "slim_attn4_decode":
        slim.slim_attn4_decode(cache, q, out, lens, f["B"], 256, HQ, 0.1, ws)
    else:
        slim.slim_attn4_decode(cache, q, out, lens, f["B"], 256, HQ, 0.1, ws, k_new=k, v_new=v)


APPEND, READ, PREFILL, PREFILL_STEP, DECODE, STEP = "slim_kv4_append", "slim_kv4_read", "slim_attn4_prefill", "slim_prefill4_step", "slim_attn4_decode", "step"
EVERY = [APPEND, READ, PREFILL, PREFILL_STEP, DECODE, STEP]


@pytest.mark.parametrize("name,kw,says", [
    *[(n, dict(rows=B - 1), "block table") for n in EVERY],
    *[(n, dict(lens=B - 1), "lengths") for n in EVERY],
    *[(n, dict(dtype=torch.int64), "lengths") for n in EVERY],
    *[(n, dict(cu=B), "lengths") for n in (APPEND, READ, PREFILL, PREFILL_STEP)],
    *[(n, dict(v=(TOKENS - 1, HKV)), "rows must") for n in (APPEND, READ, PREFILL_STEP, STEP)],
    *[(n, dict(k=(TOKENS, HKV + 1), v=(TOKENS, HKV + 1)), "rows must") for n in (APPEND, READ, PREFILL_STEP, STEP)],
    *[(n, dict(out=(TOKENS - 1, HQ)), "q and out") for n in (PREFILL, PREFILL_STEP, DECODE, STEP)],
    *[(n, dict(q=(B - 1, HQ), out=(B - 1, HQ)), "q and out") for n in (DECODE, STEP)],
    (PREFILL_STEP, dict(k=(TOKENS - 1, HKV), v=(TOKENS - 1, HKV)), "rows must"),
    (STEP, dict(k=(B - 1, HKV), v=(B - 1, HKV)), "rows must"),
])
def test_too_small(name, kw, says):
    with pytest.raises(slim.SlimError, match=says) as e:
        call(name, **kw)
    assert e.value.code == slim.SLIM_ERR_INVALID_ARG


@pytest.mark.parametrize("name", EVERY)
def test_host_memory(name):
    """Sizes that fit: what is left to refuse is that no GPU can read any of it."""
    with pytest.raises(slim.SlimError, match="not a GPU's"):
        call(name)


def test_a_smaller_table_goes_with_a_smaller_batch():
    cache = slim.SlimCache4(B, HKV, 2, device="cpu")
    cache.set_block_table(i32(B - 1, 4))
    with pytest.raises(slim.SlimError, match="block table"):
        slim.slim_attn4_decode(cache, rows(B, HQ), rows(B, HQ), i32(B), B, 256, HQ, 0.1, torch.zeros(1 << 20, dtype=torch.uint8))
    with pytest.raises(TypeError):
        slim.SlimCache4(B, HKV, 2, device="cpu", block_table=i32(B, 3))


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["k", "v", "q", "out", "cu", "lens", "ws"])
def test_one_tensor_on_the_host(which):
    where = lambda n, t: t if n == which else t.cuda()  # noqa: E731
    cache = slim.SlimCache4(B, HKV, 2)
    k, v, q, out = (where(n, rows(*GOOD[n])) for n in ("k", "v", "q", "out"))
    cu, lens, ws = where("cu", i32(B + 1)), where("lens", i32(B)), where("ws", torch.zeros(1 << 20, dtype=torch.uint8))
    calls = [(("k", "v", "cu", "lens"), lambda: slim.slim_kv4_append(cache, k, v, cu, lens, B, 2)),
             (("k", "v", "cu", "lens"), lambda: slim.slim_kv4_read(cache, k, v, cu, lens, B, 2)),
             (("q", "out", "cu", "lens", "ws"), lambda: slim.slim_attn4_prefill(cache, q, out, cu, lens, B, 2, 256, HQ, 0.1, ws)),
             (("k", "v", "q", "out", "cu", "lens", "ws"), lambda: slim.slim_prefill4_step(cache, q, k, v, out, cu, lens, B, 2, 256, HQ, 0.1, ws)),
             (("q", "out", "lens", "ws"), lambda: slim.slim_attn4_decode(cache, q, out, lens, B, 256, HQ, 0.1, ws)),
             (("k", "v", "q", "out", "lens", "ws"), lambda: slim.slim_attn4_decode(cache, q, out, lens, B, 256, HQ, 0.1, ws, k_new=k, v_new=v))]
    for takes, fn in calls:
        if which in takes:
            with pytest.raises(slim.SlimError, match="device"):
                fn()
        else:
            fn()


WS = torch.zeros(1 << 20, dtype=torch.uint8)
ONE, LENS = rows(B, HQ), i32(B)
INT8 = {
    "slim_kv_append": lambda c: slim.slim_kv_append(c, rows(B, HKV), rows(B, HKV), i32(B + 1), LENS, B, 1, STREAM),
    "slim_attn_prefill": lambda c: slim.slim_attn_prefill(c, ONE, ONE, i32(B + 1), LENS, B, 1, 256, HQ, 0.1, WS, STREAM),
    "slim_prefill_step": lambda c: slim.slim_prefill_step(c, ONE, rows(B, HKV), rows(B, HKV), ONE, i32(B + 1), LENS, B, 1, 256, HQ, 0.1, WS, STREAM),
    "slim_attn_prefill_two_pass": lambda c: slim.slim_attn_prefill_two_pass(c, ONE, ONE, i32(B + 1), LENS, B, 1, 256, HQ, 0.1, WS, STREAM),
    "slim_attn_prefill_full_row": lambda c: slim.slim_attn_prefill_full_row(c, ONE, ONE, i32(B + 1), LENS, B, 1, 256, HQ, 0.1, WS, STREAM),
    "slim_attn_decode": lambda c: slim.slim_attn_decode(c, ONE, ONE, LENS, B, 256, HQ, 0.1, WS, STREAM),
    "slim_attn_decode_split": lambda c: slim.slim_attn_decode_split(c, ONE, LENS, B, 256, HQ, 0.1, WS, STREAM),
    "slim_attn_decode_static": lambda c: slim.slim_attn_decode_static(c, ONE, ONE, LENS, B, 256, HQ, 0.1, STREAM),
    "slim_attn_decode_partial": lambda c: slim.slim_attn_decode_partial(c, ONE, WS, LENS, B, 256, HQ, 0.1, WS, STREAM),
    "slim_decode_step": lambda c: slim.slim_decode_step(c, ONE, rows(B, HKV), rows(B, HKV), ONE, LENS, B, 256, HQ, 0.1, WS, STREAM),
}


class STREAM:
    cuda_stream = 0


@pytest.mark.parametrize("name", INT8)
def test_int8_calls_on_a_smaller_table(name):
    cache = slim.SlimCache(B, HKV, 2, device="cpu")
    cache.set_block_table(i32(B - 1, 2))
    with pytest.raises(slim.SlimError, match="block table") as e:
        INT8[name](cache)
    assert e.value.code == slim.SLIM_ERR_INVALID_ARG
