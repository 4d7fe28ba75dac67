"""Arguments that the norm-and-rotation, shared-prefix, weighted-decode and eviction calls refuse, before any launch.

No GPU: every call here is answered by the host's checks.  The addresses are never followed."""
import ctypes

import pytest

from paper_2407_07304_b200 import binding as slim

A = 1 << 20        # an aligned address that nothing reads


def cache(**kw):
    f = dict(codes=A, scales=A, block_table=A, num_pages=8, page_tokens=128, num_kv_heads=2, head_dim=128, max_pages_per_seq=4)
    f.update(kw)
    return slim.SlimCacheStruct(*[f[n] for n, _ in slim.SlimCacheStruct._fields_])


def rope(**kw):
    f = dict(inv_freq=A, axis=None, q_weight=A, k_weight=A, eps=1e-6, rotary_dim=128, n_axes=1, interleaved=0)
    f.update(kw)
    return slim.SlimNormRopeStruct(*[f[n] for n, _ in slim.SlimNormRopeStruct._fields_])


INVALID, UNSUPPORTED, WORKSPACE, OK = (slim.SLIM_ERR_INVALID_ARG, slim.SLIM_ERR_UNSUPPORTED, slim.SLIM_ERR_WORKSPACE, slim.SLIM_OK)

ROPE_FIELDS = [
    (dict(rotary_dim=-16), INVALID), (dict(rotary_dim=144), UNSUPPORTED), (dict(rotary_dim=24), UNSUPPORTED), (dict(n_axes=0), INVALID),
    (dict(n_axes=5, axis=A), UNSUPPORTED), (dict(n_axes=2, axis=None), INVALID), (dict(inv_freq=None), INVALID), (dict(inv_freq=A + 4), INVALID),
    (dict(q_weight=A + 2), INVALID), (dict(k_weight=A + 8), INVALID), (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
]


def call_norm_rope(r=None, **kw):
    f = dict(nr=ctypes.byref(r if r is not None else rope()), q=A, qs=4 * 128, qo=A, k=A, ks=2 * 128, ko=A, pos=A, n=3, hq=4, hkv=2)
    f.update(kw)
    return slim.lib().slim_norm_rope(f["nr"], f["q"], f["qs"], f["qo"], f["k"], f["ks"], f["ko"], f["pos"], f["n"], f["hq"], f["hkv"], None)


@pytest.mark.parametrize("fields,want", ROPE_FIELDS)
def test_norm_rope_refuses_fields(fields, want):
    assert call_norm_rope(rope(**fields)) == want
    assert call_append(r=rope(**fields)) == want


@pytest.mark.parametrize("kw,want", [
    (dict(nr=None), INVALID), (dict(q=None), INVALID), (dict(q=A + 8), INVALID), (dict(qs=3 * 128), INVALID), (dict(qs=516), INVALID),
    (dict(qo=None), INVALID), (dict(qo=A + 2), INVALID), (dict(k=None), INVALID), (dict(ks=128), INVALID), (dict(ko=None), INVALID),
    (dict(pos=None), INVALID), (dict(n=-1), INVALID), (dict(hq=-1), INVALID), (dict(hq=0, hkv=0), INVALID), (dict(n=0, q=None), OK),
    (dict(n=1 << 26, hq=64, qs=64 * 128), UNSUPPORTED),
])
def test_norm_rope_refuses_arguments(kw, want):
    assert call_norm_rope(**kw) == want


def call_append(r=None, c=None, **kw):
    f = dict(q=A, qs=4 * 128, qo=A, k=A, ks=2 * 128, v=A, vs=2 * 128, pos=A, cu=A, start=A, B=2, n=3, hq=4)
    f.update(kw)
    return slim.lib().slim_norm_rope_append(ctypes.byref(c if c is not None else cache()), ctypes.byref(r if r is not None else rope()), f["q"], f["qs"],
                                            f["qo"], f["k"], f["ks"], f["v"], f["vs"], f["pos"], f["cu"], f["start"], f["B"], f["n"], f["hq"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), INVALID), (dict(qo=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(vs=128), INVALID), (dict(v=A + 8), INVALID),
    (dict(cu=None), INVALID), (dict(start=None), INVALID), (dict(B=-1), INVALID), (dict(B=65536), UNSUPPORTED), (dict(n=-1), INVALID), (dict(B=0), OK),
    (dict(n=0), OK), (dict(c=cache(page_tokens=64)), UNSUPPORTED), (dict(c=cache(codes=A + 8)), INVALID), (dict(c=cache(block_table=None)), INVALID),
])
def test_norm_rope_append_refuses(kw, want):
    assert call_append(**kw) == want


def call_shared(c=None, **kw):
    f = dict(q=A, k=None, v=None, out=A, cu=A, sh=A, kv=A, g=1, B=2, mg=2, ms=256, mt=128, hq=4, ws=A, n=1 << 30)
    f.update(kw)
    return slim.lib().slim_attn_decode_shared(ctypes.byref(c if c is not None else cache()), f["q"], f["k"], f["v"], f["out"], f["cu"], f["sh"], f["kv"],
                                              f["g"], f["B"], f["mg"], f["ms"], f["mt"], f["hq"], 0.1, f["ws"], f["n"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(out=A + 8), INVALID), (dict(cu=None), INVALID), (dict(sh=None), INVALID),
    (dict(kv=None), INVALID), (dict(k=A), INVALID), (dict(k=A, v=A + 8), INVALID), (dict(g=0), INVALID), (dict(g=65536), UNSUPPORTED),
    (dict(mg=0), INVALID), (dict(mg=3), INVALID), (dict(ms=-1), INVALID), (dict(ms=513), INVALID), (dict(mt=513), INVALID), (dict(hq=5), UNSUPPORTED),
    (dict(hq=34), UNSUPPORTED), (dict(B=-1), INVALID), (dict(B=0), OK), (dict(ws=None), WORKSPACE), (dict(n=1000), WORKSPACE), (dict(ws=A + 8), INVALID),
    (dict(c=cache(head_dim=64)), UNSUPPORTED),
])
def test_shared_refuses(kw, want):
    assert call_shared(**kw) == want


def call_weights(c=None, **kw):
    f = dict(q=A, k=None, v=None, out=A, wi=A, wo=A, stride=512, seen=A, kv=A, B=2, mk=512, hq=4, ws=A, n=1 << 30)
    f.update(kw)
    return slim.lib().slim_attn_decode_weights(ctypes.byref(c if c is not None else cache()), f["q"], f["k"], f["v"], f["out"], f["wi"], f["wo"], f["stride"],
                                               f["seen"], f["kv"], f["B"], f["mk"], f["hq"], 0.1, 1.0, f["ws"], f["n"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(wo=None), INVALID), (dict(wo=A + 2), INVALID), (dict(stride=511), INVALID),
    (dict(kv=None), INVALID), (dict(v=A), INVALID), (dict(mk=513, stride=513), INVALID), (dict(mk=-1), INVALID), (dict(hq=33), UNSUPPORTED),
    (dict(B=0), OK), (dict(ws=None), WORKSPACE), (dict(n=70000), WORKSPACE), (dict(q=A + 8), INVALID),
])
def test_weights_refuses(kw, want):
    assert call_weights(**kw) == want


def call_evict(c=None, **kw):
    f = dict(wi=A, wo=A, pi=A, po=A, stride=512, kv=A, placed=A, seen=A, B=2, mk=512, budget=256, sink=4, recent=32, ws=A, n=1 << 30)
    f.update(kw)
    return slim.lib().slim_kv_evict(ctypes.byref(c if c is not None else cache()), f["wi"], f["wo"], f["pi"], f["po"], f["stride"], f["kv"], f["placed"],
                                    f["seen"], f["B"], f["mk"], f["budget"], f["sink"], f["recent"], f["ws"], f["n"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(wi=None), INVALID), (dict(wo=None), INVALID), (dict(po=None), INVALID), (dict(pi=None), INVALID), (dict(kv=None), INVALID),
    (dict(stride=511), INVALID), (dict(budget=0), INVALID), (dict(sink=-1), INVALID), (dict(recent=-1), INVALID), (dict(sink=200, recent=57), INVALID),
    (dict(sink=1 << 30, recent=(1 << 31) - 1), INVALID), (dict(mk=513, stride=513), INVALID), (dict(B=65536), UNSUPPORTED), (dict(B=0), OK),
    (dict(mk=0), OK), (dict(ws=None), WORKSPACE), (dict(n=100), WORKSPACE), (dict(ws=A + 4), INVALID), (dict(wi=A + 1), INVALID),
    (dict(c=cache(num_pages=0)), INVALID),
])
def test_evict_refuses(kw, want):
    assert call_evict(**kw) == want


def test_workspace_sizes():
    L = slim.lib()
    assert L.slim_shared_workspace_bytes(0, 4, 2, 1, 1, 128, 1) == 0 and L.slim_shared_workspace_bytes(2, 5, 2, 1, 2, 128, 1) == 0
    # without a prefix of a page the call is ordinary decode, and so is its workspace
    assert L.slim_shared_workspace_bytes(3, 8, 2, 1, 3, 127, 700) == slim.slim_workspace_bytes(slim.PHASE_DECODE, 3, 8, 2, 1, 700)
    assert L.slim_shared_workspace_bytes(3, 8, 2, 1, 3, 128, 700) > L.slim_shared_workspace_bytes(3, 8, 2, 1, 3, 0, 700)
    # the scores: 4 bytes per query head and token, rounded up to whole chunks
    base = slim.slim_workspace_bytes(slim.PHASE_DECODE, 3, 8, 2, 1, 700)
    assert 3 * 8 * 768 * 4 <= L.slim_weights_workspace_bytes(3, 8, 2, 700) - base < 3 * 8 * 768 * 4 + 256
    # three lists per (sequence, kv head): never more than the budget, nor than what is cut
    assert L.slim_evict_workspace_bytes(2, 3, 1000, 990) == 2 * 3 * (1 + 3 * 10) * 4
    assert L.slim_evict_workspace_bytes(2, 3, 1000, 10) == 2 * 3 * (1 + 3 * 10) * 4
    assert L.slim_evict_workspace_bytes(2, 3, 10, 1000) == 2 * 3 * 4


def test_binding_refuses_tensors():
    import torch
    f = torch.ones(64, dtype=torch.float64)
    with pytest.raises(TypeError):
        slim.NormRope(f.float())
    with pytest.raises(TypeError):
        slim.NormRope(f, axis=torch.zeros(63, dtype=torch.uint8))
    with pytest.raises(TypeError):
        slim.NormRope(f, q_weight=torch.ones(128))
    with pytest.raises(TypeError):
        slim.NormRope(f, q_weight=torch.ones((128, 2), dtype=torch.bfloat16)[:, 0])
    nr = slim.NormRope(f)
    pos = torch.zeros(3, dtype=torch.int32)
    q = torch.zeros((3, 4, 128), dtype=torch.bfloat16)
    for bad_q, out in ((q.float(), q), (q[..., ::2], q), (q.transpose(0, 1), q), (q, q[:2]), (q, q.half()), (torch.zeros((3, 4, 64), dtype=torch.bfloat16), q)):
        with pytest.raises(slim.SlimError) as e:
            slim.slim_norm_rope(nr, bad_q, out, None, None, pos, stream=_NoStream)
        assert e.value.code == INVALID
    with pytest.raises(slim.SlimError):
        slim.slim_norm_rope(nr, q, q, None, None, pos.long(), stream=_NoStream)
    with pytest.raises(slim.SlimError):
        slim.slim_norm_rope(nr, q, q, q[:2], q[:2], pos, stream=_NoStream)


def test_binding_refuses_weights_and_positions():
    """One stride serves all of a call's arrays, so they must be of one shape."""
    import torch
    c = slim.SlimCache(2, 4, 2, device="cpu")
    w, pos, lens = torch.zeros((2, 4, 256)), torch.zeros((2, 4, 256), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    evict = lambda wi, wo, pi, po, B=2: slim.slim_kv_evict(c, wi, wo, pi, po, lens, lens, lens, B, 256, 128, 0, 0, None, stream=_NoStream)  # noqa: E731
    weigh = lambda wi, wo, B=2: slim.slim_attn_decode_weights(c, w, w, wi, wo, None, lens, B, 256, 4, 1.0, 1.0, None, stream=_NoStream)  # noqa: E731
    for wi, wo, pi, po in ((w.half(), w, pos, pos), (w, w.double(), pos, pos), (w, w, pos.long(), pos), (w, w, pos, pos[..., :255]), (w[..., :128], w, pos, pos),
                           (w, w, pos[:, :2], pos), (w, w.transpose(0, 1), pos, pos), (w, w.view(-1), pos, pos), (w.expand(2, 4, 256)[..., :1].expand(2, 4, 256), w, pos, pos)):
        with pytest.raises(slim.SlimError) as e:
            evict(wi, wo, pi, po)
        assert e.value.code == INVALID
    for wi, wo in ((w.half(), w), (None, w.double()), (w[..., :128], w), (None, w[:, :2]), (None, w[..., ::2])):
        with pytest.raises(slim.SlimError) as e:
            weigh(wi, wo)
        assert e.value.code == INVALID
    for call in (lambda: evict(w, w, pos, pos, B=3), lambda: weigh(w, w, B=3)):
        with pytest.raises(slim.SlimError) as e:
            call()
        assert e.value.code == INVALID


class _NoStream:
    cuda_stream = 0
