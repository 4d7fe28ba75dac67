"""Rows of the 4-bit cache that hold a NaN or an infinity: nothing finite is read back for them, and no other row changes."""
import pytest
import torch

from paper_2407_07304_b200 import binding as slim
from test_cache4 import D, filled, i32, rows

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def held(cache, n):
    k, v = (torch.zeros((n, cache.Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slim.slim_kv4_read(cache, k, v, i32([0, n]), i32([0]), 1, n)
    return k, v


@pytest.mark.parametrize("bad,at", [(NAN, 0), (NAN, 5), (NAN, 63), (NAN, 64), (NAN, 127), (-NAN, 70), (INF, 3), (-INF, 100)])
@pytest.mark.parametrize("step", [False, True], ids=["append", "step"])
def test_a_row_with_a_bad_value(bad, at, step):
    gen = torch.Generator().manual_seed(at)
    n, hkv, row = 70, 2, 69 if step else 40
    one, two = (slim.SlimCache4(1, hkv, 1) for _ in range(2))
    k, v = rows(gen, n, hkv).cuda(), rows(gen, n, hkv).cuda()
    bad_k, bad_v = k.clone(), v.clone()
    bad_k[row, 1, at] = bad
    bad_v[row, 0, at] = bad
    q = torch.randn(1, 4, D, generator=gen).to(torch.bfloat16).cuda()
    ws, out, want = slim.decode4_workspace(1, 4, hkv, n), torch.empty_like(q), torch.empty_like(q)
    for cache, x, y, o in ((one, bad_k, bad_v, out), (two, k, v, want)):
        if step:
            slim.slim_kv4_append(cache, x, y, i32([0, n - 1]), i32([0]), 1, n - 1)
            slim.slim_attn4_decode(cache, q, o, i32([n]), 1, n, 4, D ** -0.5, ws, k_new=x[-1:].contiguous(), v_new=y[-1:].contiguous())
        else:
            slim.slim_kv4_append(cache, x, y, i32([0, n]), i32([0]), 1, n)
            slim.slim_attn4_decode(cache, q, o, i32([n]), 1, n, 4, D ** -0.5, ws)
    good = held(two, n)
    for kind, (got, ref) in enumerate(zip(held(one, n), good)):
        head = 1 - kind
        assert not got[row, head].isfinite().any()
        ref[row, head] = got[row, head] = 0
        assert torch.equal(got, ref)
    # (queries 0 and 1 read the kv head whose V row is bad, 2 and 3 the one whose K row is)
    assert not out.isfinite().any() and want.isfinite().all()


def test_the_other_sequences_keep_their_results():
    gen = torch.Generator().manual_seed(2)
    lens, hq, hkv = [200, 65, 130], 8, 2
    cache, k, v = filled(gen, lens, hkv)
    q = torch.randn(3, hq, D, generator=gen).to(torch.bfloat16).cuda()
    ws, want, out = slim.decode4_workspace(3, hq, hkv, 200), torch.empty_like(q), torch.empty_like(q)
    slim.slim_attn4_decode(cache, q, want, i32(lens), 3, 200, hq, D ** -0.5, ws)
    k, v = k.clone(), v.clone()
    v[200 + 30, 1, 77] = NAN
    slim.slim_kv4_append(cache, k.cuda(), v.cuda(), i32([0, 200, 265, 395]), i32([0, 0, 0]), 3, 200)
    slim.slim_attn4_decode(cache, q, out, i32(lens), 3, 200, hq, D ** -0.5, ws)
    assert out[1, 4:].isnan().all()
    out[1, 4:] = want[1, 4:]
    assert torch.equal(out, want)


def test_a_bad_row_behind_the_last_token_is_not_seen():
    """A token that was cut off again may hold anything, in either direction of the attention."""
    gen = torch.Generator().manual_seed(3)
    n, hq, hkv = 150, 8, 2
    cache, k, v = filled(gen, [n], hkv)
    q = torch.randn(20, hq, D, generator=gen).to(torch.bfloat16).cuda()
    ws, wp = slim.decode4_workspace(1, hq, hkv, n), slim.workspace(slim.PHASE_PREFILL, 1, hq, hkv, 20, n)
    results = []
    for bad in (False, True):
        if bad:
            k, v = k.clone(), v.clone()
            k[140, 0, 3], v[141, 1, 90] = NAN, INF
            slim.slim_kv4_append(cache, k.cuda(), v.cuda(), i32([0, n]), i32([0]), 1, n)
        one, many = torch.empty_like(q[:1]), torch.empty_like(q)
        slim.slim_attn4_decode(cache, q[:1].contiguous(), one, i32([140]), 1, n, hq, D ** -0.5, ws)
        slim.slim_attn4_prefill(cache, q, many, i32([0, 20]), i32([140]), 1, 20, n, hq, D ** -0.5, wp)
        results.append((one, many))
    assert all(torch.equal(a, b) and a.isfinite().all() for a, b in zip(*results))
