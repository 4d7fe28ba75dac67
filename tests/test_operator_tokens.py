"""Shared-prefix and weighted decode where single tokens, and large scores, decide the result."""
import pytest
import torch

from test_operators import D, PAGE, attend, fill, gen, i32, rows_of, shared_setup

pytestmark = pytest.mark.gpu


def _slim():
    from paper_2407_07304_b200 import binding
    return binding


def rms_close(out, want, what, times=1.25):
    """Every sequence's root mean square error over its heads, against that of the exact result rounded to bf16 (1.65e-3 of the
    result's).  The kernel's own roundings are three of fp16 per term (P, V's scale, V), half a step 2^-11 each, independent
    from term to term like the terms themselves: at most 3^0.5 2^-11 = 0.85e-3 of the result's, so together
    (1.65^2 + 0.85^2)^0.5 / 1.65 = 1.13 times the rounding's; 1.25 leaves room for 1024 elements' scatter (1 / 2048^0.5 each)."""
    err = (out.double() - want).flatten(1).norm(dim=1)
    best = (want.to(torch.bfloat16).double() - want).flatten(1).norm(dim=1)
    assert torch.isfinite(out.float()).all(), what
    assert (err <= times * best + 1e-30).all(), f"{what}: {(err / (best + 1e-30)).max().item():.3f} times the rounding's error"


@pytest.mark.parametrize("hq,hkv,n", [(16, 2, 4), (16, 1, 20), (32, 32, 16)])
@pytest.mark.parametrize("offset", [40.0, 400.0, 4000.0])
def test_decode_shared_scores_with_a_large_common_part(hq, hkv, n, offset):
    """Keys whose rows share one large component, and queries that meet it: scores of `offset` that differ by a few units, as the
    keys' scales do.  A key rounded to fp16 (2^-11 of its large component) would move a score of 400 by up to 0.1."""
    slim = _slim()
    cache, B, cu = shared_setup(n, [(12, n)], hq, hkv, 2)
    codes, scales = cache.codes_view(), cache.scales_view()
    codes[:, :, 0, :, 5] = 127
    scales[:, :, 0] = 0.5 + torch.rand(scales[:, :, 0].shape, generator=gen(6)).cuda() * 4.0 / offset   # scores spread over eight units
    q = (torch.randn((B, hq, D), generator=gen(n)) * 0.02).to(torch.bfloat16).cuda()
    q[..., 5] = offset / (127 * 0.5 * D ** -0.5)
    lens = [12 * PAGE + 3 + b for b in range(B)]
    out, ref = torch.empty_like(q), torch.empty_like(q)
    ws = slim.shared_workspace(B, hq, hkv, 1, B, 12 * PAGE, 64)
    slim.slim_attn_decode_shared(cache, q, out, i32(cu), i32([12 * PAGE] * B), i32(lens), 1, B, B, 12 * PAGE, 64, hq, D ** -0.5, ws)
    slim.slim_attn_decode(cache, q, ref, i32(lens), B, max(lens), hq, D ** -0.5, slim.workspace(slim.PHASE_DECODE, B, hq, hkv, 1, max(lens)))
    torch.cuda.synchronize()
    assert slim.slim_read_status(ws) == slim.SLIM_OK
    want, probs, _ = attend(cache, q, lens, D ** -0.5)
    assert max(p.max().item() for p in probs) < 0.2      # many tokens count
    # scores of s in log2 units are sums of fp32: 128 terms of one 2^-23 of them each where the sums are cut off, 2^-16 s, and
    # three roundings behind; a weight moves by as much, independently from token to token like the roundings above
    moved = 1.4427 * offset * (2.0 ** -16 + 3 * 2.0 ** -24)
    rms_close(ref, want, "decode", 1.25 * (1 + (moved / 1.65e-3) ** 2) ** 0.5)
    rms_close(out, want, "shared", 1.25 * (1 + (moved / 1.65e-3) ** 2) ** 0.5)


TOKEN_CASES = [
    # groups (prefix pages, sequences), hq, hkv, tails per sequence (cycled; negative: shorter than the prefix by that much)
    ([(1, 1)], 8, 1, [1]), ([(3, 4)], 16, 2, [1, 2, 256, 257]), ([(9, 40)], 16, 1, [3, 515, 128]), ([(12, 3), (0, 2), (5, 7)], 24, 3, [1, 129, 300]),
    ([(17, 16)], 8, 8, [0, 1, 255]), ([(4, 9)], 16, 2, [-1, -128, -200, -384, -511, 5]), ([(2, 33)], 28, 4, [-255, 1, 128, -129]),
    ([(25, 5)], 64, 4, [513, 700]), ([(2, 2)] * 9, 32, 32, [3, 140]),
]


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("case", TOKEN_CASES, ids=range(len(TOKEN_CASES)))
def test_decode_shared_counts_every_token_once(case, append):
    """Nearly equal scores, so that every token holds about 1 / n of the result: one left out, or counted twice, at the borders of
    the prefix, its parts, pages and chunks moves the result by several times what the roundings may."""
    groups, hq, hkv, tails = case
    slim = _slim()
    cache, B, cu = shared_setup(hq + len(groups), groups, hq, hkv, max(0, max(tails)) // PAGE + 2)
    pre = [p * PAGE for p, n in groups for _ in range(n)]
    lens = [max(1, pre[b] + tails[b % len(tails)]) for b in range(B)]
    most, max_tail = max(n for _, n in groups), max(max(0, lens[b] - pre[b]) for b in range(B))
    q = (torch.randn((B, hq, D), generator=gen(B)) * 0.05).to(torch.bfloat16).cuda()
    out = torch.full_like(q, 5.0)
    new = {}
    if append:
        new = dict(k_new=torch.randn((B, hkv, D), generator=gen(1)).to(torch.bfloat16).cuda(), v_new=torch.randn((B, hkv, D), generator=gen(2)).to(torch.bfloat16).cuda())
    ws = slim.shared_workspace(B, hq, hkv, len(groups), most, max(pre), max_tail)
    slim.slim_attn_decode_shared(cache, q, out, i32(cu), i32(pre), i32(lens), len(groups), B, most, max(pre), max_tail, hq, D ** -0.5, ws, **new)
    torch.cuda.synchronize()
    assert slim.slim_read_status(ws) == slim.SLIM_OK
    want, probs, _ = attend(cache, q, lens, D ** -0.5)
    rms_close(out, want, case)
    # the check sees a single token: the exact result without it lies outside
    for b in range(0, B, max(1, B // 6)):
        best = (want[b].to(torch.bfloat16).double() - want[b]).norm()
        _, v = rows_of(cache, b, lens[b])
        for j in {0, 127, 128, 255, 256, pre[b] // 2 - 1, pre[b] // 2, pre[b] - 1, pre[b], pre[b] + 255, pre[b] + 256, lens[b] - 2, lens[b] - 1}:
            if 0 <= j < lens[b] and lens[b] > 1:
                p = probs[b][:, j, None]
                without = (want[b] - p * v[:, j].repeat_interleave(hq // hkv, 0)) / (1 - p)
                assert (without - want[b]).norm() > 3 * best, (b, j)


@pytest.mark.parametrize("lens,hq,hkv", [([1], 1, 1), ([2, 1, 257, 256, 300], 6, 3), ([272], 32, 32), ([2049, 1030, 128], 16, 2), ([9000, 33], 16, 1)])
def test_decode_weights_appends_like_the_other_calls(lens, hq, hkv):
    """With k_new and v_new: codes and scales those of slim_kv_append on a copy of the cache, the output slim_decode_step's, the
    weights those of a call without them over the copy."""
    slim = _slim()
    B, top = len(lens), max(lens)
    mp = (top + PAGE - 1) // PAGE
    table = torch.randperm(B * mp, generator=gen(top)).to(torch.int32).view(B, mp)
    caches = [slim.SlimCache(B, hkv, mp, block_table=table) for _ in range(3)]
    for c in caches:
        fill(c, hq)
    before = caches[0].codes.clone()
    g = gen(top + 1)
    q, kn, vn = (torch.randn((B, h, D), generator=g).to(torch.bfloat16).cuda() for h in (hq, hkv, hkv))
    kn[0, 0] *= 20                                          # a new key that takes weight
    out, step, plain = (torch.full_like(q, 5.0) for _ in range(3))
    w, w_ref = (torch.full((B, hkv, top), -3.0, device="cuda") for _ in range(2))
    n = i32(lens)
    slim.slim_attn_decode_weights(caches[0], q, out, None, w, None, n, B, top, hq, D ** -0.5, 1.0, slim.weights_workspace(B, hq, hkv, top), k_new=kn, v_new=vn)
    slim.slim_decode_step(caches[1], q, kn, vn, step, n, B, top, hq, D ** -0.5, slim.workspace(slim.PHASE_DECODE, B, hq, hkv, 1, top))
    slim.slim_kv_append(caches[2], kn, vn, i32(list(range(B + 1))), n - 1, B, 1)
    slim.slim_attn_decode_weights(caches[2], q, plain, None, w_ref, None, n, B, top, hq, D ** -0.5, 1.0, slim.weights_workspace(B, hq, hkv, top))
    torch.cuda.synchronize()
    assert not torch.equal(caches[0].codes, before)
    for c in caches[1:]:
        assert torch.equal(c.codes, caches[0].codes) and torch.equal(c.scales, caches[0].scales)
    assert torch.equal(out, step) and torch.equal(out, plain) and torch.equal(w, w_ref)
