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
