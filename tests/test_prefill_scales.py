"""Prefill with softmax scales of either sign and of zero, over both caches, against fp64 attention over the values held."""
import numpy as np
import pytest
import torch

from helpers import MAX_ABS, MEAN_ABS, dense_attention
from paper_2407_07304_b200 import binding as slim
from test_cache4 import D, PAGE, close, filled, i32, offsets, reference

pytestmark = pytest.mark.gpu
SCALES = [-D ** -0.5, 0.0, -0.0, -1e-4]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("hq,hkv", [(2, 2), (6, 2), (16, 1)])
def test_four_bits(hq, hkv, scale):
    """The bound is that of test_cache4's prefill (see there), with the scale's size."""
    gen = torch.Generator().manual_seed(hq)
    counts, lens = [130, 1, 260], [130, 200, 300]
    cache, _, _ = filled(gen, lens, hkv)
    q = torch.randn(sum(counts), hq, D, generator=gen).to(torch.bfloat16).cuda()
    out, cu = torch.empty_like(q), offsets(counts)
    ws = slim.workspace(slim.PHASE_PREFILL, 3, hq, hkv, 260, 300)
    slim.slim_attn4_prefill(cache, q, out, i32(cu), i32(lens), 3, 260, 300, hq, scale, ws)
    for b, (m, n) in enumerate(zip(counts, lens)):
        at = slice(cu[b], cu[b + 1])
        want, parts = reference(cache, b, n, q[at], scale, n - m + np.arange(m))
        _, score, v, _ = (np.abs(x)[..., None] for x in parts)
        close(out[at], want, 2.0 ** -8 * np.abs(want) + (2 * score + 2 * 2.0 ** -11 + n * 2.0 ** -25 + 2.0 ** -20) * v)


def test_four_bits_decode_and_prefill_agree():
    gen = torch.Generator().manual_seed(8)
    n, hq, hkv, scale = 300, 8, 2, -0.1
    cache, _, _ = filled(gen, [n], hkv)
    q = torch.randn(1, hq, D, generator=gen).to(torch.bfloat16).cuda()
    one, two = torch.empty_like(q), torch.empty_like(q)
    slim.slim_attn4_decode(cache, q, one, i32([n]), 1, n, hq, scale, slim.decode4_workspace(1, hq, hkv, n))
    slim.slim_attn4_prefill(cache, q, two, i32([0, 1]), i32([n]), 1, 1, n, hq, scale, slim.workspace(slim.PHASE_PREFILL, 1, hq, hkv, 1, n))
    want, parts = reference(cache, 0, n, q, scale)
    dec, pre, v, s = (np.abs(x)[..., None] for x in parts)
    close(one, want, 2.0 ** -8 * np.abs(want) + 2.0 ** -11 * 15 * s + (2 * dec + 2.0 ** -20) * v)
    close(two, want, 2.0 ** -8 * np.abs(want) + (2 * pre + 2 * 2.0 ** -11 + n * 2.0 ** -25 + 2.0 ** -20) * v)


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("form", ["slim_attn_prefill", "slim_attn_prefill_two_pass"])
def test_int8(form, scale):
    check_int8(form, scale, 300)


def check_int8(form, scale, n):
    gen = torch.Generator().manual_seed(4)
    hq, hkv = 4, 2
    cache = slim.SlimCache(1, hkv, (n + PAGE - 1) // PAGE)
    k, v = (torch.randn(n, hkv, D, generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    slim.slim_kv_append(cache, k, v, i32([0, n]), i32([0]), 1, n)
    q = torch.randn(n, hq, D, generator=gen).to(torch.bfloat16).cuda()
    out = torch.empty_like(q)
    getattr(slim, form)(cache, q, out, i32([0, n]), i32([n]), 1, n, n, hq, scale, slim.workspace(slim.PHASE_PREFILL, 1, hq, hkv, n, n))
    codes = cache.codes_view().permute(2, 0, 3, 1, 4).reshape(2, -1, hkv, D)[:, :n].double().cpu().numpy()
    scales = cache.scales_view().permute(2, 0, 3, 1).reshape(2, -1, hkv)[:, :n].double().cpu().numpy()
    held = codes * scales[..., None]
    err = np.abs(out.double().cpu().numpy() - dense_attention(q.double().cpu().numpy(), held[0], held[1], n, scale))
    assert err.max() <= MAX_ABS and err.mean() <= MEAN_ABS, f"max {err.max():.3e}, mean {err.mean():.3e}"


@pytest.mark.parametrize("scale", SCALES)
def test_int8_full_row(scale):
    check_int8("slim_attn_prefill_full_row", scale, 250)


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("hq,hkv", [(2, 2), (16, 2)])
def test_int8_decode(hq, hkv, scale):
    """Decode takes the same scales."""
    gen = torch.Generator().manual_seed(6)
    n = 700
    cache = slim.SlimCache(1, hkv, 6)
    k, v = (torch.randn(n, hkv, D, generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    slim.slim_kv_append(cache, k, v, i32([0, n]), i32([0]), 1, n)
    q = torch.randn(1, hq, D, generator=gen).to(torch.bfloat16).cuda()
    out = torch.empty_like(q)
    slim.slim_attn_decode(cache, q, out, i32([n]), 1, n, hq, scale, slim.workspace(slim.PHASE_DECODE, 1, hq, hkv, 1, n))
    codes = cache.codes_view().permute(2, 0, 3, 1, 4).reshape(2, -1, hkv, D)[:, :n].double().cpu().numpy()
    held = codes * cache.scales_view().permute(2, 0, 3, 1).reshape(2, -1, hkv)[:, :n].double().cpu().numpy()[..., None]
    err = np.abs(out.double().cpu().numpy() - dense_attention(q.double().cpu().numpy(), held[0], held[1], n, scale))
    assert err.max() <= MAX_ABS and err.mean() <= MEAN_ABS, f"max {err.max():.3e}, mean {err.mean():.3e}"
