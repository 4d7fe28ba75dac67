"""The 4-bit cache on a GPU: append, read-back, decode and prefill against plain implementations.

Codes, scales and offsets are compared bit for bit with the definition in numpy.  Attention is compared with fp64 softmax
attention over the values held.  Bounds (per sequence and head; all maxima over its keys and dims):
  output      half a bf16 step of the result: 2^-8 |o|
  decode      weights p s in fp16: 2^-11 each, at most 15 s times sum p = 1 in all; scores in fp32 from sums of |q| (15 s_k + |z_k|):
              2^-21 of that, twice (numerator and denominator), times the largest |v|
              (weights below 2^-14 lose at most 2^-25 each in prefill, of which there are n)
  prefill     keys, values and weights in fp16: a key's 2^-11 |k| shifts a score by at most 2^-11 sum |q k| (and fp16's smallest step,
              2^-24 of the tile's power of two, by 2^-24 max|k| sum |q|), values and weights 2^-11 of |v| each
A further 2^-20 max |v| covers exponentials and sums.
"""
import math

import numpy as np
import pytest
import torch

from paper_2407_07304_b200 import binding as slim

pytestmark = pytest.mark.gpu
PAGE, D = 128, 128


def rows(gen, *shape, spread=1.0):
    x = torch.randn(*shape, D, generator=gen)
    big = torch.rand(*shape[-1:], D, generator=gen).argsort(-1) < 3
    return (x * torch.where(big, 8.0, 1.0) * spread + 0.5).to(torch.bfloat16)


def define(x):
    """Codes [.., 128], scale and offset (fp32 values of bf16) of bf16 rows by the definition, every step in numpy fp32."""
    f = x.float().numpy()
    low, high = f.min(-1), f.max(-1)
    s = torch.from_numpy(((high - low) / np.float32(15)).astype(np.float32)).to(torch.bfloat16).float().numpy()
    with np.errstate(divide="ignore", invalid="ignore"):
        u = np.rint((f - low[..., None]) / s[..., None])
    return np.where(s[..., None] > 0, np.clip(u, 0, 15), 0).astype(np.uint8), s, low


def held_values(codes, s, z):
    return z[..., None].astype(np.float64) + codes.astype(np.float64) * s[..., None].astype(np.float64)


def unpack(cache, b, n):
    """Sequence b's first n rows as the cache holds them: codes [2, n, Hkv, 128], scale and offset [2, n, Hkv]."""
    pages = cache.block_table[b, :(n + PAGE - 1) // PAGE].long()
    c = cache.codes_view()[pages].permute(2, 0, 3, 1, 4).reshape(2, -1, cache.Hkv, D // 2)[:, :n].cpu().numpy()
    sz = cache.scales_view()[pages].permute(2, 0, 3, 1, 4).reshape(2, -1, cache.Hkv, 2)[:, :n].float().cpu().numpy()
    return np.concatenate([c & 15, c >> 4], -1), sz[..., 0], sz[..., 1]


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def offsets(counts):
    return np.concatenate([[0], np.cumsum(counts)]).tolist()


def filled(gen, lens, hkv, capacity=None, spread=1.0, extra_pages=3):
    """A cache whose sequences hold `lens` tokens on shuffled pages; what no token owns is 0xFF codes and NaN scales."""
    b, stride = len(lens), max(1, ((capacity or max(lens)) + PAGE - 1) // PAGE)
    pages = b * stride + extra_pages
    table = torch.randperm(pages, generator=gen)[:b * stride].view(b, stride).to(torch.int32)
    cache = slim.SlimCache4(b, hkv, stride, block_table=table, num_pages=pages)
    cache.codes.fill_(255)
    cache.scales.fill_(float("nan"))
    k, v = rows(gen, sum(lens), hkv, spread=spread), rows(gen, sum(lens), hkv, spread=spread)
    if sum(lens):
        slim.slim_kv4_append(cache, k.cuda(), v.cuda(), i32(offsets(lens)), i32([0] * b), b, max(lens))
    return cache, k, v


# ------------------------------------------------------------------------------------------------ append and read
@pytest.mark.parametrize("counts,start,hkv", [([1], [0], 1), ([1] * 16, [2047, 128, 127, 0] * 4, 32), ([5, 0, 130, 1], [126, 0, 127, 255], 5), ([300, 17], [0, 64], 8)])
def test_append_is_the_definition(counts, start, hkv):
    gen = torch.Generator().manual_seed(sum(counts) + hkv)
    b, stride = len(counts), (max(c + s for c, s in zip(counts, start)) + PAGE - 1) // PAGE + 1
    pages = b * stride + 2
    table = torch.randperm(pages, generator=gen)[:b * stride].view(b, stride).to(torch.int32)
    cache = slim.SlimCache4(b, hkv, stride, block_table=table, num_pages=pages)
    cache.codes.fill_(0xA5)
    before = cache.codes_view().clone()
    k, v = rows(gen, sum(counts), hkv), rows(gen, sum(counts), hkv)
    slim.slim_kv4_append(cache, k.cuda(), v.cuda(), i32(offsets(counts)), i32(start), b, max(counts))
    cu = offsets(counts)
    touched = torch.zeros(pages, PAGE, dtype=torch.bool)
    for i in range(b):
        codes, s, z = unpack(cache, i, start[i] + counts[i])
        for kv, x in enumerate((k, v)):
            want = define(x[cu[i]:cu[i + 1]])
            assert np.array_equal(codes[kv, start[i]:], want[0])
            assert np.array_equal(s[kv, start[i]:], want[1]) and np.array_equal(z[kv, start[i]:], want[2])
        for t in range(start[i], start[i] + counts[i]):
            touched[table[i, t // PAGE], t % PAGE] = True
    other = ~touched.cuda()
    assert torch.equal(cache.codes_view().permute(0, 3, 1, 2, 4)[other], before.permute(0, 3, 1, 2, 4)[other])
    # ---- and back
    k_back, v_back = torch.zeros_like(k).cuda(), torch.zeros_like(v).cuda()
    slim.slim_kv4_read(cache, k_back, v_back, i32(cu), i32(start), b, max(counts))
    for x, back in ((k, k_back), (v, v_back)):
        codes, s, z = define(x)
        want = (codes.astype(np.float32) * s[..., None] + z[..., None]).astype(np.float32)
        assert torch.equal(back.cpu(), torch.from_numpy(want).to(torch.bfloat16))


def test_append_of_odd_rows():
    """All zero, constant, one value apart, both signs' extremes, subnormal and huge rows; ties of the rounding."""
    x = torch.zeros(12, 1, D)
    x[1] = -3.5
    x[2, 0, 77] = 2.0
    x[3] = torch.linspace(-1, 1, D)
    x[4] = torch.arange(D) % 16                       # scale 1: exact
    x[5] = (torch.arange(D) % 31) / 2                 # ties at every second value
    x[6] = 2.0 ** -130 * (torch.arange(D) % 7)        # bf16 subnormals
    x[7] = 2.0 ** -133                                # the smallest subnormal, constant
    x[8] = 1e37 * torch.linspace(-1, 1, D)
    x[9] = 1000.0
    x[9, 0, 5] = 1008.0
    x[10] = 1e-25 * torch.linspace(3, 9, D)
    x[11, 0, :64] = -0.0
    x = x.to(torch.bfloat16)
    cache = slim.SlimCache4(1, 1, 1)
    slim.slim_kv4_append(cache, x.cuda(), x.cuda(), i32([0, 12]), i32([0]), 1, 12)
    codes, s, z = unpack(cache, 0, 12)
    want = define(x)
    for kv in (0, 1):
        assert np.array_equal(codes[kv], want[0]) and np.array_equal(s[kv], want[1]) and np.array_equal(z[kv], want[2])


def test_append_skips_what_is_outside():
    gen = torch.Generator().manual_seed(3)
    table = torch.tensor([[2, -1], [7, 1]], dtype=torch.int32)      # page -1, and page 7 of a pool of 4
    cache = slim.SlimCache4(2, 2, 2, block_table=table, num_pages=4)
    x = rows(gen, 400, 2).cuda()
    slim.slim_kv4_append(cache, x, x, i32([0, 200, 400]), i32([100, 100]), 2, 200)      # sequence 1 runs past its two pages
    used = cache.codes_view().flatten(1).any(1).tolist()
    assert used == [False, True, True, False]
    back = torch.full_like(x, 7.0)
    slim.slim_kv4_read(cache, back, back.clone(), i32([0, 200, 400]), i32([100, 100]), 2, 200)
    assert (back[28:200] == 7).all() and (back[200:228] == 7).all() and (back[356:] == 7).all() and not (back[:28] == 7).all(-1).any()


# ------------------------------------------------------------------------------------------------ decode
def reference(cache, b, n, q, scale, first_seen=None):
    """fp64 attention of q [rows, Hq, 128] over sequence b's n tokens, and the bound's parts [rows, Hq]: the score error of decode
    and of prefill, the largest |v|, the largest V scale."""
    codes, s, z = unpack(cache, b, n)
    k, v = held_values(codes[0], s[0], z[0]), held_values(codes[1], s[1], z[1])
    q = q.double().cpu().numpy()
    hq, group = q.shape[1], q.shape[1] // cache.Hkv
    out, parts = np.zeros(q.shape), np.zeros((4,) + q.shape[:2])
    for h in range(hq):
        g = h // group
        score = scale * (q[:, h] @ k[:, g].T)
        if first_seen is not None:
            score = np.where(np.arange(n)[None, :] <= first_seen[:, None], score, -np.inf)
        p = np.exp(score - score.max(1, keepdims=True))
        out[:, h] = (p / p.sum(1, keepdims=True)) @ v[:, g]
        size = np.abs(q[:, h])
        parts[0][:, h] = scale * size.sum(1) * (15 * s[0][:, g] + np.abs(z[0][:, g])).max() * 2.0 ** -21
        parts[1][:, h] = scale * ((size @ np.abs(k[:, g]).T).max(1) * 2.0 ** -11 + size.sum(1) * np.abs(k[:, g]).max() * 2.0 ** -24)
        parts[2][:, h], parts[3][:, h] = np.abs(v[:, g]).max(), s[1][:, g].max()
    return out, parts


def close(got, want, bound):
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.isfinite(err).all() and (err <= bound).all(), f"error {err.max():.3e}, {(err / bound).max():.2f} of the bound"


def decode_bound(want, parts):
    score, _, v, s = (x[..., None] for x in parts)
    return 2.0 ** -8 * np.abs(want) + 2.0 ** -11 * 15 * s + (2 * score + 2.0 ** -20) * v


def check_decode(cache, lens, q, out, scale):
    for b, n in enumerate(lens):
        if n <= 0:
            assert not out[b].any()
            continue
        want, parts = reference(cache, b, n, q[b:b + 1], scale)
        close(out[b:b + 1], want, decode_bound(want, parts))


LENGTHS = [[1], [0], [272], [64, 65, 0, 1, 63], [2, 15, 16, 17, 31, 33], [127, 128, 129, 255, 256, 257, 1], [1000, 3, 517], [4097]]
HEADS = [(1, 1), (2, 1), (3, 3), (14, 2), (8, 1), (9, 1), (16, 1), (32, 2), (40, 5), (32, 32)]


@pytest.mark.parametrize("lens", LENGTHS, ids=str)
@pytest.mark.parametrize("hq,hkv", HEADS)
def test_decode(lens, hq, hkv):
    gen = torch.Generator().manual_seed(hq * 100 + len(lens))
    cache, _, _ = filled(gen, lens, hkv)
    b, q = len(lens), torch.randn(len(lens), hq, D, generator=gen).to(torch.bfloat16).cuda()
    out = torch.full_like(q, 9.0)
    ws = slim.decode4_workspace(b, hq, hkv, max(lens))
    slim.slim_attn4_decode(cache, q, out, i32(lens), b, max(lens), hq, D ** -0.5, ws)
    check_decode(cache, lens, q, out, D ** -0.5)
    again = torch.empty_like(q)
    slim.slim_attn4_decode(cache, q, again, i32(lens), b, max(lens), hq, D ** -0.5, ws)
    assert torch.equal(out, again), "two calls differ"
    assert slim.slim_read_status(ws) == slim.SLIM_OK and not ws[:slim.WORKSPACE_HEADER_BYTES].any()


@pytest.mark.parametrize("lens,hq,hkv", [([32768], 32, 2), ([3000, 1, 2500, 2800], 64, 8), ([300] * 70, 16, 4), ([1, 5, 0] * 300, 4, 4), ([700], 1, 1)],
                         ids=["long", "ragged", "many", "tiny", "one"])
def test_decode_larger(lens, hq, hkv):
    gen = torch.Generator().manual_seed(len(lens))
    cache, _, _ = filled(gen, lens, hkv)
    b, q = len(lens), torch.randn(len(lens), hq, D, generator=gen).to(torch.bfloat16).cuda()
    out = torch.full_like(q, 9.0)
    slim.slim_attn4_decode(cache, q, out, i32(lens), b, max(lens), hq, D ** -0.5, slim.decode4_workspace(b, hq, hkv, max(lens)))
    check_decode(cache, lens, q, out, D ** -0.5)


@pytest.mark.parametrize("hq,hkv", [(4, 4), (16, 2), (32, 2)])
def test_decode_of_uneven_rows(hq, hkv):
    """Rows whose scales and offsets differ by orders of magnitude, a row with a few huge query channels, sharp and negative softmax scales."""
    gen = torch.Generator().manual_seed(hq)
    lens = [190, 333]
    cache, _, _ = filled(gen, lens, hkv)
    k = rows(gen, sum(lens), hkv).float() * torch.pow(10.0, torch.rand(sum(lens), 1, 1, generator=gen) * 3 - 2)
    v = rows(gen, sum(lens), hkv).float() * torch.pow(10.0, torch.rand(sum(lens), 1, 1, generator=gen) * 6 - 3)
    v[::7] = v[::7] * 1e-3 + 40.0                       # nearly constant rows with an offset
    v[3::50] = 5.0                                      # constant rows: scale 0
    v[4::50] = 0.0
    slim.slim_kv4_append(cache, k.to(torch.bfloat16).cuda(), v.to(torch.bfloat16).cuda(), i32(offsets(lens)), i32([0, 0]), 2, max(lens))
    q = torch.randn(2, hq, D, generator=gen)
    q[:, :, 17] *= 300
    q = q.to(torch.bfloat16).cuda()
    ws = slim.decode4_workspace(2, hq, hkv, max(lens))
    for scale in (D ** -0.5, 1e-4, -D ** -0.5):
        out = torch.empty_like(q)
        slim.slim_attn4_decode(cache, q, out, i32(lens), 2, max(lens), hq, scale, ws)
        for b, n in enumerate(lens):
            want, parts = reference(cache, b, n, q[b:b + 1], scale)
            parts[0] = np.abs(parts[0])
            close(out[b:b + 1], want, decode_bound(want, parts))


def test_one_token_is_its_value():
    """With one token the softmax is 1 and the result is the value row, scale 0 included."""
    gen = torch.Generator().manual_seed(11)
    cache, _, _ = filled(gen, [1, 1, 1], 2)
    v = rows(gen, 3, 2)
    v[0] = -2.75
    v[1] = 0
    slim.slim_kv4_append(cache, v.cuda(), v.cuda(), i32([0, 1, 2, 3]), i32([0, 0, 0]), 3, 1)
    q = torch.randn(3, 2, D, generator=gen).to(torch.bfloat16).cuda()
    out = torch.empty_like(q)
    slim.slim_attn4_decode(cache, q, out, i32([1, 1, 1]), 3, 128, 2, 0.3, slim.decode4_workspace(3, 2, 2, 128))
    assert (out[0] == -2.75).all() and not out[1].any()
    check_decode(cache, [1, 1, 1], q, out, 0.3)


@pytest.mark.parametrize("hq,hkv", [(4, 4), (16, 2), (32, 2)])
@pytest.mark.parametrize("lens", [[1], [64, 65, 128, 129], [5, 0, 1000, 257, 1], [2049, 2049]], ids=str)
def test_step_is_append_then_decode(lens, hq, hkv):
    gen = torch.Generator().manual_seed(hq)
    b, before = len(lens), [max(n - 1, 0) for n in lens]
    one, _, _ = filled(gen, before, hkv, capacity=max(lens))
    two = slim.SlimCache4(b, hkv, one.max_pages_per_seq, block_table=one.block_table, num_pages=one.num_pages)
    two.codes.copy_(one.codes)
    two.scales.copy_(one.scales)
    k, v, q = rows(gen, b, hkv).cuda(), rows(gen, b, hkv).cuda(), torch.randn(b, hq, D, generator=gen).to(torch.bfloat16).cuda()
    ws = slim.decode4_workspace(b, hq, hkv, max(lens))
    out, want = torch.empty_like(q), torch.empty_like(q)
    slim.slim_attn4_decode(one, q, out, i32(lens), b, max(lens), hq, D ** -0.5, ws, k_new=k, v_new=v)
    new = [1 if n > 0 else 0 for n in lens]
    kept = torch.tensor([i for i, n in enumerate(lens) if n > 0]).cuda()
    slim.slim_kv4_append(two, k[kept], v[kept], i32(offsets(new)), i32(before), b, 1)
    slim.slim_attn4_decode(two, q, want, i32(lens), b, max(lens), hq, D ** -0.5, ws)
    assert torch.equal(one.codes, two.codes) and torch.equal(one.scales.view(torch.int16), two.scales.view(torch.int16))
    assert torch.equal(out, want)
    check_decode(one, lens, q, out, D ** -0.5)


def test_lengths_beyond_the_bound():
    """kv_len beyond max_kv: the tokens that fit, and nothing appended."""
    gen = torch.Generator().manual_seed(5)
    cache, _, _ = filled(gen, [300, 300], 2)
    codes = cache.codes.clone()
    q, k = torch.randn(2, 4, D, generator=gen).to(torch.bfloat16).cuda(), rows(gen, 2, 2).cuda()
    out, want = torch.empty_like(q), torch.empty_like(q)
    ws = slim.decode4_workspace(2, 4, 2, 300)
    slim.slim_attn4_decode(cache, q, out, i32([100000, 301]), 2, 200, 4, 0.1, ws, k_new=k, v_new=k)
    assert torch.equal(codes, cache.codes)
    slim.slim_attn4_decode(cache, q, want, i32([200, 200]), 2, 200, 4, 0.1, ws)
    assert torch.equal(out, want)
    slim.slim_attn4_decode(cache, q, out, i32([-5, 0]), 2, 0, 4, 0.1, ws)
    assert not out.any()


def test_one_workspace_serves_all_shapes_and_a_graph():
    gen = torch.Generator().manual_seed(6)
    ws = slim.decode4_workspace(64, 32, 2, 65536)
    for lens, hq, hkv in (([700, 900], 32, 2), ([3], 1, 1), ([50] * 40, 8, 8), ([5000], 16, 1)):
        cache, _, _ = filled(gen, lens, hkv)
        q = torch.randn(len(lens), hq, D, generator=gen).to(torch.bfloat16).cuda()
        out = torch.empty_like(q)
        slim.slim_attn4_decode(cache, q, out, i32(lens), len(lens), max(lens), hq, D ** -0.5, ws)
        check_decode(cache, lens, q, out, D ** -0.5)
    # ---- captured on another stream, replayed with other inputs and lengths
    lens_dev, stream = i32([5000]), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        slim.slim_attn4_decode(cache, q, out, lens_dev, 1, 5000, 16, D ** -0.5, ws)
    for n in (4999, 1, 0, 2500):
        lens_dev.fill_(n)
        q.copy_(torch.randn(1, 16, D, generator=gen).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        check_decode(cache, [n], q, out, D ** -0.5)


def test_two_streams_with_a_workspace_each():
    gen = torch.Generator().manual_seed(8)
    jobs = []
    for lens, hq, hkv in (([900, 1100, 1000], 16, 4), ([6000], 32, 2)):
        cache, _, _ = filled(gen, lens, hkv)
        q = torch.randn(len(lens), hq, D, generator=gen).to(torch.bfloat16).cuda()
        jobs.append((cache, lens, q, torch.empty_like(q), slim.decode4_workspace(len(lens), hq, hkv, max(lens)), i32(lens), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for cache, lens, q, out, ws, dev, stream in jobs:
            slim.slim_attn4_decode(cache, q, out, dev, len(lens), max(lens), q.shape[1], D ** -0.5, ws, stream=stream)
    torch.cuda.synchronize()
    for cache, lens, q, out, ws, _, _ in jobs:
        check_decode(cache, lens, q, out, D ** -0.5)


def test_pages_behind_four_gigabytes():
    hkv, pages = 8, 33500                       # 4.4 GB of codes
    gen = torch.Generator().manual_seed(9)
    cache = slim.SlimCache4(1, hkv, 3, block_table=torch.tensor([[33499, 5, 33400]], dtype=torch.int32), num_pages=pages)
    n = 300
    k, v = rows(gen, n, hkv), rows(gen, n, hkv)
    slim.slim_kv4_append(cache, k.cuda(), v.cuda(), i32([0, n]), i32([0]), 1, n)
    codes, s, z = unpack(cache, 0, n)
    for kv, x in enumerate((k, v)):
        want = define(x)
        assert np.array_equal(codes[kv], want[0]) and np.array_equal(s[kv], want[1])
    q = torch.randn(1, 16, D, generator=gen).to(torch.bfloat16).cuda()
    out = torch.empty_like(q)
    slim.slim_attn4_decode(cache, q, out, i32([n]), 1, n, 16, D ** -0.5, slim.decode4_workspace(1, 16, hkv, n))
    check_decode(cache, [n], q, out, D ** -0.5)
    out4 = torch.empty((n, 16, D), dtype=torch.bfloat16, device="cuda")
    q4 = torch.randn(n, 16, D, generator=gen).to(torch.bfloat16).cuda()
    slim.slim_attn4_prefill(cache, q4, out4, i32([0, n]), i32([n]), 1, n, n, 16, D ** -0.5, slim.workspace(slim.PHASE_PREFILL, 1, 16, hkv, n, n))
    check_prefill(cache, [n], [n], q4, out4, D ** -0.5)


# ------------------------------------------------------------------------------------------------ prefill
def check_prefill(cache, q_lens, kv_lens, q, out, scale):
    cu = offsets(q_lens)
    for b, (m, n) in enumerate(zip(q_lens, kv_lens)):
        if m == 0:
            continue
        first_seen = n - m + np.arange(m)
        blind = first_seen < 0
        assert not out[cu[b]:cu[b + 1]].cpu()[torch.from_numpy(blind)].any()
        if blind.all():
            continue
        seeing = torch.from_numpy(np.flatnonzero(~blind)) + cu[b]
        want, parts = reference(cache, b, n, q.cpu()[seeing], scale, first_seen[~blind])
        _, score, v, _ = (x[..., None] for x in parts)
        close(out.cpu()[seeing], want, 2.0 ** -8 * np.abs(want) + (2 * score + 2 * 2.0 ** -11 + n * 2.0 ** -25 + 2.0 ** -20) * v)


@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 1), (15, 5)])
@pytest.mark.parametrize("q_lens,before", [([1], [0]), ([1, 0, 3], [127, 5, 128]), ([128, 129], [0, 0]), ([255, 257, 1], [1, 64, 300]), ([600], [0])], ids=str)
def test_prefill(q_lens, before, hq, hkv):
    gen = torch.Generator().manual_seed(hq + sum(q_lens))
    kv = [m + n for m, n in zip(q_lens, before)]
    cache, _, _ = filled(gen, kv, hkv)
    q = torch.randn(sum(q_lens), hq, D, generator=gen).to(torch.bfloat16).cuda()
    out = torch.full_like(q, 9.0)
    ws = slim.workspace(slim.PHASE_PREFILL, len(kv), hq, hkv, max(q_lens), max(kv))
    slim.slim_attn4_prefill(cache, q, out, i32(offsets(q_lens)), i32(kv), len(kv), max(q_lens), max(kv), hq, D ** -0.5, ws)
    check_prefill(cache, q_lens, kv, q, out, D ** -0.5)
    assert slim.slim_read_status(ws) == slim.SLIM_OK


def test_prefill_rows_that_see_nothing():
    gen = torch.Generator().manual_seed(2)
    cache, _, _ = filled(gen, [5, 0], 1, capacity=128)
    q = torch.randn(20, 2, D, generator=gen).to(torch.bfloat16).cuda()
    out = torch.full_like(q, 9.0)
    slim.slim_attn4_prefill(cache, q, out, i32([0, 10, 20]), i32([5, 0]), 2, 10, 128, 2, 0.1, slim.workspace(slim.PHASE_PREFILL, 2, 2, 1, 10, 128))
    check_prefill(cache, [10, 10], [5, 0], q, out, 0.1)


def test_prefill_step_is_append_then_prefill():
    gen = torch.Generator().manual_seed(4)
    counts, before, hq, hkv = [130, 1, 0, 300], [50, 0, 9, 129], 8, 2
    kv = [m + n for m, n in zip(counts, before)]
    one, _, _ = filled(gen, before, hkv, capacity=max(kv))
    two = slim.SlimCache4(4, hkv, one.max_pages_per_seq, block_table=one.block_table, num_pages=one.num_pages)
    two.codes.copy_(one.codes)
    two.scales.copy_(one.scales)
    k, v, q = rows(gen, sum(counts), hkv).cuda(), rows(gen, sum(counts), hkv).cuda(), torch.randn(sum(counts), hq, D, generator=gen).to(torch.bfloat16).cuda()
    cu, ws = i32(offsets(counts)), slim.workspace(slim.PHASE_PREFILL, 4, hq, hkv, 300, max(kv))
    out, want = torch.empty_like(q), torch.empty_like(q)
    slim.slim_prefill4_step(one, q, k, v, out, cu, i32(kv), 4, 300, max(kv), hq, D ** -0.5, ws)
    slim.slim_kv4_append(two, k, v, cu, i32(before), 4, 300)
    slim.slim_attn4_prefill(two, q, want, cu, i32(kv), 4, 300, max(kv), hq, D ** -0.5, ws)
    assert torch.equal(one.codes, two.codes) and torch.equal(out, want)
    check_prefill(one, counts, kv, q, out, D ** -0.5)


def test_prefill_and_decode_agree_on_the_last_row():
    gen = torch.Generator().manual_seed(14)
    n, hq, hkv = 500, 16, 4
    cache, _, _ = filled(gen, [n], hkv)
    q = torch.randn(n, hq, D, generator=gen).to(torch.bfloat16).cuda()
    out, one = torch.empty_like(q), torch.empty_like(q[:1])
    slim.slim_attn4_prefill(cache, q, out, i32([0, n]), i32([n]), 1, n, n, hq, D ** -0.5, slim.workspace(slim.PHASE_PREFILL, 1, hq, hkv, n, n))
    slim.slim_attn4_decode(cache, q[-1:].contiguous(), one, i32([n]), 1, n, hq, D ** -0.5, slim.decode4_workspace(1, hq, hkv, n))
    want, parts = reference(cache, 0, n, q[-1:], D ** -0.5)
    _, score, v, _ = (x[..., None] for x in parts)
    close(out[-1:], want, 2.0 ** -8 * np.abs(want) + (2 * score + 2 * 2.0 ** -11 + n * 2.0 ** -25 + 2.0 ** -20) * v)
    close(one, want, decode_bound(want, parts))
    assert math.isfinite(float(out.float().sum()))


@pytest.mark.parametrize("lens,bound,hq,hkv", [([100] * 16 + [0, 1, 64, 65], 8192, 16, 4), ([3000] + [2] * 19, 3000, 32, 2), ([70, 130], 30000, 4, 2)])
def test_decode_bound_far_above_the_lengths(lens, bound, hq, hkv):
    """The launch is made for max_kv: fewer units than blocks, one long sequence among short ones, few pairs on many blocks."""
    gen = torch.Generator().manual_seed(bound)
    cache, _, _ = filled(gen, lens, hkv, capacity=bound)
    b, q = len(lens), torch.randn(len(lens), hq, D, generator=gen).to(torch.bfloat16).cuda()
    out = torch.full_like(q, 9.0)
    ws = slim.decode4_workspace(b, hq, hkv, bound)
    for _ in range(2):
        slim.slim_attn4_decode(cache, q, out, i32(lens), b, bound, hq, D ** -0.5, ws)
    check_decode(cache, lens, q, out, D ** -0.5)
    assert not ws[:slim.WORKSPACE_HEADER_BYTES].any()
