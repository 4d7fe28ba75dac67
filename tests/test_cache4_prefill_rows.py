"""4-bit prefill over rows of very different size, tile by tile and row by row, against fp64 attention over the values held.

The bound is that of test_cache4 (see there) with two parts more, as rows lie far below their tile's power of two 2^e (at most the
largest |value| m of the tile): scale and offset become fp16 numbers of at least 2^-24, off by at most 2^-25 each, which up to
fifteen times the one and once the other, and the rounding of the value itself, make 17 x 2^-25 m; and a value whose size is
below its scale's fifteenfold is rounded by 2^-11 of itself, as there.  Tiles of values below 2^-100 do not occur here."""
import numpy as np
import pytest
import torch

from paper_2407_07304_b200 import binding as slim
from test_cache4 import D, PAGE, close, filled, held_values, i32, offsets, rows, unpack

pytestmark = pytest.mark.gpu


def check(cache, b, q, out, scale):
    """Query rows q [m, Hq, 128] behind which the cache ends, against fp64; the bound goes by what each row sees."""
    m, hq = q.shape[:2]
    n = int(cache.lens[b])
    codes, s, z = unpack(cache, b, n)
    k, v = held_values(codes[0], s[0], z[0]), held_values(codes[1], s[1], z[1])
    q = q.double().cpu().numpy()
    seen = np.arange(n)[None, :] <= (n - m + np.arange(m))[:, None]
    want, bound = np.zeros(q.shape), np.zeros(q.shape)
    tile = np.arange(n) // PAGE
    for h in range(hq):
        g = h // (hq // cache.Hkv)
        kt = np.array([np.abs(k[tile == t, g]).max() for t in range(tile[-1] + 1)])[tile]      # largest |key value| of a key's tile
        vt = np.array([np.abs(v[tile == t, g]).max() for t in range(tile[-1] + 1)])
        score = np.where(seen, scale * (q[:, h] @ k[:, g].T), -np.inf)
        p = np.exp(score - score.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        want[:, h] = p @ v[:, g]
        size = np.abs(q[:, h])
        # a score's error, then the change of the result: a factor of 1 + 2 error at most on every weight and on their sum
        error = abs(scale) * (size @ np.abs(k[:, g]).T * 2.0 ** -11 + size.sum(1, keepdims=True) * kt[None, :] * 17 * 2.0 ** -25)
        worst = np.where(seen, error, 0).max(1)[:, None] + 2.0 ** -20
        # weights in fp16: 2^-11 of each, or, where p 2^e(V) lies 2^-14 below the largest one, 2^-25 of that one
        top = np.max([(np.where(seen & (tile == t)[None, :], p, 0)).max(1) * max(vt[t], 2.0 ** -100) for t in range(len(vt))], axis=0)[:, None]
        weighed = p @ np.abs(v[:, g])
        bound[:, h] = (2.0 ** -8 * np.abs(want[:, h]) + (4 * worst + 2 * 2.0 ** -11) * weighed + n * 2.0 ** -25 * 2 ** 4 * top
                       + (p @ vt[tile])[:, None] * 17 * 2.0 ** -25 + 2.0 ** -20 * weighed)
    close(out, want, bound)


def sizes(gen, n, low, high):
    return torch.pow(10.0, torch.rand(n, 1, 1, generator=gen) * (high - low) + low)


def uneven(gen, n, hkv):
    """Keys of 10^-2 to 10, values of 10^-3 to 10^3; rows nearly constant about an offset, constant and zero ones; whole tiles apart."""
    k = rows(gen, n, hkv).float() * sizes(gen, n, -2, 1) / 8
    v = rows(gen, n, hkv).float() * sizes(gen, n, -3, 3)
    k[5::9] = k[5::9] * 1e-3 - 3.0
    k[6::40] = 0.25
    k[7::40] = 0.0
    v[::7] = v[::7] * 1e-6 + 40.0
    v[1::7] = v[1::7] * 1e-6 - 40.0
    v[3::50] = 5.0
    v[4::50] = 0.0
    return k, v


def run(gen, counts, lens, hq, hkv, k, v, scale=D ** -0.5):
    cache, _, _ = filled(gen, lens, hkv)
    cache.lens = lens
    cu_k = offsets(lens)
    slim.slim_kv4_append(cache, k.to(torch.bfloat16).cuda(), v.to(torch.bfloat16).cuda(), i32(cu_k), i32([0] * len(lens)), len(lens), max(lens))
    q = torch.randn(sum(counts), hq, D, generator=gen)
    q[:, :, 17] *= 30
    q = q.to(torch.bfloat16).cuda()
    out, cu = torch.full_like(q, 9.0), offsets(counts)
    ws = slim.workspace(slim.PHASE_PREFILL, len(lens), hq, hkv, max(counts), max(lens))
    slim.slim_attn4_prefill(cache, q, out, i32(cu), i32(lens), len(lens), max(counts), max(lens), hq, scale, ws)
    for b in range(len(lens)):
        check(cache, b, q[cu[b]:cu[b + 1]], out[cu[b]:cu[b + 1]], scale)


@pytest.mark.parametrize("scale", [D ** -0.5, 1e-4, -D ** -0.5])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (6, 2), (16, 1), (34, 2)])
def test_uneven_rows(hq, hkv, scale):
    gen = torch.Generator().manual_seed(hq)
    counts, lens = [70, 130, 1], [190, 400, 333]
    k, v = uneven(gen, sum(lens), hkv)
    run(gen, counts, lens, hq, hkv, k, v, scale)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (16, 1)])
def test_uneven_tiles(hq, hkv):
    """Tiles of 128 tokens a thousandfold apart, both ways; a tile of zero values, one of constant rows, one nearly so."""
    gen = torch.Generator().manual_seed(hq)
    n = 7 * PAGE + 5
    k, v = rows(gen, n, hkv).float() / 8, rows(gen, n, hkv).float()
    for t, (a, c) in enumerate([(1.0, 1e-3), (1e-3, 1.0), (1.0, 0.0), (1e-2, 1e3), (0.0, 1.0), (1.0, 1.0), (3.0, 1e-3), (1.0, 10.0)]):
        k[t * PAGE:(t + 1) * PAGE] *= a
        v[t * PAGE:(t + 1) * PAGE] *= c
    v[5 * PAGE:6 * PAGE] = -7.0
    v[6 * PAGE:7 * PAGE] += 100.0
    run(gen, [n], [n], hq, hkv, k, v)


def test_sixteen_heads_of_one_row_block():
    """Few tokens of sixteen heads: a block's rows belong to tokens that see different numbers of keys."""
    gen = torch.Generator().manual_seed(1)
    counts, lens = [17, 33, 3, 16], [17, 160, 131, 128]
    k, v = rows(gen, sum(lens), 2).float() / 8, rows(gen, sum(lens), 2).float()
    run(gen, counts, lens, 32, 2, k, v)
