"""The norm-and-rotation, shared-prefix, weighted-decode and eviction calls against plain 64-bit implementations, on a GPU.

Bounds.  A rounding is off by at most half a step: bf16 2^-8 of the value, fp16 2^-11, fp32 2^-24, a code half its row's
scale.  The arithmetic between is fp32; each bound's comment counts its terms."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

D, PAGE = 128, 128


def _slim():
    from paper_2407_07304_b200 import binding
    return binding


def gen(seed):
    return torch.Generator().manual_seed(seed)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ================================================================== norm and rotation
def rope_reference(x, w, eps, pos, axis, inv_freq, inter):
    """fp64 [tokens, heads, 128] from bf16."""
    x = x.double().cpu()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double().cpu()
    half = inv_freq.numel()
    if half == 0:
        return x
    a = pos.cpu().double()[axis.cpu().long()].T * inv_freq.cpu()[None]          # [tokens, half]
    c, s = a.cos()[:, None], a.sin()[:, None]
    y = x.clone()
    f, g = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if inter else (slice(0, half), slice(half, 2 * half))
    y[..., f] = x[..., f] * c - x[..., g] * s
    y[..., g] = x[..., f] * s + x[..., g] * c
    return y


def rope_inputs(seed, n, hq, hkv, rotary, axes, norm, far=5000, theta=10000.0):
    g = gen(seed)
    half = rotary // 2
    rows = (torch.randn((n, hq + 2 * hkv, D), generator=g) * torch.exp2(torch.randint(-3, 4, (1, hq + 2 * hkv, 1), generator=g).float())).to(torch.bfloat16).cuda()
    inv = torch.tensor([theta ** (-i / max(half, 1)) for i in range(half)], dtype=torch.float64).cuda()
    axis = torch.randint(0, axes, (half,), generator=g).to(torch.uint8).cuda()
    pos = torch.randint(-3, far, (axes, n), generator=g).to(torch.int32).cuda()
    w = [(torch.randn(D, generator=g) * 0.3 + 1).to(torch.bfloat16).cuda() if norm else None for _ in range(2)]
    return rows, inv, axis, pos, w


def rope_close(got, want, top, what):
    """bf16 rounding (2^-8 of the value) and, before it, fp32: a dozen roundings of the row's elements and an angle off by
    2^-22 of a turn, together below 2^-18 of the row's largest element before the rotation (`top`)."""
    err = (got.double().cpu() - want).abs()
    bound = want.abs() * 2.0 ** -8 + top * 2.0 ** -18
    assert torch.isfinite(got.float()).all(), what
    assert (err <= bound).all(), f"{what}: {(err - bound).max().item():.3e} over the bound"


ROPE_CASES = [
    # tokens, hq, hkv, rotary, axes, interleaved, norm
    (1, 1, 1, 128, 1, False, True), (1, 0, 1, 128, 1, False, True), (3, 2, 0, 64, 1, True, True), (2, 5, 1, 0, 1, False, True),
    (65, 1, 0, 128, 1, False, False), (7, 5, 2, 96, 2, False, True), (130, 8, 8, 32, 3, False, True), (33, 4, 1, 16, 4, True, False),
    (64, 3, 3, 112, 2, True, True), (17, 32, 8, 128, 3, False, True), (19, 7, 1, 48, 1, False, False), (5, 64, 4, 64, 1, False, True),
    (1025, 2, 1, 128, 1, True, True),
]


@pytest.mark.parametrize("case", ROPE_CASES, ids=lambda c: "-".join(map(str, c)))
def test_norm_rope(case):
    n, hq, hkv, rotary, axes, inter, norm = case
    slim = _slim()
    rows, inv, axis, pos, w = rope_inputs(n + hq, n, hq, hkv, rotary, axes, norm)
    q, k = rows[:, :hq], rows[:, hq:hq + hkv]            # views of the fused projection's rows
    nr = slim.NormRope(inv, w[0], w[1], 1e-5, axis if rotary else None, axes, inter)
    qo, ko = torch.full((n, hq, D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((n, hkv, D), 7.0, dtype=torch.bfloat16, device="cuda")
    slim.slim_norm_rope(nr, q if hq else None, qo if hq else None, k if hkv else None, ko if hkv else None, pos if rotary else None)
    torch.cuda.synchronize()
    for x, o, ww in ((q, qo, w[0]), (k, ko, w[1])):
        if x.shape[1]:
            want = rope_reference(x, ww, 1e-5, pos, axis, inv, inter)
            rope_close(o, want, rope_reference(x, ww, 1e-5, pos, axis[:0], inv[:0], inter).abs().amax(-1, keepdim=True), case)


def test_norm_rope_in_place_and_one_sided_norm():
    slim = _slim()
    rows, inv, axis, pos, w = rope_inputs(5, 37, 6, 2, 96, 2, True)
    q, k = rows[:, :6].contiguous(), rows[:, 6:8].contiguous()
    nr = slim.NormRope(inv, None, w[1], 1e-5, axis, 2, False)
    a, b = torch.empty_like(q), torch.empty_like(k)
    slim.slim_norm_rope(nr, q, a, k, b, pos)
    rope_close(a, rope_reference(q, None, 0, pos, axis, inv, False), q.double().cpu().abs().amax(-1, keepdim=True), "no norm for q")
    slim.slim_norm_rope(nr, q, q, k, k, pos)
    torch.cuda.synchronize()
    assert torch.equal(q, a) and torch.equal(k, b)


def test_norm_rope_far_positions_and_zero_rows():
    # up to 2^31 - 1: an angle formed in fp32 would be meaningless there
    slim = _slim()
    rows, inv, axis, pos, w = rope_inputs(11, 64, 2, 1, 128, 1, True, far=2 ** 31 - 1)
    pos[0, 0], pos[0, 1], pos[0, 2] = 2 ** 31 - 1, -2 ** 31, 1 << 24
    rows[3] = 0
    q, k = rows[:, :2], rows[:, 2:3]
    nr = slim.NormRope(inv, w[0], w[1], 1e-6)
    qo, ko = torch.empty((64, 2, D), dtype=torch.bfloat16, device="cuda"), torch.empty((64, 1, D), dtype=torch.bfloat16, device="cuda")
    slim.slim_norm_rope(nr, q, qo, k, ko, pos)
    torch.cuda.synchronize()
    # the reference's own angle is off by 2^31 * 2^-53 * pi at most: nothing here
    for x, o, ww in ((q, qo, w[0]), (k, ko, w[1])):
        want = rope_reference(x, ww, 1e-6, pos, torch.zeros(64), inv, False)
        rope_close(o, want, rope_reference(x, ww, 1e-6, pos, axis[:0], inv[:0], False).abs().amax(-1, keepdim=True), "far")
    assert (qo[3] == 0).all() and (ko[3] == 0).all()


APPEND_CASES = [
    # new tokens per sequence, cached before, hq, hkv, rotary, axes, interleaved, norm, positions given
    ([1], [0], 1, 1, 128, 1, False, True, False), ([1, 1, 1], [127, 128, 300], 4, 2, 64, 1, True, True, True),
    ([5, 0, 130, 0], [0, 7, 100, 3], 8, 8, 128, 3, False, True, True), ([0, 3], [0, 0], 0, 2, 96, 2, False, True, False),
    ([257, 2], [1, 383], 7, 1, 0, 1, False, True, True), ([1] * 70, [5 * i for i in range(70)], 2, 1, 128, 1, False, False, False),
]


@pytest.mark.parametrize("case", APPEND_CASES, ids=range(len(APPEND_CASES)))
def test_norm_rope_append(case):
    new, before, hq, hkv, rotary, axes, inter, norm, given = case
    slim = _slim()
    B, n, behind = len(new), sum(new), 3                 # three rows behind the last sequence (a padded batch)
    rows, inv, axis, pos, w = rope_inputs(n + hq, n + behind, hq, hkv, rotary, axes, norm)
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    mp = max((a + b + PAGE - 1) // PAGE for a, b in zip(new, before)) or 1
    table = torch.randperm(B * mp, generator=gen(1)).to(torch.int32).view(B, mp)
    cache, plain = (slim.SlimCache(B, hkv, mp, block_table=table) for _ in range(2))
    for c in (cache, plain):
        c.codes.fill_(77)
        c.scales.fill_(-1.0)
    cu = [0]
    for x in new:
        cu.append(cu[-1] + x)
    if not given:
        at = torch.cat([torch.arange(s, s + x) for s, x in zip(before, new)] + [torch.zeros(behind, dtype=torch.int64)])
        pos = at.to(torch.int32).cuda().expand(axes, -1).contiguous()
    nr = slim.NormRope(inv, w[0], w[1], 1e-5, axis if rotary else None, axes, inter)
    qo = torch.full((n + behind, hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    slim.slim_norm_rope_append(cache, nr, q if hq else None, qo if hq else None, k, v, pos if given else None, i32(cu), i32(before), B)
    torch.cuda.synchronize()
    if hq:
        want = rope_reference(q, w[0], 1e-5, pos, axis, inv, inter)[:n]
        top = rope_reference(q, w[0], 1e-5, pos, axis[:0], inv[:0], inter)[:n].abs().amax(-1, keepdim=True)
        rope_close(qo[:n], want, top, case)
        assert (qo[n:] == 7.0).all()                     # behind the last sequence: as they were
    # values: bit for bit what slim_kv_append writes; keys: within half a step of the exact row's scale, and fp32's share
    slim.slim_kv_append(plain, k.contiguous(), v.contiguous(), i32(cu), i32(before), B, max(new))
    torch.cuda.synchronize()
    codes, scales = cache.codes_view().cpu(), cache.scales_view().cpu()
    pc, ps = plain.codes_view().cpu(), plain.scales_view().cpu()
    assert torch.equal(codes[:, :, 1], pc[:, :, 1]) and torch.equal(scales[:, :, 1], ps[:, :, 1])
    exact = rope_reference(k, w[1], 1e-5, pos, axis, inv, inter)
    top = rope_reference(k, w[1], 1e-5, pos, axis[:0], inv[:0], inter).abs().amax(-1)
    touched = torch.zeros_like(scales[:, :, 0], dtype=torch.bool)
    for b in range(B):
        for t in range(new[b]):
            p = before[b] + t
            page, slot, tok = int(table[b, p // PAGE]), p % PAGE, cu[b] + t
            touched[page, :, slot] = True
            sc = scales[page, :, 0, slot].double()
            amax = exact[tok].abs().amax(-1)
            assert ((sc - amax / 127).abs() <= top[tok] * 2.0 ** -18 / 127 + amax * 2.0 ** -24).all()
            off = (codes[page, :, 0, slot].double() * sc[:, None] - exact[tok]).abs()
            assert (off <= sc[:, None] * 0.5 + top[tok][:, None] * 2.0 ** -17).all()
    assert (codes[:, :, 0][~touched] == 77).all() and (scales[:, :, 0][~touched] == -1.0).all()


def test_norm_rope_append_without_norm_and_rotation_is_the_append():
    slim = _slim()
    rows, _, _, _, _ = rope_inputs(3, 300, 2, 3, 0, 1, False)
    rows[7] = 0
    rows[8] *= 2.0 ** -70
    rows[9] *= 2.0 ** 70
    caches = [slim.SlimCache(2, 3, 2) for _ in range(2)]
    q, k, v = rows[:, :2], rows[:, 2:5], rows[:, 5:]
    qo = torch.empty((300, 2, D), dtype=torch.bfloat16, device="cuda")
    slim.slim_norm_rope_append(caches[0], slim.NormRope(), q, qo, k, v, None, i32([0, 100, 300]), i32([50, 0]), 2)
    slim.slim_kv_append(caches[1], k.contiguous(), v.contiguous(), i32([0, 100, 300]), i32([50, 0]), 2, 200)
    torch.cuda.synchronize()
    assert torch.equal(qo, q) and torch.equal(caches[0].codes, caches[1].codes) and torch.equal(caches[0].scales, caches[1].scales)


def test_norm_rope_append_skips_pages_that_do_not_exist():
    slim = _slim()
    rows, inv, axis, pos, w = rope_inputs(3, 40, 2, 1, 128, 1, True)
    cache = slim.SlimCache(2, 1, 1, block_table=torch.tensor([[5], [-1]], dtype=torch.int32), num_pages=2)   # pages that are not there
    qo = torch.empty((40, 2, D), dtype=torch.bfloat16, device="cuda")
    slim.slim_norm_rope_append(cache, slim.NormRope(inv, w[0], w[1]), rows[:, :2], qo, rows[:, 2:3], rows[:, 3:], pos, i32([0, 20, 40]), i32([120, -10]), 2)
    torch.cuda.synchronize()
    assert (cache.codes == 0).all() and (cache.scales == 0).all()
    rope_close(qo, rope_reference(rows[:, :2], w[0], 1e-6, pos, axis, inv, False), torch.full((40, 2, 1), 16.0, dtype=torch.float64), "queries")


# ================================================================== decode over a cache with given contents
def fill(cache, seed):
    """Normal rows, a few channels eight times the others', quantised by plain arithmetic into every page of the pool."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((cache.num_pages, cache.Hkv, 2, PAGE, D), generator=g, device="cuda")
    x[..., torch.randperm(D, generator=gen(seed))[:4]] *= 8
    amax = x.abs().amax(-1, keepdim=True)
    cache.codes.copy_((x / amax * 127).round().clamp(-127, 127).to(torch.int8).view(-1))
    cache.scales.copy_((amax / 127).view(-1))


def rows_of(cache, b, length):
    """fp64 K and V [Hkv, length, 128] of a sequence."""
    pages = cache.block_table[b, :(length + PAGE - 1) // PAGE].long()
    x = cache.codes_view()[pages].double() * cache.scales_view()[pages].double()[..., None]
    x = x.permute(2, 1, 0, 3, 4).reshape(2, cache.Hkv, -1, D)[:, :, :length]
    return x[0], x[1]


def attend(cache, q, lens, sm_scale):
    """fp64 outputs [B, Hq, 128], per sequence the probabilities [Hq, length], and per row what an error is measured by:
    (sum p |v|, and how far fp16 roundings of the keys move a score)."""
    B, Hq, _ = q.shape
    G = Hq // cache.Hkv
    out, probs, top = torch.zeros((B, Hq, D), dtype=torch.float64, device="cuda"), [], torch.zeros((B, Hq, 1), dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        if n <= 0:
            probs.append(torch.zeros((Hq, 0), dtype=torch.float64, device="cuda"))
            continue
        k, v = rows_of(cache, b, n)
        s = torch.einsum("hgd,hnd->hgn", q[b].double().view(cache.Hkv, G, D), k) * sm_scale
        p = torch.softmax(s, -1)
        out[b] = torch.einsum("hgn,hnd->hgd", p, v).reshape(Hq, D)
        moved = torch.einsum("hgd,hnd->hgn", q[b].double().view(cache.Hkv, G, D) ** 2, k ** 2).amax(-1).sqrt() * abs(sm_scale)
        top[b] = (torch.einsum("hgn,hnd->hgd", p, v.abs()).amax(-1) * (2.0 ** -9 + 16 * 2.0 ** -11 / 3 ** 0.5 * moved)).reshape(Hq, 1)
        probs.append(p.reshape(Hq, n))
    return out, probs, top


def out_close(got, want, slack, what):
    """bf16 rounding of the result: 2^-8 of it.  fp16 roundings of P and of V^, 2^-11 each of every term, P's fixed point and
    the fp32 sums: 2^-9 of sum p |v| in all.  Scores from fp16 keys: 128 independent roundings of at most 2^-11 of
    their terms, eight standard deviations, twice (numerator and denominator).  attend() adds the last two up (`slack`).
    On average the roundings must stay below half steps of the result and 2^-9 of the slack's terms."""
    assert torch.isfinite(got.float()).all(), what
    err = (got.double() - want).abs()
    bound = want.abs() * 2.0 ** -8 + slack + 1e-30
    assert (err <= bound).all(), f"{what}: {(err / bound).max().item():.3f} times the bound"
    assert err.mean() <= 0.5 * bound.mean(), what


def shared_setup(seed, groups, hq, hkv, tail_pages):
    """groups: list of (prefix pages, sequences).  Pages of a group's prefix are shared, every tail has pages of its own."""
    slim = _slim()
    B = sum(n for _, n in groups)
    mp = max(p for p, _ in groups) + tail_pages
    n_pages = sum(p for p, _ in groups) + B * mp
    order = torch.randperm(n_pages, generator=gen(seed)).tolist()
    table = []
    for pre, n in groups:
        head = [order.pop() for _ in range(pre)]
        table += [head + [order.pop() for _ in range(mp - pre)] for _ in range(n)]
    cache = slim.SlimCache(B, hkv, mp, block_table=torch.tensor(table, dtype=torch.int32), num_pages=n_pages)
    fill(cache, seed)
    cu = [0]
    for _, n in groups:
        cu.append(cu[-1] + n)
    return cache, B, cu


SHARED_CASES = [
    # groups (prefix pages, sequences), hq, hkv, tails per sequence (cycled; negative: shorter than the prefix by that much)
    ([(1, 1)], 1, 1, [0]), ([(1, 2)], 2, 1, [1, 2]), ([(2, 3)], 4, 4, [1, 129, 256]), ([(3, 5)], 16, 1, [300, 1, 0, 257, 128]),
    ([(7, 16)], 8, 8, [5]), ([(16, 16)], 16, 2, [1, 100, 200, 300]), ([(5, 33)], 28, 4, [17, 0, 130]), ([(9, 40)], 16, 1, [3, 515]),
    ([(4, 2), (0, 3), (11, 9), (1, 1)], 6, 3, [1, 60, 300]), ([(20, 64)], 8, 1, [2]), ([(2, 4)], 4, 2, [-1, -128, -255, -256]),
    ([(3, 70)], 15, 5, [-384, -383, 1, 0, -1, 44, -129]), ([(33, 17)], 32, 32, [127, 128, 129]), ([(40, 8)], 64, 4, [700, 1]),
    ([(2, 129)], 1, 1, [9]),
    # more prefix blocks than SMs: nine groups of 32 kv heads; thirteen row blocks of one kv head; 65 groups of one
    ([(2, 2)] * 9, 32, 32, [3, 140]), ([(4, 200)], 16, 1, [5, 1, 260]), ([(1, 1), (2, 1)] * 32 + [(0, 1)], 4, 4, [2, 130, 0]),
]


@pytest.mark.parametrize("case", SHARED_CASES, ids=range(len(SHARED_CASES)))
@pytest.mark.parametrize("append", [False, True])
def test_decode_shared(case, append):
    groups, hq, hkv, tails = case
    slim = _slim()
    g = gen(len(groups) + hq)
    tail_pages = max(0, max(tails)) // PAGE + 2
    cache, B, cu = shared_setup(hq, groups, hq, hkv, tail_pages)
    pre = [p * PAGE for p, n in groups for _ in range(n)]
    lens = [max(0, pre[b] + tails[b % len(tails)]) for b in range(B)]
    max_tail = max(max(0, lens[b] - pre[b]) for b in range(B))
    q = torch.randn((B, hq, D), generator=g).to(torch.bfloat16).cuda()
    out = torch.full_like(q, 5.0)
    ws = slim.shared_workspace(B, hq, hkv, len(groups), max(n for _, n in groups), max(pre), max_tail)
    shared = i32([p + (7 if p else 0) for p in pre])       # a length inside a page: cut to the page
    new = {}
    if append:
        kn, vn = (torch.randn((B, hkv, D), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
        new = dict(k_new=kn, v_new=vn)
        before = cache.codes.clone()
        expect = slim.SlimCache(B, hkv, cache.max_pages_per_seq, block_table=cache.block_table, num_pages=cache.num_pages)
        expect.codes.copy_(cache.codes)
        expect.scales.copy_(cache.scales)
        goes = [b for b in range(B) if lens[b] > pre[b]]
        if goes:   # the new tokens that fall behind the prefix, by the append call
            start = torch.full((B,), -1, dtype=torch.int32)
            for b in goes:
                start[b] = lens[b] - 1
            slim.slim_kv_append(expect, kn, vn, i32(list(range(B + 1))), start.cuda(), B, 1)
    slim.slim_attn_decode_shared(cache, q, out, i32(cu), shared, i32(lens), len(groups), B, max(n for _, n in groups), max(pre) + 7 if max(pre) else 0,
                                 max_tail, hq, D ** -0.5, ws, **new)
    torch.cuda.synchronize()
    assert slim.slim_read_status(ws) == slim.SLIM_OK
    if append:
        assert torch.equal(cache.codes, expect.codes) and torch.equal(cache.scales, expect.scales)
        assert any(lens[b] > pre[b] for b in range(B)) == bool((cache.codes != before).any())
    want, _, top = attend(cache, q, lens, D ** -0.5)
    out_close(out, want, top, case)
    for b in range(B):
        if lens[b] == 0:
            assert (out[b] == 0).all()


def test_decode_shared_without_prefix_is_decode():
    slim = _slim()
    cache, B, cu = shared_setup(3, [(0, 3)], 8, 2, 3)
    q = torch.randn((B, 8, D), generator=gen(4)).to(torch.bfloat16).cuda()
    lens = i32([1, 200, 300])
    a, b = torch.empty_like(q), torch.empty_like(q)
    ws = slim.shared_workspace(B, 8, 2, 1, B, 0, 300)
    slim.slim_attn_decode_shared(cache, q, a, i32(cu), i32([0, 0, 0]), lens, 1, B, B, 0, 300, 8, D ** -0.5, ws)
    slim.slim_attn_decode(cache, q, b, lens, B, 300, 8, D ** -0.5, slim.workspace(slim.PHASE_DECODE, B, 8, 2, 1, 300))
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_decode_shared_garbage_behind_the_tokens():
    # rows that no sequence has yet hold codes and scales of anything, a NaN included: they must not reach a result
    slim = _slim()
    cache, B, cu = shared_setup(9, [(3, 20)], 16, 2, 1)
    lens = [300 - (b % 3) for b in range(B)]               # inside the prefix's last page
    k = cache.scales_view()
    page = int(cache.block_table[0, 2])
    k[page, :, :, 300 - 2 * PAGE:] = float("nan")
    tail = cache.block_table[:, 3].long()
    k[tail] = float("inf")
    q = torch.randn((B, 16, D), generator=gen(4)).to(torch.bfloat16).cuda()
    out = torch.empty_like(q)
    ws = slim.shared_workspace(B, 16, 2, 1, B, 3 * PAGE, 64)
    slim.slim_attn_decode_shared(cache, q, out, i32(cu), i32([3 * PAGE] * B), i32(lens), 1, B, B, 3 * PAGE, 64, 16, D ** -0.5, ws)
    torch.cuda.synchronize()
    k[page, :, :, 300 - 2 * PAGE:] = 0.0
    want, _, top = attend(cache, q, lens, D ** -0.5)
    out_close(out, want, top, "garbage")


def test_decode_shared_growing_and_falling_maxima():
    # the prefix's scores grow from tile to tile by far more than the rescaling threshold, then fall; scales jump as well
    slim = _slim()
    for R in (3, 200):
        cache, B, cu = shared_setup(5, [(12, R)], 1, 1, 1)
        pre = cache.block_table[0, :12].long()
        k = cache.scales_view()
        f = torch.tensor([2.0 ** min(j, 14 - j) for j in range(12)], device="cuda")
        k[pre, :, 0] *= f[:, None, None]
        k[pre, :, 1] *= torch.tensor([2.0 ** ((j * 5) % 7 - 3) for j in range(12)], device="cuda")[:, None, None]
        q = torch.randn((B, 1, D), generator=gen(4)).to(torch.bfloat16).cuda()
        out = torch.empty_like(q)
        lens = [12 * PAGE + 3] * B
        ws = slim.shared_workspace(B, 1, 1, 1, B, 12 * PAGE, 3)
        slim.slim_attn_decode_shared(cache, q, out, i32(cu), i32([12 * PAGE] * B), i32(lens), 1, B, B, 12 * PAGE, 3, 1, D ** -0.5, ws)
        torch.cuda.synchronize()
        want, _, _ = attend(cache, q, lens, D ** -0.5)
        # scores reach about 700: K^'s fp16 rounding (2^-12 on average 2^-13 of 128 terms) moves them, so the weights by a factor;
        # what must hold then is that every output stays within the rows' range and finite, and that rows whose best key wins by
        # far (a margin of 20 in the exponent) agree
        assert torch.isfinite(out.float()).all()
        for b in range(B):
            kk, vv = rows_of(cache, b, lens[b])
            s = (kk[0] @ q[b, 0].double()) * D ** -0.5
            best = torch.topk(s, 2)
            if best.values[0] - best.values[1] > 20:
                v = vv[0, best.indices[0]]
                assert ((out[b, 0].double() - v).abs() <= v.abs() * 2.0 ** -8 + v.abs().max() * 2.0 ** -9).all()


@pytest.mark.parametrize("sm_scale", [-0.05, 0.0, 1e-3, 0.4])
def test_decode_shared_and_weights_any_scale(sm_scale):
    slim = _slim()
    for groups in ([(3, 4)], [(3, 40)]):                    # 16 and 160 rows per kv head
        cache, B, cu = shared_setup(12, groups, 8, 2, 2)
        q = torch.randn((B, 8, D), generator=gen(4)).to(torch.bfloat16).cuda()
        lens = [384 + (37 * b) % 200 for b in range(B)]
        out, out2 = torch.empty_like(q), torch.empty_like(q)
        ws = slim.shared_workspace(B, 8, 2, 1, B, 384, 200)
        slim.slim_attn_decode_shared(cache, q, out, i32(cu), i32([384] * B), i32(lens), 1, B, B, 384, 200, 8, sm_scale, ws)
        wt = torch.zeros((B, 2, 600), device="cuda")
        slim.slim_attn_decode_weights(cache, q, out2, None, wt, None, i32(lens), B, 600, 8, sm_scale, 1.0, slim.weights_workspace(B, 8, 2, 600))
        torch.cuda.synchronize()
        want, probs, slack = attend(cache, q, lens, sm_scale)
        out_close(out, want, slack, "shared")
        out_close(out2, want, slack, "weights")
        for b in range(B):
            assert (wt[b, :, :lens[b]].double() - probs[b].view(2, 4, -1).sum(1)).abs().max() < 1e-4


def test_decode_shared_and_weights_zero_rows():
    """Keys and values of zero (scale 0), a whole tile of them, zero queries."""
    slim = _slim()
    cache, B, cu = shared_setup(13, [(3, 30)], 8, 2, 3)
    codes, scales = cache.codes_view(), cache.scales_view()
    pre = cache.block_table[0, :3].long()
    codes[pre[1]] = 0
    scales[pre[1]] = 0.0                                    # every key and value of the second tile
    tail = cache.block_table[:, 3].long()
    codes[tail, :, :, 5:20] = 0
    scales[tail, :, :, 5:20] = 0.0
    q = torch.randn((B, 8, D), generator=gen(4)).to(torch.bfloat16).cuda()
    q[3] = 0
    q[4, 1] = 0
    lens = [384 + (23 * b) % 300 for b in range(B)]
    out, out2 = torch.empty_like(q), torch.empty_like(q)
    ws = slim.shared_workspace(B, 8, 2, 1, B, 384, 300)
    slim.slim_attn_decode_shared(cache, q, out, i32(cu), i32([384] * B), i32(lens), 1, B, B, 384, 300, 8, D ** -0.5, ws)
    wt = torch.zeros((B, 2, 700), device="cuda")
    slim.slim_attn_decode_weights(cache, q, out2, None, wt, None, i32(lens), B, 700, 8, D ** -0.5, 1.0, slim.weights_workspace(B, 8, 2, 700))
    torch.cuda.synchronize()
    want, probs, slack = attend(cache, q, lens, D ** -0.5)
    out_close(out, want, slack, "shared")
    out_close(out2, want, slack, "weights")
    for b in range(B):
        assert (wt[b, :, :lens[b]].double() - probs[b].view(2, 4, -1).sum(1)).abs().max() < 1e-5


# ================================================================== attention weights
WEIGHT_CASES = [
    # lengths, hq, hkv
    ([1], 1, 1), ([2], 4, 1), ([1, 0, 3, 256, 257, 258], 6, 3), ([300, 1, 513], 16, 1), ([272], 32, 32), ([1030, 5, 2049, 1025, 1024], 16, 2),
    ([9000, 100], 16, 1), ([700] * 20, 8, 8), ([4097], 14, 2), ([0, 0], 2, 2), ([33000], 2, 1),
]


@pytest.mark.parametrize("case", WEIGHT_CASES, ids=range(len(WEIGHT_CASES)))
@pytest.mark.parametrize("append", [False, True])
def test_decode_weights(case, append):
    lens, hq, hkv = case
    slim = _slim()
    g = gen(sum(lens) + hq)
    B, top_len = len(lens), max(lens)
    mp = max(1, (top_len + PAGE - 1) // PAGE)
    table = torch.randperm(B * mp, generator=g).to(torch.int32).view(B, mp)
    cache = slim.SlimCache(B, hkv, mp, block_table=table)
    fill(cache, hq)
    q = torch.randn((B, hq, D), generator=g).to(torch.bfloat16).cuda()
    stride = top_len + 13                                   # odd row lengths, entries behind the tokens
    w_in = torch.rand((B, hkv, stride), generator=g).cuda()
    for b in range(B):
        w_in[b, :, max(0, lens[b] - 2):] = float("nan")     # not weighed yet: anything
    weighed = i32([max(0, n - 2) for n in lens])
    w_out = torch.full((B, hkv, stride), -3.0, device="cuda")
    out, ref = torch.empty_like(q), torch.empty_like(q)
    new = {}
    if append:
        new = dict(k_new=torch.randn((B, hkv, D), generator=g).to(torch.bfloat16).cuda(), v_new=torch.randn((B, hkv, D), generator=g).to(torch.bfloat16).cuda())
    ws = slim.weights_workspace(B, hq, hkv, top_len)
    slim.slim_attn_decode_weights(cache, q, out, w_in, w_out, weighed, i32(lens), B, top_len, hq, D ** -0.5, 0.75, ws, **new)
    slim.slim_attn_decode(cache, q, ref, i32(lens), B, top_len, hq, D ** -0.5, slim.workspace(slim.PHASE_DECODE, B, hq, hkv, 1, top_len))
    torch.cuda.synchronize()
    assert slim.slim_read_status(ws) == slim.SLIM_OK
    assert torch.equal(out, ref)                            # the attention itself is slim_attn_decode's
    _, probs, _ = attend(cache, q, lens, D ** -0.5)
    for b, n in enumerate(lens):
        assert (w_out[b, :, n:] == -3.0).all()
        if n == 0:
            continue
        k, _ = rows_of(cache, b, n)
        old = torch.zeros((hkv, n), dtype=torch.float64, device="cuda")
        old[:, :max(0, n - 2)] = 0.75 * w_in[b, :, :max(0, n - 2)].double()
        p = probs[b].view(hkv, hq // hkv, n).sum(1)
        want = old + p
        # a query element is held to 2^-21 of its row's largest power of two (half a step of 2^-20, twice for that power's
        # spread), so a score is off by 2^-20 max|q| sum|k| sm_scale at most; six fp32 roundings of scores and
        # exponents up to 64 in log2 units; the denominator doubles it
        ds = D ** -0.5 * 2.0 ** -20 * q[b].double().abs().max() * k.abs().sum(-1).max() + 6 * 64 * 2.0 ** -24
        bound = 2 * ds * p + want * 2.0 ** -22 + 1e-30
        assert ((w_out[b, :, :n].double() - want).abs() <= bound).all(), (b, ((w_out[b, :, :n].double() - want).abs() / (p + 1e-30)).max().item())


def test_decode_weights_in_place_and_from_nothing():
    slim = _slim()
    cache = slim.SlimCache(2, 2, 3)
    fill(cache, 1)
    q = torch.randn((2, 8, D), generator=gen(1)).to(torch.bfloat16).cuda()
    lens, out, ws = i32([300, 40]), torch.empty_like(q), slim.weights_workspace(2, 8, 2, 300)
    a, b = torch.full((2, 2, 300), -1.0, device="cuda"), torch.full((2, 2, 300), -1.0, device="cuda")
    slim.slim_attn_decode_weights(cache, q, out, None, a, None, lens, 2, 300, 8, D ** -0.5, 1.0, ws)
    start = torch.rand((2, 2, 300), generator=gen(2)).cuda()
    b.copy_(start)
    slim.slim_attn_decode_weights(cache, q, out, b, b, i32([300, 40]), lens, 2, 300, 8, D ** -0.5, 1.0, ws)
    torch.cuda.synchronize()
    assert torch.equal(b[0], start[0] + a[0]) and torch.equal(b[1, :, :40], start[1, :, :40] + a[1, :, :40])
    assert torch.equal(b[1, :, 40:], start[1, :, 40:]) and (a[1, :, 40:] == -1.0).all()
    assert abs(a[0, 0].double().sum().item() - 4) < 1e-4    # four query heads per kv head


# ================================================================== eviction
def evict_reference(w, pos, n, budget, sink, recent, seen, placed):
    """numpy: (slots kept in their new order: source slot of every slot < min(n, budget), positions)."""
    p = np.array([pos[s] if s < placed else seen - n + s for s in range(n)], dtype=np.int64)
    if n <= budget:
        return np.arange(n), p
    safe = (p < sink) | (p >= seen - recent)
    key = np.where(np.isnan(w), -np.inf, w.astype(np.float64))
    order = sorted(range(n), key=lambda s: (not safe[s], -key[s], s))
    keep = np.zeros(n, dtype=bool)
    keep[order[:budget]] = True
    src = np.arange(budget)
    src[~keep[:budget]] = np.arange(budget, n)[keep[budget:]]
    return src, p[src]


EVICT_CASES = [
    # lengths, hkv, budget, sink, recent, placed, in place
    ([1], 1, 1, 0, 0, None, False), ([2], 1, 1, 0, 0, None, False), ([2, 1, 0], 2, 1, 1, 0, [1, 0, 0], True), ([129, 128, 127], 3, 128, 4, 32, [128, 128, 100], True),
    ([300, 45, 1000], 2, 40, 3, 17, [0, 45, 77], False), ([1000, 700], 1, 999, 0, 999, None, False), ([513], 2, 512, 0, 0, None, True),
    ([4100, 2000], 2, 1024, 4, 256, [1024, 1024], False), ([9001], 2, 9000, 4, 64, [9000], True), ([20000, 12000], 1, 500, 0, 0, [500, 0], False),
    ([260] * 9, 5, 130, 0, 10, None, False), ([60001], 1, 3000, 16, 100, [3000], True), ([55000], 1, 54990, 0, 0, None, False),
    ([16385, 70000], 1, 2000, 4, 300, [2000, 2000], True), ([66000], 1, 65990, 0, 0, None, False), ([65536], 1, 32768, 0, 0, [32768], False),
    ([8193, 3], 2, 100, 1, 1, None, True),
    ([131072], 1, 65535, 4, 64, None, True), ([131071, 70000], 1, 4000, 4, 64, [4000, 0], False), ([131072], 1, 65536, 0, 10, [65536], False),
    ([140001, 131073], 1, 30000, 4, 64, [30000, 100], True),
]


def evict_inputs(seed, lens, hkv, stride, placed, seen, kind):
    g = gen(seed)
    B = len(lens)
    w = torch.exp(3 * torch.randn((B, hkv, stride), generator=g))
    if kind == "ties":
        w = torch.floor(w)                                   # many equal ones, many zeros
    if kind == "odd":
        pick = torch.rand((B, hkv, stride), generator=g)
        w[pick < 0.05] = float("nan")
        w[(pick >= 0.05) & (pick < 0.1)] = float("inf")
        w[(pick >= 0.1) & (pick < 0.2)] = float("-inf")
        w[(pick >= 0.2) & (pick < 0.4)] *= -1
        w[(pick >= 0.4) & (pick < 0.5)] = -0.0
        w[(pick >= 0.5) & (pick < 0.6)] = 0.0
        w[(pick >= 0.6) & (pick < 0.65)] = 1e-42             # subnormal
    pos = torch.full((B, hkv, stride), -9, dtype=torch.int32)
    for b in range(B):
        p = placed[b] if placed else 0
        for h in range(hkv):
            pos[b, h, :p] = torch.randperm(seen[b] - (lens[b] - p), generator=g)[:p].to(torch.int32)
    return w, pos


@pytest.mark.parametrize("kind", ["plain", "ties", "odd"])
@pytest.mark.parametrize("case", EVICT_CASES, ids=range(len(EVICT_CASES)))
def test_evict(case, kind):
    lens, hkv, budget, sink, recent, placed, in_place = case
    slim = _slim()
    B, top = len(lens), max(lens)
    stride = top + 5
    mp = (top + PAGE - 1) // PAGE
    seen = [n + (1000 if placed else 0) for n in lens]
    w, pos = evict_inputs(top + budget, lens, hkv, stride, placed, seen, kind)
    table = torch.randperm(B * mp, generator=gen(2)).to(torch.int32).view(B, mp)
    cache = slim.SlimCache(B, hkv, mp, block_table=table)
    fill(cache, 3)
    codes0, scales0 = cache.codes_view().cpu().clone(), cache.scales_view().cpu().clone()
    wi, pi = w.cuda(), pos.cuda()
    wo, po = (wi, pi) if in_place else (torch.full_like(wi, -5.0), torch.full_like(pi, -5))
    ws = slim.evict_workspace(B, hkv, top, budget)
    ws.fill_(255)
    slim.slim_kv_evict(cache, wi, wo, pi if placed else None, po, i32(lens), i32(placed) if placed else None, i32(seen) if placed else None, B, top, budget,
                       sink, recent, ws)
    torch.cuda.synchronize()
    codes, scales = cache.codes_view().cpu(), cache.scales_view().cpu()
    same_w = lambda a, b: torch.equal(a.view(torch.int32), b.view(torch.int32))  # noqa: E731
    flat = lambda b: torch.tensor([[int(table[b, s // PAGE]), s % PAGE] for s in range(mp * PAGE)])  # noqa: E731
    for b, n in enumerate(lens):
        at = flat(b)
        for h in range(hkv):
            src, p = evict_reference(w[b, h].numpy(), pos[b, h].numpy(), n, budget, sink, recent, seen[b], placed[b] if placed else 0)
            m = len(src)
            assert po[b, h, :m].cpu().tolist() == p.tolist(), (b, h)
            assert same_w(wo[b, h, :m].cpu(), w[b, h, torch.from_numpy(src)])
            rest_w, rest_p = (w[b, h, m:], pos[b, h, m:]) if in_place else (torch.full((stride - m,), -5.0), torch.full((stride - m,), -5, dtype=torch.int32))
            if not (in_place and not placed):
                assert same_w(wo[b, h, m:].cpu(), rest_w) and torch.equal(po[b, h, m:].cpu(), rest_p)
            frm = np.arange(mp * PAGE)
            frm[:m] = src
            a, f = at, at[torch.from_numpy(frm)]
            assert torch.equal(codes[a[:, 0], h, :, a[:, 1]], codes0[f[:, 0], h, :, f[:, 1]])
            assert torch.equal(scales[a[:, 0], h, :, a[:, 1]], scales0[f[:, 0], h, :, f[:, 1]])


# ================================================================== together
def test_serving_sequence():
    """A prompt normed, rotated and appended, attended; decode steps that weigh the tokens; evictions between them; more steps on
    the cut cache: every output against the 64-bit attention over the cache's own rows, positions against a simulation."""
    slim = _slim()
    from paper_2407_07304_b200 import harness, workloads
    hq, hkv, B, budget, recent, sink = 8, 2, 3, 96, 20, 2
    prompt, steps = [150, 97, 40], 90
    g = gen(77)
    half = 64
    inv = torch.tensor([10000.0 ** (-i / half) for i in range(half)], dtype=torch.float64)
    wq, wk = ((1 + 0.1 * torch.randn(D, generator=g)).to(torch.bfloat16) for _ in range(2))
    run = harness.RotatedRun(B, hq, hkv, max_tokens=256, inv_freq=inv, q_weight=wq, k_weight=wk, budget=budget, n_sink=sink, n_recent=recent)
    qkv = torch.randn((sum(prompt), hq + 2 * hkv, D), generator=g).to(torch.bfloat16).cuda()
    outs = run.prompt(qkv, prompt)
    q_ref = rope_reference(qkv[:, :hq], wq, 1e-6, torch.cat([torch.arange(n) for n in prompt])[None], torch.zeros(half), inv, False)
    at = 0
    for b, n in enumerate(prompt):
        k, v = rows_of(run.cache, b, n)
        s = torch.einsum("thgd,hnd->thgn", q_ref[at:at + n].to(torch.bfloat16).double().cuda().view(n, hkv, hq // hkv, D), k) * D ** -0.5
        s = s.masked_fill(torch.arange(n, device="cuda")[None, None, None] > torch.arange(n, device="cuda")[:, None, None, None], -math.inf)
        p = torch.softmax(s, -1)
        want = torch.einsum("thgn,hnd->thgd", p, v).reshape(n, hq, D)
        top = torch.einsum("thgn,hnd->thgd", p, v.abs()).amax(-1, keepdim=True).reshape(n, hq, 1)
        # the query itself may round the other way (2^-8 of it): it moves a score by 2^-8 |q||k| sm_scale at worst
        err = (outs[b].double() - want).abs()
        assert (err <= want.abs() * 2.0 ** -8 + top * 2.0 ** -5).all()
        at += n
    kept = [[list(range(n)) for _ in range(hkv)] for n in prompt]       # positions in slot order
    seen = list(prompt)
    weights = [[np.zeros(n) for _ in range(hkv)] for n in prompt]
    for step in range(steps):
        qkv = torch.randn((B, hq + 2 * hkv, D), generator=g).to(torch.bfloat16).cuda()
        out = run.step(qkv)
        for b in range(B):
            for h in range(hkv):
                kept[b][h].append(seen[b])
            seen[b] += 1
        want, probs, top = attend(run.cache, run.q_last, run.lens, D ** -0.5)
        out_close(out, want, top, step)
        for b in range(B):
            n = run.lens[b]
            for h in range(hkv):
                w = np.concatenate([weights[b][h], [0.0]]) + probs[b].view(hkv, hq // hkv, n)[h].sum(0).cpu().numpy()
                got = run.weights[b, h, :n].double().cpu().numpy()
                assert np.abs(got - w).max() <= 1e-3 and len(kept[b][h]) == n
                weights[b][h] = got                                      # selection goes by the library's own fp32 sums
        if step % 16 == 15:
            run.evict()
            for b in range(B):
                for h in range(hkv):
                    src, p = evict_reference(weights[b][h].astype(np.float32), np.array(kept[b][h]), len(kept[b][h]), budget, sink, recent, seen[b], len(kept[b][h]))
                    kept[b][h] = p.tolist()
                    weights[b][h] = weights[b][h][src]
                assert run.lens[b] == len(kept[b][0]) <= budget
                assert all(run.positions[b, h, :run.lens[b]].cpu().tolist() == kept[b][h] for h in range(hkv))
    assert all(n > budget for n in seen)


def test_on_another_stream_and_in_a_graph():
    """Every call captured into one graph on a stream of its own and replayed twice: the results of plain calls."""
    slim = _slim()
    B, hq, hkv = 4, 8, 2
    cache, _, cu = shared_setup(6, [(2, B)], hq, hkv, 2)
    rows, inv, axis, pos, w = rope_inputs(9, B, hq, hkv, 128, 1, True)
    nr = slim.NormRope(inv, w[0], w[1])
    lens, shared, cu_group = i32([300, 257, 256, 290]), i32([256] * B), i32(cu)
    start = lens - 1
    ones = i32(list(range(B + 1)))
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    ws1, ws2, ws3 = slim.shared_workspace(B, hq, hkv, 1, B, 256, 64), slim.weights_workspace(B, hq, hkv, 300), slim.evict_workspace(B, hkv, 300, 200)
    own = slim.SlimCache(B, hkv, 3)
    fill(own, 2)
    state = {n: t for n, t in (("codes", own.codes.clone()), ("scales", own.scales.clone()))}

    def fresh():
        return dict(qo=torch.zeros((B, hq, D), dtype=torch.bfloat16, device="cuda"), kk=torch.zeros((B, hkv, D), dtype=torch.bfloat16, device="cuda"),
                    o1=torch.zeros((B, hq, D), dtype=torch.bfloat16, device="cuda"), o2=torch.zeros((B, hq, D), dtype=torch.bfloat16, device="cuda"),
                    wt=torch.zeros((B, hkv, 300), device="cuda"), wo=torch.zeros((B, hkv, 300), device="cuda"),
                    po=torch.zeros((B, hkv, 300), dtype=torch.int32, device="cuda"))

    def calls(t):
        slim.slim_norm_rope(nr, q, t["qo"], k, t["kk"], pos)
        slim.slim_norm_rope_append(own, nr, q, t["qo"], k, v, pos, ones, start, B)
        slim.slim_attn_decode_shared(cache, t["qo"], t["o1"], cu_group, shared, lens, 1, B, B, 256, 64, hq, D ** -0.5, ws1)
        slim.slim_attn_decode_weights(own, t["qo"], t["o2"], None, t["wt"], None, lens, B, 300, hq, D ** -0.5, 1.0, ws2)
        slim.slim_kv_evict(own, t["wt"], t["wo"], None, t["po"], lens, None, None, B, 300, 200, 1, 8, ws3)

    def restore():
        own.codes.copy_(state["codes"])
        own.scales.copy_(state["scales"])

    a, b = fresh(), fresh()
    calls(a)
    torch.cuda.synchronize()
    after = own.codes.clone()
    restore()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls(b)
    for _ in range(2):
        restore()
        for t in b.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(own.codes, after)
        for name in a:
            assert torch.equal(a[name], b[name]), name
    restore()
    c = fresh()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        calls(c)
    side.synchronize()
    assert torch.equal(own.codes, after) and all(torch.equal(a[name], c[name]) for name in a)
    for ws in (ws1, ws2):
        assert slim.slim_read_status(ws) == slim.SLIM_OK


def test_results_repeat_bit_for_bit():
    slim = _slim()
    cache, B, cu = shared_setup(8, [(9, 12), (3, 20)], 16, 4, 2)
    q = torch.randn((B, 16, D), generator=gen(8)).to(torch.bfloat16).cuda()
    pre = [9 * PAGE] * 12 + [3 * PAGE] * 20
    lens = [p + 1 + 7 * i for i, p in enumerate(pre)]
    first = None
    for _ in range(5):
        out, wt = torch.empty_like(q), torch.zeros((B, 4, max(lens)), device="cuda")
        ws = slim.shared_workspace(B, 16, 4, 2, 20, 9 * PAGE, 256)
        slim.slim_attn_decode_shared(cache, q, out, i32(cu), i32(pre), i32(lens), 2, B, 20, 9 * PAGE, 256, 16, D ** -0.5, ws)
        o2 = torch.empty_like(q)
        slim.slim_attn_decode_weights(cache, q, o2, None, wt, None, i32(lens), B, max(lens), 16, D ** -0.5, 1.0, slim.weights_workspace(B, 16, 4, max(lens)))
        torch.cuda.synchronize()
        if first is None:
            first = (out, o2, wt)
        assert all(torch.equal(x, y) for x, y in zip(first, (out, o2, wt)))


def test_pages_behind_four_gigabytes():
    """A pool of 4.6 GB of codes whose last pages are the ones in use: offsets beyond 2^32 in every call."""
    slim = _slim()
    n_pages, B, hq, hkv, mp = 140000, 2, 4, 1, 4
    table = torch.arange(n_pages - B * mp, n_pages, dtype=torch.int32).view(B, mp)
    table[1, :2] = table[0, :2]                              # a shared prefix of two pages
    cache = slim.SlimCache(B, hkv, mp, block_table=table, num_pages=n_pages)
    rows, inv, axis, pos, w = rope_inputs(21, 900, hq, hkv, 128, 1, True)
    qo = torch.empty((900, hq, D), dtype=torch.bfloat16, device="cuda")
    slim.slim_norm_rope_append(cache, slim.NormRope(inv, w[0], w[1]), rows[:, :hq], qo, rows[:, hq:hq + 1], rows[:, hq + 1:], pos, i32([0, 450, 900]),
                               i32([0, 0]), B)
    torch.cuda.synchronize()
    assert (cache.codes_view()[n_pages - B * mp].abs().amax(-1) > 0).all() and not cache.codes_view()[:1000].any()
    lens, q = [450, 300], qo[:2].contiguous()
    want, probs, slack = attend(cache, q, lens, D ** -0.5)
    out = torch.empty_like(q)
    ws = slim.shared_workspace(B, hq, hkv, 1, B, 256, 256)
    slim.slim_attn_decode_shared(cache, q, out, i32([0, 2]), i32([256, 256]), i32(lens), 1, B, B, 256, 256, hq, D ** -0.5, ws)
    out2, wt = torch.empty_like(q), torch.zeros((B, hkv, 450), device="cuda")
    slim.slim_attn_decode_weights(cache, q, out2, None, wt, None, i32(lens), B, 450, hq, D ** -0.5, 1.0, slim.weights_workspace(B, hq, hkv, 450))
    torch.cuda.synchronize()
    out_close(out, want, slack, "shared")
    out_close(out2, want, slack, "weights")
    assert (wt[0, 0].double() - probs[0].sum(0)).abs().max() < 1e-4
    # the first sequence alone is cut (the second's prefix pages are not its own)
    before = cache.codes_view()[table[0].long().cuda()].clone()
    alone = slim.SlimCache(1, hkv, mp, block_table=table[:1], num_pages=n_pages)
    alone.codes, alone.scales = cache.codes, cache.scales
    alone.struct.codes, alone.struct.scales = cache.codes.data_ptr(), cache.scales.data_ptr()
    po, wo = torch.zeros((1, hkv, 450), dtype=torch.int32, device="cuda"), torch.zeros((1, hkv, 450), device="cuda")
    slim.slim_kv_evict(alone, wt[:1].contiguous(), wo, None, po, i32([450]), None, None, 1, 450, 200, 0, 0, slim.evict_workspace(1, hkv, 450, 200))
    torch.cuda.synchronize()
    src, p = evict_reference(wt[0, 0].cpu().numpy(), np.arange(450), 450, 200, 0, 0, 450, 0)
    assert po[0, 0, :200].cpu().tolist() == p.tolist()
    flat = before.permute(1, 2, 0, 3, 4).reshape(2, mp * PAGE, D)
    after = cache.codes_view()[table[0].long().cuda()].permute(1, 2, 0, 3, 4).reshape(2, mp * PAGE, D)
    assert torch.equal(after[:, :200], flat[:, torch.from_numpy(src).cuda()]) and torch.equal(after[:, 200:], flat[:, 200:])


def test_one_workspace_for_calls_of_different_kinds():
    """A zeroed workspace serves ordinary, shared and weighted decode of different shapes in turn, its header back at zero."""
    slim = _slim()
    cache, B, cu = shared_setup(4, [(3, 6)], 8, 2, 2)
    q = torch.randn((B, 8, D), generator=gen(14)).to(torch.bfloat16).cuda()
    lens = [384 + 30 * b for b in range(B)]
    want, _, slack = attend(cache, q, lens, D ** -0.5)
    n = max(w.numel() for w in (slim.shared_workspace(B, 8, 2, 1, B, 384, 256), slim.weights_workspace(B, 8, 2, 640), slim.workspace(slim.PHASE_DECODE, B, 8, 2, 1, 640)))
    ws = torch.full((n,), 0xEE, dtype=torch.uint8, device="cuda")
    ws[:slim.WORKSPACE_HEADER_BYTES] = 0
    wt = torch.zeros((B, 2, 640), device="cuda")
    for _ in range(2):
        for call in ("shared", "weights", "decode", "shared", "decode", "weights"):
            out = torch.full_like(q, 3.0)
            if call == "shared":
                slim.slim_attn_decode_shared(cache, q, out, i32(cu), i32([384] * B), i32(lens), 1, B, B, 384, 256, 8, D ** -0.5, ws)
            elif call == "weights":
                slim.slim_attn_decode_weights(cache, q, out, None, wt, None, i32(lens), B, 640, 8, D ** -0.5, 1.0, ws)
            else:
                slim.slim_attn_decode(cache, q, out, i32(lens), B, 640, 8, D ** -0.5, ws)
            torch.cuda.synchronize()
            out_close(out, want, slack, call)
            assert slim.slim_read_status(ws) == slim.SLIM_OK and not ws[:slim.WORKSPACE_HEADER_BYTES].any()


def test_two_streams_at_once():
    """The same calls on two streams that nothing orders, each with buffers of its own: the results of calls in turn."""
    slim = _slim()
    sets = []
    for k in range(2):
        cache, B, cu = shared_setup(30 + k, [(6, 10)], 16, 4, 2)
        own = slim.SlimCache(B, 4, 8)
        fill(own, 40 + k)
        q = torch.randn((B, 16, D), generator=gen(50 + k)).to(torch.bfloat16).cuda()
        sets.append(dict(cache=cache, own=own, q=q, cu=i32(cu), shared=i32([768] * B), lens=i32([768 + 20 * b for b in range(B)]), B=B,
                         w1=slim.shared_workspace(B, 16, 4, 1, B, 768, 256), w2=slim.weights_workspace(B, 16, 4, 1024), w3=slim.evict_workspace(B, 4, 1024, 700),
                         codes=own.codes.clone(), scales=own.scales.clone()))

    def calls(s):
        o1, o2 = torch.empty_like(s["q"]), torch.empty_like(s["q"])
        wt = torch.zeros((s["B"], 4, 1024), device="cuda")
        wo, po = torch.zeros_like(wt), torch.zeros((s["B"], 4, 1024), dtype=torch.int32, device="cuda")
        for _ in range(8):
            slim.slim_attn_decode_shared(s["cache"], s["q"], o1, s["cu"], s["shared"], s["lens"], 1, s["B"], s["B"], 768, 256, 16, D ** -0.5, s["w1"])
            slim.slim_attn_decode_weights(s["own"], s["q"], o2, None, wt, None, s["lens"], s["B"], 1024, 16, D ** -0.5, 1.0, s["w2"])
        slim.slim_kv_evict(s["own"], wt, wo, None, po, s["lens"], None, None, s["B"], 1024, 700, 4, 32, s["w3"])
        return o1, o2, wt, wo, po

    turn = []
    for s in sets:
        turn.append(calls(s))
        torch.cuda.synchronize()
        s["after"] = s["own"].codes.clone()
        s["own"].codes.copy_(s["codes"])
        s["own"].scales.copy_(s["scales"])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    both = []
    for s, st in zip(sets, streams):
        with torch.cuda.stream(st):
            both.append(calls(s))
    torch.cuda.synchronize()
    for s, a, b in zip(sets, turn, both):
        assert all(torch.equal(x, y) for x, y in zip(a, b)) and torch.equal(s["own"].codes, s["after"])


def test_long_eviction_in_a_graph():
    """The cluster form and its move kernel, captured and replayed."""
    slim = _slim()
    n, budget = 20000, 5000
    w, _ = evict_inputs(5, [n], 2, n, None, [n], "ties")
    cache = slim.SlimCache(1, 2, (n + PAGE - 1) // PAGE)
    fill(cache, 6)
    codes = cache.codes.clone()
    wi, wo, po = w.cuda(), torch.zeros((1, 2, n), device="cuda"), torch.zeros((1, 2, n), dtype=torch.int32, device="cuda")
    lens, ws = i32([n]), slim.evict_workspace(1, 2, n, budget)
    call = lambda: slim.slim_kv_evict(cache, wi, wo, None, po, lens, None, None, 1, n, budget, 4, 100, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    a = (cache.codes.clone(), wo.clone(), po.clone())
    assert a[2][0, 0, :budget].cpu().tolist() == evict_reference(w[0, 0].numpy(), np.arange(n), n, budget, 4, 100, n, 0)[1].tolist()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(2):
        cache.codes.copy_(codes)
        wo.zero_()
        po.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a, (cache.codes, wo, po)))


@pytest.mark.parametrize("lens,budget", [([70000], 30000), ([66001, 90000], 45000), ([140000], 60000), ([150001, 131080], 70000)])
def test_long_eviction_with_one_side_in_place(lens, budget):
    """Weights in place and positions written anew (a sequence's first eviction), or the other way round: no walk over a
    row may take what another thread has just moved into a freed slot for the token that was there."""
    slim = _slim()
    B, top = len(lens), max(lens)
    w, _ = evict_inputs(top + budget, lens, 1, top, None, lens, "ties")
    cache = slim.SlimCache(B, 1, (top + PAGE - 1) // PAGE)
    ws = slim.evict_workspace(B, 1, top, budget)
    want = [evict_reference(w[b, 0].numpy(), np.arange(n), n, budget, 4, 300, n, 0) for b, n in enumerate(lens)]
    placed = i32(lens)
    for weights_in_place in (True, False) * 4:
        wi = w.cuda()
        pi = torch.arange(top, dtype=torch.int32, device="cuda").repeat(B, 1, 1).contiguous()
        wo, po = (wi, torch.zeros_like(pi)) if weights_in_place else (torch.zeros_like(wi), pi)
        slim.slim_kv_evict(cache, wi, wo, None if weights_in_place else pi, po, i32(lens), None if weights_in_place else placed, None, B, top, budget, 4, 300, ws)
        torch.cuda.synchronize()
        for b in range(B):
            src, p = want[b]
            assert torch.equal(po[b, 0, :budget].cpu(), torch.from_numpy(p.astype(np.int32)))
            assert torch.equal(wo[b, 0, :budget].cpu(), w[b, 0, torch.from_numpy(src)])


@pytest.mark.parametrize("into", [1, 64, 127])
def test_decode_shared_prefix_that_ends_inside_a_page(into):
    """Counted in whole pages: the page that is shared in part is the tails' (a call of the same bounds gives the same bits)."""
    slim = _slim()
    hq, hkv = 16, 2
    cache, B, cu = shared_setup(into, [(3, 4), (0, 1), (1, 2)], hq, hkv, 4)
    pre = [384] * 4 + [0] + [128] * 2
    lens = [n + 130 + 7 * b for b, n in enumerate(pre)]
    max_tail = max(n - p for n, p in zip(lens, pre))
    q = torch.randn((B, hq, D), generator=gen(into)).to(torch.bfloat16).cuda()
    outs = []
    for extra in (0, into):
        out = torch.full_like(q, 5.0)
        ws = slim.shared_workspace(B, hq, hkv, 3, 4, 384 + extra, max_tail)
        slim.slim_attn_decode_shared(cache, q, out, i32(cu), i32([p + extra for p in pre]), i32(lens), 3, B, 4, 384 + extra, max_tail, hq, D ** -0.5, ws)
        torch.cuda.synchronize()
        assert slim.slim_read_status(ws) == 0
        outs.append(out)
    assert torch.equal(*outs) and not (outs[0] == 5.0).all(-1).any()


def test_decode_shared_prefix_of_less_than_a_page_is_decode():
    slim = _slim()
    hq, hkv, lens = 8, 4, [300, 77, 1]
    cache, B, cu = shared_setup(4, [(1, 3)], hq, hkv, 3)
    q = torch.randn((B, hq, D), generator=gen(9)).to(torch.bfloat16).cuda()
    a, b = torch.full_like(q, 5.0), torch.full_like(q, 5.0)
    slim.slim_attn_decode_shared(cache, q, a, i32(cu), i32([127] * 3), i32(lens), 1, B, 3, 127, 300, hq, D ** -0.5, slim.shared_workspace(B, hq, hkv, 1, 3, 127, 300))
    slim.slim_attn_decode(cache, q, b, i32(lens), B, 300, hq, D ** -0.5, slim.workspace(slim.PHASE_DECODE, B, hq, hkv, 1, 300))
    torch.cuda.synchronize()
    assert torch.equal(a, b)
