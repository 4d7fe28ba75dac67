"""Calls whose device-side lengths and groups pass the bounds given on the host: nothing behind the bounds is written, and no
output depends on what the workspace held."""
import pytest
import torch

from test_operators import D, PAGE, attend, fill, gen, i32, out_close, rows_of, shared_setup

pytestmark = pytest.mark.gpu


def _slim():
    from paper_2407_07304_b200 import binding
    return binding


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("max_kv,lens,hq,hkv", [
    (272, [300, 512, 272, 1000], 8, 2),      # lengths inside max_kv's last chunk, at its end, at max_kv, beyond the page table
    (1, [2, 1, 256], 3, 3),                  # one entry of weight per row
    (1025, [1026, 1280, 7], 16, 1),          # the last token block has room for one token
])
def test_weights_of_lengths_beyond_max_kv_stay_in_their_rows(max_kv, lens, hq, hkv, append):
    """A row of weights holds max_kv entries; the attention takes whole chunks of 256 tokens.  With rows that lie back to back a
    value too many lands in the next head's weights, and for the last row behind the array."""
    slim = _slim()
    B, mp, guard = len(lens), (max_kv + 255) // 256 * 2, 2048
    g = gen(max_kv)
    cache = slim.SlimCache(B, hkv, mp)
    fill(cache, max_kv)
    q = torch.randn((B, hq, D), generator=g).to(torch.bfloat16).cuda()
    new = {}
    if append:
        new = dict(k_new=torch.randn((B, hkv, D), generator=g).to(torch.bfloat16).cuda(), v_new=torch.randn((B, hkv, D), generator=g).to(torch.bfloat16).cuda())
    n = B * hkv * max_kv
    held = torch.full((2, guard + n + guard), -3.0, device="cuda")
    w_in, w_out = (h[guard:guard + n].view(B, hkv, max_kv) for h in held)
    w_in.copy_(torch.rand((B, hkv, max_kv), generator=g))
    weighed = i32([max_kv + 500] * B)                       # more than there is room for: every entry of the row counts
    out = torch.empty_like(q)
    ws = slim.weights_workspace(B, hq, hkv, max_kv)
    slim.slim_attn_decode_weights(cache, q, out, w_in, w_out, weighed, i32(lens), B, max_kv, hq, D ** -0.5, 0.5, ws, **new)
    torch.cuda.synchronize()
    assert slim.slim_read_status(ws) == slim.SLIM_OK
    assert (held[:, :guard] == -3.0).all() and (held[1, guard + n:] == -3.0).all()
    # the same attention with rows of weights that have room for all of it
    room = (max_kv + 255) // 256 * 256
    wide_in, wide_out, ref = torch.zeros((B, hkv, room), device="cuda"), torch.full((B, hkv, room), -3.0, device="cuda"), torch.empty_like(q)
    wide_in[..., :max_kv] = w_in
    slim.slim_attn_decode_weights(cache, q, ref, wide_in, wide_out, weighed, i32([min(x, room) for x in lens]), B, room, hq, D ** -0.5, 0.5,
                                  slim.weights_workspace(B, hq, hkv, room))
    torch.cuda.synchronize()
    assert torch.equal(out, ref)
    for b, x in enumerate(lens):
        m = min(x, max_kv)
        assert torch.equal(w_out[b, :, :m], wide_out[b, :, :m]) and (w_out[b, :, m:] == -3.0).all()
    _, probs, _ = attend(cache, q, [min(x, room) for x in lens], D ** -0.5)
    for b, x in enumerate(lens):
        m = min(x, max_kv)
        k, _ = rows_of(cache, b, min(x, room))
        p = probs[b].view(hkv, hq // hkv, -1).sum(1)[:, :m]
        want = 0.5 * w_in[b, :, :m].double() + p
        # a query element is held to 2^-21 of its row's largest power of two, twice for that power's spread: a score is off by
        # 2^-20 max|q| sum|k| sm_scale at most; six fp32 roundings of scores and exponents up to 64 in log2 units; the
        # denominator doubles it
        ds = D ** -0.5 * 2.0 ** -20 * q[b].double().abs().max() * k.abs().sum(-1).max() + 6 * 64 * 2.0 ** -24
        assert ((w_out[b, :, :m].double() - want).abs() <= 2 * ds * p + want * 2.0 ** -22 + 1e-30).all()


def test_one_workspace_from_the_first_step_to_the_longest_tail():
    """A loop allocates for its longest tail and passes each step's own bounds: the same bits as with a workspace of the step's own."""
    slim = _slim()
    hq, hkv = 16, 2
    cache, B, cu = shared_setup(71, [(24, 16)], hq, hkv, 17)
    q = torch.randn((B, hq, D), generator=gen(71)).to(torch.bfloat16).cuda()
    ws = slim.shared_workspace(B, hq, hkv, 1, B, 24 * PAGE, 2048)
    ws[slim.WORKSPACE_HEADER_BYTES:] = 0xEE
    for tail in (1, 2, 200, 256, 257, 700, 1024, 2048):
        lens = i32([24 * PAGE + max(1, tail - b) for b in range(B)])
        a, b = torch.full_like(q, 5.0), torch.full_like(q, 6.0)
        for out, w in ((a, ws), (b, slim.shared_workspace(B, hq, hkv, 1, B, 24 * PAGE, tail))):
            slim.slim_attn_decode_shared(cache, q, out, i32(cu), i32([24 * PAGE] * B), lens, 1, B, B, 24 * PAGE, tail, hq, D ** -0.5, w)
        torch.cuda.synchronize()
        assert torch.equal(a, b) and slim.slim_read_status(ws) == slim.SLIM_OK


@pytest.mark.parametrize("hq,hkv,n", [(16, 2, 4), (4, 4, 1), (16, 1, 20)])
def test_decode_shared_prefix_beyond_its_bound_is_the_sequences_own(hq, hkv, n):
    """A shared_len beyond max_shared counts as max_shared: the bits of a call whose lengths say so."""
    slim = _slim()
    cache, B, cu = shared_setup(n, [(9, n), (2, 1)], hq, hkv, 3)
    lens = [9 * PAGE + 5 + 11 * b for b in range(n)] + [400]
    q = torch.randn((B, hq, D), generator=gen(n)).to(torch.bfloat16).cuda()
    for bound in (4 * PAGE, 4 * PAGE + 17):
        tail = max(lens) - 4 * PAGE
        outs = []
        for shared in ([9 * PAGE] * n + [2 * PAGE], [4 * PAGE] * n + [2 * PAGE]):
            out = torch.full_like(q, 5.0)
            ws = slim.shared_workspace(B, hq, hkv, 2, n, bound, tail)
            ws[slim.WORKSPACE_HEADER_BYTES:] = 0xEE
            slim.slim_attn_decode_shared(cache, q, out, i32(cu), i32(shared), i32(lens), 2, B, n, bound, tail, hq, D ** -0.5, ws)
            torch.cuda.synchronize()
            assert slim.slim_read_status(ws) == slim.SLIM_OK
            outs.append(out)
        assert torch.equal(*outs)
        want, _, slack = attend(cache, q, lens, D ** -0.5)
        out_close(outs[0], want, slack, bound)


@pytest.mark.parametrize("append", [False, True])
def test_decode_shared_tails_beyond_their_bound_are_cut(append):
    """max_tail, rounded up to a multiple of 256 tokens, is what is attended behind the prefix; a new token behind it is not appended."""
    slim = _slim()
    hq, hkv, pre = 16, 2, 3 * PAGE
    cache, B, cu = shared_setup(3, [(3, 5)], hq, hkv, 8)
    lens = [pre + x for x in (700, 257, 256, 41, 512)]
    q = torch.randn((B, hq, D), generator=gen(3)).to(torch.bfloat16).cuda()
    new, before = {}, cache.codes.clone()
    if append:
        new = dict(k_new=torch.randn((B, hkv, D), generator=gen(4)).to(torch.bfloat16).cuda(), v_new=torch.randn((B, hkv, D), generator=gen(5)).to(torch.bfloat16).cuda())
    out = torch.full_like(q, 5.0)
    ws = slim.shared_workspace(B, hq, hkv, 1, B, pre, 40)
    slim.slim_attn_decode_shared(cache, q, out, i32(cu), i32([pre] * B), i32(lens), 1, B, B, pre, 40, hq, D ** -0.5, ws, **new)
    torch.cuda.synchronize()
    assert slim.slim_read_status(ws) == slim.SLIM_OK
    want, _, slack = attend(cache, q, [min(x, pre + 256) for x in lens], D ** -0.5)
    out_close(out, want, slack, "cut")
    for b, x in enumerate(lens):
        same = torch.equal(cache.codes_view()[cache.block_table[b, 3:].long()], before.view_as(cache.codes_view())[cache.block_table[b, 3:].long()])
        assert same == (not append or x > pre + 256)


@pytest.mark.parametrize("hq,hkv,pre_pages,tail", [
    (16, 2, 4, 300),        # partials merged by a warp per row
    (1, 1, 2, 1),
    (4, 2, 4, 40 * 256),    # by a block per row
    (2, 2, 2, 300 * 256),   # by the general kernel
])
def test_decode_shared_group_beyond_max_group_attends_its_tails(hq, hkv, pre_pages, tail):
    """More sequences in a group than max_group, and sequences in no group: no prefix for them, and nothing that the workspace
    held before; the others as ever."""
    slim = _slim()
    n, most, pre = 5, 3, pre_pages * PAGE
    B = 3 * n
    mp = pre_pages + (tail + PAGE - 1) // PAGE
    table = torch.arange(pre_pages + mp, dtype=torch.int32)
    # (long tails may lie in the same pages: nothing is appended)
    table = torch.cat([table[:pre_pages], table[pre_pages:pre_pages + mp - pre_pages]]).repeat(B, 1)
    cache = slim.SlimCache(B, hkv, mp, block_table=table, num_pages=pre_pages + mp)
    fill(cache, pre_pages)
    q = torch.randn((B, hq, D), generator=gen(hq)).to(torch.bfloat16).cuda()
    lens = [pre + (0, 1, 130, tail, max(1, tail - 1))[b % 5] for b in range(B)]
    lens = [min(x, pre + tail) for x in lens]
    cu = i32([2, 2 + n, 2 * n, 2 * n + 3, B - 2, B - 2, B - 2])            # five groups of at most max_group, one of five; the first and last two sequences in none
    groups = 6
    outs = []
    for junk in (0xFF, 0x41):                               # NaN, and a large number
        out = torch.full_like(q, 5.0)
        ws = slim.shared_workspace(B, hq, hkv, groups, most, pre, tail)
        ws[slim.WORKSPACE_HEADER_BYTES:] = junk
        slim.slim_attn_decode_shared(cache, q, out, cu, i32([pre] * B), i32(lens), groups, B, most, pre, tail, hq, D ** -0.5, ws)
        torch.cuda.synchronize()
        assert slim.slim_read_status(ws) == slim.SLIM_OK
        outs.append(out)
    assert torch.equal(*outs)
    alone = {0, 1, B - 2, B - 1, 2 + most, 2 + most + 1}    # no group, or beyond the first group's three
    want, _, slack = attend(cache, q, lens, D ** -0.5)
    behind = slim.SlimCache(B, hkv, mp - pre_pages, block_table=table[:, pre_pages:], num_pages=cache.num_pages)
    behind.codes, behind.scales = cache.codes, cache.scales
    own, _, own_slack = attend(behind, q, [x - pre for x in lens], D ** -0.5)
    for b in alone:
        want[b], slack[b] = own[b], own_slack[b]
        if lens[b] == pre:
            assert (outs[0][b] == 0).all()
    out_close(outs[0], want, slack, "groups")
