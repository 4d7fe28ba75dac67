"""The 4-bit cache and the page tables at sizes far from the ordinary ones."""
import pytest
import torch

import test_pages
from paper_2407_07304_b200 import binding as slim
from test_cache4 import D, check_prefill, close, decode_bound, filled, i32, offsets, reference, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 1), (16, 1)])
def test_decode_of_units_apart(hq, hkv):
    """Units of 64 tokens whose values differ by orders of magnitude: a sequence that begins with zeros, with constant rows, with tiny
    and with large values.  Beside test_cache4's bound a weight times its scale may fall below fp16's smallest step, 2^-24 of
    a number scaled so that the largest scale counts 2^9 or more: 15 x 2^-34 of that scale per token."""
    gen = torch.Generator().manual_seed(hq)
    factors = [[0.0, 1.0, 30.0], [1e-30, 1e-3, 100.0], [1e3, 1.0, 1e-3], [1.0, 0.0, 1e-25]]
    lens = [64 * len(f) + 17 for f in factors]
    cache, k, v = filled(gen, lens, hkv)
    v = v.float()
    cu = offsets(lens)
    for b, f in enumerate(factors):
        for t, x in enumerate(f):
            v[cu[b] + 64 * t:cu[b] + 64 * (t + 1)] *= x
    v[cu[1] + 5] = 3e-20
    v[cu[3]:cu[3] + 64] = -1.5      # a whole unit of scale 0
    k = k.float() / 8
    slim.slim_kv4_append(cache, k.to(torch.bfloat16).cuda(), v.to(torch.bfloat16).cuda(), i32(cu), i32([0] * len(lens)), len(lens), max(lens))
    q = torch.randn(len(lens), hq, D, generator=gen).to(torch.bfloat16).cuda()
    out = torch.empty_like(q)
    slim.slim_attn4_decode(cache, q, out, i32(lens), len(lens), max(lens), hq, D ** -0.5, slim.decode4_workspace(len(lens), hq, hkv, max(lens)))
    for b, n in enumerate(lens):
        want, parts = reference(cache, b, n, q[b:b + 1], D ** -0.5)
        close(out[b:b + 1], want, decode_bound(want, parts) + n * 15 * 2.0 ** -34 * parts[3][..., None])


@pytest.mark.parametrize("hq", [64, 129, 300])
def test_prefill_of_many_heads_per_kv_head(hq):
    """More heads per kv head than a block has rows, and numbers that leave a token's heads in two blocks."""
    gen = torch.Generator().manual_seed(hq)
    counts, lens = [5, 1, 3], [5, 200, 130]
    cache, _, _ = filled(gen, lens, 1)
    q = torch.randn(sum(counts), hq, D, generator=gen).to(torch.bfloat16).cuda()
    out = torch.full_like(q, 9.0)
    slim.slim_attn4_prefill(cache, q, out, i32(offsets(counts)), i32(lens), 3, 5, 200, hq, D ** -0.5, slim.workspace(slim.PHASE_PREFILL, 3, hq, 1, 5, 200))
    check_prefill(cache, counts, lens, q, out, D ** -0.5)


def test_the_largest_batch():
    """65535 sequences of none to three tokens."""
    gen = torch.Generator().manual_seed(1)
    b = 65535
    lens = torch.randint(0, 4, (b,), generator=gen)
    cu = torch.cat([torch.zeros(1, dtype=torch.long), lens.cumsum(0)])
    cache = slim.SlimCache4(b, 1, 1)
    v = rows(gen, int(cu[-1]), 1).cuda()
    k = torch.zeros_like(v)                      # equal scores: the mean of the values held
    args = (cu.to(torch.int32).cuda(), torch.zeros(b, dtype=torch.int32, device="cuda"), b, 3)
    slim.slim_kv4_append(cache, k, v, *args)
    back = [torch.empty_like(v) for _ in range(2)]
    slim.slim_kv4_read(cache, *back, *args)
    assert not back[0].any()
    q = torch.randn(b, 2, D, generator=gen).to(torch.bfloat16).cuda()
    out = torch.full_like(q, 9.0)
    ws = slim.decode4_workspace(b, 2, 1, 3)
    slim.slim_attn4_decode(cache, q, out, lens.to(torch.int32).cuda(), b, 3, 2, D ** -0.5, ws)
    assert slim.slim_read_status(ws) == slim.SLIM_OK
    owner = torch.repeat_interleave(torch.arange(b), lens).cuda()
    want = torch.zeros((b, D), dtype=torch.float64, device="cuda").index_add_(0, owner, back[1][:, 0].double())
    want = want / lens.clamp(min=1).double().cuda()[:, None]
    # a value read back is rounded to bf16 (2^-8 of it, 16 at most here), the result once more; weights in fp16 as in test_cache4
    err = (out.double() - want[:, None]).abs()
    size = torch.zeros((b, D), dtype=torch.float64, device="cuda").index_reduce_(0, owner, back[1][:, 0].double().abs(), "amax")
    span = size.amax(1, keepdim=True) * 2
    assert (err <= (2.0 ** -8 * (want.abs() + size) + 2.0 ** -11 * span + 2.0 ** -20 * span)[:, None]).all()


@pytest.mark.parametrize("num_pages,rows_", [(1500, 5), (60000, 7)])
def test_a_random_run_of_wide_tables(num_pages, rows_):
    test_pages.test_a_random_run(6, num_pages, rows_, 1000)


def test_tables_of_more_entries_than_31_bits():
    """2^22 + 1 rows of 513 pages: few of them held."""
    n, stride, pages = (1 << 22) + 1, 513, 40
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    a = slim.SlimPages.empty(pages, n, stride)
    kv_len = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    kv_len[0], kv_len[n // 2], kv_len[-1] = 130, 1, 700
    result, ws = i32([0, 0]), slim.pages_workspace(pages, n)
    slim.slim_pages_grow(a, kv_len, 0, result, ws)
    assert result.tolist() == [0, pages - 9] and a.table[-1, :7].tolist() == [3, 4, 5, 6, 7, 8, -1]
    b = slim.SlimPages.empty(pages, n, stride)
    parent = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    parent[-1], parent[-2], parent[1] = n - 1, n - 1, 0
    len_out = torch.empty_like(kv_len)
    slim.slim_pages_fork(None, a, b, parent, kv_len, len_out, result, ws)
    # row n - 2 is the heir of row n - 1, whose 700 tokens leave a part of a page to copy; page 2 is free again
    assert result.tolist() == [0, pages - 9] and b.table[-2, :7].tolist() == [3, 4, 5, 6, 7, 8, -1]
    assert b.table[-1, :7].tolist() == [3, 4, 5, 6, 7, 2, -1] and b.table[1, :3].tolist() == [0, 1, -1]
    assert b.refs[:10].tolist() == [1, 1, 1, 2, 2, 2, 2, 2, 1, 0] and len_out[[0, 1, n - 2, n - 1]].tolist() == [-1, 130, 700, 700]
    parent.fill_(-1)
    parent[-1] = n - 1
    slim.slim_pages_fork(None, b, a, parent, len_out, kv_len, result, ws)
    slim.slim_pages_compact(None, a, a, result, ws)
    assert result.tolist() == [6, 2] and a.table[-1, :7].tolist() == [3, 4, 5, 0, 1, 2, -1] and kv_len[-1] == 700
    assert a.table[0].max() == -1 and a.refs[:7].tolist() == [1] * 6 + [0]
