"""SampledRun: which rows a step takes, and what it refuses."""
import pytest
import torch

from paper_2407_07304_b200 import harness


def bf16(*shape, gen=None, device="cpu"):
    return torch.randn(*shape, generator=gen).to(torch.bfloat16).to(device)


@pytest.mark.parametrize("lens,counts", [([5, 7, -1], [1, 0, 0]), ([5, 256, -1], [0, 0, 0]), ([5, 7, -1], [2, 1, 0]), ([5, -1, -1], [5, 0, 0])])
def test_step_refuses_rows_without_one_new_token(lens, counts):
    """The new token's row goes to the length's last position: without a place of its own it would overwrite a token."""
    run = harness.SampledRun(1, 4, 2, num_pages=8, rows=3, max_tokens=512, device="cpu")
    run.lens, run.counts = lens, counts
    with pytest.raises(ValueError):
        run.step(0, bf16(3, 4, 128), bf16(3, 2, 128), bf16(3, 2, 128))


def test_a_fork_ends_the_step():
    run = harness.SampledRun(1, 4, 2, num_pages=8, rows=2, max_tokens=512, device="cpu")
    with pytest.raises(ValueError):      # nothing announced yet
        run.prompt(0, bf16(3, 4, 128), bf16(3, 2, 128), bf16(3, 2, 128))
    run.lens, run.counts = [3, 3], [1, 1]
    run._forked([1, -1])
    assert run.lens == [3, -1] and run.counts == [0, 0]
    for call in (run.step, run.prompt):
        with pytest.raises(ValueError):
            call(0, bf16(2, 4, 128), bf16(2, 2, 128), bf16(2, 2, 128))


@pytest.mark.parametrize("q,k,v", [(4, 5, 5), (6, 5, 5), (5, 4, 5), (5, 5, 4)])
def test_rows_as_announced(q, k, v):
    run = harness.SampledRun(1, 4, 2, num_pages=8, rows=3, max_tokens=512, device="cpu")
    run.lens, run.counts = [2, 3, -1], [2, 3, 0]
    with pytest.raises(ValueError):
        run.prompt(0, bf16(q, 4, 128), bf16(k, 2, 128), bf16(v, 2, 128))
    run.lens, run.counts = [2, 3, -1, 1, 1], [1, 1, 0, 1, 1]
    run.rows = 5
    with pytest.raises(ValueError):
        run.step(0, bf16(q, 4, 128), bf16(k, 2, 128), bf16(v, 2, 128))


@pytest.mark.parametrize("bits", [4, 8])
def test_empty_rows_give_zeros(bits):
    run = harness.SampledRun(2, 4, 2, num_pages=4, rows=3, max_tokens=256, bits=bits, device="cpu")
    out = run.step(1, bf16(3, 4, 128), bf16(3, 2, 128), bf16(3, 2, 128))
    assert out.shape == (3, 4, 128) and not out.any()
    out = run.prompt(0, bf16(0, 4, 128), bf16(0, 2, 128), bf16(0, 2, 128))
    assert out.shape == (0, 4, 128)


@pytest.mark.parametrize("bits", [2, 16, 5])
def test_other_widths_are_refused(bits):
    with pytest.raises(ValueError):
        harness.SampledRun(1, 4, 2, num_pages=4, rows=3, max_tokens=256, bits=bits, device="cpu")


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("length", [255, 256, 257])
def test_siblings_keep_their_tokens(bits, length):
    """Fork at the end of a page, before it and behind it; each sibling's step leaves the others' tokens as they are."""
    gen = torch.Generator().manual_seed(length)
    hq, hkv = 4, 2
    run = harness.SampledRun(1, hq, hkv, num_pages=16, rows=3, max_tokens=512, bits=bits)
    draw = lambda n, h: bf16(n, h, 128, gen=gen, device="cuda")  # noqa: E731
    run.advance([length, 0, 0])
    run.prompt(0, draw(length, hq), draw(length, hkv), draw(length, hkv))
    run.fork([0, 0, 0])
    cache, q = run.caches[0], draw(3, hq)
    with pytest.raises(ValueError):
        run.step(0, q, draw(3, hkv), draw(3, hkv))

    def held(row):
        t = torch.arange(length, device="cuda")
        pages = run.pages.table[row, :3].long()[t // 128]
        return torch.cat([cache.codes_view()[pages, :, :, t % 128].flatten(1).int(), cache.scales.view(torch.int32).view(cache.num_pages, hkv, 2, 128)[pages, :, :, t % 128].flatten(1)], 1)

    before = [held(row) for row in range(3)]
    assert torch.equal(before[0], before[1]) and torch.equal(before[0], before[2])
    run.advance([1, 0, 0])
    with pytest.raises(ValueError):      # rows 1 and 2 have no new token
        run.step(0, q, draw(3, hkv), draw(3, hkv))
    run.prompt(0, q[:1].contiguous(), draw(1, hkv), draw(1, hkv))
    run.advance([1, 1, 1])
    run.step(0, q, draw(3, hkv), draw(3, hkv))
    assert all(torch.equal(a, held(row)) for row, a in enumerate(before))


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
def test_every_row_ends(bits):
    gen = torch.Generator().manual_seed(3)
    run = harness.SampledRun(1, 4, 2, num_pages=4, rows=2, max_tokens=256, bits=bits)
    run.advance([3, 1])
    run.prompt(0, *(bf16(4, h, 128, gen=gen, device="cuda") for h in (4, 2, 2)))
    run.fork([-1, -1])
    run.advance([0, 0])
    assert not run.step(0, *(bf16(2, h, 128, gen=gen, device="cuda") for h in (4, 2, 2))).any()
    run.advance([1, 0])
    assert run.step(0, *(bf16(2, h, 128, gen=gen, device="cuda") for h in (4, 2, 2)))[0].isfinite().all()
