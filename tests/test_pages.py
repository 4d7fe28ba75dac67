"""Fork, grow and compact of page tables on a GPU, against the same steps on Python lists.

Everything is chosen and moved, so every comparison is for equality."""
import random

import pytest
import torch

from paper_2407_07304_b200 import binding as slim
from paper_2407_07304_b200 import harness

pytestmark = pytest.mark.gpu
PAGE = 128


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Model:
    """The page tables as lists; pools as dicts {(page, slot): token}."""

    def __init__(self, num_pages, stride):
        self.refs, self.stride = [0] * num_pages, stride
        self.rows, self.lens = [], []
        self.slots = {}

    def take(self, n):
        free = [p for p, r in enumerate(self.refs) if r == 0]
        return free[:n] if len(free) >= n else None

    def fork(self, parents):
        heirs, refs = {}, list(self.refs)
        for row in self.rows:
            for p in row:
                refs[p] -= 1
        rows, copies, lens = [], [], []
        for i, b in enumerate(parents):
            if not 0 <= b < len(self.rows):
                rows.append([])
                lens.append(-1)
                continue
            row, n = self.rows[b], self.lens[b]
            lens.append(n)
            if b not in heirs:
                heirs[b] = i
                rows.append(list(row))
            else:
                whole = min(max(n, 0) // PAGE, len(row))
                rows.append(list(row[:whole]))
                if n % PAGE and n > 0 and whole < len(row):
                    copies.append((i, row[whole], n % PAGE))
        for row in rows:
            for p in row:
                refs[p] += 1
        free = [p for p, r in enumerate(refs) if r == 0]
        if len(free) < len(copies):
            return len(copies) - len(free), 0
        for (i, source, n), fresh in zip(copies, free):
            rows[i].append(fresh)
            refs[fresh] = 1
            for s in range(n):
                self.slots[(fresh, s)] = self.slots[(source, s)]
        self.refs, self.rows, self.lens = refs, rows, lens
        return 0, len(free) - len(copies)

    def grow(self, lens, room):
        lacks = [max(0, min(self.stride, -(-(n + room) // PAGE)) - len(row)) if n >= 0 else 0 for n, row in zip(lens, self.rows)]
        free = [p for p, r in enumerate(self.refs) if r == 0]
        if sum(lacks) > len(free):
            return sum(lacks) - len(free), 0
        it = iter(free)
        for row, n in zip(self.rows, lacks):
            for _ in range(n):
                row.append(next(it))
                self.refs[row[-1]] = 1
        return 0, len(free) - sum(lacks)

    def compact(self):
        used = [p for p, r in enumerate(self.refs) if r]
        n = len(used)
        movers, holes = [p for p in used if p >= n], [p for p in range(n) if not self.refs[p]]
        to = dict(zip(movers, holes))
        self.slots.update({(to[p], s): t for (p, s), t in list(self.slots.items()) if p in to})
        refs = [0] * len(self.refs)
        for p in used:
            refs[to.get(p, p)] = self.refs[p]
        self.refs = refs
        self.rows = [[to.get(p, p) for p in row] for row in self.rows]
        return n, len(movers)


def compare(model, pages, lens=None):
    assert pages.refs.tolist() == model.refs
    assert pages.held.tolist() == [len(r) for r in model.rows]
    assert pages.table.tolist() == [r + [-1] * (model.stride - len(r)) for r in model.rows]
    if lens is not None:
        assert lens.tolist() == model.lens


def token_words(tokens, bits):
    return tokens * 7 + bits


def write(model, caches, row, first, count, stamp):
    """Marks tokens first .. of a row in every layer: each slot's codes and scale are filled with a number of the token."""
    for t in range(first, first + count):
        page, slot = model.rows[row][t // PAGE], t % PAGE
        model.slots[(page, slot)] = stamp + t
        for i, c in enumerate(caches):
            c.codes_view()[page, :, :, slot] = (stamp + t + i) % 120
            c.scales.view(torch.int32).view(c.num_pages, c.Hkv, 2, PAGE)[page, :, :, slot] = 1000 * i + stamp + t


def check_tokens(model, caches):
    for row, n in zip(model.rows, model.lens):
        if n <= 0:
            continue
        ids = torch.tensor(row, device="cuda")[torch.arange(n) // PAGE]
        slots = torch.arange(n, device="cuda") % PAGE
        want = torch.tensor([model.slots[(row[t // PAGE], t % PAGE)] for t in range(n)], device="cuda")
        for i, c in enumerate(caches):
            codes = c.codes_view()[ids, :, :, slots]
            scales = c.scales.view(torch.int32).view(c.num_pages, c.Hkv, 2, PAGE)[ids, :, :, slots]
            assert (codes == ((want + i) % 120)[:, None, None, None].to(codes.dtype)).all()
            assert (scales == (1000 * i + want)[:, None, None].to(torch.int32)).all()


@pytest.mark.parametrize("seed,num_pages,rows,stride", [(1, 40, 5, 4), (2, 150, 17, 6), (3, 700, 70, 5), (4, 5000, 3, 40), (5, 60000, 9, 6)])
def test_a_random_run(seed, num_pages, rows, stride):
    """Twenty random steps of grow, fork (other numbers of rows too) and compact, every table after every step."""
    rng = random.Random(seed)
    caches = [slim.SlimCache(1, 2, 1, num_pages=num_pages), slim.SlimCache4(1, 3, 1, num_pages=num_pages)]
    layers, result = slim.PageLayers(caches), i32([0, 0])
    model, pages = Model(num_pages, stride), slim.SlimPages.empty(num_pages, rows, stride)
    model.rows, model.lens = [[] for _ in range(rows)], [-1] * rows
    kv_len, ws = i32(model.lens), slim.pages_workspace(num_pages, 2 * rows)
    stamp = 0
    for _ in range(20):
        kind = rng.choice(["grow", "fork", "fork", "compact"]) if any(n >= 0 for n in model.lens) else "grow"
        if kind == "grow":
            asked = [min(stride * PAGE, max(n, 0) + rng.choice([0, 1, 3, 127, 128, 200])) if rng.random() < 0.8 else n for n in model.lens]
            room = rng.choice([0, 0, 1, 130, 10 ** 6])
            want = model.grow(asked, room)
            kv_len = i32(asked)
            slim.slim_pages_grow(pages, kv_len, room, result, ws)
            assert result.tolist() == list(want)
            if want[0] == 0:
                for i, n in enumerate(asked):
                    write(model, caches, i, max(model.lens[i], 0), max(n, 0) - max(model.lens[i], 0), stamp)
                    stamp += 1
                model.lens = asked
            kv_len = i32(model.lens)
            compare(model, pages)
        elif kind == "fork":
            n_out = rng.choice([rows, rows, rng.randrange(1, 2 * rows)])
            parents = [rng.choice([-1, rng.randrange(len(model.rows)), rng.randrange(len(model.rows)), min(i, len(model.rows) - 1)]) for i in range(n_out)]
            if rng.random() < 0.2:
                parents[0] = len(model.rows) + 3
            same = rng.random() < 0.5      # the counters in place, or others
            other = slim.SlimPages.empty(num_pages, n_out, stride)
            if same:
                other = slim.SlimPages(pages.refs, other.table, other.held)
            len_out, before = i32([7] * n_out), [t.clone() for t in (pages.refs, pages.table, pages.held)]
            want = model.fork(parents)
            slim.slim_pages_fork(layers, pages, other, i32(parents), kv_len, len_out, result, ws)
            assert result.tolist() == list(want)
            if want[0]:
                assert all(torch.equal(a, b) for a, b in zip(before, (pages.refs, pages.table, pages.held)))
                assert len_out.tolist() == [7] * n_out and (other.table == -1).all()
            else:
                pages, kv_len = other, len_out
                compare(model, pages, kv_len)
        else:
            other = pages if rng.random() < 0.5 else slim.SlimPages.empty(num_pages, len(model.rows), stride)
            want = model.compact()
            slim.slim_pages_compact(layers, pages, other, result, ws)
            pages = other
            assert result.tolist() == list(want)
            compare(model, pages)
        check_tokens(model, caches)


def test_no_rows_and_no_free_page():
    pages = slim.SlimPages(i32([1, 1, 1]), i32([[2, 0], [1, -1]]), i32([2, 1]))
    ws, result = slim.pages_workspace(3, 2), i32([5, 5])
    slim.slim_pages_grow(pages, i32([128, 200]), 100, result, ws)
    assert result.tolist() == [2 - 1, 0] and pages.held.tolist() == [2, 1]          # row 1 lacks two pages of which its stride allows one
    dst = slim.SlimPages.empty(3, 3, 2)
    slim.slim_pages_fork(None, pages, dst, i32([0, 0, 1]), i32([200, 100]), i32([0] * 3), result, slim.pages_workspace(3, 3))
    assert result.tolist() == [1, 0] and (dst.table == -1).all() and not dst.refs.any()
    dst = slim.SlimPages.empty(3, 3, 2)
    len_out = i32([0] * 3)
    slim.slim_pages_fork(None, pages, dst, i32([0, 0, -1]), i32([200, 100]), len_out, result, slim.pages_workspace(3, 3))
    assert result.tolist() == [0, 0] and dst.table.tolist() == [[2, 0], [2, 1], [-1, -1]] and dst.refs.tolist() == [1, 1, 2]   # row 1's page serves the copy
    assert len_out.tolist() == [200, 200, -1] and dst.held.tolist() == [2, 2, 0]
    none = slim.SlimPages.empty(3, 0, 2)
    slim.slim_pages_fork(None, dst, none, i32([]), len_out, i32([]), result, slim.pages_workspace(3, 3))
    assert result.tolist() == [0, 3] and none.refs.tolist() == [0, 0, 0]
    slim.slim_pages_compact(None, none, none, result, ws)
    assert result.tolist() == [0, 0]


def test_pages_that_other_holders_count():
    """A page that the caller keeps (a counter one higher) survives its rows, and page ids outside the pool are not followed."""
    pages = slim.SlimPages(i32([2, 0, 1, 0]), i32([[0, 2, -1], [9, -4, -1]]), i32([2, 2]))
    dst, result = slim.SlimPages.empty(4, 2, 3), i32([0, 0])
    slim.slim_pages_fork(None, pages, dst, i32([-1, 1]), i32([130, 256]), i32([0, 0]), result, slim.pages_workspace(4, 2))
    assert dst.refs.tolist() == [1, 0, 0, 0] and result.tolist() == [0, 3] and dst.table.tolist() == [[-1] * 3, [9, -4, -1]]


def test_captured_and_replayed():
    pages = slim.SlimPages.empty(64, 4, 4)
    kv_len, result, ws = i32([100, 200, -1, 300]), i32([0, 0]), slim.pages_workspace(64, 8)
    cache = slim.SlimCache4(1, 2, 1, num_pages=64)
    cache.codes.copy_(torch.randint(0, 255, cache.codes.shape, dtype=torch.uint8))
    layers, dst = slim.PageLayers([cache]), slim.SlimPages.empty(64, 8, 4)
    slim.slim_pages_grow(pages, kv_len, 0, result, ws)
    parent, len_out = i32([0, 0, 1, 1, 1, 3, 3, 2]), i32([0] * 8)
    slim.slim_pages_fork(layers, pages, dst, parent, kv_len, len_out, result, ws)
    eager = [t.clone() for t in (dst.table, dst.refs, dst.held, len_out, cache.codes)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        slim.slim_pages_fork(layers, pages, dst, parent, kv_len, len_out, result, ws)
        slim.slim_pages_compact(layers, dst, dst, result, ws)
    dst.table.fill_(5)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, (dst.table, dst.refs, dst.held, len_out, cache.codes)))   # (the pages were together already)


# ------------------------------------------------------------------------------------------------ a run of them
@pytest.mark.parametrize("bits", [4, 8])
def test_sampled_run(bits):
    """Prompts, forks, ends, steps and a compaction, against the same attention over contiguous caches rebuilt for every call."""
    gen = torch.Generator().manual_seed(bits)
    hq, hkv, rows, n_layers = 8, 2, 6, 2
    run = harness.SampledRun(n_layers, hq, hkv, num_pages=24, rows=rows, max_tokens=640, bits=bits)
    draw = lambda n, h: torch.randn(n, h, 128, generator=gen).to(torch.bfloat16).cuda()  # noqa: E731
    past = [[None] * n_layers for _ in range(rows)]      # per row and layer: all its keys and values

    def plain(layer, row, q):
        """The same attention over a cache that holds only this row, on pages in order."""
        k, v = past[row][layer]
        n = len(k)
        kind, append = (slim.SlimCache4, slim.slim_kv4_append) if bits == 4 else (slim.SlimCache, slim.slim_kv_append)
        cache = kind(1, hkv, (n + PAGE - 1) // PAGE)
        append(cache, k.contiguous(), v.contiguous(), i32([0, n]), i32([0]), 1, n)
        out = torch.empty_like(q)
        if len(q) > 1:
            fn = slim.slim_attn4_prefill if bits == 4 else slim.slim_attn_prefill
            fn(cache, q, out, i32([0, len(q)]), i32([n]), 1, len(q), n, hq, run.sm_scale, slim.workspace(slim.PHASE_PREFILL, 1, hq, hkv, len(q), n))
        elif bits == 4:
            slim.slim_attn4_decode(cache, q, out, i32([n]), 1, n, hq, run.sm_scale, slim.decode4_workspace(1, hq, hkv, n))
        else:
            slim.slim_attn_decode(cache, q, out, i32([n]), 1, n, hq, run.sm_scale, slim.workspace(slim.PHASE_DECODE, 1, hq, hkv, 1, n))
        return out

    def same(a, b):
        # a bf16 step apart at most, and the 4-bit decode's weights in fp16 are rounded where the batch's division puts them:
        # 2^-11 of the largest less the smallest value of a row (below 10 here), on both sides
        torch.testing.assert_close(a.float(), b.float(), rtol=2.0 ** -7, atol=2 * 10 * 2.0 ** -11 if bits == 4 else 2e-4)

    def prompt(counts):
        run.advance(counts)
        for layer in range(n_layers):
            n = sum(counts)
            q, k, v = draw(n, hq), draw(n, hkv), draw(n, hkv)
            out, at = run.prompt(layer, q, k, v), 0
            for row, c in enumerate(counts):
                if c:
                    old = past[row][layer]
                    new = (k[at:at + c], v[at:at + c])
                    past[row][layer] = new if old is None else tuple(torch.cat([a, b]) for a, b in zip(old, new))
                    same(out[at:at + c], plain(layer, row, q[at:at + c]))
                at += c

    def step():
        live = [1 if n >= 0 else 0 for n in run.lens]
        run.advance(live)
        for layer in range(n_layers):
            q, k, v = draw(rows, hq), draw(rows, hkv), draw(rows, hkv)
            out = run.step(layer, q, k, v)
            for row in range(rows):
                if not live[row]:
                    assert not out[row].any()
                    continue
                past[row][layer] = tuple(torch.cat([a, b[row:row + 1]]) for a, b in zip(past[row][layer], (k, v)))
                same(out[row:row + 1], plain(layer, row, q[row:row + 1]))

    def fork(parents):
        nonlocal past
        run.fork(parents)
        past = [list(past[p]) if p >= 0 else [None] * n_layers for p in parents]

    prompt([200, 0, 256, 0, 0, 0])
    fork([0, 0, 2, 2, 2, -1])
    step()
    step()
    fork([4, 1, 1, -1, 4, 0])
    for _ in range(3):
        step()
    prompt([0, 2, 0, 130, 0, 0])
    fork([1, 3, -1, -1, 5, 5])
    used = run.compact()
    assert used == int((run.pages.refs > 0).sum()) and int(run.pages.table.max()) == used - 1
    step()
    with pytest.raises(MemoryError):
        run.advance([640 - max(n, 0) for n in run.lens])
    step()
