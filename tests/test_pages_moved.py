"""Pages that someone beside the page table holds, across a compaction."""
import random

import pytest
import torch

from paper_2407_07304_b200 import binding as slim

pytestmark = pytest.mark.gpu


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("num_pages", [7, 300, 60000])
def test_other_holders_follow(num_pages):
    rng = random.Random(num_pages)
    n = min(num_pages, 200)
    ids = rng.sample(range(num_pages), n // 2)
    rows = [sorted(ids[:n // 5]), sorted(ids[n // 5:n // 4])]       # two rows; the last ids are held by others alone
    kept = ids[n // 4:] + rows[0][:2]                                 # and two of a row's by both
    refs, stride = [0] * num_pages, max(len(r) for r in rows) + 1
    for p in rows[0] + rows[1] + kept:
        refs[p] += 1
    pages = slim.SlimPages(i32(refs), i32([r + [-1] * (stride - len(r)) for r in rows]), i32([len(r) for r in rows]))
    cache = slim.SlimCache4(1, 1, 1, num_pages=num_pages)
    cache.scales.view(torch.int32).view(num_pages, -1)[:] = torch.arange(num_pages, dtype=torch.int32, device="cuda")[:, None]
    cache.codes.view(torch.int32).view(num_pages, -1)[:] = 3 * torch.arange(num_pages, dtype=torch.int32, device="cuda")[:, None]
    result, ws = i32([0, 0]), slim.pages_workspace(num_pages, 2)
    slim.slim_pages_compact(slim.PageLayers([cache]), pages, pages, result, ws)
    used, moved = result.tolist()
    assert used == len(set(ids)) and moved == sum(p >= used for p in ids)
    old, new = (t[:moved].tolist() for t in slim.pages_moved(ws, num_pages))
    assert old == sorted(p for p in ids if p >= used) and new == sorted(set(range(used)) - set(ids))
    to = dict(zip(old, new))
    for p in kept:
        at = to.get(p, p)
        assert (cache.scales.view(torch.int32).view(num_pages, -1)[at] == p).all() and (cache.codes.view(torch.int32).view(num_pages, -1)[at] == 3 * p).all()
    after = pages.refs.tolist()
    assert all(after[to.get(p, p)] == refs[p] for p in ids) and sum(after) == sum(refs) and not any(after[used:])
    assert pages.table.tolist() == [[to.get(p, p) for p in r] + [-1] * (stride - len(r)) for r in rows]
