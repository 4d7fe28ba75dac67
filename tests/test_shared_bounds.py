"""The bounds of the shared-prefix decode on the host: what they must cover, and the workspace that they size.  No GPU."""
import random

import pytest

from paper_2407_07304_b200 import binding as slim
from test_operator_refusals import INVALID, WORKSPACE, cache, call_shared


@pytest.mark.parametrize("kw", [dict(g=1, B=2, mg=1), dict(g=3, B=7, mg=2), dict(g=1, B=65535, mg=65534)])
def test_groups_too_small_for_the_batch_are_refused(kw):
    # the sequences beyond them would have no prefix partials: their result would be what the workspace held
    assert call_shared(**kw, n=1 << 40) == INVALID


def test_groups_that_just_cover_the_batch_are_taken():
    # (as far as the next check: a workspace that is not there)
    for kw in (dict(g=1, B=2, mg=2), dict(g=4, B=7, mg=2), dict(g=65535, B=65535, mg=1)):
        assert call_shared(**kw, ws=None) == WORKSPACE


def _sizes(seed, count):
    """Pairs of calls of one head layout, the second within the first's batch, groups and bounds."""
    rng = random.Random(seed)
    for _ in range(count):
        hkv = rng.choice([1, 2, 4, 5, 8, 32])
        hq = hkv * rng.choice([1, 2, 7, 8, 16])

        def call(most=None):
            upto = lambda i, top: rng.randint(1, min(top, most[i]) if most else top)  # noqa: E731
            groups, per = upto(1, 64), upto(2, 200)
            top = min(groups * per, most[0] if most else 2048)
            return (max(per, rng.randint(1, top)), groups, per, rng.randint(0, most[3] if most else 40000), rng.randint(0, most[4] if most else 9000))

        big = call()
        small = call(big)
        if small[0] <= big[0]:
            yield hq, hkv, big, small


def test_a_workspace_made_for_the_largest_call_serves_the_smaller_ones():
    size = lambda hq, hkv, c: slim.lib().slim_shared_workspace_bytes(c[0], hq, hkv, *c[1:])  # noqa: E731
    assert [size(16, 2, (16, 1, 16, 16384, t)) for t in (1, 256, 1024, 2048)] == sorted(size(16, 2, (16, 1, 16, 16384, t)) for t in (1, 256, 1024, 2048))
    n = 0
    for hq, hkv, big, small in _sizes(11, 20000):
        assert size(hq, hkv, small) <= size(hq, hkv, big), (hq, hkv, big, small)
        n += 1
    assert n > 10000
    # one bound at a time
    for hq, hkv in ((1, 1), (16, 2), (64, 8), (32, 32)):
        for i, steps in ((3, [0, 127, 128, 300, 2048, 8192, 65536]), (4, [0, 1, 256, 257, 2048, 30000]), (2, [2, 3, 8, 16, 17, 40])):
            at = [80, 40, 40, 8192, 1024]
            row = []
            for x in steps:
                at[i] = x
                row.append(size(hq, hkv, tuple(at)))
            assert row == sorted(row)


def test_a_smaller_call_is_taken_with_the_largest_workspace():
    """(as far as the next check: an address that is not aligned)"""
    c = cache(max_pages_per_seq=1000, num_pages=4000)
    most = slim.lib().slim_shared_workspace_bytes(16, 16, 2, 1, 16, 16384, 2048)
    for tail in (0, 1, 256, 1024, 2048):
        for shared in (0, 128, 1000, 16384):
            assert call_shared(c=c, B=16, mg=16, hq=16, ms=shared, mt=tail, n=most, ws=(1 << 20) + 8) == INVALID
            assert call_shared(c=c, B=16, mg=16, hq=16, ms=shared, mt=tail, n=1000, ws=(1 << 20) + 8) == WORKSPACE
