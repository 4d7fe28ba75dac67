"""The bounds of the shared-prefix decode on the host: what they must cover, and the workspace that they size.  No GPU."""
import pytest

from test_operator_refusals import INVALID, WORKSPACE, call_shared


@pytest.mark.parametrize("kw", [dict(g=1, B=2, mg=1), dict(g=3, B=7, mg=2), dict(g=1, B=65535, mg=65534)])
def test_groups_too_small_for_the_batch_are_refused(kw):
    # the sequences beyond them would have no prefix partials: their result would be what the workspace held
    assert call_shared(**kw, n=1 << 40) == INVALID


def test_groups_that_just_cover_the_batch_are_taken():
    # (as far as the next check: a workspace that is not there)
    for kw in (dict(g=1, B=2, mg=2), dict(g=4, B=7, mg=2), dict(g=65535, B=65535, mg=1)):
        assert call_shared(**kw, ws=None) == WORKSPACE
