"""What the serving loop refuses before anything is launched.  No GPU: its buffers lie on the CPU and no call is made."""
import pytest
import torch

from paper_2407_07304_b200 import binding as slim
from paper_2407_07304_b200 import harness


def make(**kw):
    return harness.RotatedRun(3, 4, 2, max_tokens=128, inv_freq=torch.ones(64, dtype=torch.float64), device="cpu", **kw)


@pytest.mark.parametrize("counts", [[], [5], [5, 5], [5, 5, 5, 5], [5, -1, 5]])
def test_prompt_refuses_counts_that_are_not_one_per_sequence(counts):
    """A shorter list would leave the call with fewer row starts than sequences, and the run with fewer lengths."""
    run = make()
    rows = torch.zeros((sum(counts), 8, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        run.prompt(rows, counts)
    assert run.lens == [0, 0, 0] and run.seen == [0, 0, 0]


@pytest.mark.parametrize("rows", [0, 14, 16])
def test_prompt_refuses_rows_that_are_not_the_counts(rows):
    run = make()
    with pytest.raises(slim.SlimError):
        run.prompt(torch.zeros((rows, 8, 128), dtype=torch.bfloat16), [5, 5, 5])
    with pytest.raises(slim.SlimError):
        run.step(torch.zeros((rows, 8, 128), dtype=torch.bfloat16))
    assert run.lens == [0, 0, 0] and run.seen == [0, 0, 0]


def test_a_full_cache_is_refused():
    run = make()
    run.lens = [128, 3, 4]
    with pytest.raises(ValueError):
        run.step(torch.zeros((3, 8, 128), dtype=torch.bfloat16))
