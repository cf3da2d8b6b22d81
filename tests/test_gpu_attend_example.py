"""What the attention step's example finds: how far a 4-bit cache is off, and that smaller groups hold values closer."""

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_example_shows_what_groups_cost():
    """Keys and values are close to normal.  A group of 32, 64 or 128 of them spans 4.1, 4.7 or 5.3 of their deviations in the mean,
    so a value is off by span / 15 / sqrt(12) of one in the root of squares.  Averages of values are off by the same share as
    the values; keys' errors, at scores of deviation 1, change each weight by as much again: together sqrt(2) times, 11,
    13 and 14 %.  Rows with few positions have less of the second, and the weights of the head norms spread the scores: within a
    factor of 1.5."""
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import attend
    found = attend.main(["--prompt", "300", "--steps", "4", "--heads", "4", "--kv-heads", "2", "--head-size", "128"])
    assert found[32] < found[64] < found[128]
    for group, span in ((32, 4.1), (64, 4.7), (128, 5.3)):
        about = 2 ** 0.5 * span / 15 / 12 ** 0.5
        assert about / 1.5 < found[group] < 1.5 * about
