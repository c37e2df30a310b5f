"""Sizes and limits of the operators that learn from hypotheses, as the host computes them (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2510_09085_amd import binding

FAKE = 256 * 4096  # an address that no refused call may touch
OK, NULL, SHAPE, BEAM, SPACE, VOCAB, ALIGN, OPTION = 0, -1, -2, -3, -5, -6, -8, -9


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2510_09085_amd import build
        build.build()
    return binding.load()


def up(n):
    return (n + 255) // 256 * 256


@pytest.mark.parametrize("T", [1, 2, 509])
@pytest.mark.parametrize("B", [1, 3, 64, 65, 256, 1700, 1800, 5000])
def test_policy_workspaces_hold_either_loss(lib, B, T):
    """Over scores: four sums of a row.  Over logits, also of one token a row: the frames of each row, then three sums of
    each of up to 2048 workgroups and the number of all frames."""
    over_scores = up(B * 4 * 8)
    over_logits = up(B * 4) + up((3 * 2048 + 1) * 8)
    assert lib.fltop_policy_workspace_bytes(B, T) >= max(over_scores, over_logits)
    rows = binding.FltopRows(FAKE, FAKE, T * 40, 40, B, T, 40, 0)
    policy = binding.FltopPolicy(0, 0, 0.2, 0.2, 0.1, 1.0)
    for n in (over_scores, over_logits):
        if n < max(over_scores, over_logits):
            assert lib.fltop_policy_loss_logits(ctypes.byref(rows), FAKE, FAKE, None, FAKE, 0, ctypes.byref(policy), FAKE, n,
                                                FAKE, FAKE, FAKE, None) == SPACE
