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


def rows(**change):
    x = binding.FltopRows(FAKE, FAKE, 10 * 32, 32, 2, 10, 32, 0)
    for k, v in change.items():
        setattr(x, k, v)
    return ctypes.byref(x)


@pytest.mark.parametrize("most", [2 ** 31 - 1, 2 ** 31 - 8, 2 ** 31 - 8192])
def test_counts_that_loops_in_32_bits_would_step_past(lib, most):
    """Loops go on by up to 8192 behind the last frame, logit or entry."""
    hyps = binding.FltopHypotheses(FAKE, FAKE, None, 3 * 8, 8, 3, 3, 8)
    policy = ctypes.byref(binding.FltopPolicy(0, 0, 0.2, 0.2, 0.1, 1.0))
    long = rows(B=1, T=most, V=2)
    assert lib.fltop_ctc_score(long, ctypes.byref(hyps), FAKE, None, 0, None) == SHAPE
    assert lib.fltop_ctc_score_grad(long, ctypes.byref(hyps), FAKE, FAKE, 1 << 62, FAKE, None) == SHAPE
    for x in (long, rows(B=1, T=1, V=most)):
        assert lib.fltop_policy_loss_logits(x, FAKE, FAKE, None, FAKE, 0, policy, FAKE, 1 << 62, FAKE, FAKE, FAKE,
                                            None) == SHAPE
    assert lib.fltop_policy_loss(FAKE, FAKE, None, FAKE, None, 1, most, policy, FAKE, 1 << 62, FAKE, FAKE, None) == SHAPE
    assert lib.fltop_policy_workspace_bytes(1, most) == 0
    assert lib.fltop_policy_workspace_bytes(1, 2 ** 31 - 8193) > 0
