"""The operators that learn from hypotheses at the edges of their ranges: single tokens, ends of utterances at the border
of two wavefronts, one utterance's numbers beside another's, references that are only watched."""
import math

import numpy as np
import pytest
import torch

import learn_reference as ref
from paper_2510_09085_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.load()
    return torch.device("cuda:0")


def guarded(dev, need):
    """A workspace of `need` bytes inside a buffer, and whether all around it is as it was."""
    buffer = torch.full((need + (1 << 17),), 0x5A, dtype=torch.uint8, device=dev)
    start = -buffer.data_ptr() % 256 + 256
    whole = lambda: bool((buffer[:start] == 0x5A).all()) and bool((buffer[start + need:] == 0x5A).all())  # noqa: E731
    return buffer[start:start + need], whole


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,V", [(1, 1, 32), (5, 1, 40), (64, 1, 5000), (1, 2, 32), (3, 50, 33), (1800, 1, 24)])
def test_workspace_of_the_loss_over_logits(dev, B, T, V, dtype):
    """Exactly its size: single tokens a row and several, the results those of a workspace of the call's own."""
    gen = torch.Generator(device=dev).manual_seed(B + T)
    x = torch.randn((B, T, V), generator=gen, device=dev).to(dtype)
    tok = torch.randint(0, V, (B, T), generator=gen, device=dev).to(torch.int32)
    lengths = torch.full((B,), T, dtype=torch.int32, device=dev)
    old = torch.full((B, T), -math.log(V), device=dev)
    A = torch.randn((B,), generator=gen, device=dev)
    go = lambda **more: binding.policy_loss_logits(x, tok, lengths, old, A, ref_logps=old, kl_weight=0.1, **more)  # noqa: E731
    ws, whole = guarded(dev, binding.load().fltop_policy_workspace_bytes(B, T))
    got, want = go(workspace=ws), go()
    torch.cuda.synchronize()
    assert whole()
    for k in want:
        assert torch.equal(got[k], want[k]), k
    # the loss from the call's own log-probabilities, in 64 bits: ratios, their products and the sum of B T terms in fp32
    l, o, a = got["logps"].double(), old.double(), A.double()[:, None]
    r, gap = torch.exp(l - o), o - l
    f = torch.maximum(-r * a, -r.clamp(0.8, 1.2) * a) + 0.1 * (torch.expm1(gap) - gap)
    assert abs(float(got["loss"]) - float(f.mean())) <= 2.0 ** -20 * float(f.abs().mean() + 1)
    with pytest.raises(binding.FltopError):
        go(workspace=ws[:-256])
