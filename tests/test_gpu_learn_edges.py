"""The operators that learn from hypotheses at the edges of their ranges: single tokens, ends of utterances at the border
of two wavefronts, one utterance's numbers beside another's, references that are only watched."""
import ctypes
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


def log_lattice(lp, tokens):
    """(ln P, occupancies [T, V]) of a hypothesis in the domain of logarithms, fp64: for masses below the 80-bit range."""
    z = np.array(ref.states_of(tokens))
    e = lp.astype(np.float64)[:, z]
    S = len(z)
    skip = np.where((np.arange(S) > 1) & (z != 0) & (z != np.roll(z, 2)), 0.0, -np.inf)
    up = lambda x, by: np.concatenate((np.full(by, -np.inf), x))[:S]  # noqa: E731
    down = lambda x, by: np.concatenate((x, np.full(by, -np.inf)))[by:]  # noqa: E731
    with np.errstate(invalid="ignore"):
        a = [np.where(np.arange(S) < 2, e[0], -np.inf)]
        for t in range(1, len(lp)):
            a.append(np.logaddexp(np.logaddexp(a[-1], up(a[-1], 1)), up(a[-1], 2) + skip) + e[t])
        b = [np.where(np.arange(S) >= S - 2, 0.0, -np.inf)]
        for t in range(len(lp) - 2, -1, -1):
            y = b[-1] + e[t + 1]
            b.append(np.logaddexp(np.logaddexp(y, down(y, 1)), down(y + skip, 2)))
        total = np.logaddexp(a[-1][-1], a[-1][-2]) if S > 1 else a[-1][-1]
        share = np.exp(np.array(a) + np.array(b[::-1]) - total)
    out = np.zeros(lp.shape)
    np.add.at(out.T, z, share.T)
    return total, out


@pytest.mark.parametrize("L,U,V,T,cost", [
    (128, 128, 32, 257, 35), (128, 128, 32, 257, 36), (128, 128, 80, 257, 36), (128, 1100, 32, 257, 36),
    (256, 1920, 32, 513, 64), (256, 1920, 32, 517, 64), (256, 1920, 80, 517, 63), (256, 256, 32, 515, 36)])
def test_the_last_token_at_the_border_of_two_wavefronts(dev, L, U, V, T, cost):
    """An utterance that ends within a block: the last token is the last of a wavefront's states, the blank behind it the
    next one's first, and only one of them has masses close enough together for one exponent.  Every token costs e^-cost (in
    the last block e^-38 at most), so that there is little but the one alignment, and the last token alone is likely in
    the last two frames, where the blank is not."""
    R = 4 if U >= 1920 else 8
    lp = np.full((1, T, V), -float(cost), np.float32)
    lp[0, (T - 1) // R * R:, :] = -float(min(cost, 38))
    lp[0, :, 0] = -0.001
    lp[0, T - 2:, V - 1] = -0.01
    lp[0, T - 2:, 0] = -20.0
    tok = np.zeros((1, 1, U), np.int32)
    tok[0, 0, :L] = 1 + np.arange(L) % (V - 3)
    tok[0, 0, L - 1] = V - 1
    x = torch.from_numpy(lp).to(dev)
    args = [torch.tensor(a, dtype=torch.int32, device=dev) for a in ([T], tok, [[L]])]
    out = binding.ctc_score(x, *args, want_grad=True)
    alone = binding.ctc_score(x, *args)["scores"]
    grad = binding.ctc_score_grad(x, *args, torch.ones((1, 1), dtype=torch.float64, device=dev), out["workspace"])
    want, share = log_lattice(lp[0], tok[0, 0, :L])
    # the reference's own: each frame adds numbers of the score's size a few times, each time half a step of that off
    slack = 4 * T * 2.0 ** -53 * abs(want)
    for s in (out["scores"], alone):
        assert abs(float(s) - want) <= slack + ref.score_tolerance(T, want)
    near = ref.grad_tolerance("f32", T, share[None], share[None], np.array([2.0 * L + 1]))[0] + 4 * slack * share
    assert np.all(np.abs(grad[0].double().cpu().numpy() - share) <= near)


@pytest.mark.parametrize("V", [32, 90])
def test_frames_behind_the_end_are_not_read(dev, V):
    """Room for a million frames in the call's shapes, memory for those of the utterance: same bits as without the room."""
    frames, T, U = 43, 1 << 20, 9
    gen = torch.Generator(device=dev).manual_seed(V)
    x = torch.log_softmax(2 * torch.randn((1, frames, V), generator=gen, device=dev), 2)
    lengths = torch.tensor([frames], dtype=torch.int32, device=dev)
    tok = torch.randint(1, V, (1, 1, U), generator=gen, device=dev).to(torch.int32)
    tl = torch.tensor([[U]], dtype=torch.int32, device=dev)
    w = torch.ones((1, 1), dtype=torch.float64, device=dev)
    out = binding.ctc_score(x, lengths, tok, tl, want_grad=True)
    want = binding.ctc_score_grad(x, lengths, tok, tl, w, out["workspace"])

    lib = binding.load()
    rows = binding.FltopRows(x.data_ptr(), lengths.data_ptr(), T * V, V, 1, T, V, 0)
    hyps = binding.FltopHypotheses(tok.data_ptr(), tl.data_ptr(), None, U, U, 1, 1, U)
    ws = torch.empty(lib.fltop_ctc_score_workspace_bytes(1, T, 1, U), dtype=torch.uint8, device=dev)
    stream = torch.cuda.current_stream(dev).cuda_stream
    for space in (None, ws):
        score = torch.zeros((1, 1), dtype=torch.float64, device=dev)
        assert lib.fltop_ctc_score(ctypes.byref(rows), ctypes.byref(hyps), score.data_ptr(),
                                   None if space is None else space.data_ptr(), 0 if space is None else space.numel(),
                                   stream) == 0
        alone = binding.ctc_score(x, lengths, tok, tl)["scores"] if space is None else out["scores"]
        assert torch.equal(score, alone)
    grad = torch.full((1, T, V), 7.0, device=dev)
    assert lib.fltop_ctc_score_grad(ctypes.byref(rows), ctypes.byref(hyps), w.data_ptr(), ws.data_ptr(), ws.numel(),
                                    grad.data_ptr(), stream) == 0
    assert torch.equal(grad[:, :frames], want) and not grad[:, frames:].any()

    # rows of logits alike
    per_frame = lambda v: torch.full((1, T), v, device=dev)  # noqa: E731
    tokens = torch.randint(0, V, (1, T), generator=gen, device=dev).to(torch.int32)
    old, A, policy = per_frame(-3.0), torch.ones(1, device=dev), binding.FltopPolicy(0, 0, 0.2, 0.2, 0.0, 1.0)
    ws = torch.empty(lib.fltop_policy_workspace_bytes(1, T), dtype=torch.uint8, device=dev)
    summary, logps = torch.zeros(3, device=dev), per_frame(7.0)
    assert lib.fltop_policy_loss_logits(ctypes.byref(rows), tokens.data_ptr(), old.data_ptr(), None, A.data_ptr(), 0,
                                        ctypes.byref(policy), ws.data_ptr(), ws.numel(), summary.data_ptr(),
                                        logps.data_ptr(), grad.data_ptr(), stream) == 0
    want = binding.policy_loss_logits(x, tokens[:, :frames].contiguous(), lengths, old[:, :frames].contiguous(), A)
    assert torch.equal(grad[:, :frames], want["grad_logits"]) and not grad[:, frames:].any()
    assert torch.equal(logps[:, :frames], want["logps"]) and not logps[:, frames:].any()


@pytest.mark.parametrize("V", [32, 90])
def test_lengths_as_far_below_zero_as_there_are(dev, V):
    """Clamped to no frames, in each block of the room: no gradient."""
    B, T, U = 3, 40, 4
    x = torch.log_softmax(torch.randn((B, T, V), generator=torch.Generator(device=dev).manual_seed(V), device=dev), 2)
    lengths = torch.tensor([-2 ** 31, -2 ** 31 + 1, 40], dtype=torch.int32, device=dev)
    tok = torch.ones((B, 2, U), dtype=torch.int32, device=dev)
    tl = torch.tensor([[0, 2]] * B, dtype=torch.int32, device=dev)
    ws = torch.zeros(binding.score_workspace_bytes(B, T, 2, U), dtype=torch.uint8, device=dev)
    out = binding.ctc_score(x, lengths, tok, tl, want_grad=True, workspace=ws)
    grad = binding.ctc_score_grad(x, lengths, tok, tl, torch.ones((B, 2), dtype=torch.float64, device=dev), ws)
    assert out["scores"][:2].tolist() == [[0.0, -math.inf]] * 2 and torch.isfinite(out["scores"][2]).all()
    assert not grad[:2].any() and grad[2].any()
    old = torch.zeros((B, T), device=dev)
    told = binding.policy_loss_logits(x, torch.ones((B, T), dtype=torch.int32, device=dev), lengths, old, old[:, 0].contiguous() + 1)
    assert not told["grad_logits"][:2].any() and not told["logps"][:2].any() and told["grad_logits"][2].any()


def test_lists_of_pairs_of_as_many_utterances_as_a_launch_takes(dev):
    """2^22 utterances, of more pairs than a small workgroup is taken for: the same number everywhere."""
    B, M = 1 << 22, 513
    pairs = torch.zeros((B, M, 2), dtype=torch.int32, device=dev)
    pairs[:, :, 1] = 1
    scores = torch.tensor([[3.0, 1.0]], dtype=torch.float64, device=dev).expand(B, 2).contiguous()
    out = binding.preference_loss(scores, pairs, beta=0.5, scale=float(B))
    del pairs
    assert bool((out["margins"] == 2.0).all())
    del out["margins"]
    # each loss ln(1 + 1/e); sums of M and of B terms, half a step each at most
    assert abs(float(out["loss"]) - math.log1p(math.exp(-1.0))) <= (B + M) * 2.0 ** -53
    want = -0.5 / (1.0 + math.e)
    got = out["grad_scores"]
    assert torch.equal(got, got[:1].expand_as(got))
    assert abs(float(got[0, 0]) - want) <= M * 2.0 ** -52 and float(got[0, 1]) == -float(got[0, 0])
    torch.cuda.empty_cache()


@pytest.mark.parametrize("V", [30, 9000])
def test_a_reference_over_logits_that_is_only_watched(dev, V):
    """kl_weight 0: a KL that overflows, and that of a token without mass, touch neither loss nor gradient."""
    gen = torch.Generator(device=dev).manual_seed(V)
    x = torch.randn((2, 3, V), generator=gen, device=dev)
    tok = torch.full((2, 3), 5, dtype=torch.int32, device=dev)
    x[1, 1, 5] = -math.inf
    lengths = torch.full((2,), 3, dtype=torch.int32, device=dev)
    old = torch.full((2, 3), -math.log(V), device=dev)
    A = torch.tensor([1.0, -0.5], device=dev)
    far = old.clone()
    far[0, 1] += 100.0
    go = lambda q, w: binding.policy_loss_logits(x, tok, lengths, old, A, ref_logps=q, kl_weight=w)  # noqa: E731
    alone = go(None, 0.0)
    assert math.isfinite(float(alone["loss"])) and float(alone["kl"]) == 0.0
    for q in (far, old):
        seen = go(q, 0.0)
        for k in ("loss", "clipped", "logps", "grad_logits"):
            assert torch.equal(seen[k], alone[k]), k
        assert float(seen["kl"]) == math.inf
    # with a weight they are what the formulas give
    assert float(go(far, 0.1)["loss"]) == math.inf
    # a reference that rules a token out: infinite KL, of slope 1
    x[1, 1, 5] = 0.0
    far[:] = old
    far[0, 0] = -math.inf
    ruled, near = go(far, 0.25), go(old, 0.25)
    assert float(ruled["loss"]) == math.inf and float(ruled["kl"]) == math.inf
    l = ruled["logps"][0, 0].double()
    # d/dl: 1 in place of 1 - exp(ref - l), of six frames, at the token times 1 - p
    want = 0.25 / 6 * math.exp(float(old[0, 0]) - float(l)) * (1 - math.exp(float(l)))
    got = float(ruled["grad_logits"][0, 0, 5].double() - near["grad_logits"][0, 0, 5].double())
    # both derivatives below 4 and their parts rounded to fp32 some 20 times
    assert abs(got - want) <= 4 * 20 * 2.0 ** -24
    assert torch.equal(ruled["grad_logits"][:, 1:], near["grad_logits"][:, 1:])


@pytest.mark.parametrize("B,N", [(2, 3), (40, 64)])
def test_a_reference_of_scores_that_is_only_watched(dev, B, N):
    """The same over scores, in one launch and in two: a gap of 800, and one that no double holds."""
    s = -20 * torch.rand((B, N), dtype=torch.float64, generator=torch.Generator(device=dev).manual_seed(N), device=dev)
    A = torch.ones_like(s)
    go = lambda q, w: binding.policy_loss(s, s + 0.1, A, ref_scores=q, kl_weight=w)  # noqa: E731
    alone = go(None, 0.0)
    for gap in (800.0, 1.7e308):
        q = s.clone()
        q[1, 2] += gap
        seen = go(q, 0.0)
        for k in ("loss", "clipped", "grad_scores"):
            assert torch.equal(seen[k], alone[k]), k
        assert float(seen["kl"]) == math.inf and float(go(q, 0.1)["loss"]) == math.inf
    s[1, 2], q[1, 2] = -1.7e308, 1.7e308
    assert float(binding.policy_loss(s, s, A, ref_scores=q)["kl"]) == math.inf
    assert math.isfinite(float(binding.policy_loss(s, s, A, ref_scores=q)["loss"]))


@pytest.mark.parametrize("B", [2, 64, 2000])
@pytest.mark.parametrize("kind", ["sigmoid", "square"])
def test_one_utterance_does_not_set_the_digits_of_another(dev, kind, B):
    """A derivative of 1e17, or ones of e^-40, beside those of other utterances: each keeps 50 bits of its own, in a batch of
    one launch (up to 2048 scores) as in a larger one."""
    rng = np.random.default_rng(B)
    s = -20 * rng.random((B, 2))
    s[0] = (1e17, 0.0) if kind == "square" else (-20.0, 0.0)
    s[1:, 0] += 0.0 if kind == "square" else 450.0
    pairs = np.tile(np.array([[[0, 1]]], np.int32), (B, 1, 1))
    S, P = torch.from_numpy(s).to(dev), torch.from_numpy(pairs).to(dev)
    got = binding.preference_loss(S, P, kind=kind, beta=0.1)["grad_scores"].cpu().numpy()
    h = s[:, 0] - s[:, 1]
    want = (2 * (h - 5.0) if kind == "square" else -0.1 / (1.0 + np.exp(0.1 * h))) / B
    # the margin's difference, beta's product with it (45 * 2^-53 in e^x) and some ten roundings; a step of 2^-50
    tol = (45 + 20) * 2.0 ** -53 + 2.0 ** -50
    scale = np.abs(want) + (2 * 2.0 ** -53 * (np.abs(s).sum(1) + 5.0) / B / tol if kind == "square" else 0.0)
    assert np.all(np.abs(got[:, 0] - want) <= tol * scale) and np.array_equal(got[:, 1], -got[:, 0])


@pytest.mark.parametrize("B", [1, 3000])
def test_a_margin_that_beta_takes_out_of_range(dev, B):
    """Won by more than a double holds: no loss and no gradient; lost by as much: an infinite loss of slope -beta."""
    s = torch.tensor([[1e300, -1e300]], dtype=torch.float64, device=dev).repeat(B, 1)
    won = torch.tensor([[[0, 1]]], dtype=torch.int32, device=dev).repeat(B, 1, 1)
    out = binding.preference_loss(s, won, beta=1e10)
    assert float(out["loss"]) == 0.0 and not out["grad_scores"].any()
    out = binding.preference_loss(s, won.flip(2).contiguous(), beta=1e10, scale=float(B))
    assert float(out["loss"]) == math.inf and out["grad_scores"][-1].tolist() == [1e10, -1e10]
    for smoothed in (won, won.flip(2).contiguous()):
        out = binding.preference_loss(s, smoothed, beta=1e10, label_smoothing=0.25)
        assert float(out["loss"]) == math.inf and torch.isfinite(out["grad_scores"]).all()


@pytest.mark.parametrize("B", [1, 3, 3000])
def test_lists_without_pairs(dev, B):
    """A batch of which nothing can be paired: no loss, no gradient, no margins."""
    s = -10 * torch.rand((B, 4), dtype=torch.float64, device=dev)
    none = torch.empty((B, 0, 2), dtype=torch.int32, device=dev)
    for more in ({}, {"pair_counts": torch.zeros(B, dtype=torch.int32, device=dev)},
                 {"pair_counts": torch.full((B,), 7, dtype=torch.int32, device=dev), "kind": "square", "ref_scores": s}):
        out = binding.preference_loss(s, none, **more)
        assert float(out["loss"]) == 0.0 and out["margins"].shape == (B, 0)
        assert out["grad_scores"].shape == s.shape and not out["grad_scores"].any()
    with pytest.raises(binding.FltopError):
        binding.preference_loss(s, none, beta=-1.0)


def test_inputs_that_require_a_gradient(dev):
    """They are read as they are; what comes back carries no history, and backward(gradient) goes on from it."""
    logits = torch.randn((2, 20, 12), generator=torch.Generator(device=dev).manual_seed(1), device=dev, requires_grad=True)
    x = torch.log_softmax(logits, 2)
    lengths = torch.tensor([20, 13], dtype=torch.int32, device=dev)
    tok = torch.randint(1, 12, (2, 1, 5), device=dev).to(torch.int32)
    tl = torch.full((2, 1), 5, dtype=torch.int32, device=dev)
    out = binding.ctc_score(x, lengths, tok, tl, want_grad=True)
    grad = binding.ctc_score_grad(x, lengths, tok, tl, torch.ones_like(out["scores"]), out["workspace"])
    assert not out["scores"].requires_grad and not grad.requires_grad
    x.backward(grad)
    plain = binding.ctc_score(x.detach(), lengths, tok, tl)["scores"]
    assert torch.equal(out["scores"], plain) and logits.grad is not None and logits.grad.any()


@pytest.mark.parametrize("cost", [400.0, 900.0, 5000.0])
@pytest.mark.parametrize("L,U,V", [(40, 40, 60), (40, 40, 90), (140, 140, 60), (40, 1920, 60), (40, 1920, 90), (140, 1920, 90)])
def test_one_costly_token_among_as_many_as_there_are_frames(dev, L, U, V, cost):
    """As many frames as tokens: one alignment, a new token in each frame, whatever the emissions are.  One of the tokens,
    another one for each utterance, costs e^-cost in every frame, so that what lies above it at a border of a block is that
    much likelier to get to the end than what the alignment has there."""
    B = L
    word = 1 + np.arange(L) % (V - 2)   # (no two neighbours alike)
    lp = np.full((B, L, V), -2.0, np.float32)
    for b in range(B):
        lp[b, :, word[b]] = -cost
    tok = np.ones((B, 1, U), np.int32)
    tok[:, 0, :L] = word
    x = torch.from_numpy(lp).to(dev)
    args = [torch.from_numpy(a).to(dev) for a in (np.full(B, L, np.int32), tok, np.full((B, 1), L, np.int32))]
    out = binding.ctc_score(x, *args, want_grad=True)
    grad = binding.ctc_score_grad(x, *args, torch.ones((B, 1), dtype=torch.float64, device=dev), out["workspace"])
    total = lp[:, np.arange(L), word].astype(np.float64).sum(1)
    want = np.zeros((L, V))
    want[np.arange(L), word] = 1.0
    for b in range(B):
        assert abs(float(out["scores"][b, 0]) - total[b]) <= ref.score_tolerance(L, total[b]), b
    got = grad.double().cpu().numpy()
    near = ref.grad_tolerance("f32", L, want[None], want[None], np.array([2.0 * L + 1]))[0]
    off = [b for b in range(B) if np.any(np.abs(got[b] - want) > near)]
    assert not off, off


@pytest.mark.parametrize("kind", ["steep", "heavy tails", "costly tokens", "levels", "masked"])
@pytest.mark.parametrize("L,U,V,T", [(0, 1, 5, 9), (7, 7, 12, 7), (63, 70, 32, 71), (64, 64, 80, 64), (112, 113, 32, 121),
                                     (128, 128, 65, 131), (129, 1000, 20, 150), (128, 2004, 65, 138), (256, 1920, 12, 259)])
def test_emissions_of_mixed_regimes(dev, kind, L, U, V, T):
    """Masses that lie far apart in some lanes and not in others, with little room for alignments: both ways through a block
    side by side, scores with and without the borders, and the gradient."""
    gen = torch.Generator().manual_seed(L + V + len(kind))
    x = torch.randn((2, T, V), generator=gen)
    if kind == "steep":
        x = torch.full((2, T, V), -36.0)
        x[:, :, 0] = -0.001
        x[1, T // 2:, 0] = -39.0
    elif kind == "heavy tails":
        x = torch.log_softmax(x / torch.randn((2, T, V), generator=gen).abs().clamp_min(1e-3), 2)
    elif kind == "costly tokens":
        x = x - 900.0 * (torch.rand((2, 1, V), generator=gen) < 0.2) * torch.rand((2, 1, V), generator=gen)
    elif kind == "levels":
        x = x + 100.0 * (torch.rand((2, T, 1), generator=gen) - 0.7)
    else:
        x = torch.log_softmax(x, 2).masked_fill(torch.rand((2, T, V), generator=gen) < 0.005, -math.inf)
    tok = (1 + (torch.arange(U) + torch.randint(0, V, (2, 1, 1), generator=gen)) % (V - 1)).expand(2, 1, U).to(torch.int32)
    lengths, tl = torch.tensor([T, max(T - 2, min(T, L))]), torch.tensor([[L], [max(0, L - 1)]])
    args = [x.to(dev)] + [a.to(torch.int32).contiguous().to(dev) for a in (lengths, tok, tl)]
    out = binding.ctc_score(*args, want_grad=True)
    alone = binding.ctc_score(*args)["scores"]
    grad = binding.ctc_score_grad(*args, torch.ones((2, 1), dtype=torch.float64, device=dev), out["workspace"])
    for b in range(2):
        n, frames = int(tl[b, 0]), int(lengths[b])
        want, share = log_lattice(x[b, :frames].numpy(), tok[b, 0, :n].numpy())
        got = grad[b].double().cpu().numpy()
        if not np.isfinite(want):
            assert float(out["scores"][b, 0]) == -math.inf and float(alone[b, 0]) == -math.inf and not got.any()
            continue
        # the reference's own: each frame adds numbers of the score's size a few times, each time half a step of that off
        slack = 4 * T * 2.0 ** -53 * max(abs(want), 1.0)
        for s in (out["scores"], alone):
            assert abs(float(s[b, 0]) - want) <= slack + ref.score_tolerance(T, want)
        near = ref.grad_tolerance("f32", T, share[None], share[None], np.array([2.0 * n + 1]))[0] + 4 * slack * share
        assert np.all(np.abs(got[:frames] - share) <= near) and not got[frames:].any()
