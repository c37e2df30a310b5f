"""ctc_score and ctc_score_grad against the lattice summed in 80 bits, all alignments enumerated, and differences."""
import math

import numpy as np
import pytest
import torch

import learn_reference as ref
from paper_2510_09085_amd import binding, synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.load()
    return torch.device("cuda:0")


def make(seed, B, N, T, V, U, lengths=None, token_lengths=None, flat=2.0, repeats=0.2):
    """Emissions [B,T,V] fp64-drawn fp32, lengths, tokens with some repeats, token lengths in 0..U."""
    rng = np.random.default_rng(seed)
    lp = synth.random_emissions(seed + 1, B, T, V, flat=flat)
    ln = np.asarray(lengths if lengths is not None else rng.integers(max(1, T // 2), T + 1, B), dtype=np.int32)
    tok = rng.integers(1, V, (B, N, U)).astype(np.int32)
    again = rng.random((B, N, U)) < repeats
    again[:, :, 0] = False
    for u in range(1, U):
        tok[:, :, u] = np.where(again[:, :, u], tok[:, :, u - 1], tok[:, :, u])
    tl = np.asarray(token_lengths if token_lengths is not None else rng.integers(0, U + 1, (B, N)), dtype=np.int32)
    w = rng.standard_normal((B, N))
    return lp, ln, tok, tl.reshape(B, N), w


def on_gpu(dev, lp, ln, tok, tl, w, dtype="f32", counts=None, poison=True, **options):
    x = torch.from_numpy(lp).to(dev).to(ref.DTYPES[dtype])
    args = [torch.from_numpy(np.ascontiguousarray(a)).to(dev) for a in (ln, tok, tl)]
    c = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=dev)
    ws = None
    if poison:
        ws = torch.full((binding.score_workspace_bytes(*x.shape[:2], *tok.shape[1:]),), 0xA5, dtype=torch.uint8, device=dev)
    out = binding.ctc_score(x, *args, c, want_grad=True, workspace=ws, **options)
    grad = binding.ctc_score_grad(x, *args, torch.from_numpy(w).to(dev), out["workspace"], c, **options)
    alone = binding.ctc_score(x, *args, c, **options)["scores"]
    torch.cuda.synchronize()
    return x.double().cpu().numpy(), out["scores"].cpu().numpy(), alone.cpu().numpy(), grad.double().cpu().numpy()


def check(dev, lp, ln, tok, tl, w, dtype="f32", counts=None, **options):
    x, scores, alone, grad = on_gpu(dev, lp, ln, tok, tl, w, dtype, counts, **options)
    want, g, size, quanta = ref.scores_and_grad(x, ln, tok, tl, w, counts)
    T = x.shape[1]
    for got in (scores, alone):
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(np.isneginf(got), np.isneginf(want))
        fine = np.isfinite(want)
        assert np.all(np.abs(got[fine] - want[fine]) <= ref.score_tolerance(T, want[fine]))
    assert np.all(np.abs(grad - g) <= ref.grad_tolerance(dtype, T, g, size, quanta))
    for b in range(x.shape[0]):  # frames behind the last are written, with zeros
        assert not grad[b, max(0, ln[b]):].any()
    return scores, grad


@pytest.mark.parametrize("T,V", [(1, 2), (1, 4), (2, 3), (3, 4), (5, 3), (6, 2)])
def test_every_alignment_enumerated(dev, T, V):
    words = [()] + [(a,) for a in range(1, V)] + [(a, b) for a in range(1, V) for b in range(1, V)] + [(1, 1, 1)]
    U = 3
    tok = np.full((1, len(words), U), 2 ** 31 - 1, dtype=np.int32)  # what lies behind a hypothesis is not read
    for n, word in enumerate(words):
        tok[0, n, :len(word)] = word
    tl = np.array([[len(word) for word in words]], dtype=np.int32)
    lp = synth.random_emissions(5 + T, 1, T, V, flat=1.5)
    w = np.random.default_rng(3).standard_normal((1, len(words)))
    x, scores, alone, grad = on_gpu(dev, lp, np.array([T], np.int32), tok, tl, w)
    want = np.zeros((T, V))
    size = np.zeros((T, V))
    for n, word in enumerate(words):
        total, share = ref.enumerated(x[0], word)
        if total == 0.0:
            assert scores[0, n] == -np.inf and alone[0, n] == -np.inf
        else:
            # the enumeration's own sum: up to 729 terms of 2^-53
            tol = ref.score_tolerance(T, math.log(total)) + 729 * 2.0 ** -53
            assert abs(scores[0, n] - math.log(total)) <= tol and abs(alone[0, n] - math.log(total)) <= tol
        want += w[0, n] * share
        size += abs(w[0, n]) * share
    quanta = np.array([np.abs(w).max() * 7 * len(words)])
    assert np.all(np.abs(grad[0] - want) <= ref.grad_tolerance("f32", T, want[None], size[None], quanta)[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", [
    (1, 1, 1, 2, 1), (2, 3, 7, 5, 4), (3, 2, 40, 29, 20), (2, 2, 130, 32, 62), (2, 2, 131, 32, 63), (2, 2, 140, 32, 64),
    (1, 2, 150, 31, 65), (5, 7, 33, 130, 9), (2, 1, 260, 24, 127), (1, 1, 261, 24, 128), (1, 2, 64, 1024, 30),
    (1, 33, 24, 4096, 6)])
def test_shapes_against_the_80_bit_lattice(dev, shape, dtype):
    B, N, T, V, U = shape
    check(dev, *make(sum(shape), B, N, T, V, U), dtype)


@pytest.mark.parametrize("L", [200, 255, 256, 257, 511, 512, 513, 700, 1023, 1024, 1100])
def test_long_hypotheses(dev, L):
    T = 2 * L + 9
    lp, ln, tok, tl, w = make(L, 1, 2, T, 32, L, lengths=[T], token_lengths=[[L, L - 1]], flat=1.0, repeats=0.05)
    check(dev, lp, ln, tok, tl, w)


def test_the_longest_hypothesis_there_may_be(dev):
    L = binding.MAX_LABELS
    T = L + 5
    rng = np.random.default_rng(2)
    tok = np.zeros((1, 1, L), np.int32)
    tok[0, 0, 0::2] = rng.integers(1, 8, (L + 1) // 2)
    tok[0, 0, 1::2] = rng.integers(8, 16, L // 2)  # no repeats: it fits
    lp = synth.random_emissions(4, 1, T, 16, flat=0.3)
    check(dev, lp, np.array([T], np.int32), tok, np.array([[L]], np.int32), np.array([[0.7]]))


def test_lengths_of_zero_and_one(dev):
    lp, ln, tok, tl, w = make(8, 6, 4, 9, 6, 3, lengths=[0, 1, 1, 9, 0, 2],
                              token_lengths=[[0, 1, 2, 3], [0, 1, 2, 3], [1, 1, 0, 0], [0, 3, 2, 1], [0, 0, 0, 0],
                                             [1, 2, 0, 3]])
    scores, grad = check(dev, lp, ln, tok, tl, w)
    assert scores[0].tolist() == [0.0] + [-np.inf] * 3  # no frames: the empty hypothesis has all the mass
    assert not grad[0].any()


def test_lengths_outside_their_range_are_clamped(dev):
    lp, ln, tok, tl, w = make(9, 3, 2, 11, 7, 4, lengths=[-3, 40, 11])
    check(dev, lp, ln, tok, tl, w)


def test_hypotheses_that_are_not_there(dev):
    lp, ln, tok, tl, w = make(10, 4, 5, 20, 9, 6, lengths=[20, 20, 20, 20], token_lengths=np.full((4, 5), 4))
    tl[0, 2] = -1
    tl[1, 1] = 7       # longer than U: not scored
    tl[1, 3] = 2 ** 31 - 1
    tok[2, 0, 3] = 0   # the blank is no token
    tok[2, 1, 0] = 9   # nor is V
    tok[2, 2, 2] = -5
    tok[2, 3, 1] = 2 ** 31 - 1
    w[0, 2] = np.nan   # weights of what takes no part do not matter
    w[1, 1] = np.inf
    w[3, 4] = np.nan
    counts = [5, 5, 5, 3]
    tl[3, 3] = 10 ** 6
    scores, _ = check(dev, lp, ln, tok, tl, w, counts=counts)
    assert np.isnan(scores[1]).tolist() == [False, True, False, True, False]
    assert np.isneginf(scores[3]).tolist() == [False] * 3 + [True] * 2
    w[3, 4] = 0.5
    for counts in ([0, 0, 0, 0], [-4, 99, 1, 5]):
        check(dev, lp, ln, tok, tl, w, counts=counts)


@pytest.mark.parametrize("dtype,low", [("f32", -math.inf), ("f32", torch.finfo(torch.float32).min), ("f32", -1e30),
                                       ("bf16", torch.finfo(torch.bfloat16).min), ("f16", -math.inf)])
def test_masked_emissions_have_no_mass(dev, dtype, low):
    lp, ln, tok, tl, w = make(11, 4, 3, 24, 8, 6, lengths=[24, 24, 20, 24], token_lengths=np.full((4, 3), 5))
    lp[0, 3, 1:] = low          # only the blank
    lp[1, 5, :] = low           # nothing at all: no hypothesis has an alignment
    lp[2, :, int(tok[2, 1, 2])] = low
    lp[2, 7:9, 0] = low         # no blank in two frames
    lp[3, 2::3, 4] = low
    lp[2, 20:] = np.nan         # behind the last frame
    scores, grad = check(dev, lp, ln, tok, tl, w, dtype) if math.isinf(low) else compare_to_inf(dev, lp, ln, tok, tl, w, dtype, low)
    assert np.isneginf(scores[1]).all() and not grad[1].any()


def compare_to_inf(dev, lp, ln, tok, tl, w, dtype, low):
    """A type's lowest value counts as -inf: bit for bit the same."""
    a = on_gpu(dev, lp, ln, tok, tl, w, dtype)
    b = on_gpu(dev, np.where(lp == np.float32(low), np.float32(-np.inf), lp), ln, tok, tl, w, dtype)
    for x, y in zip(a[1:], b[1:]):
        assert x.tobytes() == y.tobytes()
    return a[1], a[3]


def test_a_finite_mask_of_float16(dev):
    """-65504 is a number: a hypothesis that has to pass it has a finite score."""
    lp, ln, tok, tl, w = make(12, 1, 1, 30, 6, 5, lengths=[30], token_lengths=[[5]])
    lp[0, 4, :] = -65504.0
    x, scores, _, grad = on_gpu(dev, lp, ln, tok, tl, w, "f16")
    # frame 4 multiplies every alignment alike: exactly the score of an emission of 0 there, less 65504
    even = x.copy()
    even[0, 4] = 0.0
    want, g, size, quanta = ref.scores_and_grad(even, ln, tok, tl, w)
    assert abs(scores[0, 0] - (want[0, 0] - 65504.0)) <= ref.score_tolerance(30, 65504.0)
    assert np.all(np.abs(grad - g) <= ref.grad_tolerance("f16", 30, g, size, quanta))


def test_hypotheses_far_from_the_emissions(dev):
    """Every frame says blank with e^-0.001 and any token with e^-60: 150 tokens have a score near -9000, while the
    masses of a frame differ by e^9000.  The reference goes down to e^-11000."""
    T, V, L = 400, 12, 150
    lp = np.full((1, T, V), -60.0, np.float32) - np.random.default_rng(1).random((1, T, V)).astype(np.float32)
    lp[:, :, 0] = -0.001
    tok = np.random.default_rng(2).integers(1, V, (1, 2, L)).astype(np.int32)
    scores, _ = check(dev, lp, np.array([T], np.int32), tok, np.array([[L, 3]], np.int32), np.array([[1.0, -0.5]]))
    assert scores[0, 0] < -8000


@pytest.mark.parametrize("level", [-40.0, -120.0, -600.0, -5000.0, -1e6])
def test_levels_of_emissions_beyond_any_float(dev, level):
    """Rows need not be normalised: c added to every emission adds c T to the scores and leaves the gradient alone."""
    lp, ln, tok, tl, w = make(13, 2, 2, 60, 9, 12, lengths=[60, 41])
    base = on_gpu(dev, lp, ln, tok, tl, w)
    moved_lp = (lp.astype(np.float64) + level).astype(np.float32)
    moved = on_gpu(dev, moved_lp, ln, tok, tl, w)
    want, g, size, quanta = ref.scores_and_grad(moved[0] - level, ln, tok, tl, w)
    fine = np.isfinite(want)
    shift = (level * ln)[:, None] + 0 * want
    assert np.all(np.abs(moved[1][fine] - (want + shift)[fine]) <= ref.score_tolerance(60, (want + shift)[fine]))
    assert np.all(np.abs(moved[3] - g) <= ref.grad_tolerance("f32", 60, g, size, quanta))
    assert np.isfinite(base[3]).all()


def test_one_token_far_below_and_then_needed(dev):
    """A state that is e^-3000 below the others of its frame is the only one that the hypothesis can end with."""
    T, V = 50, 5
    lp = np.full((1, T, V), -3.0, np.float32)
    lp[0, :, 1] = -100.0   # 30 frames of token 1 cost e^-3000
    lp[0, 10:40, 0] = -np.inf
    lp[0, 10:40, 2:] = -0.5
    lp[0, 40:, 2:] = -np.inf
    tok = np.array([[[1], [2]]], np.int32)
    check(dev, lp, np.array([T], np.int32), tok, np.array([[1, 1]], np.int32), np.array([[1.0, 1.0]]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_orders(dev, dtype):
    """Time-major emissions transposed, rows inside wider ones, slices of the n-best arrays."""
    B, N, T, V, U = 3, 2, 37, 21, 9
    lp, ln, tok, tl, w = make(14, B, N, T, V, U)
    plain = on_gpu(dev, lp, ln, tok, tl, w, dtype)
    x = torch.from_numpy(lp).to(dev).to(ref.DTYPES[dtype])
    wide = torch.full((T, B + 1, V + 4), float("nan"), dtype=x.dtype, device=dev)
    wide[:, 1:, 3:3 + V] = x.transpose(0, 1)
    view = wide[:, 1:, 3:3 + V].transpose(0, 1)
    assert view.stride(0) != T * V and view.stride(1) != V
    more_tok = torch.full((B, N + 5, U + 11), -7, dtype=torch.int32, device=dev)
    more_tok[:, 2:2 + N, 1:1 + U] = torch.from_numpy(tok).to(dev)
    more_tl = torch.full((B, N + 5), 10 ** 9, dtype=torch.int32, device=dev)
    more_tl[:, 2:2 + N] = torch.from_numpy(tl).to(dev)
    args = (view, torch.from_numpy(ln).to(dev), more_tok[:, 2:2 + N, 1:1 + U], more_tl[:, 2:2 + N])
    out = binding.ctc_score(*args, want_grad=True)
    grad = binding.ctc_score_grad(*args, torch.from_numpy(w).to(dev), out["workspace"])
    assert grad.is_contiguous()
    assert out["scores"].cpu().numpy().tobytes() == plain[1].tobytes()
    assert grad.double().cpu().numpy().tobytes() == plain[3].tobytes()


def test_one_emission_for_all_utterances(dev):
    """An expanded batch (stride 0) is read as such."""
    lp, ln, tok, tl, w = make(15, 1, 3, 25, 8, 6, lengths=[25])
    x = torch.from_numpy(lp).to(dev).expand(4, 25, 8)
    args = (x, torch.full((4,), 25, dtype=torch.int32, device=dev), torch.from_numpy(tok).to(dev).expand(4, 3, 6),
            torch.from_numpy(tl).to(dev).expand(4, 3))
    s = binding.ctc_score(*args)["scores"].cpu().numpy()
    assert (s == s[:1]).all() and np.isfinite(s[0, tl[0] <= 5]).any()


@pytest.mark.parametrize("shape", [(2, 2, 12, 6, 4), (1, 1, 90, 8, 70)])
def test_gradient_against_differences(dev, shape):
    """Central differences of the scores: error h^2/6 times a third derivative of at most 1 (a third central moment of
    a variable in [0,1] is below 1/4), and the scores' own error over h."""
    B, N, T, V, U = shape
    lp, ln, tok, tl, w = make(16, B, N, T, V, U, lengths=[T] * B, token_lengths=np.full((B, N), max(1, U // 2)))
    _, scores, _, grad = on_gpu(dev, lp, ln, tok, tl, w)
    args = [torch.from_numpy(a).to(dev) for a in (ln, tok, tl)]
    rng = np.random.default_rng(0)
    h = 2.0 ** -10
    x = torch.from_numpy(lp).to(dev)
    # values on a grid of 2^-12, so that adding h is exact in fp32
    x = torch.round(x * 4096) / 4096
    out = binding.ctc_score(x, *args, want_grad=True)
    grad = binding.ctc_score_grad(x, *args, torch.from_numpy(w).to(dev), out["workspace"]).double().cpu().numpy()
    for _ in range(40):
        b, t = rng.integers(B), rng.integers(T)
        v = int(rng.choice([0, *tok[b, 0, :tl[b, 0]]]))
        said = []
        for sign in (1, -1):
            y = x.clone()
            y[b, t, v] += sign * h
            said.append((binding.ctc_score(y, *args)["scores"].cpu().numpy() * w)[b].sum())
        want = (said[0] - said[1]) / (2 * h)
        tol = np.abs(w[b]).sum() * (h * h / 6 + 5 * 2.0 ** -24 + ref.score_tolerance(T, scores[b].min()) / h)
        assert abs(grad[b, t, v] - want) <= tol


def test_gradient_from_one_workspace_again_and_other_weights(dev):
    lp, ln, tok, tl, w = make(17, 3, 4, 50, 32, 15)
    x = torch.from_numpy(lp).to(dev)
    args = [torch.from_numpy(a).to(dev) for a in (ln, tok, tl)]
    out = binding.ctc_score(x, *args, want_grad=True)
    W = torch.from_numpy(w).to(dev)
    first = binding.ctc_score_grad(x, *args, W, out["workspace"])
    other = binding.ctc_score_grad(x, *args, -2.0 * W, out["workspace"])
    again = binding.ctc_score_grad(x, *args, W, out["workspace"])
    assert torch.equal(first, again) and torch.equal(other, -2.0 * first)
    zero = binding.ctc_score_grad(x, *args, torch.zeros_like(W), out["workspace"])
    assert not zero.any()
    bad = W.clone()
    bad[1, 0] = float("nan")
    tl_fine = np.isfinite(out["scores"].cpu().numpy())
    odd = binding.ctc_score_grad(x, *args, bad, out["workspace"])
    if tl_fine[1, 0]:
        assert torch.isnan(odd[1, :int(ln[1])]).all()
    assert torch.equal(odd[0], first[0]) and torch.equal(odd[2], first[2])


def test_workspace_of_exactly_its_size_and_outputs_stay_inside(dev):
    lp, ln, tok, tl, w = make(18, 2, 3, 31, 17, 11)
    x = torch.from_numpy(lp).to(dev)
    args = [torch.from_numpy(a).to(dev) for a in (ln, tok, tl)]
    n = binding.score_workspace_bytes(2, 31, 3, 11)
    buffer = torch.full((n + 8192,), 0x5A, dtype=torch.uint8, device=dev)
    start = -buffer.data_ptr() % 256 + 256
    ws = buffer[start:start + n]
    out = binding.ctc_score(x, *args, want_grad=True, workspace=ws)
    grad = binding.ctc_score_grad(x, *args, torch.from_numpy(w).to(dev), ws)
    fresh = on_gpu(dev, lp, ln, tok, tl, w)
    assert out["scores"].cpu().numpy().tobytes() == fresh[1].tobytes()
    assert grad.double().cpu().numpy().tobytes() == fresh[3].tobytes()
    assert bool((buffer[:start] == 0x5A).all()) and bool((buffer[start + n:] == 0x5A).all())
    with pytest.raises(binding.FltopError):
        binding.ctc_score(x, *args, workspace=ws[:-256])


def test_same_bits_again_and_on_another_stream(dev):
    lp, ln, tok, tl, w = make(19, 9, 6, 120, 32, 40)
    base = on_gpu(dev, lp, ln, tok, tl, w)
    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    for stream in (None, side, side):
        got = on_gpu(dev, lp, ln, tok, tl, w, stream=stream) if stream is None else None
        if got is None:
            x = torch.from_numpy(lp).to(dev)
            args = [torch.from_numpy(a).to(dev) for a in (ln, tok, tl)]
            W = torch.from_numpy(w).to(dev)
            side.wait_stream(torch.cuda.current_stream(dev))
            out = binding.ctc_score(x, *args, want_grad=True, stream=side)
            grad = binding.ctc_score_grad(x, *args, W, out["workspace"], stream=side)
            torch.cuda.synchronize()
            got = (None, out["scores"].cpu().numpy(), None, grad.double().cpu().numpy())
        assert got[1].tobytes() == base[1].tobytes() and got[3].tobytes() == base[3].tobytes()


def test_captured_and_replayed(dev):
    lp, ln, tok, tl, w = make(20, 4, 2, 70, 32, 20)
    x = torch.from_numpy(lp).to(dev)
    args = [torch.from_numpy(a).to(dev) for a in (ln, tok, tl)]
    W = torch.from_numpy(w).to(dev)
    binding.ctc_score(x, *args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = binding.ctc_score(x, *args, want_grad=True)
        grad = binding.ctc_score_grad(x, *args, W, out["workspace"])
    for turn in range(4):
        y = torch.roll(torch.from_numpy(lp).to(dev), turn, 0)
        x.copy_(y)
        W.mul_(-0.5)
        graph.replay()
        torch.cuda.synchronize()
        eager = binding.ctc_score(y, *args, want_grad=True)
        want = binding.ctc_score_grad(y, *args, W, eager["workspace"])
        torch.cuda.synchronize()
        assert torch.equal(out["scores"], eager["scores"]) and torch.equal(grad, want)


def test_scores_of_the_search_are_reached_when_nothing_is_pruned(dev):
    """With every token kept and a beam that no prefix falls out of, the search's masses are the full likelihood."""
    B, T, V, beam = 3, 5, 4, 1024
    lp = synth.random_emissions(21, B, T, V, flat=1.0)
    ln = np.array([5, 4, 5], np.int32)
    x, lengths = torch.from_numpy(lp).to(dev), torch.from_numpy(ln).to(dev)
    out = binding.decode(x, lengths, beam, 0.0, want_nbest=True)
    got = binding.ctc_score(x, lengths, out["nbest_tokens"], out["nbest_lengths"], out["nbest_count"])["scores"].cpu().numpy()
    mass = np.logaddexp(out["nbest_pb"].cpu().numpy(), out["nbest_pnb"].cpu().numpy())
    count = out["nbest_count"].cpu().numpy()
    for b in range(B):
        assert count[b] > 50
        # both sides round each of T frames a few times, in fp64
        assert np.all(np.abs(got[b, :count[b]] - mass[b, :count[b]]) <= 64 * 2.0 ** -52 * (1 + np.abs(mass[b, :count[b]])))
        assert np.isneginf(got[b, count[b]:]).all()
        # every prefix is there, so they are certain together
        assert abs(np.exp(got[b, :count[b]]).sum() - 1.0) <= 1e-5  # emissions are normalised to fp32


def test_pruned_search_bounds_from_below(dev):
    w = synth.WORKLOADS["cfg2_batch64"]
    lp, ln = synth.make_emissions(w, utterances=range(6))
    x, lengths = torch.from_numpy(lp).to(dev), torch.from_numpy(ln).to(dev)
    out = binding.decode(x, lengths, 16, 0.01, want_nbest=True)
    longest = int(out["nbest_lengths"].max())
    got = binding.ctc_score(x, lengths, out["nbest_tokens"][:, :, :longest], out["nbest_lengths"],
                            out["nbest_count"])["scores"].cpu().numpy()
    mass = np.logaddexp(out["nbest_pb"].cpu().numpy(), out["nbest_pnb"].cpu().numpy())
    for b in range(6):
        n = int(out["nbest_count"][b])
        assert np.all(got[b, :n] >= mass[b, :n] - 1e-9)
        assert np.all(got[b, :n] <= 1e-4)  # rows are normalised to fp32: 500 frames of 2^-24 and more


def test_places_beyond_32_bits(dev):
    """More than 2^31 kept pairs of states, 16 bytes each: the last hypotheses are as good as the first."""
    B, N, T, U, V = 112, 32, 1400, 1900, 8
    assert binding.score_workspace_bytes(B, T, N, U) > 2 ** 35
    lp, ln, tok, tl, w = make(22, 1, 1, T, V, 30, lengths=[T], token_lengths=[[30]])
    x = torch.from_numpy(lp).to(dev).expand(B, T, V)
    tokens = torch.zeros((B, N, U), dtype=torch.int32, device=dev)
    tokens[:, :, :30] = torch.from_numpy(tok[0, 0]).to(dev)
    lengths = torch.full((B,), T, dtype=torch.int32, device=dev)
    tls = torch.full((B, N), 30, dtype=torch.int32, device=dev)
    out = binding.ctc_score(x, lengths, tokens, tls, want_grad=True)
    weights = torch.zeros((B, N), dtype=torch.float64, device=dev)
    weights[:, -1] = w[0, 0]
    grad = binding.ctc_score_grad(x, lengths, tokens, tls, weights, out["workspace"])
    s = out["scores"].cpu().numpy()
    want, g, size, quanta = ref.scores_and_grad(lp.astype(np.float64), ln, tok, tl, w)
    assert (s == s[0, 0]).all() and abs(s[0, 0] - want[0, 0]) <= ref.score_tolerance(T, want[0, 0])
    got = grad[-1].double().cpu().numpy()
    assert torch.equal(grad[0], grad[-1])
    assert np.all(np.abs(got - g[0]) <= ref.grad_tolerance("f32", T, g, size, quanta * 2000)[0])


@pytest.mark.parametrize("V", [32, 65])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 15, 16, 17, 23, 24, 25])
def test_ends_of_utterances_within_a_block(dev, T, V):
    """Lengths of every remainder, hypotheses that fill them and that are empty."""
    lengths = [T, T - 1, max(0, T - 3), max(0, T - 6), T]
    rng = np.random.default_rng(T)
    tl = [[0, (n + 1) // 2, rng.integers(0, T + 1)] for n in lengths]
    check(dev, *make(T + V, 5, 3, T, V, T, lengths=lengths, token_lengths=tl, repeats=0.1))


@pytest.mark.parametrize("V", [29, 90])
@pytest.mark.parametrize("U", [127, 128, 383, 384, 511, 512, 767, 768, 895, 896, 959, 960])
def test_room_at_the_borders_of_the_builds(dev, U, V):
    """Room of U tokens, hypotheses that take all of it and less; only the room chooses how the lattice is laid out."""
    T = U + U // 8 + 3
    lp, ln, tok, tl, w = make(U + V, 1, 3, T, V, U, lengths=[T], token_lengths=[[U, U // 2, 3]], flat=0.5, repeats=0.02)
    check(dev, lp, ln, tok, tl, w)


@pytest.mark.parametrize("V", [32, 100])
def test_many_hypotheses(dev, V):
    """So many that workgroups of more wavefronts a compute unit are taken."""
    check(dev, *make(V, 18, 30, 40, V, 12))


@pytest.mark.parametrize("V", [32, 70])
def test_rows_of_an_untrained_model(dev, V):
    """Far from each alignment being alike: masses of neighbours lie hundreds of nats apart."""
    rng = np.random.default_rng(V)
    lp, ln, tok, tl, w = make(V, 2, 2, 300, V, 110, lengths=[300, 293], token_lengths=[[100, 20], [110, 1]])
    x = rng.standard_normal(lp.shape) * 4
    lp = (x - np.log(np.exp(x).sum(-1, keepdims=True))).astype(np.float32)
    check(dev, lp, ln, tok, tl, w)


@pytest.mark.parametrize("V", [12, 80])
@pytest.mark.parametrize("shift", [9.0, 11.0, 60.0, -35.0, -60.0])
def test_rows_that_are_not_normalised(dev, V, shift):
    """Emissions far above 0 or far below are as good as any; the occupancies do not see a shift."""
    lp, ln, tok, tl, w = make(V, 2, 3, 43, V, 12, lengths=[43, 40])
    check(dev, lp + np.float32(shift), ln, tok, tl, w)


def test_a_vocabulary_whose_sums_are_taken_in_ranges(dev):
    lp, ln, tok, tl, w = make(77, 2, 3, 21, binding.MAX_VOCAB - 1, 9, lengths=[21, 18])
    check(dev, lp, ln, tok, tl, w)


def test_two_calls_at_once(dev):
    """Two streams, each with a workspace of its own."""
    data = [make(50 + i, 3, 4, 90 + i, 32, 20) for i in range(2)]
    streams = [torch.cuda.Stream(dev) for _ in range(2)]
    put = [[torch.from_numpy(np.ascontiguousarray(a)).to(dev) for a in d] for d in data]
    alone = []
    for x, ln, tok, tl, w in put:
        out = binding.ctc_score(x, ln, tok, tl, want_grad=True)
        alone.append((out["scores"], binding.ctc_score_grad(x, ln, tok, tl, w, out["workspace"])))
    torch.cuda.synchronize()
    for _ in range(3):
        outs = [binding.ctc_score(*p[:4], want_grad=True, stream=s) for p, s in zip(put, streams)]
        grads = [binding.ctc_score_grad(*p[:5], o["workspace"], stream=s) for p, o, s in zip(put, outs, streams)]
        torch.cuda.synchronize()
        for (scores, grad), o, g in zip(alone, outs, grads):
            assert torch.equal(scores, o["scores"]) and torch.equal(grad, g)
