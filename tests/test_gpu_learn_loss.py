"""preference_loss, policy_loss and policy_loss_logits against their formulas in 64 bits and against differences, and a
training step from the search's n-best list to the gradient of the emissions."""
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


def put(dev, *arrays):
    return [None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dev) for a in arrays]


# exp, log1p and the few operations around them, each within two half steps of fp64, and sums of n terms
def loss_tolerance(n, size):
    return (n + 40) * 2.0 ** -52 * size


# ---- pairs -------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("kind", ["sigmoid", "hinge", "square"])
@pytest.mark.parametrize("B,N,M", [(1, 1, 1), (1, 2, 1), (64, 2, 1), (3, 5, 10), (7, 4, 3), (2, 100, 4950), (5, 1024, 77),
                                   (1, 7, 257), (300, 3, 2)])
def test_pairs(dev, kind, B, N, M):
    rng = np.random.default_rng(B + N + M)
    s, q = -100 * rng.random((B, N)), -100 * rng.random((B, N))
    pairs = rng.integers(0, N, (B, M, 2)).astype(np.int32)  # the same pair twice, and a hypothesis against itself, too
    eps = 0.1 if kind == "sigmoid" else 0.0
    S, P, Q = put(dev, s, pairs, q)
    for r, R in ((None, None), (q, Q)):
        out = binding.preference_loss(S, P, ref_scores=R, kind=kind, beta=0.3, label_smoothing=eps, scale=3.0)
        loss, margins, grad, used = ref.preference(s, pairs, r, None, kind, 0.3, eps, 3.0)
        # a margin is three sums of numbers below 100, a loss's slope at most 2 (square), its derivative's 2
        err = 4 * 2.0 ** -53 * 200
        top = {"sigmoid": 0.3, "hinge": 0.3, "square": 2 * 200.0 + 4}[kind]
        assert np.all(np.abs(out["margins"].cpu().numpy() - margins) <= err)
        assert abs(float(out["loss"]) - loss) <= top * err + loss_tolerance(used, abs(loss) + 1)
        worst = np.zeros((B, N))
        for b in range(B):
            np.add.at(worst[b], pairs[b].ravel(), 3.0 / used)
        assert np.all(np.abs(out["grad_scores"].cpu().numpy() - grad) <= worst * (2 * err + loss_tolerance(2 * M, top)))


def test_pairs_that_take_no_part(dev):
    rng = np.random.default_rng(1)
    B, N, M = 6, 5, 8
    s, q = -10 * rng.random((B, N)), -10 * rng.random((B, N))
    s[0, 1], s[1, 0], q[2, 3], q[3, 4] = -np.inf, np.nan, -np.inf, np.inf
    pairs = rng.integers(0, N, (B, M, 2)).astype(np.int32)
    pairs[4, 2] = (-1, 0)
    pairs[4, 3] = (0, N)
    pairs[4, 4] = (2 ** 31 - 1, -2 ** 31)
    counts = np.array([8, 99, 5, 0, 8, -3], np.int32)
    S, P, Q, C = put(dev, s, pairs, q, counts)
    out = binding.preference_loss(S, P, ref_scores=Q, pair_counts=C, beta=0.5)
    loss, margins, grad, _ = ref.preference(s, pairs, q, counts, beta=0.5)
    got = out["margins"].cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(margins))
    np.testing.assert_allclose(got, margins, rtol=0, atol=1e-13)
    np.testing.assert_allclose(float(out["loss"]), loss, rtol=0, atol=loss_tolerance(48, 8))
    np.testing.assert_allclose(out["grad_scores"].cpu().numpy(), grad, rtol=0, atol=loss_tolerance(48, 1))
    none = binding.preference_loss(S, P, pair_counts=torch.zeros_like(C))
    assert float(none["loss"]) == 0.0 and not none["grad_scores"].any() and torch.isnan(none["margins"]).all()


def test_margins_far_out(dev):
    """Log ratios of thousands: no overflow, and the loss is linear there."""
    s = np.array([[0.0, -5000.0, 5000.0, -1e300, 1e300]])
    pairs = np.array([[[0, 1], [1, 0], [2, 1], [1, 2]]], np.int32)
    S, P = put(dev, s, pairs)
    out = binding.preference_loss(S, P, beta=1.0)
    assert float(out["loss"]) == (0.0 + 5000.0 + 0.0 + 10000.0) / 4
    assert out["grad_scores"].cpu().numpy()[0].tolist() == [0.25, -0.5, 0.25, 0.0, 0.0]
    far = binding.preference_loss(S, put(dev, np.array([[[3, 4]]], np.int32))[0], beta=0.1)
    assert abs(float(far["loss"]) - 2e299) <= 2e299 * 2.0 ** -50 and far["grad_scores"].cpu().numpy()[0, 3] == -0.1


def test_preference_gradient_against_differences(dev):
    rng = np.random.default_rng(5)
    s, q = -20 * rng.random((3, 6)), -20 * rng.random((3, 6))
    pairs = rng.integers(0, 6, (3, 9, 2)).astype(np.int32)
    S, P, Q = put(dev, s, pairs, q)
    for kind, eps in (("sigmoid", 0.2), ("square", 0.0)):
        go = lambda x: binding.preference_loss(x, P, ref_scores=Q, kind=kind, beta=0.2, label_smoothing=eps)  # noqa: E731
        grad, h = go(S)["grad_scores"].cpu().numpy(), 1e-5
        for b, n in ((0, 0), (1, 3), (2, 5), (2, 1)):
            d = torch.zeros_like(S)
            d[b, n] = h
            want = (float(go(S + d)["loss"]) - float(go(S - d)["loss"])) / (2 * h)
            # third derivatives are below beta^3, the losses below 1600 and rounded to 2^-50
            assert abs(grad[b, n] - want) <= h * h + 1600 * 2.0 ** -48 / h


# ---- the policy loss over log-probabilities ------------------------------------------------------------------------------


def policy_inputs(seed, B, N):
    rng = np.random.default_rng(seed)
    l = -50 * rng.random((B, N))
    old, q = l + 0.3 * rng.standard_normal((B, N)), l + 0.5 * rng.standard_normal((B, N))
    return l, old, q, rng.standard_normal((B, N))


@pytest.mark.parametrize("reduction", ["token", "sequence", "sum"])
@pytest.mark.parametrize("B,N", [(1, 1), (1, 5), (64, 2), (3, 255), (2, 256), (9, 257), (1, 5000), (700, 7), (4097, 1)])
def test_policy(dev, reduction, B, N):
    l, old, q, A = policy_inputs(B + N, B, N)
    rng = np.random.default_rng(B * N)
    for counts in (None, rng.integers(-1, N + 2, B).astype(np.int32)):
        for r in (None, q):
            L, O, Q, Adv, C = put(dev, l, old, r, A, counts)
            out = binding.policy_loss(L, O, Adv, ref_scores=Q, counts=C, clip_low=0.1, clip_high=0.3, kl_weight=0.4,
                                      reduction=reduction, scale=-2.0)
            part = np.arange(N) < (np.full((B, 1), N) if counts is None else counts[:, None])
            want = ref.policy(l, old, A, part, r, 0.1, 0.3, 0.4, reduction, -2.0)
            n = part.sum() if reduction == "sum" else 1
            # ratios below e^2, advantages below 6, KL below e^3; scores of 50 round to 50 * 2^-52 in each difference
            tol = loss_tolerance(200, 100) * max(n, 1)
            assert abs(float(out["loss"]) - want[0]) <= tol and abs(float(out["kl"]) - want[1]) <= tol
            assert abs(float(out["clipped"]) - want[2]) <= 2.0 ** -50
            assert np.all(np.abs(out["grad_scores"].cpu().numpy() - want[3]) <= 2 * loss_tolerance(200, 100))
            assert not out["grad_scores"].cpu().numpy()[~part].any()


def test_policy_numbers_that_are_not_finite_take_no_part(dev):
    l, old, q, A = policy_inputs(3, 5, 6)
    part = np.ones((5, 6), bool)
    for x, at, v in ((l, (0, 1), -np.inf), (old, (1, 2), -np.inf), (q, (2, 3), np.nan), (A, (3, 4), np.inf),
                     (l, (4, 0), np.nan)):
        x[at] = v
        part[at] = False
    l[4] = -np.inf
    part[4] = False  # a whole row
    for reduction in ("token", "sequence", "sum"):
        L, O, Q, Adv = put(dev, l, old, q, A)
        out = binding.policy_loss(L, O, Adv, ref_scores=Q, kl_weight=0.1, reduction=reduction)
        want = ref.policy(l, old, A, part, q, kl_weight=0.1, reduction=reduction)
        np.testing.assert_allclose([float(out[k]) for k in ("loss", "kl", "clipped")], want[:3], rtol=0, atol=1e-11)
        np.testing.assert_allclose(out["grad_scores"].cpu().numpy(), want[3], rtol=0, atol=1e-11)
    L.fill_(float("nan"))
    out = binding.policy_loss(L, O, Adv)
    assert [float(out[k]) for k in ("loss", "kl", "clipped")] == [0.0, 0.0, 0.0] and not out["grad_scores"].any()


def test_policy_borders(dev):
    """At a ratio of one nothing is clipped; the gradient goes through where A r equals its clipped value."""
    one = np.zeros((1, 4))
    A = np.array([[1.0, -1.0, 0.0, 2.0]])
    L, Adv = put(dev, one, A)
    out = binding.policy_loss(L, L, Adv, clip_low=0.0, clip_high=0.0, reduction="sum")
    assert out["grad_scores"].cpu().numpy().tolist() == (-A).tolist() and float(out["clipped"]) == 0.0
    old = np.array([[-2.0, -2.0, 2.0, 2.0]])  # r = e^2, e^2, e^-2, e^-2
    A = np.array([[1.0, -1.0, 1.0, -1.0]])
    O, Adv = put(dev, old, A)
    out = binding.policy_loss(L, O, Adv, clip_low=0.25, clip_high=0.5, reduction="sum")
    g = out["grad_scores"].cpu().numpy()[0]
    assert g[0] == 0.0 and g[3] == 0.0 and abs(g[1] - np.exp(2)) < 1e-14 and abs(g[2] + np.exp(-2)) < 1e-15
    assert float(out["clipped"]) == 0.5 and abs(float(out["loss"]) - (-1.5 + np.exp(2) - np.exp(-2) + 0.75)) < 1e-14


def test_policy_ratios_that_overflow_are_what_the_formula_gives(dev):
    L, O = put(dev, np.array([[0.0, 0.0]]), np.array([[-800.0, 800.0]]))
    (A,) = put(dev, np.array([[-1.0, 1.0]]))
    out = binding.policy_loss(L, O, A, reduction="sum")
    assert float(out["loss"]) == np.inf and out["grad_scores"].cpu().numpy()[0].tolist() == [np.inf, 0.0]


# ---- the policy loss over logits -----------------------------------------------------------------------------------------


def logits_inputs(seed, B, T, V, dtype, flat=2.0):
    gen = torch.Generator().manual_seed(seed)
    x = (flat * torch.randn((B, T, V), generator=gen)).to(ref.DTYPES[dtype])
    tok = torch.randint(0, V, (B, T), generator=gen).to(torch.int32)
    lp = torch.log_softmax(x.double(), 2).gather(2, tok[..., None].long())[..., 0]
    old, q = (lp + 0.2 * torch.randn((B, T), generator=gen)).float(), (lp + 0.3 * torch.randn((B, T), generator=gen)).float()
    for border in (np.log(0.8), np.log(1.3)):  # decided alike by fp32 and fp64 statistics
        near = ((lp - old.double()) - border).abs() < 1e-3
        old = torch.where(near, old - 4e-3, old)
    A = torch.randn((B, T), generator=gen)
    lengths = torch.randint(0, T + 1, (B,), generator=gen).to(torch.int32)
    lengths[0] = T
    return x, tok, lengths, old, q, A


def check_logits(dev, x, tok, lengths, old, q, A, dtype, reduction="token", scale=1.0, stream=None, view=None):
    B, T, V = x.shape
    args = [a.to(dev) for a in (tok, lengths, old, A)]
    out = binding.policy_loss_logits(x.to(dev) if view is None else view, *args,
                                     ref_logps=None if q is None else q.to(dev), clip_low=0.2, clip_high=0.3,
                                     kl_weight=0.1, reduction=reduction, scale=scale, stream=stream)
    torch.cuda.synchronize()
    X = x.double().numpy()
    part = (np.arange(T) < lengths.numpy()[:, None]) & (tok.numpy() >= 0) & (tok.numpy() < V)
    t = np.where(part, tok.numpy(), 0)[..., None]
    with np.errstate(all="ignore"):
        top = X.max(2, keepdims=True)
        e = np.exp(X - top)
        p = e / e.sum(2, keepdims=True)
        others = e.sum(2) - np.take_along_axis(e, t, 2)[..., 0]
        l = np.take_along_axis(X - top, t, 2)[..., 0] - np.log(e.sum(2))
    adv = (A if A.dim() == 2 else A[:, None]).double().numpy() * np.ones((B, T))
    loss, kl, clipped, d = ref.policy(l, old.double().numpy(), adv, part, None if q is None else q.double().numpy(), 0.2, 0.3,
                                      0.1, reduction, scale)
    # fp32 exponentials of x - top: the difference rounded (|x - top| up to 24 matter: 24 * 2^-24), the exponential two
    # steps, and their sum as deep as a thread's share of the row
    err = (24 + 4 + 8 + V / 64) * 2.0 ** -24
    got = {k: v.double().cpu().numpy() for k, v in out.items()}
    fine = np.where(part, l, 0.0)
    assert np.all(np.abs(got["logps"] - fine) <= err + 2.0 ** -24 * np.abs(fine))
    assert not got["logps"][~part].any()
    n = part.sum() if reduction == "sum" else 1
    size = np.where(part, np.abs(adv) * 1.5 + 5, 0).max(initial=1)
    assert abs(got["loss"] - loss) <= n * size * err + 2.0 ** -24 * abs(loss)
    assert abs(got["kl"] - kl) <= n * 5 * err + 2.0 ** -24 * abs(kl)
    assert abs(got["clipped"] - clipped) <= 2.0 ** -24
    onehot = np.zeros_like(X)
    np.put_along_axis(onehot, t, 1.0, 2)
    want = np.where(part, d, 0.0)[..., None] * (onehot - np.where(part[..., None], p, 0.0))
    # d itself is off by |A| r e^... times err; every entry is a product of d and a probability
    dd = (np.abs(adv) * 3 + 5) * np.abs(scale) * err * weights(part, reduction)
    tol = (np.abs(d) * 3 * err + dd)[..., None] * np.where(onehot > 0, np.where(part, 1 - np.take_along_axis(p, t, 2)[..., 0], 0)[..., None], p)
    tol = np.where(part[..., None], tol + 1e-37, 0.0) + ref.HALF_STEP[dtype] * 1.01 * np.abs(want) + ref.SMALLEST[dtype]
    assert np.all(np.abs(got["grad_logits"] - want) <= tol)
    assert not got["grad_logits"][~part].any()
    return got


def weights(part, reduction):
    n = part.sum(1, keepdims=True)
    if reduction == "token":
        return part / max(part.sum(), 1)
    if reduction == "sequence":
        return part / (np.maximum(n, 1) * max((n > 0).sum(), 1))
    return part.astype(float)


VOCABULARIES = [1, 2, 3, 7, 24, 29, 31, 32, 33, 63, 64, 65, 127, 128, 130, 255, 256, 257, 511, 512, 513, 1000, 1024, 1025,
                2047, 2048, 2049, 4095, 4096, 4097, 8192, 8193, 16384, 16391, 32768, 32771, 50021, 65536, 65541]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", VOCABULARIES)
def test_vocabularies(dev, V, dtype):
    B, T = (3, 50) if V < 2000 else (2, 9)
    x, tok, lengths, old, q, A = logits_inputs(V, B, T, V, dtype)
    scale = 256.0 if dtype == "f16" else 1.0
    check_logits(dev, x, tok, lengths, old, q, A, dtype, scale=scale)


@pytest.mark.parametrize("V", [131072, 200003])
def test_very_large_vocabularies(dev, V):
    for dtype in ("f32", "bf16"):
        x, tok, lengths, old, q, A = logits_inputs(V, 1, 3, V, dtype)
        check_logits(dev, x, tok, lengths, old, q, A, dtype)


@pytest.mark.parametrize("reduction", ["token", "sequence", "sum"])
@pytest.mark.parametrize("B,T,V", [(1, 1, 32), (1, 1, 5000), (5, 1, 40), (300, 3, 32), (1, 2500, 29), (17, 130, 100),
                                   (2000, 2, 24)])
def test_shapes_and_reductions(dev, B, T, V, reduction):
    x, tok, lengths, old, q, A = logits_inputs(B + T, B, T, V, "f32")
    check_logits(dev, x, tok, lengths, old, q, A, "f32", reduction)
    check_logits(dev, x, tok, lengths, old, None, A[:, 0].contiguous(), "f32", reduction)


def test_frames_that_take_no_part(dev):
    x, tok, lengths, old, q, A = logits_inputs(4, 5, 20, 37, "f32")
    lengths[:] = torch.tensor([20, 0, -5, 99, 20])
    tok[0, :7] = -1          # a prompt
    tok[0, 9] = 37
    tok[3, 3] = 2 ** 31 - 1
    tok[3, 5] = -2 ** 31
    tok[4] = -100            # a row of which nothing takes part
    x[1], old[1], q[1], A[1] = (float("nan"),) * 4
    x[0, :7], old[0, :7], q[0, :7], A[0, :7] = (float("nan"),) * 4
    lengths_in = torch.clamp(lengths, max=20)
    for reduction in ("token", "sequence", "sum"):
        check_logits(dev, x, tok, lengths_in, old, q, A, "f32", reduction)
    got = check_logits(dev, x, torch.full_like(tok, -1), lengths, old, q, A, "f32")
    assert got["loss"] == 0 and got["kl"] == 0 and got["clipped"] == 0


def test_lengths_beyond_the_frames_are_clamped(dev):
    x, tok, lengths, old, q, A = logits_inputs(41, 3, 9, 33, "f32")
    a = check_logits(dev, x, tok, torch.tensor([9, 9, 4], dtype=torch.int32), old, q, A, "f32")
    b = check_logits(dev, x, tok, torch.tensor([2 ** 31 - 1, 10, 4], dtype=torch.int32), old, q, A, "f32")
    assert a["grad_logits"].tobytes() == b["grad_logits"].tobytes()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [32, 1000, 20000])
def test_masked_logits(dev, dtype, V):
    """-inf, the type's lowest value, and equal rows."""
    x, tok, lengths, old, q, A = logits_inputs(6, 2, 12, V, dtype)
    lengths[:] = 12
    low = torch.finfo(x.dtype).min
    for t, value in enumerate((-float("inf"), low, low / 2)):
        x[0, t, 1::2] = value
        x[0, 3 + t, :] = value
        x[0, 3 + t, 5] = 1.0   # all the mass on one token
        tok[0, t], tok[0, 3 + t] = 4, 5
    x[0, 6] = low              # a row of the lowest value: uniform
    x[0, 7] = 0.0
    x[1, 0] = 60000.0 if dtype == "f16" else 3e38
    lp = torch.log_softmax(x.double(), 2).gather(2, tok[..., None].long())[..., 0]
    assert torch.isfinite(lp).all()
    old, q = (lp + 0.05).float(), (lp - 0.1).float()
    check_logits(dev, x, tok, lengths, old, q, A, dtype, scale=64.0)


def test_a_token_without_mass(dev):
    """Its logit is -inf: the ratio is 0, and without a reference there is no gradient."""
    x, tok, lengths, old, _, A = logits_inputs(7, 1, 3, 40, "f32")
    tok[0, 0] = 3
    x[0, 0, 3] = -float("inf")
    A[0] = torch.tensor([1.0, 0.5, -0.5])
    args = [a.to(dev) for a in (x, tok, lengths, old, A)]
    out = binding.policy_loss_logits(*args, reduction="sum")
    assert float(out["logps"][0, 0]) == -np.inf and np.isfinite(float(out["loss"]))
    assert not out["grad_logits"][0, 0].any() and out["grad_logits"][0, 1].any()


def test_nearly_certain_tokens_keep_their_digits(dev):
    """p = 1 - 1e-9: ln p and the token's own gradient are not lost in 1 - 1."""
    V = 100
    x = torch.zeros((1, 4, V))
    x[0, :, 7] = torch.tensor([10.0, 20.0, 25.0, 30.0])
    tok = torch.full((1, 4), 7, dtype=torch.int32)
    lengths = torch.tensor([4], dtype=torch.int32)
    old, A = torch.zeros((1, 4)), torch.ones((1, 4))
    out = binding.policy_loss_logits(*[a.to(dev) for a in (x, tok, lengths, old, A)], reduction="sum")
    others = (V - 1) * np.exp(-x[0, :, 7].double().numpy())
    want = -np.log1p(others)
    # as many roundings as elsewhere, but all of them relative
    err = (24 + 4 + 8 + V / 64) * 2.0 ** -24
    assert np.all(np.abs(out["logps"][0].double().cpu().numpy() - want) <= err * np.abs(want))
    own = out["grad_logits"][0, :, 7].double().cpu().numpy()
    r = np.exp(want)
    assert np.all(np.abs(own + r * others / (1 + others)) <= 3 * err * others)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [32, 33, 1024, 1025, 20000])
def test_strides_of_logits(dev, dtype, V):
    x, tok, lengths, old, q, A = logits_inputs(8, 3, 14, V, dtype)
    plain = check_logits(dev, x, tok, lengths, old, q, A, dtype)
    wide = torch.full((14, 4, V + 5), float("nan"), dtype=x.dtype, device=dev)
    for at in (1, 3, 4, 5):  # alignments of the first value
        wide.fill_(float("nan"))
        view = wide[:, 1:, at:at + V].transpose(0, 1)
        view.copy_(x)
        if at + V <= V + 5:
            got = check_logits(dev, x, tok, lengths, old, q, A, dtype, view=view)
            assert got["grad_logits"].tobytes() == plain["grad_logits"].tobytes()
            assert got["loss"].tobytes() == plain["loss"].tobytes()


def test_rows_beyond_32_bits(dev):
    """More than 2^31 logits: the last rows as good as the first."""
    B, T, V = 2, 30000, 40000
    x = torch.empty((B, T, V), dtype=torch.bfloat16, device=dev)
    x.zero_()
    x[:, :, 5] = 3.0
    tok = torch.full((B, T), 5, dtype=torch.int32, device=dev)
    lengths = torch.full((B,), T, dtype=torch.int32, device=dev)
    one = torch.ones((B,), device=dev)
    out = binding.policy_loss_logits(x, tok, lengths, torch.full((B, T), -7.0, device=dev), one, reduction="sum")
    assert torch.equal(out["logps"], out["logps"][:1, :1].expand(B, T))
    assert abs(float(out["logps"][-1, -1]) - (3 - np.log(V - 1 + np.exp(3)))) <= 1e-4
    assert torch.equal(out["grad_logits"][1, T - 1], out["grad_logits"][0, 0])


def test_policy_logits_gradient_against_differences(dev):
    x, tok, lengths, old, q, A = logits_inputs(9, 2, 6, 30, "f32", flat=1.0)
    lengths[:] = 6
    x = torch.round(x * 1024) / 1024
    args = [a.to(dev) for a in (tok, lengths, old, A)]
    go = lambda y: binding.policy_loss_logits(y.to(dev), *args, ref_logps=q.to(dev), clip_low=0.2, clip_high=0.3,  # noqa: E731
                                              kl_weight=0.2, reduction="sum")
    grad, h = go(x)["grad_logits"].cpu(), 2.0 ** -6
    rng = np.random.default_rng(3)
    for _ in range(20):
        b, t = rng.integers(2), rng.integers(6)
        v = int(tok[b, t]) if rng.random() < 0.5 else int(rng.integers(30))
        gap = float(go(x)["logps"][b, t].cpu()) - float(old[b, t])
        if min(abs(gap - np.log(0.8)), abs(gap - np.log(1.3))) < 2 * h:
            continue  # the loss has a kink there
        up, down = x.clone(), x.clone()
        up[b, t, v] += h
        down[b, t, v] -= h
        want = (float(go(up)["loss"]) - float(go(down)["loss"])) / (2 * h)
        # third derivatives below 10 (|A| r and the KL's exponential), the loss below 30 and rounded to fp32
        assert abs(float(grad[b, t, v]) - want) <= 10 * h * h / 6 + 30 * 2.0 ** -23 / h


def test_same_bits_on_another_stream_and_in_a_graph(dev):
    x, tok, lengths, old, q, A = logits_inputs(10, 40, 60, 257, "bf16")
    X, K, N, O, Q, Adv = [a.to(dev) for a in (x, tok, lengths, old, q, A)]
    s = -50 * torch.rand((40, 60), dtype=torch.float64, device=dev)
    pairs = torch.randint(0, 60, (40, 30, 2), dtype=torch.int32, device=dev)

    def all_of_them(stream=None):
        a = binding.policy_loss_logits(X, K, N, O, Adv, ref_logps=Q, kl_weight=0.1, reduction="sequence", stream=stream)
        b = binding.policy_loss(s, s + 0.1, s, ref_scores=s - 0.2, kl_weight=0.3, stream=stream)
        c = binding.preference_loss(s, pairs, stream=stream)
        return [t for o in (a, b, c) for _, t in sorted(o.items())]

    base = [t.clone() for t in all_of_them()]
    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    other = all_of_them(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = all_of_them()
    same = lambda p, q: all(u.cpu().numpy().tobytes() == v.cpu().numpy().tobytes()  # noqa: E731
                            for u, v in zip((t.float() if t.dtype == torch.bfloat16 else t for t in p),
                                            (t.float() if t.dtype == torch.bfloat16 else t for t in q)))
    assert same(base, other)
    for _ in range(3):
        X.copy_(torch.roll(X, 1, 1))
        s.add_(-0.25)
        graph.replay()
        torch.cuda.synchronize()
        assert same(held, all_of_them())
        torch.cuda.synchronize()


def test_workspaces_of_exactly_their_size(dev):
    l, old, q, A = put(dev, *policy_inputs(2, 7, 9))
    for need, call in ((binding.load().fltop_policy_workspace_bytes(7, 1),
                        lambda ws: binding.policy_loss(l, old, A, workspace=ws)),
                       (binding.load().fltop_preference_workspace_bytes(7),
                        lambda ws: binding.preference_loss(l, torch.zeros((7, 3, 2), dtype=torch.int32, device=dev),
                                                           workspace=ws))):
        buffer = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device=dev)
        start = -buffer.data_ptr() % 256 + 256
        call(buffer[start:start + need])
        torch.cuda.synchronize()
        assert bool((buffer[:start] == 0x5A).all()) and bool((buffer[start + need:] == 0x5A).all())
        with pytest.raises(binding.FltopError):
            call(buffer[start:start + need - 256])


@pytest.mark.parametrize("call", ["preference", "policy"])
def test_a_training_step_from_the_search(dev, call):
    """decode -> scores of its n-best list -> loss -> gradient of the emissions -> a model's logits, as a trainer runs
    them, against the same in 64 bits."""
    w = synth.WORKLOADS["cfg2_batch64"]
    B, N, frames = 4, 6, 80
    lp, _ = synth.make_emissions(w, utterances=range(B))
    logits = torch.from_numpy(np.ascontiguousarray(lp[:, :frames])).to(dev).requires_grad_()
    emissions = torch.log_softmax(logits, 2)
    lengths = torch.tensor([80, 61, 80, 40], dtype=torch.int32, device=dev)
    found = binding.decode(emissions.detach(), lengths, 16, 0.001, want_nbest=True)
    U = int(found["nbest_lengths"].max())
    hyps = (found["nbest_tokens"][:, :N, :U], found["nbest_lengths"][:, :N], found["nbest_count"].clamp(max=N))
    x = emissions.detach()
    out = binding.ctc_score(x, lengths, *hyps, want_grad=True)
    gen = torch.Generator().manual_seed(1)
    shift = 0.1 * torch.randn((B, N), generator=gen, dtype=torch.float64)
    advantages = torch.randn((B, N), generator=gen, dtype=torch.float64)
    pairs = torch.randint(0, N, (B, 5, 2), generator=gen).to(torch.int32)
    old = out["scores"] + shift.to(dev)
    if call == "policy":
        told = binding.policy_loss(out["scores"], old, advantages.to(dev), ref_scores=old - 0.05, counts=hyps[2],
                                   kl_weight=0.1)
    else:
        told = binding.preference_loss(out["scores"], pairs.to(dev), ref_scores=old, beta=0.3)
    grad = binding.ctc_score_grad(x, lengths, hyps[0], hyps[1], told["grad_scores"], out["workspace"], hyps[2])
    emissions.backward(grad)

    tokens, tls, counts = (t.cpu().numpy() for t in hyps)
    xs = x.double().cpu().numpy()
    s, _, _, _ = ref.scores_and_grad(xs, lengths.cpu().numpy(), tokens, tls, np.ones((B, N)), counts)
    o = old.cpu().numpy()
    part = (np.arange(N) < counts[:, None]) & np.isfinite(s) & np.isfinite(o)
    if call == "policy":
        loss, _, _, d = ref.policy(s, o, advantages.numpy(), part, o - 0.05, kl_weight=0.1)
    else:
        loss, _, d, _ = ref.preference(s, pairs.numpy(), o, beta=0.3)
    assert part.sum() > 10 and abs(float(told["loss"]) - loss) <= 1e-11
    assert np.all(np.abs(told["grad_scores"].cpu().numpy() - d) <= 1e-11)
    _, g, size, quanta = ref.scores_and_grad(xs, lengths.cpu().numpy(), tokens, tls, np.where(part, d, 0.0), counts)
    got = grad.double().cpu().numpy()
    near = ref.grad_tolerance("f32", frames, g, size, quanta) + 1e-10
    assert np.all(np.abs(got - g) <= near)
    # the softmax's own gradient on top, in 64 bits from the same emissions: fp32 sums of 32 terms
    p = np.exp(xs)
    want = g - p * g.sum(2, keepdims=True)
    assert np.all(np.abs(logits.grad.double().cpu().numpy() - want) <= 34 * 2.0 ** -23 * (np.abs(g).sum(2, keepdims=True) + 1e-3))


@pytest.mark.parametrize("kind", ["sigmoid", "square"])
@pytest.mark.parametrize("B,N,M", [(64, 32, 64), (1, 2048, 4096), (3, 683, 5), (64, 32, 65), (2, 2048, 513), (1, 1, 4096),
                                   (4096, 1, 1), (2, 3, 5000)])
def test_pairs_at_the_borders_of_the_launches(dev, kind, B, N, M):
    if N > binding.MAX_BEAM:
        N = binding.MAX_BEAM
    rng = np.random.default_rng(B * N + M)
    s = -100 * rng.random((B, N))
    pairs = rng.integers(0, N, (B, M, 2)).astype(np.int32)
    out = binding.preference_loss(*put(dev, s, pairs), kind=kind, beta=0.3, scale=2.0)
    loss, margins, grad, used = ref.preference(s, pairs, None, None, kind, 0.3, 0.0, 2.0)
    err = 2.0 ** -53 * 200
    top = {"sigmoid": 0.3, "square": 2 * 100.0 + 4}[kind]
    assert np.all(np.abs(out["margins"].cpu().numpy() - margins) <= err)
    assert abs(float(out["loss"]) - loss) <= top * err + loss_tolerance(used, abs(loss) + 1)
    worst = np.zeros((B, N))
    for b in range(B):
        np.add.at(worst[b], pairs[b].ravel(), 2.0 / used)
    assert np.all(np.abs(out["grad_scores"].cpu().numpy() - grad) <= worst * (2 * err + loss_tolerance(2 * M, top)))


@pytest.mark.parametrize("B", [1, 5000])
def test_small_slopes_keep_their_digits(dev, B):
    """Where all pairs are won by far each derivative is e^-40 of beta, and still a number of 50 bits."""
    rng = np.random.default_rng(B)
    s = np.stack([np.zeros(B), -400 - 20 * rng.random(B)], 1)
    pairs = np.tile(np.array([[[0, 1]]], np.int32), (B, 1, 1))
    got = binding.preference_loss(*put(dev, s, pairs), beta=0.1)["grad_scores"].cpu().numpy()
    x = 0.1 * (s[:, 0] - s[:, 1])
    want = -0.1 / (1.0 + np.exp(x)) / B
    # beta times a margin is rounded once (42 * 2^-53 in e^x), the rest as in the other losses
    np.testing.assert_allclose(got, np.stack([want, -want], 1), rtol=42 * 2.0 ** -53 + loss_tolerance(2, 1), atol=0)


def test_pairs_at_an_odd_place(dev):
    """A list of pairs need not begin at a multiple of 8 bytes."""
    rng = np.random.default_rng(3)
    s = -10 * rng.random((2, 5))
    pairs = rng.integers(0, 5, (2, 6, 2)).astype(np.int32)
    room = torch.zeros(25, dtype=torch.int32, device=dev)
    view = room[1:].view(2, 6, 2)
    view.copy_(torch.from_numpy(pairs))
    S, P = put(dev, s, pairs)
    a, b = binding.preference_loss(S, P), binding.preference_loss(S, view)
    assert all(torch.equal(a[k], b[k]) for k in ("loss", "margins", "grad_scores"))


@pytest.mark.parametrize("reduction", ["token", "sequence", "sum"])
@pytest.mark.parametrize("B,N", [(1, 2048), (2, 1025), (2048, 1), (2049, 1), (31, 66), (33, 63)])
def test_policy_at_the_borders_of_the_launches(dev, B, N, reduction):
    test_policy(dev, reduction, B, N)
