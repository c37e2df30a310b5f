"""The operators that learn from hypotheses: what of them is measured, in their plain form and as the framework's calls.

    ctc_score, ctc_score_grad   log-probability of N hypotheses per utterance under its emissions, summed over all their
                                alignments, and its gradient to the emissions
    preference_loss             paired log ratios of an utterance's hypotheses, with gradient
    policy_loss                 clipped policy loss with a KL term over hypotheses, with gradient
    policy_loss_logits          the same over the frames (or tokens) of [B,T,V] logits, log-softmax inside, with gradient

`listed()` names a dozen calls, `draw(rng)` gives one more of the same ranges:

    batch       1 .. 256 utterances of 20 .. 1500 frames, equal or ragged lengths, 1 .. 32 hypotheses each
    vocabulary  24 .. 4096 tokens; rows of logits up to 50021, odd sizes among them
    pairs       1 .. 4950 of an utterance, up to 100 hypotheses
    types       float32, bfloat16, float16 emissions and logits; float64 scores

Emissions follow the recipe of `synth.py`: sharply peaked rows, most frames blank; hypotheses are the path's own tokens
with substitutions and deletions, as an n-best list holds them.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CLIP_LOW, CLIP_HIGH, KL_WEIGHT, BETA, SMOOTHING = 0.2, 0.25, 0.05, 0.2, 0.05
LOSS_SCALE = {"f16": 1024.0}  # gradients in float16 are scaled, as trainers do, to stay clear of its smallest numbers
MOST_LATTICE = 256 * 1500 * 1351  # frames times states, of the largest listed
MOST_ROWS_BYTES = 2 * 8 * 509 * 50021


def _ctc(name, kind, B, N, T, V, **more):
    case = {"name": name, "kind": kind, "B": B, "N": N, "T": T, "V": V, "dtype": "f32", "ragged": False,
            "p_blank": 0.65}
    case.update(more)
    return case


def _pairs(name, B, N, M, loss):
    return {"name": name, "kind": "preference", "B": B, "N": N, "M": M, "loss": loss}


def _rows(name, B, T, V, dtype, **more):
    case = {"name": name, "kind": "rows", "B": B, "T": T, "V": V, "dtype": dtype, "ragged": True, "prompt": 0.0,
            "reduce": "token"}
    case.update(more)
    return case


def listed():
    return [
        # one short utterance and its transcript: the latency of a single training call
        _ctc("ctc_single", "ctc", 1, 1, 200, 32),
        # an ordinary training batch of characters: one transcript each, scores and gradient
        _ctc("ctc_batch64", "ctc", 64, 1, 500, 32),
        # a corpus batch with utterances of 5 to 30 s
        _ctc("ctc_varlen256", "ctc", 256, 1, 1500, 32, ragged=True),
        # sub-words, mixed precision, eight hypotheses of an n-best list each
        _ctc("ctc_subword_nbest", "ctc", 32, 8, 400, 1024, dtype="bf16", ragged=True, p_blank=0.85),
        # rescoring: full likelihoods of the search's final beam, no gradient
        _ctc("rescore_nbest", "rescore", 64, 32, 500, 32),
        # a step of preference training from end to end: scores, pairs, gradient to the emissions
        _ctc("train_preference", "train", 32, 4, 500, 32, M=6),
        # one pair for each utterance of a batch: the smallest call
        _pairs("pair_each", 64, 2, 1, "sigmoid"),
        # every pair of a long n-best list
        _pairs("all_pairs", 128, 100, 4950, "sigmoid"),
        # a group of hypotheses for each utterance, lists of different lengths
        {"name": "policy_nbest", "kind": "policy", "B": 256, "N": 32, "reduce": "sequence"},
        # frames of character emissions: short rows
        _rows("frames_chars", 256, 1500, 32, "f32"),
        # sub-word rows in bfloat16
        _rows("frames_subword", 128, 400, 1024, "bf16", reduce="sequence"),
        # tokens of a large odd vocabulary behind a prompt that takes no part
        _rows("tokens_large_vocab", 8, 509, 50021, "f16", prompt=0.25),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(("ctc", "ctc", "rescore", "train", "preference", "policy", "rows", "rows"))
        dtype = rng.choice(("f32", "f32", "bf16", "f16"))
        if kind == "preference":
            N = _log_int(rng, 2, 100)
            c = _pairs("", _log_int(rng, 1, 128), N, _log_int(rng, 1, N * (N - 1) // 2),
                       rng.choice(("sigmoid", "hinge", "square")))
        elif kind == "policy":
            c = {"kind": "policy", "B": _log_int(rng, 1, 256), "N": _log_int(rng, 1, 32), "name": "",
                 "reduce": rng.choice(("token", "sequence", "sum"))}
        elif kind == "rows":
            c = _rows("", _log_int(rng, 1, 256), _log_int(rng, 1, 1500),
                      rng.choice((29, 32, _log_int(rng, 24, 4096), _log_int(rng, 4096, 50021))), dtype,
                      ragged=rng.random() < 0.7, prompt=rng.choice((0.0, 0.25)),
                      reduce=rng.choice(("token", "sequence", "sum")))
            if DTYPES[dtype].itemsize * c["B"] * c["T"] * c["V"] > MOST_ROWS_BYTES:
                continue
        else:
            V = rng.choice((29, 32, 32, _log_int(rng, 24, 4096)))
            N = rng.choice((1, _log_int(rng, 1, 32)))
            c = _ctc("", kind, _log_int(rng, 1, 256), N, _log_int(rng, 20, 1500), V, dtype=dtype,
                     ragged=rng.random() < 0.5, p_blank=0.65 if V < 256 else 0.85)
            if kind == "train":
                c["N"] = max(2, N)
                c["M"] = rng.randint(1, 8)
            if c["B"] * c["N"] * c["T"] * (2 * _most_labels(c) + 1) > MOST_LATTICE:
                continue
            if c["B"] * c["T"] * V > 1 << 27:
                continue
        del c["name"]
        return c


def _most_labels(c):
    """Room for the tokens of a hypothesis."""
    return int((1.1 - c["p_blank"]) * c["T"]) + 4


def work(case):
    """Inputs read and outputs written once.  A lattice has two states for each token and one more; each takes three
    products and sums per frame and direction, and two for its share of the gradient.  Ragged batches at their mean."""
    c = case
    if c["kind"] == "preference":
        return {"bytes": c["B"] * (3.0 * 8 * c["N"] + 16.0 * c["M"]), "flops": 40.0 * c["B"] * c["M"]}
    if c["kind"] == "policy":
        return {"bytes": c["B"] * (40.0 * c["N"] + 4.0), "flops": 60.0 * c["B"] * c["N"]}
    share = 7.0 / 12.0 if c["ragged"] else 1.0
    size = DTYPES[c["dtype"]].itemsize
    frames = c["B"] * c["T"]
    if c["kind"] == "rows":
        part = share * (1.0 - c["prompt"])
        return {"bytes": size * c["V"] * frames * (1.0 + part) + 16.0 * frames, "flops": 8.0 * c["V"] * frames * part}
    labels = (1.0 - c["p_blank"]) * c["T"] * share
    needed = min(c["V"], 1.5 * labels + 1.0)
    grad = c["kind"] != "rescore"
    return {"bytes": size * (needed * frames * share + c["V"] * frames * grad) + 4.0 * c["B"] * c["N"] * labels,
            "flops": frames * share * c["N"] * (2.0 * labels + 1.0) * (8.0 if grad else 3.0)}


# ---- inputs ----------------------------------------------------------------------------------------------------------


def _uniform(gen, dev, shape, lo=0.0, hi=1.0):
    return lo + (hi - lo) * torch.rand(shape, generator=gen, device=dev, dtype=torch.float64)


def _lengths(gen, dev, c):
    if c["ragged"]:
        return torch.randint(max(1, c["T"] // 6), c["T"] + 1, (c["B"],), generator=gen, device=dev).to(torch.int32)
    return torch.full((c["B"],), c["T"], dtype=torch.int32, device=dev)


def _emissions(gen, dev, c):
    """Log-softmax rows [B,T,V] in the case's type, and each frame's strongest token [B,T]."""
    B, T, V = c["B"], c["T"], c["V"]
    x = torch.randn((B, T, V), generator=gen, device=dev, dtype=torch.float32)
    blank = _uniform(gen, dev, (B, T)) < c["p_blank"]
    primary = torch.where(blank, 0, torch.randint(1, V, (B, T), generator=gen, device=dev))
    x.scatter_add_(2, primary[..., None], _uniform(gen, dev, (B, T, 1), 6.0, 12.0).float())
    other = torch.randint(0, V, (B, T, 1), generator=gen, device=dev)
    second = torch.where(_uniform(gen, dev, (B, T, 1)) < 0.15, _uniform(gen, dev, (B, T, 1), 4.0, 8.0), 0.0)
    x.scatter_add_(2, other, second.float())
    return torch.log_softmax(x, 2).to(DTYPES[c["dtype"]]), primary


def _packed(tokens, keep, room):
    """The kept tokens of each row [..., n] moved to its front, and how many they are; `room` places."""
    at = torch.where(keep, keep.cumsum(-1) - 1, room).clamp_max(room)
    out = torch.zeros(tokens.shape[:-1] + (room + 1,), dtype=tokens.dtype, device=tokens.device)
    out.scatter_(-1, at, tokens)
    return out[..., :room], keep.sum(-1).clamp_max(room)


def _hypotheses(gen, dev, c, primary, lengths):
    """int32 [B,N,U] tokens and [B,N] lengths: the path's own tokens, in all but the first of each list 5% replaced and
    3% left out."""
    B, N, V, U = c["B"], c["N"], c["V"], _most_labels(c)
    frame = torch.arange(c["T"], device=dev)
    before = torch.nn.functional.pad(primary[:, :-1], (1, 0))
    tokens, count = _packed(primary, (primary != 0) & (primary != before) & (frame < lengths[:, None]), U)
    tokens = tokens[:, None].expand(B, N, U)
    later = (torch.arange(N, device=dev) > 0)[:, None]
    replaced = later & (_uniform(gen, dev, (B, N, U)) < 0.05)
    tokens = torch.where(replaced, torch.randint(1, V, (B, N, U), generator=gen, device=dev), tokens)
    keep = torch.arange(U, device=dev) < count[:, None, None]
    keep = keep & ~(later & (_uniform(gen, dev, (B, N, U)) < 0.03))
    tokens, count = _packed(tokens, keep, U)
    return tokens.to(torch.int32).contiguous(), count.to(torch.int32)


def _log_ratios(gen, dev, shape, spread):
    """Log ratios that stay a thousandth off the borders where the loss is clipped, so that 32 bits decide alike."""
    x = spread * torch.randn(shape, generator=gen, device=dev, dtype=torch.float64)
    for border in (math.log(1.0 - CLIP_LOW), math.log(1.0 + CLIP_HIGH)):
        x = torch.where((x - border).abs() < 1e-3, x + 2e-3, x)
    return x


def _some_pairs(gen, dev, B, N, M):
    """int32 [B,M,2]: M of the N(N-1)/2 pairs of each list, the better one first by a random order of the list."""
    i, j = torch.triu_indices(N, N, 1, device=dev)
    pick = _uniform(gen, dev, (B, i.numel())).argsort(1)[:, torch.arange(M, device=dev) % i.numel()]
    order = _uniform(gen, dev, (B, N)).argsort(1)
    return torch.stack((order.gather(1, i[pick]), order.gather(1, j[pick])), 2).to(torch.int32)


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    c = case
    s = {"case": c, "scale": LOSS_SCALE.get(c.get("dtype"), 1.0)}
    if c["kind"] == "preference":
        s["scores"] = -_uniform(gen, dev, (c["B"], c["N"]), 20.0, 400.0)
        s["ref_scores"] = s["scores"] + 4.0 * torch.randn((c["B"], c["N"]), generator=gen, device=dev,
                                                          dtype=torch.float64)
        s["pairs"] = _some_pairs(gen, dev, c["B"], c["N"], c["M"])
    elif c["kind"] == "policy":
        shape = (c["B"], c["N"])
        s["scores"] = -_uniform(gen, dev, shape, 20.0, 400.0)
        s["old"] = s["scores"] - _log_ratios(gen, dev, shape, 0.2)
        s["ref"] = s["scores"] + 0.3 * torch.randn(shape, generator=gen, device=dev, dtype=torch.float64)
        s["advantages"] = torch.randn(shape, generator=gen, device=dev, dtype=torch.float64)
        s["counts"] = torch.randint(1, c["N"] + 1, (c["B"],), generator=gen, device=dev).to(torch.int32)
    elif c["kind"] == "rows":
        B, T, V = c["B"], c["T"], c["V"]
        x = torch.randn((B, T, V), generator=gen, device=dev, dtype=torch.float32).mul_(2.0)
        tokens = torch.randint(0, V, (B, T), generator=gen, device=dev)
        x.scatter_add_(2, tokens[..., None], _uniform(gen, dev, (B, T, 1), 0.0, 12.0).float())
        s["logits"] = x.to(DTYPES[c["dtype"]])
        del x
        lp = torch.empty((B, T), dtype=torch.float64, device=dev)
        for b in range(B):  # one sequence at a time: 64 bits of all would be large
            lp[b] = torch.log_softmax(s["logits"][b].double(), 1).gather(1, tokens[b, :, None])[:, 0]
        s["lengths"] = _lengths(gen, dev, c)
        s["old"] = (lp - _log_ratios(gen, dev, (B, T), 0.15)).float()
        s["ref"] = (lp + 0.2 * torch.randn((B, T), generator=gen, device=dev, dtype=torch.float64)).float()
        s["advantages"] = torch.randn((B,), generator=gen, device=dev, dtype=torch.float32)
        prompt = torch.arange(T, device=dev) < torch.floor(c["prompt"] * s["lengths"])[:, None]
        s["tokens"] = torch.where(prompt, -1, tokens).to(torch.int32)
    else:
        s["logprobs"], primary = _emissions(gen, dev, c)
        s["lengths"] = _lengths(gen, dev, c)
        s["tokens"], s["token_lengths"] = _hypotheses(gen, dev, c, primary, s["lengths"])
        if c["kind"] == "ctc":
            s["weights"] = -_uniform(gen, dev, (c["B"], c["N"]), 0.5, 1.5) * (s["scale"] / (c["B"] * c["N"]))
        elif c["kind"] == "train":
            s["ref_scores"] = -_uniform(gen, dev, (c["B"], c["N"]), 60.0, 90.0)
            s["pairs"] = _some_pairs(gen, dev, c["B"], c["N"], c["M"])
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------


def _log_sum(*terms):
    top = terms[0]
    for x in terms[1:]:
        top = torch.maximum(top, x)
    top = top.clamp_min(-1e300)
    total = torch.exp(terms[0] - top)
    for x in terms[1:]:
        total = total + torch.exp(x - top)
    return top + torch.log(total)


def _plain_lattice(s, weights):
    """Scores [B,N]; where `weights` is a function of them, also the gradient of sum(weights * scores) [B,T,V].  Sums over
    hundreds of frames: 64 bits."""
    lp, lengths, tokens, count = s["logprobs"], s["lengths"].long(), s["tokens"].long(), s["token_lengths"].long()
    (B, T, V), (N, U) = lp.shape, tokens.shape[1:]
    S = 2 * U + 1
    z = torch.zeros((B, N, S), dtype=torch.long, device=lp.device)
    z[:, :, 1::2] = tokens
    place = torch.arange(S, device=lp.device)
    minus = torch.full((B, N, S), -math.inf, dtype=torch.float64, device=lp.device)
    skip = torch.where((z != 0) & (z != torch.roll(z, 2, 2)) & (place > 1), 0.0, minus)
    states = 2 * count[..., None] + 1
    p = lambda t: torch.gather(lp[:, t].double(), 1, z.view(B, N * S)).view(B, N, S)  # noqa: E731

    def shifted(x, by):
        y = torch.roll(x, by, 2)
        y[:, :, :by] = -math.inf if by > 0 else y[:, :, :by]
        if by < 0:
            y[:, :, by:] = -math.inf
        return y

    first = torch.where((place < 2) & (place < states), 0.0, minus)
    last = torch.where((place < states) & (place >= states - 2), 0.0, minus)
    alphas, a = [], None
    end = torch.where(place == 0, 0.0, minus)
    for t in range(T):
        a_new = (first if a is None else _log_sum(a, shifted(a, 1), shifted(a, 2) + skip)) + p(t)
        inside = (t < lengths)[:, None, None]
        end = torch.where(inside, a_new, end)
        a = a_new
        if weights is not None:
            alphas.append(a)
    total = end + last
    top = total.amax(2, keepdim=True).clamp_min(-1e300)
    scores = (top + torch.log(torch.exp(total - top).sum(2, keepdim=True)))[..., 0]
    if weights is None:
        return scores, None
    weights = weights(scores)
    scale = torch.where(torch.isfinite(scores), weights, 0.0)[..., None]
    per = torch.where(torch.isfinite(scores), scores, 0.0)[..., None]
    grad = torch.zeros((B, T, V), dtype=torch.float64, device=lp.device)
    flat = z.view(B, N * S)
    skip_on = shifted(skip, -2)
    b = minus
    for t in range(T - 1, -1, -1):
        at_end = (t == lengths - 1)[:, None, None]
        if t < T - 1:
            up = b + p(t + 1)
            b = _log_sum(up, shifted(up, -1), shifted(up, -2) + skip_on)
        b = torch.where(at_end, last, b)
        gamma = torch.exp(alphas[t] + b - per) * scale * (t < lengths)[:, None, None]
        grad[:, t].scatter_add_(1, flat, gamma.view(B, N * S))
    return scores, grad.to(lp.dtype)


def _plain_preference(scores, ref_scores, pairs, loss, scale):
    won, lost = pairs[..., 0].long(), pairs[..., 1].long()
    ratio = scores - ref_scores
    h = ratio.gather(1, won) - ratio.gather(1, lost)
    n = h.numel()
    step = scale / n
    if loss == "sigmoid":
        soft = lambda x: torch.clamp_min(x, 0.0) + torch.log1p(torch.exp(-x.abs()))  # noqa: E731
        f = (1.0 - SMOOTHING) * soft(-BETA * h) + SMOOTHING * soft(BETA * h)
        d = BETA * (1.0 / (1.0 + torch.exp(-BETA * h)) - (1.0 - SMOOTHING))
    elif loss == "hinge":
        f = torch.clamp_min(1.0 - BETA * h, 0.0)
        d = torch.where(BETA * h < 1.0, torch.full_like(h, -BETA), 0.0)
    else:
        f = (h - 0.5 / BETA) ** 2
        d = 2.0 * (h - 0.5 / BETA)
    grad = torch.zeros_like(scores)
    grad.scatter_add_(1, won, d * step)
    grad.scatter_add_(1, lost, -d * step)
    return f.sum() / n, h, grad


def _plain_policy(lp, old, ref, advantages, part, reduce):
    """Loss, KL, share of clipped places, and the loss's derivative to each log-probability."""
    n = part.sum(1, keepdim=True).to(lp.dtype)
    if reduce == "token":
        weight = part / n.sum().clamp_min(1.0)
    elif reduce == "sequence":
        weight = part / (n.clamp_min(1.0) * (n > 0).sum().clamp_min(1))
    else:
        weight = part.to(lp.dtype)
    zero = torch.zeros_like(lp)
    r = torch.exp(torch.where(part, lp - old, zero))
    plain, cut = r * advantages, r.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * advantages
    gap = torch.where(part, ref - lp, zero)
    kl = torch.exp(gap) - gap - 1.0
    f = torch.maximum(-plain, -cut) + KL_WEIGHT * kl
    d = torch.where(plain <= cut, -plain, 0.0) + KL_WEIGHT * (1.0 - torch.exp(gap))
    clipped = (part & (plain > cut)).sum() / n.sum().clamp_min(1.0)
    return (f * weight).sum(), (kl * weight).sum(), clipped, d * weight


def _plain_rows(s):
    x = s["logits"].float()
    tokens = s["tokens"].long()
    part = (torch.arange(x.shape[1], device=x.device) < s["lengths"][:, None]) & (tokens >= 0)
    at = tokens.clamp_min(0)[..., None]
    top = x.amax(2, keepdim=True)
    total = torch.exp(x - top).sum(2, keepdim=True)
    lp = torch.where(part, (x.gather(2, at) - top - torch.log(total))[..., 0], 0.0)
    loss, kl, clipped, d = _plain_policy(lp, s["old"], s["ref"], s["advantages"][:, None], part, s["case"]["reduce"])
    d = d * s["scale"]
    grad = torch.exp(x - top) / total * -d[..., None]
    grad.scatter_add_(2, at, d[..., None])
    return {"loss": loss, "kl": kl, "clipped": clipped, "logps": lp, "grad_logits": grad.to(s["logits"].dtype)}


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "rescore":
        return {"scores": _plain_lattice(s, None)[0]}
    if c["kind"] == "ctc":
        scores, grad = _plain_lattice(s, lambda _: s["weights"])
        return {"scores": scores, "grad_logprobs": grad}
    if c["kind"] == "train":
        told = {}

        def weights(scores):
            told["loss"], told["margins"], grad_scores = _plain_preference(scores, s["ref_scores"], s["pairs"], "sigmoid",
                                                                             s["scale"])
            return grad_scores

        scores, grad = _plain_lattice(s, weights)
        return {"scores": scores, "grad_logprobs": grad, **told}
    if c["kind"] == "preference":
        loss, h, grad = _plain_preference(s["scores"], s["ref_scores"], s["pairs"], c["loss"], s["scale"])
        return {"loss": loss, "margins": h, "grad_scores": grad}
    if c["kind"] == "policy":
        part = torch.arange(c["N"], device=s["scores"].device) < s["counts"][:, None]
        loss, kl, clipped, grad = _plain_policy(s["scores"], s["old"], s["ref"], s["advantages"], part, c["reduce"])
        return {"loss": loss, "kl": kl, "clipped": clipped, "grad_scores": grad}
    return _plain_rows(s)


# ---- the framework's calls -------------------------------------------------------------------------------------------


def _run_own(s):
    from paper_2510_09085_amd import binding

    c = s["case"]
    if c["kind"] in ("ctc", "rescore", "train"):
        lattice = (s["logprobs"], s["lengths"], s["tokens"], s["token_lengths"])
        if c["kind"] == "rescore":
            return {"scores": binding.ctc_score(*lattice)["scores"]}
        out = binding.ctc_score(*lattice, want_grad=True)
        if c["kind"] == "ctc":
            told, grad_scores = {}, s["weights"]
        else:
            told = binding.preference_loss(out["scores"], s["pairs"], ref_scores=s["ref_scores"], beta=BETA,
                                           label_smoothing=SMOOTHING, scale=s["scale"])
            grad_scores = told["grad_scores"]
            told = {"loss": told["loss"], "margins": told["margins"]}
        grad = binding.ctc_score_grad(*lattice, grad_scores, out["workspace"])
        return {"scores": out["scores"], "grad_logprobs": grad, **told}
    if c["kind"] == "preference":
        out = binding.preference_loss(s["scores"], s["pairs"], ref_scores=s["ref_scores"], kind=c["loss"], beta=BETA,
                                      label_smoothing=SMOOTHING if c["loss"] == "sigmoid" else 0.0)
        return {k: out[k] for k in ("loss", "margins", "grad_scores")}
    settings = {"clip_low": CLIP_LOW, "clip_high": CLIP_HIGH, "kl_weight": KL_WEIGHT, "reduction": c["reduce"]}
    if c["kind"] == "policy":
        out = binding.policy_loss(s["scores"], s["old"], s["advantages"], ref_scores=s["ref"], counts=s["counts"],
                                  **settings)
        return {k: out[k] for k in ("loss", "kl", "clipped", "grad_scores")}
    out = binding.policy_loss_logits(s["logits"], s["tokens"], s["lengths"], s["old"], s["advantages"],
                                     ref_logps=s["ref"], scale=s["scale"], **settings)
    return {k: out[k] for k in ("loss", "kl", "clipped", "logps", "grad_logits")}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- from the definitions, in 64 bits: values by sums, gradients by differentiating them -----------------------------


def _exact_scores(s, lp):
    """A path either stays, steps or skips: probabilities of being at each state, rescaled to sum to one in each frame
    so that they stay in range, with the logarithms of the scales added up."""
    tokens, count, lengths = s["tokens"].long(), s["token_lengths"].long(), s["lengths"].long()
    B, N, U = tokens.shape
    p_frames = torch.exp(lp).unbind(1)
    label = torch.arange(U, device=lp.device)
    fresh = torch.ones((B, N, U), dtype=torch.float64, device=lp.device)
    fresh[:, :, 1:] = (tokens[:, :, 1:] != tokens[:, :, :-1]).double()
    used = (label < count[..., None]).double()
    blanks = torch.zeros((B, N, U + 1), dtype=torch.float64, device=lp.device)
    blanks[:, :, 0] = 1.0  # before the first frame: at the first blank, with nothing emitted
    labels = torch.zeros((B, N, U), dtype=torch.float64, device=lp.device)
    logs = torch.zeros((B, N, 1), dtype=torch.float64, device=lp.device)
    pad = torch.nn.functional.pad
    for t in range(int(lengths.max())):
        p = p_frames[t]
        p_label = p.gather(1, tokens.reshape(B, N * U)).view(B, N, U) * used
        came = pad(labels, (1, 0))[:, :, :U]
        b = (blanks + pad(labels, (1, 0))) * p[:, None, :1]
        l = (labels + blanks[:, :, :U] + fresh * came) * p_label
        scale = b.sum(2, keepdim=True) + l.sum(2, keepdim=True)
        live = (t < lengths)[:, None, None]
        blanks = torch.where(live, b / scale, blanks)
        labels = torch.where(live, l / scale, labels)
        logs = torch.where(live, logs + torch.log(scale), logs)
    ends = blanks.gather(2, count[..., None]) + torch.where(
        count[..., None] > 0, labels.gather(2, (count[..., None] - 1).clamp_min(0)), 0.0)
    return (logs + torch.log(ends))[..., 0]


def _exact_pairs(scores, ref, pairs, loss):
    i, j = pairs.long().unbind(2)
    h = (scores.gather(1, i) - scores.gather(1, j)) - (ref.gather(1, i) - ref.gather(1, j))
    sig = torch.nn.functional.logsigmoid
    f = {"sigmoid": lambda: -(1.0 - SMOOTHING) * sig(BETA * h) - SMOOTHING * sig(-BETA * h),
         "hinge": lambda: torch.relu(1.0 - BETA * h), "square": lambda: (h - 1.0 / (2.0 * BETA)).square()}[loss]()
    return f.mean(), h


def _exact_policy(lp, old, ref, advantages, part, reduce):
    r = torch.exp(lp - old)
    worst = torch.minimum(r * advantages, torch.clamp(r, 1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * advantages)
    kl = torch.expm1(ref - lp) - (ref - lp)
    out = []
    for x in (KL_WEIGHT * kl - worst, kl, (worst < r * advantages).double()):
        x = torch.where(part, x, 0.0)
        if reduce == "token" or len(out) == 2:
            out.append(x.sum() / part.sum())
        elif reduce == "sequence":
            some = part.any(1)
            out.append((x.sum(1)[some] / part.sum(1)[some]).mean())
        else:
            out.append(x.sum())
    return out


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["kind"] == "preference":
        x = s["scores"].clone().requires_grad_()
        loss, h = _exact_pairs(x, s["ref_scores"], s["pairs"], c["loss"])
        return {"loss": loss.detach(), "margins": h.detach(), "grad_scores": torch.autograd.grad(loss, x)[0]}
    if c["kind"] == "policy":
        x = s["scores"].clone().requires_grad_()
        part = torch.arange(c["N"], device=x.device) < s["counts"][:, None]
        loss, kl, clipped = _exact_policy(x, s["old"], s["ref"], s["advantages"], part, c["reduce"])
        return {"loss": loss.detach(), "kl": kl.detach(), "clipped": clipped.detach(),
                "grad_scores": torch.autograd.grad(loss, x)[0]}
    if c["kind"] == "rows":
        x = s["logits"].double().requires_grad_()
        tokens = s["tokens"].long()
        part = (torch.arange(c["T"], device=x.device) < s["lengths"][:, None]) & (tokens >= 0)
        lp = torch.log_softmax(x, 2).gather(2, tokens.clamp_min(0)[..., None])[..., 0]
        lp = torch.where(part, lp, 0.0)
        loss, kl, clipped = _exact_policy(lp, s["old"].double(), s["ref"].double(), s["advantages"].double()[:, None],
                                          part, c["reduce"])
        return {"loss": loss.detach(), "kl": kl.detach(), "clipped": clipped.detach(), "logps": lp.detach(),
                "grad_logits": torch.autograd.grad(loss * s["scale"], x)[0]}
    if c["kind"] == "rescore":
        with torch.no_grad():
            return {"scores": _exact_scores(s, s["logprobs"].double())}
    x = s["logprobs"].double().requires_grad_()
    scores = _exact_scores(s, x)
    told = {}
    if c["kind"] == "train":
        value, h = _exact_pairs(scores, s["ref_scores"], s["pairs"], "sigmoid")
        told = {"loss": value.detach(), "margins": h.detach()}
        value = value * s["scale"]
    else:
        value = (s["weights"] * scores).sum()
    return {"scores": scores.detach(), "grad_logprobs": torch.autograd.grad(value, x)[0], **told}
