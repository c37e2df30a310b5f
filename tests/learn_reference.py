"""Plain 64-bit (and, for the lattice, 80-bit) forms of the operators that learn from hypotheses.

The lattice is summed in linear domain with numpy's long doubles, whose exponents reach e^-11000, each frame relative
to its likeliest state: no logarithms on the way, no rounding that matters beside fp64.  Nothing here is shared with the
kernels."""
import itertools
import math

import numpy as np
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# half a step of the type: the largest relative error of one rounding
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SMALLEST = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


def states_of(tokens):
    z = [0]
    for t in tokens:
        z += [int(t), 0]
    return z


def lattice(lp, tokens):
    """(ln P, occupancies [T, states]) as long doubles of one hypothesis under lp [T, V] (already cut to its frames).  Each
    frame is taken relative to its likeliest state, which keeps long products in range."""
    z = states_of(tokens)
    T, S = lp.shape[0], len(z)
    if T == 0:
        return (0.0 if S == 1 else -np.inf), np.zeros((0, S), np.longdouble)
    e = lp.astype(np.longdouble)[:, z]
    top = e.max(1, keepdims=True)
    top = np.where(np.isfinite(top), top, 0)
    em = np.exp(e - top)
    enter = [s for s in range(S)]
    skip = np.array([s > 1 and z[s] != 0 and z[s] != z[s - 2] for s in enter])
    a = np.zeros((T, S), np.longdouble)
    a[0, :2] = em[0, :2]
    for t in range(1, T):
        x = a[t - 1].copy()
        x[1:] += a[t - 1, :-1]
        x[2:] += np.where(skip[2:], a[t - 1, :-2], 0)
        a[t] = x * em[t]
    b = np.zeros((T, S), np.longdouble)
    b[T - 1, S - 1] = 1
    if S > 1:
        b[T - 1, S - 2] = 1
    for t in range(T - 2, -1, -1):
        y = b[t + 1] * em[t + 1]
        x = y.copy()
        x[:-1] += y[1:]
        x[:-2] += np.where(skip[2:], y[2:], 0)
        b[t] = x
    total = a[T - 1, S - 1] + (a[T - 1, S - 2] if S > 1 else 0)
    if total <= 0:
        return -np.inf, np.zeros_like(a)
    return np.log(total) + top.sum(), a * b / total


def possible(tokens, V):
    return all(1 <= int(t) < V for t in tokens)


def scores_and_grad(lp, lengths, tokens, token_lengths, weights, counts=None):
    """Scores [B,N], gradient [B,T,V], the sum of |weight| * occupancy [B,T,V] (what roundings are relative to) and the
    largest |weight| times states [B] (what they are absolute to)."""
    B, T, V = lp.shape
    N, U = tokens.shape[1:]
    scores = np.full((B, N), -np.inf)
    grad = np.zeros((B, T, V), np.longdouble)
    size = np.zeros((B, T, V), np.longdouble)
    quanta = np.zeros(B)
    for b in range(B):
        frames = min(max(int(lengths[b]), 0), T)
        states = 0
        most = 0.0
        for n in range(N if counts is None else min(max(int(counts[b]), 0), N)):
            L = int(token_lengths[b, n])
            if L > U:
                scores[b, n] = np.nan
                continue
            if L < 0 or not possible(tokens[b, n, :L], V):
                continue
            total, share = lattice(lp[b, :frames], tokens[b, n, :L])
            if total == -np.inf:
                continue
            scores[b, n] = float(total)
            states += 2 * L + 1
            most = max(most, abs(float(weights[b, n])))
            for s, v in enumerate(states_of(tokens[b, n, :L])):
                grad[b, :frames, v] += weights[b, n] * share[:, s]
                size[b, :frames, v] += abs(weights[b, n]) * share[:, s]
        quanta[b] = most * states
    return scores, grad.astype(np.float64), size.astype(np.float64), quanta


def enumerated(lp, tokens):
    """(P, occupancies [T, V]) by going through all V^T alignments."""
    T, V = lp.shape
    total, share = 0.0, np.zeros((T, V))
    for path in itertools.product(range(V), repeat=T):
        said = [v for i, v in enumerate(path) if v != 0 and (i == 0 or path[i - 1] != v)]
        if said == list(tokens):
            p = math.exp(sum(float(lp[t, v]) for t, v in enumerate(path)))
            total += p
            for t, v in enumerate(path):
                share[t, v] += p
    return total, (share / total if total > 0 else share)


def score_tolerance(T, score):
    """Relative roundings of a frame (three sums, a product, the series of exp, whose ln2 split and Horner steps
    round four times at most in effect): 8 * 2^-53; the logarithm and the exponent's product once each."""
    return 8 * T * 2.0 ** -53 + 2.0 ** -51 * abs(score)


def grad_tolerance(dtype, T, grad, size, quanta):
    """Of an occupancy: both kept masses, the share and its place in the gradient rounded to fp32 (four half steps, and
    as much as one for their products and the fp64 sums), whole multiples of 2^-50 of the largest weight (half of one
    for each state), and the rounding to the gradient's own type."""
    near = 5 * 2.0 ** -24 * size + 2.0 ** -51 * quanta[:, None, None] + 1e-30
    return near + (HALF_STEP[dtype] * (np.abs(grad) + near) + SMALLEST[dtype] if dtype != "f32" else 0.0)


# ---- losses ------------------------------------------------------------------------------------------------------------


def softplus(x):
    return np.logaddexp(0.0, x)


def preference(scores, pairs, ref=None, pair_counts=None, kind="sigmoid", beta=0.1, eps=0.0, scale=1.0):
    B, N = scores.shape
    M = pairs.shape[1]
    margins = np.full((B, M), np.nan)
    slope = np.zeros((B, M))
    total, used = 0.0, 0
    for b in range(B):
        for m in range(M if pair_counts is None else min(max(int(pair_counts[b]), 0), M)):
            i, j = (int(v) for v in pairs[b, m])
            if not (0 <= i < N and 0 <= j < N):
                continue
            numbers = [scores[b, i], scores[b, j]] + ([] if ref is None else [ref[b, i], ref[b, j]])
            if not np.all(np.isfinite(numbers)):
                continue
            h = scores[b, i] - scores[b, j] - (0.0 if ref is None else ref[b, i] - ref[b, j])
            margins[b, m] = h
            used += 1
            if kind == "sigmoid":
                total += (1 - eps) * softplus(-beta * h) + eps * softplus(beta * h)
                slope[b, m] = -(1 - eps) * beta / (1 + np.exp(beta * h)) + eps * beta / (1 + np.exp(-beta * h))
            elif kind == "hinge":
                total += max(0.0, 1 - beta * h)
                slope[b, m] = -beta if beta * h < 1 else 0.0
            else:
                total += (h - 1 / (2 * beta)) ** 2
                slope[b, m] = 2 * (h - 1 / (2 * beta))
    grad = np.zeros((B, N))
    for b in range(B):
        for m in range(M):
            if np.isfinite(margins[b, m]):
                grad[b, pairs[b, m, 0]] += slope[b, m] * scale / used
                grad[b, pairs[b, m, 1]] -= slope[b, m] * scale / used
    return total / max(used, 1), margins, grad, used


def policy(l, old, advantages, part, ref=None, lo=0.2, hi=0.2, kl_weight=0.0, reduction="token", scale=1.0):
    """Loss, KL, clipped share, derivative to l (all fp64; `part` says what takes part)."""
    with np.errstate(all="ignore"):
        r = np.exp(l - old)
        plain, cut = r * advantages, np.clip(r, 1 - lo, 1 + hi) * advantages
        gap = np.zeros_like(l) if ref is None else ref - l
        kl = np.expm1(gap) - gap
        f = np.maximum(-plain, -cut) + kl_weight * kl
        d = np.where(plain <= cut, -plain, 0.0) - kl_weight * np.expm1(gap)
    n = part.sum(1, keepdims=True)
    some = max(int((n > 0).sum()), 1)
    weight = {"token": part / max(int(n.sum()), 1), "sequence": part / (np.maximum(n, 1) * some),
              "sum": part.astype(np.float64)}[reduction]
    pick = lambda x: np.where(part, x, 0.0)  # noqa: E731
    return ((pick(f) * weight).sum(), (pick(kl) * weight).sum(), pick(plain > cut).sum() / max(int(n.sum()), 1),
            pick(d) * weight * scale)
