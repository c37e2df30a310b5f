"""Refusals of the operators that learn from hypotheses: every bad call fails in the host's checks, before anything is
enqueued (no GPU needed), and the binding's structures have the C compiler's layout."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2510_09085_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 256 * 4096  # an address that no refused call may touch
OK, NULL, SHAPE, BEAM, SPACE, VOCAB, ALIGN, OPTION = 0, -1, -2, -3, -5, -6, -8, -9


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2510_09085_amd import build
        build.build()
    return binding.load()


def rows(**change):
    x = binding.FltopRows(FAKE, FAKE, 10 * 32, 32, 2, 10, 32, 0)
    for k, v in change.items():
        setattr(x, k, v)
    return x


def hyps(**change):
    h = binding.FltopHypotheses(FAKE, FAKE, None, 3 * 8, 8, 3, 3, 8)
    for k, v in change.items():
        setattr(h, k, v)
    return h


BAD_ROWS = [({"data": None}, NULL), ({"lengths": None}, NULL), ({"B": 0}, SHAPE), ({"T": 0}, SHAPE), ({"V": 1}, SHAPE),
            ({"B": 70000, "T": 70000}, SHAPE), ({"batch_stride": -1}, SHAPE), ({"frame_stride": -32}, SHAPE),
            ({"V": binding.MAX_VOCAB + 1}, VOCAB), ({"type": 3}, OPTION), ({"type": -1}, OPTION)]
BAD_HYPS = [({"tokens": None}, NULL), ({"lengths": None}, NULL), ({"N": 0}, SHAPE), ({"U": 0}, SHAPE),
            ({"U": binding.MAX_LABELS + 1}, SHAPE), ({"token_stride": -8}, SHAPE), ({"token_batch_stride": -1}, SHAPE),
            ({"length_batch_stride": -1}, SHAPE), ({"N": binding.MAX_BEAM + 1}, BEAM)]


def test_score_refusals(lib):
    need = lib.fltop_ctc_score_workspace_bytes(2, 10, 3, 8)

    def score(x=None, h=None, out=FAKE, ws=FAKE, n=need):
        return lib.fltop_ctc_score(ctypes.byref(x or rows()), ctypes.byref(h or hyps()), out, ws, n, None)

    def grad(x=None, h=None, g=FAKE, ws=FAKE, n=need, out=FAKE):
        return lib.fltop_ctc_score_grad(ctypes.byref(x or rows()), ctypes.byref(h or hyps()), g, ws, n, out, None)

    for call in (score, grad):
        for change, code in BAD_ROWS:
            assert call(x=rows(**change)) == code, change
        for change, code in BAD_HYPS:
            assert call(h=hyps(**change)) == code, change
        assert call(out=None) == NULL
        assert call(n=need - 1) == SPACE
        assert call(ws=FAKE + 8) == ALIGN
    assert grad(g=None) == NULL
    assert grad(ws=None) == NULL
    assert lib.fltop_ctc_score(None, ctypes.byref(hyps()), FAKE, None, 0, None) == NULL
    assert lib.fltop_ctc_score(ctypes.byref(rows()), None, FAKE, None, 0, None) == NULL


def test_workspace_sizes(lib):
    assert lib.fltop_ctc_score_workspace_bytes(2, 10, 3, 8) % 256 == 0
    for bad in ((0, 10, 3, 8), (2, 0, 3, 8), (2, 10, 0, 8), (2, 10, 3, 0), (2, 10, 3, binding.MAX_LABELS + 1),
                (1 << 30, 10, 1024, 8), (2, 10, binding.MAX_BEAM + 1, 8)):
        assert lib.fltop_ctc_score_workspace_bytes(*bad) == 0
    # beyond 32 bits
    assert lib.fltop_ctc_score_workspace_bytes(256, 1500, 8, 700) > 2 ** 32
    assert lib.fltop_preference_workspace_bytes(0) == 0 and lib.fltop_preference_workspace_bytes(3) % 256 == 0
    assert lib.fltop_policy_workspace_bytes(0, 4) == 0 and lib.fltop_policy_workspace_bytes(4, 0) == 0
    assert lib.fltop_policy_workspace_bytes(70000, 70000) == 0
    assert lib.fltop_policy_workspace_bytes(3, 7) % 256 == 0


def test_preference_refusals(lib):
    need = lib.fltop_preference_workspace_bytes(2)

    def call(ws=FAKE, n=need, **change):
        p = binding.FltopPreference(FAKE, FAKE, FAKE, None, 2, 4, 6, 0, 0.1, 0.1, 1.0, FAKE, FAKE, FAKE)
        for k, v in change.items():
            setattr(p, k, v)
        return lib.fltop_preference_loss(ctypes.byref(p), ws, n, None)

    for name in ("scores", "pairs", "loss", "margins", "grad_scores"):
        assert call(**{name: None}) == NULL
    for name in ("B", "N", "M"):
        assert call(**{name: 0}) == SHAPE
    assert call(M=1 << 30) == SHAPE
    assert call(N=binding.MAX_BEAM + 1) == BEAM
    for change in ({"kind": 3}, {"kind": -1}, {"beta": 0.0}, {"beta": -1.0}, {"beta": float("nan")},
                   {"beta": float("inf")}, {"label_smoothing": -0.1}, {"label_smoothing": 0.6},
                   {"label_smoothing": float("nan")}, {"kind": 1, "label_smoothing": 0.1}, {"scale": float("inf")}):
        assert call(**change) == OPTION, change
    assert call(n=need - 1) == SPACE
    assert call(ws=FAKE + 16) == ALIGN
    assert call(ws=None) == NULL
    assert lib.fltop_preference_loss(None, FAKE, need, None) == NULL


BAD_POLICY = [{"reduction": 3}, {"reduction": -1}, {"clip_low": -0.1}, {"clip_low": 1.1}, {"clip_low": float("nan")},
              {"clip_high": -0.1}, {"clip_high": float("inf")}, {"kl_weight": float("nan")}, {"scale": float("inf")}]


def settings(**change):
    p = binding.FltopPolicy(0, 0, 0.2, 0.2, 0.1, 1.0)
    for k, v in change.items():
        setattr(p, k, v)
    return p


def test_policy_refusals(lib):
    need = lib.fltop_policy_workspace_bytes(2, 1)
    good = dict(scores=FAKE, old=FAKE, ref=None, adv=FAKE, counts=None, B=2, N=4, policy=settings(), ws=FAKE, n=need,
                summary=FAKE, grad=FAKE)

    def call(**change):
        a = {**good, **change}
        return lib.fltop_policy_loss(a["scores"], a["old"], a["ref"], a["adv"], a["counts"], a["B"], a["N"],
                                     ctypes.byref(a["policy"]) if a["policy"] else None, a["ws"], a["n"], a["summary"],
                                     a["grad"], None)

    for name in ("scores", "old", "adv", "policy", "ws", "summary", "grad"):
        assert call(**{name: None}) == NULL, name
    assert call(B=0) == SHAPE and call(N=0) == SHAPE
    assert call(n=need - 1) == SPACE and call(ws=FAKE + 4) == ALIGN
    for change in BAD_POLICY:
        assert call(policy=settings(**change)) == OPTION, change


def test_policy_logits_refusals(lib):
    need = lib.fltop_policy_workspace_bytes(2, 10)
    good = dict(x=rows(), tokens=FAKE, old=FAKE, ref=None, adv=FAKE, policy=settings(), ws=FAKE, n=need, summary=FAKE,
                logps=FAKE, grad=FAKE)

    def call(**change):
        a = {**good, **change}
        return lib.fltop_policy_loss_logits(ctypes.byref(a["x"]), a["tokens"], a["old"], a["ref"], a["adv"], 0,
                                            ctypes.byref(a["policy"]) if a["policy"] else None, a["ws"], a["n"],
                                            a["summary"], a["logps"], a["grad"], None)

    for name in ("tokens", "old", "adv", "policy", "ws", "summary", "logps", "grad"):
        assert call(**{name: None}) == NULL, name
    for change, code in BAD_ROWS:
        if change not in ({"V": 1}, {"V": binding.MAX_VOCAB + 1}):  # any vocabulary here
            assert call(x=rows(**change)) == code, change
    assert call(x=rows(V=0)) == SHAPE
    assert call(n=need - 1) == SPACE and call(ws=FAKE + 4) == ALIGN
    for change in BAD_POLICY:
        assert call(policy=settings(**change)) == OPTION, change


def test_binding_refuses_host_tensors():
    lp = torch.zeros((1, 4, 8))
    ln = torch.zeros(1, dtype=torch.int32)
    tok = torch.zeros((1, 1, 2), dtype=torch.int32)
    one = torch.zeros((1, 1), dtype=torch.int32)
    score = torch.zeros((1, 2), dtype=torch.float64)
    calls = [lambda: binding.ctc_score(lp, ln, tok, one),
             lambda: binding.ctc_score_grad(lp, ln, tok, one, score[:, :1], torch.zeros(4096, dtype=torch.uint8)),
             lambda: binding.preference_loss(score, tok),
             lambda: binding.policy_loss(score, score, score),
             lambda: binding.policy_loss_logits(lp, torch.zeros((1, 4), dtype=torch.int32), ln, lp[..., 0], lp[:, 0, 0])]
    for call in calls:
        with pytest.raises(ValueError):
            call()


def test_structures_have_the_compilers_layout(tmp_path):
    pairs = [("fltop_rows", binding.FltopRows), ("fltop_hypotheses", binding.FltopHypotheses),
             ("fltop_preference", binding.FltopPreference), ("fltop_policy", binding.FltopPolicy)]
    prog = ['#include <stddef.h>', '#include <stdio.h>', '#include "fltop_ctc.h"', 'int main(void) {']
    for name, mirror in pairs:
        prog.append(f'  printf("{name} %zu\\n", sizeof({name}));')
        prog += [f'  printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in mirror._fields_]
    prog += ['  return 0;', '}']
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(prog) + "\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"),
                    str(src), "-o", str(exe)], check=True)
    said = dict(line.split() for line in subprocess.run([str(exe)], capture_output=True, text=True,
                                                        check=True).stdout.splitlines())
    for name, mirror in pairs:
        assert int(said[name]) == ctypes.sizeof(mirror)
        for f, _ in mirror._fields_:
            assert int(said[f"{name}.{f}"]) == getattr(mirror, f).offset, f


def test_constants_match_the_header():
    import re
    text = open(os.path.join(ROOT, "include", "fltop_ctc.h")).read()
    said = {k: int(v) for k, v in re.findall(r"#define FLTOP_((?:TYPE|PREFERENCE|REDUCE)_[A-Z0-9]+|MAX_LABELS)\s+(\d+)", text)}
    assert said["MAX_LABELS"] == binding.MAX_LABELS
    assert {"sigmoid": said["PREFERENCE_SIGMOID"], "hinge": said["PREFERENCE_HINGE"],
            "square": said["PREFERENCE_SQUARE"]} == binding.PREFERENCE_KINDS
    assert {"token": said["REDUCE_TOKEN"], "sequence": said["REDUCE_SEQUENCE"], "sum": said["REDUCE_SUM"]} == binding.REDUCTIONS
    assert binding.ROW_TYPES == {torch.float32: said["TYPE_F32"], torch.bfloat16: said["TYPE_BF16"],
                                 torch.float16: said["TYPE_F16"]}


def test_more_than_a_launch_can_take(lib):
    """Batches whose launches would have 2^32 threads or more are refused before anything is enqueued."""
    big = 1 << 24
    assert lib.fltop_ctc_score(ctypes.byref(rows(B=big)), ctypes.byref(hyps()), FAKE, None, 0, None) == SHAPE
    many = ctypes.byref(rows(B=1 << 12)), ctypes.byref(hyps(N=512))
    assert lib.fltop_ctc_score(*many, FAKE, None, 0, None) == SHAPE
    long = ctypes.byref(rows(B=1 << 12, T=1 << 13)), ctypes.byref(hyps())
    assert lib.fltop_ctc_score(*long, FAKE, FAKE, 1 << 62, None) == SHAPE
    assert lib.fltop_ctc_score_grad(*long, FAKE, FAKE, 1 << 62, FAKE, None) == SHAPE
    assert lib.fltop_ctc_score_workspace_bytes(1 << 12, 1 << 13, 3, 8) == 0
    assert lib.fltop_ctc_score_workspace_bytes(1 << 12, 10, 512, 8) == 0
    p = binding.FltopPreference(FAKE, None, FAKE, None, big, 4, 6, 0, 0.1, 0.1, 1.0, FAKE, FAKE, FAKE)
    assert lib.fltop_preference_loss(ctypes.byref(p), FAKE, 1 << 62, None) == SHAPE
    assert lib.fltop_preference_workspace_bytes(big) == 0 and lib.fltop_policy_workspace_bytes(big, 1) == 0
    assert lib.fltop_policy_loss(FAKE, FAKE, None, FAKE, None, big, 4, ctypes.byref(settings()), FAKE, 1 << 62, FAKE, FAKE,
                                 None) == SHAPE
    assert lib.fltop_policy_loss_logits(ctypes.byref(rows(B=big)), FAKE, FAKE, None, FAKE, 0, ctypes.byref(settings()), FAKE,
                                        1 << 62, FAKE, FAKE, FAKE, None) == SHAPE
