"""Thin ctypes binding of the C ABI in include/fltop_ctc.h (argument marshalling only).

Every step of the decode runs in the HIP library; torch is used for device
memory and the current stream.  There is no fallback: if the shared library is
missing, loading raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("FLTOP_CTC_LIB") or os.path.join(_PKG, "libfltop_ctc.so")

MAX_BEAM = 1024
MAX_BEAM_STREAMING = 512      # the streaming entry points
MAX_VOCAB_WIDE_BEAM = 2048    # vocabulary limit of decodes with beam > 512
MAX_VOCAB = 4096

STATIC_SCRATCH_BYTES = 64 << 20

EXPORTS = ("fltop_ctc_workspace_bytes", "fltop_ctc_workspace_bytes_for", "fltop_ctc_decode",
           "fltop_ctc_decode_static",
           "fltop_ctc_prune", "fltop_ctc_search",
           "fltop_ctc_unpack_survivors", "fltop_ctc_token_ranks", "fltop_ctc_stream_state_bytes",
           "fltop_ctc_stream_begin", "fltop_ctc_stream_decode", "fltop_ctc_log_add",
           "fltop_ctc_score_workspace_bytes", "fltop_ctc_score", "fltop_ctc_score_grad",
           "fltop_preference_workspace_bytes", "fltop_preference_loss",
           "fltop_policy_workspace_bytes", "fltop_policy_loss", "fltop_policy_loss_logits",
           "fltop_status_string")

MAX_LABELS = 4095             # tokens of a hypothesis in ctc_score


class FltopParams(ctypes.Structure):
    _fields_ = [
        ("beam", ctypes.c_int32),
        ("rel_threshold", ctypes.c_float),
        ("top_n", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("beam_threshold", ctypes.c_double),
        ("lm_table", ctypes.c_void_p),
        ("lm_weight", ctypes.c_float),
        ("insertion_bonus", ctypes.c_float),
        ("nbest_count", ctypes.c_void_p),
        ("nbest_tokens", ctypes.c_void_p),
        ("nbest_lengths", ctypes.c_void_p),
        ("nbest_pb", ctypes.c_void_p),
        ("nbest_pnb", ctypes.c_void_p),
        ("frame_beam", ctypes.c_void_p),
        ("out_token_frames", ctypes.c_void_p),
    ]


class FltopRows(ctypes.Structure):
    _fields_ = [
        ("data", ctypes.c_void_p),
        ("lengths", ctypes.c_void_p),
        ("batch_stride", ctypes.c_int64),
        ("frame_stride", ctypes.c_int64),
        ("B", ctypes.c_int32),
        ("T", ctypes.c_int32),
        ("V", ctypes.c_int32),
        ("type", ctypes.c_int32),
    ]


class FltopHypotheses(ctypes.Structure):
    _fields_ = [
        ("tokens", ctypes.c_void_p),
        ("lengths", ctypes.c_void_p),
        ("counts", ctypes.c_void_p),
        ("token_batch_stride", ctypes.c_int64),
        ("token_stride", ctypes.c_int64),
        ("length_batch_stride", ctypes.c_int64),
        ("N", ctypes.c_int32),
        ("U", ctypes.c_int32),
    ]


class FltopPreference(ctypes.Structure):
    _fields_ = [
        ("scores", ctypes.c_void_p),
        ("ref_scores", ctypes.c_void_p),
        ("pairs", ctypes.c_void_p),
        ("pair_counts", ctypes.c_void_p),
        ("B", ctypes.c_int32),
        ("N", ctypes.c_int32),
        ("M", ctypes.c_int32),
        ("kind", ctypes.c_int32),
        ("beta", ctypes.c_double),
        ("label_smoothing", ctypes.c_double),
        ("scale", ctypes.c_double),
        ("loss", ctypes.c_void_p),
        ("margins", ctypes.c_void_p),
        ("grad_scores", ctypes.c_void_p),
    ]


class FltopPolicy(ctypes.Structure):
    _fields_ = [
        ("reduction", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("clip_low", ctypes.c_double),
        ("clip_high", ctypes.c_double),
        ("kl_weight", ctypes.c_double),
        ("scale", ctypes.c_double),
    ]


STATS_FIELDS = ("frames", "sum_survivors", "sum_candidates", "peak_candidates", "sum_beam",
                "select_passes", "exact_rankings", "overflow_drops", "survivor_records",
                "record_overflows")
# words to allocate for a fltop_stats block: the ten counters, and room for the 4 x 16 phase
# clocks that a profiling build of the library (-DFLTOP_PHASE_CLOCKS) appends
STATS_WORDS = len(STATS_FIELDS) + 64

_lib = None


class FltopError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def load():
    """Load the HIP library built in-tree; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2510_09085_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
    lib.fltop_ctc_workspace_bytes.restype = sz
    lib.fltop_ctc_workspace_bytes.argtypes = [i32, i32, i32, i32]
    lib.fltop_ctc_workspace_bytes_for.restype = sz
    lib.fltop_ctc_workspace_bytes_for.argtypes = [i32, i32, i32, i32, ctypes.c_uint64]
    lib.fltop_ctc_decode.restype = ctypes.c_int
    lib.fltop_ctc_decode.argtypes = [vp, vp, i32, i32, i32, ctypes.POINTER(FltopParams), vp, sz,
                                     vp, vp, vp, vp, vp]
    lib.fltop_ctc_decode_static.restype = ctypes.c_int
    lib.fltop_ctc_decode_static.argtypes = [vp, vp, i32, i32, i32, ctypes.POINTER(FltopParams),
                                            vp, vp, vp, vp, vp]
    lib.fltop_ctc_search.restype = ctypes.c_int
    lib.fltop_ctc_search.argtypes = [vp, i32, i32, i32, ctypes.POINTER(FltopParams), vp, sz,
                                     vp, vp, vp, vp, vp]
    lib.fltop_ctc_prune.restype = ctypes.c_int
    lib.fltop_ctc_prune.argtypes = [vp, vp, i32, i32, i32, i32, f32, i32, vp, sz, vp]
    lib.fltop_ctc_token_ranks.restype = ctypes.c_int
    lib.fltop_ctc_token_ranks.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.fltop_ctc_unpack_survivors.restype = ctypes.c_int
    lib.fltop_ctc_unpack_survivors.argtypes = [vp, sz, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.fltop_ctc_stream_state_bytes.restype = sz
    lib.fltop_ctc_stream_state_bytes.argtypes = [i32, i32, i32]
    lib.fltop_ctc_stream_begin.restype = ctypes.c_int
    lib.fltop_ctc_stream_begin.argtypes = [vp, sz, i32, i32, i32, vp]
    lib.fltop_ctc_stream_decode.restype = ctypes.c_int
    lib.fltop_ctc_stream_decode.argtypes = [vp, vp, i32, i32, i32, ctypes.POINTER(FltopParams),
                                            vp, sz, vp, sz, i32, vp, vp, vp, vp, vp]
    lib.fltop_ctc_log_add.restype = ctypes.c_int
    lib.fltop_ctc_log_add.argtypes = [vp, vp, vp, ctypes.c_int64, vp]
    rows, hyps = ctypes.POINTER(FltopRows), ctypes.POINTER(FltopHypotheses)
    policy = ctypes.POINTER(FltopPolicy)
    lib.fltop_ctc_score_workspace_bytes.restype = sz
    lib.fltop_ctc_score_workspace_bytes.argtypes = [i32, i32, i32, i32]
    lib.fltop_ctc_score.restype = ctypes.c_int
    lib.fltop_ctc_score.argtypes = [rows, hyps, vp, vp, sz, vp]
    lib.fltop_ctc_score_grad.restype = ctypes.c_int
    lib.fltop_ctc_score_grad.argtypes = [rows, hyps, vp, vp, sz, vp, vp]
    lib.fltop_preference_workspace_bytes.restype = sz
    lib.fltop_preference_workspace_bytes.argtypes = [i32]
    lib.fltop_preference_loss.restype = ctypes.c_int
    lib.fltop_preference_loss.argtypes = [ctypes.POINTER(FltopPreference), vp, sz, vp]
    lib.fltop_policy_workspace_bytes.restype = sz
    lib.fltop_policy_workspace_bytes.argtypes = [i32, i32]
    lib.fltop_policy_loss.restype = ctypes.c_int
    lib.fltop_policy_loss.argtypes = [vp, vp, vp, vp, vp, i32, i32, policy, vp, sz, vp, vp, vp]
    lib.fltop_policy_loss_logits.restype = ctypes.c_int
    lib.fltop_policy_loss_logits.argtypes = [rows, vp, vp, vp, vp, i32, policy, vp, sz, vp, vp, vp,
                                             vp]
    lib.fltop_status_string.restype = ctypes.c_char_p
    lib.fltop_status_string.argtypes = [ctypes.c_int]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().fltop_status_string(int(status)).decode()


def workspace_bytes(B: int, T: int, V: int, beam: int, max_records: Optional[int] = None) -> int:
    """Bytes that hold any input of these shapes, or (max_records given) the fixed regions plus
    room for that many survivor records beyond the six per frame that sit in the headers."""
    if max_records is None:
        return int(load().fltop_ctc_workspace_bytes(B, T, V, beam))
    return int(load().fltop_ctc_workspace_bytes_for(B, T, V, beam, int(max_records)))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream_handle(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _check_inputs(logprobs: torch.Tensor, lengths: torch.Tensor):
    if not (logprobs.is_cuda and lengths.is_cuda):
        raise ValueError("logprobs and lengths must be device tensors")
    if logprobs.dtype != torch.float32 or lengths.dtype != torch.int32:
        raise ValueError("logprobs must be float32 and lengths int32")
    if logprobs.dim() != 3 or not logprobs.is_contiguous() or not lengths.is_contiguous():
        raise ValueError("logprobs must be a contiguous [B,T,V] tensor")
    if lengths.numel() != logprobs.shape[0]:
        raise ValueError("lengths must have B entries")


def alloc_workspace(B: int, T: int, V: int, beam: int, device,
                    max_records: Optional[int] = None) -> torch.Tensor:
    n = workspace_bytes(B, T, V, beam, max_records)
    if n == 0:
        raise FltopError(-2, "fltop_ctc_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def decode_raw(logprobs, lengths, params: FltopParams, workspace, workspace_nbytes, out_tokens,
               out_lengths, out_scores, stats, stream=None) -> int:
    """Direct call of fltop_ctc_decode; returns the status code (no checks, no allocation)."""
    B, T, V = logprobs.shape
    return int(load().fltop_ctc_decode(_ptr(logprobs), _ptr(lengths), B, T, V,
                                       ctypes.byref(params), _ptr(workspace), workspace_nbytes,
                                       _ptr(out_tokens), _ptr(out_lengths), _ptr(out_scores),
                                       _ptr(stats), _stream_handle(stream)))


def decode_static_raw(logprobs, lengths, params: FltopParams, out_tokens, out_lengths, out_scores,
                      stats, stream=None) -> int:
    """Direct call of fltop_ctc_decode_static (workspace inside the library); returns the status."""
    B, T, V = logprobs.shape
    return int(load().fltop_ctc_decode_static(_ptr(logprobs), _ptr(lengths), B, T, V,
                                              ctypes.byref(params), _ptr(out_tokens),
                                              _ptr(out_lengths), _ptr(out_scores), _ptr(stats),
                                              _stream_handle(stream)))


def search_raw(lengths, shape, params: FltopParams, workspace, workspace_nbytes, out_tokens,
               out_lengths, out_scores, stats, stream=None) -> int:
    """Direct call of fltop_ctc_search on a workspace fltop_ctc_prune has filled."""
    B, T, V = shape
    return int(load().fltop_ctc_search(_ptr(lengths), B, T, V, ctypes.byref(params),
                                       _ptr(workspace), workspace_nbytes, _ptr(out_tokens),
                                       _ptr(out_lengths), _ptr(out_scores), _ptr(stats),
                                       _stream_handle(stream)))


def prune_raw(logprobs, lengths, beam, rel_threshold, workspace, workspace_nbytes,
              stream=None, top_n: int = 0) -> int:
    """Direct call of fltop_ctc_prune; returns the status code."""
    B, T, V = logprobs.shape
    return int(load().fltop_ctc_prune(_ptr(logprobs), _ptr(lengths), B, T, V, int(beam),
                                      float(rel_threshold), int(top_n), _ptr(workspace),
                                      workspace_nbytes, _stream_handle(stream)))


def decode(logprobs: torch.Tensor, lengths: torch.Tensor, beam: int, rel_threshold: float, *,
           top_n: int = 0, beam_threshold: float = 0.0,
           lm_table: Optional[torch.Tensor] = None, lm_weight: float = 0.0,
           insertion_bonus: float = 0.0, workspace: Optional[torch.Tensor] = None,
           want_stats: bool = False, want_nbest: bool = False, want_traces: bool = False,
           stream=None) -> dict:
    """fltop_ctc_decode on device tensors.  Returns device tensors (no host sync):
    tokens [B,T] int32, lengths [B] int32, scores [B] fp32, and optionally stats
    (uint64, see STATS_FIELDS), the n-best export, and the statistics traces
    (frame_beam [B,T], token_frames [B,T], both int32 and -1 where nothing was written)."""
    _check_inputs(logprobs, lengths)
    B, T, V = logprobs.shape
    dev = logprobs.device
    if workspace is None:
        workspace = alloc_workspace(B, T, V, beam, dev)
    out = {
        "tokens": torch.full((B, T), -1, dtype=torch.int32, device=dev),
        "lengths": torch.zeros(B, dtype=torch.int32, device=dev),
        "scores": torch.zeros(B, dtype=torch.float32, device=dev),
    }
    p = FltopParams()
    p.beam = int(beam)
    p.rel_threshold = float(rel_threshold)
    p.top_n = int(top_n)
    p.beam_threshold = float(beam_threshold)
    p.lm_weight = float(lm_weight)
    p.insertion_bonus = float(insertion_bonus)
    if lm_table is not None:
        if not (lm_table.is_cuda and lm_table.dtype == torch.float32 and lm_table.is_contiguous()
                and tuple(lm_table.shape) == (V, V)):
            raise ValueError("lm_table must be a contiguous float32 [V,V] device tensor")
        p.lm_table = lm_table.data_ptr()
    if want_nbest:
        out["nbest_count"] = torch.zeros(B, dtype=torch.int32, device=dev)
        out["nbest_tokens"] = torch.full((B, beam, T), -1, dtype=torch.int32, device=dev)
        out["nbest_lengths"] = torch.zeros((B, beam), dtype=torch.int32, device=dev)
        out["nbest_pb"] = torch.zeros((B, beam), dtype=torch.float64, device=dev)
        out["nbest_pnb"] = torch.zeros((B, beam), dtype=torch.float64, device=dev)
        p.nbest_count = out["nbest_count"].data_ptr()
        p.nbest_tokens = out["nbest_tokens"].data_ptr()
        p.nbest_lengths = out["nbest_lengths"].data_ptr()
        p.nbest_pb = out["nbest_pb"].data_ptr()
        p.nbest_pnb = out["nbest_pnb"].data_ptr()
    if want_traces:
        out["frame_beam"] = torch.full((B, T), -1, dtype=torch.int32, device=dev)
        out["token_frames"] = torch.full((B, T), -1, dtype=torch.int32, device=dev)
        p.frame_beam = out["frame_beam"].data_ptr()
        p.out_token_frames = out["token_frames"].data_ptr()
    stats = None
    if want_stats:
        stats = torch.zeros(STATS_WORDS, dtype=torch.int64, device=dev)
        out["stats"] = stats
    rc = decode_raw(logprobs, lengths, p, workspace, workspace.numel(), out["tokens"],
                    out["lengths"], out["scores"], stats, stream)
    if rc != 0:
        raise FltopError(rc, "fltop_ctc_decode")
    out["workspace"] = workspace
    return out


def prune(logprobs: torch.Tensor, lengths: torch.Tensor, beam: int, rel_threshold: float, *,
          top_n: int = 0, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """fltop_ctc_prune: survivor lists into the workspace (returned)."""
    _check_inputs(logprobs, lengths)
    B, T, V = logprobs.shape
    if workspace is None:
        workspace = alloc_workspace(B, T, V, beam, logprobs.device)
    rc = int(load().fltop_ctc_prune(_ptr(logprobs), _ptr(lengths), B, T, V, int(beam),
                                    float(rel_threshold), int(top_n), _ptr(workspace),
                                    workspace.numel(), _stream_handle(stream)))
    if rc != 0:
        raise FltopError(rc, "fltop_ctc_prune")
    return workspace


def unpack_survivors(workspace: torch.Tensor, lengths: torch.Tensor, B: int, T: int, V: int,
                     beam: int, stream=None):
    """fltop_ctc_unpack_survivors -> (counts [B*T], tokens [B*T,V], values [B*T,V], frame_max [B*T])."""
    dev = workspace.device
    counts = torch.zeros(B * T, dtype=torch.int32, device=dev)
    tokens = torch.full((B * T, V), -1, dtype=torch.int32, device=dev)
    values = torch.zeros((B * T, V), dtype=torch.float32, device=dev)
    fmax = torch.zeros(B * T, dtype=torch.float32, device=dev)
    rc = int(load().fltop_ctc_unpack_survivors(_ptr(workspace), workspace.numel(),
                                               _ptr(lengths), B, T, V,
                                               int(beam), _ptr(counts), _ptr(tokens),
                                               _ptr(values), _ptr(fmax), _stream_handle(stream)))
    if rc != 0:
        raise FltopError(rc, "fltop_ctc_unpack_survivors")
    return counts, tokens, values, fmax


def token_ranks(logprobs: torch.Tensor, tokens: torch.Tensor, token_frames: torch.Tensor,
                token_counts: torch.Tensor, stream=None):
    """fltop_ctc_token_ranks -> (ranks [B,T] int32 (-1 where unused), rank_count [V] int64,
    rank_lp_sum [V] float64)."""
    B, T, V = logprobs.shape
    dev = logprobs.device
    ranks = torch.full((B, T), -1, dtype=torch.int32, device=dev)
    count = torch.zeros(V, dtype=torch.int64, device=dev)
    lp_sum = torch.zeros(V, dtype=torch.float64, device=dev)
    rc = int(load().fltop_ctc_token_ranks(_ptr(logprobs), B, T, V, _ptr(tokens),
                                          _ptr(token_frames), _ptr(token_counts), _ptr(ranks),
                                          _ptr(count), _ptr(lp_sum), _stream_handle(stream)))
    if rc != 0:
        raise FltopError(rc, "fltop_ctc_token_ranks")
    return ranks, count, lp_sum


class Stream:
    """Chunked decoding of a batch of B streams of up to T_total frames each: owns the
    carried state, the output tensors and a workspace for chunks of up to T_chunk frames.
    feed() enqueues one chunk; the outputs then describe everything decoded so far."""

    def __init__(self, B: int, T_total: int, T_chunk: int, V: int, beam: int,
                 rel_threshold: float, device, *, top_n: int = 0, beam_threshold: float = 0.0,
                 lm_table: Optional[torch.Tensor] = None, lm_weight: float = 0.0,
                 insertion_bonus: float = 0.0, want_traces: bool = False):
        lib = load()
        self.B, self.T_total, self.T_chunk, self.V = B, T_total, T_chunk, V
        nbytes = int(lib.fltop_ctc_stream_state_bytes(B, T_total, beam))
        if nbytes == 0:
            raise FltopError(-2, "fltop_ctc_stream_state_bytes")
        self.state = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.workspace = alloc_workspace(B, T_chunk, V, beam, device)
        self.tokens = torch.full((B, T_total), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(B, dtype=torch.int32, device=device)
        self.scores = torch.zeros(B, dtype=torch.float32, device=device)
        self.stats = torch.zeros(STATS_WORDS, dtype=torch.int64, device=device)
        p = FltopParams()
        p.beam = int(beam)
        p.rel_threshold = float(rel_threshold)
        p.top_n = int(top_n)
        p.beam_threshold = float(beam_threshold)
        p.lm_weight = float(lm_weight)
        p.insertion_bonus = float(insertion_bonus)
        self._lm = lm_table
        if lm_table is not None:
            p.lm_table = lm_table.data_ptr()
        self.frame_beam = self.token_frames = None
        if want_traces:
            self.frame_beam = torch.full((B, T_total), -1, dtype=torch.int32, device=device)
            self.token_frames = torch.full((B, T_total), -1, dtype=torch.int32, device=device)
            p.frame_beam = self.frame_beam.data_ptr()
            p.out_token_frames = self.token_frames.data_ptr()
        self.params = p
        self.begin()

    def begin(self, stream=None):
        rc = int(load().fltop_ctc_stream_begin(_ptr(self.state), self.state.numel(), self.B,
                                               self.T_total, self.params.beam,
                                               _stream_handle(stream)))
        if rc != 0:
            raise FltopError(rc, "fltop_ctc_stream_begin")

    def feed(self, logprobs: torch.Tensor, lengths: torch.Tensor, stream=None):
        """logprobs [B,Tc,V] (Tc <= T_chunk), lengths [B]: valid frames of this chunk."""
        _check_inputs(logprobs, lengths)
        B, Tc, V = logprobs.shape
        if B != self.B or V != self.V or Tc > self.T_chunk:
            raise ValueError("chunk shape does not fit this stream")
        rc = int(load().fltop_ctc_stream_decode(
            _ptr(logprobs), _ptr(lengths), B, Tc, V, ctypes.byref(self.params),
            _ptr(self.workspace), self.workspace.numel(), _ptr(self.state), self.state.numel(),
            self.T_total, _ptr(self.tokens), _ptr(self.lengths), _ptr(self.scores),
            _ptr(self.stats), _stream_handle(stream)))
        if rc != 0:
            raise FltopError(rc, "fltop_ctc_stream_decode")


def log_add(a: torch.Tensor, b: torch.Tensor, stream=None) -> torch.Tensor:
    """fltop_ctc_log_add on two float64 device tensors of equal size."""
    if not (a.is_cuda and b.is_cuda and a.dtype == torch.float64 and b.dtype == torch.float64
            and a.is_contiguous() and b.is_contiguous() and a.numel() == b.numel()):
        raise ValueError("a and b must be contiguous float64 device tensors of one size")
    out = torch.empty_like(a)
    rc = int(load().fltop_ctc_log_add(_ptr(a), _ptr(b), _ptr(out), a.numel(),
                                      _stream_handle(stream)))
    if rc != 0:
        raise FltopError(rc, "fltop_ctc_log_add")
    return out


def stats_dict(stats: torch.Tensor) -> dict:
    vals = stats.cpu().tolist()
    out = dict(zip(STATS_FIELDS, vals))
    out.update({f"clk{i}": v for i, v in enumerate(vals[len(STATS_FIELDS):])})
    return out


# ---- learning from hypotheses ------------------------------------------------------------------
#
# Calls on plain device memory, as decode is: nothing that they return carries autograd history, also
# where an input requires a gradient.  Gradients are results of their own (grad_scores, grad_logits,
# ctc_score_grad's) and reach a model by `tensor.backward(gradient)`.

ROW_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
PREFERENCE_KINDS = {"sigmoid": 0, "hinge": 1, "square": 2}
REDUCTIONS = {"token": 0, "sequence": 1, "sum": 2}


class _On:
    """The device of `t` made current, and outputs and workspaces taken on the stream that the call
    is enqueued on, so that they outlive their use there.  `stream` None: that device's current one."""

    __slots__ = ("_managers", "_index", "_stream")

    def __init__(self, t: torch.Tensor, stream):
        self._index, self._stream, self._managers = t.device.index, stream, ()
        if self._index != torch.cuda.current_device():
            self._managers += (torch.cuda.device(t.device),)
        if stream is not None:
            self._managers += (torch.cuda.stream(stream),)

    def __enter__(self):
        for manager in self._managers:
            manager.__enter__()
        stream = torch.cuda.current_stream(self._index) if self._stream is None else self._stream
        return stream.cuda_stream

    def __exit__(self, *what):
        for manager in reversed(self._managers):
            manager.__exit__(*what)


def _need(ok: bool, message: str):
    if not ok:
        raise ValueError(message)


def _device_tensor(t, name: str, dtype, shape, device):
    """Checks a dense tensor of one call (all of a call's tensors are on one device)."""
    if t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous():
        return
    if not (t.is_cuda and t.device == device):
        raise ValueError(f"{name} must be on {device}, where the call's other tensors are")
    raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {list(shape)}")


def _rows(x: torch.Tensor, lengths: torch.Tensor, name: str) -> FltopRows:
    _need(x.is_cuda, f"{name} must be a device tensor")
    kind = ROW_TYPES.get(x.dtype)
    _need(kind is not None, f"{name} must be float32, bfloat16 or float16")
    _need(x.dim() == 3 and x.numel() > 0, f"{name} must be a [B,T,V] tensor")
    B, T, V = x.shape
    by_batch, by_frame, by_value = x.stride()
    _need(by_value == 1 or V == 1, f"{name}: the V values of a row must be adjacent")
    _device_tensor(lengths, "lengths", torch.int32, (B,), x.device)
    return FltopRows(x.data_ptr(), lengths.data_ptr(), by_batch, by_frame, B, T, V, kind)


def _hypotheses(tokens, token_lengths, counts, B: int, device) -> FltopHypotheses:
    _need(tokens.dim() == 3 and tokens.shape[0] == B and tokens.numel() > 0
          and tokens.dtype == torch.int32 and tokens.device == device,
          f"tokens must be an int32 [B,N,U] tensor on {device}")
    _, N, U = tokens.shape
    by_batch, by_hypothesis, by_token = tokens.stride()
    _need(by_token == 1 or U == 1, "the tokens of a hypothesis must be adjacent")
    _need(token_lengths.shape == (B, N) and token_lengths.dtype == torch.int32
          and token_lengths.device == device, f"token_lengths must be an int32 [B,N] tensor on {device}")
    lengths_by_batch, by_length = token_lengths.stride()
    _need(by_length == 1 or N == 1, "the token lengths of an utterance must be adjacent")
    if counts is not None:
        _device_tensor(counts, "counts", torch.int32, (B,), device)
    return FltopHypotheses(tokens.data_ptr(), token_lengths.data_ptr(), _address(counts), by_batch,
                           by_hypothesis, lengths_by_batch, N, U)


def _address(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _raise(rc: int, where: str):
    if rc != 0:
        raise FltopError(rc, where)


@functools.lru_cache(maxsize=256)
def _bytes(where: str, *shape: int) -> int:
    n = int(getattr(load(), where)(*shape))
    if n == 0:
        raise FltopError(-2, where)
    return n


def _workspace(workspace, device, where: str, *shape: int) -> torch.Tensor:
    """The caller's workspace, or one of the size that the library's function `where` gives."""
    if workspace is None:
        return torch.empty(_bytes(where, *shape), dtype=torch.uint8, device=device)
    _need(workspace.device == device and workspace.is_contiguous() and workspace.dtype == torch.uint8,
          f"the workspace must be a contiguous uint8 tensor on {device}")
    return workspace


def score_workspace_bytes(B: int, T: int, N: int, U: int) -> int:
    """Bytes that ctc_score leaves for ctc_score_grad (0 if the shapes are invalid)."""
    return int(load().fltop_ctc_score_workspace_bytes(B, T, N, U))


def ctc_score(logprobs: torch.Tensor, lengths: torch.Tensor, tokens: torch.Tensor,
              token_lengths: torch.Tensor, counts: Optional[torch.Tensor] = None, *,
              want_grad: bool = False, workspace: Optional[torch.Tensor] = None,
              stream=None) -> dict:
    """fltop_ctc_score: log-probability of N hypotheses of each utterance, over all alignments.

    logprobs [B,T,V] float32, bfloat16 or float16 with adjacent values in a row (a [T,B,V] tensor
    transposed is fine), lengths [B]; tokens [B,N,U] and token_lengths [B,N] int32 as decode's
    n-best export gives them (slices too: `nbest_tokens[:, :8, :200]`), counts [B] its nbest_count.
    Returns scores [B,N] float64; with want_grad also the workspace that ctc_score_grad needs
    (about 4 * B * N * T * U bytes, twice that from U = 1920 on: slice the tokens to the longest
    hypothesis).  The scores carry no autograd history, whether or not logprobs does: their gradient is
    what ctc_score_grad returns."""
    x = _rows(logprobs, lengths, "logprobs")
    dev = logprobs.device
    h = _hypotheses(tokens, token_lengths, counts, x.B, dev)
    with _On(logprobs, stream) as handle:
        out = {"scores": torch.empty((x.B, h.N), dtype=torch.float64, device=dev)}
        if want_grad or workspace is not None:
            out["workspace"] = _workspace(workspace, dev, "fltop_ctc_score_workspace_bytes", x.B, x.T, h.N, h.U)
        ws = out.get("workspace")
        _raise(load().fltop_ctc_score(ctypes.byref(x), ctypes.byref(h), _address(out["scores"]), _address(ws),
                                      0 if ws is None else ws.numel(), handle), "fltop_ctc_score")
    return out


def ctc_score_grad(logprobs: torch.Tensor, lengths: torch.Tensor, tokens: torch.Tensor,
                   token_lengths: torch.Tensor, grad_scores: torch.Tensor,
                   workspace: torch.Tensor, counts: Optional[torch.Tensor] = None, *,
                   stream=None) -> torch.Tensor:
    """fltop_ctc_score_grad: from the derivative of a loss to ctc_score's scores (float64 [B,N])
    its derivative to logprobs, [B,T,V] of their type.  The other arguments as given to ctc_score,
    `workspace` as it returned it.  A model's gradient follows by `logprobs.backward(grad)`."""
    x = _rows(logprobs, lengths, "logprobs")
    dev = logprobs.device
    h = _hypotheses(tokens, token_lengths, counts, x.B, dev)
    _device_tensor(grad_scores, "grad_scores", torch.float64, (x.B, h.N), dev)
    _need(workspace is not None, "workspace must be the one that ctc_score returned")
    ws = _workspace(workspace, dev, "fltop_ctc_score_workspace_bytes", x.B, x.T, h.N, h.U)
    with _On(logprobs, stream) as handle:
        grad = torch.empty((x.B, x.T, x.V), dtype=logprobs.dtype, device=dev)
        _raise(load().fltop_ctc_score_grad(ctypes.byref(x), ctypes.byref(h), _address(grad_scores), _address(ws),
                                           ws.numel(), _address(grad), handle), "fltop_ctc_score_grad")
    return grad


def preference_loss(scores: torch.Tensor, pairs: torch.Tensor, *,
                    ref_scores: Optional[torch.Tensor] = None,
                    pair_counts: Optional[torch.Tensor] = None, kind: str = "sigmoid",
                    beta: float = 0.1, label_smoothing: float = 0.0, scale: float = 1.0,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> dict:
    """fltop_preference_loss: mean loss over pairs (won, lost) of an utterance's hypotheses.

    scores, ref_scores float64 [B,N] (ctc_score's), pairs int32 [B,M,2] of places in [0,N) (a pair
    with any other place takes no part; M may be 0), pair_counts int32 [B]; kind "sigmoid", "hinge"
    or "square".
    Returns loss (float64), margins [B,M] and grad_scores [B,N], the gradient of scale * loss."""
    _need(scores.is_cuda and scores.dim() == 2, "scores must be a [B,N] device tensor")
    dev, (B, N) = scores.device, scores.shape
    _device_tensor(scores, "scores", torch.float64, (B, N), dev)
    _need(pairs.dim() == 3, "pairs must be an int32 [B,M,2] tensor")
    M = pairs.shape[1]
    _device_tensor(pairs, "pairs", torch.int32, (B, M, 2), dev)
    if ref_scores is not None:
        _device_tensor(ref_scores, "ref_scores", torch.float64, (B, N), dev)
    if pair_counts is not None:
        _device_tensor(pair_counts, "pair_counts", torch.int32, (B,), dev)
    if kind not in PREFERENCE_KINDS:
        raise ValueError(f"kind must be one of {', '.join(PREFERENCE_KINDS)}")
    with _On(scores, stream) as handle:
        if M == 0:  # the library takes lists of one pair and more: one that takes no part
            pairs = torch.full((B, 1, 2), -1, dtype=torch.int32, device=dev)
        room = pairs.shape[1]
        grad = torch.empty_like(scores)
        loss = torch.empty((), dtype=torch.float64, device=dev)
        margins = torch.empty((B, room), dtype=torch.float64, device=dev)
        ws = _workspace(workspace, dev, "fltop_preference_workspace_bytes", B)
        p = FltopPreference(scores.data_ptr(), _address(ref_scores),
                            pairs.data_ptr(), _address(pair_counts),
                            B, N, room, PREFERENCE_KINDS[kind], beta, label_smoothing, scale,
                            loss.data_ptr(), margins.data_ptr(), grad.data_ptr())
        _raise(load().fltop_preference_loss(ctypes.byref(p), _address(ws), ws.numel(), handle),
               "fltop_preference_loss")
    return {"loss": loss, "margins": margins if M else margins[:, :0], "grad_scores": grad}


def _policy(reduction, clip_low, clip_high, kl_weight, scale) -> FltopPolicy:
    if reduction not in REDUCTIONS:
        raise ValueError(f"reduction must be one of {', '.join(REDUCTIONS)}")
    return FltopPolicy(REDUCTIONS[reduction], 0, clip_low, clip_high, kl_weight, scale)


def policy_loss(scores: torch.Tensor, old_scores: torch.Tensor, advantages: torch.Tensor, *,
                ref_scores: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None,
                clip_low: float = 0.2, clip_high: float = 0.2, kl_weight: float = 0.0,
                reduction: str = "token", scale: float = 1.0,
                workspace: Optional[torch.Tensor] = None, stream=None) -> dict:
    """fltop_policy_loss: clipped policy loss with a KL term over log-probabilities, float64 [B,N]
    throughout (ctc_score's scores of an utterance's hypotheses); counts int32 [B].  `reduction`
    "token" (mean of all entries), "sequence" (mean of the rows' means) or "sum".  Returns loss, kl,
    clipped (share of entries) and grad_scores [B,N], the gradient of scale * loss."""
    _need(scores.is_cuda and scores.dim() == 2, "scores must be a [B,N] device tensor")
    dev, (B, N) = scores.device, scores.shape
    for name, t in (("scores", scores), ("old_scores", old_scores), ("advantages", advantages),
                    ("ref_scores", ref_scores)):
        if t is not None:
            _device_tensor(t, name, torch.float64, (B, N), dev)
    if counts is not None:
        _device_tensor(counts, "counts", torch.int32, (B,), dev)
    p = _policy(reduction, clip_low, clip_high, kl_weight, scale)
    with _On(scores, stream) as handle:
        grad = torch.empty_like(scores)
        summary = torch.empty(3, dtype=torch.float64, device=dev)
        ws = _workspace(workspace, dev, "fltop_policy_workspace_bytes", B, 1)
        _raise(load().fltop_policy_loss(_address(scores), _address(old_scores), _address(ref_scores), _address(advantages),
                                        _address(counts), B, N, ctypes.byref(p), _address(ws), ws.numel(),
                                        _address(summary), _address(grad), handle), "fltop_policy_loss")
    loss, kl, clipped = summary.unbind()
    return {"loss": loss, "kl": kl, "clipped": clipped, "grad_scores": grad}


def policy_loss_logits(logits: torch.Tensor, tokens: torch.Tensor, lengths: torch.Tensor,
                       old_logps: torch.Tensor, advantages: torch.Tensor, *,
                       ref_logps: Optional[torch.Tensor] = None, clip_low: float = 0.2,
                       clip_high: float = 0.2, kl_weight: float = 0.0, reduction: str = "token",
                       scale: float = 1.0, workspace: Optional[torch.Tensor] = None,
                       stream=None) -> dict:
    """fltop_policy_loss_logits: the same loss over the frames (or tokens) of [B,T,V] logits.

    logits float32, bfloat16 or float16 with adjacent values in a row, tokens int32 [B,T] (a place
    with a token outside [0,V), such as -1, takes no part), lengths int32 [B], old_logps and
    ref_logps float32 [B,T], advantages float32 [B] or [B,T].  Returns loss, kl, clipped, logps
    [B,T] float32 and grad_logits [B,T,V] of the logits' type, the gradient of scale * loss."""
    x = _rows(logits, lengths, "logits")
    dev, shape = logits.device, (x.B, x.T)
    _device_tensor(tokens, "tokens", torch.int32, shape, dev)
    _device_tensor(old_logps, "old_logps", torch.float32, shape, dev)
    if ref_logps is not None:
        _device_tensor(ref_logps, "ref_logps", torch.float32, shape, dev)
    per_frame = advantages.dim() == 2
    _device_tensor(advantages, "advantages", torch.float32, shape if per_frame else (x.B,), dev)
    p = _policy(reduction, clip_low, clip_high, kl_weight, scale)
    with _On(logits, stream) as handle:
        grad = torch.empty((x.B, x.T, x.V), dtype=logits.dtype, device=dev)
        logps = torch.empty(shape, dtype=torch.float32, device=dev)
        summary = torch.empty(3, dtype=torch.float32, device=dev)
        ws = _workspace(workspace, dev, "fltop_policy_workspace_bytes", x.B, x.T)
        _raise(load().fltop_policy_loss_logits(ctypes.byref(x), _address(tokens), _address(old_logps),
                                               _address(ref_logps), _address(advantages), int(per_frame),
                                               ctypes.byref(p), _address(ws), ws.numel(), _address(summary),
                                               _address(logps), _address(grad), handle),
               "fltop_policy_loss_logits")
    loss, kl, clipped = summary.unbind()
    return {"loss": loss, "kl": kl, "clipped": clipped, "logps": logps, "grad_logits": grad}
