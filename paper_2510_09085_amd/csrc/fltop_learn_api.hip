// C ABI of the operators that learn from hypotheses: argument checks and launches.
// See include/fltop_ctc.h for the contract of every entry point.
#include <cmath>

#include "fltop_learn.h"

namespace {

// A launch has fewer than 2^32 threads: of 256 in a workgroup for each row of a batch, of 1024 in two workgroups for each
// hypothesis, of 256 in four for each block of frames.
constexpr int64_t kMostBatch = (1 << 24) - 1, kMostHypotheses = (1 << 21) - 1, kMostBlocks = (1 << 22) - 1;
// Loops over a batch's frames, a row's logits and a row's entries count in 32 bits, up to 8192 beyond the last one.
constexpr int64_t kMostPlaces = (int64_t)INT32_MAX - 8192;

int check_rows(const fltop_rows* x, bool decodes) {
    if (!x || !x->data || !x->lengths) return FLTOP_ERR_NULL_POINTER;
    if (x->B < 1 || x->T < 1 || x->V < (decodes ? 2 : 1)) return FLTOP_ERR_BAD_SHAPE;
    if (x->batch_stride < 0 || x->frame_stride < 0) return FLTOP_ERR_BAD_SHAPE;
    if (x->B > kMostBatch || (int64_t)x->B * x->T > kMostPlaces || x->V > kMostPlaces) return FLTOP_ERR_BAD_SHAPE;
    if (decodes && x->V > FLTOP_MAX_VOCAB) return FLTOP_ERR_VOCAB_TOO_BIG;
    if (x->type < FLTOP_TYPE_F32 || x->type > FLTOP_TYPE_F16) return FLTOP_ERR_BAD_OPTION;
    return FLTOP_OK;
}

bool lattice_shapes(int32_t B, int32_t T, int32_t N, int32_t U) {
    return B >= 1 && T >= 1 && (int64_t)B * T <= kMostPlaces && N >= 1 && N <= FLTOP_MAX_BEAM && U >= 1 &&
           U <= FLTOP_MAX_LABELS && (int64_t)B * N <= kMostHypotheses;
}

// Whether the borders of these lattices can be addressed (their places as bytes within 63 bits), and their blocks launched.
bool lattice_fits(int32_t B, int32_t T, int32_t N, int32_t U) {
    return lattice_shapes(B, T, N, U) && (int64_t)B * (T / 8 + 1) <= kMostBlocks &&
           (double)B * N * T * (2.0 * U + 1100.0) < 7e16;
}

int check_hypotheses(const fltop_rows* x, const fltop_hypotheses* h) {
    if (!h || !h->tokens || !h->lengths) return FLTOP_ERR_NULL_POINTER;
    if (h->N > FLTOP_MAX_BEAM) return FLTOP_ERR_BAD_BEAM;
    if (!lattice_shapes(x->B, x->T, h->N, h->U)) return FLTOP_ERR_BAD_SHAPE;
    if (h->token_batch_stride < 0 || h->token_stride < 0 || h->length_batch_stride < 0) return FLTOP_ERR_BAD_SHAPE;
    return FLTOP_OK;
}

int check_space(const void* ws, size_t bytes, size_t need) {
    if (!ws) return FLTOP_ERR_NULL_POINTER;
    if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return FLTOP_ERR_ALIGNMENT;
    return bytes < need ? FLTOP_ERR_WORKSPACE : FLTOP_OK;
}

int check_policy(const fltop_policy* p) {
    if (!p) return FLTOP_ERR_NULL_POINTER;
    const bool fine = p->reduction >= FLTOP_REDUCE_TOKEN && p->reduction <= FLTOP_REDUCE_SUM && p->clip_low >= 0.0 &&
                      p->clip_low <= 1.0 && p->clip_high >= 0.0 && std::isfinite(p->clip_high) &&
                      std::isfinite(p->kl_weight) && std::isfinite(p->scale);
    return fine ? FLTOP_OK : FLTOP_ERR_BAD_OPTION;
}

int launched(hipError_t e) { return e == hipSuccess ? FLTOP_OK : FLTOP_ERR_HIP; }

}  // namespace

extern "C" size_t fltop_ctc_score_workspace_bytes(int32_t B, int32_t T, int32_t N, int32_t U) {
    return lattice_fits(B, T, N, U) ? fltop::carve_score(nullptr, B, T, N, U).bytes : 0;
}

extern "C" int fltop_ctc_score(const fltop_rows* logprobs, const fltop_hypotheses* hyps, double* out_scores,
                               void* workspace, size_t workspace_bytes, void* hip_stream) {
    int rc = check_rows(logprobs, true);
    if (rc != FLTOP_OK) return rc;
    rc = check_hypotheses(logprobs, hyps);
    if (rc != FLTOP_OK) return rc;
    if (!out_scores) return FLTOP_ERR_NULL_POINTER;
    const fltop::ScoreSpace ws = fltop::carve_score(workspace, logprobs->B, logprobs->T, hyps->N, hyps->U);
    if (workspace) {
        if (!lattice_fits(logprobs->B, logprobs->T, hyps->N, hyps->U)) return FLTOP_ERR_BAD_SHAPE;
        rc = check_space(workspace, workspace_bytes, ws.bytes);
        if (rc != FLTOP_OK) return rc;
    }
    return launched(fltop::launch_score(*logprobs, *hyps, out_scores, workspace ? &ws : nullptr,
                                        static_cast<hipStream_t>(hip_stream)));
}

extern "C" int fltop_ctc_score_grad(const fltop_rows* logprobs, const fltop_hypotheses* hyps, const double* grad_scores,
                                    void* workspace, size_t workspace_bytes, void* grad_logprobs, void* hip_stream) {
    int rc = check_rows(logprobs, true);
    if (rc != FLTOP_OK) return rc;
    rc = check_hypotheses(logprobs, hyps);
    if (rc != FLTOP_OK) return rc;
    if (!grad_scores || !grad_logprobs) return FLTOP_ERR_NULL_POINTER;
    if (!lattice_fits(logprobs->B, logprobs->T, hyps->N, hyps->U)) return FLTOP_ERR_BAD_SHAPE;
    const fltop::ScoreSpace ws = fltop::carve_score(workspace, logprobs->B, logprobs->T, hyps->N, hyps->U);
    rc = check_space(workspace, workspace_bytes, ws.bytes);
    if (rc != FLTOP_OK) return rc;
    return launched(fltop::launch_score_grad(*logprobs, *hyps, grad_scores, ws, grad_logprobs,
                                             static_cast<hipStream_t>(hip_stream)));
}

extern "C" size_t fltop_preference_workspace_bytes(int32_t B) {
    return B < 1 || B > kMostBatch ? 0 : fltop::align_up((size_t)B * 2 * sizeof(double), 256);
}

extern "C" int fltop_preference_loss(const fltop_preference* p, void* workspace, size_t workspace_bytes,
                                     void* hip_stream) {
    if (!p || !p->scores || !p->pairs || !p->loss || !p->margins || !p->grad_scores) return FLTOP_ERR_NULL_POINTER;
    if (p->B < 1 || p->B > kMostBatch || p->N < 1 || p->M < 1 || p->M > (1 << 29)) return FLTOP_ERR_BAD_SHAPE;
    if (p->N > FLTOP_MAX_BEAM) return FLTOP_ERR_BAD_BEAM;
    const bool sigmoid = p->kind == FLTOP_PREFERENCE_SIGMOID;
    if (p->kind < FLTOP_PREFERENCE_SIGMOID || p->kind > FLTOP_PREFERENCE_SQUARE || !(p->beta > 0.0) ||
        !std::isfinite(p->beta) || !(p->label_smoothing >= 0.0 && p->label_smoothing <= (sigmoid ? 0.5 : 0.0)) ||
        !std::isfinite(p->scale))
        return FLTOP_ERR_BAD_OPTION;
    const int rc = check_space(workspace, workspace_bytes, fltop_preference_workspace_bytes(p->B));
    if (rc != FLTOP_OK) return rc;
    return launched(fltop::launch_preference(*p, workspace, static_cast<hipStream_t>(hip_stream)));
}

extern "C" size_t fltop_policy_workspace_bytes(int32_t B, int32_t T) {
    if (B < 1 || B > kMostBatch || T < 1 || (int64_t)B * T > kMostPlaces) return 0;
    // (both policy losses are asked for with T = 1: rows of hypotheses, and one token a row)
    const size_t sums = fltop::policy_sums_bytes(B), rows = fltop::row_workspace_bytes(B);
    return sums > rows ? sums : rows;
}

extern "C" int fltop_policy_loss(const double* scores, const double* old_scores, const double* ref_scores,
                                 const double* advantages, const int32_t* counts, int32_t B, int32_t N,
                                 const fltop_policy* policy, void* workspace, size_t workspace_bytes, double* summary,
                                 double* grad_scores, void* hip_stream) {
    if (!scores || !old_scores || !advantages || !summary || !grad_scores) return FLTOP_ERR_NULL_POINTER;
    if (B < 1 || B > kMostBatch || N < 1 || N > kMostPlaces) return FLTOP_ERR_BAD_SHAPE;
    int rc = check_policy(policy);
    if (rc != FLTOP_OK) return rc;
    rc = check_space(workspace, workspace_bytes, fltop_policy_workspace_bytes(B, 1));
    if (rc != FLTOP_OK) return rc;
    return launched(fltop::launch_policy(scores, old_scores, ref_scores, advantages, counts, B, N, *policy, workspace,
                                         summary, grad_scores, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int fltop_policy_loss_logits(const fltop_rows* logits, const int32_t* tokens, const float* old_logps,
                                        const float* ref_logps, const float* advantages, int32_t advantages_per_frame,
                                        const fltop_policy* policy, void* workspace, size_t workspace_bytes,
                                        float* summary, float* logps, void* grad_logits, void* hip_stream) {
    int rc = check_rows(logits, false);
    if (rc != FLTOP_OK) return rc;
    if (!tokens || !old_logps || !advantages || !summary || !logps || !grad_logits) return FLTOP_ERR_NULL_POINTER;
    rc = check_policy(policy);
    if (rc != FLTOP_OK) return rc;
    rc = check_space(workspace, workspace_bytes, fltop_policy_workspace_bytes(logits->B, logits->T));
    if (rc != FLTOP_OK) return rc;
    return launched(fltop::launch_policy_logits(*logits, tokens, old_logps, ref_logps, advantages,
                                                advantages_per_frame != 0, *policy, workspace, summary, logps,
                                                grad_logits, static_cast<hipStream_t>(hip_stream)));
}
