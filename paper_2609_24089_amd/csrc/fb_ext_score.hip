// C ABI of the attention over capped scores, distance biases and spans: validation and
// dispatch.  The entry points are declared (and documented) in include/flashbob.h.
#include "fb_ext_score.h"

namespace fb {

// Returns BOB_OK to proceed, or an error; sets *empty where there is nothing to compute.
static int32_t score_check(const ScoreProblem& p, bool* empty) {
  const int32_t rc = ext_check(p, empty);
  if (rc != BOB_OK) return rc;
  // the argument of the tanh and the capped score stay finite
  if (!(p.cap >= 0.f) || !std::isfinite(p.cap)) return BOB_EINVAL;
  if (p.cap > 0.f && (p.cap < 1e-6f || p.cap > 1e6f || std::fabs(p.scale) > 1e6f)) return BOB_EINVAL;
  if ((reinterpret_cast<uintptr_t>(p.spans) & 15) != 0 || (reinterpret_cast<uintptr_t>(p.slopes) & 3) != 0)
    return BOB_EINVAL;
  if (p.spans != nullptr && p.causal != 0) return BOB_EINVAL;
  if (p.slopes != nullptr && !*empty && ext_group(p) > kMaxSlopeGroup) return BOB_EINVAL;
  return BOB_OK;
}

static ScoreProblem score_problem(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t d,
                                  float scale, int32_t causal, const attn_score* score) {
  ScoreProblem p{};
  static_cast<ExtProblem&>(p) = ExtProblem{dtype, B, H, Hkv, Nq, Nk, d, scale, causal, attn_ext{}};
  if (score != nullptr) {
    p.x.q_lens = score->q_lens;
    p.x.kv_lens = score->kv_lens;
    p.x.q_starts = score->q_starts;
    p.spans = score->spans;
    p.slopes = score->slopes;
    p.cap = score->cap;
  }
  return p;
}

static ExtPlan plan_fwd(const ScoreProblem& p) { FB_EXT_DISPATCH(p, score_fwd_plan, p); }
static ExtPlan plan_rows(const ScoreProblem& p) { FB_EXT_DISPATCH(p, score_rows_plan, p); }
static ExtPlan plan_cols(const ScoreProblem& p) { FB_EXT_DISPATCH(p, score_cols_plan, p); }
static ExtPlan plan_pass1(const ScoreProblem& p) { FB_EXT_DISPATCH(p, score_pass1_plan, p); }
static ExtPlan plan_pass2(const ScoreProblem& p) { FB_EXT_DISPATCH(p, score_pass2_plan, p); }
static int32_t go_fwd(const ScoreProblem& p, const void* Q, const void* K, const void* V, void* O, void* Orest,
                      float* L, float* ws, hipStream_t s) {
  FB_EXT_DISPATCH(p, score_launch_fwd, p, Q, K, V, O, Orest, L, ws, s);
}
static int32_t go_bwd(const ScoreProblem& p, const void* Q, const void* K, const void* V, const void* O,
                      const void* Orest, const void* dO, const float* L, void* dQ, void* dK, void* dV, float* D,
                      float* row_parts, float* parts, hipStream_t s) {
  FB_EXT_DISPATCH(p, score_launch_bwd, p, Q, K, V, O, Orest, dO, L, dQ, dK, dV, D, row_parts, parts, s);
}
static int32_t go_pass1(const ScoreProblem& p, const void* Q, const void* K, const void* V, const void* O,
                        const void* Orest, const void* dO, const void* UQ, const void* UK, const void* UV,
                        const float* L, const float* D, const void* dQ, void* Qt, void* dOt, float* alpha,
                        float* E, float* parts, hipStream_t s) {
  FB_EXT_DISPATCH(p, score_launch_pass1, p, Q, K, V, O, Orest, dO, UQ, UK, UV, L, D, dQ, Qt, dOt, alpha, E, parts, s);
}
static int32_t go_pass2(const ScoreProblem& p, const void* Q, const void* K, const void* V, const void* dO,
                        const void* UQ, const void* UK, const void* UV, const float* L, const float* D,
                        const float* alpha, const float* E, void* Kt, void* Vt, float* parts, hipStream_t s) {
  FB_EXT_DISPATCH(p, score_launch_pass2, p, Q, K, V, dO, UQ, UK, UV, L, D, alpha, E, Kt, Vt, parts, s);
}

static int64_t rows_bytes(const ScoreProblem& p) { return ext_row_bytes(p, plan_rows(p), p.d + 1); }
// The parts' fp32 sums of a column kernel.
static int64_t parts_bytes(const ScoreProblem& p, const ExtPlan& c) {
  return c.parts > 1 ? (int64_t)c.parts * 2 * ext_slices(p, c).rows * p.d * 4 : 0;
}
static int64_t call_bytes(int32_t call, const ScoreProblem& p) {
  switch (call) {
    case ATTN_SCORE_FWD: return p.Nq == 0 ? 0 : ext_row_bytes(p, plan_fwd(p), p.d + kFwdScalars);
    case ATTN_SCORE_BWD: return rows_bytes(p) + parts_bytes(p, plan_cols(p));
    case ATTN_SCORE_PASS1: return p.Nq == 0 ? 0 : ext_row_bytes(p, plan_pass1(p), 3 * p.d + 2);
    default: return parts_bytes(p, plan_pass2(p));
  }
}
// Orest: NULL, or as the other matrices of n rows.
static bool score_rest(int64_t n, const void* Orest) { return n == 0 || Orest == nullptr || aligned16(Orest); }
static bool workspace_fits(int64_t need, const void* workspace, int64_t bytes) {
  return need == 0 || (bytes >= need && aligned16(workspace));
}

}  // namespace fb

using fb::ScoreProblem;

extern "C" {

int32_t attn_score_fwd_lse(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t d,
                           float scale, int32_t causal, const attn_score* score, const void* Q, const void* K,
                           const void* V, void* O, void* Orest, float* L, void* workspace, int64_t workspace_bytes,
                           void* stream) {
  const ScoreProblem p = fb::score_problem(dtype, B, H, Hkv, Nq, Nk, d, scale, causal, score);
  bool empty;
  const int32_t rc = fb::score_check(p, &empty);
  if (rc != BOB_OK || empty || Nq == 0) return rc;
  if (!fb::score_rest(Nq, Orest) || !fb::ext_ptrs(Nq, {Q, O, L}) || !fb::ext_ptrs(Nk, {K, V})) return BOB_EINVAL;
  if (!fb::workspace_fits(fb::call_bytes(ATTN_SCORE_FWD, p), workspace, workspace_bytes)) return BOB_EINVAL;
  return fb::go_fwd(p, Q, K, V, O, Orest, L, (float*)workspace, (hipStream_t)stream);
}

int32_t attn_score_bwd(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t d,
                       float scale, int32_t causal, const attn_score* score, const void* Q, const void* K,
                       const void* V, const void* O, const void* Orest, const void* dO, const float* L, void* dQ,
                       void* dK, void* dV, float* D, void* workspace, int64_t workspace_bytes, void* stream) {
  const ScoreProblem p = fb::score_problem(dtype, B, H, Hkv, Nq, Nk, d, scale, causal, score);
  bool empty;
  const int32_t rc = fb::score_check(p, &empty);
  if (rc != BOB_OK || empty) return rc;
  if (!fb::score_rest(Nq, Orest) || !fb::ext_ptrs(Nq, {Q, O, dO, L, dQ, D}) || !fb::ext_ptrs(Nk, {K, V, dK, dV}))
    return BOB_EINVAL;
  if (!fb::workspace_fits(fb::call_bytes(ATTN_SCORE_BWD, p), workspace, workspace_bytes)) return BOB_EINVAL;
  char* const ws = (char*)workspace;
  return fb::go_bwd(p, Q, K, V, O, Orest, dO, L, dQ, dK, dV, D, (float*)ws, (float*)(ws + fb::rows_bytes(p)),
                    (hipStream_t)stream);
}

int32_t attn_score_pass1_rows(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t d,
                              float scale, int32_t causal, const attn_score* score, const void* Q, const void* K,
                              const void* V, const void* O, const void* Orest, const void* dO, const void* gdQ,
                              const void* gdK, const void* gdV, const float* L, const float* D, const void* dQ,
                              void* Qt, void* dOt, float* alpha, float* E, void* workspace, int64_t workspace_bytes,
                              void* stream) {
  const ScoreProblem p = fb::score_problem(dtype, B, H, Hkv, Nq, Nk, d, scale, causal, score);
  bool empty;
  const int32_t rc = fb::score_check(p, &empty);
  if (rc != BOB_OK || empty || Nq == 0) return rc;
  if (!fb::score_rest(Nq, Orest) || !fb::ext_ptrs(Nq, {Q, O, dO, gdQ, L, D, dQ, Qt, dOt, alpha, E}) ||
      !fb::ext_ptrs(Nk, {K, V, gdK, gdV}))
    return BOB_EINVAL;
  if (!fb::workspace_fits(fb::call_bytes(ATTN_SCORE_PASS1, p), workspace, workspace_bytes)) return BOB_EINVAL;
  return fb::go_pass1(p, Q, K, V, O, Orest, dO, gdQ, gdK, gdV, L, D, dQ, Qt, dOt, alpha, E, (float*)workspace,
                      (hipStream_t)stream);
}

int32_t attn_score_pass2_cols(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t d,
                              float scale, int32_t causal, const attn_score* score, const void* Q, const void* K,
                              const void* V, const void* dO, const void* gdQ, const void* gdK, const void* gdV,
                              const float* L, const float* D, const float* alpha, const float* E, void* Kt, void* Vt,
                              void* workspace, int64_t workspace_bytes, void* stream) {
  const ScoreProblem p = fb::score_problem(dtype, B, H, Hkv, Nq, Nk, d, scale, causal, score);
  bool empty;
  const int32_t rc = fb::score_check(p, &empty);
  if (rc != BOB_OK || empty || Nk == 0) return rc;
  if (!fb::ext_ptrs(Nq, {Q, dO, gdQ, L, D, alpha, E}) || !fb::ext_ptrs(Nk, {K, V, gdK, gdV, Kt, Vt}))
    return BOB_EINVAL;
  if (!fb::workspace_fits(fb::call_bytes(ATTN_SCORE_PASS2, p), workspace, workspace_bytes)) return BOB_EINVAL;
  return fb::go_pass2(p, Q, K, V, dO, gdQ, gdK, gdV, L, D, alpha, E, Kt, Vt, (float*)workspace, (hipStream_t)stream);
}

int64_t attn_score_workspace_bytes(int32_t call, int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq,
                                   int64_t Nk, int64_t d, int32_t causal, const attn_score* score) {
  const ScoreProblem p = fb::score_problem(dtype, B, H, Hkv, Nq, Nk, d, 1.0f, causal, score);
  bool empty;
  if (call < ATTN_SCORE_FWD || call > ATTN_SCORE_PASS2 || fb::score_check(p, &empty) != BOB_OK || empty) return 0;
  return fb::call_bytes(call, p);
}

int32_t attn_score_layout(int32_t kernel, int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk,
                          int64_t d, int32_t causal, const attn_score* score, attn_ext_launch* launch) {
  if (kernel < ATTN_EXT_FWD || kernel > ATTN_EXT_PASS2 || launch == nullptr) return BOB_EINVAL;
  const ScoreProblem p = fb::score_problem(dtype, B, H, Hkv, Nq, Nk, d, 1.0f, causal, score);
  bool empty;
  const int32_t rc = fb::score_check(p, &empty);
  if (rc != BOB_OK) return rc;
  *launch = attn_ext_launch{};
  const bool columns = kernel == ATTN_EXT_COLS || kernel == ATTN_EXT_PASS2;
  if (empty || (columns ? Nk : Nq) == 0) return BOB_OK;
  const fb::ExtPlan c = kernel == ATTN_EXT_FWD     ? fb::plan_fwd(p)
                        : kernel == ATTN_EXT_ROWS  ? fb::plan_rows(p)
                        : kernel == ATTN_EXT_COLS  ? fb::plan_cols(p)
                        : kernel == ATTN_EXT_PASS1 ? fb::plan_pass1(p)
                                                   : fb::plan_pass2(p);
  *launch = attn_ext_launch{16 * c.blocks, c.sets, c.parts, c.fold ? 1 : 0, c.resident};
  return BOB_OK;
}

}  // extern "C"
