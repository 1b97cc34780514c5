// Host side of the attention over capped scores, distance biases and spans
// (fb_ext_score_kernels.h): problem and launchers, shared by its translation units.
// fb_ext_score.hip holds the C ABI.
#pragma once
#include "fb_ext.h"
#include "fb_ext_score_kernels.h"

namespace fb {

// A column workgroup keeps the slopes of a key/value head's query heads in LDS.
constexpr int64_t kMaxSlopeGroup = 1024;

struct ScoreProblem : ExtProblem {
  const int32_t* spans;
  const float* slopes;
  float cap;  // 0: none
};
inline bool ext_variant(const ScoreProblem& p) { return p.cap > 0.f; }

template <typename T>
ScoreArgs score_args(const ScoreProblem& p, const ExtPlan& c, int64_t heads, int64_t rows) {
  ScoreArgs a{};
  static_cast<ExtArgs&>(a) = ext_args(p, c, heads, rows, nullptr);
  a.spans = p.spans;
  a.slopes = p.slopes;
  if (p.cap > 0.f) {
    a.cap_out = p.cap * kLog2e;
    a.cap_k = 2.f / p.cap;
    // x: S / c of a score of Q K^T = 1, taken into the polynomial while its powers stay in fp32
    double x = (double)p.scale / p.cap;
    a.cap_pre = std::fabs(x) >= 1e-4 && std::fabs(x) <= 1e4 ? 1.f : (float)x;
    x = a.cap_pre == 1.f ? x : 1.0;
    a.cap_in = (float)(x * kCapArg<T>);
    const bool far = p.cap > kCapMinimax;
    const double(&poly)[4] = far ? kCapTaylor : kCapPoly;
    a.cap_far = far ? 1 : 0;
    a.cap_near = (float)((far ? kCapNearFar : kCapNear) / std::fabs(x));
    for (int i = 0; i < 4; ++i) a.cap_poly[i] = (float)(poly[i] * std::pow(x, 2 * i + 1));
  }
  return a;
}
inline int64_t score_cols_lds(const ScoreProblem& p) {
  return p.slopes != nullptr ? (ext_group(p) * 4 + 15) / 16 * 16 : 0;
}

// Launches (defined per translation unit; instantiated for every (dtype, head dim)).
template <typename T, int D> ExtPlan score_fwd_plan(const ScoreProblem& p);
template <typename T, int D>
int32_t score_launch_fwd(const ScoreProblem& p, const void* Q, const void* K, const void* V, void* O, void* Orest,
                         float* L, float* ws, hipStream_t s);
template <typename T, int D> ExtPlan score_rows_plan(const ScoreProblem& p);
template <typename T, int D> ExtPlan score_cols_plan(const ScoreProblem& p);
template <typename T, int D>
int32_t score_launch_bwd(const ScoreProblem& p, const void* Q, const void* K, const void* V, const void* O,
                         const void* Orest, const void* dO, const float* L, void* dQ, void* dK, void* dV, float* Dv,
                         float* row_parts, float* parts, hipStream_t s);
template <typename T, int D> ExtPlan score_pass1_plan(const ScoreProblem& p);
template <typename T, int D>
int32_t score_launch_pass1(const ScoreProblem& p, const void* Q, const void* K, const void* V, const void* O,
                           const void* Orest, const void* dO, const void* UQ, const void* UK, const void* UV,
                           const float* L, const float* Dv, const void* dQ, void* Qt, void* dOt, float* alpha,
                           float* E, float* parts, hipStream_t s);
template <typename T, int D> ExtPlan score_pass2_plan(const ScoreProblem& p);
template <typename T, int D>
int32_t score_launch_pass2(const ScoreProblem& p, const void* Q, const void* K, const void* V, const void* dO,
                           const void* UQ, const void* UK, const void* UV, const float* L, const float* Dv,
                           const float* alpha, const float* E, void* Kt, void* Vt, float* parts, hipStream_t s);

}  // namespace fb
