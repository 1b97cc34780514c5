// The forward over capped scores, distance biases and spans: its forms and launches.
#include "fb_ext_score.h"

namespace fb {

template <typename T, int D> struct ScoreFwd {
  static constexpr ExtShape shape(int form, bool capped) {
    constexpr Shape w = Cfg<T, D>::kFwd;
    return form == 0   ? ExtShape{w.mr, w.nw, w.occ, 1}
           : form == 4 ? ext_two_sets<T, D>(w, 2, 0)
                       : ext_sets<T, D>(kFormWaves[form], 2, 0, 16, form == 2 ? 1 : w.occ);
  }
  template <int F, bool kCap> static __host__ constexpr auto kernel() {
    constexpr ExtShape s = shape(F, kCap);
    return &score_fwd_kernel<T, D, s.mr, s.nw, s.occ, s.ks, kCap>;
  }
};

// As ext_fwd_plan: a few query rows of a group's heads are one matrix, and 16 rows or fewer run
// one wave a set.
constexpr int kScoreFoldRows = 32;
template <typename T, int D> ExtPlan score_fwd_plan(const ScoreProblem& p) {
  ExtPlan c;
  const int grp = ext_group(p);
  int64_t rows, heads;
  const auto few = [&](bool fold) {
    c.fold = fold;
    rows = fold ? grp * p.Nq : p.Nq;
    heads = p.B * (fold ? p.Hkv : p.H);
    return heads * ((rows + 15) / 16) <= UINT32_MAX / 1024 && ext_form_of<ScoreFwd<T, D>, 2>(p, 0, 1.0).resident > 0;
  };
  const bool fits = (grp > 1 && p.Nq <= kScoreFoldRows && few(true)) || few(false);
  const int64_t tiles = std::max<int64_t>((p.Nk + kBS - 1) / kBS, 1);
  const FormQuery q{device_cus(), heads, rows, tiles, triangular(p), block_us<T>(2, D), kFwdStep<T>, merge_us(1, D),
                    kRowMargin};
  const unsigned forms = rows <= 16 && fits ? 1u << 2 : c.fold ? 1u << 1 | 1u << 2 | 1u << 3 : kAnyForm;
  ext_pick<ScoreFwd<T, D>>(p, q, kFwdStep<T>.narrow, [](const ExtShape&) { return int64_t(0); }, forms, 1, 1,
                           heads * rows * (D + kFwdScalars) * 4, &c);
  return c;
}

template <typename T, int D>
int32_t score_launch_fwd(const ScoreProblem& p, const void* Q, const void* K, const void* V, void* O, void* Orest,
                         float* L, float* ws, hipStream_t s) {
  const ExtPlan c = score_fwd_plan<T, D>(p);
  const int64_t rows = c.fold ? ext_group(p) * p.Nq : p.Nq, heads = p.B * (c.fold ? p.Hkv : p.H);
  const ScoreArgs a = score_args<T>(p, c, heads, rows);
  const int32_t rc = ext_dispatch<ScoreFwd<T, D>>(c.form, p, dim3(a.total, c.parts), 0, s, a, (const T*)Q, (const T*)K,
                                                  (const T*)V, (T*)O, (T*)Orest, L, ws);
  if (rc != BOB_OK || c.parts == 1) return rc;
  const int64_t all = heads * rows;
  hipLaunchKernelGGL((score_fwd_join_kernel<T, D>), dim3((unsigned)((all * (D / 4) + 255) / 256)), dim3(256), 0, s, a,
                     (const float*)ws, all, (T*)O, (T*)Orest, L);
  return finish_launch();
}

#define FB_INST(T, D, ...)                                                                                       \
  template ExtPlan score_fwd_plan<T, D>(const ScoreProblem&);                                                    \
  template int32_t score_launch_fwd<T, D>(const ScoreProblem&, const void*, const void*, const void*, void*,     \
                                          void*, float*, float*, hipStream_t);
FB_EXT_EACH(FB_INST)

}  // namespace fb
