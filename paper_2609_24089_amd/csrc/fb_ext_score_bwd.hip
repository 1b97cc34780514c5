// The first backward over capped scores, distance biases and spans: its forms and launches.
#include "fb_ext_score.h"

namespace fb {

// Whole blocks at bf16 d = 64: 16 rows a wave and five waves per SIMD on the row side, three (168
// registers) on the column side.  With 32 rows and three waves the row side of B4 H12 N4096 took,
// causal with a cap, 287 us for 277, and under packed documents 74 for 63; the forward (151 for 147
// us) and the column side (271 for 232) were slower with 16.
template <typename T, int D> constexpr bool kNarrowHeads = std::is_same_v<T, bf16> && D == 64;

template <typename T, int D> struct ScoreRowsBwd {
  static constexpr ExtShape shape(int form, bool capped) {
    constexpr Shape w = Cfg<T, D>::kRows;
    return form == 0   ? kNarrowHeads<T, D> ? ExtShape{1, 4, 4, 1} : ExtShape{w.mr, w.nw, w.occ, 1}
           : form == 4 ? ext_two_sets<T, D>(w, 2, 0)
                       : ext_sets<T, D>(kFormWaves[form], 2, 0, 16, w.occ);
  }
  template <int F, bool kCap> static __host__ constexpr auto kernel() {
    constexpr ExtShape s = shape(F, kCap);
    return &score_bwd_rows_kernel<T, D, s.mr, s.nw, s.occ, s.ks, kCap>;
  }
};

template <typename T, int D> struct ScoreColsBwd {
  static constexpr int kExtra = 4 * 2 * kBS * (int)sizeof(float) + 1024;  // raw and transformed L, D; slopes
  static constexpr ExtShape shape(int form, bool capped) {
    constexpr Shape w = Cfg<T, D>::kCols;
    constexpr int waves = D * (int)sizeof(T) <= 128 ? 16 : 8;
    return form == 0   ? ExtShape{w.mr, w.nw, kNarrowHeads<T, D> ? 3 : w.occ, 1}
           : form == 4 ? ext_two_sets<T, D>(w, 2, 2 * kExtra + (w.kl ? 4 * Geo<T, D>::kTileElems * (int)sizeof(T) : 0))
           : form == 1 && D == 256
               ? kNotBuilt  // spilled 127 registers
               : ext_sets<T, D>(kFormWaves[form], 2, kExtra, waves, w.occ);
  }
  template <int F, bool kCap> static __host__ constexpr auto kernel() {
    constexpr ExtShape s = shape(F, kCap);
    return &score_bwd_cols_kernel<T, D, s.mr, s.nw, s.occ, s.ks, (F == 0 || F == 4) && Cfg<T, D>::kCols.kl != 0, kCap>;
  }
};

template <typename T, int D> ExtPlan score_rows_plan(const ScoreProblem& p) {
  ExtPlan c;
  const FormQuery q{device_cus(), p.B * p.H, std::max<int64_t>(p.Nq, 1), std::max<int64_t>((p.Nk + kBS - 1) / kBS, 1),
                    triangular(p), block_us<T>(3, D), kRowsStep<T>, merge_us(1, D), kRowMargin};
  ext_pick<ScoreRowsBwd<T, D>>(p, q, kRowsStep<T>.narrow, [](const ExtShape&) { return int64_t(0); }, kAnyForm, 1, 1,
                               p.B * p.H * p.Nq * (D + 1) * 4, &c);
  return c;
}

template <typename T, int D> ExtPlan score_cols_plan(const ScoreProblem& p) {
  const int grp = ext_group(p);
  ExtPlan c;
  const FormQuery q{device_cus(), p.B * p.Hkv, std::max<int64_t>(p.Nk, 1),
                    std::max<int64_t>((p.Nq + kBS - 1) / kBS, 1) * grp, triangular(p), block_us<T>(4, D), kColsStep<T>,
                    merge_us(2, D), 1.0};
  ext_pick<ScoreColsBwd<T, D>>(p, q, kColsStep<T>.narrow, [&](const ExtShape&) { return score_cols_lds(p); }, kAnyForm,
                               1, grp, 2 * p.B * p.Hkv * p.Nk * D * 4, &c, kLongChain);
  return c;
}

template <typename T, int D>
int32_t score_launch_bwd(const ScoreProblem& p, const void* Q, const void* K, const void* V, const void* O,
                         const void* Orest, const void* dO, const float* L, void* dQ, void* dK, void* dV, float* Dv,
                         float* row_parts, float* parts, hipStream_t s) {
  int32_t rc = BOB_OK;
  if (p.Nq > 0) {
    const ExtPlan r = score_rows_plan<T, D>(p);
    const ScoreArgs a = score_args<T>(p, r, p.B * p.H, p.Nq);
    rc = ext_dispatch<ScoreRowsBwd<T, D>>(r.form, p, dim3(a.total, r.parts), 0, s, a, (const T*)Q, (const T*)K,
                                          (const T*)V, (const T*)O, (const T*)Orest, (const T*)dO, L, (T*)dQ, Dv,
                                          row_parts);
    if (rc == BOB_OK && r.parts > 1) rc = ext_join_bwd<T, D>(a, row_parts, p.B * p.H * p.Nq, dQ, Dv, s);
  }
  if (rc != BOB_OK || p.Nk == 0) return rc;
  const ExtPlan c = score_cols_plan<T, D>(p);
  return ext_launch_columns(p, c, score_args<T>(p, c, p.B * p.Hkv, p.Nk), parts, dK, dV, s,
                            [&](const ScoreArgs& a, dim3 grid) {
                              return ext_dispatch<ScoreColsBwd<T, D>>(c.form, p, grid, score_cols_lds(p), s, a,
                                                                      (const T*)Q, (const T*)K, (const T*)V,
                                                                      (const T*)dO, L, (const float*)Dv, (T*)dK,
                                                                      (T*)dV, parts);
                            });
}

#define FB_INST(T, D, ...)                                                                                         \
  template ExtPlan score_rows_plan<T, D>(const ScoreProblem&);                                                     \
  template ExtPlan score_cols_plan<T, D>(const ScoreProblem&);                                                     \
  template int32_t score_launch_bwd<T, D>(const ScoreProblem&, const void*, const void*, const void*, const void*, \
                                          const void*, const void*, const float*, void*, void*, void*, float*, float*,     \
                                          float*, hipStream_t);
FB_EXT_EACH(FB_INST)

}  // namespace fb
