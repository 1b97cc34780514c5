// The two BoB passes over capped scores, distance biases and spans: their forms and launches,
// for the translation units that build them.
#pragma once
#include "fb_ext_score.h"

namespace fb {

template <typename T, int D> struct ScorePass1 {
  static constexpr ExtShape shape(int form, bool capped) {
    constexpr Shape w = Cfg<T, D>::kP1;
    constexpr bool kThreeWaves = std::is_same_v<T, bf16> && D == 64;  // 168 registers
    return form == 0   ? ExtShape{w.mr, w.nw, kThreeWaves ? 3 : w.occ, 1}
           : form == 4 ? ext_two_sets<T, D>(w, 4, 0)
                       : ext_sets<T, D>(kFormWaves[form], 4, 0, 8, w.occ);
  }
  template <int F, bool kCap> static __host__ constexpr auto kernel() {
    constexpr ExtShape s = shape(F, kCap);
    // fragments read ahead (bf16 d = 128) where the registers hold them: with a cap, or in sets, they
    // spilled hundreds (B2 H16 N2048 causal with a cap: five times as long)
    constexpr int pf = F == 0 && !kCap ? Cfg<T, D>::kP1.pf : 0;
    return &score_pass1_kernel<T, D, s.mr, s.nw, s.occ, s.ks, pf, kCap>;
  }
};
template <typename T, int D> struct ScorePass2 {
  static constexpr int kExtra = 4 * 4 * kBS * (int)sizeof(float) + 1024;
  static constexpr ExtShape shape(int form, bool capped) {
    // 16 columns a wave, three waves per SIMD, where a cap's tanh spilled 63 registers of the 32
    // columns' 256 (B4 H12 N4096 causal 750 us for 520)
    constexpr bool kNarrow = std::is_same_v<T, bf16> && D == 64;
    constexpr Shape w = Cfg<T, D>::kP2;
    return form == 0   ? capped && kNarrow ? ExtShape{1, 4, 3, 1} : ExtShape{w.mr, w.nw, w.occ, 1}
           : form == 4 ? capped && kNarrow ? kNotBuilt : ext_two_sets<T, D>(w, 3, 2 * kExtra)
           : sizeof(T) == 2 && D == 32 && form == 1
               ? kNotBuilt  // three tensors of two 1 KB blocks do not deal out over four waves
               : ext_sets<T, D>(kFormWaves[form], 3, kExtra, 8, w.occ);
  }
  template <int F, bool kCap> static __host__ constexpr auto kernel() {
    constexpr ExtShape s = shape(F, kCap);
    return &score_pass2_kernel<T, D, s.mr, s.nw, s.occ, s.ks, Cfg<T, D>::kP2.pf != 0, kCap>;
  }
};

template <typename T, int D> ExtPlan score_pass1_plan(const ScoreProblem& p) {
  ExtPlan c;
  const FormQuery q{device_cus(), p.B * p.H, std::max<int64_t>(p.Nq, 1), std::max<int64_t>((p.Nk + kBS - 1) / kBS, 1),
                    triangular(p), block_us<T>(10, D), kP1Step<T>, merge_us(3, D), kRowMargin};
  ext_pick<ScorePass1<T, D>>(p, q, kP1Step<T>.narrow, [](const ExtShape&) { return int64_t(0); }, kAnyForm, 1, 1,
                             p.B * p.H * p.Nq * (3 * D + 2) * 4, &c);
  return c;
}

template <typename T, int D>
int32_t score_launch_pass1(const ScoreProblem& p, const void* Q, const void* K, const void* V, const void* O,
                           const void* Orest, const void* dO, const void* UQ, const void* UK, const void* UV,
                           const float* L, const float* Dv, const void* dQ, void* Qt, void* dOt, float* alpha,
                           float* E, float* parts, hipStream_t s) {
  const ExtPlan c = score_pass1_plan<T, D>(p);
  const ScoreArgs a = score_args<T>(p, c, p.B * p.H, p.Nq);
  const int32_t rc = ext_dispatch<ScorePass1<T, D>>(
      c.form, p, dim3(a.total, c.parts), 0, s, a, (const T*)Q, (const T*)K, (const T*)V, (const T*)O,
      (const T*)Orest, (const T*)dO, (const T*)UQ, (const T*)UK, (const T*)UV, L, Dv, (const T*)dQ, (T*)Qt, (T*)dOt,
      alpha, E, parts);
  if (rc != BOB_OK || c.parts == 1) return rc;
  const int64_t all = p.B * p.H * p.Nq;
  hipLaunchKernelGGL((score_pass1_join_kernel<T, D>), dim3((unsigned)((all * (D / 4) + 255) / 256)), dim3(256), 0, s, a,
                     (const float*)parts, all, (const T*)O, (const T*)Orest, Dv, (const T*)dQ, (T*)Qt, (T*)dOt, alpha,
                     E);
  return finish_launch();
}

template <typename T, int D> ExtPlan score_pass2_plan(const ScoreProblem& p) {
  const int grp = ext_group(p);
  ExtPlan c;
  const FormQuery q{device_cus(), p.B * p.Hkv, std::max<int64_t>(p.Nk, 1),
                    std::max<int64_t>((p.Nq + kBS - 1) / kBS, 1) * grp, triangular(p), block_us<T>(8, D), kP2Step<T>,
                    merge_us(2, D), 1.0};
  ext_pick<ScorePass2<T, D>>(p, q, kP2Step<T>.narrow, [&](const ExtShape&) { return score_cols_lds(p); }, kAnyForm, 1,
                             grp, 2 * p.B * p.Hkv * p.Nk * D * 4, &c, kLongChain);
  return c;
}

template <typename T, int D>
int32_t score_launch_pass2(const ScoreProblem& p, const void* Q, const void* K, const void* V, const void* dO,
                           const void* UQ, const void* UK, const void* UV, const float* L, const float* Dv,
                           const float* alpha, const float* E, void* Kt, void* Vt, float* parts, hipStream_t s) {
  const ExtPlan c = score_pass2_plan<T, D>(p);
  return ext_launch_columns(p, c, score_args<T>(p, c, p.B * p.Hkv, p.Nk), parts, Kt, Vt, s,
                            [&](const ScoreArgs& a, dim3 grid) {
                              return ext_dispatch<ScorePass2<T, D>>(
                                  c.form, p, grid, score_cols_lds(p), s, a, (const T*)Q, (const T*)K, (const T*)V,
                                  (const T*)dO, (const T*)UQ, (const T*)UK, (const T*)UV, L, Dv, alpha, E, (T*)Kt,
                                  (T*)Vt, parts);
                            });
}

#define FB_SCORE_PASS1(T, D, ...)                                                                                     \
  template ExtPlan score_pass1_plan<T, D>(const ScoreProblem&);                                                       \
  template int32_t score_launch_pass1<T, D>(const ScoreProblem&, const void*, const void*, const void*, const void*, \
                                            const void*, const void*, const void*, const void*, const void*,         \
                                            const float*, const float*, const void*, void*, void*, float*, float*,   \
                                            float*,                                                                  \
                                            hipStream_t);
#define FB_SCORE_PASS2(T, D, ...)                                                                                     \
  template ExtPlan score_pass2_plan<T, D>(const ScoreProblem&);                                                       \
  template int32_t score_launch_pass2<T, D>(const ScoreProblem&, const void*, const void*, const void*, const void*, \
                                            const void*, const void*, const void*, const float*, const float*,       \
                                            const float*, const float*, void*, void*, float*, hipStream_t);

}  // namespace fb
