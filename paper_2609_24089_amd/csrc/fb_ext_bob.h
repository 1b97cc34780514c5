// The two BoB passes between sequences of two lengths: their forms and launches, for the
// translation units that build them.
#pragma once
#include "fb_ext.h"

namespace fb {

template <typename T, int D> struct ExtPass1 {
  static constexpr ExtShape shape(int form, bool bias) {
    constexpr Shape w = Cfg<T, D>::kP1;
    return form == 0   ? ExtShape{w.mr, w.nw, w.occ, 1}
           : form == 4 ? ext_two_sets<T, D>(w, 4, 0)
                       : ext_sets<T, D>(kFormWaves[form], 4, 0, 8, w.occ);
  }
  template <int F, bool kBias> static __host__ constexpr auto kernel() {
    constexpr ExtShape s = shape(F, kBias);
    return &ext_pass1_kernel<T, D, s.mr, s.nw, s.occ, s.ks, Cfg<T, D>::kP1.pf, kBias>;
  }
};
template <typename T, int D> struct ExtPass2 {
  static constexpr int kExtra = 4 * 4 * kBS * (int)sizeof(float) + 1024;
  static constexpr ExtShape shape(int form, bool bias) {
    constexpr Shape w = Cfg<T, D>::kP2;
    return form == 0   ? ExtShape{w.mr, w.nw, w.occ, 1}
           : form == 4 ? ext_two_sets<T, D>(w, 3, 2 * kExtra)
           : sizeof(T) == 2 && D == 32 && form == 1
               ? kNotBuilt  // three tensors of two 1 KB blocks do not deal out over four waves
               : ext_sets<T, D>(kFormWaves[form], 3, kExtra, 8, w.occ);
  }
  template <int F, bool kBias> static __host__ constexpr auto kernel() {
    constexpr ExtShape s = shape(F, kBias);
    return &ext_pass2_kernel<T, D, s.mr, s.nw, s.occ, s.ks, Cfg<T, D>::kP2.pf != 0, kBias>;
  }
};

inline int64_t pass2_dynamic(const ExtProblem& p, const ExtShape& s) {
  return has_bias(p) ? 2 * ext_steps_bytes(p) + (int64_t)s.nw * s.ks * StepSums::kBufFloats * 4 : 0;
}

template <typename T, int D> ExtPlan ext_pass1_plan(const ExtProblem& p) {
  ExtPlan c;
  const FormQuery q{device_cus(), p.B * p.H, std::max<int64_t>(p.Nq, 1), std::max<int64_t>((p.Nk + kBS - 1) / kBS, 1),
                    triangular(p), block_us<T>(10, D), kP1Step<T>, merge_us(3, D), kRowMargin};
  const int64_t steps = 2 * ext_steps_bytes(p);
  ext_pick<ExtPass1<T, D>>(p, q, kP1Step<T>.narrow, [&](const ExtShape&) { return steps; }, kAnyForm, 1, 1,
                           p.B * p.H * p.Nq * (3 * D + 4) * 4, &c);
  return c;
}

template <typename T, int D>
int32_t ext_launch_pass1(const ExtProblem& p, const void* Q, const void* K, const void* V, const void* O,
                         const void* dO, const void* UQ, const void* UK, const void* UV, const void* UT,
                         const float* L, const float* Dv, const void* dQ, void* Qt, void* dOt, float* alpha, float* E,
                         float* parts, hipStream_t s) {
  const ExtPlan c = ext_pass1_plan<T, D>(p);
  const ExtArgs a = ext_args(p, c, p.B * p.H, p.Nq, UT);
  const int32_t rc = ext_dispatch<ExtPass1<T, D>>(
      c.form, p, dim3(a.total, c.parts), 2 * ext_steps_bytes(p), s, a, (const T*)Q, (const T*)K, (const T*)V,
      (const T*)O, (const T*)dO, (const T*)UQ, (const T*)UK, (const T*)UV, L, Dv, (const T*)dQ, (T*)Qt, (T*)dOt, alpha,
      E, parts);
  if (rc != BOB_OK || c.parts == 1) return rc;
  const int64_t all = p.B * p.H * p.Nq;
  hipLaunchKernelGGL((ext_pass1_join_kernel<T, D>), dim3((unsigned)((all * (D / 4) + 255) / 256)), dim3(256), 0, s, a,
                     (const float*)parts, all, (const T*)O, Dv, (const T*)dQ, (T*)Qt, (T*)dOt, alpha, E);
  return finish_launch();
}

template <typename T, int D> ExtPlan ext_pass2_plan(const ExtProblem& p) {
  using C = ExtPass2<T, D>;
  const int grp = ext_group(p);
  ExtPlan c;
  const int base = has_bias(p) ? grp : 1;
  const FormQuery q{device_cus(), p.B * p.Hkv, std::max<int64_t>(p.Nk, 1),
                    std::max<int64_t>((p.Nq + kBS - 1) / kBS, 1) * grp, triangular(p), block_us<T>(8, D), kP2Step<T>,
                    merge_us(2, D), 1.0};
  ext_pick<C>(p, q, kP2Step<T>.narrow, [&](const ExtShape& s) { return pass2_dynamic(p, s); }, kAnyForm, base, grp,
              2 * p.B * p.Hkv * p.Nk * D * 4, &c, kLongChain);
  return c;
}

template <typename T, int D>
int32_t ext_launch_pass2(const ExtProblem& p, const void* Q, const void* K, const void* V, const void* dO,
                         const void* UQ, const void* UK, const void* UV, const void* UT, const float* L,
                         const float* Dv, const float* alpha, const float* E, void* Kt, void* Vt, float* parts,
                         float* sums, hipStream_t s) {
  using C = ExtPass2<T, D>;
  const ExtPlan c = ext_pass2_plan<T, D>(p);
  const int64_t dynamic = pass2_dynamic(p, C::shape(c.form, has_bias(p)));
  return ext_launch_columns(p, c, ext_args(p, c, p.B * p.Hkv, p.Nk, UT), parts, Kt, Vt, s,
                            [&](const ExtArgs& a, dim3 grid) {
                              return ext_dispatch<C>(c.form, p, grid, dynamic, s, a, (const T*)Q, (const T*)K,
                                                     (const T*)V, (const T*)dO, (const T*)UQ, (const T*)UK,
                                                     (const T*)UV, L, Dv, alpha, E, (T*)Kt, (T*)Vt, parts, sums);
                            });
}

#define FB_EXT_PASS1(T, D, ...)                                                                                      \
  template ExtPlan ext_pass1_plan<T, D>(const ExtProblem&);                                                          \
  template int32_t ext_launch_pass1<T, D>(const ExtProblem&, const void*, const void*, const void*, const void*,    \
                                          const void*, const void*, const void*, const void*, const void*,          \
                                          const float*, const float*, const void*, void*, void*, float*, float*,    \
                                          float*, hipStream_t);
#define FB_EXT_PASS2(T, D, ...)                                                                                     \
  template ExtPlan ext_pass2_plan<T, D>(const ExtProblem&);                                                         \
  template int32_t ext_launch_pass2<T, D>(const ExtProblem&, const void*, const void*, const void*, const void*,    \
                                          const void*, const void*, const void*, const void*, const float*,         \
                                          const float*, const float*, const float*, void*, void*, float*, float*,   \
                                          hipStream_t);

}  // namespace fb
