// The forward between sequences of two lengths: its forms and launches.
#include "fb_ext.h"

namespace fb {

template <typename T, int D> struct ExtFwd {
  static constexpr ExtShape shape(int form, bool bias) {
    constexpr Shape w = Cfg<T, D>::kFwd;
    return form == 0   ? ExtShape{w.mr, w.nw, w.occ, 1}
           : form == 4 ? ext_two_sets<T, D>(w, 2, 0)
                       : ext_sets<T, D>(kFormWaves[form], 2, 0, 16, form == 2 ? 1 : w.occ);
  }
  template <int F, bool kBias> static __host__ constexpr auto kernel() {
    constexpr ExtShape s = shape(F, kBias);
    return &ext_fwd_kernel<T, D, s.mr, s.nw, s.occ, s.ks, kBias>;
  }
};

template <typename T, int D> ExtPlan ext_fwd_plan(const ExtProblem& p) {
  ExtPlan c;
  const int64_t steps = ext_steps_bytes(p);
  const int grp = ext_group(p);
  const auto few = [&](int64_t dynamic) { return ext_form_of<ExtFwd<T, D>, 2>(p, dynamic, 1.0).resident > 0; };
  // the query heads of a group together read each key and value once: a few rows a head
  c.fold = grp > 1 && p.Nq <= 16 && few(steps * std::min(grp, 16));
  const int64_t rows = c.fold ? grp * p.Nq : p.Nq, heads = p.B * (c.fold ? p.Hkv : p.H);
  const int64_t tiles = std::max<int64_t>((p.Nk + kBS - 1) / kBS, 1);
  const FormQuery q{device_cus(), heads, rows, tiles, triangular(p), block_us<T>(2, D), kFwdStep<T>, merge_us(1, D),
                    kRowMargin};
  const int64_t dynamic = steps * (c.fold ? std::min(grp, 16) : 1);
  ext_pick<ExtFwd<T, D>>(p, q, kFwdStep<T>.narrow, [&](const ExtShape&) { return dynamic; },
                         c.fold || (rows <= 16 && few(steps)) ? 2 : -1, 1, 1, heads * rows * (D + 2) * 4, &c);
  return c;
}

template <typename T, int D>
int32_t ext_launch_fwd(const ExtProblem& p, const void* Q, const void* K, const void* V, void* O, float* L, float* ws,
                       hipStream_t s) {
  const ExtPlan c = ext_fwd_plan<T, D>(p);
  const int64_t rows = c.fold ? ext_group(p) * p.Nq : p.Nq, heads = p.B * (c.fold ? p.Hkv : p.H);
  const ExtArgs a = ext_args(p, c, heads, rows, nullptr);
  const int64_t dynamic = ext_steps_bytes(p) * (c.fold ? std::min(ext_group(p), 16) : 1);
  int32_t rc = ext_dispatch<ExtFwd<T, D>>(c.form, p, dim3(a.total, c.parts), dynamic, s, a, (const T*)Q, (const T*)K,
                                          (const T*)V, (T*)O, L, ws);
  if (rc != BOB_OK || c.parts == 1) return rc;
  const int64_t all = heads * rows;
  hipLaunchKernelGGL((ext_fwd_join_kernel<T, D>), dim3((unsigned)((all * (D / 4) + 255) / 256)), dim3(256), 0, s, a,
                     (const float*)ws, all, (T*)O, L);
  return finish_launch();
}

#define FB_INST(T, D, ...)                                  \
  template ExtPlan ext_fwd_plan<T, D>(const ExtProblem&);   \
  template int32_t ext_launch_fwd<T, D>(const ExtProblem&, const void*, const void*, const void*, void*, float*, float*, \
                                        hipStream_t);
FB_EXT_EACH(FB_INST)

}  // namespace fb
