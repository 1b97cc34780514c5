// The first backward between sequences of two lengths: its forms and launches.
#include "fb_ext.h"

namespace fb {

template <typename T, int D> struct ExtRowsBwd {
  static constexpr ExtShape shape(int form, bool bias) {
    constexpr Shape w = Cfg<T, D>::kRows;
    return form == 0   ? ExtShape{w.mr, w.nw, w.occ, 1}
           : form == 4 ? ext_two_sets<T, D>(w, 2, 0)
                       : ext_sets<T, D>(kFormWaves[form], 2, 0, 16, w.occ);
  }
  template <int F, bool kBias> static __host__ constexpr auto kernel() {
    constexpr ExtShape s = shape(F, kBias);
    return &ext_bwd_rows_kernel<T, D, s.mr, s.nw, s.occ, s.ks, kBias>;
  }
};

template <typename T, int D> struct ExtColsBwd {
  static constexpr int kExtra = 4 * 2 * kBS * (int)sizeof(float) + 1024;  // raw and transformed L, D; bias buffers
  static constexpr ExtShape shape(int form, bool bias) {
    constexpr Shape w = Cfg<T, D>::kCols;
    constexpr int waves = D * (int)sizeof(T) <= 128 ? 16 : 8;
    // three waves per SIMD for some spills beside the near tiles: 814 us for 881 with two at
    // B4 H12 N4096 dense, 462 for 485 causal (first backward)
    constexpr bool kThree = std::is_same_v<T, bf16> && D == 64;
    const ExtShape s =
        form == 0   ? ExtShape{w.mr, w.nw, bias && kThree ? 3 : w.occ, 1}
        : form == 4 ? ext_two_sets<T, D>(w, 2, 2 * kExtra + (w.kl ? 4 * Geo<T, D>::kTileElems * (int)sizeof(T) : 0))
                    : ext_sets<T, D>(kFormWaves[form], 2, kExtra, waves, w.occ);
    // one-wave sets that leave no room for their buffers of step sums (16 waves at bf16 d = 32)
    const int ring = 4 * Geo<T, D>::kTileElems * (int)sizeof(T) + 4 * 2 * kBS * (int)sizeof(float);
    return bias && form == 2 && s.ks * (ring + StepSums::kBufFloats * 4) > kMaxLds ? kNotBuilt : s;
  }
  template <int F, bool kBias> static __host__ constexpr auto kernel() {
    constexpr ExtShape s = shape(F, kBias);
    return &ext_bwd_cols_kernel<T, D, s.mr, s.nw, s.occ, s.ks, (F == 0 || F == 4) && Cfg<T, D>::kCols.kl != 0, kBias>;
  }
};

// Beside the bias, a buffer of step sums for every wave.
static int64_t cols_dynamic(const ExtProblem& p, const ExtShape& s) {
  return has_bias(p) ? ext_steps_bytes(p) + (int64_t)s.nw * s.ks * StepSums::kBufFloats * 4 : 0;
}

template <typename T, int D> ExtPlan ext_rows_plan(const ExtProblem& p) {
  ExtPlan c;
  const FormQuery q{device_cus(), p.B * p.H, std::max<int64_t>(p.Nq, 1), std::max<int64_t>((p.Nk + kBS - 1) / kBS, 1),
                    triangular(p), block_us<T>(3, D), kRowsStep<T>, merge_us(1, D), kRowMargin};
  const int64_t steps = ext_steps_bytes(p);
  ext_pick<ExtRowsBwd<T, D>>(p, q, kRowsStep<T>.narrow, [&](const ExtShape&) { return steps; }, kAnyForm, 1, 1,
                             p.B * p.H * p.Nq * (D + 1) * 4, &c);
  return c;
}

template <typename T, int D> ExtPlan ext_cols_plan(const ExtProblem& p) {
  using C = ExtColsBwd<T, D>;
  const int grp = ext_group(p);
  ExtPlan c;
  // with a bias each query head of a group has its own table: one part a head
  const int base = has_bias(p) ? grp : 1;
  const FormQuery q{device_cus(), p.B * p.Hkv, std::max<int64_t>(p.Nk, 1),
                    std::max<int64_t>((p.Nq + kBS - 1) / kBS, 1) * grp, triangular(p), block_us<T>(4, D), kColsStep<T>,
                    merge_us(2, D), 1.0};
  ext_pick<C>(p, q, kColsStep<T>.narrow, [&](const ExtShape& s) { return cols_dynamic(p, s); }, kAnyForm, base, grp,
              2 * p.B * p.Hkv * p.Nk * D * 4, &c, kLongChain);
  return c;
}

template <typename T, int D>
int32_t ext_launch_bwd(const ExtProblem& p, const void* Q, const void* K, const void* V, const void* O, const void* dO,
                       const float* L, void* dQ, void* dK, void* dV, float* Dv, float* row_parts, float* parts,
                       float* sums, hipStream_t s) {
  int32_t rc = BOB_OK;
  if (p.Nq > 0) {
    const ExtPlan r = ext_rows_plan<T, D>(p);
    const ExtArgs a = ext_args(p, r, p.B * p.H, p.Nq, nullptr);
    rc = ext_dispatch<ExtRowsBwd<T, D>>(r.form, p, dim3(a.total, r.parts), ext_steps_bytes(p), s, a, (const T*)Q,
                                        (const T*)K, (const T*)V, (const T*)O, (const T*)dO, L, (T*)dQ, Dv, row_parts);
    if (rc == BOB_OK && r.parts > 1) rc = ext_join_bwd<T, D>(a, row_parts, p.B * p.H * p.Nq, dQ, Dv, s);
  }
  if (rc != BOB_OK || p.Nk == 0) return rc;
  const ExtPlan c = ext_cols_plan<T, D>(p);
  using C = ExtColsBwd<T, D>;
  const int64_t dynamic = cols_dynamic(p, C::shape(c.form, has_bias(p)));
  return ext_launch_columns(p, c, ext_args(p, c, p.B * p.Hkv, p.Nk, nullptr), parts, dK, dV, s,
                            [&](const ExtArgs& a, dim3 grid) {
                              return ext_dispatch<C>(c.form, p, grid, dynamic, s, a, (const T*)Q, (const T*)K,
                                                     (const T*)V, (const T*)dO, L, (const float*)Dv, (T*)dK, (T*)dV,
                                                     parts, sums);
                            });
}

template <typename T, int D>
int32_t ext_join_bwd(const ExtArgs& a, const float* parts, int64_t all, void* dQ, float* Dv, hipStream_t s) {
  hipLaunchKernelGGL((ext_bwd_join_kernel<T, D>), dim3((unsigned)((all * (D / 4) + 255) / 256)), dim3(256), 0, s, a,
                     parts, all, (T*)dQ, Dv);
  return finish_launch();
}

#define FB_INST(T, D, ...)                                                                                        \
  template ExtPlan ext_rows_plan<T, D>(const ExtProblem&);                                                        \
  template ExtPlan ext_cols_plan<T, D>(const ExtProblem&);                                                        \
  template int32_t ext_launch_bwd<T, D>(const ExtProblem&, const void*, const void*, const void*, const void*,    \
                                        const void*, const float*, void*, void*, void*, float*, float*, float*,   \
                                        float*,                                                                   \
                                        hipStream_t);                                                             \
  template int32_t ext_join_bwd<T, D>(const ExtArgs&, const float*, int64_t, void*, float*, hipStream_t);
FB_EXT_EACH(FB_INST)

}  // namespace fb
