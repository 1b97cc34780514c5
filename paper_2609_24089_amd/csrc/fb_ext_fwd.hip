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

// The tables by steps of a block's heads: folded, at most every one of the group that its
// rows touch.
static int64_t fwd_dynamic(const ExtProblem& p, const ExtShape& s, bool fold) {
  const int64_t heads = fold ? std::min<int64_t>(ext_group(p), (16 * s.blocks() - 2) / p.Nq + 2) : 1;
  return ext_steps_bytes(p) * heads;
}

// A few query rows of a group's heads are one matrix (fold), so that each key and value is
// read once for all of them.  A lane's rows then have positions up to kFoldRows apart, which
// the steps kept beyond R allow for.  Measured (us), folded / not, bf16 B32 H32 Hkv8 d128
// against 4096 keys: 1 row 101 / 184, 16 rows 107 / 185, 32 rows 142 / 248; where the keys stay
// in the caches, as B16 H16 Hkv8 d64, 32 rows, 2048 keys: 16.5 / 15.4.
constexpr int kFoldRows = 32;
static_assert(kFoldRows - 1 + kBS - 1 < kStepPad, "steps of a near tile");
template <typename T, int D> ExtPlan ext_fwd_plan(const ExtProblem& p) {
  ExtPlan c;
  const int grp = ext_group(p);
  int64_t rows, heads;
  // whether the one-wave form takes it: the tables of a block's heads fit, and a grid of 1024
  // threads a block at most
  const auto few = [&](bool fold) {
    c.fold = fold;
    rows = fold ? grp * p.Nq : p.Nq;
    heads = p.B * (fold ? p.Hkv : p.H);
    return heads * ((rows + 15) / 16) <= UINT32_MAX / 1024 &&
           ext_form_of<ExtFwd<T, D>, 2>(p, fwd_dynamic(p, ExtFwd<T, D>::shape(2, has_bias(p)), fold), 1.0).resident > 0;
  };
  const bool fits = (grp > 1 && p.Nq <= kFoldRows && few(true)) || few(false);
  const int64_t tiles = std::max<int64_t>((p.Nk + kBS - 1) / kBS, 1);
  const FormQuery q{device_cus(), heads, rows, tiles, triangular(p), block_us<T>(2, D), kFwdStep<T>, merge_us(1, D),
                    kRowMargin};
  // Bits of the forms to choose from.  16 rows or fewer: one wave a set, each on its own
  // (against the estimate's choice 7.1 / 7.3 us on 700 keys, the same on long ones).  More
  // folded rows: the forms of one 16-row block a wave (in the one-wave form, whose blocks
  // each read the keys, 64 rows of the first figures' grid took 182 us for 108).
  const unsigned forms = rows <= 16 && fits ? 1u << 2 : c.fold ? 1u << 1 | 1u << 2 | 1u << 3 : kAnyForm;
  ext_pick<ExtFwd<T, D>>(p, q, kFwdStep<T>.narrow, [&](const ExtShape& s) { return fwd_dynamic(p, s, c.fold); }, forms,
                         1, 1, heads * rows * (D + 2) * 4, &c);
  return c;
}

template <typename T, int D>
int32_t ext_launch_fwd(const ExtProblem& p, const void* Q, const void* K, const void* V, void* O, float* L, float* ws,
                       hipStream_t s) {
  const ExtPlan c = ext_fwd_plan<T, D>(p);
  const int64_t rows = c.fold ? ext_group(p) * p.Nq : p.Nq, heads = p.B * (c.fold ? p.Hkv : p.H);
  const ExtArgs a = ext_args(p, c, heads, rows, nullptr);
  const int64_t dynamic = fwd_dynamic(p, ExtFwd<T, D>::shape(c.form, has_bias(p)), c.fold);
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
