// Host side of the attention between sequences of two lengths (fb_ext_kernels.h): problem,
// validation, launch forms and the per-(dtype, head dim) launchers, shared by its
// translation units.  fb_ext.hip holds the C ABI.
#pragma once
#include "fb_ext_kernels.h"
#include "fb_launch.h"

namespace fb {

constexpr int kMaxDistance = 1024;     // R: two tables of 2 (R + 64) + 1 floats beside the largest rings
constexpr int kMaxBuckets = 1 << 16;
constexpr int64_t kMaxLds = 160 * 1024;

struct ExtProblem {
  int32_t dtype;
  int64_t B, H, Hkv, Nq, Nk, d;
  float scale;
  int32_t causal;
  attn_ext x;   // zeros where the caller gave none
};
inline bool has_bias(const ExtProblem& p) { return p.x.table != nullptr; }
inline int ext_group(const ExtProblem& p) { return (int)(p.H / p.Hkv); }
inline int64_t ext_width(const ExtProblem& p) { return 2 * (int64_t)p.x.max_distance + 3; }

// How a launch runs: blocks of 16 `blocks` stationary rows, `sets` wave sets, `parts`
// workgroups a block; folded rows (row kernels).
struct ExtPlan {
  int form = 0, blocks = 4, sets = 1, waves = 4, parts = 1;
  int resident = 0;  // workgroups a compute unit, as the estimate takes them
  bool fold = false;
};

inline ExtArgs ext_args(const ExtProblem& p, const ExtPlan& c, int64_t heads, int64_t rows, const void* dir) {
  ExtArgs a{};
  a.H = (int)p.H;
  a.grp = ext_group(p);
  a.Nq = (int)p.Nq;
  a.Nk = (int)p.Nk;
  a.nRB = (int)((rows + 16 * c.blocks - 1) / (16 * c.blocks));
  a.total = a.blocks = (int)(heads * a.nRB);
  a.causal = p.causal;
  a.fold = c.fold ? 1 : 0;
  a.scale = p.scale;
  a.nparts = c.parts;
  a.q_lens = p.x.q_lens;
  a.kv_lens = p.x.kv_lens;
  a.q_starts = p.x.q_starts;
  a.table = p.x.table;
  a.dir = dir;
  a.buckets = p.x.buckets;
  a.table_bf16 = p.x.table_dtype == BOB_BF16 ? 1 : 0;
  a.num_buckets = p.x.num_buckets;
  a.R = p.x.max_distance;
  return a;
}

// LDS of the bias tables, in bytes.
inline int64_t ext_steps_bytes(const ExtProblem& p) {
  return has_bias(p) ? 4 * ((2 * (int64_t)(p.x.max_distance + kStepPad) + 1 + 3) / 4 * 4) : 0;
}

// Launches (defined per translation unit; instantiated for every (dtype, head dim)).
template <typename T, int D> ExtPlan ext_fwd_plan(const ExtProblem& p);
template <typename T, int D>
int32_t ext_launch_fwd(const ExtProblem& p, const void* Q, const void* K, const void* V, void* O, float* L, float* ws,
                       hipStream_t s);
template <typename T, int D> ExtPlan ext_rows_plan(const ExtProblem& p);
template <typename T, int D> ExtPlan ext_cols_plan(const ExtProblem& p);
template <typename T, int D>
int32_t ext_launch_bwd(const ExtProblem& p, const void* Q, const void* K, const void* V, const void* O, const void* dO,
                       const float* L, void* dQ, void* dK, void* dV, float* Dv, float* row_parts, float* parts, float* sums,
                       hipStream_t s);
template <typename T, int D> ExtPlan ext_pass1_plan(const ExtProblem& p);
template <typename T, int D>
int32_t ext_launch_pass1(const ExtProblem& p, const void* Q, const void* K, const void* V, const void* O,
                         const void* dO, const void* UQ, const void* UK, const void* UV, const void* UT,
                         const float* L, const float* Dv, const void* dQ, void* Qt, void* dOt, float* alpha, float* E,
                         float* parts, hipStream_t s);
template <typename T, int D> ExtPlan ext_pass2_plan(const ExtProblem& p);
template <typename T, int D>
int32_t ext_launch_pass2(const ExtProblem& p, const void* Q, const void* K, const void* V, const void* dO,
                         const void* UQ, const void* UK, const void* UV, const void* UT, const float* L,
                         const float* Dv, const float* alpha, const float* E, void* Kt, void* Vt, float* parts,
                         float* sums, hipStream_t s);
#define FB_EXT_EACH(M, ...) \
  M(bf16, 32, __VA_ARGS__) M(bf16, 64, __VA_ARGS__) M(bf16, 128, __VA_ARGS__) M(bf16, 256, __VA_ARGS__) \
  M(float, 32, __VA_ARGS__) M(float, 64, __VA_ARGS__) M(float, 128, __VA_ARGS__)

// Adds the parts of a column kernel ([nparts][2][a.rows][d]) into X and Y.
int32_t ext_add_parts(const ExtProblem& p, const ExtArgs& a, const float* parts, void* X, void* Y, hipStream_t s);

// A column kernel in parts keeps its parts' sums in at most kSliceBytes of workspace (or one
// block's, if that is more): where all blocks' would take more, it runs a slice of consecutive
// blocks at a time and adds each slice's parts before the next.  4 to 8 thousand workgroups a
// slice, ten rounds and more, so that a slice's last round costs a few percent of it.  Without
// slices bf16 B4 H64 Hkv8 N32768 d128 with a bias, whose heads of a group have a part each,
// took 8.6 GB beside outputs of 0.5.
constexpr int64_t kSliceBytes = int64_t(512) << 20;
struct ExtSlices {
  int64_t blocks, rows;  // of a slice, the last one's may be fewer
};
inline ExtSlices ext_slices(const ExtProblem& p, const ExtPlan& c) {
  const int64_t all = p.B * p.Hkv * p.Nk, blocks = p.B * p.Hkv * ((p.Nk + 16 * c.blocks - 1) / (16 * c.blocks));
  const int64_t row_bytes = (int64_t)c.parts * 2 * p.d * 4, block_rows = std::min<int64_t>(16 * c.blocks, p.Nk);
  if (c.parts == 1 || all * row_bytes <= kSliceBytes) return {blocks, all};
  const int64_t most = std::max<int64_t>(1, kSliceBytes / (block_rows * row_bytes)), count = (blocks + most - 1) / most;
  const int64_t each = (blocks + count - 1) / count;
  return {each, std::min(each * block_rows, all)};
}

// Runs launch(a, grid) for every slice of the column kernel's blocks, and adds its parts.
template <typename Launch>
int32_t ext_launch_columns(const ExtProblem& p, const ExtPlan& c, ExtArgs a, float* parts, void* X, void* Y,
                           hipStream_t s, Launch&& launch) {
  const int64_t each = ext_slices(p, c).blocks;
  auto row = [&](int64_t block) { return block / a.nRB * p.Nk + block % a.nRB * (16 * c.blocks); };
  for (int64_t first = 0; first < a.total; first += each) {
    a.block0 = (int)first;
    a.blocks = (int)std::min<int64_t>(each, a.total - first);
    a.row0 = a.blocks < a.total ? row(first) : 0;
    a.rows = a.blocks < a.total ? row(first + a.blocks) - a.row0 : p.B * p.Hkv * p.Nk;
    int32_t rc = launch(a, dim3(a.blocks, c.parts));
    if (rc == BOB_OK && c.parts > 1) rc = ext_add_parts(p, a, parts, X, Y, s);
    if (rc != BOB_OK) return rc;
  }
  return BOB_OK;
}

// A kernel's LDS beside its dynamic part, as the runtime tells it, and 1 (0: it does not tell).
template <auto kKernel> int64_t static_lds() {
  static std::atomic<int> known;
  return read_once(known, [] {
    hipFuncAttributes at;
    if (hipFuncGetAttributes(&at, (const void*)kKernel) != hipSuccess) return 0;
    return (int)at.sharedSizeBytes + 1;  // 0 is read again
  });
}

// Workgroups of kKernel that fit one CU with `dynamic` bytes of LDS beside the kernel's own: the
// occupancy query knows the registers and the kernel's own LDS alone.
template <auto kKernel> int ext_resident(int threads, int64_t dynamic) {
  int n = resident_blocks<kKernel>(threads);
  if (dynamic > 0) {
    const int64_t each = std::max<int64_t>(static_lds<kKernel>(), 1) - 1 + dynamic;
    while (n > 1 && n * each > kMaxLds) --n;
  }
  return n;
}

// ---------------------------------------------------------------------------
// Kernels: whole blocks, and 64-, 32- and 16-row blocks in wave sets.
// Kern::kernel<form, bias>() names the kernel, Kern::shape(form, bias) its shape.
// ---------------------------------------------------------------------------
struct ExtShape {
  int mr, nw, occ, ks;
  constexpr int threads() const { return 64 * nw * ks; }
  constexpr int blocks() const { return mr * nw; }
  constexpr bool built() const { return mr > 0; }
};
constexpr ExtShape kNotBuilt{0, 1, 1, 1};
// Forms: 0 whole blocks, 1 to 3 blocks of this many waves of 16 rows in wave sets, 4 whole
// blocks of 32 rows a wave in two sets (with 16 rows a wave those are form 1's).
constexpr int kFormWaves[4] = {0, 4, 1, 2};
constexpr int kForms = 5;

// Sets of `tensors` streamed tensors in blocks of nw waves of 16 rows, if more than one fits.
template <typename T, int D> constexpr ExtShape ext_sets(int nw, int tensors, int extra, int max_waves, int occ) {
  const SetShape s = set_shape<T, D>(nw, tensors, extra, max_waves, 1);
  const int lds = s.ks * (2 * tensors * Geo<T, D>::kTileElems * (int)sizeof(T) + extra);
  // as many waves a SIMD as the workgroups that the LDS holds bring, `occ` at most
  const int fit = s.ks * nw * (160 * 1024 / lds) / 4;
  return s.ks > 1 ? ExtShape{1, nw, std::max({1, s.ks * nw / 4, std::min(occ, fit)}), s.ks} : kNotBuilt;
}

// Whole blocks in two wave sets, two waves per SIMD; `beside` bytes of LDS beside the rings.
template <typename T, int D> constexpr ExtShape ext_two_sets(const Shape& w, int tensors, int beside) {
  const int ring = 2 * tensors * Geo<T, D>::kTileElems * (int)sizeof(T);
  const bool fits = w.mr == 2 && w.nw == 4 && 2 * ring + beside <= 144 * 1024 &&
                    2 * ring >= w.nw * Geo<T, D>::kNB * w.mr * 1024;
  return fits ? ExtShape{w.mr, w.nw, 2, 2} : kNotBuilt;
}

template <typename Kern, int F> Form ext_form_of(const ExtProblem& p, int64_t dynamic, double narrow) {
  auto form = [&](auto bias) -> Form {
    constexpr bool kBias = decltype(bias)::value;
    constexpr ExtShape s = Kern::shape(F, kBias);
    if constexpr (s.built()) {
      if (F > 0 && static_lds<Kern::template kernel<F, kBias>()>() + dynamic > kMaxLds) return {};
      const int fit = ext_resident<Kern::template kernel<F, kBias>()>(s.threads(), kBias ? dynamic : 0);
      return {s.blocks(), s.ks, fit, s.threads(), 1, 0.0, F == 0 || F == 4 ? 1.0 : narrow};
    }
    return {};
  };
  return has_bias(p) ? form(std::true_type{}) : form(std::false_type{});
}

// Launches form F of Kern, whose first argument is a.
template <typename Kern, int F, typename... Args>
int32_t ext_go(const ExtProblem& p, dim3 grid, int64_t dynamic, hipStream_t stream, ExtArgs a, Args... args) {
  auto go = [&](auto bias) -> int32_t {
    constexpr bool kBias = decltype(bias)::value;
    constexpr ExtShape s = Kern::shape(F, kBias);
    if constexpr (s.built()) {
      constexpr auto kernel = Kern::template kernel<F, kBias>();
      a.fit = ext_resident<kernel>(s.threads(), kBias ? dynamic : 0);
      if (p.causal != 0 && grid.y == 1) a.resident = balanced_order(a.total, a.fit, device_cus());
      (void)hipGetLastError();
      hipLaunchKernelGGL(kernel, grid, dim3(s.threads()), (unsigned)(kBias ? dynamic : 0), stream, a, args...);
      return finish_launch();
    }
    return BOB_EUNSUPPORTED;
  };
  return has_bias(p) ? go(std::true_type{}) : go(std::false_type{});
}
template <typename Kern, typename... Args>
int32_t ext_dispatch(int form, const ExtProblem& p, dim3 grid, int64_t dynamic, hipStream_t stream, const ExtArgs& a,
                     Args... args) {
  if (form == 4) return ext_go<Kern, 4>(p, grid, dynamic, stream, a, args...);
  if (form == 3) return ext_go<Kern, 3>(p, grid, dynamic, stream, a, args...);
  if (form == 2) return ext_go<Kern, 2>(p, grid, dynamic, stream, a, args...);
  if (form == 1) return ext_go<Kern, 1>(p, grid, dynamic, stream, a, args...);
  return ext_go<Kern, 0>(p, grid, dynamic, stream, a, args...);
}

// The form (of the bits in `allowed`) and the parts with the least estimated time.
// dynamic(shape): its LDS of the bias; base: parts that a block has in any case (1, or a
// group's query heads); others are multiples of `unit`; part_bytes: of fp32 sums that a part
// of all blocks stores.  A part costs what its sums take to write and to read back at 4 TB/s,
// all of them the joining launch; grids of at most four rounds (causal ones, whose order
// balances them: two workgroups a compute unit) and kMaxPartBytes are offered parts of four
// tiles a set or more.  Beyond two workgroups a unit they even out the last round: bf16 B2 H24
// Hkv12, 3622 queries, 1426 keys, d64, column side 387 -> 304 us with the row side, Pass 2 429
// -> 307; Pass 1 of B1 H8, 1301 queries, 5846 keys 121 -> 96; two of 110 shapes lost a tenth.
// max_chain: tiles that one accumulator of a column kernel may sum: longer ones drift
// (SectionSums), so they are split whatever it costs, in slices of kSliceBytes.  Measured, one
// part -> chosen (us): a token against 16384 keys, bf16 B1 H16 d64 46 -> 24, B1 H32 Hkv4 d128
// 131 -> 24; fp32 B4 H8 Hkv4, 424 queries, 298 keys, d128 Hessian-vector product 617 -> 475.  On
// 110 drawn problems the choice is 1 to 4% slower than the best form and parts on average; the
// worst of 35 us and more are the forward's 1.39 and Pass 1's 1.33.
constexpr double kJoinUs = 6.0;
constexpr int64_t kMaxPartBytes = int64_t(128) << 20;
constexpr unsigned kAnyForm = (1u << kForms) - 1;
template <typename Kern, typename Dynamic>
void ext_pick(const ExtProblem& p, const FormQuery& q, double narrow, Dynamic&& dynamic, unsigned allowed, int base,
              int unit, int64_t part_bytes, ExtPlan* c, int64_t max_chain = int64_t(1) << 40) {
  const bool b = has_bias(p);
  const Form forms[kForms] = {ext_form_of<Kern, 0>(p, dynamic(Kern::shape(0, b)), 1.0),
                              ext_form_of<Kern, 1>(p, dynamic(Kern::shape(1, b)), narrow),
                              ext_form_of<Kern, 2>(p, dynamic(Kern::shape(2, b)), narrow),
                              ext_form_of<Kern, 3>(p, dynamic(Kern::shape(3, b)), narrow),
                              ext_form_of<Kern, 4>(p, dynamic(Kern::shape(4, b)), narrow)};
  double least = 0;
  bool found = false, fills = false;
  c->form = __builtin_ctz(allowed);  // an unknown device
  c->parts = base;
  for (int i = 0; i < kForms && q.cus > 0; ++i) {
    Form f = forms[i];
    if (f.resident == 0 || (allowed >> i & 1) == 0) continue;
    const int64_t blocks = q.heads * ((q.N + 16 * f.blocks - 1) / (16 * f.blocks));
    if (i == 0) fills = f.resident > 1 && blocks * base > q.cus * f.resident;
    if (i > 0 && fills) continue;
    const auto too_long = [&](int64_t parts) { return q.tiles > max_chain * f.sets * parts; };
    for (int64_t m = 0;; m = m == 0 ? 1 : 2 * m) {
      // 16 parts a unit are enough but for chains that are still too long
      if (m > 16 && !too_long(unit * (m / 2))) break;
      if (m > 0 && unit * m > 65535) break;  // a grid's second dimension
      f.parts = (int)(m == 0 ? base : unit * m);
      if (m > 0 && f.parts <= base) continue;
      const int64_t total = blocks * f.parts;
      if (too_long(f.parts)) continue;
      const int64_t most = q.cus * (q.causal ? 2 : std::max<int64_t>(2, 4 * f.resident));
      const bool few = total <= most && f.parts * part_bytes <= kMaxPartBytes && q.tiles >= (int64_t)4 * f.sets * f.parts;
      if (m > 0 && !few && !too_long(base)) break;
      // a launch takes fewer than 2^32 threads; slices of parts stay far below
      if (f.parts == 1 && (total > INT32_MAX / 16 || total * f.threads > (int64_t)UINT32_MAX)) continue;
      double t = form_us(q, f) * (f.parts > base ? 1.08 : i > 0 ? q.margin : 1.0);
      if (f.parts > 1) t += kJoinUs + 2.0 * f.parts * (double)part_bytes / 4.0e6;
      if (!found || t < least) {
        least = t;
        found = true;
        c->form = i;
        c->parts = f.parts;
      }
    }
  }
  const ExtShape s = Kern::shape(c->form, b);
  c->blocks = s.blocks();
  c->sets = s.ks;
  c->resident = q.cus > 0 ? forms[c->form].resident : 0;
  c->waves = s.ks * s.nw;
}

// A causal problem whose queries start its keys: the blocks' work grows to the diagonal.
inline bool triangular(const ExtProblem& p) { return p.causal != 0 && p.Nq == p.Nk; }

}  // namespace fb
