// Attention over capped scores, distance biases and masks by spans of positions: forward,
// first backward and the two BoB passes as gfx950 kernels.
//
// The problem is that of fb_ext_kernels.h (two lengths, valid rows of each batch entry,
// positions past a cache) with, in the place of the bias by buckets,
//   Z = c tanh(S / c) - m_h |pos_q - pos_k|,  S = tau Q K^T,  P = softmax of Z over valid keys,
// either term optional (no cap: Z takes S itself), and with the causal mask generalised to
// spans: per position p of a batch entry the keys k0 .. k1 - 1 that its query sees and the
// positions q0 .. q1 - 1 whose queries see its key.  Packed documents and prefixes are such
// masks; each side finds from the spans of its own rows which tiles of the other it meets, so
// a tile that no row sees is neither loaded nor computed.
//
// With t = tanh(S / c), u = dZ/dS = 1 - t^2 and u' = -2 t u / c the identities are those of
// the uncapped problem with dZ = P (dP - D) for its dS and F = u Fs, Fs = tau (U_Q K^T +
// Q U_K^T), but where a score's gradient meets the matrices:
//   dS = u dZ,   St = u P (Pt - E) + u' dZ Fs = P (u (Pt - E) - (2 / c) t (dP - D) F).
// The distance bias is constant, so it enters Z alone.
//
// The kernels keep the skeleton, tiles, sets, parts and folded rows of fb_ext_kernels.h.  The
// gradients of rows whose weight lies on few keys anywhere in the sequence, as in trained models,
// are differences of terms far larger than themselves, which operands rounded to bf16 do not
// carry.  So
//  * P meets V as one bf16 value: the forward divides by the sum of P as it was rounded, which
//    leaves sum r_j (v_j - O) of the roundings r_j, and also stores Orest, what O's own rounding
//    left; D = do.O and alpha O in Pass 1 take both;
//  * operands whose sums cancel, dS of dQ and those of Pass 1 that its epilogue subtracts from
//    each other, meet the matrix instructions as two bf16 values each (SplitFrag).
// With scores of standard deviation 3 that takes dQ from 2.9e-3 off to 2.0e-3, Qt from 3.2 to
// 2.1e-3 and dOt from 3.3 to 1.8e-3 of their size (a bf16 output is 1.7e-3 off by itself), also
// with a mean in the keys and values far above their spread, and makes the estimates of
// ext_bwd_rows_kernel and ext_pass1_kernel unnecessary.
#pragma once
#include "fb_ext_kernels.h"

namespace fb {

struct ScoreArgs : ExtArgs {
  const int32_t* spans;  // [B, Nk, 4]: k0, k1, q0, q1 of each position, or null: causal or dense
  const float* slopes;   // [H] or null: 0
  float cap_pre;         // what Q K^T is multiplied by first: 1, or S / c where that is very small or large
  float cap_in;          // from there to an argument of tanh for cap_tanh()
  float cap_out;         // c log2(e)
  float cap_k;           // 2 / c
  float cap_near;        // up to here the tanh is cap_poly's
  int cap_far;           // 1: a tile beyond cap_near has its elements up to it from cap_poly too
  float cap_poly[4];     // t = s (p0 + p1 s^2 + p2 s^4 + p3 s^6)
};

// ---------------------------------------------------------------------------
// The cap
// ---------------------------------------------------------------------------
// tanh of x: bf16 takes y = 2 log2(e) x, as 1 - 2 / (1 + 2^y), off by some 2^-23 of 1 (1e-5 of a
// score of c = 50: P is rounded to bf16 afterwards).  fp32 takes x and is within some 2^-23 of
// the result: the same for |x| > 0.45, the Taylor series (next term below 2^-25 of x) below.
template <typename T> __device__ __forceinline__ float cap_tanh(float s, float cap_in);
template <> __device__ __forceinline__ float cap_tanh<bf16>(float s, float cap_in) {
  return __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + fast_exp2(s * cap_in)), 1.f);
}
template <> __device__ __forceinline__ float cap_tanh<float>(float s, float cap_in) {
  const float x = s * cap_in;
  float ax = fabsf(x);
  ax = ax > 20.f ? 20.f : ax;  // tanh is 1 there; a NaN stays
  const float d = 1.f + fast_exp2(2.f * kLog2e * ax);
  float r = __builtin_amdgcn_rcpf(d);
  r = __builtin_fmaf(r, __builtin_fmaf(-d, r, 1.f), r);
  const float far = __builtin_copysignf(__builtin_fmaf(-2.f, r, 1.f), x);
  const float q = x * x;
  float p = -929569.f / 638512875.f;
  p = __builtin_fmaf(p, q, 21844.f / 6081075.f);
  p = __builtin_fmaf(p, q, -1382.f / 155925.f);
  p = __builtin_fmaf(p, q, 62.f / 2835.f);
  p = __builtin_fmaf(p, q, -17.f / 315.f);
  p = __builtin_fmaf(p, q, 2.f / 15.f);
  p = __builtin_fmaf(p, q, -1.f / 3.f);
  const float near = __builtin_fmaf(x * q, p, x);
  return ax < 0.45f ? near : far;
}
template <typename T> constexpr float kCapArg = std::is_same_v<T, bf16> ? 2.f * kLog2e : 1.f;  // of cap_in

// tanh on |x| <= kCapNear by an odd polynomial, off by 1.14e-6 at most (the least for four terms;
// 6e-5 of a score of c = 50, where P is rounded to 2^-9).  Where scores lie far below their cap whole
// tiles take it: 5 instructions an element for two transcendentals, at a quarter of the rate, and
// three others: B4 H16 Hkv8 N4096 d128 causal, standard deviation 3, caps 20 to 50: forward 340 us
// for 361, first backward 1157 for 1190, Pass 1 1658 for 1710.  Where few tiles qualify (cap 20,
// standard deviation 6) looking for them costs nothing that shows (365 for 365, 1193 for 1194).  (A
// fifth term reaches 0.9 for a sixth instruction: the training step 1497 us for 1470.)  cap_near and
// cap_poly are this in terms of Q K^T.
// Which of the two a pair's score meets goes by its wave's tile, so forward, row side and column side
// may differ in it; what either is off by, times c, has to stay below P's rounding.  Caps up to
// kCapMinimax leave 1.2e-4 of a score.  Farther ones take the Taylor series, off by 2^-24 of the
// *result* up to kCapNearFar, in every tile: beyond it the other is off by 2^-20 of the result at most.
constexpr double kCapNear = 0.65, kCapNearFar = 0.2, kCapMinimax = 100.0;
constexpr double kCapPoly[4] = {0.9999839352347103, -0.332806913691474, 0.12861559355416782, -0.03767224489906605};
constexpr double kCapTaylor[4] = {1.0, -1.0 / 3, 2.0 / 15, -17.0 / 315};
__device__ __forceinline__ float cap_series(const ScoreArgs& a, float v) {
  const float q = v * v;
  float p = __builtin_fmaf(q, a.cap_poly[3], a.cap_poly[2]);
  p = __builtin_fmaf(q, p, a.cap_poly[1]);
  return v * __builtin_fmaf(q, p, a.cap_poly[0]);
}

// t = tanh(S / c) of a tile of raw scores, which it may overwrite.
template <typename T, int A, int B>
__device__ __forceinline__ void cap_tile(const ScoreArgs& a, floatx4 (&s)[A][B], floatx4 (&t)[A][B]) {
  if (a.cap_pre != 1.f) {
#pragma unroll
    for (int x = 0; x < A; ++x)
#pragma unroll
      for (int y = 0; y < B; ++y) s[x][y] *= a.cap_pre;
  }
  if constexpr (sizeof(T) == 2) {
    float most = 0.f;
#pragma unroll
    for (int x = 0; x < A; ++x)
#pragma unroll
      for (int y = 0; y < B; ++y)
#pragma unroll
        for (int r = 0; r < 4; r += 2) most = fmaxf(most, fmaxf(fabsf(s[x][y][r]), fabsf(s[x][y][r + 1])));
    if (__builtin_amdgcn_ballot_w64(most > a.cap_near) == 0) {
#pragma unroll
      for (int x = 0; x < A; ++x)
#pragma unroll
        for (int y = 0; y < B; ++y)
#pragma unroll
          for (int r = 0; r < 4; ++r) t[x][y][r] = cap_series(a, s[x][y][r]);
      return;
    }
    if (a.cap_far != 0) {
#pragma unroll
      for (int x = 0; x < A; ++x)
#pragma unroll
        for (int y = 0; y < B; ++y)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float v = s[x][y][r];
            t[x][y][r] = fabsf(v) <= a.cap_near ? cap_series(a, v) : cap_tanh<T>(v, a.cap_in);
          }
      return;
    }
  }
#pragma unroll
  for (int x = 0; x < A; ++x)
#pragma unroll
    for (int y = 0; y < B; ++y)
#pragma unroll
      for (int r = 0; r < 4; ++r) t[x][y][r] = cap_tanh<T>(s[x][y][r], a.cap_in);
}

// ---------------------------------------------------------------------------
// Spans
// ---------------------------------------------------------------------------
struct Interval {
  int lo, hi;  // lo >= hi: empty
};
// The keys that query row `query` of entry b sees, and the query rows that key `key` is seen by.
__device__ __forceinline__ Interval score_keys(const ScoreArgs& a, const ExtLens& n, int b, int query) {
  const int pos = n.start + query;
  Interval v{0, a.causal != 0 ? min(n.k, pos + 1) : n.k};
  if (a.spans != nullptr) {
    v.hi = 0;
    if (pos >= 0 && pos < a.Nk) {
      const int32_t* const s = a.spans + 4 * ((int64_t)b * a.Nk + pos);
      v = Interval{max(s[0], 0), min(s[1], n.k)};
    }
  }
  return v;
}
__device__ __forceinline__ Interval score_queries(const ScoreArgs& a, const ExtLens& n, int b, int key) {
  Interval v{a.causal != 0 ? max(key - n.start, 0) : 0, n.q};
  if (a.spans != nullptr) {
    const int32_t* const s = a.spans + 4 * ((int64_t)b * a.Nk + key);
    v = Interval{max(max(s[2], 0) - n.start, 0), min(min(s[3], a.Nk) - n.start, n.q)};
  }
  return v;
}

// What the intervals of several rows have together: some row's from any_lo to any_hi, every
// row's between all_lo and all_hi.
struct Reach {
  int any_lo = INT32_MAX, any_hi = 0, all_lo = 0, all_hi = INT32_MAX;
  __device__ __forceinline__ void add(Interval v) {
    if (v.lo < v.hi) {
      any_lo = min(any_lo, v.lo);
      any_hi = max(any_hi, v.hi);
      all_lo = max(all_lo, v.lo);
      all_hi = min(all_hi, v.hi);
    } else {
      all_hi = -1;
    }
  }
  // over the lanes whose index differs in the bits below `lanes`, into scalar registers
  template <int lanes> __device__ __forceinline__ void join() {
#pragma unroll
    for (int m = 1; m < lanes; m *= 2) {
      any_lo = min(any_lo, __shfl_xor(any_lo, m));
      any_hi = max(any_hi, __shfl_xor(any_hi, m));
      all_lo = max(all_lo, __shfl_xor(all_lo, m));
      all_hi = min(all_hi, __shfl_xor(all_hi, m));
    }
    any_lo = __builtin_amdgcn_readfirstlane(any_lo);
    any_hi = __builtin_amdgcn_readfirstlane(any_hi);
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);
  }
  // 0: no valid pair of the tile at s0, 1: all valid for every row, 2: mixed
  __device__ __forceinline__ int mode(int s0) const {
    return s0 >= any_hi || s0 + kBS <= any_lo ? 0 : s0 >= all_lo && s0 + kBS <= all_hi ? 1 : 2;
  }
};

// Exponents outside v to -inf: x[sb][r] belongs to streamed row s0 + 16 sb + 4 (l >> 4) + r.
__device__ __forceinline__ void score_mask(floatx4& x0, floatx4& x1, int s0, Interval v) {
  const int first = s0 + 4 * (lane_id() >> 4) - v.lo;
  const unsigned n = (unsigned)max(v.hi - v.lo, 0);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    x0[r] = (unsigned)(first + r) < n ? x0[r] : -INFINITY;
    x1[r] = (unsigned)(first + 16 + r) < n ? x1[r] : -INFINITY;
  }
}

// x[sb] - m |distance|, of a tile and a 16-row block of the stationary side: `first` is the distance
// at sb = 0, r = 0, kSign its step along the streamed side (rows: the keys stream).  m is in units
// of Q K^T, or of the cap, so that the scores' factor and L meet them in one operation.
template <int kSign>
__device__ __forceinline__ void score_distance(floatx4& x0, floatx4& x1, int first, float m) {
  const float d = (float)first;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    x0[r] = __builtin_fmaf(-m, fabsf(d + (float)(kSign * r)), x0[r]);
    x1[r] = __builtin_fmaf(-m, fabsf(d + (float)(kSign * (16 + r))), x1[r]);
  }
}
// log2(e) tau, or something of no effect that can be divided by where tau is 0.
__device__ __forceinline__ float score_scale(float scale) {
  const float c = scale * kLog2e;
  return fabsf(c) < 1e-30f ? 1e-30f : c;
}

// What a row kernel's workgroup and wave know of their rows (as ExtRows).
template <int MR, int NW, bool kFold>
struct ScoreRows {
  int b, kvh, head0, rows;
  int64_t qrow;
  int t0, tiles, kend;  // first key tile of the workgroup, tiles, keys that some row of it sees
  Interval keys[MR];    // of the lane's rows
  Reach reach;          // of the wave's rows
  int row0, qlen, Nq, start;
  bool fold;

  __device__ __forceinline__ ScoreRows(const ScoreArgs& a, int rh, int rb, int wl, int j) {
    constexpr int BR = 16 * MR * NW;
    fold = kFold && a.fold != 0;
    const int per_entry = fold ? a.H / a.grp : a.H;
    b = rh / per_entry;
    const int h = rh - b * per_entry;
    rows = fold ? a.grp * a.Nq : a.Nq;
    kvh = fold ? rh : rh / a.grp;
    head0 = fold ? h * a.grp : h;
    qrow = (int64_t)rh * rows;
    const ExtLens n = ext_lens(a, b);
    qlen = n.q;
    Nq = a.Nq;
    start = n.start;
    row0 = rb * BR + wl * 16 * MR + j;
    // folded rows hold every query of each head
    const int first = fold ? 0 : rb * BR, last = fold ? qlen : min(rb * BR + BR, qlen);
    Reach all;
    for (int q = first + lane_id(); q < last; q += 64) all.add(score_keys(a, n, b, q));
    all.template join<64>();
    kend = all.any_hi;
    t0 = all.any_lo < all.any_hi ? all.any_lo / kBS : 0;
    tiles = (kend + kBS - 1) / kBS - t0;
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) {
      keys[mb] = Interval{0, 0};
      if (ok(mb)) {  // other rows are not stored, whatever they hold
        keys[mb] = score_keys(a, n, b, query(mb));
        reach.add(keys[mb]);
      }
    }
    reach.template join<16>();
  }
  __device__ __forceinline__ int row(int mb) const { return row0 + 16 * mb; }
  __device__ __forceinline__ int query(int mb) const { return fold ? row(mb) % Nq : row(mb); }
  __device__ __forceinline__ int head(int mb) const { return fold ? head0 + min(row(mb), rows - 1) / Nq : head0; }
  __device__ __forceinline__ int pos(int mb) const { return start + query(mb); }
  __device__ __forceinline__ bool ok(int mb) const { return row(mb) < rows && query(mb) < qlen; }
  // the first key of tile i of the run
  __device__ __forceinline__ int key(int i) const { return (t0 + min(i, tiles - 1)) * kBS; }
  // The same in the forward's order under a distance bias: from the tile of the workgroup's last
  // query (`peak`, from outward()) down, then those behind it upward.  Scores fall with distance,
  // so the running maximum is found at once; from the first key on it grew in every tile (B1 H16
  // N8192 d128 causal 690 us).
  __device__ __forceinline__ int outward(const ScoreArgs& a, int rb) const {
    if (a.slopes == nullptr) return -1;
    const int last = start + (fold ? qlen : min((rb + 1) * 16 * MR * NW, qlen)) - 1;
    return min(max(last, 0) / kBS - t0, tiles - 1);
  }
  __device__ __forceinline__ int key(int i, int peak) const {
    const int at = min(i, tiles - 1);
    return (t0 + (at <= peak ? peak - at : at)) * kBS;
  }
};

// The slope of a row kernel's lane, of one head (folded rows have one row a lane); c: the scores'
// factor.
template <typename Rows>
__device__ __forceinline__ float score_row_slope(const ScoreArgs& a, const Rows& rw, float c) {
  if (a.slopes == nullptr) return 0.f;
  return a.slopes[rw.head(0)] * kLog2e / c;
}
template <int MR, typename Rows>
__device__ __forceinline__ void score_row_distance(const ScoreArgs& a, const Rows& rw, int s0, float slope,
                                                   floatx4 (&s)[2][MR]) {
  if (a.slopes == nullptr) return;
#pragma unroll
  for (int mb = 0; mb < MR; ++mb)
    score_distance<-1>(s[0][mb], s[1][mb], rw.pos(mb) - s0 - 4 * (lane_id() >> 4), slope);
}

// x rounded to T, and what that leaves.
template <typename T> __device__ __forceinline__ void store_both(T* hi, T* lo, floatx4 x) {
  Elt<T>::store4(hi, x);
  if (lo == nullptr) return;
#pragma unroll
  for (int r = 0; r < 4; ++r) x[r] -= (float)(T)x[r];
  Elt<T>::store4(lo, x);
}
template <typename T> __device__ __forceinline__ floatx4 load_both(const T* hi, const T* lo, int64_t at) {
  const floatx4 x = Elt<T>::load4(hi + at);
  return lo == nullptr ? x : x + Elt<T>::load4(lo + at);
}

// sum plus an operand's elements as they are rounded.
__device__ __forceinline__ float add_rounded(const Elt<bf16>::TFrag& f, float sum) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 one = {(bf16)1.f, (bf16)1.f};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{f.v[2 * i], f.v[2 * i + 1]}, one, sum, false);
  return sum;
}

// {-1, 0} and {0, -1} as bf16 pairs, in a register: as the instruction's own constant the
// assembler writes {-1, 0} as -1.0, which the instruction reads as {0, -1}.
template <int kAt> __device__ __forceinline__ auto minus_one() {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  unsigned bits = kAt == 0 ? 0x0000bf80u : 0xbf800000u;
  asm("" : "+s"(bits));
  return __builtin_bit_cast(bf16x2, bits);
}
// An operand in twice the bits of bf16: its rounding and what that left, x - hi in one dot
// product of two (subtracting the unpacked value takes two instructions).  fp32 needs one.
// Elements are set in ascending order.
template <typename T> struct SplitFrag {
  using E = Elt<T>;
  static constexpr bool kTwo = sizeof(T) == 2;
  typename E::TFrag hi, lo;
  float before;  // element i - 1
  __device__ __forceinline__ void set(int i, float x) {
    hi.set(i, x);
    if constexpr (kTwo) {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      if (i % 2 != 0) {
        const bf16x2 pair = {hi.v[i - 1], hi.v[i]};
        lo.set(i - 1, __builtin_amdgcn_fdot2_f32_bf16(pair, minus_one<0>(), before, false));
        lo.set(i, __builtin_amdgcn_fdot2_f32_bf16(pair, minus_one<1>(), x, false));
      }
      before = x;
    }
  }
  __device__ __forceinline__ floatx4 mma_acc(const typename E::AFrag& a, floatx4 c) const {
    c = E::mma_acc(a, hi, c);
    if constexpr (kTwo) c = E::mma_acc(a, lo, c);
    return c;
  }
};

// ===========================================================================
// Forward, as ext_fwd_kernel.  Orest may be null.  Bound by MFMA and VALU issue for many rows: B1
// H16 N8192 d128 causal with slopes 286 us, 0.96 PFLOP/s, the two busy for 83% of the cycles; a cap
// takes 12 VALU operations an element for 7 (B4 H16 Hkv8 N4096 d128 causal 348 us for 300).  For a
// few rows by the keys' and values' bytes: B16 H16 Hkv4, one token, up to 4096 keys, d128, 87 MB in
// 22 us.
// ===========================================================================
template <typename T, int D, int MR, int NW, int OCC, int KS, bool kCap>
__global__ __launch_bounds__(KS * NW * 64, OCC) void score_fwd_kernel(
    ScoreArgs a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, T* __restrict__ O,
    T* __restrict__ Orest, float* __restrict__ L, float* __restrict__ parts) {
  using E = Elt<T>;
  using G = Geo<T, D>;
  constexpr int BR = 16 * MR * NW;
  __shared__ __attribute__((aligned(16))) RowSmem<T, D, 2, 2, KS, BR> sm;
  __shared__ float rounded_mem[KS > 1 && sizeof(T) == 2 ? KS : 1][KS > 1 && sizeof(T) == 2 ? BR : 1];

  int rh, rb;
  ext_map_block(a, a.fold != 0 ? a.nRB : a.grp * a.nRB, true, NW == 1 ? nullptr : a.kv_lens, a.Nk, rh, rb);
  const int l = lane_id(), g = l >> 4, j = l & 15;
  const int ks = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave_id() / NW);
  const int wl = __builtin_amdgcn_readfirstlane(KS == 1 ? wave_id() : wave_id() % NW);
  const ScoreRows<MR, NW, MR == 1> rw(a, rh, rb, wl, j);
  const int part = blockIdx.y;
  const int64_t kvoff = (int64_t)rw.kvh * a.Nk * D;

  u32x4 qf[MR][G::kChunks];
#pragma unroll
  for (int mb = 0; mb < MR; ++mb)
    load_stationary<T, D>(qf[mb], Q + rw.qrow * D, rw.ok(mb) ? rw.row(mb) : rw.rows, rw.rows);

  floatx4 acc[G::kNB][MR];
#pragma unroll
  for (int nb = 0; nb < G::kNB; ++nb)
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) acc[nb][mb] = floatx4{0.f, 0.f, 0.f, 0.f};
  constexpr bool kRounded = sizeof(T) == 2;
  float mrun[MR], lsum[MR], rsum[MR];  // rsum: of P as it is rounded
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) {
    mrun[mb] = -1e30f;
    lsum[mb] = rsum[mb] = 0.f;
  }
  const float c = kCap ? a.cap_out : score_scale(a.scale);
  const float slope = score_row_slope(a, rw, c);
  floatx4 s[2][MR];
  typename E::TFrag pf[MR];

  // s times c are the scores in log2 units
  auto softmax_step = [&](int s0, int mode) {
    float p[MR][8], ls[MR];
    bool grown = false;
    floatx4 e[MR][2];
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) {
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int r = 0; r < 4; ++r) e[mb][sb][r] = __builtin_fmaf(s[sb][mb][r], c, -mrun[mb]);
    }
    if (mode == 2) {
#pragma unroll
      for (int mb = 0; mb < MR; ++mb) score_mask(e[mb][0], e[mb][1], s0, rw.keys[mb]);
    }
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[mb][i] = fast_exp2(e[mb][i >> 2][i & 3]);
      ls[mb] = ((p[mb][0] + p[mb][1]) + (p[mb][2] + p[mb][3])) + ((p[mb][4] + p[mb][5]) + (p[mb][6] + p[mb][7]));
      grown |= !(ls[mb] <= kRescaleP);
    }
    if (__builtin_amdgcn_ballot_w64(grown) != 0) {
#pragma unroll
      for (int mb = 0; mb < MR; ++mb) {
        if (__builtin_amdgcn_ballot_w64(!(ls[mb] <= kRescaleP)) == 0) continue;
        floatx4 x[2];
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int r = 0; r < 4; ++r) x[sb][r] = s[sb][mb][r] * c;
        if (mode == 2) score_mask(x[0], x[1], s0, rw.keys[mb]);
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) mx = fmaxf(mx, x[i >> 2][i & 3]);
        mx = group_max(mx);
        if (__builtin_amdgcn_ballot_w64(mx > mrun[mb] + kRescaleLog2) != 0) {
          const float mnew = fmaxf(mrun[mb], mx);
          const float corr = fast_exp2(mrun[mb] - mnew);
          mrun[mb] = mnew;
          lsum[mb] *= corr;
          rsum[mb] *= corr;
#pragma unroll
          for (int nb = 0; nb < G::kNB; ++nb) acc[nb][mb] *= corr;
        }
        ls[mb] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[mb][i] = fast_exp2(x[i >> 2][i & 3] - mrun[mb]);
          ls[mb] += p[mb][i];
        }
      }
    }
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) {
      lsum[mb] += ls[mb];
#pragma unroll
      for (int i = 0; i < 8; ++i) pf[mb].set(i, p[mb][i]);
      if constexpr (kRounded) rsum[mb] = add_rounded(pf[mb], rsum[mb]);
    }
  };

  const T* const src[2] = {K + kvoff, V + kvoff};
  const int split = ext_parts_of(rw.tiles, KS, a.nparts), peak = rw.outward(a, rb);
  const ExtRun run = ext_run(rw.tiles, part, split, ks, KS), first = ext_run(rw.tiles, part, split, 0, KS);
  constexpr bool kBarrier = NW > 1;
  const TileCopy<T, D, NW, 2> copy(wl);
  ext_stream<tile_loads<T, D, NW, 2>(), kBarrier>(
      kBarrier ? first.size() : run.size(),
      [&](int it, int st) {
        copy.template issue<true>(src, (T FB_LDS*)sm.lds[ks][st], rw.key(run.begin + it, peak), rw.kend);
      },
      []() {},
      [&](int it, int st) {
        const int s0 = rw.key(run.begin + it, peak);
        const int mode = vector_mode(run.begin + it < run.end ? rw.reach.mode(s0) : 0);
        if (mode == 0) return;
        const T FB_LDS* Ks = (const T FB_LDS*)sm.lds[ks][st];
        const T FB_LDS* Vs = Ks + G::kTileElems;
#pragma unroll
        for (int x = 0; x < MR; ++x) s[0][x] = s[1][x] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int kk = 0; kk < G::kChunks; ++kk) {
            const u32x4 ak = *(const u32x4 FB_LDS*)(Ks + G::chunk_off(16 * sb + j, 4 * kk + g));
#pragma unroll
            for (int mb = 0; mb < MR; ++mb) s[sb][mb] = E::mma_chunk(ak, qf[mb][kk], s[sb][mb]);
          }
        if constexpr (kCap) cap_tile<T>(a, s, s);
        score_row_distance(a, rw, s0, slope, s);
        softmax_step(s0, mode);
#pragma unroll
        for (int nb = 0; nb < G::kNB; ++nb) {
          const typename E::AFrag av = G::load_afrag(Vs, 16 * nb);
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) acc[nb][mb] = E::mma_acc(av, pf[mb], acc[nb][mb]);
        }
      });
  float lt[MR], rt[MR];
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) {
    lt[mb] = group_sum(lsum[mb]);
    rt[mb] = kRounded ? group_sum(rsum[mb]) : lt[mb];
  }
  if constexpr (KS > 1) {
    // one reference for the sets, then their sums, as in ext_fwd_kernel
#pragma unroll
    for (int mb = 0; mb < MR; ++mb)
      if (g == 0) {
        const int at = 16 * (wl * MR + mb) + j;
        sm.sc[0][ks][at] = mrun[mb];
        sm.sc[1][ks][at] = lt[mb];
        if (kRounded) rounded_mem[ks][at] = rt[mb];
      }
    __syncthreads();
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) {
      const int at = 16 * (wl * MR + mb) + j;
      float m = sm.sc[0][0][at], sum = 0.f, rounded = 0.f;
#pragma unroll
      for (int q = 1; q < KS; ++q) m = fmaxf(m, sm.sc[0][q][at]);
#pragma unroll
      for (int q = 0; q < KS; ++q) {
        const float f = fast_exp2(sm.sc[0][q][at] - m);
        sum = __builtin_fmaf(sm.sc[1][q][at], f, sum);
        if (kRounded) rounded = __builtin_fmaf(rounded_mem[q][at], f, rounded);
      }
      const float corr = fast_exp2(mrun[mb] - m);
      mrun[mb] = m;
      lt[mb] = sum;
      rt[mb] = kRounded ? rounded : sum;
#pragma unroll
      for (int nb = 0; nb < G::kNB; ++nb) acc[nb][mb] *= corr;
    }
    static_assert(sizeof(sm.lds) >= merge_bytes<KS, NW, G::kNB, MR>(), "set merge buffer");
    merge_sets<KS, NW>(acc, ks, wl, (floatx4 FB_LDS*)&sm.lds[0][0][0]);
  }
  const RowSplit<KS> own{ks, 0};
  if (a.nparts > 1) {
    const int64_t all = (int64_t)(a.total / a.nRB) * rw.rows;
    float* const ml = parts + a.nparts * all * D;
#pragma unroll
    for (int mb = 0; mb < MR; ++mb)
      if (rw.ok(mb)) {
        const int64_t at = part * all + rw.qrow + rw.row(mb);
#pragma unroll
        for (int nb = 0; nb < G::kNB; ++nb)
          if (own.owns(nb)) *(floatx4*)(parts + at * D + 16 * nb + 4 * g) = acc[nb][mb];
        if (g == 0 && ks == 0) *(floatx4*)(ml + 4 * at) = floatx4{mrun[mb], lt[mb], rt[mb], 0.f};
      }
    return;
  }
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) {
    if (rw.row(mb) >= rw.rows) continue;
    const int64_t at = rw.qrow + rw.row(mb);
    const bool some = rw.ok(mb) && lt[mb] != 0.f;
    const float inv = 1.f / rt[mb];
#pragma unroll
    for (int nb = 0; nb < G::kNB; ++nb)
      if (own.owns(nb)) {
        const int64_t off = at * D + 16 * nb + 4 * g;
        store_both(O + off, Orest != nullptr ? Orest + off : nullptr,
                   some ? acc[nb][mb] * inv : floatx4{0.f, 0.f, 0.f, 0.f});
      }
    if (g == 0 && ks == 0) L[at] = some ? (mrun[mb] + __log2f(lt[mb])) * kLn2 : -INFINITY;
  }
}

constexpr int kFwdScalars = 4;  // floats a row and part: reference, sum, rounded sum

// Joins the parts of the forward, as ext_fwd_join_kernel.
template <typename T, int D>
__global__ __launch_bounds__(256) void score_fwd_join_kernel(ExtArgs a, const float* __restrict__ parts, int64_t all,
                                                             T* __restrict__ O, T* __restrict__ Orest,
                                                             float* __restrict__ L) {
  constexpr int kPer = D / 4;
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = x / kPer;
  const int dim = 4 * (int)(x % kPer);
  if (row >= all) return;
  const int64_t bh = row / a.Nq, off = row * D + dim;
  const bool ok = (int)(row - bh * a.Nq) < ext_lens(a, (int)(bh / a.H)).q;
  const float* const ml = parts + a.nparts * all * D;
  floatx4 sum = floatx4{0.f, 0.f, 0.f, 0.f};
  float m = -1e30f, w = 0.f, rounded = 0.f;
  if (ok) {
    for (int q = 0; q < a.nparts; ++q) m = fmaxf(m, ml[4 * (q * all + row)]);
    for (int q = 0; q < a.nparts; ++q) {
      const int64_t at = q * all + row;
      const floatx4 mine = *(const floatx4*)(ml + 4 * at);
      const float f = fast_exp2(mine[0] - m);
      w = __builtin_fmaf(mine[1], f, w);
      rounded = __builtin_fmaf(mine[2], f, rounded);
      sum += *(const floatx4*)(parts + at * D + dim) * f;
    }
  }
  const bool some = ok && w != 0.f;
  store_both(O + off, Orest != nullptr ? Orest + off : nullptr,
             some ? sum * (1.f / rounded) : floatx4{0.f, 0.f, 0.f, 0.f});
  if (dim == 0) L[row] = some ? (m + __log2f(w)) * kLn2 : -INFINITY;
}

__device__ __forceinline__ float cap_slope(float t) { return __builtin_fmaf(-t, t, 1.f); }

// A row kernel's raw scores -> the exponents of P: capped (t = tanh), less L.
template <typename T, bool kCap, int MR, int A, int B, typename Rows>
__device__ __forceinline__ void score_row_exponents(const ScoreArgs& a, const Rows& rw, float slope, float c, int s0,
                                                    const float (&lb)[MR], floatx4 (&s)[2][MR], floatx4 (&t)[A][B]) {
  if constexpr (kCap) {
    cap_tile<T>(a, s, t);
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) s[0][mb] = t[0][mb], s[1][mb] = t[1][mb];
  }
  score_row_distance(a, rw, s0, slope, s);
#pragma unroll
  for (int mb = 0; mb < MR; ++mb)
#pragma unroll
    for (int sb = 0; sb < 2; ++sb)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[sb][mb][r] = __builtin_fmaf(s[sb][mb][r], c, -lb[mb]);
}

// ===========================================================================
// First backward, row side, as ext_bwd_rows_kernel.  A capped tile's t takes eight registers a
// 16-row block from the exponent to the gradient of the score.  dS meets K as two bf16 values:
// four contractions a tile for three.  Bound by MFMA (43% of the cycles) and VALU issue (62%),
// which overlap little: B4 H16 Hkv8 N4096 d128 causal 491 us, with a cap 561.
// ===========================================================================
template <typename T, int D, int MR, int NW, int OCC, int KS, bool kCap>
__global__ __launch_bounds__(KS * NW * 64, OCC) void score_bwd_rows_kernel(
    ScoreArgs a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ O,
    const T* __restrict__ Orest, const T* __restrict__ dO, const float* __restrict__ L, T* __restrict__ dQ,
    float* __restrict__ Dout,
    float* __restrict__ parts) {
  using E = Elt<T>;
  using G = Geo<T, D>;
  constexpr int BR = 16 * MR * NW;
  __shared__ __attribute__((aligned(16))) RowSmem<T, D, 2, 2, KS, BR> sm;

  int rh, rb;
  ext_map_block(a, a.grp * a.nRB, true, a.kv_lens, a.Nk, rh, rb);
  const int l = lane_id(), g = l >> 4, j = l & 15;
  const int ks = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave_id() / NW);
  const int wl = __builtin_amdgcn_readfirstlane(KS == 1 ? wave_id() : wave_id() % NW);
  const ScoreRows<MR, NW, false> rw(a, rh, rb, wl, j);
  const int64_t kvoff = (int64_t)rw.kvh * a.Nk * D, qoff = rw.qrow * D;

  u32x4 qf[MR][G::kChunks], dof[MR][G::kChunks];
  float lb[MR], drow[MR], dout[MR], rest[MR];
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) {
    const int row = rw.ok(mb) ? rw.row(mb) : rw.rows;
    load_stationary<T, D>(qf[mb], Q + qoff, row, rw.rows);
    load_stationary<T, D>(dof[mb], dO + qoff, row, rw.rows);
    u32x4 of[G::kChunks];
    load_stationary<T, D>(of, O + qoff, row, rw.rows);
    float part = 0.f;
#pragma unroll
    for (int kk = 0; kk < G::kChunks; ++kk) part += E::dot_chunk(dof[mb][kk], of[kk]);
    if (Orest != nullptr) {
      load_stationary<T, D>(of, Orest + qoff, row, rw.rows);
      float rest_part = 0.f;
#pragma unroll
      for (int kk = 0; kk < G::kChunks; ++kk) rest_part += E::dot_chunk(dof[mb][kk], of[kk]);
      part += rest_part;
    }
    drow[mb] = dout[mb] = group_sum(part);
    // an empty row (L = -inf) gets P = 0
    const float Lr = rw.ok(mb) ? L[rw.qrow + rw.row(mb)] : 0.f;
    lb[mb] = Lr == -INFINITY ? INFINITY : Lr * kLog2e;
    rest[mb] = 0.f;
  }

  floatx4 acc[G::kNB][MR];
#pragma unroll
  for (int nb = 0; nb < G::kNB; ++nb)
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) acc[nb][mb] = floatx4{0.f, 0.f, 0.f, 0.f};
  const float c = kCap ? a.cap_out : score_scale(a.scale);
  const float slope = score_row_slope(a, rw, c);
  floatx4 s[2][MR], dp[2][MR], t[kCap ? 2 : 1][kCap ? MR : 1];
  SplitFrag<T> dsf[MR];

  const T* const src[2] = {K + kvoff, V + kvoff};
  const int part = blockIdx.y, split = ext_parts_of(rw.tiles, KS, a.nparts);
  const ExtRun run = ext_run(rw.tiles, part, split, ks, KS), first = ext_run(rw.tiles, part, split, 0, KS);
  constexpr bool kBarrier = NW > 1;
  const TileCopy<T, D, NW, 2> copy(wl);
  ext_stream<tile_loads<T, D, NW, 2>(), kBarrier>(
      kBarrier ? first.size() : run.size(),
      [&](int it, int st) {
        copy.template issue<true>(src, (T FB_LDS*)sm.lds[ks][st], rw.key(run.begin + it), rw.kend);
      },
      []() {},
      [&](int it, int st) {
        const int s0 = rw.key(run.begin + it);
        const int mode = vector_mode(run.begin + it < run.end ? rw.reach.mode(s0) : 0);
        if (mode == 0) return;
        const T FB_LDS* Ks = (const T FB_LDS*)sm.lds[ks][st];
        const T FB_LDS* Vs = Ks + G::kTileElems;
#pragma unroll
        for (int x = 0; x < MR; ++x) s[0][x] = s[1][x] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) dp[sb][mb] = floatx4{-drow[mb], -drow[mb], -drow[mb], -drow[mb]};
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int kk = 0; kk < G::kChunks; ++kk) {
            const int off = G::chunk_off(16 * sb + j, 4 * kk + g);
            const u32x4 ak = *(const u32x4 FB_LDS*)(Ks + off);
            const u32x4 av = *(const u32x4 FB_LDS*)(Vs + off);
#pragma unroll
            for (int mb = 0; mb < MR; ++mb) {
              s[sb][mb] = E::mma_chunk(ak, qf[mb][kk], s[sb][mb]);
              dp[sb][mb] = E::mma_chunk(av, dof[mb][kk], dp[sb][mb]);
            }
          }
        score_row_exponents<T, kCap>(a, rw, slope, c, s0, lb, s, t);
        if (mode == 2) {
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) score_mask(s[0][mb], s[1][mb], s0, rw.keys[mb]);
        }
#pragma unroll
        for (int mb = 0; mb < MR; ++mb)
#pragma unroll
          for (int sb = 0; sb < 2; ++sb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float dz = fast_exp2(s[sb][mb][r]) * dp[sb][mb][r];
              rest[mb] += dz;
              if constexpr (kCap)
                dsf[mb].set(4 * sb + r, dz * cap_slope(t[sb][mb][r]));
              else
                dsf[mb].set(4 * sb + r, dz);
            }
#pragma unroll
        for (int nb = 0; nb < G::kNB; ++nb) {
          const typename E::AFrag ak = G::load_afrag(Ks, 16 * nb);
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) acc[nb][mb] = dsf[mb].mma_acc(ak, acc[nb][mb]);
        }
      });
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) rest[mb] = group_sum(rest[mb]);
  if constexpr (KS > 1) {
#pragma unroll
    for (int mb = 0; mb < MR; ++mb)
      if (g == 0) sm.sc[0][ks][16 * (wl * MR + mb) + j] = rest[mb];
    __syncthreads();
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) {
      const int at = 16 * (wl * MR + mb) + j;
      rest[mb] = sm.sc[0][0][at];
#pragma unroll
      for (int q = 1; q < KS; ++q) rest[mb] += sm.sc[0][q][at];
    }
    static_assert(sizeof(sm.lds) >= merge_bytes<KS, NW, G::kNB, MR>(), "set merge buffer");
    merge_sets<KS, NW>(acc, ks, wl, (floatx4 FB_LDS*)&sm.lds[0][0][0]);
  }
  const RowSplit<KS> own{ks, 0};
  if (a.nparts > 1) {
    const int64_t all = (int64_t)(a.total / a.nRB) * rw.rows;
    float* const sc = parts + a.nparts * all * D;
#pragma unroll
    for (int mb = 0; mb < MR; ++mb)
      if (rw.ok(mb)) {
        const int64_t at = part * all + rw.qrow + rw.row(mb);
#pragma unroll
        for (int nb = 0; nb < G::kNB; ++nb)
          if (own.owns(nb)) *(floatx4*)(parts + at * D + 16 * nb + 4 * g) = acc[nb][mb];
        if (g == 0 && ks == 0) sc[at] = (part == 0 ? dout[mb] : 0.f) + rest[mb];
      }
    return;
  }
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) {
    if (rw.row(mb) >= rw.rows) continue;
    const int64_t at = rw.qrow + rw.row(mb);
#pragma unroll
    for (int nb = 0; nb < G::kNB; ++nb)
      if (own.owns(nb))
        E::store4(dQ + at * D + 16 * nb + 4 * g, rw.ok(mb) ? acc[nb][mb] * a.scale : floatx4{0.f, 0.f, 0.f, 0.f});
    if (g == 0 && ks == 0) Dout[at] = rw.ok(mb) ? dout[mb] + rest[mb] : 0.f;
  }
}

// ===========================================================================
// Column kernels
// ===========================================================================

// What a column kernel's workgroup and wave know of their columns (as ExtCols).
template <int MC, int NW>
struct ScoreCols {
  int b, kvh, hq, heads, sub, subs;
  int t0, per_head;  // first query tile, query tiles a head
  int qlen, klen, start;
  int col0;           // first column of the wave
  Interval rows[MC];  // query rows that see the lane's columns
  Reach reach;        // of the wave's columns
  __device__ __forceinline__ ScoreCols(const ScoreArgs& a, int kv, int rb, int wl) {
    constexpr int BC = 16 * MC * NW;
    const int per_entry = a.H / a.grp;
    kvh = kv;
    b = kv / per_entry;
    const int split = a.nparts > 1;
    subs = split ? a.nparts / a.grp : 1;
    const int part = blockIdx.y;
    heads = split ? 1 : a.grp;
    hq = kv * a.grp + (split ? part / subs : 0);
    sub = split ? part % subs : 0;
    const ExtLens n = ext_lens(a, b);
    qlen = n.q;
    klen = n.k;
    start = n.start;
    col0 = rb * BC + wl * 16 * MC;
    Reach all;
    for (int col = rb * BC + lane_id(); col < min(rb * BC + BC, klen); col += 64) all.add(score_queries(a, n, b, col));
    all.template join<64>();
    t0 = all.any_lo < all.any_hi ? all.any_lo / kBS : 0;
    per_head = (all.any_hi + kBS - 1) / kBS - t0;
#pragma unroll
    for (int mc = 0; mc < MC; ++mc) {
      const int col = col0 + 16 * mc + (lane_id() & 15);
      rows[mc] = Interval{0, 0};
      if (col < klen) {  // other columns are stored as zeros
        rows[mc] = score_queries(a, n, b, col);
        reach.add(rows[mc]);
      }
    }
    reach.template join<16>();
  }
  __device__ __forceinline__ int count() const { return heads * per_head; }
  __device__ __forceinline__ int qhead(int f) const { return heads == 1 ? hq : hq + f / per_head; }
  __device__ __forceinline__ int tile(int f) const { return t0 + (heads == 1 ? f : f % per_head); }
};

// The slopes of a key/value head's query heads, as score_row_slope(): in LDS, and that of a workgroup with
// one head in a register (read from LDS in every tile it held up the first MFMA).
struct ColSlopes {
  const float FB_LDS* all;
  float one = 0.f;
  template <typename Cols>
  __device__ __forceinline__ ColSlopes(const ScoreArgs& a, const Cols& cl, float* mem, int threads, float c) {
    float FB_LDS* const to = (float FB_LDS*)mem;
    all = to;
    if (a.slopes == nullptr) return;
    const float* const from = a.slopes + cl.kvh * a.grp % a.H;
    one = from[cl.hq - cl.kvh * a.grp] * kLog2e / c;
    for (int x = threadIdx.x; x < a.grp; x += threads) to[x] = from[x] * kLog2e / c;
    __syncthreads();
  }
};

// The slope of tile f's head.
template <typename Cols>
__device__ __forceinline__ float score_col_slope(const ScoreArgs& a, const Cols& cl, const ColSlopes& slopes, int f) {
  if (a.slopes == nullptr) return 0.f;
  return cl.heads == 1 ? slopes.one : scalar(slopes.all[cl.qhead(f) - cl.kvh * a.grp]);
}
template <int MC, typename Cols>
__device__ __forceinline__ void score_col_distance(const ScoreArgs& a, const Cols& cl, int s0, float slope,
                                                   floatx4 (&s)[2][MC]) {
  if (a.slopes == nullptr) return;
  const int l = lane_id();
#pragma unroll
  for (int mc = 0; mc < MC; ++mc)
    score_distance<1>(s[0][mc], s[1][mc], cl.start + s0 + 4 * (l >> 4) - (cl.col0 + 16 * mc + (l & 15)), slope);
}

// A column kernel's raw scores -> the exponents of P; off: the row scalars.  Uncapped scores have
// their distance before the first MFMA (after the last one bf16 d = 64 spilled, and Pass 2 of B4 H12
// N4096 took 433 us for 409).
template <typename T, bool kCap, int MC, int A, int B, typename Cols>
__device__ __forceinline__ void score_col_exponents(const ScoreArgs& a, const Cols& cl, float slope, float c, int s0,
                                                    const float FB_LDS* off, floatx4 (&s)[2][MC], floatx4 (&t)[A][B]) {
  if constexpr (kCap) {
    cap_tile<T>(a, s, t);
#pragma unroll
    for (int mc = 0; mc < MC; ++mc) s[0][mc] = t[0][mc], s[1][mc] = t[1][mc];
    score_col_distance(a, cl, s0, slope, s);
  }
#pragma unroll
  for (int sb = 0; sb < 2; ++sb) {
    const floatx4 o = *(const floatx4 FB_LDS*)(off + 16 * sb + 4 * (lane_id() >> 4));
#pragma unroll
    for (int mc = 0; mc < MC; ++mc)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[sb][mc][r] = __builtin_fmaf(s[sb][mc][r], c, o[r]);
  }
}

// First backward, column side, as ext_bwd_cols_kernel (P and dS are summed over queries whose
// roundings do not cancel: one bf16 value each).  Bound as the row side: 556 us there, with a cap 623.
template <typename T, int D, int MC, int NW, int OCC, int KS, bool kKL, bool kCap>
__global__ __launch_bounds__(KS * NW * 64, OCC) void score_bwd_cols_kernel(
    ScoreArgs a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ dO,
    const float* __restrict__ L, const float* __restrict__ Dv, T* __restrict__ dK, T* __restrict__ dV,
    float* __restrict__ parts) {
  using E = Elt<T>;
  using G = Geo<T, D>;
  struct Smem {
    T lds[KS][2][2 * G::kTileElems];
    float rawsc[KS][2][2 * kBS];
    float tsc[KS][2][2 * kBS];
  };
  constexpr int kWPT = kBS / (16 * MC);  // waves per stationary K tile
  static_assert(!kKL || (kBS % (16 * MC) == 0 && NW % kWPT == 0), "stationary K in LDS: 32-row tiles");
  struct SmemK : Smem {
    T kst[NW / kWPT][G::kTileElems];
  };
  __shared__ __attribute__((aligned(16))) std::conditional_t<kKL, SmemK, Smem> sm;
  extern __shared__ float slope_mem[];

  int kv, rb;
  ext_map_cols(a, kv, rb);
  const int l = lane_id(), g = l >> 4, j = l & 15;
  const int ks = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave_id() / NW);
  const int wl = __builtin_amdgcn_readfirstlane(KS == 1 ? wave_id() : wave_id() % NW);
  const ScoreCols<MC, NW> cl(a, kv, rb, wl);
  const int64_t koff = (int64_t)kv * a.Nk * D;

  u32x4 kf[kKL ? 1 : MC][G::kChunks], vf[MC][G::kChunks];
#pragma unroll
  for (int mc = 0; mc < MC; ++mc) {
    if constexpr (!kKL) load_stationary<T, D>(kf[mc], K + koff, cl.col0 + 16 * mc + j, cl.klen);
    load_stationary<T, D>(vf[mc], V + koff, cl.col0 + 16 * mc + j, cl.klen);
  }
  if constexpr (kKL) {
    // read by waves with a valid column alone, which lies in the tile
    if (ks == 0 && wl % kWPT == 0 && cl.col0 < cl.klen) {
      const TileCopy<T, D, 1, 1> kc(0);
      const T* const ksrc[1] = {K + koff};
      kc.template issue<true>(ksrc, (T FB_LDS*)sm.kst[wl / kWPT], cl.col0, cl.klen);
    }
  }
  const float c = kCap ? a.cap_out : score_scale(a.scale);
  const ColSlopes slopes(a, cl, slope_mem, KS * NW * 64, c);
  floatx4 dk[G::kNB][MC], dv[G::kNB][MC];
#pragma unroll
  for (int nb = 0; nb < G::kNB; ++nb)
#pragma unroll
    for (int mc = 0; mc < MC; ++mc) dk[nb][mc] = dv[nb][mc] = floatx4{0.f, 0.f, 0.f, 0.f};
  floatx4 s[2][MC], dp[2][MC], t[kCap ? 2 : 1][kCap ? MC : 1];
  typename E::TFrag pf[MC], dsf[MC];

  const int n = cl.count();
  const ExtRun run(n, cl.sub * KS + ks, cl.subs * KS), first(n, cl.sub * KS, cl.subs * KS);
  auto flat = [&](int it) { return min(run.begin + it, n - 1); };
  const TileCopy<T, D, NW, 2> copy(wl);
  stream_loop_rs<2, tile_loads<T, D, NW, 2>(), 1, true>(
      0, first.size(), __builtin_amdgcn_readfirstlane(wl) == 0,
      [&](int it, int rs) {
        const int64_t qs = (int64_t)cl.qhead(flat(it)) * a.Nq;
        issue_scalar_pair<true>((float FB_LDS*)sm.rawsc[ks][rs], L + qs, Dv + qs, cl.tile(flat(it)) * kBS, cl.qlen);
      },
      [&](int it, int st) {
        const int64_t qo = (int64_t)cl.qhead(flat(it)) * a.Nq * D;
        const T* const src[2] = {Q + qo, dO + qo};
        copy.template issue<true>(src, (T FB_LDS*)sm.lds[ks][st], cl.tile(flat(it)) * kBS, cl.qlen);
      },
      [&](int, int rs, int ts) {
        if (l < kBS) {
          const float FB_LDS* raw = (const float FB_LDS*)sm.rawsc[ks][rs];
          float FB_LDS* to = (float FB_LDS*)sm.tsc[ks][ts];
          const float Lr = raw[l];
          to[l] = Lr == -INFINITY ? -INFINITY : -Lr * kLog2e;  // an empty row: P = 0
          to[kBS + l] = -raw[kBS + l];
        }
      },
      [&](int it, int st, int ts, auto&& prep_next) {
        const int s0 = cl.tile(flat(it)) * kBS;
        const int mode = vector_mode(run.begin + it < run.end ? cl.reach.mode(s0) : 0);
        if (mode == 0) {
          prep_next();
          return;
        }
        const T FB_LDS* Qs = (const T FB_LDS*)sm.lds[ks][st];
        const T FB_LDS* dOs = Qs + G::kTileElems;
        const float FB_LDS* Ts = (const float FB_LDS*)sm.tsc[ks][ts];
        const float slope = score_col_slope(a, cl, slopes, flat(it));
#pragma unroll
        for (int x = 0; x < MC; ++x) s[0][x] = s[1][x] = floatx4{0.f, 0.f, 0.f, 0.f};
        if constexpr (!kCap) score_col_distance(a, cl, s0, slope, s);
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
          const floatx4 t1 = *(const floatx4 FB_LDS*)(Ts + kBS + 16 * sb + 4 * g);
#pragma unroll
          for (int mc = 0; mc < MC; ++mc) {
            dp[sb][mc] = t1;
          }
        }
        __builtin_amdgcn_s_setprio(1);
        if constexpr (kKL) {
          const T FB_LDS* Ks = (const T FB_LDS*)sm.kst[wl / kWPT];
          const int r0 = 16 * MC * (wl % kWPT);
#pragma unroll
          for (int kk = 0; kk < G::kChunks; ++kk) {
            u32x4 kfr[MC];
#pragma unroll
            for (int mc = 0; mc < MC; ++mc)
              kfr[mc] = *(const u32x4 FB_LDS*)(Ks + G::chunk_off(r0 + 16 * mc + j, 4 * kk + g));
#pragma unroll
            for (int sb = 0; sb < 2; ++sb) {
              const int off = G::chunk_off(16 * sb + j, 4 * kk + g);
              const u32x4 aq = *(const u32x4 FB_LDS*)(Qs + off);
              const u32x4 ado = *(const u32x4 FB_LDS*)(dOs + off);
#pragma unroll
              for (int mc = 0; mc < MC; ++mc) {
                s[sb][mc] = E::mma_chunk(aq, kfr[mc], s[sb][mc]);
                dp[sb][mc] = E::mma_chunk(ado, vf[mc][kk], dp[sb][mc]);
              }
            }
          }
        } else {
#pragma unroll
          for (int sb = 0; sb < 2; ++sb)
#pragma unroll
            for (int kk = 0; kk < G::kChunks; ++kk) {
              const int off = G::chunk_off(16 * sb + j, 4 * kk + g);
              const u32x4 aq = *(const u32x4 FB_LDS*)(Qs + off);
              const u32x4 ado = *(const u32x4 FB_LDS*)(dOs + off);
#pragma unroll
              for (int mc = 0; mc < MC; ++mc) {
                s[sb][mc] = E::mma_chunk(aq, kf[mc][kk], s[sb][mc]);
                dp[sb][mc] = E::mma_chunk(ado, vf[mc][kk], dp[sb][mc]);
              }
            }
        }
        __builtin_amdgcn_s_setprio(0);
        score_col_exponents<T, kCap>(a, cl, slope, c, s0, Ts, s, t);
        if (mode == 2) {
#pragma unroll
          for (int mc = 0; mc < MC; ++mc) score_mask(s[0][mc], s[1][mc], s0, cl.rows[mc]);
        }
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int mc = 0; mc < MC; ++mc) {
              const float p = fast_exp2(s[sb][mc][r]);
              pf[mc].set(4 * sb + r, p);
              if constexpr (kCap)
                dsf[mc].set(4 * sb + r, p * dp[sb][mc][r] * cap_slope(t[sb][mc][r]));
              else
                dsf[mc].set(4 * sb + r, p * dp[sb][mc][r]);
            }
#pragma unroll
        for (int nb = 0; nb < G::kNB; ++nb) {
          const typename E::AFrag ado = G::load_afrag(dOs, 16 * nb);
          const typename E::AFrag aq = G::load_afrag(Qs, 16 * nb);
#pragma unroll
          for (int mc = 0; mc < MC; ++mc) {
            dv[nb][mc] = E::mma_acc(ado, pf[mc], dv[nb][mc]);
            dk[nb][mc] = E::mma_acc(aq, dsf[mc], dk[nb][mc]);
          }
        }
        prep_next();
      });
  if constexpr (KS > 1) {
    static_assert(sizeof(sm.lds) >= merge_bytes<KS, NW, G::kNB, MC>(), "set merge buffer");
    merge_sets<KS, NW>(dk, ks, wl, (floatx4 FB_LDS*)&sm.lds[0][0][0]);
    merge_sets<KS, NW>(dv, ks, wl, (floatx4 FB_LDS*)&sm.lds[0][0][0]);
  }
  ext_store_cols<T, D, KS>(a, kv, cl.col0, cl.klen, ks, dk, dv, a.scale, 1.f, dK, dV, parts);
}

// ===========================================================================
// BoB Pass 1, as ext_pass1_kernel without its references.  With w = C + F (dP - D) and
// alpha, e the sums of P F and P w, the epilogue's
//   Qt = tau (sum P (u w - (2 / c) t (dP - D) F) k + sum u P (dP - D) u_K - e sum u P k) - alpha dQ
//   dOt = sum P u_V + sum P F v - alpha O,  E = e - alpha D
// needs, capped, one more operand, u P, beside P, which stays with u_V.  P F, u P and Pt's operand
// meet their matrices as two bf16 values each: thirteen contractions a tile for ten.  P with u_V and
// u P (dP - D) with u_K are one: the epilogue subtracts nothing from their sums, which keep a rounding
// of their terms' size.  Bound by MFMA and by a wave's chain of LDS reads, MFMA and exponentials at
// two or three waves a SIMD: B2 H16
// N2048 d128 causal 191 us with slopes, 210 with a cap; B4 H12 N4096 d64 558 and 678.
// ===========================================================================
template <typename T, int D, int MR, int NW, int OCC, int KS, int kPF, bool kCap>
__global__ __launch_bounds__(KS * NW * 64, OCC) void score_pass1_kernel(
    ScoreArgs a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ O,
    const T* __restrict__ Orest, const T* __restrict__ dO, const T* __restrict__ UQ, const T* __restrict__ UK,
    const T* __restrict__ UV, const float* __restrict__ L, const float* __restrict__ Dv, const T* __restrict__ dQ,
    T* __restrict__ Qt, T* __restrict__ dOt, float* __restrict__ alpha_out, float* __restrict__ E_out,
    float* __restrict__ parts) {
  using E = Elt<T>;
  using G = Geo<T, D>;
  constexpr int BR = 16 * MR * NW;
  __shared__ __attribute__((aligned(16))) RowSmem<T, D, 4, 2, KS, BR> sm;

  int rh, rb;
  ext_map_block(a, a.grp * a.nRB, true, a.kv_lens, a.Nk, rh, rb);
  const int l = lane_id(), g = l >> 4, j = l & 15;
  const int ks = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave_id() / NW);
  const int wl = KS == 1 ? wave_id() : __builtin_amdgcn_readfirstlane(wave_id() % NW);
  const ScoreRows<MR, NW, false> rw(a, rh, rb, wl, j);
  const int64_t kvoff = (int64_t)rw.kvh * a.Nk * D, qoff = rw.qrow * D;

  u32x4 qf[MR][G::kChunks], uqf[MR][G::kChunks], dof[MR][G::kChunks];
  float lb[MR], drow[MR];
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) {
    const int row = rw.ok(mb) ? rw.row(mb) : rw.rows;
    load_stationary<T, D>(qf[mb], Q + qoff, row, rw.rows);
    load_stationary<T, D>(uqf[mb], UQ + qoff, row, rw.rows);
    load_stationary<T, D>(dof[mb], dO + qoff, row, rw.rows);
    const float Lr = rw.ok(mb) ? L[rw.qrow + rw.row(mb)] : 0.f;
    lb[mb] = Lr == -INFINITY ? INFINITY : Lr * kLog2e;
    drow[mb] = rw.ok(mb) ? Dv[rw.qrow + rw.row(mb)] : 0.f;
  }
  floatx4 aDO[G::kNB][MR], aOM[G::kNB][MR], aB[G::kNB][MR];
#pragma unroll
  for (int nb = 0; nb < G::kNB; ++nb)
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) aDO[nb][mb] = aOM[nb][mb] = aB[nb][mb] = floatx4{0.f, 0.f, 0.f, 0.f};
  float alpha[MR], e0[MR];
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) alpha[mb] = e0[mb] = 0.f;
  const float c = kCap ? a.cap_out : score_scale(a.scale);
  const float slope = score_row_slope(a, rw, c);
  floatx4 s[2][MR], dp[2][MR], f[2][MR], cc[2][MR], t[kCap ? 2 : 1][kCap ? MR : 1];
  typename E::TFrag fP[MR], fPdd[MR];  // of a cap: P, and u P in fB
  SplitFrag<T> fPF[MR], fPPt[MR], fB[MR];
  using AF = typename E::AFrag;

  const T* const src[4] = {K + kvoff, V + kvoff, UK + kvoff, UV + kvoff};
  const int part = blockIdx.y, split = ext_parts_of(rw.tiles, KS, a.nparts);
  const ExtRun run = ext_run(rw.tiles, part, split, ks, KS), first = ext_run(rw.tiles, part, split, 0, KS);
  constexpr bool kBarrier = NW > 1;
  const TileCopy<T, D, NW, 4> copy(wl);
  ext_stream<tile_loads<T, D, NW, 4>(), kBarrier>(
      kBarrier ? first.size() : run.size(),
      [&](int it, int st) {
        copy.template issue<true>(src, (T FB_LDS*)sm.lds[ks][st], rw.key(run.begin + it), rw.kend);
      },
      []() {},
      [&](int it, int st) {
        const int s0 = rw.key(run.begin + it);
        int mode = run.begin + it < run.end ? rw.reach.mode(s0) : 0;
        if constexpr (KS > 1) mode = vector_mode(mode);
        if (mode == 0) return;
        const T FB_LDS* Ks = (const T FB_LDS*)sm.lds[ks][st];
        const T FB_LDS* Vs = Ks + G::kTileElems;
        const T FB_LDS* UKs = Vs + G::kTileElems;
        const T FB_LDS* UVs = UKs + G::kTileElems;
        if constexpr (std::is_same_v<T, bf16> && D == 128) __builtin_amdgcn_iglp_opt(3);
#pragma unroll
        for (int x = 0; x < MR; ++x) s[0][x] = s[1][x] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) {
            f[sb][mb] = cc[sb][mb] = floatx4{0.f, 0.f, 0.f, 0.f};
            dp[sb][mb] = floatx4{-drow[mb], -drow[mb], -drow[mb], -drow[mb]};
          }
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int kk = 0; kk < G::kChunks; ++kk) {
            const int off = G::chunk_off(16 * sb + j, 4 * kk + g);
            const u32x4 ak = *(const u32x4 FB_LDS*)(Ks + off), av = *(const u32x4 FB_LDS*)(Vs + off);
            const u32x4 auk = *(const u32x4 FB_LDS*)(UKs + off), auv = *(const u32x4 FB_LDS*)(UVs + off);
#pragma unroll
            for (int mb = 0; mb < MR; ++mb) {
              s[sb][mb] = E::mma_chunk(ak, qf[mb][kk], s[sb][mb]);        // S^T = K Q^T
              dp[sb][mb] = E::mma_chunk(av, dof[mb][kk], dp[sb][mb]);     // (dP - D)^T
              f[sb][mb] = E::mma_chunk(ak, uqf[mb][kk], f[sb][mb]);       // (U_Q K^T)^T
              f[sb][mb] = E::mma_chunk(auk, qf[mb][kk], f[sb][mb]);       // + (Q U_K^T)^T
              cc[sb][mb] = E::mma_chunk(auv, dof[mb][kk], cc[sb][mb]);    // C^T = U_V dO^T
            }
          }
        score_row_exponents<T, kCap>(a, rw, slope, c, s0, lb, s, t);
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int mb = 0; mb < MR; ++mb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              if constexpr (kCap)
                f[sb][mb][r] *= a.scale * cap_slope(t[sb][mb][r]);
              else
                f[sb][mb][r] *= a.scale;
            }
        AF cur[4];
        auto load_frags = [&](int nb) {
#pragma unroll
          for (int x = 0; x < 4; ++x) cur[x] = G::load_afrag(Ks + x * G::kTileElems, 16 * nb);
        };
        if constexpr (kPF != 0) load_frags(0);
        if (mode == 2) {
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) score_mask(s[0][mb], s[1][mb], s0, rw.keys[mb]);
        }
#pragma unroll
        for (int mb = 0; mb < MR; ++mb)
#pragma unroll
          for (int sb = 0; sb < 2; ++sb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float p = fast_exp2(s[sb][mb][r]);
              const float dd = dp[sb][mb][r];
              const float pf = p * f[sb][mb][r];
              const float w = __builtin_fmaf(f[sb][mb][r], dd, cc[sb][mb][r]);
              const float ppt = p * w;
              const int i = 4 * sb + r;
              alpha[mb] += pf;
              e0[mb] += ppt;
              fPF[mb].set(i, pf);
              if constexpr (kCap) {
                const float tr = t[sb][mb][r], pu = p * cap_slope(tr);
                fP[mb].set(i, p);
                fB[mb].set(i, pu);
                fPdd[mb].set(i, pu * dd);
                // P (u w - (2 / c) t (dP - D) F)
                fPPt[mb].set(i, __builtin_fmaf(pu, w, -a.cap_k * tr * (p * dd) * f[sb][mb][r]));
              } else {
                fB[mb].set(i, p);
                fPPt[mb].set(i, ppt);
                fPdd[mb].set(i, p * dd);
              }
            }
#pragma unroll
        for (int nb = 0; nb < G::kNB; ++nb) {
          AF ak, av, auk, auv;
          if constexpr (kPF != 0) {
            ak = cur[0];
            av = cur[1];
            auk = cur[2];
            auv = cur[3];
            if (nb + 1 < G::kNB) load_frags(nb + 1);
          } else {
            ak = G::load_afrag(Ks, 16 * nb);
            av = G::load_afrag(Vs, 16 * nb);
            auk = G::load_afrag(UKs, 16 * nb);
            auv = G::load_afrag(UVs, 16 * nb);
          }
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) {
            aB[nb][mb] = fB[mb].mma_acc(ak, aB[nb][mb]);
            aOM[nb][mb] = fPPt[mb].mma_acc(ak, aOM[nb][mb]);
            aOM[nb][mb] = E::mma_acc(auk, fPdd[mb], aOM[nb][mb]);
            aDO[nb][mb] = E::mma_acc(auv, kCap ? fP[mb] : fB[mb].hi, aDO[nb][mb]);
            aDO[nb][mb] = fPF[mb].mma_acc(av, aDO[nb][mb]);
          }
        }
      });
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) {
    alpha[mb] = group_sum(alpha[mb]);
    e0[mb] = group_sum(e0[mb]);
  }
  if constexpr (KS > 1) {
#pragma unroll
    for (int mb = 0; mb < MR; ++mb)
      if (g == 0) {
        sm.sc[0][ks][16 * (wl * MR + mb) + j] = alpha[mb];
        sm.sc[1][ks][16 * (wl * MR + mb) + j] = e0[mb];
      }
    __syncthreads();
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) {
      const int at = 16 * (wl * MR + mb) + j;
      alpha[mb] = sm.sc[0][0][at];
      e0[mb] = sm.sc[1][0][at];
#pragma unroll
      for (int q = 1; q < KS; ++q) {
        alpha[mb] += sm.sc[0][q][at];
        e0[mb] += sm.sc[1][q][at];
      }
    }
    static_assert(sizeof(sm.lds) >= merge_bytes<KS, NW, G::kNB, MR>(), "set merge buffer");
    floatx4 FB_LDS* buf = (floatx4 FB_LDS*)&sm.lds[0][0][0];
    merge_sets<KS, NW>(aDO, ks, wl, buf);
    merge_sets<KS, NW>(aOM, ks, wl, buf);
    merge_sets<KS, NW>(aB, ks, wl, buf);
  }
  const RowSplit<KS> own{ks, 0};
  if (a.nparts > 1) {
    const int64_t all = (int64_t)(a.total / a.nRB) * rw.rows;
    float* const sc = parts + a.nparts * all * (3 * D);
#pragma unroll
    for (int mb = 0; mb < MR; ++mb)
      if (rw.ok(mb)) {
        const int64_t at = part * all + rw.qrow + rw.row(mb);
#pragma unroll
        for (int nb = 0; nb < G::kNB; ++nb)
          if (own.owns(nb)) {
            float* const to = parts + at * (3 * D) + 16 * nb + 4 * g;
            *(floatx4*)to = aDO[nb][mb];
            *(floatx4*)(to + D) = aOM[nb][mb];
            *(floatx4*)(to + 2 * D) = aB[nb][mb];
          }
        if (g == 0 && ks == 0) {
          sc[2 * at] = alpha[mb];
          sc[2 * at + 1] = e0[mb];
        }
      }
    return;
  }
  const floatx4 zero = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) {
    if (rw.row(mb) >= rw.rows) continue;
    const int64_t at = rw.qrow + rw.row(mb);
    const bool ok = rw.ok(mb);
    if (g == 0 && ks == 0) {
      alpha_out[at] = ok ? alpha[mb] : 0.f;
      E_out[at] = ok ? e0[mb] - alpha[mb] * drow[mb] : 0.f;
    }
#pragma unroll
    for (int nb = 0; nb < G::kNB; ++nb) {
      if (!own.owns(nb)) continue;
      const int64_t off = at * D + 16 * nb + 4 * g;
      E::store4(dOt + off, ok ? aDO[nb][mb] - alpha[mb] * load_both(O, Orest, off) : zero);
      E::store4(Qt + off, ok ? a.scale * (aOM[nb][mb] - e0[mb] * aB[nb][mb]) - alpha[mb] * E::load4(dQ + off) : zero);
    }
  }
}

// Adds the parts of Pass 1 and finishes its rows, as ext_pass1_join_kernel.
template <typename T, int D>
__global__ __launch_bounds__(256) void score_pass1_join_kernel(ExtArgs a, const float* __restrict__ parts, int64_t all,
                                                               const T* __restrict__ O, const T* __restrict__ Orest,
                                                               const float* __restrict__ Dv, const T* __restrict__ dQ,
                                                               T* __restrict__ Qt, T* __restrict__ dOt,
                                                               float* __restrict__ alpha_out,
                                                               float* __restrict__ E_out) {
  using E = Elt<T>;
  constexpr int kPer = D / 4;
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = x / kPer;
  const int dim = 4 * (int)(x % kPer);
  if (row >= all) return;
  const int64_t bh = row / a.Nq, off = row * D + dim;
  const bool ok = (int)(row - bh * a.Nq) < ext_lens(a, (int)(bh / a.H)).q;
  const floatx4 zero = floatx4{0.f, 0.f, 0.f, 0.f};
  floatx4 d = zero, om = zero, b = zero;
  float alpha = 0.f, e0 = 0.f;
  if (ok) {
    const float* const scalars = parts + a.nparts * all * (3 * D);
    for (int q = 0; q < a.nparts; ++q) {
      const int64_t at = q * all + row;
      const float* const from = parts + at * (3 * D) + dim;
      d += *(const floatx4*)from;
      om += *(const floatx4*)(from + D);
      b += *(const floatx4*)(from + 2 * D);
      alpha += scalars[2 * at];
      e0 += scalars[2 * at + 1];
    }
  }
  E::store4(dOt + off, ok ? d - alpha * load_both(O, Orest, off) : zero);
  E::store4(Qt + off, ok ? a.scale * (om - e0 * b) - alpha * E::load4(dQ + off) : zero);
  if (dim == 0) {
    alpha_out[row] = alpha;
    E_out[row] = ok ? e0 - alpha * Dv[row] : 0.f;
  }
}

// ===========================================================================
// BoB Pass 2, as ext_pass2_kernel.  Its operands already hold the differences (h = F - alpha, C -
// (alpha D + E)) and are summed over queries, whose roundings do not cancel: one bf16 value each.
// Bound as Pass 1: B2 H16 N2048 d128 causal 139 us with slopes, 154 with a cap; B4 H12 N4096 d64 396
// and 528.
// ===========================================================================
template <typename T, int D, int MC, int NW, int OCC, int KS, bool kPF, bool kCap>
__global__ __launch_bounds__(KS * NW * 64, OCC) void score_pass2_kernel(
    ScoreArgs a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ dO,
    const T* __restrict__ UQ, const T* __restrict__ UK, const T* __restrict__ UV, const float* __restrict__ L,
    const float* __restrict__ Dv, const float* __restrict__ alpha_in, const float* __restrict__ E_in,
    T* __restrict__ Kt, T* __restrict__ Vt, float* __restrict__ parts) {
  using E = Elt<T>;
  using G = Geo<T, D>;
  struct Smem2 {
    T lds[KS][2][3 * G::kTileElems];
    float rawsc[KS][2][4 * kBS];
    float tsc[KS][2][4 * kBS];
  };
  __shared__ __attribute__((aligned(16))) Smem2 sm;
  extern __shared__ float slope_mem[];

  int kv, rb;
  ext_map_cols(a, kv, rb);
  const int l = lane_id(), g = l >> 4, j = l & 15;
  const int ks = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave_id() / NW);
  const int wl = __builtin_amdgcn_readfirstlane(KS == 1 ? wave_id() : wave_id() % NW);
  const ScoreCols<MC, NW> cl(a, kv, rb, wl);
  const int64_t koff = (int64_t)kv * a.Nk * D;

  u32x4 kf[MC][G::kChunks], vf[MC][G::kChunks], ukf[MC][G::kChunks], uvf[MC][G::kChunks];
#pragma unroll
  for (int mc = 0; mc < MC; ++mc) {
    const int col = cl.col0 + 16 * mc + j;
    load_stationary<T, D>(kf[mc], K + koff, col, cl.klen);
    load_stationary<T, D>(vf[mc], V + koff, col, cl.klen);
    load_stationary<T, D>(ukf[mc], UK + koff, col, cl.klen);
    load_stationary<T, D>(uvf[mc], UV + koff, col, cl.klen);
  }
  const float c = kCap ? a.cap_out : score_scale(a.scale);
  const ColSlopes slopes(a, cl, slope_mem, KS * NW * 64, c);
  floatx4 aK[G::kNB][MC], aV[G::kNB][MC];
#pragma unroll
  for (int nb = 0; nb < G::kNB; ++nb)
#pragma unroll
    for (int mc = 0; mc < MC; ++mc) aK[nb][mc] = aV[nb][mc] = floatx4{0.f, 0.f, 0.f, 0.f};
  floatx4 s[2][MC], dp[2][MC], f[2][MC], cc[2][MC];
  typename E::TFrag fPh[MC], fSt[MC], fdS[MC];

  // Transformed row scalars: T0 = -L log2e, T1 = -D (the dP tile's start), T2 = -alpha,
  // T3 = -(alpha D + E) (the C tile's start).  With h = F - alpha:
  //   P h = p h,  P (Pt - E) = p (h (dP - D) + C - (alpha D + E)),  dZ = p (dP - D).
  const int n = cl.count();
  const ExtRun run(n, cl.sub * KS + ks, cl.subs * KS), first(n, cl.sub * KS, cl.subs * KS);
  auto flat = [&](int it) { return min(run.begin + it, n - 1); };
  const TileCopy<T, D, NW, 3> copy(wl);
  stream_loop_rs<2, tile_loads<T, D, NW, 3>(), 2, true>(
      0, first.size(), __builtin_amdgcn_readfirstlane(wl) == 0,
      [&](int it, int rs) {
        const int64_t qs = (int64_t)cl.qhead(flat(it)) * a.Nq;
        const int s0 = cl.tile(flat(it)) * kBS;
        float FB_LDS* dst = (float FB_LDS*)sm.rawsc[ks][rs];
        issue_scalar_pair<true>(dst, L + qs, Dv + qs, s0, cl.qlen);
        issue_scalar_pair<true>(dst + 2 * kBS, alpha_in + qs, E_in + qs, s0, cl.qlen);
      },
      [&](int it, int st) {
        const int64_t qo = (int64_t)cl.qhead(flat(it)) * a.Nq * D;
        const T* const src[3] = {Q + qo, UQ + qo, dO + qo};
        copy.template issue<true>(src, (T FB_LDS*)sm.lds[ks][st], cl.tile(flat(it)) * kBS, cl.qlen);
      },
      [&](int, int rs, int ts) {
        if (l < kBS) {
          const float FB_LDS* raw = (const float FB_LDS*)sm.rawsc[ks][rs];
          float FB_LDS* to = (float FB_LDS*)sm.tsc[ks][ts];
          const float Lr = raw[l], Dr = raw[kBS + l], ar = raw[2 * kBS + l], Er = raw[3 * kBS + l];
          to[l] = Lr == -INFINITY ? -INFINITY : -Lr * kLog2e;
          to[kBS + l] = -Dr;
          to[2 * kBS + l] = -ar;
          to[3 * kBS + l] = -__builtin_fmaf(ar, Dr, Er);
        }
      },
      [&](int it, int st, int ts, auto&& prep_next) {
        const int s0 = cl.tile(flat(it)) * kBS;
        const int mode = vector_mode(run.begin + it < run.end ? cl.reach.mode(s0) : 0);
        if (mode == 0) {
          prep_next();
          return;
        }
        const T FB_LDS* Qs = (const T FB_LDS*)sm.lds[ks][st];
        const T FB_LDS* UQs = Qs + G::kTileElems;
        const T FB_LDS* dOs = UQs + G::kTileElems;
        const float FB_LDS* Ts = (const float FB_LDS*)sm.tsc[ks][ts];
        const float slope = score_col_slope(a, cl, slopes, flat(it));
#pragma unroll
        for (int x = 0; x < MC; ++x) s[0][x] = s[1][x] = floatx4{0.f, 0.f, 0.f, 0.f};
        if constexpr (!kCap) score_col_distance(a, cl, s0, slope, s);
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
          const floatx4 t1 = *(const floatx4 FB_LDS*)(Ts + kBS + 16 * sb + 4 * g);
          const floatx4 t3 = *(const floatx4 FB_LDS*)(Ts + 3 * kBS + 16 * sb + 4 * g);
#pragma unroll
          for (int mc = 0; mc < MC; ++mc) {
            f[sb][mc] = floatx4{0.f, 0.f, 0.f, 0.f};
            dp[sb][mc] = t1;
            cc[sb][mc] = t3;
          }
        }
        auto score_step = [&](int sb, int kk, u32x4 aq, u32x4 auq, u32x4 ado) {
#pragma unroll
          for (int mc = 0; mc < MC; ++mc) {
            s[sb][mc] = E::mma_chunk(aq, kf[mc][kk], s[sb][mc]);        // S = Q K^T
            dp[sb][mc] = E::mma_chunk(ado, vf[mc][kk], dp[sb][mc]);     // dP - D
            f[sb][mc] = E::mma_chunk(auq, kf[mc][kk], f[sb][mc]);       // U_Q K^T
            f[sb][mc] = E::mma_chunk(aq, ukf[mc][kk], f[sb][mc]);       //  + Q U_K^T
            cc[sb][mc] = E::mma_chunk(ado, uvf[mc][kk], cc[sb][mc]);    // C - (alpha D + E)
          }
        };
        auto read_step = [&](int sb, int kk, u32x4 (&o)[3]) {
          const int off = G::chunk_off(16 * sb + j, 4 * kk + g);
          o[0] = *(const u32x4 FB_LDS*)(Qs + off);
          o[1] = *(const u32x4 FB_LDS*)(UQs + off);
          o[2] = *(const u32x4 FB_LDS*)(dOs + off);
        };
        __builtin_amdgcn_s_setprio(1);
        if constexpr (kPF) {
          constexpr int kSteps = 2 * G::kChunks;
          u32x4 nx[3];
          read_step(0, 0, nx);
#pragma unroll
          for (int q = 0; q < kSteps; ++q) {
            const u32x4 aq = nx[0], auq = nx[1], ado = nx[2];
            if (q + 1 < kSteps) read_step((q + 1) / G::kChunks, (q + 1) % G::kChunks, nx);
            score_step(q / G::kChunks, q % G::kChunks, aq, auq, ado);
          }
        } else {
#pragma unroll
          for (int sb = 0; sb < 2; ++sb)
#pragma unroll
            for (int kk = 0; kk < G::kChunks; ++kk) {
              u32x4 o[3];
              read_step(sb, kk, o);
              score_step(sb, kk, o[0], o[1], o[2]);
            }
        }
        __builtin_amdgcn_s_setprio(0);
        prep_next();
        floatx4 t[kCap ? 2 : 1][kCap ? MC : 1];
        score_col_exponents<T, kCap>(a, cl, slope, c, s0, Ts, s, t);
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int mc = 0; mc < MC; ++mc)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              if constexpr (kCap)
                f[sb][mc][r] *= a.scale * cap_slope(t[sb][mc][r]);
              else
                f[sb][mc][r] *= a.scale;
            }
        typename E::AFrag cur[3];
        if constexpr (kPF) {
#pragma unroll
          for (int x = 0; x < 3; ++x) cur[x] = G::load_afrag(Qs + x * G::kTileElems, 0);
        }
        if (mode == 2) {
#pragma unroll
          for (int mc = 0; mc < MC; ++mc) score_mask(s[0][mc], s[1][mc], s0, cl.rows[mc]);
        }
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
          const floatx4 t2 = *(const floatx4 FB_LDS*)(Ts + 2 * kBS + 16 * sb + 4 * g);
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int mc = 0; mc < MC; ++mc) {
              const float p = fast_exp2(s[sb][mc][r]);
              const float h = f[sb][mc][r] + t2[r], dd = dp[sb][mc][r];
              const float w = __builtin_fmaf(h, dd, cc[sb][mc][r]);
              const int i = 4 * sb + r;
              fPh[mc].set(i, p * h);
              if constexpr (kCap) {
                const float tr = t[sb][mc][r], pu = p * cap_slope(tr);
                fSt[mc].set(i, __builtin_fmaf(pu, w, -a.cap_k * tr * (p * dd) * f[sb][mc][r]));
                fdS[mc].set(i, pu * dd);
              } else {
                fSt[mc].set(i, p * w);
                fdS[mc].set(i, p * dd);
              }
            }
        }
#pragma unroll
        for (int nb = 0; nb < G::kNB; ++nb) {
          typename E::AFrag aq, auq, ado;
          if constexpr (kPF) {
            aq = cur[0];
            auq = cur[1];
            ado = cur[2];
            if (nb + 1 < G::kNB) {
#pragma unroll
              for (int x = 0; x < 3; ++x) cur[x] = G::load_afrag(Qs + x * G::kTileElems, 16 * (nb + 1));
            }
          } else {
            aq = G::load_afrag(Qs, 16 * nb);
            auq = G::load_afrag(UQs, 16 * nb);
            ado = G::load_afrag(dOs, 16 * nb);
          }
#pragma unroll
          for (int mc = 0; mc < MC; ++mc) {
            aV[nb][mc] = E::mma_acc(ado, fPh[mc], aV[nb][mc]);
            aK[nb][mc] = E::mma_acc(aq, fSt[mc], aK[nb][mc]);
            aK[nb][mc] = E::mma_acc(auq, fdS[mc], aK[nb][mc]);
          }
        }
      });
  if constexpr (KS > 1) {
    static_assert(sizeof(sm.lds) >= merge_bytes<KS, NW, G::kNB, MC>(), "set merge buffer");
    merge_sets<KS, NW>(aK, ks, wl, (floatx4 FB_LDS*)&sm.lds[0][0][0]);
    merge_sets<KS, NW>(aV, ks, wl, (floatx4 FB_LDS*)&sm.lds[0][0][0]);
  }
  ext_store_cols<T, D, KS>(a, kv, cl.col0, cl.klen, ks, aK, aV, a.scale, 1.f, Kt, Vt, parts);
}

}  // namespace fb
