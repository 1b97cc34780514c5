// Normalised, rotated heads: each head vector of the queries and keys divided by its root mean
// square and multiplied by a weight (optional), then rotated by the angles of its position,
// forward, backward and the backward of that, and the C ABI.
//
// Per vector x of d elements with weight w, g = R^T dy (R: the rotation), a = w g, u the
// cotangent on dx, uw that on dw, and xh = r x, r = (mean x^2 + eps)^-1/2:
//   y  = R (w xh)
//   dx = r (a - (a.xh) xh / d),  dw = sum g xh
//   the gradients of <dx, u> + <dw, uw>, with A = a.u, B = a.xh, C = u.xh, S = (uw g).xh:
//   xt = r uw g - r ((r A + S) xh + r C a + r B u) / d + 3 r^2 B C xh / d^2
//   wt = sum (r g u - r C g xh / d)
//   gt = r w u - r C w xh / d + uw xh,  dyt = R gt
// Without a weight y = R x, dx = R^T dy and dyt = R u.
//
// Everything is bound by memory: each call reads and writes every vector once, whatever the
// layout (strides of batch entry, head and token), so the way from a projection's [B,N,heads,d]
// to an attention's [B,heads,N,d] is part of it.  A lane holds two runs of 16 bytes of a vector:
// a run of pairs' first halves and that of their second ones (neighbours paired: two runs of whole
// pairs, half a vector apart), so a rotation needs no other lane, and the lanes of a vector read
// and write neighbouring runs (in runs of 16 elements a lane fp32 B8 H6 N1395 d64 of neighbours
// took 33 us forward for 24).  A workgroup makes the cosines and sines of its tokens once for all heads
// of the queries or keys.
#include "fb_ext.h"

namespace fb {

// Tensor of head vectors: element strides of batch entry, head and token.
struct Heads {
  void* data;
  int64_t b, h, n;
};

struct RotaryArgs {
  int B, N, H[2];         // H: heads of the queries, of the keys
  int tokens;             // a workgroup takes at a time: a power of two up to kMaxTokens
  int pairs, num_axes;
  const int32_t* positions;  // [num_axes, B, N]
  const double* freqs;       // [pairs]: radians a position
  const int32_t* axes;       // [pairs] or null: axis 0
  const void* w[2];          // [d] or null: no norm
  const void* uw[2];         // cotangents on dw, or null: 0
  int w_bf16;
  float eps, sign;           // of the angles: -1 rotates back
  // x; y (forward) or dx; dy; u; x~; dy~
  Heads x[2], out[2], dy[2], u[2], xt[2], dyt[2];
  float* sums;               // [2][gridDim.x][d]: sums of dw or wt, or null
};

constexpr int kRotaryThreads = 256, kMaxTokens = 16;
constexpr double kTurns = 0.15915494309189535;  // 1 / (2 pi)

// Elements of a run, and lanes that share a vector (2 to 32).
template <typename T> constexpr int kRun = 16 / sizeof(T);
template <typename T, int D> constexpr int kLanes = D / (2 * kRun<T>);

// Sum over the LPV lanes that share a vector: all of them get it.
template <int LPV> __device__ __forceinline__ float vector_sum(float v) {
  auto add = [&](auto ctrl) {
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf,
                                                               0xf, true));
  };
  if constexpr (LPV >= 2) add(std::integral_constant<int, 0xb1>{});   // quad_perm 1,0,3,2
  if constexpr (LPV >= 4) add(std::integral_constant<int, 0x4e>{});   // quad_perm 2,3,0,1
  if constexpr (LPV >= 8) add(std::integral_constant<int, 0x141>{});  // row_half_mirror
  if constexpr (LPV >= 16) add(std::integral_constant<int, 0x140>{}); // row_mirror
  if constexpr (LPV >= 32) v += __shfl_xor(v, 16);
  return v;
}

// Where a lane's two runs lie in a vector, and the pair of each of its elements: E / 2 pairs from
// pair[0] and as many from pair[1] (halves apart: E in a row).  turned: whether those are rotated.
struct LanePairs {
  int a, b;
  int pair[2];
  bool turned[2];
};
template <typename T, int D, bool kNeighbours> __device__ __forceinline__ LanePairs lane_pairs(int p, int pairs) {
  constexpr int E = kRun<T>;
  LanePairs l;
  if (kNeighbours) {
    l.a = E * p;
    l.b = D / 2 + E * p;
    l.pair[0] = l.a / 2;
    l.pair[1] = l.b / 2;
  } else {
    const bool turned = E * p < pairs;
    l.a = turned ? E * p : 2 * E * p;
    l.b = turned ? pairs + E * p : 2 * E * p + E;
    l.pair[0] = E * p;
    l.pair[1] = E * p + E / 2;
  }
  l.turned[0] = l.pair[0] < pairs;
  l.turned[1] = l.pair[1] < pairs;
  return l;
}

template <typename T> __device__ __forceinline__ void unpack(u32x4 raw, float (&x)[kRun<T>]) {
  if constexpr (sizeof(T) == 2) {
    const bf16x8 v = __builtin_bit_cast(bf16x8, raw);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
  } else {
    const floatx4 v = __builtin_bit_cast(floatx4, raw);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
  }
}
// Element i of the run: of(i).
template <typename T, class F> __device__ __forceinline__ void store_run(T* p, F&& of) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (bf16)of(i);
    *(u32x4*)p = __builtin_bit_cast(u32x4, v);
  } else {
    *(floatx4*)p = floatx4{of(0), of(1), of(2), of(3)};
  }
}

// The lane's elements as E pairs (a[i], b[i]).
template <int E> struct Pairs {
  float a[E], b[E];
};
// Neighbours come as the elements of the two runs.
template <int E> __device__ __forceinline__ Pairs<E> from_neighbours(const Pairs<E>& e) {
  Pairs<E> p;
#pragma unroll
  for (int i = 0; i < E / 2; ++i) {
    p.a[i] = e.a[2 * i], p.b[i] = e.a[2 * i + 1];
    p.a[E / 2 + i] = e.b[2 * i], p.b[E / 2 + i] = e.b[2 * i + 1];
  }
  return p;
}
template <int E> __device__ __forceinline__ Pairs<E> to_neighbours(const Pairs<E>& p) {
  Pairs<E> e;
#pragma unroll
  for (int i = 0; i < E / 2; ++i) {
    e.a[2 * i] = p.a[i], e.a[2 * i + 1] = p.b[i];
    e.b[2 * i] = p.a[E / 2 + i], e.b[2 * i + 1] = p.b[E / 2 + i];
  }
  return e;
}
// The pairs of a run as it lies in memory: a load on its way.
template <typename T> struct RawPairs {
  u32x4 a, b;
  __device__ __forceinline__ void load(const T* v, const LanePairs& l) {
    a = *(const u32x4*)(v + l.a);
    b = *(const u32x4*)(v + l.b);
  }
  template <bool kNeighbours> __device__ __forceinline__ Pairs<kRun<T>> pairs() const {
    Pairs<kRun<T>> p;
    unpack<T>(a, p.a);
    unpack<T>(b, p.b);
    if constexpr (kNeighbours) return from_neighbours(p);
    return p;
  }
};
template <typename T, bool kNeighbours>
__device__ __forceinline__ void store_pairs(T* v, const LanePairs& l, const Pairs<kRun<T>>& x) {
  if constexpr (kNeighbours) {
    store_run(v + l.a, [&](int i) { return i % 2 == 0 ? x.a[i / 2] : x.b[i / 2]; });
    store_run(v + l.b, [&](int i) { return i % 2 == 0 ? x.a[(kRun<T> + i) / 2] : x.b[(kRun<T> + i) / 2]; });
  } else {
    store_run(v + l.a, [&](int i) { return x.a[i]; });
    store_run(v + l.b, [&](int i) { return x.b[i]; });
  }
}
// The lane's elements of a weight, whose type may be another than the heads'.
template <int E, bool kNeighbours>
__device__ __forceinline__ Pairs<E> load_weight(const void* w, int w_bf16, const LanePairs& l) {
  Pairs<E> p;
  auto load = [&](auto w) {
#pragma unroll
    for (int i = 0; i < E; ++i) p.a[i] = (float)w[l.a + i], p.b[i] = (float)w[l.b + i];
  };
  if (w_bf16 != 0)
    load((const bf16*)w);
  else
    load((const float*)w);
  if constexpr (kNeighbours) return from_neighbours(p);
  return p;
}

// x turned by the angles (sign 1) or back (-1).
template <int E> __device__ __forceinline__ Pairs<E> turn(const Pairs<E>& x, const Pairs<E>& cs, float sign) {
  Pairs<E> y;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float s = sign * cs.b[i];
    y.a[i] = __builtin_fmaf(x.a[i], cs.a[i], -(x.b[i] * s));
    y.b[i] = __builtin_fmaf(x.a[i], s, x.b[i] * cs.a[i]);
  }
  return y;
}
template <int E, class F> __device__ __forceinline__ Pairs<E> each(F&& f) {
  Pairs<E> y;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    y.a[i] = f([i](const Pairs<E>& p) { return p.a[i]; });
    y.b[i] = f([i](const Pairs<E>& p) { return p.b[i]; });
  }
  return y;
}
template <int LPV, int E> __device__ __forceinline__ float dot(const Pairs<E>& x, const Pairs<E>& y) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) s = __builtin_fmaf(x.a[i], y.a[i], __builtin_fmaf(x.b[i], y.b[i], s));
  return vector_sum<LPV>(s);
}

// The cosines and sines of the workgroup's tokens: four floats between tokens keep the lanes of
// different tokens on different banks.
template <int D> struct AngleMem {
  static constexpr int kStride = D / 2 + 4;
  float cs[2][kMaxTokens][kStride];
};

// What one vector's work reads.
template <typename T> struct VectorIn {
  RawPairs<T> x, g, u;
};
template <typename T, int kMode>
__device__ __forceinline__ void load_vector(const RotaryArgs& a, int k, int64_t b, int h, int64_t n, const LanePairs& l,
                                            bool norm, VectorIn<T>& v) {
  auto at = [&](const Heads& t) { return (const T*)t.data + b * t.b + h * t.h + n * t.n; };
  if (kMode == 0 || norm) v.x.load(at(a.x[k]), l);
  if (kMode == 1 || (kMode == 2 && norm)) v.g.load(at(a.dy[k]), l);
  if (kMode == 2 && a.u[k].data != nullptr) v.u.load(at(a.u[k]), l);
}

// One vector's work; kMode 0: y (or, with sign -1 and no weights, x from y); 1: dx, dw; 2: x~, dy~, w~.
template <typename T, int D, int kMode, bool kNeighbours>
__device__ __forceinline__ void rotary_vector(const RotaryArgs& a, int k, int64_t b, int h, int64_t n,
                                              const LanePairs& l, const Pairs<kRun<T>>& cs, bool norm,
                                              const Pairs<kRun<T>>& w,
                                              const Pairs<kRun<T>>& uw, const VectorIn<T>& v,
                                              Pairs<kRun<T>>& sum) {
  constexpr int LPV = kLanes<T, D>, E = kRun<T>;
  auto at = [&](const Heads& t) { return (T*)t.data + b * t.b + h * t.h + n * t.n; };
  if constexpr (kMode == 0) {
    Pairs<E> x = v.x.template pairs<kNeighbours>();
    if (norm) {
      const float r = rsqrtf(dot<LPV>(x, x) * (1.f / D) + a.eps);
      x = each<E>([&](auto of) { return of(x) * r * of(w); });
    }
    store_pairs<T, kNeighbours>(at(a.out[k]), l, turn(x, cs, 1.f));
  } else if constexpr (kMode == 1) {
    Pairs<E> g = v.g.template pairs<kNeighbours>();
    if (!norm) {
      store_pairs<T, kNeighbours>(at(a.out[k]), l, turn(g, cs, -1.f));
      return;
    }
    Pairs<E> x = v.x.template pairs<kNeighbours>();
    g = turn(g, cs, -1.f);
    const float r = rsqrtf(dot<LPV>(x, x) * (1.f / D) + a.eps);
    x = each<E>([&](auto of) { return of(x) * r; });
    const Pairs<E> aw = each<E>([&](auto of) { return of(w) * of(g); });
    const float B = dot<LPV>(aw, x) * (1.f / D);
    sum = each<E>([&](auto of) { return __builtin_fmaf(of(g), of(x), of(sum)); });
    store_pairs<T, kNeighbours>(at(a.out[k]), l,
                                each<E>([&](auto of) { return r * __builtin_fmaf(-B, of(x), of(aw)); }));
  } else {
    Pairs<E> u;
#pragma unroll
    for (int i = 0; i < E; ++i) u.a[i] = u.b[i] = 0.f;
    if (a.u[k].data != nullptr) u = v.u.template pairs<kNeighbours>();
    if (!norm) {
      store_pairs<T, kNeighbours>(at(a.dyt[k]), l, turn(u, cs, 1.f));
      return;
    }
    Pairs<E> g = v.g.template pairs<kNeighbours>(), x = v.x.template pairs<kNeighbours>();
    g = turn(g, cs, -1.f);
    const float r = rsqrtf(dot<LPV>(x, x) * (1.f / D) + a.eps);
    x = each<E>([&](auto of) { return of(x) * r; });
    const Pairs<E> aw = each<E>([&](auto of) { return of(w) * of(g); });
    const Pairs<E> ug = each<E>([&](auto of) { return of(uw) * of(g); });
    const float A = dot<LPV>(aw, u) * (1.f / D), B = dot<LPV>(aw, x) * (1.f / D);
    const float C = dot<LPV>(u, x) * (1.f / D), S = dot<LPV>(ug, x) * (1.f / D);
    const float by_x = __builtin_fmaf(3.f * r, B * C, -__builtin_fmaf(r, A, S));
    sum = each<E>([&](auto of) { return __builtin_fmaf(r * of(g), __builtin_fmaf(-C, of(x), of(u)), of(sum)); });
    store_pairs<T, kNeighbours>(at(a.xt[k]), l, each<E>([&](auto of) {
                                  const float m = __builtin_fmaf(C, of(aw), B * of(u));
                                  return r * (of(ug) + __builtin_fmaf(by_x, of(x), -r * m));
                                }));
    const Pairs<E> gt = each<E>([&](auto of) {
      return __builtin_fmaf(r * of(w), __builtin_fmaf(-C, of(x), of(u)), of(uw) * of(x));
    });
    store_pairs<T, kNeighbours>(at(a.dyt[k]), l, turn(gt, cs, 1.f));
  }
}

// A workgroup takes a.tokens tokens at a time, for which it makes the angles once, and shares the
// heads of each out over 256 / LPV / tokens slots of LPV lanes.  bf16, 16384 tokens, 16 + 8 heads of
// 128: forward 37 us (5.5 TB/s), backward 62 (4.9 TB/s, with the weights' sums); 4094 tokens, 12 + 12
// heads of 64: 10, 16 and 25 us, a chain of position, angles, vector and store a workgroup.
template <typename T, int D, int kMode, bool kNeighbours>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryArgs a) {
  constexpr int LPV = kLanes<T, D>, E = kRun<T>, kSlots = kRotaryThreads / LPV;
  __shared__ union Mem {
    AngleMem<D> angles;
    float rows[kMode == 0 ? 1 : kSlots][D + 4];  // four more: slots on different banks
  } mem;
  const int slot = threadIdx.x / LPV, p = threadIdx.x % LPV;
  const int token = slot % a.tokens, hs = slot / a.tokens, head_slots = kSlots / a.tokens;
  const LanePairs l = lane_pairs<T, D, kNeighbours>(p, a.pairs);
  const int64_t tokens = (int64_t)a.B * a.N;
  // blockIdx.y: the queries' heads, then the keys'
  const int k = blockIdx.y;
  const bool norm = a.w[k] != nullptr;
  Pairs<E> w, uw, sum;
#pragma unroll
  for (int i = 0; i < E; ++i) w.a[i] = w.b[i] = 1.f, uw.a[i] = uw.b[i] = sum.a[i] = sum.b[i] = 0.f;
  if (norm) {
    w = load_weight<E, kNeighbours>(a.w[k], a.w_bf16, l);
    if (kMode == 2 && a.uw[k] != nullptr) uw = load_weight<E, kNeighbours>(a.uw[k], a.w_bf16, l);
  }
  for (int64_t t0 = (int64_t)blockIdx.x * a.tokens; t0 < tokens; t0 += (int64_t)gridDim.x * a.tokens) {
    // a vector is on its way while the angles, or the one before it, are worked on
    const int64_t t = t0 + token;
    const unsigned b = (unsigned)t / (unsigned)a.N, n = (unsigned)t - b * (unsigned)a.N;  // t < 2^31, or not used
    const int heads = t < tokens ? a.H[k] : 0;
    VectorIn<T> v;
    if (hs < heads) load_vector<T, kMode>(a, k, b, hs, n, l, norm, v);
    for (int x = threadIdx.x; x < a.tokens * a.pairs; x += kRotaryThreads) {
      const int tk = x / a.pairs, pair = x - tk * a.pairs;
      const int axis = a.axes != nullptr ? min(max(a.axes[pair], 0), a.num_axes - 1) : 0;
      // the angle in turns, without its whole ones, in 64 bits: far positions keep their fraction
      const double turns = a.freqs[pair] * kTurns * (double)a.positions[(int64_t)axis * tokens + min(t0 + tk, tokens - 1)];
      float s, c;
      sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
      mem.angles.cs[0][tk][pair] = c;
      mem.angles.cs[1][tk][pair] = a.sign * s;
    }
    __syncthreads();
    Pairs<E> cs;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int half = i / (E / 2), pair = l.pair[half] + i % (E / 2);
      cs.a[i] = l.turned[half] ? mem.angles.cs[0][token][pair] : 1.f;
      cs.b[i] = l.turned[half] ? mem.angles.cs[1][token][pair] : 0.f;
    }
    __syncthreads();
    for (int h = hs; h < heads; h += head_slots) {
      const VectorIn<T> now = v;
      if (h + head_slots < heads) load_vector<T, kMode>(a, k, b, h + head_slots, n, l, norm, v);
      rotary_vector<T, D, kMode, kNeighbours>(a, k, b, h, n, l, cs, norm, w, uw, now, sum);
    }
  }
  if constexpr (kMode != 0) {
    if (a.sums == nullptr || !norm) return;
    // the workgroup's sums in one row
    Pairs<E> e = sum;
    if constexpr (kNeighbours) e = to_neighbours(sum);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      mem.rows[slot][l.a + i] = e.a[i];
      mem.rows[slot][l.b + i] = e.b[i];
    }
    __syncthreads();
    float* const to = a.sums + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * D;
    for (int x = threadIdx.x; x < D; x += kRotaryThreads) {
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < kSlots; ++s) v[s & 3] += mem.rows[s][x];
      to[x] = (v[0] + v[1]) + (v[2] + v[3]);
    }
  }
}

// Adds the workgroups' rows of sums: 16 columns of the queries' (blockIdx.y 0) or keys' weight a
// workgroup, 64 threads a column with eight loads in flight each, for all of it is latency
// (1024 rows: 16 threads a column 14 us for 7).
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void rotary_sums_kernel(const float* __restrict__ sums, int d, int rows,
                                                                  void* out_q, void* out_k, int w_bf16) {
  __shared__ float part[64][17];
  void* const out = blockIdx.y == 0 ? out_q : out_k;
  if (out == nullptr) return;
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, col = blockIdx.x * 16 + x;
  const float* const from = sums + (int64_t)blockIdx.y * rows * d + col;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 0.f;
  for (int r = y; r < rows; r += 512)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (r + 64 * i < rows) v[i] += from[(int64_t)(r + 64 * i) * d];
  part[y][x] = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  __syncthreads();
  if (threadIdx.x < 16) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 64; ++i) s += part[i][threadIdx.x];
    const int at = blockIdx.x * 16 + threadIdx.x;
    if (w_bf16 != 0)
      ((bf16*)out)[at] = (bf16)s;
    else
      ((float*)out)[at] = s;
  }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
struct RotaryProblem {
  int32_t dtype;
  int64_t B, H, Hkv, N, d;
  attn_rotary r;
};

// Returns BOB_OK to proceed, or an error; sets *empty where there are no vectors.
static int32_t rotary_check(const RotaryProblem& p, bool* empty) {
  *empty = false;
  if (p.dtype != BOB_F32 && p.dtype != BOB_BF16) return BOB_EINVAL;
  if (p.B < 0 || p.H < 0 || p.Hkv < 0 || p.N < 0) return BOB_EINVAL;
  if (p.d != 32 && p.d != 64 && p.d != 128 && p.d != 256) return BOB_EUNSUPPORTED;
  if (p.r.pairs < 0 || p.r.pairs % 8 != 0 || 2 * (int64_t)p.r.pairs > p.d) return BOB_EINVAL;
  if (p.r.interleaved != 0 && p.r.interleaved != 1) return BOB_EINVAL;
  auto aligned = [](const void* q, uintptr_t n) { return (reinterpret_cast<uintptr_t>(q) & (n - 1)) == 0; };
  if (p.r.q_weight != nullptr || p.r.k_weight != nullptr) {
    if (p.r.weight_dtype != BOB_F32 && p.r.weight_dtype != BOB_BF16) return BOB_EINVAL;
    if (!aligned(p.r.q_weight, 16) || !aligned(p.r.k_weight, 16)) return BOB_EINVAL;
    if (!(p.r.eps >= 0.f) || !std::isfinite(p.r.eps)) return BOB_EINVAL;
  }
  if (p.B == 0 || p.N == 0 || p.H + p.Hkv == 0) {
    *empty = true;
    return BOB_OK;
  }
  if (p.r.pairs > 0) {
    if (p.r.num_axes < 1 || p.r.positions == nullptr || p.r.freqs == nullptr) return BOB_EINVAL;
    if (!aligned(p.r.positions, 4) || !aligned(p.r.freqs, 8) || !aligned(p.r.axes, 4)) return BOB_EINVAL;
    if (p.r.num_axes > 1 && p.r.axes == nullptr) return BOB_EINVAL;
  }
  if (p.N > kMaxN || p.B > INT32_MAX || p.B * p.N > (int64_t(1) << 31) || p.H > 65535 || p.Hkv > 65535 ||
      p.H + p.Hkv > 65535)
    return BOB_EINVAL;
  return BOB_OK;
}

// How a launch runs: tokens a workgroup takes at a time, workgroups for the queries and as many
// for the keys.
struct RotaryPlan {
  int tokens;
  int64_t groups;
};
// At least as many tokens at a time as leave no slot without a head (bf16 B2 H12 N2047 d64, whose
// 32 slots met 12 heads: 12.8 us forward for 10), and more while kEnough workgroups are left.  Calls
// that sum a weight's gradient have at most kMaxSums rows of sums a weight, in workgroups that go
// on to as many further tokens as each other; a launch takes fewer than 2^32 threads.
constexpr int64_t kEnough = 1024, kMaxSums = 1024, kMaxBlocks = int64_t(1) << 22;
static RotaryPlan rotary_plan(const RotaryProblem& p, bool sums) {
  RotaryPlan c;
  const int64_t all = p.B * p.N;
  const int slots = kRotaryThreads / ((int)p.d / (p.dtype == BOB_BF16 ? 16 : 8)), most = std::min(kMaxTokens, slots);
  auto groups = [&] { return (all + c.tokens - 1) / c.tokens; };
  c.tokens = 1;
  while (c.tokens < most && slots / (2 * c.tokens) >= std::max(p.H, p.Hkv)) c.tokens *= 2;
  while (c.tokens < most && all >= 2 * kEnough * c.tokens) c.tokens *= 2;
  while (sums && c.tokens < most && groups() > kMaxSums) c.tokens *= 2;
  const int64_t limit = sums ? kMaxSums : kMaxBlocks, each = (groups() + limit - 1) / limit;
  c.groups = (groups() + each - 1) / std::max<int64_t>(each, 1);
  return c;
}
static int64_t rotary_bytes(const RotaryProblem& p) {
  if (p.r.q_weight == nullptr && p.r.k_weight == nullptr) return 0;
  return 2 * rotary_plan(p, true).groups * p.d * 4;
}

// A tensor of head vectors of `heads` heads: present, aligned, in strides that keep 16 bytes.
static bool heads_ok(const RotaryProblem& p, int64_t heads, const attn_heads* v, bool required) {
  if (heads == 0) return true;
  if (v == nullptr || v->data == nullptr) return !required;
  const int64_t unit = p.dtype == BOB_BF16 ? 8 : 4;
  return aligned16(v->data) && v->stride_b % unit == 0 && v->stride_h % unit == 0 && v->stride_n % unit == 0;
}
static Heads heads_of(const attn_heads* v) {
  return v == nullptr ? Heads{} : Heads{v->data, v->stride_b, v->stride_h, v->stride_n};
}

static RotaryArgs rotary_args(const RotaryProblem& p, const RotaryPlan& c) {
  RotaryArgs a{};
  a.B = (int)p.B;
  a.N = (int)p.N;
  a.H[0] = (int)p.H;
  a.H[1] = (int)p.Hkv;
  a.tokens = c.tokens;
  a.pairs = p.r.pairs;
  a.num_axes = p.r.num_axes;
  a.positions = p.r.positions;
  a.freqs = p.r.freqs;
  a.axes = p.r.axes;
  a.w[0] = p.r.q_weight;
  a.w[1] = p.r.k_weight;
  a.w_bf16 = p.r.weight_dtype == BOB_BF16 ? 1 : 0;
  a.eps = p.r.eps;
  a.sign = 1.f;
  return a;
}

template <int kMode> static int32_t rotary_launch(const RotaryProblem& p, const RotaryPlan& c, const RotaryArgs& a,
                                                  hipStream_t s) {
  const dim3 grid((unsigned)c.groups, 2);
  (void)hipGetLastError();
  auto go = [&](auto type, auto dim) {
    using T = decltype(type);
    constexpr int D = decltype(dim)::value;
    if (p.r.interleaved != 0)
      hipLaunchKernelGGL((rotary_kernel<T, D, kMode, true>), grid, dim3(kRotaryThreads), 0, s, a);
    else
      hipLaunchKernelGGL((rotary_kernel<T, D, kMode, false>), grid, dim3(kRotaryThreads), 0, s, a);
  };
  auto dims = [&](auto type) {
    if (p.d == 32) go(type, std::integral_constant<int, 32>{});
    if (p.d == 64) go(type, std::integral_constant<int, 64>{});
    if (p.d == 128) go(type, std::integral_constant<int, 128>{});
    if (p.d == 256) go(type, std::integral_constant<int, 256>{});
  };
  if (p.dtype == BOB_BF16)
    dims(bf16{});
  else
    dims(float{});
  return finish_launch();
}

// The workgroups' sums -> the weights' gradients.
static int32_t rotary_gather(const RotaryProblem& p, const RotaryPlan& c, const float* sums, void* out_q, void* out_k,
                             hipStream_t s) {
  hipLaunchKernelGGL(rotary_sums_kernel, dim3((unsigned)(p.d / 16), 2), dim3(kSumThreads), 0, s, sums, (int)p.d,
                     (int)c.groups, out_q, out_k, p.r.weight_dtype == BOB_BF16 ? 1 : 0);
  return finish_launch();
}

static RotaryProblem rotary_problem(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t N, int64_t d,
                                    const attn_rotary* r) {
  RotaryProblem p{dtype, B, H, Hkv, N, d, attn_rotary{}};
  if (r != nullptr) p.r = *r;
  return p;
}
// A weight's gradient: not without the weight, aligned to its type.
static bool weight_ptr(const RotaryProblem& p, const void* weight, const void* grad, uintptr_t align) {
  if (grad == nullptr) return true;
  return weight != nullptr && (reinterpret_cast<uintptr_t>(grad) & (align - 1)) == 0;
}

}  // namespace fb

using fb::RotaryProblem;

extern "C" {

int32_t attn_rotary_fwd(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t N, int64_t d, int32_t inverse,
                        const attn_rotary* rotary, const attn_heads* Q, const attn_heads* K, const attn_heads* Qr,
                        const attn_heads* Kr, void* stream) {
  const RotaryProblem p = fb::rotary_problem(dtype, B, H, Hkv, N, d, rotary);
  bool empty;
  const int32_t rc = fb::rotary_check(p, &empty);
  if (rc != BOB_OK) return rc;
  if (rotary == nullptr || (inverse != 0 && inverse != 1)) return BOB_EINVAL;
  if (inverse != 0 && (p.r.q_weight != nullptr || p.r.k_weight != nullptr)) return BOB_EINVAL;
  if (empty) return BOB_OK;
  if (!fb::heads_ok(p, H, Q, true) || !fb::heads_ok(p, Hkv, K, true) || !fb::heads_ok(p, H, Qr, true) ||
      !fb::heads_ok(p, Hkv, Kr, true))
    return BOB_EINVAL;
  const fb::RotaryPlan c = fb::rotary_plan(p, false);
  fb::RotaryArgs a = fb::rotary_args(p, c);
  a.sign = inverse != 0 ? -1.f : 1.f;
  a.x[0] = fb::heads_of(Q);
  a.x[1] = fb::heads_of(K);
  a.out[0] = fb::heads_of(Qr);
  a.out[1] = fb::heads_of(Kr);
  return fb::rotary_launch<0>(p, c, a, (hipStream_t)stream);
}

int32_t attn_rotary_bwd(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t N, int64_t d,
                        const attn_rotary* rotary, const attn_heads* Q, const attn_heads* K, const attn_heads* dQr,
                        const attn_heads* dKr, const attn_heads* dQ, const attn_heads* dK, void* dWq, void* dWk,
                        void* workspace, int64_t workspace_bytes, void* stream) {
  const RotaryProblem p = fb::rotary_problem(dtype, B, H, Hkv, N, d, rotary);
  bool empty;
  int32_t rc = fb::rotary_check(p, &empty);
  if (rc != BOB_OK) return rc;
  const uintptr_t align = p.r.weight_dtype == BOB_F32 ? 4 : 2;
  if (rotary == nullptr || !fb::weight_ptr(p, p.r.q_weight, dWq, align) ||
      !fb::weight_ptr(p, p.r.k_weight, dWk, align))
    return BOB_EINVAL;
  const bool sums = dWq != nullptr || dWk != nullptr;
  if (empty && !sums) return BOB_OK;
  fb::RotaryPlan c{};
  if (!empty) {
    if (!fb::heads_ok(p, H, Q, p.r.q_weight != nullptr) || !fb::heads_ok(p, Hkv, K, p.r.k_weight != nullptr) ||
        !fb::heads_ok(p, H, dQr, true) || !fb::heads_ok(p, Hkv, dKr, true) || !fb::heads_ok(p, H, dQ, true) ||
        !fb::heads_ok(p, Hkv, dK, true))
      return BOB_EINVAL;
    if (sums && (workspace_bytes < fb::rotary_bytes(p) || !fb::aligned16(workspace))) return BOB_EINVAL;
    c = fb::rotary_plan(p, sums);
    fb::RotaryArgs a = fb::rotary_args(p, c);
    a.x[0] = fb::heads_of(Q);
    a.x[1] = fb::heads_of(K);
    a.dy[0] = fb::heads_of(dQr);
    a.dy[1] = fb::heads_of(dKr);
    a.out[0] = fb::heads_of(dQ);
    a.out[1] = fb::heads_of(dK);
    a.sums = sums ? (float*)workspace : nullptr;
    rc = fb::rotary_launch<1>(p, c, a, (hipStream_t)stream);
  }
  return rc == BOB_OK && sums ? fb::rotary_gather(p, c, (const float*)workspace, dWq, dWk, (hipStream_t)stream) : rc;
}

int32_t attn_rotary_bwd2(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t N, int64_t d,
                         const attn_rotary* rotary, const attn_heads* Q, const attn_heads* K, const attn_heads* dQr,
                         const attn_heads* dKr, const attn_heads* gdQ, const attn_heads* gdK, const void* gdWq,
                         const void* gdWk, const attn_heads* Qt, const attn_heads* Kt, const attn_heads* dQrt,
                         const attn_heads* dKrt, void* Wqt, void* Wkt, void* workspace, int64_t workspace_bytes,
                         void* stream) {
  const RotaryProblem p = fb::rotary_problem(dtype, B, H, Hkv, N, d, rotary);
  bool empty;
  int32_t rc = fb::rotary_check(p, &empty);
  if (rc != BOB_OK) return rc;
  const uintptr_t align = p.r.weight_dtype == BOB_F32 ? 4 : 2;
  if (rotary == nullptr || !fb::weight_ptr(p, p.r.q_weight, Wqt, align) ||
      !fb::weight_ptr(p, p.r.k_weight, Wkt, align) || !fb::weight_ptr(p, p.r.q_weight, gdWq, 16) ||
      !fb::weight_ptr(p, p.r.k_weight, gdWk, 16))
    return BOB_EINVAL;
  const bool sums = Wqt != nullptr || Wkt != nullptr;
  if (empty && !sums) return BOB_OK;
  fb::RotaryPlan c{};
  if (!empty) {
    const bool nq = p.r.q_weight != nullptr, nk = p.r.k_weight != nullptr;
    if (!fb::heads_ok(p, H, Q, nq) || !fb::heads_ok(p, Hkv, K, nk) || !fb::heads_ok(p, H, dQr, nq) ||
        !fb::heads_ok(p, Hkv, dKr, nk) || !fb::heads_ok(p, H, gdQ, false) || !fb::heads_ok(p, Hkv, gdK, false) ||
        !fb::heads_ok(p, H, Qt, nq) || !fb::heads_ok(p, Hkv, Kt, nk) || !fb::heads_ok(p, H, dQrt, true) ||
        !fb::heads_ok(p, Hkv, dKrt, true))
      return BOB_EINVAL;
    if (sums && (workspace_bytes < fb::rotary_bytes(p) || !fb::aligned16(workspace))) return BOB_EINVAL;
    c = fb::rotary_plan(p, sums);
    fb::RotaryArgs a = fb::rotary_args(p, c);
    a.x[0] = fb::heads_of(Q);
    a.x[1] = fb::heads_of(K);
    a.dy[0] = fb::heads_of(dQr);
    a.dy[1] = fb::heads_of(dKr);
    a.u[0] = fb::heads_of(gdQ);
    a.u[1] = fb::heads_of(gdK);
    a.uw[0] = gdWq;
    a.uw[1] = gdWk;
    a.xt[0] = fb::heads_of(Qt);
    a.xt[1] = fb::heads_of(Kt);
    a.dyt[0] = fb::heads_of(dQrt);
    a.dyt[1] = fb::heads_of(dKrt);
    a.sums = sums ? (float*)workspace : nullptr;
    rc = fb::rotary_launch<2>(p, c, a, (hipStream_t)stream);
  }
  return rc == BOB_OK && sums ? fb::rotary_gather(p, c, (const float*)workspace, Wqt, Wkt, (hipStream_t)stream) : rc;
}

int64_t attn_rotary_workspace_bytes(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t N, int64_t d,
                                    const attn_rotary* rotary) {
  const RotaryProblem p = fb::rotary_problem(dtype, B, H, Hkv, N, d, rotary);
  bool empty;
  return fb::rotary_check(p, &empty) != BOB_OK || empty ? 0 : fb::rotary_bytes(p);
}

}  // extern "C"
