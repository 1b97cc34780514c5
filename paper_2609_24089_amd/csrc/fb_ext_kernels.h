// Attention between sequences of two lengths, with an optional bias on the scores that
// depends on the bucket of the key's position minus the query's: forward, first backward
// and the two BoB passes as gfx950 kernels.
//
// The problem generalises that of fb_kernels.h.  Per batch entry and query head
//   S = tau Q K^T + T[bucket(clamp(pos_k - pos_q, -R, R))],  P = softmax over valid keys,
// with Nq query and Nk key rows, of which the first q_len and kv_len are valid; key row j
// has position j, query row i position start + i, and under the causal mask key j is valid
// for query i where j <= start + i.  A row without a valid key has P = 0, O = 0, L = -inf.
// The first backward adds dT[c] = sum of dS over the pairs of bucket c (S holds the bias
// with factor 1), so the BoB's F gains U_T[bucket] (U_T the cotangent on dT) where it has
// tau (U_Q K^T + Q U_K^T), and Tt[c] is the sum of St over bucket c; every other identity
// stands as it is.
//
// The kernels keep the skeleton of fb_common.h: a workgroup owns stationary rows, the
// other side streams through LDS in 32-row tiles.  What is new:
//  * Bias.  The workgroup writes its head's bias for every step of position from -(R + 64)
//    to R + 64 into LDS, times log2(e).  A wave's tile covers at most 63 steps, so a tile
//    that meets (-R, R) reads one float an element at a fixed offset from one lane address,
//    with no clamp, and every other tile has one bias for all its elements, added where the
//    row's maximum or L is.  Long sequences are nearly all of the second kind.
//  * Table gradients.  A column kernel's wave streams query tiles in order, so the steps
//    that a tile meets lie in two windows of 32, the upper of which no later tile meets.
//    A near tile's blocks of equal step are added, summed along their diagonals by shifts
//    inside a row of 16 lanes, and the four lane groups meet in a small LDS buffer of the
//    wave's own; the upper window is stored, the lower carried in a register; far tiles add
//    to one sum a side.  Each wave stores its own row of sums, so there are no atomics and
//    the order is fixed; one kernel adds the rows and gathers the steps into buckets (from
//    257 rows a head on after another that adds most of them).
//  * Sets and parts.  Wave sets (KS) and workgroups (parts) that share stationary rows
//    take one run of consecutive tiles each.
#pragma once
#include "fb_common.h"

namespace fb {

constexpr int kStepPad = 64;  // steps of bias kept beyond R on either side

struct ExtArgs {
  int H, grp;          // query heads of a batch entry, query heads that share a key/value head
  int Nq, Nk;
  int nRB, total;      // blocks a head, blocks of the problem
  int block0, blocks;  // column kernels: those of this launch are block0 .. block0 + blocks - 1
  int64_t row0, rows;  // and their key rows, counted over all key/value heads
  int causal;
  int fold;            // row kernels: the rows of the grp query heads of a key/value head form one matrix
  float scale;
  int nparts;
  int resident;        // of balanced_order(): causal grids of a few rounds
  int fit;             // workgroups of the kernel that fit a compute unit
  const int32_t* q_lens;    // [B] or null: every row is valid
  const int32_t* kv_lens;
  const int32_t* q_starts;  // [B] or null: 0
  const void* table;        // [num_buckets, H], fp32 or bf16
  const void* dir;          // U_T in the same layout and type, or null: 0
  const int32_t* buckets;   // [2 R + 1]
  int table_bf16, num_buckets, R;
};

// Valid rows of a batch entry, and the position of its first query.
struct ExtLens {
  int q, k, start;
};
__device__ __forceinline__ ExtLens ext_lens(const ExtArgs& a, int b) {
  ExtLens n;
  n.q = a.q_lens != nullptr ? min(max(a.q_lens[b], 0), a.Nq) : a.Nq;
  n.k = a.kv_lens != nullptr ? min(max(a.kv_lens[b], 0), a.Nk) : a.Nk;
  // positions stay far from the ends of an int
  n.start = a.q_starts != nullptr ? min(max(a.q_starts[b], -(1 << 29)), 1 << 29) : 0;
  return n;
}

// ---------------------------------------------------------------------------
// Bias by steps of position
// ---------------------------------------------------------------------------
__device__ __forceinline__ int ext_steps(const ExtArgs& a) { return 2 * (a.R + kStepPad) + 1; }

__device__ __forceinline__ float ext_table(const ExtArgs& a, const void* t, int bucket, int head) {
  const int64_t at = (int64_t)bucket * a.H + head;
  return a.table_bf16 != 0 ? (float)((const bf16*)t)[at] : ((const float*)t)[at];
}

// The bias of heads head0 .. head0 + heads - 1 at every step, `count` threads of the
// workgroup at work: dst[hh * steps + R + kStepPad + step].  As an exponent (kExp) it is
// times log2(e), and an entry of kMaskedEntry or less masks its bucket's keys.  At that size a
// score in fp32 has no fraction left: L rounds its logarithm of the weights' sum away, and P,
// which the backward kernels take from L, would be that sum too large in a row that sees such
// keys alone; the product with log2(e) of a lowest value overflows.
constexpr float kMaskedEntry = -16777216.f;
template <bool kExp>
__device__ __forceinline__ void ext_fill_steps(const ExtArgs& a, const void* t, int head0, int heads, float FB_LDS* dst,
                                               int count) {
  const int steps = ext_steps(a);
  for (int x = threadIdx.x; x < heads * steps; x += count) {
    float v = 0.f;
    if (t != nullptr) {
      const int hh = x / steps, at = x - hh * steps - kStepPad;
      const int bucket = min(max(a.buckets[min(max(at, 0), 2 * a.R)], 0), a.num_buckets - 1);
      v = ext_table(a, t, bucket, head0 + hh);
      if (kExp) v = v <= kMaskedEntry ? -INFINITY : v * kLog2e;
    }
    dst[x] = v;
  }
}

// A wave's tile whose steps are lo .. hi: -1 all at or below -R, 1 all at or above R (one
// bias each), 0 mixed.
__device__ __forceinline__ int ext_side(int lo, int hi, int R) { return hi <= -R ? -1 : lo >= R ? 1 : 0; }

// ---------------------------------------------------------------------------
// Tile loop of the row kernels: as stream_loop with opaque copies into a ring of two stages,
// a callback that runs while the first tiles are on their way, and (kBarrier false: one wave
// a set, which alone writes and reads its ring) no barrier but the first.
// ---------------------------------------------------------------------------
template <int LT, bool kBarrier, class Issue, class Pro, class Body>
__device__ __forceinline__ void ext_stream(int n, Issue&& issue, Pro&& pro, Body&& body) {
  if (n > 0) issue(0, 0);
  if (!kBarrier && n > 1) issue(1, 1);
  pro();
  if constexpr (kBarrier) wait_copies<true>();
  __syncthreads();
  auto step = [&](int k, auto cur) {
    constexpr int kCur = decltype(cur)::value;
    if constexpr (kBarrier) {
      if (k + 1 < n) issue(k + 1, 1 - kCur);
      body(k, kCur);
      wait_copies<true>();
      __syncthreads();
    } else {
      if (k + 1 < n)
        wait_vm<LT>();
      else
        wait_copies<true>();
      body(k, kCur);
      // the stage is filled again as soon as its tile is done: the wave's own reads of it have
      // to be back before (lgkmcnt(0), the other counters at their maxima)
      __builtin_amdgcn_s_waitcnt(0xc07f);
      if (k + 2 < n) issue(k + 2, kCur);
    }
  };
  for (int k = 0; k < n; k += 2) {
    step(k, std::integral_constant<int, 0>{});
    if (k + 1 < n) step(k + 1, std::integral_constant<int, 1>{});
  }
}

// A tile's mode in a vector register: the wave indices are scalar, and a branch on a scalar
// mode made the compiler merge the tile's body with the loop around it and spill hundreds of
// registers (cross attention's column kernel at d = 128: 2.9 ms for 0.47 ms).
__device__ __forceinline__ int vector_mode(int mode) {
  asm volatile("" : "+v"(mode));
  return mode;
}

// A value that is the same in all lanes of the wave, in a scalar register.
__device__ __forceinline__ float scalar(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}

// Run `index` of `count` equal runs over n tiles.  The division leaves its ends in vector
// registers: there Pass 1 with a bias at d = 64 took 188 of them for 168 and lost its third wave
// per SIMD (B4 H12 N4096 dense 1021 us for 967), and at d = 128 it
// spilled ten in its loop (B2 H16 N4096 1631 us for 1135).
struct ExtRun {
  int begin, end;
  __device__ __forceinline__ ExtRun(int n, int index, int count) {
    const int per = (n + count - 1) / count;
    begin = __builtin_amdgcn_readfirstlane(min(index * per, n));
    end = __builtin_amdgcn_readfirstlane(min(begin + per, n));
  }
  __device__ __forceinline__ int size() const { return end - begin; }
};

// The parts that split a row block's tiles, of nparts: each set of a part gets four tiles at
// least, the parts beyond take none.
__device__ __forceinline__ int ext_parts_of(int tiles, int sets, int nparts) {
  return min(max(tiles / (4 * sets), 1), nparts);
}
// The run of set ks of part `part`.
__device__ __forceinline__ ExtRun ext_run(int tiles, int part, int split, int ks, int sets) {
  ExtRun r(tiles, min(part, split) * sets + ks, split * sets);
  return r;
}

// What a row kernel's workgroup and wave know of their rows.  kFold: the kernel may run
// folded rows (a.fold); the others keep one lane position instead of one a 16-row block.
template <int MR, int NW, bool kFold>
struct ExtRows {
  int b, kvh, head0, rows;   // batch entry, key/value head, first query head, rows of the matrix
  int64_t qrow;              // its first row among all query rows
  int kvis, tiles;           // keys that some row of the workgroup sees, their tiles
  int lo, hi;                // least and largest last valid key over the wave's rows
  int plo, phi;              // least and largest query position of the wave
  int row0, qlen, Nq, start; // the lane's first row; valid rows of the entry, its rows, its first position
  bool fold, causal;

  __device__ __forceinline__ ExtRows(const ExtArgs& a, int rh, int rb, int wl, int j) {
    constexpr int BR = 16 * MR * NW;
    fold = kFold && a.fold != 0;
    causal = a.causal != 0;
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
    const int first = rb * BR + wl * 16 * MR;
    row0 = first + j;
    // the last valid query of the workgroup; folded rows hold every query of each head
    const int last = fold ? n.q - 1 : min(rb * BR + BR, n.q) - 1;
    const bool none = fold ? n.q == 0 : n.q <= rb * BR;
    kvis = none ? 0 : causal ? max(min(n.k, n.start + last + 1), 0) : n.k;
    tiles = (kvis + kBS - 1) / kBS;
    plo = n.start + (fold ? 0 : first);
    phi = fold ? n.start + a.Nq - 1 : plo + 16 * MR - 1;
    lo = causal ? min(kvis - 1, plo) : kvis - 1;
    hi = causal ? min(kvis - 1, phi) : kvis - 1;
  }
  __device__ __forceinline__ int row(int mb) const { return row0 + 16 * mb; }
  __device__ __forceinline__ int query(int mb) const { return fold ? row(mb) % Nq : row(mb); }
  __device__ __forceinline__ int pos(int mb) const { return start + query(mb); }
  __device__ __forceinline__ int klim(int mb) const { return causal ? min(kvis - 1, pos(mb)) : kvis - 1; }  // last valid key
  __device__ __forceinline__ bool ok(int mb) const { return row(mb) < rows && query(mb) < qlen; }
  // 0: no valid key of the tile at s0, 1: all valid for every row, 2: mixed
  __device__ __forceinline__ int mode(int s0) const { return s0 > hi ? 0 : s0 + kBS - 1 <= lo ? 1 : 2; }
};

// The batch entry with the `rank`-th largest length (equal ones in order), 2 to 64 entries:
// each lane ranks one.
__device__ __forceinline__ int entry_of_rank(const int32_t* lens, int entries, int limit, int rank) {
  const int l = lane_id();
  const int n = l < entries ? min(max(lens[l], 0), limit) : -1;
  int above = 0;
  for (int q = 0; q < entries; ++q) {
    const int other = __builtin_amdgcn_readlane(n, q);
    above += other > n || (other == n && q < l) ? 1 : 0;
  }
  return __builtin_ctzll(__builtin_amdgcn_ballot_w64(l < entries && above == rank));
}

// Which block a workgroup runs.  As map_block, one head's blocks stay on one XCD, whose L2
// its key/value head's tensors then pass once; but units of heads that share a key/value
// head go round the XCDs one by one where their number allows it, so that the entries of a
// ragged batch spread over all of them (in map_block's runs of consecutive heads an XCD got
// the longest entry's heads and another the shortest's: 3 to 10% slower on such batches).
// `lens`: the streamed side's lengths, or null.  With them the longest entries' blocks start
// first, and in the rounds that become resident together each XCD deals them to its CUs in
// alternating direction, as map_block_causal does: a CU gets a long block and a short one.
// Causal grids of a few rounds run in map_block_causal's order.  `per`: blocks of one unit.
__device__ __forceinline__ void ext_map_block(const ExtArgs& a, int per, bool last_heavy, const int32_t* lens, int limit,
                                              int& head, int& rb) {
  if (a.resident > 0) {
    map_block_causal(a.nRB, a.total, a.resident, last_heavy, head, rb);
    return;
  }
  const int units = a.total / per, entry_units = a.H / a.grp, entries = units / entry_units;
  if (units % kXCDs != 0) {
    map_block(a.nRB, a.total, head, rb, last_heavy && a.causal != 0);
    return;
  }
  const int xcd = blockIdx.x % kXCDs;
  int i = blockIdx.x / kXCDs;
  const bool ranked = lens != nullptr && entries > 1 && entries <= 64;
  if (ranked) {
    const int round = i / kCUsPerXCD, first = round * kCUsPerXCD;
    const int m = min(kCUsPerXCD, a.total / kXCDs - first);
    if ((round & 1) != 0 && round < a.fit) i = first + m - 1 - (i - first);
  }
  int u = i / per;
  const int at = i - u * per, h = at / a.nRB;
  u = u * kXCDs + xcd;
  if (ranked) {
    const int rank = u / entry_units;
    u += (entry_of_rank(lens, entries, limit, rank) - rank) * entry_units;
  }
  head = u * (per / a.nRB) + h;
  rb = at - h * a.nRB;
  if (last_heavy && a.causal != 0) rb = a.nRB - 1 - rb;
}

// The block of a column kernel's workgroup.  A slice of the problem's blocks has a run of
// consecutive ones on each XCD.
__device__ __forceinline__ void ext_map_cols(const ExtArgs& a, int& head, int& rb) {
  if (a.blocks == a.total) {
    ext_map_block(a, a.nRB, false, a.q_lens, a.Nq, head, rb);
    return;
  }
  const int xcd = blockIdx.x % kXCDs, each = a.blocks / kXCDs, more = a.blocks % kXCDs;
  const int id = a.block0 + xcd * each + min(xcd, more) + blockIdx.x / kXCDs;
  head = id / a.nRB;
  rb = id - head * a.nRB;
}

// Exponents of invalid keys to -inf: x[sb][r] belongs to key s0 + 16 sb + 4 (l >> 4) + r.
__device__ __forceinline__ void ext_mask1(floatx4 (&x)[2], int s0, int klim) {
  const int g = lane_id() >> 4;
#pragma unroll
  for (int sb = 0; sb < 2; ++sb)
#pragma unroll
    for (int r = 0; r < 4; ++r) x[sb][r] = s0 + 16 * sb + 4 * g + r <= klim ? x[sb][r] : -INFINITY;
}

// ===========================================================================
// Forward.  As attn_fwd_kernel (online softmax against a lazily moved reference), over the
// keys of another sequence, with the bias.  A part (gridDim.y of them) takes a run of the
// key tiles (none, if the block has few) and stores its unnormalised sums, reference and weight instead of O and L;
// ext_fwd_join_kernel joins them.  One wave a set (NW = 1) runs without barriers: the form
// of a few query rows against a long cache, which reads each key and value once.
// Bound by the keys' and values' bytes for a few rows (B32 H32 Hkv8, one token, up to 4096
// keys, d128: 403 MB in 77 us, 5.2 TB/s, what a large copy reaches), by MFMA and VALU issue
// for many (B1 H16 N8192 d128 causal with a bias: 262 us, 1.05 PFLOP/s; B4 H12 N4096 d64 0.85 and
// dense 0.92, where an element's exponential meets half the MFMA work).
// ===========================================================================
template <typename T, int D, int MR, int NW, int OCC, int KS, bool kBias>
__global__ __launch_bounds__(KS * NW * 64, OCC) void ext_fwd_kernel(
    ExtArgs a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, T* __restrict__ O,
    float* __restrict__ L, float* __restrict__ parts) {
  using E = Elt<T>;
  using G = Geo<T, D>;
  constexpr int BR = 16 * MR * NW;
  __shared__ __attribute__((aligned(16))) RowSmem<T, D, 2, 2, KS, BR> sm;
  extern __shared__ float steps_mem[];
  float FB_LDS* const steps = (float FB_LDS*)steps_mem;

  int rh, rb;
  // a few rows a head: every workgroup is resident, whatever the order
  ext_map_block(a, a.fold != 0 ? a.nRB : a.grp * a.nRB, true, NW == 1 ? nullptr : a.kv_lens, a.Nk, rh, rb);
  const int l = lane_id(), g = l >> 4, j = l & 15;
  const int ks = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave_id() / NW);
  const int wl = __builtin_amdgcn_readfirstlane(KS == 1 ? wave_id() : wave_id() % NW);
  const ExtRows<MR, NW, MR == 1> rw(a, rh, rb, wl, j);
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
  float mrun[MR], lsum[MR], blo[MR], bhi[MR];
  int tb[MR];  // the lane's head in `steps`, at key 0
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) {
    mrun[mb] = -1e30f;
    lsum[mb] = blo[mb] = bhi[mb] = 0.f;
    tb[mb] = 0;
  }
  const float c = a.scale * kLog2e;
  floatx4 s[2][MR];
  typename E::TFrag pf[MR];

  // s times cf plus kb are the scores in log2 units (cf = 1 and kb = 0 where a near tile's
  // bias went into s)
  auto softmax_step = [&](int s0, int mode, float cf, const float (&kb)[MR]) {
    float p[MR][8], ls[MR];
    bool grown = false;
    floatx4 e[MR][2];
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) {
      const float off = kb[mb] - mrun[mb];
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int r = 0; r < 4; ++r) e[mb][sb][r] = __builtin_fmaf(s[sb][mb][r], cf, off);
    }
    if (mode == 2) {
#pragma unroll
      for (int mb = 0; mb < MR; ++mb) ext_mask1(e[mb], s0, rw.klim(mb));
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
          for (int r = 0; r < 4; ++r) x[sb][r] = __builtin_fmaf(s[sb][mb][r], cf, kb[mb]);
        if (mode == 2) ext_mask1(x, s0, rw.klim(mb));
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) mx = fmaxf(mx, x[i >> 2][i & 3]);
        mx = group_max(mx);
        if (__builtin_amdgcn_ballot_w64(mx > mrun[mb] + kRescaleLog2) != 0) {
          const float mnew = fmaxf(mrun[mb], mx);
          const float corr = fast_exp2(mrun[mb] - mnew);
          mrun[mb] = mnew;
          lsum[mb] *= corr;
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
    }
  };

  const T* const src[2] = {K + kvoff, V + kvoff};
  // every set of a workgroup with barriers runs as long as its first, whose run is the longest
  const int split = ext_parts_of(rw.tiles, KS, a.nparts);
  const ExtRun run = ext_run(rw.tiles, part, split, ks, KS), first = ext_run(rw.tiles, part, split, 0, KS);
  constexpr bool kBarrier = NW > 1;
  const int iters = kBarrier ? first.size() : run.size();
  const TileCopy<T, D, NW, 2> copy(wl);
  ext_stream<tile_loads<T, D, NW, 2>(), kBarrier>(
      iters,
      [&](int it, int st) {
        copy.template issue<true>(src, (T FB_LDS*)sm.lds[ks][st], min(run.begin + it, rw.tiles - 1) * kBS, rw.kvis);
      },
      [&]() {
        if constexpr (kBias) {
          const int n = ext_steps(a);
          const int h0 = rw.fold ? rb * BR / a.Nq : 0;  // folded: the heads of this block's rows
          const int h1 = rw.fold ? (min(rb * BR + BR, rw.rows) - 1) / a.Nq : 0;
          ext_fill_steps<true>(a, a.table, rw.head0 + h0, h1 - h0 + 1, steps, KS * NW * 64);
          __syncthreads();
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) {
            const int hh = rw.fold ? min(rw.row(mb), rw.rows - 1) / a.Nq - h0 : 0;
            blo[mb] = steps[hh * n];
            bhi[mb] = steps[hh * n + n - 1];
            tb[mb] = hh * n + a.R + kStepPad - rw.pos(mb);
          }
        }
      },
      [&](int it, int st) {
        const int s0 = min(run.begin + it, rw.tiles - 1) * kBS;
        const int mode = vector_mode(run.begin + it < run.end ? rw.mode(s0) : 0);
        if (mode == 0) return;
        const T FB_LDS* Ks = (const T FB_LDS*)sm.lds[ks][st];
        const T FB_LDS* Vs = Ks + G::kTileElems;
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) s[sb][mb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int kk = 0; kk < G::kChunks; ++kk) {
            const u32x4 ak = *(const u32x4 FB_LDS*)(Ks + G::chunk_off(16 * sb + j, 4 * kk + g));
#pragma unroll
            for (int mb = 0; mb < MR; ++mb) s[sb][mb] = E::mma_chunk(ak, qf[mb][kk], s[sb][mb]);
          }
        float cf = c, kb[MR];
#pragma unroll
        for (int mb = 0; mb < MR; ++mb) kb[mb] = 0.f;
        if constexpr (kBias) {
          const int side = ext_side(s0 - rw.phi, s0 + kBS - 1 - rw.plo, a.R);
          if (side != 0) {
#pragma unroll
            for (int mb = 0; mb < MR; ++mb) kb[mb] = side < 0 ? blo[mb] : bhi[mb];
          } else {
            cf = 1.f;
#pragma unroll
            for (int mb = 0; mb < MR; ++mb) {
              const float FB_LDS* bias = steps + tb[mb] + s0 + 4 * g;
#pragma unroll
              for (int sb = 0; sb < 2; ++sb)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[sb][mb][r] = __builtin_fmaf(s[sb][mb][r], c, bias[16 * sb + r]);
            }
          }
        }
        softmax_step(s0, mode, cf, kb);
#pragma unroll
        for (int nb = 0; nb < G::kNB; ++nb) {
          const typename E::AFrag av = G::load_afrag(Vs, 16 * nb);
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) acc[nb][mb] = E::mma_acc(av, pf[mb], acc[nb][mb]);
        }
      });
  float lt[MR];
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) lt[mb] = group_sum(lsum[mb]);
  if constexpr (KS > 1) {
    // bring the sets to one reference and add them, as in attn_fwd_kernel; without the
    // loop's barriers the rings are free once every wave is here
#pragma unroll
    for (int mb = 0; mb < MR; ++mb)
      if (g == 0) {
        sm.sc[0][ks][16 * (wl * MR + mb) + j] = mrun[mb];
        sm.sc[1][ks][16 * (wl * MR + mb) + j] = lt[mb];
      }
    __syncthreads();
#pragma unroll
    for (int mb = 0; mb < MR; ++mb) {
      const int at = 16 * (wl * MR + mb) + j;
      float m = sm.sc[0][0][at], sum = 0.f;
#pragma unroll
      for (int q = 1; q < KS; ++q) m = fmaxf(m, sm.sc[0][q][at]);
#pragma unroll
      for (int q = 0; q < KS; ++q) sum = __builtin_fmaf(sm.sc[1][q][at], fast_exp2(sm.sc[0][q][at] - m), sum);
      const float corr = fast_exp2(mrun[mb] - m);
      mrun[mb] = m;
      lt[mb] = sum;
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
        if (g == 0 && ks == 0) {
          ml[2 * at] = mrun[mb];
          ml[2 * at + 1] = lt[mb];
        }
      }
    return;
  }
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) {
    if (rw.row(mb) >= rw.rows) continue;
    const int64_t at = rw.qrow + rw.row(mb);
    const bool some = rw.ok(mb) && lt[mb] != 0.f;
    const float inv = 1.f / lt[mb];
#pragma unroll
    for (int nb = 0; nb < G::kNB; ++nb)
      if (own.owns(nb))
        E::store4(O + at * D + 16 * nb + 4 * g, some ? acc[nb][mb] * inv : floatx4{0.f, 0.f, 0.f, 0.f});
    if (g == 0 && ks == 0) L[at] = some ? (mrun[mb] + __log2f(lt[mb])) * kLn2 : -INFINITY;
  }
}

// Joins the parts of the forward: every part's sums brought to the largest reference.
// One thread for four head dims of a row.
template <typename T, int D>
__global__ __launch_bounds__(256) void ext_fwd_join_kernel(ExtArgs a, const float* __restrict__ parts, int64_t all,
                                                           T* __restrict__ O, float* __restrict__ L) {
  using E = Elt<T>;
  constexpr int kPer = D / 4;
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = x / kPer;
  const int dim = 4 * (int)(x % kPer);
  if (row >= all) return;
  const int64_t bh = row / a.Nq;
  const bool ok = (int)(row - bh * a.Nq) < ext_lens(a, (int)(bh / a.H)).q;
  const float* const ml = parts + a.nparts * all * D;
  floatx4 sum = floatx4{0.f, 0.f, 0.f, 0.f};
  float m = -1e30f, w = 0.f;
  if (ok) {
    for (int q = 0; q < a.nparts; ++q) m = fmaxf(m, ml[2 * (q * all + row)]);
    for (int q = 0; q < a.nparts; ++q) {
      const int64_t at = q * all + row;
      const float f = fast_exp2(ml[2 * at] - m);
      w = __builtin_fmaf(ml[2 * at + 1], f, w);
      sum += *(const floatx4*)(parts + at * D + dim) * f;
    }
  }
  const bool some = ok && w != 0.f;
  E::store4(O + row * D + dim, some ? sum * (1.f / w) : floatx4{0.f, 0.f, 0.f, 0.f});
  if (dim == 0) L[row] = some ? (m + __log2f(w)) * kLn2 : -INFINITY;
}

// ===========================================================================
// First backward, row side: as attn_bwd_rows_kernel.  D is the exact sum_j P_ij dP_ij in
// fp32: the tiles form dP minus do_i . o_i, whose o_i is rounded to the tensors' type, and
// D_i adds what sum_j P_ij (dP_ij - do_i . o_i) is off zero.  The table's gradient is a
// sum over many rows of fp32 products, and that rounding of o would be its largest error
// by far (2^-8 of D a row against 2^-24).  In dQ it matters where few keys share a row's
// weight (a row of one key has dQ = 0): a row whose whole weight lies in a set's first tile
// takes D from that tile.  MFMA and VALU issue bound it (47 and 38% busy at 1.6 waves
// a SIMD, a quarter of the waves' time in waits): B4 H16 of 2048 ragged queries and 4096 keys,
// d128, 305 us (1.02 PFLOP/s); B4 H12 N4096 d64 causal with a bias 173 us (0.89).
// ===========================================================================
template <typename T, int D, int MR, int NW, int OCC, int KS, bool kBias>
__global__ __launch_bounds__(KS * NW * 64, OCC) void ext_bwd_rows_kernel(
    ExtArgs a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ O,
    const T* __restrict__ dO, const float* __restrict__ L, T* __restrict__ dQ, float* __restrict__ Dout, float* __restrict__ parts) {
  using E = Elt<T>;
  using G = Geo<T, D>;
  constexpr int BR = 16 * MR * NW;
  __shared__ __attribute__((aligned(16))) RowSmem<T, D, 2, 2, KS, BR> sm;
  extern __shared__ float steps_mem[];
  float FB_LDS* const steps = (float FB_LDS*)steps_mem;

  int rh, rb;
  ext_map_block(a, a.grp * a.nRB, true, a.kv_lens, a.Nk, rh, rb);
  const int l = lane_id(), g = l >> 4, j = l & 15;
  const int ks = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave_id() / NW);
  const int wl = __builtin_amdgcn_readfirstlane(KS == 1 ? wave_id() : wave_id() % NW);
  const ExtRows<MR, NW, false> rw(a, rh, rb, wl, j);
  const int64_t kvoff = (int64_t)rw.kvh * a.Nk * D, qoff = rw.qrow * D;

  u32x4 qf[MR][G::kChunks], dof[MR][G::kChunks];
  float lb[MR], drow[MR], dout[MR], rest[MR];
  bool centred = false;
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
  const float c = a.scale * kLog2e;
  floatx4 s[2][MR], dp[2][MR];
  typename E::TFrag dsf[MR];

  const T* const src[2] = {K + kvoff, V + kvoff};
  const int part = blockIdx.y, split = ext_parts_of(rw.tiles, KS, a.nparts);
  const ExtRun run = ext_run(rw.tiles, part, split, ks, KS), first = ext_run(rw.tiles, part, split, 0, KS);
  constexpr bool kBarrier = NW > 1;
  const TileCopy<T, D, NW, 2> copy(wl);
  float blo = 0.f, bhi = 0.f;
  ext_stream<tile_loads<T, D, NW, 2>(), kBarrier>(
      kBarrier ? first.size() : run.size(),
      [&](int it, int st) {
        copy.template issue<true>(src, (T FB_LDS*)sm.lds[ks][st], min(run.begin + it, rw.tiles - 1) * kBS, rw.kvis);
      },
      [&]() {
        if constexpr (kBias) {
          ext_fill_steps<true>(a, a.table, rw.head0, 1, steps, KS * NW * 64);
          __syncthreads();
          blo = steps[0];
          bhi = steps[ext_steps(a) - 1];
        }
      },
      [&](int it, int st) {
        const int s0 = min(run.begin + it, rw.tiles - 1) * kBS;
        const int mode = vector_mode(run.begin + it < run.end ? rw.mode(s0) : 0);
        if (mode == 0) return;
        const T FB_LDS* Ks = (const T FB_LDS*)sm.lds[ks][st];
        const T FB_LDS* Vs = Ks + G::kTileElems;
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) {
            s[sb][mb] = floatx4{0.f, 0.f, 0.f, 0.f};
            dp[sb][mb] = floatx4{-drow[mb], -drow[mb], -drow[mb], -drow[mb]};
          }
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
        float off[MR];
#pragma unroll
        for (int mb = 0; mb < MR; ++mb) off[mb] = -lb[mb];
        if constexpr (kBias) {
          const int side = ext_side(s0 - rw.phi, s0 + kBS - 1 - rw.plo, a.R);
          const float kb = side < 0 ? blo : side > 0 ? bhi : 0.f;
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) off[mb] += kb;
        }
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int mb = 0; mb < MR; ++mb)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[sb][mb][r] = __builtin_fmaf(s[sb][mb][r], c, off[mb]);
        if constexpr (kBias) {
          if (ext_side(s0 - rw.phi, s0 + kBS - 1 - rw.plo, a.R) == 0) {
#pragma unroll
            for (int mb = 0; mb < MR; ++mb) {
              const float FB_LDS* bias = steps + (a.R + kStepPad + s0 - rw.pos(mb) + 4 * g);
#pragma unroll
              for (int sb = 0; sb < 2; ++sb)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[sb][mb][r] += bias[16 * sb + r];
            }
          }
        }
        if (mode == 2) {
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) {
            floatx4 x[2] = {s[0][mb], s[1][mb]};
            ext_mask1(x, s0, rw.klim(mb));
            s[0][mb] = x[0];
            s[1][mb] = x[1];
          }
        }
        if (!centred) {
          centred = true;
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) {
            float w = 0.f, wd = 0.f;
#pragma unroll
            for (int sb = 0; sb < 2; ++sb)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float p = fast_exp2(s[sb][mb][r]);
                w += p;
                wd = __builtin_fmaf(p, dp[sb][mb][r], wd);
              }
            w = group_sum(w);
            wd = group_sum(wd);
            // L and the weights are off by a few 2^-24 of L's size
            const float by = w > 1.f - 0x1p-16f ? wd / w : 0.f;
            drow[mb] += by;
            rest[mb] = g == 0 ? by : 0.f;
#pragma unroll
            for (int sb = 0; sb < 2; ++sb) dp[sb][mb] -= by;
          }
        }
#pragma unroll
        for (int mb = 0; mb < MR; ++mb)
#pragma unroll
          for (int sb = 0; sb < 2; ++sb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float ds = fast_exp2(s[sb][mb][r]) * dp[sb][mb][r];
              rest[mb] += ds;
              dsf[mb].set(4 * sb + r, ds);
            }
#pragma unroll
        for (int nb = 0; nb < G::kNB; ++nb) {
          const typename E::AFrag ak = G::load_afrag(Ks, 16 * nb);
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) acc[nb][mb] = E::mma_acc(ak, dsf[mb], acc[nb][mb]);
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

// Adds the parts of the row side: dQ = tau times the sums, D their scalars' sum.  One
// thread for four head dims of a row.
template <typename T, int D>
__global__ __launch_bounds__(256) void ext_bwd_join_kernel(ExtArgs a, const float* __restrict__ parts, int64_t all,
                                                           T* __restrict__ dQ, float* __restrict__ Dout) {
  constexpr int kPer = D / 4;
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = x / kPer;
  const int dim = 4 * (int)(x % kPer);
  if (row >= all) return;
  const int64_t bh = row / a.Nq;
  floatx4 sum = floatx4{0.f, 0.f, 0.f, 0.f};
  float d = 0.f;
  if ((int)(row - bh * a.Nq) < ext_lens(a, (int)(bh / a.H)).q) {
    const float* const sc = parts + a.nparts * all * D;
    for (int q = 0; q < a.nparts; ++q) {
      const int64_t at = q * all + row;
      sum += *(const floatx4*)(parts + at * D + dim);
      d += sc[at];
    }
  }
  Elt<T>::store4(dQ + row * D + dim, sum * a.scale);
  if (dim == 0) Dout[row] = d;
}

// ===========================================================================
// Column kernels
// ===========================================================================

// What a column kernel's workgroup and wave know of their columns.  The streamed tiles are
// the query tiles t0 .. t0 + per_head - 1 of `heads` query heads from head `hq` on: all of
// a group's, or (parts: part = head of the group x sub-run) one head's.
template <int MC, int NW>
struct ExtCols {
  int b, kvh, hq, heads, sub, subs;
  int t0, per_head;       // first query tile, query tiles a head
  int qlen, klen, start;
  int col0, col1;         // the wave's columns col0 .. col1 - 1 that are valid keys
  __device__ __forceinline__ ExtCols(const ExtArgs& a, int kv, int rb, int wl) {
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
    col1 = min(col0 + 16 * MC, n.k);
    // the first query that sees the block's first key; a block behind the keys has no tiles
    const int q0 = a.causal != 0 ? max(rb * BC - n.start, 0) : 0;
    const int nT = rb * BC < n.k ? (n.q + kBS - 1) / kBS : 0;
    t0 = min(q0 / kBS, nT);
    per_head = nT - t0;
  }
  __device__ __forceinline__ int count() const { return heads * per_head; }
  __device__ __forceinline__ int qhead(int f) const { return heads == 1 ? hq : hq + f / per_head; }
  __device__ __forceinline__ int tile(int f) const { return t0 + (heads == 1 ? f : f % per_head); }
  // 0: no valid pair of the tile at s0, 1: every pair valid, 2: mixed
  __device__ __forceinline__ int mode(int s0, bool causal) const {
    if (col0 >= col1 || (causal && start + s0 + kBS - 1 < col0)) return 0;
    return s0 + kBS <= qlen && col1 == col0 + 16 * MC && (!causal || start + s0 >= col0 + 16 * MC - 1) ? 1 : 2;
  }
};

// Exponents of invalid pairs to -inf: x[sb][mc][r] belongs to query s0 + 16 sb + 4 g + r
// and key t + 16 mc.
template <int MC>
__device__ __forceinline__ void ext_mask_cols(floatx4 (&x)[2][MC], int s0, int t, int qlen, int klen, int start,
                                              bool causal) {
  const int g = lane_id() >> 4;
#pragma unroll
  for (int mc = 0; mc < MC; ++mc) {
    const int key = t + 16 * mc;
    // queries qlo .. qlen - 1 see the key
    const int qlo = key >= klen ? 1 << 30 : causal ? key - start : 0;
#pragma unroll
    for (int sb = 0; sb < 2; ++sb)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int q = s0 + 16 * sb + 4 * g + r;
        x[sb][mc][r] = q < qlen && q >= qlo ? x[sb][mc][r] : -INFINITY;
      }
  }
}

// Sums of a wave's score-like tiles by step of position (key - query): see the head of
// this file.  tile() takes the tiles in order of their queries; x[sb][mc][r] belongs to
// query 16 sb + 4 g + r and key 16 mc + j of the tile, `base` is the step of its first
// key and first query.  buf: kBufFloats floats of LDS of this wave.  out: 2 R + 3 sums:
// steps -R .. R, then all below -R, then all above R.
struct StepSums {
  static constexpr int kStride = 76, kBufFloats = 4 * kStride;
  float* out;
  int R;
  float carry, below, above;  // the window below the last near tile's; the far sums
  // The row starts at zero: the loop's first wait for its copies waits for these stores too.
  __device__ __forceinline__ void init(float* row, int r, float FB_LDS* buf) {
    out = row;
    R = r;
    carry = below = above = 0.f;
    for (int x = lane_id(); x < kBufFloats; x += 64) buf[x] = 0.f;  // columns that no tile writes stay so
    for (int x = lane_id(); x < 2 * R + 1; x += 64) out[x] = 0.f;
  }
  // The sums of steps at .. at + 31, one a lane; every window is stored once.
  __device__ __forceinline__ void emit(int at, float v) {
    const int l = lane_id(), step = at + l;
    if (l < 32) {
      if (step > R)
        above += v;
      else if (step < -R)
        below += v;
      else
        out[step + R] = v;
    }
  }
  template <int MC>
  __device__ __forceinline__ void far(const floatx4 (&x)[2][MC], int base, int side) {
    // the first tile below the near ones: its upper window is what they left
    if (side < 0 && base + 31 + 16 * MC > -R) {
      emit(base, carry);
      carry = 0.f;
    }
    float sum = 0.f;
#pragma unroll
    for (int mc = 0; mc < MC; ++mc) {
      const floatx4 v = x[0][mc] + x[1][mc];
      sum += (v[0] + v[1]) + (v[2] + v[3]);
    }
    if (side < 0)
      below += sum;
    else
      above += sum;
  }
  // The sum of a 16x16 block x_r (query 4 g + r, key j) along its diagonals for one lane
  // group g: same[c] over key - r = c, next[c] over key - r = c - 16.
  static __device__ __forceinline__ void diagonals(floatx4 x, float& same, float& next) {
    same = shifted<0x101>(shifted<0x101>(shifted<0x101>(x[3]) + x[2]) + x[1]) + x[0];  // lane c takes lane c + 1
    next = shifted<0x11f>(x[1]) + (shifted<0x11e>(x[2]) + shifted<0x11d>(x[3]));       // lane c takes c - 15, - 14, - 13
  }
  template <int kCtrl> static __device__ __forceinline__ float shifted(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl, 0xf, 0xf, true));
  }
  // A tile with steps of their own sums.  Blocks of equal key - query are added first, each
  // is summed along its diagonals inside its lane group by shifts in the row of 16 lanes,
  // and the four groups, whose steps lie 4 apart, meet in LDS: row g of the buffer holds its
  // 64 sums 4 g to the left, so that lane l finds step l - 32 in one column.  (Summing the
  // diagonals from a whole tile in LDS, 16 reads and 110 vector instructions for 4 and 35,
  // took B8 H12 N512 d64, all of it near, 41 us for the column kernel.)
  template <int MC>
  __device__ __forceinline__ void near(const floatx4 (&x)[2][MC], int base, float FB_LDS* buf) {
    int l = lane_id();
    asm volatile("" : "+v"(l));  // the addresses are made anew in every tile, not kept
    float a0, n0, am, nm, a1 = 0.f, n1 = 0.f;
    diagonals(MC == 2 ? x[0][0] + x[1][MC - 1] : x[0][0], a0, n0);
    diagonals(x[1][0], am, nm);
    if constexpr (MC == 2) diagonals(x[0][1], a1, n1);
    float FB_LDS* const to = buf + (kStride - 4) * (l >> 4) + (l & 15) + 12;  // row g, 4 g to the left
    to[0] = nm;
    to[16] = am + n0;
    to[32] = a0 + n1;
    if constexpr (MC == 2) to[48] = a1;
    const float FB_LDS* const from = buf + l + 12;
    const float sum = (from[0] + from[kStride]) + (from[2 * kStride] + from[3 * kStride]);
    // lanes 32 .. 63: the upper window, which no later tile meets
    const float other = __shfl_xor(sum, 32);
    emit(base, (l < 32 ? other : sum) + carry);
    carry = sum;
  }
  // last: `base` of the last tile of the run (of any tile if the run is empty)
  __device__ __forceinline__ void finish(int last) {
    emit(last - 32, carry);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      below += __shfl_xor(below, m);
      above += __shfl_xor(above, m);
    }
    if (lane_id() == 0) {
      out[2 * R + 1] = below;
      out[2 * R + 2] = above;
    }
  }
};

// The column kernels' LDS beside the rings: the bias by steps (and the direction's), then
// the waves' StepSums buffers.
template <bool kBias, int KS, int NW, bool kDir>
struct ExtColMem {
  float FB_LDS* steps;
  float FB_LDS* dirs;
  float FB_LDS* buf;
  __device__ __forceinline__ ExtColMem(float* mem, const ExtArgs& a, int head) {
    steps = dirs = buf = (float FB_LDS*)mem;
    if constexpr (kBias) {
      const int n = (ext_steps(a) + 3) & ~3;
      dirs = steps + n;
      buf = steps + (kDir ? 2 : 1) * n + __builtin_amdgcn_readfirstlane(wave_id()) * StepSums::kBufFloats;
      ext_fill_steps<true>(a, a.table, head, 1, steps, KS * NW * 64);
      if constexpr (kDir) ext_fill_steps<false>(a, a.dir, head, 1, dirs, KS * NW * 64);
    }
  }
};

// One wave's row in the workspace of step sums: the rows of a query head lie together,
// [H][B][nRB][subs][waves].
__device__ __forceinline__ float* ext_step_row(float* sums, const ExtArgs& a, int qhead, int b, int rb, int sub,
                                               int subs, int waves) {
  const int batch = a.total / a.nRB / (a.H / a.grp);
  const int64_t row = ((((int64_t)(qhead - b * a.H) * batch + b) * a.nRB + rb) * subs + sub) * waves +
                      __builtin_amdgcn_readfirstlane(wave_id());
  return sums + row * (2 * a.R + 3);
}

// Stores the two key-side accumulators: to the outputs, or as one part's fp32 sums
// ([nparts][2][the launch's key rows][D]).  Columns that are no valid key get zeros.
template <typename T, int D, int KS, int NB, int MC>
__device__ __forceinline__ void ext_store_cols(const ExtArgs& a, int kvh, int col0, int klen, int ks,
                                               const floatx4 (&x)[NB][MC], const floatx4 (&y)[NB][MC], float fx, float fy,
                                               T* __restrict__ X, T* __restrict__ Y, float* __restrict__ parts) {
  const int l = lane_id(), g = l >> 4, j = l & 15;
  const int64_t plane = a.rows * D, first = a.row0 * D;
  const floatx4 zero = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int mc = 0; mc < MC; ++mc) {
    const int col = col0 + 16 * mc + j;
    if (col >= a.Nk) continue;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (KS > 1 && nb % KS != ks) continue;
      const int64_t off = ((int64_t)kvh * a.Nk + col) * D + 16 * nb + 4 * g;
      const floatx4 vx = col < klen ? x[nb][mc] * fx : zero, vy = col < klen ? y[nb][mc] * fy : zero;
      if (a.nparts > 1) {
        *(floatx4*)(parts + 2 * blockIdx.y * plane + off - first) = vx;
        *(floatx4*)(parts + (2 * blockIdx.y + 1) * plane + off - first) = vy;
      } else {
        Elt<T>::store4(X + off, vx);
        Elt<T>::store4(Y + off, vy);
      }
    }
  }
}

// Adds the parts of the column kernels in order and rounds.
template <typename T>
__global__ __launch_bounds__(256) void ext_parts_kernel(const float* __restrict__ parts, int nparts, int64_t plane,
                                                        T* __restrict__ X, T* __restrict__ Y) {
  const int64_t n4 = plane / 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < 2 * n4; i += (int64_t)gridDim.x * 256) {
    const int t = i < n4 ? 0 : 1;
    const int64_t off = 4 * (i - t * n4);
    floatx4 acc = *(const floatx4*)(parts + t * plane + off);
    for (int q = 1; q < nparts; ++q) acc += *(const floatx4*)(parts + (2 * (int64_t)q + t) * plane + off);
    Elt<T>::store4((t == 0 ? X : Y) + off, acc);
  }
}

// First backward, column side: as attn_bwd_cols_kernel (its K rows in LDS with kKL), with
// the table's step sums (`sums`, or null).  Waits bound it, a third of
// the waves' time (copies, barriers and LDS reads at 1.7 waves a SIMD; MFMA 44% and VALU 28% busy):
// B4 H16 of 2048 ragged queries and 4096 keys, d128, 415 us (1.00 PFLOP/s); B4 H12 N4096 d64
// causal with a bias 238 us (0.87), without 204; dense 439 us (0.94), without 383.
template <typename T, int D, int MC, int NW, int OCC, int KS, bool kKL, bool kBias>
__global__ __launch_bounds__(KS * NW * 64, OCC) void ext_bwd_cols_kernel(
    ExtArgs a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ dO,
    const float* __restrict__ L, const float* __restrict__ Dv, T* __restrict__ dK, T* __restrict__ dV,
    float* __restrict__ parts, float* __restrict__ sums) {
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
  extern __shared__ float steps_mem[];

  int kv, rb;
  ext_map_cols(a, kv, rb);
  const int l = lane_id(), g = l >> 4, j = l & 15;
  const int ks = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave_id() / NW);
  const int wl = __builtin_amdgcn_readfirstlane(KS == 1 ? wave_id() : wave_id() % NW);
  const ExtCols<MC, NW> cl(a, kv, rb, wl);
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
  const ExtColMem<kBias, KS, NW, false> mem(steps_mem, a, cl.hq - cl.b * a.H);
  StepSums tab;
  if constexpr (kBias)
    if (sums != nullptr) tab.init(ext_step_row(sums, a, cl.hq, cl.b, rb, cl.sub, cl.subs, KS * NW), a.R, mem.buf);
  floatx4 dk[G::kNB][MC], dv[G::kNB][MC];
#pragma unroll
  for (int nb = 0; nb < G::kNB; ++nb)
#pragma unroll
    for (int mc = 0; mc < MC; ++mc) dk[nb][mc] = dv[nb][mc] = floatx4{0.f, 0.f, 0.f, 0.f};
  const float c = a.scale * kLog2e;
  floatx4 s[2][MC], dp[2][MC];
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
          float FB_LDS* t = (float FB_LDS*)sm.tsc[ks][ts];
          const float Lr = raw[l];
          t[l] = Lr == -INFINITY ? -INFINITY : -Lr * kLog2e;  // an empty row: P = 0
          t[kBS + l] = -raw[kBS + l];
        }
      },
      [&](int it, int st, int ts, auto&& prep_next) {
        const int s0 = cl.tile(flat(it)) * kBS;
        const int mode = vector_mode(run.begin + it < run.end ? cl.mode(s0, a.causal != 0) : 0);
        if (mode == 0) {
          prep_next();
          return;
        }
        const T FB_LDS* Qs = (const T FB_LDS*)sm.lds[ks][st];
        const T FB_LDS* dOs = Qs + G::kTileElems;
        const float FB_LDS* Ts = (const float FB_LDS*)sm.tsc[ks][ts];
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
          const floatx4 t1 = *(const floatx4 FB_LDS*)(Ts + kBS + 16 * sb + 4 * g);
#pragma unroll
          for (int mc = 0; mc < MC; ++mc) {
            s[sb][mc] = floatx4{0.f, 0.f, 0.f, 0.f};
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
        const int base = cl.col0 - (cl.start + s0);  // step of the tile's first key and query
        const int side = kBias ? ext_side(base - (kBS - 1), base + 16 * MC - 1, a.R) : 0;
        const float kb = !kBias || side == 0 ? 0.f : mem.steps[side < 0 ? 0 : ext_steps(a) - 1];
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
          floatx4 t0 = *(const floatx4 FB_LDS*)(Ts + 16 * sb + 4 * g);
          if constexpr (kBias) t0 += kb;
#pragma unroll
          for (int mc = 0; mc < MC; ++mc)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[sb][mc][r] = __builtin_fmaf(s[sb][mc][r], c, t0[r]);
        }
        if constexpr (kBias) {
          if (side == 0) {
            const float FB_LDS* bias = mem.steps + (a.R + kStepPad + base + j - 4 * g - 19);
#pragma unroll
            for (int sb = 0; sb < 2; ++sb)
#pragma unroll
              for (int mc = 0; mc < MC; ++mc)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[sb][mc][r] += bias[19 + 16 * mc - 16 * sb - r];
          }
        }
        if (mode == 2) ext_mask_cols(s, s0, cl.col0 + j, cl.qlen, cl.klen, cl.start, a.causal != 0);
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int mc = 0; mc < MC; ++mc) {
              const float p = fast_exp2(s[sb][mc][r]);
              pf[mc].set(4 * sb + r, p);
              dp[sb][mc][r] *= p;
              dsf[mc].set(4 * sb + r, dp[sb][mc][r]);
            }
        if constexpr (kBias) {
          if (sums != nullptr) {
            if (side != 0)
              tab.far(dp, base, side);
            else
              tab.near(dp, base, mem.buf);
          }
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
  if constexpr (kBias)
    if (sums != nullptr) tab.finish(cl.col0 - (cl.start + cl.tile(max(run.end - 1, 0)) * kBS));
  if constexpr (KS > 1) {
    static_assert(sizeof(sm.lds) >= merge_bytes<KS, NW, G::kNB, MC>(), "set merge buffer");
    merge_sets<KS, NW>(dk, ks, wl, (floatx4 FB_LDS*)&sm.lds[0][0][0]);
    merge_sets<KS, NW>(dv, ks, wl, (floatx4 FB_LDS*)&sm.lds[0][0][0]);
  }
  ext_store_cols<T, D, KS>(a, kv, cl.col0, cl.klen, ks, dk, dv, a.scale, 1.f, dK, dV, parts);
}

// ===========================================================================
// BoB Pass 1: as bob_pass1_kernel's form with the first backward's dQ, but for the
// reference of its sums.  The affine epilogue takes E B from Omega and alpha O from dOt, and
// rows of few keys are what these differences leave of the operands' rounding (a row of one
// key has Qt = 0 and kept 2^-8 of tau C k).  So F and Pt enter the sums less an estimate
// alpha*, E* of their means under P, which the first tile gives (all keys of such rows):
//   F' = F - alpha*,  w = C + F' (dP - D) - E*,  da = sum P F',  de = sum P w,
//   Qt = tau (sum P w k + sum P (dP - D) u_K - de sum P k) - da dQ,
//   dOt = sum P u_V + sum P F' v - da O,  alpha = alpha* + da,  E = E* + de - alpha D,
// since Pt - E = w - da (dP - D) - de.  It costs nothing after the first tile: alpha* rides
// on the fma that scales F, -E* is where the C tile starts.  Wave sets share one estimate.
// MFMA and VALU issue bound it: B4 H12 N4096 d64 dense with a bias 963 us (1.07 PFLOP/s of the
// ten contractions), without 929; a wave's chain of LDS reads, MFMA and VALU where the grid
// leaves one or two waves a SIMD (B2 H8 of 1000 queries and 2047 keys: 52 us, 0.56 PFLOP/s).
// ===========================================================================
template <typename T, int D, int MR, int NW, int OCC, int KS, int kPF, bool kBias>
__global__ __launch_bounds__(KS * NW * 64, OCC) void ext_pass1_kernel(
    ExtArgs a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ O,
    const T* __restrict__ dO, const T* __restrict__ UQ, const T* __restrict__ UK, const T* __restrict__ UV,
    const float* __restrict__ L, const float* __restrict__ Dv, const T* __restrict__ dQ, T* __restrict__ Qt,
    T* __restrict__ dOt, float* __restrict__ alpha_out, float* __restrict__ E_out, float* __restrict__ parts) {
  using E = Elt<T>;
  using G = Geo<T, D>;
  constexpr int BR = 16 * MR * NW;
  __shared__ __attribute__((aligned(16))) RowSmem<T, D, 4, 2, KS, BR> sm;
  __shared__ float ref_mem[KS == 1 ? 1 : 5 * KS * BR];
  extern __shared__ float steps_mem[];
  float FB_LDS* const steps = (float FB_LDS*)steps_mem;
  float FB_LDS* const dirs = steps + (kBias ? (ext_steps(a) + 3) & ~3 : 0);

  int rh, rb;
  ext_map_block(a, a.grp * a.nRB, true, a.kv_lens, a.Nk, rh, rb);
  const int l = lane_id(), g = l >> 4, j = l & 15;
  const int ks = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave_id() / NW);
  // scalar, one set at d = 64 takes 174 registers for 166 and loses its third wave per SIMD
  const int wl = KS == 1 ? wave_id() : __builtin_amdgcn_readfirstlane(wave_id() % NW);
  const ExtRows<MR, NW, false> rw(a, rh, rb, wl, j);
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
  const float c = a.scale * kLog2e;
  floatx4 s[2][MR], dp[2][MR], f[2][MR], cc[2][MR];
  typename E::TFrag fP[MR], fPF[MR], fPPt[MR], fPdd[MR];
  using AF = typename E::AFrag;

  const T* const src[4] = {K + kvoff, V + kvoff, UK + kvoff, UV + kvoff};
  const int part = blockIdx.y, split = ext_parts_of(rw.tiles, KS, a.nparts);
  const ExtRun run = ext_run(rw.tiles, part, split, ks, KS), first = ext_run(rw.tiles, part, split, 0, KS);
  constexpr bool kBarrier = NW > 1 || KS > 1;  // the sets meet in the first tile
  const TileCopy<T, D, NW, 4> copy(wl);
  float blo = 0.f, bhi = 0.f, ulo = 0.f, uhi = 0.f;
  float aref[MR], eref[MR];
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) aref[mb] = eref[mb] = 0.f;
  // parts that share a block take their sums from 0: each row of theirs has many keys in view
  bool centred = false;
  ext_stream<tile_loads<T, D, NW, 4>(), kBarrier>(
      kBarrier ? first.size() : run.size(),
      [&](int it, int st) {
        copy.template issue<true>(src, (T FB_LDS*)sm.lds[ks][st], min(run.begin + it, rw.tiles - 1) * kBS, rw.kvis);
      },
      [&]() {
        if constexpr (kBias) {
          ext_fill_steps<true>(a, a.table, rw.head0, 1, steps, KS * NW * 64);
          ext_fill_steps<false>(a, a.dir, rw.head0, 1, dirs, KS * NW * 64);
          __syncthreads();
          const int n = ext_steps(a);
          blo = scalar(steps[0]);
          bhi = scalar(steps[n - 1]);
          ulo = scalar(dirs[0]);
          uhi = scalar(dirs[n - 1]);
        }
      },
      [&](int it, int st) {
        const int s0 = min(run.begin + it, rw.tiles - 1) * kBS;
        int mode = run.begin + it < run.end ? rw.mode(s0) : 0;
        if constexpr (KS > 1) mode = vector_mode(mode);
        if (mode == 0 && (KS == 1 || it > 0 || split > 1)) return;
        const T FB_LDS* Ks = (const T FB_LDS*)sm.lds[ks][st];
        const T FB_LDS* Vs = Ks + G::kTileElems;
        const T FB_LDS* UKs = Vs + G::kTileElems;
        const T FB_LDS* UVs = UKs + G::kTileElems;
        if constexpr (std::is_same_v<T, bf16> && D == 128) __builtin_amdgcn_iglp_opt(3);
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) {
            s[sb][mb] = f[sb][mb] = floatx4{0.f, 0.f, 0.f, 0.f};
            cc[sb][mb] = floatx4{-eref[mb], -eref[mb], -eref[mb], -eref[mb]};
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
              cc[sb][mb] = E::mma_chunk(auv, dof[mb][kk], cc[sb][mb]);    // C^T - E* = U_V dO^T - E*
            }
          }
        int side = 0;
        float kb = 0.f, ku = 0.f;
        if constexpr (kBias) {
          side = ext_side(s0 - rw.phi, s0 + kBS - 1 - rw.plo, a.R);
          if (side != 0) {
            kb = side < 0 ? blo : bhi;
            ku = side < 0 ? ulo : uhi;
          }
        }
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int mb = 0; mb < MR; ++mb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              s[sb][mb][r] = __builtin_fmaf(s[sb][mb][r], c, kb - lb[mb]);
              f[sb][mb][r] = __builtin_fmaf(f[sb][mb][r], a.scale, ku - aref[mb]);
            }
        AF cur[4];
        auto load_frags = [&](int nb) {
#pragma unroll
          for (int t = 0; t < 4; ++t) cur[t] = G::load_afrag(Ks + t * G::kTileElems, 16 * nb);
        };
        if constexpr (kPF != 0) load_frags(0);
        if constexpr (kBias) {
          if (side == 0) {
#pragma unroll
            for (int mb = 0; mb < MR; ++mb) {
              const int at = a.R + kStepPad + s0 - rw.pos(mb) + 4 * g;
#pragma unroll
              for (int sb = 0; sb < 2; ++sb)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  s[sb][mb][r] += steps[at + 16 * sb + r];
                  f[sb][mb][r] += dirs[at + 16 * sb + r];
                }
            }
          }
        }
        if (mode == 2) {
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) {
            floatx4 x[2] = {s[0][mb], s[1][mb]};
            ext_mask1(x, s0, rw.klim(mb));
            s[0][mb] = x[0];
            s[1][mb] = x[1];
          }
        }
        // every wave of a workgroup with sets comes here in its first iteration (a barrier)
        if (split == 1 && (KS > 1 ? it == 0 : !centred)) {
          centred = true;
#pragma unroll
          for (int mb = 0; mb < MR; ++mb) {
            float w = 0.f, wf = 0.f, wd = 0.f, wc = 0.f, wfd = 0.f;  // sums of P, P F, P (dP - D), P C, P F (dP - D)
            if (mode != 0) {
#pragma unroll
              for (int sb = 0; sb < 2; ++sb)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  const float p = fast_exp2(s[sb][mb][r]), pf = p * f[sb][mb][r];
                  w += p;
                  wf += pf;
                  wd = __builtin_fmaf(p, dp[sb][mb][r], wd);
                  wc = __builtin_fmaf(p, cc[sb][mb][r], wc);
                  wfd = __builtin_fmaf(pf, dp[sb][mb][r], wfd);
                }
            }
            w = group_sum(w);
            wf = group_sum(wf);
            wd = group_sum(wd);
            wc = group_sum(wc);
            wfd = group_sum(wfd);
            if constexpr (KS > 1) {
              float FB_LDS* at = (float FB_LDS*)ref_mem + 16 * (wl * MR + mb) + j;
              if (g == 0) {
                at[(5 * ks + 0) * BR] = w;
                at[(5 * ks + 1) * BR] = wf;
                at[(5 * ks + 2) * BR] = wd;
                at[(5 * ks + 3) * BR] = wc;
                at[(5 * ks + 4) * BR] = wfd;
              }
              __syncthreads();
              w = wf = wd = wc = wfd = 0.f;
#pragma unroll
              for (int q = 0; q < KS; ++q) {
                w += at[(5 * q + 0) * BR];
                wf += at[(5 * q + 1) * BR];
                wd += at[(5 * q + 2) * BR];
                wc += at[(5 * q + 3) * BR];
                wfd += at[(5 * q + 4) * BR];
              }
            }
            // rows without weight here (or of NaN) keep the reference 0
            if (w > 0.f) {
              aref[mb] = wf / w;
              eref[mb] = (wc + (wfd - aref[mb] * wd)) / w;
            }
#pragma unroll
            for (int sb = 0; sb < 2; ++sb) {
              f[sb][mb] -= aref[mb];
              cc[sb][mb] -= eref[mb];
            }
          }
        }
        if (KS > 1 && mode == 0) return;
#pragma unroll
        for (int mb = 0; mb < MR; ++mb)
#pragma unroll
          for (int sb = 0; sb < 2; ++sb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float p = fast_exp2(s[sb][mb][r]);
              const float dd = dp[sb][mb][r];
              const float pf = p * f[sb][mb][r];
              const float ppt = p * __builtin_fmaf(f[sb][mb][r], dd, cc[sb][mb][r]);
              const int i = 4 * sb + r;
              alpha[mb] += pf;
              e0[mb] += ppt;
              fP[mb].set(i, p);
              fPF[mb].set(i, pf);
              fPPt[mb].set(i, ppt);
              fPdd[mb].set(i, p * dd);
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
            aB[nb][mb] = E::mma_acc(ak, fP[mb], aB[nb][mb]);
            aOM[nb][mb] = E::mma_acc(ak, fPPt[mb], aOM[nb][mb]);
            aOM[nb][mb] = E::mma_acc(auk, fPdd[mb], aOM[nb][mb]);
            aDO[nb][mb] = E::mma_acc(auv, fP[mb], aDO[nb][mb]);
            aDO[nb][mb] = E::mma_acc(av, fPF[mb], aDO[nb][mb]);
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
        if (g == 0 && ks == 0) *(floatx4*)(sc + 4 * at) = floatx4{alpha[mb], e0[mb], aref[mb], eref[mb]};
      }
    return;
  }
  const floatx4 zero = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int mb = 0; mb < MR; ++mb) {
    if (rw.row(mb) >= rw.rows) continue;
    const int64_t at = rw.qrow + rw.row(mb);
    if (g == 0 && ks == 0) {
      const float al = aref[mb] + alpha[mb];
      alpha_out[at] = rw.ok(mb) ? al : 0.f;
      E_out[at] = rw.ok(mb) ? eref[mb] + e0[mb] - al * drow[mb] : 0.f;
    }
#pragma unroll
    for (int nb = 0; nb < G::kNB; ++nb) {
      if (!own.owns(nb)) continue;
      const int64_t off = at * D + 16 * nb + 4 * g;
      if (rw.ok(mb)) {
        E::store4(dOt + off, aDO[nb][mb] - alpha[mb] * E::load4(O + off));
        E::store4(Qt + off, a.scale * (aOM[nb][mb] - e0[mb] * aB[nb][mb]) - alpha[mb] * E::load4(dQ + off));
      } else {
        E::store4(dOt + off, zero);
        E::store4(Qt + off, zero);
      }
    }
  }
}

// Adds the parts of Pass 1 and finishes its rows.  One thread for four head dims of a row.
template <typename T, int D>
__global__ __launch_bounds__(256) void ext_pass1_join_kernel(ExtArgs a, const float* __restrict__ parts, int64_t all,
                                                             const T* __restrict__ O, const float* __restrict__ Dv,
                                                             const T* __restrict__ dQ, T* __restrict__ Qt,
                                                             T* __restrict__ dOt, float* __restrict__ alpha_out,
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
  floatx4 d = zero, om = zero, b = zero, sc = zero;
  if (ok) {
    const float* const scalars = parts + a.nparts * all * (3 * D);
    for (int q = 0; q < a.nparts; ++q) {
      const int64_t at = q * all + row;
      const float* const from = parts + at * (3 * D) + dim;
      d += *(const floatx4*)from;
      om += *(const floatx4*)(from + D);
      b += *(const floatx4*)(from + 2 * D);
      sc += *(const floatx4*)(scalars + 4 * at);
    }
    E::store4(dOt + off, d - sc[0] * E::load4(O + off));
    E::store4(Qt + off, a.scale * (om - sc[1] * b) - sc[0] * E::load4(dQ + off));
  } else {
    E::store4(dOt + off, zero);
    E::store4(Qt + off, zero);
  }
  if (dim == 0) {
    const float al = sc[2] + sc[0];
    alpha_out[row] = al;
    E_out[row] = ok ? sc[3] + sc[1] - al * Dv[row] : 0.f;
  }
}

// ===========================================================================
// BoB Pass 2: as bob_pass2_kernel, with the second-order table sums (`sums`, or null).  Bound
// as Pass 1: B4 H12 N4096 d64 dense with a bias 792 us (1.04 PFLOP/s of the eight
// contractions), without 705: the near tiles' bias reads and step sums, and registers.
// ===========================================================================
template <typename T, int D, int MC, int NW, int OCC, int KS, bool kPF, bool kBias>
__global__ __launch_bounds__(KS * NW * 64, OCC) void ext_pass2_kernel(
    ExtArgs a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ dO,
    const T* __restrict__ UQ, const T* __restrict__ UK, const T* __restrict__ UV, const float* __restrict__ L,
    const float* __restrict__ Dv, const float* __restrict__ alpha_in, const float* __restrict__ E_in,
    T* __restrict__ Kt, T* __restrict__ Vt, float* __restrict__ parts, float* __restrict__ sums) {
  using E = Elt<T>;
  using G = Geo<T, D>;
  struct Smem2 {
    T lds[KS][2][3 * G::kTileElems];
    float rawsc[KS][2][4 * kBS];
    float tsc[KS][2][4 * kBS];
  };
  __shared__ __attribute__((aligned(16))) Smem2 sm;
  extern __shared__ float steps_mem[];

  int kv, rb;
  ext_map_cols(a, kv, rb);
  const int l = lane_id(), g = l >> 4, j = l & 15;
  const int ks = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave_id() / NW);
  const int wl = __builtin_amdgcn_readfirstlane(KS == 1 ? wave_id() : wave_id() % NW);
  const ExtCols<MC, NW> cl(a, kv, rb, wl);
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
  const ExtColMem<kBias, KS, NW, true> mem(steps_mem, a, cl.hq - cl.b * a.H);
  StepSums tab;
  if constexpr (kBias)
    if (sums != nullptr) tab.init(ext_step_row(sums, a, cl.hq, cl.b, rb, cl.sub, cl.subs, KS * NW), a.R, mem.buf);
  floatx4 aK[G::kNB][MC], aV[G::kNB][MC];
#pragma unroll
  for (int nb = 0; nb < G::kNB; ++nb)
#pragma unroll
    for (int mc = 0; mc < MC; ++mc) aK[nb][mc] = aV[nb][mc] = floatx4{0.f, 0.f, 0.f, 0.f};
  const float c = a.scale * kLog2e;
  floatx4 s[2][MC], dp[2][MC], f[2][MC], cc[2][MC];
  typename E::TFrag fPh[MC], fSt[MC], fdS[MC];

  // Transformed row scalars: T0 = -L log2e, T1 = -D (the dP tile's start), T2 = -alpha,
  // T3 = -(alpha D + E) (the C tile's start).  With h = F - alpha:
  //   P h = p h,  St = P (Pt - E) = p (h (dP - D) + C - (alpha D + E)),  dS = p (dP - D).
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
          float FB_LDS* t = (float FB_LDS*)sm.tsc[ks][ts];
          const float Lr = raw[l], Dr = raw[kBS + l], ar = raw[2 * kBS + l], Er = raw[3 * kBS + l];
          t[l] = Lr == -INFINITY ? -INFINITY : -Lr * kLog2e;
          t[kBS + l] = -Dr;
          t[2 * kBS + l] = -ar;
          t[3 * kBS + l] = -__builtin_fmaf(ar, Dr, Er);
        }
      },
      [&](int it, int st, int ts, auto&& prep_next) {
        const int s0 = cl.tile(flat(it)) * kBS;
        const int mode = vector_mode(run.begin + it < run.end ? cl.mode(s0, a.causal != 0) : 0);
        if (mode == 0) {
          prep_next();
          return;
        }
        const T FB_LDS* Qs = (const T FB_LDS*)sm.lds[ks][st];
        const T FB_LDS* UQs = Qs + G::kTileElems;
        const T FB_LDS* dOs = UQs + G::kTileElems;
        const float FB_LDS* Ts = (const float FB_LDS*)sm.tsc[ks][ts];
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
          const floatx4 t1 = *(const floatx4 FB_LDS*)(Ts + kBS + 16 * sb + 4 * g);
          const floatx4 t3 = *(const floatx4 FB_LDS*)(Ts + 3 * kBS + 16 * sb + 4 * g);
#pragma unroll
          for (int mc = 0; mc < MC; ++mc) {
            s[sb][mc] = f[sb][mc] = floatx4{0.f, 0.f, 0.f, 0.f};
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
        const int base = cl.col0 - (cl.start + s0);
        const int side = kBias ? ext_side(base - (kBS - 1), base + 16 * MC - 1, a.R) : 0;
        float kb = 0.f, ku = 0.f;
        if constexpr (kBias) {
          if (side != 0) {
            const int end = side < 0 ? 0 : ext_steps(a) - 1;
            kb = mem.steps[end];
            ku = mem.dirs[end];
          }
        }
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
          floatx4 t0 = *(const floatx4 FB_LDS*)(Ts + 16 * sb + 4 * g);
          floatx4 t2 = *(const floatx4 FB_LDS*)(Ts + 2 * kBS + 16 * sb + 4 * g);
          if constexpr (kBias) {
            t0 += kb;
            t2 += ku;
          }
#pragma unroll
          for (int mc = 0; mc < MC; ++mc)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              s[sb][mc][r] = __builtin_fmaf(s[sb][mc][r], c, t0[r]);
              f[sb][mc][r] = __builtin_fmaf(f[sb][mc][r], a.scale, t2[r]);   // h
            }
        }
        typename E::AFrag cur[3];
        if constexpr (kPF) {
#pragma unroll
          for (int t = 0; t < 3; ++t) cur[t] = G::load_afrag(Qs + t * G::kTileElems, 0);
        }
        if constexpr (kBias) {
          if (side == 0) {
            const int at = a.R + kStepPad + base + j - 4 * g - 19;
#pragma unroll
            for (int sb = 0; sb < 2; ++sb)
#pragma unroll
              for (int mc = 0; mc < MC; ++mc)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  s[sb][mc][r] += mem.steps[at + (19 + 16 * mc - 16 * sb - r)];
                  f[sb][mc][r] += mem.dirs[at + (19 + 16 * mc - 16 * sb - r)];
                }
          }
        }
        if (mode == 2) ext_mask_cols(s, s0, cl.col0 + j, cl.qlen, cl.klen, cl.start, a.causal != 0);
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int mc = 0; mc < MC; ++mc) {
              const float p = fast_exp2(s[sb][mc][r]);
              const float h = f[sb][mc][r], dd = dp[sb][mc][r];
              const int i = 4 * sb + r;
              fPh[mc].set(i, p * h);
              cc[sb][mc][r] = p * __builtin_fmaf(h, dd, cc[sb][mc][r]);
              fSt[mc].set(i, cc[sb][mc][r]);
              fdS[mc].set(i, p * dd);
            }
        if constexpr (kBias) {
          if (sums != nullptr) {
            if (side != 0)
              tab.far(cc, base, side);
            else
              tab.near(cc, base, mem.buf);
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
              for (int t = 0; t < 3; ++t) cur[t] = G::load_afrag(Qs + t * G::kTileElems, 16 * (nb + 1));
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
  if constexpr (kBias)
    if (sums != nullptr) tab.finish(cl.col0 - (cl.start + cl.tile(max(run.end - 1, 0)) * kBS));
  if constexpr (KS > 1) {
    static_assert(sizeof(sm.lds) >= merge_bytes<KS, NW, G::kNB, MC>(), "set merge buffer");
    merge_sets<KS, NW>(aK, ks, wl, (floatx4 FB_LDS*)&sm.lds[0][0][0]);
    merge_sets<KS, NW>(aV, ks, wl, (floatx4 FB_LDS*)&sm.lds[0][0][0]);
  }
  ext_store_cols<T, D, KS>(a, kv, cl.col0, cl.klen, ks, aK, aV, a.scale, 1.f, Kt, Vt, parts);
}

}  // namespace fb
