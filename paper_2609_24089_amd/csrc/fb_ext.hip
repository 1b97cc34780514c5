// C ABI of the attention between sequences of two lengths: validation and dispatch, and the
// kernels that add parts and gather the bias table's gradients.  The entry points are
// declared (and documented) in include/flashbob.h.
#include "fb_ext.h"

namespace fb {

// The sum of rows r0, r0 + by, ... below `rows` of column x, eight loads in flight: the
// rows are few and far apart, so one load after another was all latency.
__device__ __forceinline__ float sum_rows(const float* __restrict__ m, int64_t r0, int64_t rows, int64_t by, int width,
                                          int x) {
  float v[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) v[u] = 0.f;
  int64_t r = r0;
  for (; r + 7 * by < rows; r += 8 * by)
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] += m[(r + u * by) * width + x];
#pragma unroll
  for (int u = 0; u < 7; ++u)
    if (r + u * by < rows) v[u] += m[(r + u * by) * width + x];
  return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}

// Adds the waves' rows of step sums (StepSums) of head blockIdx.y: workgroup s of S takes
// rows s, s + S, ... of the head's `rows` and writes one row of `mid` ([H][S][width]).
__global__ __launch_bounds__(256) void ext_step_rows_kernel(const float* __restrict__ sums, int64_t rows, int width,
                                                            float* __restrict__ mid) {
  const float* const head = sums + (int64_t)blockIdx.y * rows * width;
  float* const out = mid + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * width;
  for (int x = threadIdx.x; x < width; x += 256) out[x] = sum_rows(head, blockIdx.x, rows, gridDim.x, width, x);
}

// Gathers head blockIdx.x's sums by step into its buckets: four groups of 256 threads add
// every fourth row of a step, then `lanes` threads share a bucket's steps.  The order of the
// sums is fixed.  All of it is latency: with eight threads a bucket, which read the four
// groups' sums, a gather of 16 rows of 259 steps took 7.4 us.
constexpr int kMaxWidth = 2 * kMaxDistance + 3;
constexpr int kGroups = 4, kGatherThreads = 256 * kGroups;
__global__ __launch_bounds__(kGatherThreads) void ext_buckets_kernel(const float* __restrict__ rows, int n, int lanes,
                                                                     ExtArgs a, void* __restrict__ out) {
  __shared__ float part[kGroups][kMaxWidth];
  __shared__ int bucket[kMaxWidth];
  const int width = 2 * a.R + 3, group = threadIdx.x >> 8;
  const float* const mine = rows + (int64_t)blockIdx.x * n * width;
  for (int x = threadIdx.x & 255; x < width; x += 256) {
    if (group == 0) {
      // the two sums beyond the steps belong to the buckets of the ends
      const int step = x <= 2 * a.R ? x : x == 2 * a.R + 1 ? 0 : 2 * a.R;
      bucket[x] = min(max(a.buckets[step], 0), a.num_buckets - 1);
    }
    part[group][x] = sum_rows(mine, group, n, kGroups, width, x);
  }
  __syncthreads();
  for (int x = threadIdx.x; x < width; x += kGatherThreads)
    part[0][x] = (part[0][x] + part[1][x]) + (part[2][x] + part[3][x]);
  __syncthreads();
  const int lane = threadIdx.x & (lanes - 1), at_once = kGatherThreads / lanes;
  for (int c0 = 0; c0 < a.num_buckets; c0 += at_once) {
    const int c = c0 + threadIdx.x / lanes;
    float v = 0.f;
    for (int x = lane; x < width; x += lanes) v += bucket[x] == c ? part[0][x] : 0.f;
    for (int m = 1; m < lanes; m *= 2) v += __shfl_xor(v, m);
    if (lane == 0 && c < a.num_buckets) {
      const int64_t at = (int64_t)c * a.H + blockIdx.x;
      if (a.table_bf16 != 0)
        ((bf16*)out)[at] = (bf16)v;
      else
        ((float*)out)[at] = v;
    }
  }
}

int32_t ext_add_parts(const ExtProblem& p, const ExtArgs& a, const float* parts, void* X, void* Y, hipStream_t s) {
  const int64_t plane = a.rows * p.d, first = a.row0 * p.d;
  const unsigned blocks = (unsigned)std::min<int64_t>((plane / 2 + 255) / 256, 8192);
  (void)hipGetLastError();
  if (p.dtype == BOB_BF16)
    hipLaunchKernelGGL(ext_parts_kernel<bf16>, dim3(blocks), dim3(256), 0, s, parts, a.nparts, plane, (bf16*)X + first,
                       (bf16*)Y + first);
  else
    hipLaunchKernelGGL(ext_parts_kernel<float>, dim3(blocks), dim3(256), 0, s, parts, a.nparts, plane, (float*)X + first,
                       (float*)Y + first);
  return finish_launch();
}

int32_t ext_check(const ExtProblem& p, bool* empty) {
  *empty = false;
  if (p.dtype != BOB_F32 && p.dtype != BOB_BF16) return BOB_EINVAL;
  if (p.B < 0 || p.H < 0 || p.Nq < 0 || p.Nk < 0 || p.d < 1) return BOB_EINVAL;
  if (!std::isfinite(p.scale)) return BOB_EINVAL;
  if (p.causal != 0 && p.causal != 1) return BOB_EINVAL;
  if (p.Hkv < 0 || (p.H > 0 && (p.Hkv < 1 || p.H % p.Hkv != 0))) return BOB_EINVAL;
  if (!supported(p.dtype, p.d)) return BOB_EUNSUPPORTED;
  auto aligned = [](const void* q, uintptr_t n) { return (reinterpret_cast<uintptr_t>(q) & (n - 1)) == 0; };
  if (!aligned(p.x.q_lens, 4) || !aligned(p.x.kv_lens, 4) || !aligned(p.x.q_starts, 4)) return BOB_EINVAL;
  if (has_bias(p)) {
    if (p.x.table_dtype != BOB_F32 && p.x.table_dtype != BOB_BF16) return BOB_EINVAL;
    if (!aligned(p.x.table, p.x.table_dtype == BOB_F32 ? 4 : 2)) return BOB_EINVAL;
    if (p.x.buckets == nullptr || !aligned(p.x.buckets, 4)) return BOB_EINVAL;
    if (p.x.num_buckets < 1 || p.x.num_buckets > kMaxBuckets) return BOB_EINVAL;
    if (p.x.max_distance < 1 || p.x.max_distance > kMaxDistance) return BOB_EINVAL;
  }
  if (p.H == 0 || (p.B == 0 && !has_bias(p))) {
    *empty = true;
    return BOB_OK;
  }
  if (p.Nq > kMaxN || p.Nk > kMaxN) return BOB_EINVAL;
  // 2^30 rows of all heads: a launch takes fewer than 2^32 threads, and the whole blocks have
  // 64 rows or more in 256 threads.  A column block streams a group's query tiles in one loop.
  if (p.B > INT32_MAX || p.H > 65535) return BOB_EINVAL;
  const int64_t heads = p.B * p.H, rows = std::max(p.Nq, p.Nk);
  if (heads > INT32_MAX) return BOB_EINVAL;
  if (heads * ((rows + 63) / 64) >= int64_t(1) << 24) return BOB_EINVAL;
  if (ext_group(p) * p.Nq > INT32_MAX / 2) return BOB_EINVAL;
  return BOB_OK;
}

static ExtProblem ext_problem(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t d,
                              float scale, int32_t causal, const attn_ext* ext) {
  ExtProblem p{dtype, B, H, Hkv, Nq, Nk, d, scale, causal, attn_ext{}};
  if (ext != nullptr) p.x = *ext;
  return p;
}

static int64_t fwd_bytes(const ExtProblem& p, const ExtPlan& c) { return ext_row_bytes(p, c, p.d + 2); }
static int64_t rows_bytes(const ExtProblem& p, const ExtPlan& c) { return ext_row_bytes(p, c, p.d + 1); }
static int64_t pass1_bytes(const ExtProblem& p, const ExtPlan& c) { return ext_row_bytes(p, c, 3 * p.d + 4); }
// Workspace of a column kernel: the parts' fp32 sums, then the waves' rows of step sums and
// what ext_step_rows_kernel makes of them.
struct ColBytes {
  int64_t parts = 0, rows = 0, sums = 0, mid = 0;  // rows: of step sums of one head
  int S = 0;  // rows a head that ext_step_rows_kernel makes of them; 0: it does not run
  int64_t all() const { return parts + sums + mid; }
};
static ColBytes col_bytes(const ExtProblem& p, const ExtPlan& c) {
  ColBytes b;
  if (c.parts > 1) b.parts = (int64_t)c.parts * 2 * ext_slices(p, c).rows * p.d * 4;
  if (has_bias(p)) {
    const int64_t blocks = (p.Nk + 16 * c.blocks - 1) / (16 * c.blocks);
    const int subs = c.parts > 1 ? c.parts / ext_group(p) : 1;
    b.rows = p.B * blocks * subs * c.waves;
    // few rows go straight to the gather, for one launch less: 256 rows of 259 steps 8.0 us for
    // 5.4 + 4.9
    b.S = b.rows <= 256 ? 0 : (int)std::min<int64_t>(16, b.rows / 8);
    auto pad = [](int64_t n) { return (n + 15) / 16 * 16; };
    b.sums = pad(b.rows * p.H * ext_width(p) * 4);
    b.mid = pad(b.S * p.H * ext_width(p) * 4);
  }
  return b;
}

static ExtPlan plan_fwd(const ExtProblem& p) { FB_EXT_DISPATCH(p, ext_fwd_plan, p); }
static ExtPlan plan_rows(const ExtProblem& p) { FB_EXT_DISPATCH(p, ext_rows_plan, p); }
static ExtPlan plan_pass1(const ExtProblem& p) { FB_EXT_DISPATCH(p, ext_pass1_plan, p); }
static ExtPlan plan_cols(const ExtProblem& p) { FB_EXT_DISPATCH(p, ext_cols_plan, p); }
static ExtPlan plan_pass2(const ExtProblem& p) { FB_EXT_DISPATCH(p, ext_pass2_plan, p); }
static int32_t go_fwd(const ExtProblem& p, const void* Q, const void* K, const void* V, void* O, float* L, float* ws,
                      hipStream_t s) {
  FB_EXT_DISPATCH(p, ext_launch_fwd, p, Q, K, V, O, L, ws, s);
}
static int32_t go_bwd(const ExtProblem& p, const void* Q, const void* K, const void* V, const void* O, const void* dO,
                      const float* L, void* dQ, void* dK, void* dV, float* D, float* row_parts, float* parts,
                      float* sums, hipStream_t s) {
  FB_EXT_DISPATCH(p, ext_launch_bwd, p, Q, K, V, O, dO, L, dQ, dK, dV, D, row_parts, parts, sums, s);
}
static int32_t go_pass1(const ExtProblem& p, const void* Q, const void* K, const void* V, const void* O,
                        const void* dO, const void* UQ, const void* UK, const void* UV, const void* UT, const float* L,
                        const float* D, const void* dQ, void* Qt, void* dOt, float* alpha, float* E, float* parts,
                        hipStream_t s) {
  FB_EXT_DISPATCH(p, ext_launch_pass1, p, Q, K, V, O, dO, UQ, UK, UV, UT, L, D, dQ, Qt, dOt, alpha, E, parts, s);
}
static int32_t go_pass2(const ExtProblem& p, const void* Q, const void* K, const void* V, const void* dO,
                        const void* UQ, const void* UK, const void* UV, const void* UT, const float* L, const float* D,
                        const float* alpha, const float* E, void* Kt, void* Vt, float* parts, float* sums,
                        hipStream_t s) {
  FB_EXT_DISPATCH(p, ext_launch_pass2, p, Q, K, V, dO, UQ, UK, UV, UT, L, D, alpha, E, Kt, Vt, parts, sums, s);
}

// The rows of step sums -> the table's gradient.
static int32_t gather_table(const ExtProblem& p, const ColBytes& b, const float* sums, float* mid, void* out,
                            hipStream_t s) {
  const int width = (int)ext_width(p);
  const ExtArgs a = ext_args(p, ExtPlan{}, 0, 0, nullptr);
  int lanes = 64;
  while (lanes > 1 && lanes * p.x.num_buckets > kGatherThreads) lanes /= 2;
  (void)hipGetLastError();
  if (b.S > 0)
    hipLaunchKernelGGL(ext_step_rows_kernel, dim3(b.S, (unsigned)p.H), dim3(256), 0, s, sums, b.rows, width, mid);
  hipLaunchKernelGGL(ext_buckets_kernel, dim3((unsigned)p.H), dim3(kGatherThreads), 0, s,
                     b.S > 0 ? (const float*)mid : sums, b.S > 0 ? b.S : (int)b.rows, lanes, a, out);
  return finish_launch();
}

// A table's gradient pointer: not without a table, aligned to its type.
static bool table_ptr(const ExtProblem& p, const void* t) {
  if (t == nullptr) return true;
  return has_bias(p) && (reinterpret_cast<uintptr_t>(t) & (p.x.table_dtype == BOB_F32 ? 3u : 1u)) == 0;
}

}  // namespace fb

using fb::ExtProblem;

extern "C" {

int32_t attn_ext_fwd_lse(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t d,
                         float scale, int32_t causal, const attn_ext* ext, const void* Q, const void* K, const void* V,
                         void* O, float* L, void* workspace, int64_t workspace_bytes, void* stream) {
  const ExtProblem p = fb::ext_problem(dtype, B, H, Hkv, Nq, Nk, d, scale, causal, ext);
  bool empty;
  const int32_t rc = fb::ext_check(p, &empty);
  if (rc != BOB_OK || empty || B == 0 || Nq == 0) return rc;
  if (!fb::ext_ptrs(Nq, {Q, O, L}) || !fb::ext_ptrs(Nk, {K, V})) return BOB_EINVAL;
  const int64_t need = fb::fwd_bytes(p, fb::plan_fwd(p));
  if (need > 0 && (workspace_bytes < need || !fb::aligned16(workspace))) return BOB_EINVAL;
  return fb::go_fwd(p, Q, K, V, O, L, (float*)workspace, (hipStream_t)stream);
}

int32_t attn_ext_bwd(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t d, float scale,
                     int32_t causal, const attn_ext* ext, const void* Q, const void* K, const void* V, const void* O,
                     const void* dO, const float* L, void* dQ, void* dK, void* dV, float* D, void* dT, void* workspace,
                     int64_t workspace_bytes, void* stream) {
  const ExtProblem p = fb::ext_problem(dtype, B, H, Hkv, Nq, Nk, d, scale, causal, ext);
  bool empty;
  int32_t rc = fb::ext_check(p, &empty);
  if (rc != BOB_OK || empty) return rc;
  if (!fb::ext_ptrs(B * Nq, {Q, O, dO, L, dQ, D}) || !fb::ext_ptrs(B * Nk, {K, V, dK, dV}) || !fb::table_ptr(p, dT))
    return BOB_EINVAL;
  const fb::ColBytes b = fb::col_bytes(p, fb::plan_cols(p));
  const int64_t rows = fb::rows_bytes(p, fb::plan_rows(p)), need = rows + b.all();
  if (need > 0 && (workspace_bytes < need || !fb::aligned16(workspace))) return BOB_EINVAL;
  char* const row_ws = (char*)workspace;
  char* const ws = row_ws + rows;
  float* const sums = dT != nullptr ? (float*)(ws + b.parts) : nullptr;
  if (B > 0)
    rc = fb::go_bwd(p, Q, K, V, O, dO, L, dQ, dK, dV, D, (float*)row_ws, (float*)ws, sums, (hipStream_t)stream);
  if (rc != BOB_OK || dT == nullptr) return rc;
  return fb::gather_table(p, b, sums, (float*)(ws + b.parts + b.sums), dT, (hipStream_t)stream);
}

int32_t attn_ext_pass1_rows(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t d,
                            float scale, int32_t causal, const attn_ext* ext, const void* Q, const void* K,
                            const void* V, const void* O, const void* dO, const void* gdQ, const void* gdK,
                            const void* gdV, const void* gdT, const float* L, const float* D, const void* dQ, void* Qt,
                            void* dOt, float* alpha, float* E, void* workspace, int64_t workspace_bytes,
                            void* stream) {
  const ExtProblem p = fb::ext_problem(dtype, B, H, Hkv, Nq, Nk, d, scale, causal, ext);
  bool empty;
  const int32_t rc = fb::ext_check(p, &empty);
  if (rc != BOB_OK || empty || B == 0 || Nq == 0) return rc;
  if (!fb::ext_ptrs(Nq, {Q, O, dO, gdQ, L, D, dQ, Qt, dOt, alpha, E}) || !fb::ext_ptrs(Nk, {K, V, gdK, gdV}) ||
      !fb::table_ptr(p, gdT))
    return BOB_EINVAL;
  const int64_t need = fb::pass1_bytes(p, fb::plan_pass1(p));
  if (need > 0 && (workspace_bytes < need || !fb::aligned16(workspace))) return BOB_EINVAL;
  return fb::go_pass1(p, Q, K, V, O, dO, gdQ, gdK, gdV, gdT, L, D, dQ, Qt, dOt, alpha, E, (float*)workspace,
                      (hipStream_t)stream);
}

int32_t attn_ext_pass2_cols(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t d,
                            float scale, int32_t causal, const attn_ext* ext, const void* Q, const void* K,
                            const void* V, const void* dO, const void* gdQ, const void* gdK, const void* gdV,
                            const void* gdT, const float* L, const float* D, const float* alpha, const float* E,
                            void* Kt, void* Vt, void* Tt, void* workspace, int64_t workspace_bytes, void* stream) {
  const ExtProblem p = fb::ext_problem(dtype, B, H, Hkv, Nq, Nk, d, scale, causal, ext);
  bool empty;
  int32_t rc = fb::ext_check(p, &empty);
  if (rc != BOB_OK || empty) return rc;
  if (!fb::ext_ptrs(B * Nq, {Q, dO, gdQ, L, D, alpha, E}) || !fb::ext_ptrs(B * Nk, {K, V, gdK, gdV, Kt, Vt}) ||
      !fb::table_ptr(p, gdT) || !fb::table_ptr(p, Tt))
    return BOB_EINVAL;
  const fb::ColBytes b = fb::col_bytes(p, fb::plan_pass2(p));
  const int64_t need = b.all();
  if (need > 0 && (workspace_bytes < need || !fb::aligned16(workspace))) return BOB_EINVAL;
  char* const ws = (char*)workspace;
  float* const sums = Tt != nullptr ? (float*)(ws + b.parts) : nullptr;
  if (B > 0 && Nk > 0)
    rc = fb::go_pass2(p, Q, K, V, dO, gdQ, gdK, gdV, gdT, L, D, alpha, E, Kt, Vt, (float*)ws, sums,
                      (hipStream_t)stream);
  if (rc != BOB_OK || Tt == nullptr) return rc;
  return fb::gather_table(p, b, sums, (float*)(ws + b.parts + b.sums), Tt, (hipStream_t)stream);
}

int64_t attn_ext_fwd_workspace_bytes(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk,
                                     int64_t d, int32_t causal, const attn_ext* ext) {
  const ExtProblem p = fb::ext_problem(dtype, B, H, Hkv, Nq, Nk, d, 1.0f, causal, ext);
  bool empty;
  if (fb::ext_check(p, &empty) != BOB_OK || empty || B == 0 || Nq == 0) return 0;
  return fb::fwd_bytes(p, fb::plan_fwd(p));
}

int64_t attn_ext_bwd_workspace_bytes(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk,
                                     int64_t d, int32_t causal, const attn_ext* ext) {
  const ExtProblem p = fb::ext_problem(dtype, B, H, Hkv, Nq, Nk, d, 1.0f, causal, ext);
  bool empty;
  if (fb::ext_check(p, &empty) != BOB_OK || empty) return 0;
  return fb::rows_bytes(p, fb::plan_rows(p)) + fb::col_bytes(p, fb::plan_cols(p)).all();
}

int64_t attn_ext_pass1_workspace_bytes(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk,
                                       int64_t d, int32_t causal, const attn_ext* ext) {
  const ExtProblem p = fb::ext_problem(dtype, B, H, Hkv, Nq, Nk, d, 1.0f, causal, ext);
  bool empty;
  if (fb::ext_check(p, &empty) != BOB_OK || empty || B == 0 || Nq == 0) return 0;
  return fb::pass1_bytes(p, fb::plan_pass1(p));
}

int64_t attn_ext_pass2_workspace_bytes(int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk,
                                       int64_t d, int32_t causal, const attn_ext* ext) {
  const ExtProblem p = fb::ext_problem(dtype, B, H, Hkv, Nq, Nk, d, 1.0f, causal, ext);
  bool empty;
  if (fb::ext_check(p, &empty) != BOB_OK || empty) return 0;
  return fb::col_bytes(p, fb::plan_pass2(p)).all();
}

int32_t attn_ext_layout(int32_t kernel, int32_t dtype, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t Nk,
                        int64_t d, int32_t causal, const attn_ext* ext, attn_ext_launch* launch) {
  if (kernel < ATTN_EXT_FWD || kernel > ATTN_EXT_PASS2 || launch == nullptr) return BOB_EINVAL;
  const ExtProblem p = fb::ext_problem(dtype, B, H, Hkv, Nq, Nk, d, 1.0f, causal, ext);
  bool empty;
  const int32_t rc = fb::ext_check(p, &empty);
  if (rc != BOB_OK) return rc;
  *launch = attn_ext_launch{};
  const bool columns = kernel == ATTN_EXT_COLS || kernel == ATTN_EXT_PASS2;
  if (empty || B == 0 || (columns ? Nk : Nq) == 0) return BOB_OK;
  const fb::ExtPlan c = kernel == ATTN_EXT_FWD     ? fb::plan_fwd(p)
                        : kernel == ATTN_EXT_ROWS  ? fb::plan_rows(p)
                        : kernel == ATTN_EXT_COLS  ? fb::plan_cols(p)
                        : kernel == ATTN_EXT_PASS1 ? fb::plan_pass1(p)
                                                   : fb::plan_pass2(p);
  *launch = attn_ext_launch{16 * c.blocks, c.sets, c.parts, c.fold ? 1 : 0, c.resident};
  return BOB_OK;
}

}  // extern "C"
