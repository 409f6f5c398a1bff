// C-ABI front end of the operators around the long convolution: the gated linear
// recurrence, and the norms before and behind a residual block.  Validation and sizing are pure host code; nothing here touches
// the GPU before every check has passed.
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <cmath>

#include "../../include/hyenand.h"
#include "kernels.hpp"
#include "norm.hpp"
#include "scan.hpp"

namespace hyenand {

hyenand_status set_last_error(hyenand_status s, const char* msg);

namespace {

hyenand_status fail(hyenand_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return set_last_error(s, buf);
}

// A device buffer of a call.
struct Buffer {
  const char* name;
  const void* p;
  size_t bytes, align;
  bool out, optional;
};

bool overlap(const Buffer& a, const Buffer& b) {
  const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
  return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}

// Required buffers given, all aligned, no output overlapping another buffer
// (same: an output that may be the very buffer of that input).
template <int N>
hyenand_status check_buffers(const Buffer (&b)[N], const char* same_out = "", const char* same_in = "") {
  for (const Buffer& x : b)
    if (!x.p && !x.optional) return fail(HYENAND_ERR_INVALID_ARGUMENT, "%s is NULL", x.name);
  for (const Buffer& x : b)
    if (x.p && (uintptr_t)x.p % x.align != 0)
      return fail(HYENAND_ERR_INVALID_ARGUMENT, "%s is not %zu-byte aligned", x.name, x.align);
  for (const Buffer& x : b) {
    if (!x.p || !x.out) continue;
    for (const Buffer& y : b) {
      if (&x == &y || !y.p || (y.out && &y > &x) || !overlap(x, y)) continue;
      if (x.p == y.p && !strcmp(x.name, same_out) && !strcmp(y.name, same_in)) continue;
      return fail(HYENAND_ERR_INVALID_ARGUMENT, "%s overlaps %s", x.name, y.name);
    }
  }
  return HYENAND_OK;
}

constexpr int64_t kMaxRows = (int64_t(1) << 26) - 4;  // B * C: 64 work-items a row, 4 rows a workgroup, fewer than 2^32 in a launch

hyenand_status check_shape(int64_t B, int64_t C, int64_t L, const char* last, int dtype) {
  if (dtype != HYENAND_DTYPE_F32 && dtype != HYENAND_DTYPE_BF16)
    return fail(HYENAND_ERR_INVALID_ARGUMENT, "dtype must be 0 (f32) or 1 (bf16), got %d", dtype);
  if (B < 1 || C < 1 || L < 1)
    return fail(HYENAND_ERR_INVALID_ARGUMENT, "B = %lld, C = %lld and %s = %lld must be >= 1", (long long)B,
                (long long)C, last, (long long)L);
  if (B > kMaxRows || C > kMaxRows || B * C > kMaxRows)
    return fail(HYENAND_ERR_UNSUPPORTED, "B * C = %lld x %lld (b, c) rows exceed the %lld one call takes", (long long)B,
                (long long)C, (long long)kMaxRows);
  if (L > (int64_t(1) << 40) || B * C > (int64_t(1) << 46) / L) return fail(HYENAND_ERR_UNSUPPORTED, "tensor too large");
  return HYENAND_OK;
}

hyenand_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return HYENAND_OK;
  if (!ws || bytes < need)
    return fail(HYENAND_ERR_WORKSPACE_TOO_SMALL, "the call needs %zu workspace bytes, got %zu", need, ws ? bytes : (size_t)0);
  if ((uintptr_t)ws % 16 != 0) return fail(HYENAND_ERR_INVALID_ARGUMENT, "workspace is not 16-byte aligned");
  return HYENAND_OK;
}

hyenand_status launched(hipError_t e) {
  return e == hipSuccess ? HYENAND_OK : fail(HYENAND_ERR_HIP, "HIP error %d: %s", (int)e, hipGetErrorString(e));
}

hyenand_status check_norm_shape(int64_t B, int64_t C, int64_t P, int dtype) {
  const hyenand_status st = check_shape(B, C, P, "P", dtype);
  if (st != HYENAND_OK) return st;
  if (P > kMaxNormPoints / B)
    return fail(HYENAND_ERR_UNSUPPORTED, "B * P = %lld x %lld points exceed the %lld one call takes", (long long)B,
                (long long)P, (long long)kMaxNormPoints);
  return HYENAND_OK;
}

int64_t scan_states_of(int64_t L) { return (L + kScanTile - 1) / kScanTile; }
static_assert(kScanTile == HYENAND_SCAN_BLOCK, "a state is kept before every tile");

// The arguments that the norms' forward and backward share; x is x_out in the
// backward.
hyenand_status check_norm(const void* z, const void* gate, const void* w_post, const void* scale, float eps_post,
                          float eps_pre, float p, const void* rng, NormArgs* a) {
  if (!z && (gate || w_post || scale))
    return fail(HYENAND_ERR_INVALID_ARGUMENT, "gate, w_post and scale belong to a branch z: without it they are NULL");
  if (z && !w_post) return fail(HYENAND_ERR_INVALID_ARGUMENT, "w_post is NULL");
  if (!(eps_post >= 0.f) || !(eps_pre >= 0.f) || !std::isfinite(eps_post) || !std::isfinite(eps_pre))
    return fail(HYENAND_ERR_INVALID_ARGUMENT, "eps_post = %g and eps_pre = %g must be finite and >= 0", (double)eps_post,
                (double)eps_pre);
  if (!(p >= 0.f && p < 1.f)) return fail(HYENAND_ERR_INVALID_ARGUMENT, "dropout_p = %g must be in [0, 1)", (double)p);
  if (p > 0.f && !z) return fail(HYENAND_ERR_INVALID_ARGUMENT, "dropout belongs to a branch z");
  if (p > 0.f && !rng) return fail(HYENAND_ERR_INVALID_ARGUMENT, "rng is NULL: dropout takes a seed and an offset");
  const double drop = std::floor((double)p * 65536.0 + 0.5);
  a->drop = drop > 65535.0 ? 65535u : (uint32_t)drop;
  a->kept = (float)(65536.0 / (65536.0 - a->drop));
  a->eps_post = eps_post;
  a->eps_pre = eps_pre;
  return HYENAND_OK;
}

hyenand_status workspace_size(int64_t B, int64_t C, int64_t L, int dtype, bool backward, size_t* bytes_out) {
  if (!bytes_out) return fail(HYENAND_ERR_INVALID_ARGUMENT, "bytes_out is NULL");
  const hyenand_status st = check_shape(B, C, L, "L", dtype);
  if (st == HYENAND_OK) *bytes_out = scan_workspace_bytes(B * C, L, backward);
  return st;
}

}  // namespace
}  // namespace hyenand

using namespace hyenand;

extern "C" {

hyenand_status hyenand_scan_workspace_size(int64_t B, int64_t C, int64_t L, hyenand_dtype dtype, size_t* bytes_out) {
  return workspace_size(B, C, L, dtype, false, bytes_out);
}

hyenand_status hyenand_scan_backward_workspace_size(int64_t B, int64_t C, int64_t L, hyenand_dtype dtype,
                                                    size_t* bytes_out) {
  return workspace_size(B, C, L, dtype, true, bytes_out);
}

hyenand_status hyenand_scan(const void* x1, const void* x2, const void* v, const void* log_a, const void* D,
                            const float* h0, const int64_t* lengths, void* y, float* h_last, float* states, int64_t B,
                            int64_t C, int64_t L, hyenand_dtype dtype, void* workspace, size_t workspace_bytes,
                            void* stream) {
  hyenand_status st = check_shape(B, C, L, "L", dtype);
  if (st != HYENAND_OK) return st;
  const size_t es = dtype == HYENAND_DTYPE_BF16 ? 2 : 4, rows = (size_t)(B * C), n = rows * (size_t)L * es;
  const size_t need = scan_workspace_bytes(B * C, L, false);
  const Buffer bufs[] = {{"x1", x1, n, es, false, false},
                         {"x2", x2, n, es, false, false},
                         {"v", v, n, es, false, false},
                         {"log_a", log_a, n, es, false, false},
                         {"D", D, (size_t)C * es, es, false, false},
                         {"h0", h0, rows * 4, 4, false, true},
                         {"lengths", lengths, (size_t)B * 8, 8, false, true},
                         {"y", y, n, es, true, false},
                         {"h_last", h_last, rows * 4, 4, true, true},
                         {"states", states, rows * (size_t)scan_states_of(L) * 4, 4, true, true},
                         {"workspace", need ? workspace : nullptr, need, 1, true, true}};
  st = check_workspace(workspace, workspace_bytes, need);
  if (st == HYENAND_OK) st = check_buffers(bufs, "h_last", "h0");
  if (st != HYENAND_OK) return st;
  ScanArgs a;
  memset(&a, 0, sizeof a);
  a.x1 = x1;
  a.x2 = x2;
  a.v = v;
  a.la = log_a;
  a.D = D;
  a.h0 = h0;
  a.len = lengths;
  a.y = y;
  a.h_last = h_last;
  a.states = states;
  a.R = B * C;
  a.L = L;
  a.C = (int)C;
  a.nst = scan_states_of(L);
  a.bf16 = dtype == HYENAND_DTYPE_BF16;
  clear_pending_error();
  return launched(launch_scan(a, workspace, (hipStream_t)stream));
}

hyenand_status hyenand_scan_backward(const void* x1, const void* x2, const void* v, const void* log_a, const void* D,
                                     const int64_t* lengths, const float* states, const void* gy, const float* gh_last,
                                     void* gx1, void* gx2, void* gv, void* glog_a, void* gD, float* gh0, int64_t B,
                                     int64_t C, int64_t L, hyenand_dtype dtype, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  hyenand_status st = check_shape(B, C, L, "L", dtype);
  if (st != HYENAND_OK) return st;
  const size_t es = dtype == HYENAND_DTYPE_BF16 ? 2 : 4, rows = (size_t)(B * C), n = rows * (size_t)L * es;
  const size_t need = scan_workspace_bytes(B * C, L, true);
  const Buffer bufs[] = {{"x1", x1, n, es, false, false},
                         {"x2", x2, n, es, false, false},
                         {"v", v, n, es, false, false},
                         {"log_a", log_a, n, es, false, false},
                         {"D", D, (size_t)C * es, es, false, false},
                         {"lengths", lengths, (size_t)B * 8, 8, false, true},
                         {"states", states, rows * (size_t)scan_states_of(L) * 4, 4, false, false},
                         {"gy", gy, n, es, false, false},
                         {"gh_last", gh_last, rows * 4, 4, false, true},
                         {"gx1", gx1, n, es, true, false},
                         {"gx2", gx2, n, es, true, false},
                         {"gv", gv, n, es, true, false},
                         {"glog_a", glog_a, n, es, true, false},
                         {"gD", gD, (size_t)C * es, es, true, false},
                         {"gh0", gh0, rows * 4, 4, true, true},
                         {"workspace", need ? workspace : nullptr, need, 1, true, true}};
  st = check_workspace(workspace, workspace_bytes, need);
  if (st == HYENAND_OK) st = check_buffers(bufs);
  if (st != HYENAND_OK) return st;
  ScanArgs a;
  memset(&a, 0, sizeof a);
  a.x1 = x1;
  a.x2 = x2;
  a.v = v;
  a.la = log_a;
  a.D = D;
  a.len = lengths;
  a.states = const_cast<float*>(states);
  a.gy = gy;
  a.gh_last = gh_last;
  a.gx1 = gx1;
  a.gx2 = gx2;
  a.gv = gv;
  a.gla = glog_a;
  a.gD = gD;
  a.gh0 = gh0;
  a.R = B * C;
  a.L = L;
  a.C = (int)C;
  a.nst = scan_states_of(L);
  a.bf16 = dtype == HYENAND_DTYPE_BF16;
  clear_pending_error();
  return launched(launch_scan_backward(a, workspace, (hipStream_t)stream));
}

hyenand_status hyenand_scan_step(const void* x1, const void* x2, const void* v, const void* log_a, const void* D,
                                 const int64_t* slots, float* state, void* y, int64_t B, int64_t C, int64_t num_slots,
                                 hyenand_dtype dtype, void* stream) {
  hyenand_status st = check_shape(B, C, 1, "L", dtype);
  if (st != HYENAND_OK) return st;
  if (B > 65535) return fail(HYENAND_ERR_UNSUPPORTED, "B = %lld exceeds the 65535 one step takes", (long long)B);
  if (num_slots < 1 || (!slots && num_slots < B))
    return fail(HYENAND_ERR_INVALID_ARGUMENT, "num_slots = %lld: without slots every one of the %lld rows has a state",
                (long long)num_slots, (long long)B);
  if (num_slots > (int64_t(1) << 46) / C) return fail(HYENAND_ERR_UNSUPPORTED, "state too large");
  const size_t es = dtype == HYENAND_DTYPE_BF16 ? 2 : 4, n = (size_t)(B * C) * es;
  const Buffer bufs[] = {{"x1", x1, n, es, false, false},
                         {"x2", x2, n, es, false, false},
                         {"v", v, n, es, false, false},
                         {"log_a", log_a, n, es, false, false},
                         {"D", D, (size_t)C * es, es, false, false},
                         {"slots", slots, (size_t)B * 8, 8, false, true},
                         {"state", state, (size_t)num_slots * (size_t)C * 4, 4, true, false},
                         {"y", y, n, es, true, false}};
  st = check_buffers(bufs);
  if (st != HYENAND_OK) return st;
  const ScanStepArgs a = {x1, x2, v, log_a, D, slots, state, y, B, num_slots, (int)C, dtype == HYENAND_DTYPE_BF16};
  clear_pending_error();
  return launched(launch_scan_step(a, (hipStream_t)stream));
}

hyenand_status hyenand_block_norm(const void* x, const void* z, const void* gate, const void* w_post, const void* scale,
                                  const void* w_pre, float eps_post, float eps_pre, float dropout_p,
                                  const uint64_t* rng, void* x_out, void* n, int64_t B, int64_t C, int64_t P,
                                  hyenand_dtype dtype, void* stream) {
  hyenand_status st = check_norm_shape(B, C, P, dtype);
  if (st != HYENAND_OK) return st;
  NormArgs a;
  memset(&a, 0, sizeof a);
  st = check_norm(z, gate, w_post, scale, eps_post, eps_pre, dropout_p, rng, &a);
  if (st != HYENAND_OK) return st;
  if (!z != !x_out) return fail(HYENAND_ERR_INVALID_ARGUMENT, "z and x_out must both be given or both be NULL");
  if (!w_pre != !n) return fail(HYENAND_ERR_INVALID_ARGUMENT, "w_pre and n must both be given or both be NULL");
  if (!z && !n) return fail(HYENAND_ERR_INVALID_ARGUMENT, "neither a branch z nor a norm n is asked for");
  const size_t es = dtype == HYENAND_DTYPE_BF16 ? 2 : 4, bytes = (size_t)(B * C) * (size_t)P * es, row = (size_t)C * es;
  const Buffer bufs[] = {{"x", x, bytes, es, false, false},        {"z", z, bytes, es, false, true},
                         {"gate", gate, bytes, es, false, true},   {"w_post", w_post, row, es, false, true},
                         {"scale", scale, row, es, false, true},   {"w_pre", w_pre, row, es, false, true},
                         {"rng", rng, 16, 8, false, true},         {"x_out", x_out, bytes, es, true, true},
                         {"n", n, bytes, es, true, true}};
  st = check_buffers(bufs);
  if (st != HYENAND_OK) return st;
  a.x = x;
  a.z = z;
  a.g = gate;
  a.w_post = w_post;
  a.scale = scale;
  a.w_pre = w_pre;
  a.rng = rng;
  a.x_out = x_out;
  a.n = n;
  a.B = B;
  a.C = (int)C;
  a.P = P;
  a.bf16 = dtype == HYENAND_DTYPE_BF16;
  clear_pending_error();
  return launched(launch_norm(a, (hipStream_t)stream));
}

hyenand_status hyenand_block_norm_backward_workspace_size(int64_t B, int64_t C, int64_t P, hyenand_dtype dtype,
                                                          size_t* bytes_out) {
  if (!bytes_out) return fail(HYENAND_ERR_INVALID_ARGUMENT, "bytes_out is NULL");
  const hyenand_status st = check_norm_shape(B, C, P, dtype);
  if (st == HYENAND_OK) *bytes_out = norm_backward_workspace_bytes(B, C, P, dtype == HYENAND_DTYPE_BF16);
  return st;
}

hyenand_status hyenand_block_norm_backward(const void* x_out, const void* z, const void* gate, const void* w_post,
                                           const void* scale, const void* w_pre, float eps_post, float eps_pre,
                                           float dropout_p, const uint64_t* rng, const void* gx_out, const void* gn,
                                           void* gx, void* gz, void* ggate, void* gw_post, void* gscale, void* gw_pre,
                                           int64_t B, int64_t C, int64_t P, hyenand_dtype dtype, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  hyenand_status st = check_norm_shape(B, C, P, dtype);
  if (st != HYENAND_OK) return st;
  NormArgs a;
  memset(&a, 0, sizeof a);
  st = check_norm(z, gate, w_post, scale, eps_post, eps_pre, dropout_p, rng, &a);
  if (st != HYENAND_OK) return st;
  if (!gx_out && !gn) return fail(HYENAND_ERR_INVALID_ARGUMENT, "neither gx_out nor gn is given");
  const struct {
    const void* of;
    const char* name;
    const void* grad;
    const char* grad_name;
  } pairs[] = {{z, "z", gz, "gz"}, {gate, "gate", ggate, "ggate"}, {w_post, "w_post", gw_post, "gw_post"},
               {scale, "scale", gscale, "gscale"}, {gn, "gn", w_pre, "w_pre"}, {gn, "gn", gw_pre, "gw_pre"}};
  for (const auto& q : pairs)
    if (!q.of != !q.grad)
      return fail(HYENAND_ERR_INVALID_ARGUMENT, "%s and %s must both be given or both be NULL", q.name, q.grad_name);
  const size_t es = dtype == HYENAND_DTYPE_BF16 ? 2 : 4, bytes = (size_t)(B * C) * (size_t)P * es, row = (size_t)C * es;
  const size_t need = norm_backward_workspace_bytes(B, C, P, dtype == HYENAND_DTYPE_BF16);
  const Buffer bufs[] = {{"x_out", x_out, bytes, es, false, false}, {"z", z, bytes, es, false, true},
                         {"gate", gate, bytes, es, false, true},    {"w_post", w_post, row, es, false, true},
                         {"scale", scale, row, es, false, true},    {"w_pre", w_pre, row, es, false, true},
                         {"rng", rng, 16, 8, false, true},          {"gx_out", gx_out, bytes, es, false, true},
                         {"gn", gn, bytes, es, false, true},        {"gx", gx, bytes, es, true, false},
                         {"gz", gz, bytes, es, true, true},         {"ggate", ggate, bytes, es, true, true},
                         {"gw_post", gw_post, row, es, true, true}, {"gscale", gscale, row, es, true, true},
                         {"gw_pre", gw_pre, row, es, true, true},   {"workspace", workspace, need, 1, true, true}};
  st = check_workspace(workspace, workspace_bytes, need);
  if (st == HYENAND_OK) st = check_buffers(bufs);
  if (st != HYENAND_OK) return st;
  a.x = x_out;
  a.z = z;
  a.g = gate;
  a.w_post = w_post;
  a.scale = scale;
  a.w_pre = w_pre;
  a.rng = rng;
  a.gx_out = gx_out;
  a.gn = gn;
  a.gx = gx;
  a.gz = gz;
  a.gg = ggate;
  a.gw_post = gw_post;
  a.gscale = gscale;
  a.gw_pre = gw_pre;
  a.partial = reinterpret_cast<float2*>(workspace);
  a.B = B;
  a.C = (int)C;
  a.P = P;
  a.bf16 = dtype == HYENAND_DTYPE_BF16;
  clear_pending_error();
  return launched(launch_norm_backward(a, (hipStream_t)stream));
}

}  // extern "C"
