// Gradients of the norms around a block (block_norm.hip).  With q = 1 / rms(x),
// r = 1 / rms(t), means over the C channels of a point, x the forward's x_out:
//
//   gx = gx_out + q (gn w_pre - x q^2 mean(gn w_pre x))
//   gm = scale drop(gx),  gt = r (gm w_post - t r^2 mean(gm w_post t))
//   gz = gt sigmoid(g),   gg = gt t (1 - sigmoid(g))
//   gw_pre = sum gn x q,  gw_post = scale S, gscale = w_post S,
//   S = sum drop(gx) t r  (over samples and points)
//
// Bound by HBM: five tensors read and three written.  The dropped points are drawn
// again from the counter.  A workgroup takes tile after tile and adds its weight
// sums up in registers; a second kernel adds those of the workgroups, in order.
#include "norm_device.hpp"

namespace hyenand {

using namespace rows;
using namespace norm_dev;

namespace {

// The raw inputs of V points of a channel.
template <typename TS, int V>
struct BwdRow {
  Raw<TS, V> x, gn, gxo, z, g;
};

template <typename TS, int V>
__device__ __forceinline__ void load_row(BwdRow<TS, V>& r, const NormArgs& a, int64_t o, int n) {
  r.x = load<TS, V>(reinterpret_cast<const TS*>(a.x) + o, n);
  if (a.gn) r.gn = load<TS, V>(reinterpret_cast<const TS*>(a.gn) + o, n);
  if (a.z) {
    r.z = load<TS, V>(reinterpret_cast<const TS*>(a.z) + o, n);
    if (a.g) r.g = load<TS, V>(reinterpret_cast<const TS*>(a.g) + o, n);
  }
  if (a.gx_out) r.gxo = load<TS, V>(reinterpret_cast<const TS*>(a.gx_out) + o, n);
}

// t = sigmoid(g) z of a point
template <typename TS, int V>
__device__ __forceinline__ float branch(const BwdRow<TS, V>& r, const NormArgs& a, int j, float* sig, float* rest) {
  *sig = 1.f;
  *rest = 0.f;
  if (a.g) gates(get(r.g, j), sig, rest);
  return *sig * get(r.z, j);
}

// The sums of the first kind: squares of x, gn w_pre x, squares of t.
template <typename TS, int V>
__device__ __forceinline__ void first_sums(const BwdRow<TS, V>& r, const NormArgs& a, float w_pre, float (&acc)[3][V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if (a.gn) {
      const float x = get(r.x, j);
      acc[0][j] = fmaf(x, x, acc[0][j]);
      acc[1][j] = fmaf(get(r.gn, j) * w_pre, x, acc[1][j]);
    }
    if (a.z) {
      float sig, rest;
      const float t = branch(r, a, j, &sig, &rest);
      acc[2][j] = fmaf(t, t, acc[2][j]);
    }
  }
}

// gx of V points; what reaches the branch's norm, and its sum with t (the second kind)
template <typename TS, int V>
__device__ __forceinline__ void second_sums(const BwdRow<TS, V>& r, const NormArgs& a, int64_t row, int64_t p, int c,
                                            uint64_t seed, uint64_t offset, const float (&acc)[3][V], float (&gx)[V],
                                            float (&gmw)[V], float (&sum)[1][V], float2* weights) {
  const float w_pre = a.gn ? weight<TS>(a.w_pre, c) : 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    gx[j] = a.gx_out ? get(r.gxo, j) : 0.f;
    if (a.gn) {
      const float q = acc[0][j], gn = get(r.gn, j), xq = get(r.x, j) * q;
      gx[j] += q * fmaf(-xq, acc[1][j], gn * w_pre);
      weights->x = fmaf(gn, xq, weights->x);
    }
  }
  if (!a.z) return;
  const float w = weight<TS>(a.w_post, c) * weight<TS>(a.scale, c);
  float f[V];
#pragma unroll
  for (int j = 0; j < V; ++j) f[j] = 1.f;
  if (a.drop) keep_factors<V>(a, seed, offset, row, p, f);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    float sig, rest;
    const float t = branch(r, a, j, &sig, &rest), kept = f[j] * gx[j];
    gmw[j] = kept * w;
    sum[0][j] = fmaf(gmw[j], t, sum[0][j]);
    weights->y = fmaf(kept, t * acc[2][j], weights->y);
  }
}

// gz and gg of V points
template <typename TS, int V>
__device__ __forceinline__ void last_row(const BwdRow<TS, V>& r, const NormArgs& a, int64_t o, int n, const float (&rinv)[V],
                                         const float (&mean)[V], const float (&gmw)[V]) {
  float gz[V], gg[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    float sig, rest;
    const float t = branch(r, a, j, &sig, &rest);
    const float gt = rinv[j] * fmaf(-t * rinv[j], mean[j], gmw[j]);
    gz[j] = gt * sig;
    gg[j] = gt * t * rest;
  }
  store<TS, V>(reinterpret_cast<TS*>(a.gz) + o, gz, n);
  if (a.gg) store<TS, V>(reinterpret_cast<TS*>(a.gg) + o, gg, n);
}

// q, q mean(gn w_pre x) and r from the first sums
__device__ __forceinline__ void finish_first(const NormArgs& a, float (&s)[3]) {
  s[0] = a.gn ? inverse_rms(s[0], a.C, a.eps_pre) : 0.f;
  s[1] = s[1] / (float)a.C * s[0];
  s[2] = inverse_rms(s[2], a.C, a.eps_post);
}

template <typename TS, int V, int K>
__global__ void __launch_bounds__(kMaxNT) norm_backward(NormArgs a) {
  __shared__ Joint<3> lds;
  __shared__ Joint<1> lds1;
  const uint64_t seed = a.drop ? a.rng[0] : 0, offset = a.drop ? a.rng[1] : 0;
  float2 weights[K];
#pragma unroll
  for (int k = 0; k < K; ++k) weights[k] = make_float2(0.f, 0.f);
  for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const Spot<V> at(a, tile);
    const int64_t base = (at.b * a.C + at.cl) * a.P + at.p, step = (int64_t)at.CL * a.P;
    auto count = [&](int k) { return at.cl + k * at.CL < a.C ? at.n : 0; };
    BwdRow<TS, V> r[K];
#pragma unroll
    for (int k = 0; k < K; ++k) load_row(r[k], a, base + k * step, count(k));
    float acc[3][V], sum[1][V], gmw[K][V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[0][j] = acc[1][j] = acc[2][j] = sum[0][j] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (count(k)) first_sums(r[k], a, a.gn ? weight<TS>(a.w_pre, at.cl + k * at.CL) : 0.f, acc);
    over_channels(acc, lds, a.lp, at.pg, [&](float (&s)[3]) { finish_first(a, s); });
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = at.cl + k * at.CL;
      if (!count(k)) continue;
      float gx[V];
      second_sums(r[k], a, at.b * a.C + c, at.p, c, seed, offset, acc, gx, gmw[k], sum, &weights[k]);
      store<TS, V>(reinterpret_cast<TS*>(a.gx) + base + k * step, gx, count(k));
    }
    if (!a.z) continue;
    over_channels(sum, lds1, a.lp, at.pg, [&](float (&s)[1]) { s[0] /= (float)a.C; });
#pragma unroll
    for (int j = 0; j < V; ++j) sum[0][j] *= acc[2][j];
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (count(k)) last_row(r[k], a, base + k * step, count(k), acc[2], sum[0], gmw[k]);
  }
  const int cl = threadIdx.x >> a.lp, CL = blockDim.x >> a.lp;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    for (int d = 1; d < (1 << a.lp); d *= 2) {
      weights[k].x += __shfl_xor(weights[k].x, d);
      weights[k].y += __shfl_xor(weights[k].y, d);
    }
    const int c = cl + k * CL;
    if ((threadIdx.x & ((1 << a.lp) - 1)) == 0 && c < a.C) a.partial[(int64_t)blockIdx.x * a.C + c] = weights[k];
  }
}

// More channels than registers hold: the tile is read again for each sum, and
// the weight sums are added up in the workspace, each by its own thread.
template <typename TS, int V>
__global__ void __launch_bounds__(kMaxNT) norm_backward_reread(NormArgs a) {
  __shared__ Joint<3> lds;
  __shared__ Joint<1> lds1;
  const uint64_t seed = a.drop ? a.rng[0] : 0, offset = a.drop ? a.rng[1] : 0;
  float2* partial = a.partial + (int64_t)blockIdx.x * a.C;  // lp = 0: a channel is one thread's
  for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const Spot<V> at(a, tile);
    auto where = [&](int c) { return (at.b * a.C + c) * a.P + at.p; };
    BwdRow<TS, V> r;
    float acc[3][V], sum[1][V], gx[V], gmw[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[0][j] = acc[1][j] = acc[2][j] = sum[0][j] = 0.f;
    for (int c = at.cl; c < a.C; c += at.CL) {
      load_row(r, a, where(c), at.n);
      first_sums(r, a, a.gn ? weight<TS>(a.w_pre, c) : 0.f, acc);
    }
    over_channels(acc, lds, a.lp, at.pg, [&](float (&s)[3]) { finish_first(a, s); });
    for (int c = at.cl; c < a.C; c += at.CL) {
      load_row(r, a, where(c), at.n);
      float2 w = tile == blockIdx.x ? make_float2(0.f, 0.f) : partial[c];
      second_sums(r, a, at.b * a.C + c, at.p, c, seed, offset, acc, gx, gmw, sum, &w);
      partial[c] = w;
      if (!a.z) store<TS, V>(reinterpret_cast<TS*>(a.gx) + where(c), gx, at.n);
    }
    if (!a.z) continue;
    over_channels(sum, lds1, a.lp, at.pg, [&](float (&s)[1]) { s[0] /= (float)a.C; });
#pragma unroll
    for (int j = 0; j < V; ++j) sum[0][j] *= acc[2][j];
    for (int c = at.cl; c < a.C; c += at.CL) {
      load_row(r, a, where(c), at.n);
      float unused[1][V];
      float2 none = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < V; ++j) unused[0][j] = 0.f;
      second_sums(r, a, at.b * a.C + c, at.p, c, seed, offset, acc, gx, gmw, unused, &none);
      store<TS, V>(reinterpret_cast<TS*>(a.gx) + where(c), gx, at.n);
      last_row(r, a, where(c), at.n, acc[2], sum[0], gmw);
    }
  }
}

// The weights' gradients: the workgroups' sums, 32 channels a workgroup, every
// 32nd of them a thread.
template <typename TS>
__global__ void __launch_bounds__(1024) norm_weights(NormArgs a) {
  __shared__ double sx[32][33], sy[32][33];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  double x = 0.0, y = 0.0;
  if (c < a.C)
    for (int i = part; i < a.groups; i += 32) {
      const float2 w = a.partial[(int64_t)i * a.C + c];
      x += w.x;
      y += w.y;
    }
  sx[part][lane] = x;
  sy[part][lane] = y;
  __syncthreads();
  if (part == 0 && c < a.C) {
    for (int i = 1; i < 32; ++i) {
      x += sx[i][lane];
      y += sy[i][lane];
    }
    if (a.gw_pre) st1(reinterpret_cast<TS*>(a.gw_pre) + c, (float)x);
    if (a.gw_post) st1(reinterpret_cast<TS*>(a.gw_post) + c, (float)(y * weight<TS>(a.scale, c)));
    if (a.gscale) st1(reinterpret_cast<TS*>(a.gscale) + c, (float)(y * weight<TS>(a.w_post, c)));
  }
}

int groups_of(int64_t tiles) { return (int)(tiles < 1024 ? tiles : 1024); }

template <typename TS>
hipError_t backward(const NormArgs& a, const NormShape& s, hipStream_t st) {
  const dim3 grid((unsigned)a.groups), block((unsigned)s.NT);
#define HY_CASE(v, k) \
  if (s.V == v && s.K == k) hipLaunchKernelGGL((norm_backward<TS, v, k>), grid, block, 0, st, a);
  HY_CASE(1, 1) HY_CASE(1, 4) HY_CASE(1, 16) HY_CASE(8, 1) HY_CASE(8, 2)
  if constexpr (sizeof(TS) == 2) {
    HY_CASE(8, 4)
  }
#undef HY_CASE
  if (s.K == 0) {
    if (s.V == 1) hipLaunchKernelGGL((norm_backward_reread<TS, 1>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((norm_backward_reread<TS, 8>), grid, block, 0, st, a);
  }
  hipLaunchKernelGGL((norm_weights<TS>), dim3((unsigned)((a.C + 31) / 32)), dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t norm_backward_workspace_bytes(int64_t B, int64_t C, int64_t P, bool bf16) {
  NormArgs a;
  a.B = B;
  a.C = (int)C;
  a.P = P;
  norm_tiles(a, norm_shape(C, P, bf16, true));
  return (size_t)groups_of(a.tiles) * (size_t)C * sizeof(float2);
}

hipError_t launch_norm_backward(const NormArgs& args, hipStream_t st) {
  NormArgs a = args;
  const NormShape s = norm_shape(a.C, a.P, a.bf16, true);
  norm_tiles(a, s);
  a.groups = groups_of(a.tiles);
  return a.bf16 ? backward<uint16_t>(a, s, st) : backward<float>(a, s, st);
}

}  // namespace hyenand
