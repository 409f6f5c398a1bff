// The norms before and behind a residual block, with its gate, dropout and
// residual scale, forward:
//
//   t = sigmoid(g) z,  m = t / rms(t) w_post,  x_out = x + scale drop(m),
//   n = x_out / rms(x_out) w_pre            (rms over the channels of a point)
//
// Bound by HBM: three tensors read and two written.
#include "norm_device.hpp"

namespace hyenand {

using namespace rows;
using namespace norm_dev;

namespace {

// The tile in registers: K channels a thread.
template <typename TS, int V, int K>
__global__ void __launch_bounds__(kMaxNT) norm_forward(NormArgs a) {
  __shared__ Joint<1> lds;
  for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const Spot<V> at(a, tile);
    Raw<TS, V> x[K], z[K], g[K];
    const int64_t base = (at.b * a.C + at.cl) * a.P + at.p, step = (int64_t)at.CL * a.P;
    auto count = [&](int k) { return at.cl + k * at.CL < a.C ? at.n : 0; };
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (a.z) z[k] = load<TS, V>(reinterpret_cast<const TS*>(a.z) + base + k * step, count(k));
      if (a.g) g[k] = load<TS, V>(reinterpret_cast<const TS*>(a.g) + base + k * step, count(k));
      x[k] = load<TS, V>(reinterpret_cast<const TS*>(a.x) + base + k * step, count(k));
    }
    float y[K][V];  // the branch, then the sum
    float acc[1][V];
    if (a.z) {
#pragma unroll
      for (int j = 0; j < V; ++j) acc[0][j] = 0.f;
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float sig = 1.f, rest;
          if (a.g) gates(get(g[k], j), &sig, &rest);
          y[k][j] = sig * get(z[k], j);
          acc[0][j] = fmaf(y[k][j], y[k][j], acc[0][j]);
        }
      over_channels(acc, lds, a.lp, at.pg, [&](float (&s)[1]) { s[0] = inverse_rms(s[0], a.C, a.eps_post); });
      const uint64_t seed = a.drop ? a.rng[0] : 0, offset = a.drop ? a.rng[1] : 0;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = at.cl + k * at.CL;
        const float w = c < a.C ? weight<TS>(a.w_post, c) * weight<TS>(a.scale, c) : 0.f;
        float f[V];
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = 1.f;
        if (a.drop) keep_factors<V>(a, seed, offset, at.b * a.C + c, at.p, f);
#pragma unroll
        for (int j = 0; j < V; ++j) y[k][j] = fmaf(f[j] * w, y[k][j] * acc[0][j], get(x[k], j));
        store<TS, V>(reinterpret_cast<TS*>(a.x_out) + base + k * step, y[k], count(k));
      }
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) y[k][j] = get(x[k], j);
    }
    if (!a.n) continue;
#pragma unroll
    for (int j = 0; j < V; ++j) acc[0][j] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) acc[0][j] = fmaf(y[k][j], y[k][j], acc[0][j]);
    over_channels(acc, lds, a.lp, at.pg, [&](float (&s)[1]) { s[0] = inverse_rms(s[0], a.C, a.eps_pre); });
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = at.cl + k * at.CL;
      const float w = c < a.C ? weight<TS>(a.w_pre, c) : 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) y[k][j] *= acc[0][j] * w;
      store<TS, V>(reinterpret_cast<TS*>(a.n) + base + k * step, y[k], count(k));
    }
  }
}

// More channels than registers hold: the tile is read again for each sum.
template <typename TS, int V>
__global__ void __launch_bounds__(kMaxNT) norm_forward_reread(NormArgs a) {
  __shared__ Joint<1> lds;
  for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const Spot<V> at(a, tile);
    const uint64_t seed = a.drop ? a.rng[0] : 0, offset = a.drop ? a.rng[1] : 0;
    float post[1][V], pre[1][V];
    auto branch = [&](int c, float (&t)[V]) {
      const int64_t o = (at.b * a.C + c) * a.P + at.p;
      const Raw<TS, V> z = load<TS, V>(reinterpret_cast<const TS*>(a.z) + o, at.n);
      Raw<TS, V> g;
      if (a.g) g = load<TS, V>(reinterpret_cast<const TS*>(a.g) + o, at.n);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float sig = 1.f, rest;
        if (a.g) gates(get(g, j), &sig, &rest);
        t[j] = sig * get(z, j);
      }
    };
    auto sum = [&](int c, float (&y)[V]) {
      const Raw<TS, V> x = load<TS, V>(reinterpret_cast<const TS*>(a.x) + (at.b * a.C + c) * a.P + at.p, at.n);
      if (!a.z) {
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = get(x, j);
        return;
      }
      branch(c, y);
      const float w = weight<TS>(a.w_post, c) * weight<TS>(a.scale, c);
      float f[V];
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = 1.f;
      if (a.drop) keep_factors<V>(a, seed, offset, at.b * a.C + c, at.p, f);
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] = fmaf(f[j] * w, y[j] * post[0][j], get(x, j));
    };
#pragma unroll
    for (int j = 0; j < V; ++j) post[0][j] = pre[0][j] = 0.f;
    if (a.z) {
      for (int c = at.cl; c < a.C; c += at.CL) {
        float t[V];
        branch(c, t);
#pragma unroll
        for (int j = 0; j < V; ++j) post[0][j] = fmaf(t[j], t[j], post[0][j]);
      }
      over_channels(post, lds, a.lp, at.pg, [&](float (&s)[1]) { s[0] = inverse_rms(s[0], a.C, a.eps_post); });
    }
    for (int c = at.cl; c < a.C; c += at.CL) {
      float y[V];
      sum(c, y);
      if (a.z) store<TS, V>(reinterpret_cast<TS*>(a.x_out) + (at.b * a.C + c) * a.P + at.p, y, at.n);
#pragma unroll
      for (int j = 0; j < V; ++j) pre[0][j] = fmaf(y[j], y[j], pre[0][j]);
    }
    if (!a.n) continue;
    over_channels(pre, lds, a.lp, at.pg, [&](float (&s)[1]) { s[0] = inverse_rms(s[0], a.C, a.eps_pre); });
    for (int c = at.cl; c < a.C; c += at.CL) {
      float y[V];
      sum(c, y);
      const float w = weight<TS>(a.w_pre, c);
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] *= pre[0][j] * w;
      store<TS, V>(reinterpret_cast<TS*>(a.n) + (at.b * a.C + c) * a.P + at.p, y, at.n);
    }
  }
}

constexpr int64_t kMaxGrid = int64_t(1) << 20;  // workgroups of a launch (fewer than 2^32 work-items)

template <typename TS>
hipError_t forward(const NormArgs& a, const NormShape& s, hipStream_t st) {
  const dim3 grid((unsigned)(a.tiles < kMaxGrid ? a.tiles : kMaxGrid)), block((unsigned)s.NT);
#define HY_CASE(v, k) \
  if (s.V == v && s.K == k) hipLaunchKernelGGL((norm_forward<TS, v, k>), grid, block, 0, st, a);
  HY_CASE(1, 1) HY_CASE(1, 4) HY_CASE(1, 16) HY_CASE(8, 1) HY_CASE(8, 2) HY_CASE(8, 4)
#undef HY_CASE
  if (s.K == 0) {
    if (s.V == 1) hipLaunchKernelGGL((norm_forward_reread<TS, 1>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((norm_forward_reread<TS, 8>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace

NormShape norm_shape(int64_t C, int64_t P, bool bf16, bool backward) {
  NormShape s;
  s.V = P == 1 ? 1 : 8;
  s.lp = 0;
  const int64_t groups = (P + s.V - 1) / s.V;
  // a cache line of a row (128 bytes) where the row is as long
  const int most = s.V == 1 ? 0 : (bf16 ? 3 : 2);
  while (s.lp < most && (int64_t(1) << s.lp) < groups) ++s.lp;
  const int ks_many[] = {1, 4, 16}, ks_fwd[] = {1, 2, 4}, ks_bwd[] = {1, 2, bf16 ? 4 : 2};
  const int(&ks)[3] = s.V == 1 ? ks_many : (backward ? ks_bwd : ks_fwd);
  // channels a thread: the fewest of which 1024 threads hold all; fewer points
  // a tile where the most are not enough
  for (;; --s.lp) {
    for (int k : ks) {
      const int64_t nt = ((C + k - 1) / k << s.lp) + 63;
      if (nt / 64 * 64 <= kMaxNT) {
        s.K = k;
        s.NT = (int)(nt / 64 * 64);
        return s;
      }
    }
    if (s.lp == 0) break;
  }
  s.K = 0;
  s.NT = kMaxNT;
  return s;
}

void norm_tiles(NormArgs& a, const NormShape& s) {
  a.lp = s.lp;
  const int64_t points = (int64_t)s.V << s.lp;
  a.row_tiles = (a.P + points - 1) / points;
  a.tiles = a.row_tiles * a.B;
}

hipError_t launch_norm(const NormArgs& args, hipStream_t st) {
  NormArgs a = args;
  const NormShape s = norm_shape(a.C, a.P, a.bf16, false);
  norm_tiles(a, s);
  return a.bf16 ? forward<uint16_t>(a, s, st) : forward<float>(a, s, st);
}

}  // namespace hyenand
