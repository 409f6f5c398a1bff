// Gradients of the gated linear recurrence (scan.hip).  With z = h + D u,
// gz = gy x2 and c_t = a_t gh_t, what position t hands to the state before it:
//
//   gx2 = gy z,  gh_t = gz_t + c_{t+1},  glog_a_t = c_t h_{t-1},
//   gu = gh + D gz,  gx1 = gu v,  gv = gu x1,  gD = sum of gz u,  gh0 = c_0
//
// c runs through the same decays as h, from the row's end.  The forward keeps the
// state before every tile of 512 positions, so a tile's states are computed from
// its own inputs while it is taken, and five tensors are read and four written
// once: the HBM bound.
#include "scan_device.hpp"

namespace hyenand {

using namespace rows;
using namespace scan_dev;

namespace {

template <typename TS>
struct BwdTile {
  Raw<TS> x1, v, la, x2, gy;
};

template <typename TS>
__device__ __forceinline__ void load_bwd(BwdTile<TS>& t, const ScanArgs& a, int64_t off, int n) {
  t.la = load(reinterpret_cast<const TS*>(a.la) + off, n);
  t.x1 = load(reinterpret_cast<const TS*>(a.x1) + off, n);
  t.v = load(reinterpret_cast<const TS*>(a.v) + off, n);
  t.x2 = load(reinterpret_cast<const TS*>(a.x2) + off, n);
  t.gy = load(reinterpret_cast<const TS*>(a.gy) + off, n);
}

__device__ __forceinline__ int64_t row_length(const ScanArgs& a, int64_t row) {
  if (!a.len) return a.L;
  const int64_t n = a.len[(uint32_t)row / (uint32_t)a.C];
  return n < 0 ? 0 : (n > a.L ? a.L : n);
}

template <int G>
__device__ __forceinline__ Span mirror(Span x) {
  if constexpr (G == 1) return x;
  return {__shfl_xor(x.s, G - 1), __shfl_xor(x.u, G - 1)};
}

// c of a lane's eight positions when nothing comes from behind
__device__ __forceinline__ float lane_back(const float (&s)[kScanV], const float (&e)[kScanV], const float (&gz)[kScanV]) {
  float c = 0.f;
#pragma unroll
  for (int j = kScanV - 1; j >= 0; --j) c = s[j] == neg_inf() ? 0.f : e[j] * (gz[j] + c);
  return c;
}

__device__ __forceinline__ double sum_lanes(double x, int lanes) {
  for (int d = lanes / 2; d > 0; d /= 2) x += __shfl_xor(x, d);
  return x;
}

// G lanes a row (G < 64: a row is one tile), W wavefronts a row.
template <typename TS, int G, int W>
__global__ void __launch_bounds__(W == 16 ? 1024 : 256) scan_gradients(ScanArgs a) {
  __shared__ Span joint[2][W > 1 ? W : 1];
  __shared__ double sums[W];
  const Place<G, W> at(a.R);
  const int64_t len = row_length(a, at.row), base = at.row * a.L;
  const float D = ld1(reinterpret_cast<const TS*>(a.D) + (uint32_t)at.row % (uint32_t)a.C);
  const int64_t seg = blockIdx.y, first = seg * a.seg_tiles;
  const int64_t ntiles = G < 64 ? 1 : (a.L + kScanTile - 1) / kScanTile;
  const int64_t end = first + a.seg_tiles < ntiles ? first + a.seg_tiles : ntiles;
  float c = a.seg_in ? a.seg_in[at.row * a.nseg + seg] : (a.gh_last ? a.gh_last[at.row] : 0.f);
  const int64_t in_tile = (int64_t)(at.lane & (G - 1)) * kScanV;
  const int64_t wave = W > 1 ? at.wave : 0;
  auto pos = [&](int64_t tile) { return (tile + wave) * kScanTile + in_tile; };
  auto count = [&](int64_t tile) { return tile + wave < end ? clamp_count<kScanV>(len - pos(tile)) : 0; };
  auto state = [&](int64_t tile) { return tile + wave < end ? a.states[at.row * a.nst + tile + wave] : 0.f; };
  double gD = 0.0;
  int64_t tile = first + (end - first - 1) / W * W;
  BwdTile<TS> cur, nxt;
  load_bwd(cur, a, base + pos(tile), count(tile));
  float h_cur = state(tile), h_nxt = 0.f;
  int buf = 0;
  for (; tile >= first; tile -= W) {
    const int64_t p = pos(tile), off = base + p;
    const int n = count(tile);
    const int w = at.live && tile + wave < end ? clamp_count<kScanV>(a.L - p) : 0;
    if (tile > first) {
      load_bwd(nxt, a, base + pos(tile - W), count(tile - W));
      h_nxt = state(tile - W);
    }
    float s[kScanV], e[kScanV], u[kScanV], gz[kScanV], before[kScanV], out[kScanV];
    Span sp = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kScanV; ++j) {
      decay(get(cur.la, j), j < n, &s[j], &e[j]);
      u[j] = j < n ? get(cur.x1, j) * get(cur.v, j) : 0.f;
      gz[j] = j < n ? get(cur.gy, j) * get(cur.x2, j) : 0.f;
      sp.u = advance(s[j], e[j], sp.u, u[j]);
      sp.s += s[j];
    }
    // the states, from the one before the tile on
    float x = through(below<G>(prefix<G>(sp, at.lane), at.lane), h_cur);
    float dsum = 0.f;
#pragma unroll
    for (int j = 0; j < kScanV; ++j) {
      before[j] = x;
      x = advance(s[j], e[j], x, u[j]);
      out[j] = j < n ? get(cur.gy, j) * fmaf(D, u[j], x) : 0.f;
      dsum = fmaf(gz[j], u[j], dsum);
    }
    gD += dsum;
    store(reinterpret_cast<TS*>(a.gx2) + off, out, w);
    // c, from behind: the lanes in reverse order
    const Span back = prefix<G>(mirror<G>({sp.s, lane_back(s, e, gz)}), at.lane);
    Span all = {0.f, 0.f};
    float c_tile = c;
    if constexpr (W > 1) {
      c_tile = through(across_waves<W>({read_lane(back.s, 63), read_lane(back.u, 63)}, joint[buf], W - 1 - at.wave, at.lane, &all), c);
      buf ^= 1;
    }
    float g = through(mirror<G>(below<G>(back, at.lane)), c_tile);
    float gx1[kScanV], gv[kScanV];
#pragma unroll
    for (int j = kScanV - 1; j >= 0; --j) {
      const bool start = s[j] == neg_inf();
      g += gz[j];
      const float gu = fmaf(D, gz[j], g);
      gx1[j] = j < n ? gu * get(cur.v, j) : 0.f;
      gv[j] = j < n ? gu * get(cur.x1, j) : 0.f;
      g = start ? 0.f : e[j] * g;
      out[j] = j < n && !start ? g * before[j] : 0.f;
    }
    store(reinterpret_cast<TS*>(a.gx1) + off, gx1, w);
    store(reinterpret_cast<TS*>(a.gv) + off, gv, w);
    store(reinterpret_cast<TS*>(a.gla) + off, out, w);
    if constexpr (G < 64) {
      if (a.gh0 && at.live && (at.lane & (G - 1)) == 0) a.gh0[at.row] = g;
    } else if constexpr (W == 1) {
      c = read_lane(g, 0);
    } else {
      c = through(all, c);
    }
    cur = nxt;
    h_cur = h_nxt;
  }
  if constexpr (G == 64) {
    if (a.gh0 && at.live && first == 0 && wave == 0 && at.lane == 0) a.gh0[at.row] = c;
  }
  gD = sum_lanes(gD, G);
  if constexpr (W > 1) {
    if (at.lane == 0) sums[at.wave] = gD;
    __syncthreads();
    gD = 0.0;
#pragma unroll
    for (int i = 0; i < W; ++i) gD += sums[i];
    if (threadIdx.x == 0) a.partial[at.row * a.nseg + seg] = gD;
  } else {
    if (at.live && (at.lane & (G - 1)) == 0) a.partial[at.row * a.nseg + seg] = gD;
  }
}

// What each segment of a row does to a c that passes through it, from its end.
template <typename TS, int W>
__global__ void __launch_bounds__(W == 16 ? 1024 : 256) scan_segment_back(ScanArgs a) {
  __shared__ Span joint[2][W];
  const Place<64, W> at(a.R);
  const int64_t len = row_length(a, at.row), base = at.row * a.L;
  const int64_t seg = blockIdx.y, first = seg * a.seg_tiles;
  const int64_t ntiles = (a.L + kScanTile - 1) / kScanTile;
  const int64_t end = first + a.seg_tiles < ntiles ? first + a.seg_tiles : ntiles;
  const int64_t in_tile = (int64_t)at.lane * kScanV;
  auto pos = [&](int64_t tile) { return (tile + at.wave) * kScanTile + in_tile; };
  auto count = [&](int64_t tile) { return tile + at.wave < end ? clamp_count<kScanV>(len - pos(tile)) : 0; };
  auto fetch = [&](BwdTile<TS>& t, int64_t tile) {
    const int64_t off = base + pos(tile);
    const int n = count(tile);
    t.la = load(reinterpret_cast<const TS*>(a.la) + off, n);
    t.x2 = load(reinterpret_cast<const TS*>(a.x2) + off, n);
    t.gy = load(reinterpret_cast<const TS*>(a.gy) + off, n);
  };
  Span sum = {0.f, 0.f};
  int64_t tile = first + (end - first - 1) / W * W;
  BwdTile<TS> cur, nxt;
  fetch(cur, tile);
  int buf = 0;
  for (; tile >= first; tile -= W) {
    const int n = count(tile);
    if (tile > first) fetch(nxt, tile - W);
    float s[kScanV], e[kScanV], gz[kScanV], total = 0.f;
#pragma unroll
    for (int j = 0; j < kScanV; ++j) {
      decay(get(cur.la, j), j < n, &s[j], &e[j]);
      gz[j] = j < n ? get(cur.gy, j) * get(cur.x2, j) : 0.f;
      total += s[j];
    }
    const Span back = prefix<64>(mirror<64>({total, lane_back(s, e, gz)}), at.lane);
    Span all;
    across_waves<W>({read_lane(back.s, 63), read_lane(back.u, 63)}, joint[buf], W - 1 - at.wave, at.lane, &all);
    buf ^= 1;
    sum = then(sum, all);
    cur = nxt;
  }
  if (threadIdx.x == 0) a.seg[at.row * a.nseg + seg] = make_float2(sum.s, sum.u);
}

// The c that enters each segment from behind, a wavefront a row.
__global__ void __launch_bounds__(256) scan_join_back(ScanArgs a) {
  const Place<64, 1> at(a.R);
  const int64_t i = a.nseg - 1 - at.lane;
  const float2 m = i >= 0 ? a.seg[at.row * a.nseg + i] : make_float2(0.f, 0.f);
  const Span in = below<64>(prefix<64>({m.x, m.y}, at.lane), at.lane);
  if (at.live && i >= 0) a.seg_in[at.row * a.nseg + i] = through(in, a.gh_last ? a.gh_last[at.row] : 0.f);
}

// gD[c]: the rows' sums in a fixed order, a workgroup a channel.
template <typename TS>
__global__ void __launch_bounds__(256) scan_sum_D(ScanArgs a) {
  __shared__ double part[4];
  const int64_t c = blockIdx.x, per = a.R / a.C * a.nseg;
  double x = 0.0;
  for (int64_t i = threadIdx.x; i < per; i += 256) x += a.partial[(i / a.nseg * a.C + c) * a.nseg + i % a.nseg];
  x = sum_lanes(x, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  if (threadIdx.x == 0) st1(reinterpret_cast<TS*>(a.gD) + c, (float)(part[0] + part[1] + part[2] + part[3]));
}

template <typename TS, int W>
hipError_t gradient_rows(const ScanArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(W > 1 ? a.R : (a.R + 3) / 4), (unsigned)a.nseg), block(W > 4 ? 64 * W : 256);
  if constexpr (W == 16) {
    if (a.nseg > 1) {
      hipLaunchKernelGGL((scan_segment_back<TS, W>), grid, block, 0, s, a);
      hipLaunchKernelGGL(scan_join_back, dim3((unsigned)((a.R + 3) / 4)), dim3(256), 0, s, a);
    }
  }
  hipLaunchKernelGGL((scan_gradients<TS, 64, W>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <typename TS, int G>
hipError_t gradient_short(const ScanArgs& a, hipStream_t s) {
  const int64_t rows = 4 * (64 / G);
  hipLaunchKernelGGL((scan_gradients<TS, G, 1>), dim3((unsigned)((a.R + rows - 1) / rows)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename TS>
hipError_t gradients(const ScanArgs& a, const ScanShape& p, hipStream_t s) {
  hipError_t err;
  switch (p.lanes) {
    case 1: err = gradient_short<TS, 1>(a, s); break;
    case 2: err = gradient_short<TS, 2>(a, s); break;
    case 4: err = gradient_short<TS, 4>(a, s); break;
    case 8: err = gradient_short<TS, 8>(a, s); break;
    case 16: err = gradient_short<TS, 16>(a, s); break;
    case 32: err = gradient_short<TS, 32>(a, s); break;
    default: err = p.waves == 1 ? gradient_rows<TS, 1>(a, s) : (p.waves == 4 ? gradient_rows<TS, 4>(a, s) : gradient_rows<TS, 16>(a, s));
  }
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL((scan_sum_D<TS>), dim3((unsigned)a.C), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_scan_backward(const ScanArgs& args, void* ws, hipStream_t s) {
  ScanArgs a = args;
  const ScanShape p = scan_shape(a.R, a.L, true);
  a.nseg = p.nseg;
  a.seg_tiles = p.seg_tiles;
  a.seg = nullptr;
  a.seg_in = nullptr;
  a.partial = reinterpret_cast<double*>(ws);
  if (p.nseg > 1) {
    a.seg = reinterpret_cast<float2*>(a.partial + a.R * p.nseg);
    a.seg_in = reinterpret_cast<float*>(a.seg + a.R * p.nseg);
  }
  return a.bf16 ? gradients<uint16_t>(a, p, s) : gradients<float>(a, p, s);
}

}  // namespace hyenand
