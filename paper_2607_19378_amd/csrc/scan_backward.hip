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

template <int G>
__device__ __forceinline__ Span mirror(Span x) {
  if constexpr (G == 1) return x;
  return {__shfl_xor(x.s, G - 1), __shfl_xor(x.u, G - 1)};
}

template <typename TS>
__device__ __forceinline__ float input(const BwdTile<TS>& t, int j) {
  return get(t.x1, j) * get(t.v, j);
}
template <typename TS>
__device__ __forceinline__ float grad_z(const BwdTile<TS>& t, int j) {
  return get(t.gy, j) * get(t.x2, j);
}

__device__ __forceinline__ double sum_lanes(double x, int lanes) {
  for (int d = lanes / 2; d > 0; d /= 2) x += __shfl_xor(x, d);
  return x;
}

// G lanes a row (G < 64: a row is one tile), W wavefronts a row, or (LINKED) a
// segment of one.
template <typename TS, int G, int W, bool LINKED>
__global__ void __launch_bounds__(W > 4 ? 64 * W : 256, LINKED ? 4 : 1) scan_gradients(ScanArgs a) {
  __shared__ Span joint[2][W > 1 ? W : 1];
  __shared__ double sums[W];
  const uint32_t group = LINKED ? link_row(a) : blockIdx.x, turn = LINKED ? link_draw(a, group) : 0;
  if (LINKED && turn >= (uint32_t)a.nseg) return;
  const uint32_t seg = LINKED ? a.nseg - 1 - turn : 0;
  const Place<G, W> at(a.R, group);
  const int64_t len = row_length(a, at.row), base = at.row * a.L;
  const float D = ld1(reinterpret_cast<const TS*>(a.D) + (uint32_t)at.row % (uint32_t)a.C);
  const int64_t ntiles = G < 64 ? 1 : (a.L + kScanTile - 1) / kScanTile, first = (int64_t)seg * W;
  const int64_t end = LINKED && first + W < ntiles ? first + W : ntiles;
  float c = a.gh_last ? a.gh_last[at.row] : 0.f;
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
    if (!LINKED && tile > first) {
      load_bwd(nxt, a, base + pos(tile - W), count(tile - W));
      h_nxt = state(tile - W);
    }
    float e[kScanV], before[kScanV], out[kScanV];
    Span sp = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kScanV; ++j) {
      const float s = decay(get(cur.la, j));
      e[j] = pow2f(s);
      sp.u = advance(e[j], sp.u, input(cur, j));
      sp.s = join(sp.s, s);
    }
    keep_packed(cur.x1);
    keep_packed(cur.v);
    // the states, from the one before the tile on
    float x = through(below<G>(prefix<G>(sp, at.lane), at.lane), h_cur);
    float dsum = 0.f;
#pragma unroll
    for (int j = 0; j < kScanV; ++j) {
      const float u = input(cur, j);
      before[j] = x;
      x = advance(e[j], x, u);
      out[j] = get(cur.gy, j) * fmaf(D, u, x);
      dsum = fmaf(grad_z(cur, j), u, dsum);
    }
    gD += dsum;
    only(out, n);
    store(reinterpret_cast<TS*>(a.gx2) + off, out, w);
    keep_packed(cur.x1);
    keep_packed(cur.v);
    keep_packed(cur.gy);
    keep_packed(cur.x2);
    // c, from behind: the lanes in reverse order
    float back_u = 0.f;
#pragma unroll
    for (int j = kScanV - 1; j >= 0; --j) back_u = advance(e[j], grad_z(cur, j) + back_u, 0.f);
    keep_packed(cur.gy);
    keep_packed(cur.x2);
    const Span back = prefix<G>(mirror<G>({sp.s, back_u}), at.lane);
    Span all = {0.f, 0.f};
    float c_tile = c;
    if constexpr (W > 1) {
      const Span behind = across_waves<W>({read_lane(back.s, 63), read_lane(back.u, 63)}, joint[buf], W - 1 - at.wave, at.lane, &all);
      if constexpr (LINKED) {
        __shared__ float entered;
        if (at.wave == 0) {
          const float from = link_enter(a.links + 2 * at.row * a.nseg, turn, all, c, at.lane);
          if (at.lane == 0) entered = from;
        }
        __syncthreads();
        c = entered;
      }
      c_tile = through(behind, c);
      buf ^= 1;
    }
    float g = through(mirror<G>(below<G>(back, at.lane)), c_tile);
    float gx1[kScanV], gv[kScanV];
#pragma unroll
    for (int j = kScanV - 1; j >= 0; --j) {
      const float gz = grad_z(cur, j);
      g += gz;
      const float gu = fmaf(D, gz, g);
      gx1[j] = gu * get(cur.v, j);
      gv[j] = gu * get(cur.x1, j);
      g = advance(e[j], g, 0.f);
      out[j] = e[j] == 0.f ? 0.f : g * before[j];
    }
    only(gx1, n);
    only(gv, n);
    only(out, n);
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
    if (!LINKED) {
      cur = nxt;
      h_cur = h_nxt;
    }
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
    if (threadIdx.x != 0) return;
  } else {
    if (!at.live || (at.lane & (G - 1)) != 0) return;
  }
  if (!LINKED && a.R == a.C)
    st1(reinterpret_cast<TS*>(a.gD) + at.row, (float)gD);  // one sample: the whole sum
  else
    a.partial[at.row * a.nseg + seg] = gD;
}

// gD[c]: the rows' sums in a fixed order, a workgroup a channel.
template <typename TS>
__global__ void __launch_bounds__(256) scan_sum_D(ScanArgs a) {
  __shared__ double part[4];
  const uint32_t nseg = a.nseg, per = (uint32_t)a.R / a.C * nseg;
  for (int c = blockIdx.x; c < a.C; c += gridDim.x) {
    double x = 0.0;
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < per; i += 256) x += a.partial[((int64_t)(i / nseg) * a.C + c) * nseg + i % nseg];
    x = sum_lanes(x, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    if (threadIdx.x == 0) st1(reinterpret_cast<TS*>(a.gD) + c, (float)(part[0] + part[1] + part[2] + part[3]));
    __syncthreads();  // read before the next channel's
  }
}

template <typename TS, int W>
hipError_t gradient_rows(const ScanArgs& a, hipStream_t s) {
  const dim3 block(W > 4 ? 64 * W : 256);
  if (W == kLinkedWaves && a.nseg > 1) {
    const hipError_t e = launch_scan_links(a, s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((scan_gradients<TS, 64, kLinkedWaves, true>), dim3((unsigned)(a.R * a.nseg)), block, 0, s, a);
  } else {
    hipLaunchKernelGGL((scan_gradients<TS, 64, W, false>), dim3((unsigned)(W > 1 ? a.R : (a.R + 3) / 4)), block, 0, s, a);
  }
  return hipGetLastError();
}

template <typename TS, int G>
hipError_t gradient_short(const ScanArgs& a, hipStream_t s) {
  const int64_t rows = 4 * (64 / G);
  hipLaunchKernelGGL((scan_gradients<TS, G, 1, false>), dim3((unsigned)((a.R + rows - 1) / rows)), dim3(256), 0, s, a);
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
    default: err = p.waves == 1 ? gradient_rows<TS, 1>(a, s) : (p.waves == 4 ? gradient_rows<TS, 4>(a, s) : gradient_rows<TS, 8>(a, s));
  }
  if (err != hipSuccess || (a.R == a.C && a.nseg == 1)) return err;
  const int most = 1 << 20;  // workgroups (fewer than 2^32 work-items)
  hipLaunchKernelGGL((scan_sum_D<TS>), dim3((unsigned)(a.C < most ? a.C : most)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_scan_backward(const ScanArgs& args, void* ws, hipStream_t s) {
  ScanArgs a = args;
  const ScanShape p = scan_shape(a.R, a.L);
  a.nseg = p.nseg;
  a.links = reinterpret_cast<uint64_t*>(ws);
  a.partial = reinterpret_cast<double*>(reinterpret_cast<char*>(ws) + scan_link_bytes(p, a.R));
  return a.bf16 ? gradients<uint16_t>(a, p, s) : gradients<float>(a, p, s);
}

}  // namespace hyenand
