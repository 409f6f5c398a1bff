// Gated linear recurrence along the last axis, forward and one step:
//
//   u = x1 v,  h_t = exp(log_a_t) h_{t-1} + u_t,  y = x2 (h + D u)
//
// Bound by HBM: four tensors read and one written, about 8 flops a position.  A
// wavefront takes a tile of 512 positions, eight consecutive ones a lane (16 bytes
// of bf16, 32 of fp32); the lanes' spans are joined by a prefix over the lanes (DPP
// moves, no LDS), then each lane walks its eight positions from the state that
// enters them.
#include "scan_device.hpp"

namespace hyenand {

using namespace rows;
using namespace scan_dev;

namespace {

template <typename TS>
struct FwdTile {
  Raw<TS> x1, v, la, x2;
};

template <typename TS, bool WITH_X2>
__device__ __forceinline__ void load_fwd(FwdTile<TS>& t, const ScanArgs& a, int64_t off, int n) {
  t.x1 = load(reinterpret_cast<const TS*>(a.x1) + off, n);
  t.v = load(reinterpret_cast<const TS*>(a.v) + off, n);
  t.la = load(reinterpret_cast<const TS*>(a.la) + off, n);
  if constexpr (WITH_X2) t.x2 = load(reinterpret_cast<const TS*>(a.x2) + off, n);
}

__device__ __forceinline__ int64_t row_length(const ScanArgs& a, int64_t row) {
  if (!a.len) return a.L;
  const int64_t n = a.len[(uint32_t)row / (uint32_t)a.C];
  return n < 0 ? 0 : (n > a.L ? a.L : n);
}

// The span of a lane's eight positions.
template <typename TS>
__device__ __forceinline__ Span lane_span(const FwdTile<TS>& t, int n, float (&s)[kScanV], float (&e)[kScanV],
                                          float (&u)[kScanV]) {
  Span sp = {0.f, 0.f};
#pragma unroll
  for (int j = 0; j < kScanV; ++j) {
    decay(get(t.la, j), j < n, &s[j], &e[j]);
    u[j] = j < n ? get(t.x1, j) * get(t.v, j) : 0.f;
    sp.u = advance(s[j], e[j], sp.u, u[j]);
    sp.s += s[j];
  }
  return sp;
}

// G lanes a row (G < 64: a row is one tile), W wavefronts a row.
template <typename TS, int G, int W>
__global__ void __launch_bounds__(W == 16 ? 1024 : 256) scan_forward(ScanArgs a) {
  __shared__ Span joint[2][W > 1 ? W : 1];
  const Place<G, W> at(a.R);
  const int64_t len = row_length(a, at.row), base = at.row * a.L;
  const float D = ld1(reinterpret_cast<const TS*>(a.D) + (uint32_t)at.row % (uint32_t)a.C);
  const int64_t seg = blockIdx.y, first = seg * a.seg_tiles;
  const int64_t ntiles = G < 64 ? 1 : (a.L + kScanTile - 1) / kScanTile;
  const int64_t end = first + a.seg_tiles < ntiles ? first + a.seg_tiles : ntiles;
  float h = a.seg_in ? a.seg_in[at.row * a.nseg + seg] : (a.h0 ? a.h0[at.row] : 0.f);
  const int64_t in_tile = (int64_t)(at.lane & (G - 1)) * kScanV;
  const int64_t wave = W > 1 ? at.wave : 0;
  auto pos = [&](int64_t tile) { return (tile + wave) * kScanTile + in_tile; };
  auto count = [&](int64_t tile) { return tile + wave < end ? clamp_count<kScanV>(len - pos(tile)) : 0; };
  FwdTile<TS> cur, nxt;
  load_fwd<TS, true>(cur, a, base + pos(first), count(first));
  int buf = 0;
  for (int64_t tile = first; tile < end; tile += W) {
    const int64_t p = pos(tile);
    const int n = count(tile);
    if (tile + W < end) load_fwd<TS, true>(nxt, a, base + pos(tile + W), count(tile + W));
    float s[kScanV], e[kScanV], u[kScanV], y[kScanV];
    const Span lanes = prefix<G>(lane_span(cur, n, s, e, u), at.lane);
    Span in = below<G>(lanes, at.lane), all;
    float h_tile = h;  // the state that enters this wavefront's tile
    if constexpr (W > 1) {
      h_tile = through(across_waves<W>({read_lane(lanes.s, 63), read_lane(lanes.u, 63)}, joint[buf], at.wave, at.lane, &all), h);
      buf ^= 1;
    }
    float x = through(in, h_tile);
    if (a.states && at.live && (at.lane & (G - 1)) == 0 && tile + wave < end) a.states[at.row * a.nst + tile + wave] = h_tile;
#pragma unroll
    for (int j = 0; j < kScanV; ++j) {
      x = advance(s[j], e[j], x, u[j]);
      y[j] = j < n ? get(cur.x2, j) * fmaf(D, u[j], x) : 0.f;
    }
    if (at.live && tile + wave < end) store(reinterpret_cast<TS*>(a.y) + base + p, y, clamp_count<kScanV>(a.L - p));
    if constexpr (G < 64) {
      if (a.h_last && at.live && (at.lane & (G - 1)) == G - 1) a.h_last[at.row] = x;
    } else if constexpr (W == 1) {
      h = read_lane(x, 63);
    } else {
      h = through(all, h);
    }
    cur = nxt;
  }
  if constexpr (G == 64) {
    if (a.h_last && at.live && end == ntiles && wave == 0 && at.lane == 0) a.h_last[at.row] = h;
  }
}

// What each segment of a row does to a state that passes through it.
template <typename TS, int W>
__global__ void __launch_bounds__(W == 16 ? 1024 : 256) scan_segment(ScanArgs a) {
  __shared__ Span joint[2][W];
  const Place<64, W> at(a.R);
  const int64_t len = row_length(a, at.row), base = at.row * a.L;
  const int64_t seg = blockIdx.y, first = seg * a.seg_tiles;
  const int64_t ntiles = (a.L + kScanTile - 1) / kScanTile;
  const int64_t end = first + a.seg_tiles < ntiles ? first + a.seg_tiles : ntiles;
  const int64_t in_tile = (int64_t)at.lane * kScanV;
  auto pos = [&](int64_t tile) { return (tile + at.wave) * kScanTile + in_tile; };
  auto count = [&](int64_t tile) { return tile + at.wave < end ? clamp_count<kScanV>(len - pos(tile)) : 0; };
  Span sum = {0.f, 0.f};
  FwdTile<TS> cur, nxt;
  load_fwd<TS, false>(cur, a, base + pos(first), count(first));
  int buf = 0;
  for (int64_t tile = first; tile < end; tile += W) {
    const int n = count(tile);
    if (tile + W < end) load_fwd<TS, false>(nxt, a, base + pos(tile + W), count(tile + W));
    float s[kScanV], e[kScanV], u[kScanV];
    const Span lanes = prefix<64>(lane_span(cur, n, s, e, u), at.lane);
    Span all;
    across_waves<W>({read_lane(lanes.s, 63), read_lane(lanes.u, 63)}, joint[buf], at.wave, at.lane, &all);
    buf ^= 1;
    sum = then(sum, all);
    cur = nxt;
  }
  if (threadIdx.x == 0) a.seg[at.row * a.nseg + seg] = make_float2(sum.s, sum.u);
}

// The state that enters each segment, a wavefront a row.
__global__ void __launch_bounds__(256) scan_join(ScanArgs a) {
  const Place<64, 1> at(a.R);
  const float2 m = at.lane < a.nseg ? a.seg[at.row * a.nseg + at.lane] : make_float2(0.f, 0.f);
  const Span in = below<64>(prefix<64>({m.x, m.y}, at.lane), at.lane);
  if (at.live && at.lane < a.nseg) a.seg_in[at.row * a.nseg + at.lane] = through(in, a.h0 ? a.h0[at.row] : 0.f);
}

template <typename TS, int W>
hipError_t forward_rows(const ScanArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(W > 1 ? a.R : (a.R + 3) / 4), (unsigned)a.nseg), block(W > 4 ? 64 * W : 256);
  if constexpr (W == 16) {
    if (a.nseg > 1) {
      hipLaunchKernelGGL((scan_segment<TS, W>), grid, block, 0, s, a);
      hipLaunchKernelGGL(scan_join, dim3((unsigned)((a.R + 3) / 4)), dim3(256), 0, s, a);
    }
  }
  hipLaunchKernelGGL((scan_forward<TS, 64, W>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <typename TS, int G>
hipError_t forward_short(const ScanArgs& a, hipStream_t s) {
  const int64_t rows = 4 * (64 / G);
  hipLaunchKernelGGL((scan_forward<TS, G, 1>), dim3((unsigned)((a.R + rows - 1) / rows)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename TS>
hipError_t forward(const ScanArgs& a, const ScanShape& p, hipStream_t s) {
  switch (p.lanes) {
    case 1: return forward_short<TS, 1>(a, s);
    case 2: return forward_short<TS, 2>(a, s);
    case 4: return forward_short<TS, 4>(a, s);
    case 8: return forward_short<TS, 8>(a, s);
    case 16: return forward_short<TS, 16>(a, s);
    case 32: return forward_short<TS, 32>(a, s);
    default: break;
  }
  if (p.waves == 1) return forward_rows<TS, 1>(a, s);
  return p.waves == 4 ? forward_rows<TS, 4>(a, s) : forward_rows<TS, 16>(a, s);
}

constexpr int kStepNT = 256;

// One position of every sequence, a thread a channel.  Rows with the same slot
// are positions of one sequence, in the order of the batch: the workgroup of the
// first of them takes all, those of the others end.
template <typename TS>
__global__ void __launch_bounds__(kStepNT) scan_step(ScanStepArgs a) {
  __shared__ int earlier, next;
  int64_t b = blockIdx.y;
  const int c = blockIdx.x * kStepNT + threadIdx.x;
  const int64_t slot = a.slots ? a.slots[b] : b;
  const bool in_pool = slot >= 0 && slot < a.nslots;
  int later = (int)a.B;
  if (a.slots) {
    if (threadIdx.x == 0) {
      earlier = 0;
      next = (int)a.B;
    }
    __syncthreads();
    if (in_pool)
      for (int i = threadIdx.x; i < a.B; i += kStepNT)
        if (a.slots[i] == slot && i != b) {
          if (i < b) earlier = 1;
          else atomicMin(&next, i);
        }
    __syncthreads();
    if (earlier) return;
    later = next;
  }
  float h = in_pool && c < a.C ? a.state[slot * a.C + c] : 0.f;
  for (;;) {
    if (c < a.C) {
      const int64_t i = b * a.C + c;
      float y = 0.f;
      if (in_pool) {
        float s, e;
        decay(ld1(reinterpret_cast<const TS*>(a.la) + i), true, &s, &e);
        const float u = ld1(reinterpret_cast<const TS*>(a.x1) + i) * ld1(reinterpret_cast<const TS*>(a.v) + i);
        h = advance(s, e, h, u);
        y = ld1(reinterpret_cast<const TS*>(a.x2) + i) * fmaf(ld1(reinterpret_cast<const TS*>(a.D) + c), u, h);
      }
      st1(reinterpret_cast<TS*>(a.y) + i, y);
    }
    if (later >= a.B) break;
    // the row after this one with the same slot, if there is one more
    b = later;
    __syncthreads();
    if (threadIdx.x == 0) next = (int)a.B;
    __syncthreads();
    for (int i = (int)b + 1 + threadIdx.x; i < a.B; i += kStepNT)
      if (a.slots[i] == slot) atomicMin(&next, i);
    __syncthreads();
    later = next;
  }
  if (in_pool && c < a.C) a.state[slot * a.C + c] = h;
}

}  // namespace

ScanShape scan_shape(int64_t R, int64_t L, bool backward) {
  ScanShape p = {64, 1, 1, 0};
  const int64_t tiles = (L + kScanTile - 1) / kScanTile;
  p.seg_tiles = tiles;
  if (L <= 32 * kScanV) {
    p.lanes = 1;
    while (p.lanes * kScanV < L) p.lanes *= 2;
    return p;
  }
  if (R < 2048 && tiles > 1) p.waves = R < 512 && tiles > 4 ? 16 : 4;
  if (p.waves == 16 && R < 128) {
    int64_t n = (256 + R - 1) / R;  // a workgroup a CU at least
    if (n > kScanMaxSeg) n = kScanMaxSeg;
    if (n > tiles / 16) n = tiles / 16;
    if (n > 1) {
      p.seg_tiles = ((tiles + n - 1) / n + 15) / 16 * 16;
      p.nseg = (int)((tiles + p.seg_tiles - 1) / p.seg_tiles);
    }
  }
  (void)backward;
  return p;
}

size_t scan_segment_bytes(const ScanShape& p, int64_t R) {
  return p.nseg > 1 ? (size_t)R * p.nseg * (sizeof(float2) + sizeof(float)) : 0;
}

size_t scan_workspace_bytes(int64_t R, int64_t L, bool backward) {
  const ScanShape p = scan_shape(R, L, backward);
  return scan_segment_bytes(p, R) + (backward ? (size_t)R * p.nseg * sizeof(double) : 0);
}

hipError_t launch_scan(const ScanArgs& args, void* ws, hipStream_t s) {
  ScanArgs a = args;
  const ScanShape p = scan_shape(a.R, a.L, false);
  a.nseg = p.nseg;
  a.seg_tiles = p.seg_tiles;
  a.seg = nullptr;
  a.seg_in = nullptr;
  if (p.nseg > 1) {
    a.seg = reinterpret_cast<float2*>(ws);
    a.seg_in = reinterpret_cast<float*>(a.seg + a.R * p.nseg);
  }
  return a.bf16 ? forward<uint16_t>(a, p, s) : forward<float>(a, p, s);
}

hipError_t launch_scan_step(const ScanStepArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.C + kStepNT - 1) / kStepNT), (unsigned)a.B);
  if (a.bf16)
    hipLaunchKernelGGL((scan_step<uint16_t>), grid, dim3(kStepNT), 0, s, a);
  else
    hipLaunchKernelGGL((scan_step<float>), grid, dim3(kStepNT), 0, s, a);
  return hipGetLastError();
}

}  // namespace hyenand
