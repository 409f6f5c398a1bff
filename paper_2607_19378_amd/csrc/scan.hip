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

template <typename TS>
__device__ __forceinline__ void load_fwd(FwdTile<TS>& t, const ScanArgs& a, int64_t off, int n) {
  t.x1 = load(reinterpret_cast<const TS*>(a.x1) + off, n);
  t.v = load(reinterpret_cast<const TS*>(a.v) + off, n);
  t.la = load(reinterpret_cast<const TS*>(a.la) + off, n);
  t.x2 = load(reinterpret_cast<const TS*>(a.x2) + off, n);
}

template <typename TS>
__device__ __forceinline__ float input(const FwdTile<TS>& t, int j) {
  return get(t.x1, j) * get(t.v, j);
}

// The span of a lane's eight positions, and their decays.
template <typename TS>
__device__ __forceinline__ Span lane_span(const FwdTile<TS>& t, float (&e)[kScanV]) {
  Span sp = {0.f, 0.f};
#pragma unroll
  for (int j = 0; j < kScanV; ++j) {
    const float s = decay(get(t.la, j));
    e[j] = pow2f(s);
    sp.u = advance(e[j], sp.u, input(t, j));
    sp.s = join(sp.s, s);
  }
  return sp;
}

// G lanes a row (G < 64: a row is one tile), W wavefronts a row, or (LINKED) a
// segment of one.
template <typename TS, int G, int W, bool LINKED>
__global__ void __launch_bounds__(W > 4 ? 64 * W : 256) scan_forward(ScanArgs a) {
  __shared__ Span joint[2][W > 1 ? W : 1];
  const uint32_t group = LINKED ? link_row(a) : blockIdx.x, seg = LINKED ? link_draw(a, group) : 0;
  if (LINKED && seg >= (uint32_t)a.nseg) return;
  const Place<G, W> at(a.R, group);
  const int64_t len = row_length(a, at.row), base = at.row * a.L;
  const float D = ld1(reinterpret_cast<const TS*>(a.D) + (uint32_t)at.row % (uint32_t)a.C);
  const int64_t ntiles = G < 64 ? 1 : (a.L + kScanTile - 1) / kScanTile, first = (int64_t)seg * W;
  const int64_t end = LINKED && first + W < ntiles ? first + W : ntiles;
  float h = a.h0 ? a.h0[at.row] : 0.f;
  const int64_t in_tile = (int64_t)(at.lane & (G - 1)) * kScanV;
  const int64_t wave = W > 1 ? at.wave : 0;
  auto pos = [&](int64_t tile) { return (tile + wave) * kScanTile + in_tile; };
  auto count = [&](int64_t tile) { return tile + wave < end ? clamp_count<kScanV>(len - pos(tile)) : 0; };
  FwdTile<TS> cur, nxt;
  load_fwd(cur, a, base + pos(first), count(first));
  int buf = 0;
  for (int64_t tile = first; tile < end; tile += W) {
    const int64_t p = pos(tile);
    const int n = count(tile);
    if (!LINKED && tile + W < end) load_fwd(nxt, a, base + pos(tile + W), count(tile + W));
    float e[kScanV], y[kScanV];
    const Span lanes = prefix<G>(lane_span(cur, e), at.lane);
    keep_packed(cur.x1);
    keep_packed(cur.v);
    Span in = below<G>(lanes, at.lane), all;
    float h_tile = h;  // the state that enters this wavefront's tile
    if constexpr (W > 1) {
      const Span before = across_waves<W>({read_lane(lanes.s, 63), read_lane(lanes.u, 63)}, joint[buf], at.wave, at.lane, &all);
      if constexpr (LINKED) {
        __shared__ float entered;
        if (at.wave == 0) {
          const float x = link_enter(a.links + 2 * at.row * a.nseg, seg, all, h, at.lane);
          if (at.lane == 0) entered = x;
        }
        __syncthreads();
        h = entered;
      }
      h_tile = through(before, h);
      buf ^= 1;
    }
    float x = through(in, h_tile);
    if (a.states && at.live && (at.lane & (G - 1)) == 0 && tile + wave < end) a.states[at.row * a.nst + tile + wave] = h_tile;
#pragma unroll
    for (int j = 0; j < kScanV; ++j) {
      const float u = input(cur, j);
      x = advance(e[j], x, u);
      y[j] = get(cur.x2, j) * fmaf(D, u, x);
    }
    only(y, n);
    if (at.live && tile + wave < end) store(reinterpret_cast<TS*>(a.y) + base + p, y, clamp_count<kScanV>(a.L - p));
    if constexpr (G < 64) {
      if (a.h_last && at.live && (at.lane & (G - 1)) == G - 1) a.h_last[at.row] = x;
    } else if constexpr (W == 1) {
      h = read_lane(x, 63);
    } else {
      h = through(all, h);
    }
    if (!LINKED) cur = nxt;
  }
  if constexpr (G == 64) {
    if (a.h_last && at.live && end == ntiles && wave == 0 && at.lane == 0) a.h_last[at.row] = h;
  }
}

__global__ void __launch_bounds__(256) scan_clear_links(uint64_t* links, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) links[i] = 0;
}

template <typename TS, int W>
hipError_t forward_rows(const ScanArgs& a, hipStream_t s) {
  const dim3 block(W > 4 ? 64 * W : 256);
  if (W == kLinkedWaves && a.nseg > 1) {
    const hipError_t e = launch_scan_links(a, s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((scan_forward<TS, 64, kLinkedWaves, true>), dim3((unsigned)(a.R * a.nseg)), block, 0, s, a);
  } else {
    hipLaunchKernelGGL((scan_forward<TS, 64, W, false>), dim3((unsigned)(W > 1 ? a.R : (a.R + 3) / 4)), block, 0, s, a);
  }
  return hipGetLastError();
}

template <typename TS, int G>
hipError_t forward_short(const ScanArgs& a, hipStream_t s) {
  const int64_t rows = 4 * (64 / G);
  hipLaunchKernelGGL((scan_forward<TS, G, 1, false>), dim3((unsigned)((a.R + rows - 1) / rows)), dim3(256), 0, s, a);
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
  return p.waves == 4 ? forward_rows<TS, 4>(a, s) : forward_rows<TS, 8>(a, s);
}

constexpr int kStepNT = 256;
constexpr int kStepLook = 8 * kStepNT;  // rows looked at before the workgroup compares

// One position of every sequence, a thread a channel.  Rows with the same slot
// are positions of one sequence, in the order of the batch: the workgroup of the
// first of them takes all, those of the others end.  A search of the batch ends
// with the first kStepLook rows that hold the slot: searches through all of it cost
// the square of the rows with one state (16384 of them: 1220 ms, now 12).
template <typename TS>
__global__ void __launch_bounds__(kStepNT) scan_step(ScanStepArgs a) {
  __shared__ int first[2][kStepNT / 64];
  int b = blockIdx.y, turn = 0;
  const int c = blockIdx.x * kStepNT + threadIdx.x, B = (int)a.B;
  const int64_t slot = a.slots ? a.slots[b] : b;
  const bool in_pool = slot >= 0 && slot < a.nslots;
  // the first of the rows from ... to, but for row b, with this slot (B: none)
  auto look = [&](int from, int to) {
    int mine = B;
    for (int i = from + (int)threadIdx.x; i < to; i += kStepNT)
      if (a.slots[i] == slot && i != b) mine = min(mine, i);
    if (__ballot(mine < B))
      for (int d = 32; d > 0; d /= 2) mine = min(mine, __shfl_xor(mine, d));
    if ((threadIdx.x & 63) == 0) first[turn][threadIdx.x >> 6] = mine;
    __syncthreads();  // (and the results of the look before the last one have been read)
    int found = B;
#pragma unroll
    for (int w = 0; w < kStepNT / 64; ++w) found = min(found, first[turn][w]);
    turn ^= 1;
    return found;
  };
  auto search = [&](int from) {
    int found = B;
    for (; from < B && found == B; from += kStepLook) found = look(from, min(from + kStepLook, B));
    return found;
  };
  int later = B;
  if (a.slots && in_pool) {
    later = search(0);
    if (later < b) return;
  }
  float h = in_pool && c < a.C ? a.state[slot * a.C + c] : 0.f;
  for (;;) {
    if (c < a.C) {
      const int64_t i = (int64_t)b * a.C + c;
      float y = 0.f;
      if (in_pool) {
        const float e = pow2f(decay(ld1(reinterpret_cast<const TS*>(a.la) + i)));
        const float u = ld1(reinterpret_cast<const TS*>(a.x1) + i) * ld1(reinterpret_cast<const TS*>(a.v) + i);
        h = advance(e, h, u);
        y = ld1(reinterpret_cast<const TS*>(a.x2) + i) * fmaf(ld1(reinterpret_cast<const TS*>(a.D) + c), u, h);
      }
      st1(reinterpret_cast<TS*>(a.y) + i, y);
    }
    if (later >= B) break;
    b = later;
    later = look(b + 1, min(b + 1 + kStepNT, B));  // (neighbours, most often)
    if (later == B) later = search(b + 1 + kStepNT);
  }
  if (in_pool && c < a.C) a.state[slot * a.C + c] = h;
}

}  // namespace

// Eight wavefronts a row as long as the rows alone do not fill the chip (256 rows of
// 65536 backward, bf16: 56 us against 71 with four and 222 with one), four from 1024 rows
// on (1024 of 16384 backward, bf16: 57 against 58 and 70 us), one from 4096 (4096 of 4096:
// 58 against 61 us with four).  Rows so few that most CUs would have none are split into
// linked segments, from the length on where these pay for their two more steps (128
// rows backward, fp32: 130 against 163 us for 2^17 positions, 39 against 45 us for 2^15, 32
// against 28 us for 2^14; 200 rows: equal).
ScanShape scan_shape(int64_t R, int64_t L) {
  ScanShape p = {64, 1, 1};
  const int64_t tiles = (L + kScanTile - 1) / kScanTile;
  if (L <= 32 * kScanV) {
    p.lanes = 1;
    while (p.lanes * kScanV < L) p.lanes *= 2;
    return p;
  }
  if (tiles > 1 && R < 4096) p.waves = R < 1024 && tiles > 4 ? 8 : 4;
  // A launch has fewer than 2^32 work-items: segments of 2^35 positions in all, more than five tensors in a
  // card's memory.  (One row of 2^33, bf16, forward: 135 ms, against 3640 for one workgroup.)
  const int64_t nseg = (tiles + kLinkedWaves - 1) / kLinkedWaves;
  if (R < 192 && tiles > 32 && nseg <= ((int64_t(1) << 32) - 1) / (64 * kLinkedWaves) / R) {
    p.waves = kLinkedWaves;
    p.nseg = (int)nseg;
  }
  return p;
}

size_t scan_link_bytes(const ScanShape& p, int64_t R) { return p.nseg > 1 ? ((size_t)R * (p.nseg * 2 + kLinkStride)) * sizeof(uint64_t) : 0; }

size_t scan_workspace_bytes(int64_t R, int64_t L, bool backward) {
  const ScanShape p = scan_shape(R, L);
  return scan_link_bytes(p, R) + (backward ? (size_t)R * p.nseg * sizeof(double) : 0);
}

hipError_t launch_scan_links(const ScanArgs& a, hipStream_t s) {
  const int64_t n = a.R * (2 * a.nseg + kLinkStride);
  hipLaunchKernelGGL(scan_clear_links, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a.links, n);
  return hipGetLastError();
}

hipError_t launch_scan(const ScanArgs& args, void* ws, hipStream_t s) {
  ScanArgs a = args;
  const ScanShape p = scan_shape(a.R, a.L);
  a.nseg = p.nseg;
  a.links = reinterpret_cast<uint64_t*>(ws);
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
