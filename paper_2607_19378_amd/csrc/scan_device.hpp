// Device parts of the gated linear recurrence h_t = a_t h_{t-1} + u_t, shared by
// its forward and backward.
//
// A span of positions maps the state that enters it to the one that leaves it,
// h -> a h + U, and two spans compose to another: (a2 a1, a2 U1 + U2).  a is kept
// as s = log2 a: sums of s stay exact to an fp32 rounding of the sum where the
// product of thousands of factors near one would add up their roundings (memories
// of 4096 positions: 4e-6 against 1.3e-7 relative to 64 bits).  s = -inf marks a
// span with a start of a sequence in it: nothing that enters it leaves it, not
// even an infinity or a NaN, so the product is skipped there instead of formed.
#pragma once

#include "kernels.hpp"
#include "row_access.hpp"
#include "scan.hpp"

namespace hyenand {
namespace scan_dev {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kStart = -87.f;  // log_a below this (a < 2^-125) starts a sequence

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
__device__ __forceinline__ float pow2f(float s) { return __builtin_amdgcn_exp2f(s); }

// a x + u, and u alone where s = log2 a marks a start
__device__ __forceinline__ float advance(float s, float a, float x, float u) {
  const float r = fmaf(a, x, u);
  return s == neg_inf() ? u : r;
}

struct Span {
  float s, u;
};

// first, then second
__device__ __forceinline__ Span then(Span first, Span second) {
  return {first.s + second.s, advance(second.s, pow2f(second.s), first.u, second.u)};
}

__device__ __forceinline__ float through(Span sp, float x) { return advance(sp.s, pow2f(sp.s), x, sp.u); }

// DPP move; lanes without a source (or in a row that row_mask leaves out) get 0
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ Span dpp(Span x) {
  return {dpp<CTRL, ROWS>(x.s), dpp<CTRL, ROWS>(x.u)};
}

constexpr int kRowShr = 0x110;   // + n: from n lanes below, within 16 lanes
constexpr int kWaveShr1 = 0x138;
constexpr int kBcast15 = 0x142;  // lane 15 of a row of 16 to the next row
constexpr int kBcast31 = 0x143;  // lane 31 to the upper half

// Inclusive prefix over groups of G lanes (a power of two), lower lanes first.
// Lanes that have no lane to combine with combine with (0, 0), which changes nothing.
template <int G>
__device__ __forceinline__ Span prefix(Span x, int lane) {
  auto step = [&](auto shr, int d) {
    Span p = shr(x);
    if (G < 16 && (lane & (G - 1)) < d) p = {0.f, 0.f};
    x = then(p, x);
  };
  if constexpr (G > 1) step([](Span t) { return dpp<kRowShr + 1>(t); }, 1);
  if constexpr (G > 2) step([](Span t) { return dpp<kRowShr + 2>(t); }, 2);
  if constexpr (G > 4) step([](Span t) { return dpp<kRowShr + 4>(t); }, 4);
  if constexpr (G > 8) step([](Span t) { return dpp<kRowShr + 8>(t); }, 8);
  if constexpr (G > 16) x = then(dpp<kBcast15, 0xa>(x), x);
  if constexpr (G > 32) x = then(dpp<kBcast31, 0xc>(x), x);
  return x;
}

// The inclusive prefix of the lane below, (0, 0) in a group's first lane.
template <int G>
__device__ __forceinline__ Span below(Span x, int lane) {
  Span p = dpp<kWaveShr1>(x);
  if ((lane & (G - 1)) == 0) p = {0.f, 0.f};
  return p;
}

__device__ __forceinline__ float read_lane(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}

// Spans of the W tiles that the wavefronts of a workgroup hold: the one of all
// before wavefront w, and the one of all W.  `at`: W spans in LDS, of which no
// wavefront writes the next ones before every other has read these (two
// buffers, one barrier an iteration).
template <int W>
__device__ __forceinline__ Span across_waves(Span mine, Span* at, int wave, int lane, Span* all) {
  static_assert(W >= 2 && W <= 16, "one row of 16 lanes holds the spans");
  if (lane == 0) at[wave] = mine;
  __syncthreads();
  Span x = at[lane & (W - 1)];
  x = prefix<W>(x, lane);
  *all = {read_lane(x.s, W - 1), read_lane(x.u, W - 1)};
  if (wave == 0) return {0.f, 0.f};
  return {read_lane(x.s, wave - 1), read_lane(x.u, wave - 1)};
}

// log2 a and a of element j; behind the sample's end (j >= n) the state stays as it is
__device__ __forceinline__ void decay(float la, bool live, float* s, float* e) {
  float t = la < kStart ? neg_inf() : la * kLog2e;
  t = live ? t : 0.f;
  *s = t;
  *e = pow2f(t);
}

// Where a lane works: its row and the tile of a wavefront.
template <int G, int W>
struct Place {
  int lane, wave;
  int64_t row;
  bool live;  // false: a lane beyond the last row, which computes on the last one and writes nothing
  __device__ __forceinline__ explicit Place(int64_t R) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if constexpr (W > 1) {
      row = blockIdx.x;
    } else if constexpr (G == 64) {
      row = (int64_t)blockIdx.x * 4 + wave;
    } else {
      row = ((int64_t)blockIdx.x * 4 + wave) * (64 / G) + lane / G;
    }
    live = row < R;
    if (!live) row = R - 1;
  }
};

}  // namespace scan_dev
}  // namespace hyenand
