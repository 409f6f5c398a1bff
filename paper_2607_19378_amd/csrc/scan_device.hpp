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

// a x + u, and u alone where a = 0, which only a start has: a decay that is none
// is 2^-126 at least
__device__ __forceinline__ float advance(float a, float x, float u) {
  const float r = fmaf(a, x, u);
  return a == 0.f ? u : r;
}

struct Span {
  float s, u;
};

// log2 of a product of two decays; a start in either one stays one, also beside a
// NaN or a decay of infinity (whose NaN is in u, too)
__device__ __forceinline__ float join(float a, float b) {
  const float s = a + b;
  return s == s ? s : fminf(a, b);
}

// first, then second
__device__ __forceinline__ Span then(Span first, Span second) {
  const float r = fmaf(pow2f(second.s), first.u, second.u);
  return {join(first.s, second.s), second.s == neg_inf() ? second.u : r};
}

__device__ __forceinline__ float through(Span sp, float x) {
  const float r = fmaf(pow2f(sp.s), x, sp.u);
  return sp.s == neg_inf() ? sp.u : r;
}

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

// log2 a; behind a sample's end, where log_a is loaded as 0, the state stays as it is
__device__ __forceinline__ float decay(float la) { return la < kStart ? neg_inf() : la * kLog2e; }

// zeros behind a sample's end, where the state goes on
__device__ __forceinline__ void only(float (&x)[kScanV], int n) {
  if (n < kScanV)
#pragma unroll
    for (int j = 0; j < kScanV; ++j) x[j] = j < n ? x[j] : 0.f;
}

__device__ __forceinline__ int64_t row_length(const ScanArgs& a, int64_t row) {
  if (!a.len) return a.L;
  const int64_t n = a.len[(uint32_t)row / (uint32_t)a.C];
  return n < 0 ? 0 : (n > a.L ? a.L : n);
}

// Segments of a split row are taken by workgroups of one launch, each of which
// reads its inputs once and holds them while it learns the state that enters it: a
// prefix in a single pass with look-back (Merrill and Garland, "Single-pass Parallel
// Prefix Scan with Decoupled Look-back", 2016).
// A workgroup draws its segment from its row's counter, so that every segment before
// its own in the row is finished or being worked on.  It publishes what its segment
// does to a state (its span) before it waits for anything, then looks for the nearest segment before it that has published the
// state behind it, and takes the spans between from there on in their order, so
// that the roundings do not depend on the timing.  Each wait ends: a row's first
// segment waits for nothing, and each other one for segments that are being worked on.
// (Two calls at once on one workspace, which callers may not make, spoil the words: a
// draw beyond the row's segments takes none, and a wait that lasts for seconds gives
// up, with NaN.)
//
// Two words a segment, each written at once with its flag in the upper half:
// word 0 (kSpan, s); word 1 (kSpan, u), later (kState, the state behind it).
constexpr uint64_t kSpan = 1, kState = 2;
constexpr int kMostPolls = 1 << 22;

__device__ __forceinline__ uint64_t link_word(uint64_t flag, float x) { return flag << 32 | __float_as_uint(x); }
__device__ __forceinline__ float link_value(uint64_t w) { return __uint_as_float((uint32_t)w); }
__device__ __forceinline__ uint64_t link_load(const uint64_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void link_store(uint64_t* p, uint64_t w) {
  __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The row that this workgroup works on; each row gets nseg of them.  Of few rows,
// eight workgroups, one for each XCD, share one before the next eight go to the next
// (16 rows of 2^20: 47 against 69 us forward, 81 against 106 us backward, bf16); of
// more, neighbours take different ones (128 rows of 2^17 backward, fp32: 131 against 157 us).
__device__ __forceinline__ uint32_t link_row(const ScanArgs& a) {
  const uint32_t R = (uint32_t)a.R;
  if (R >= 64) return blockIdx.x % R;
  const uint32_t turn = blockIdx.x / (8 * R), in = blockIdx.x - turn * 8 * R, left = (uint32_t)a.nseg - 8 * turn;
  return in / (left < 8 ? left : 8);
}

// The segment that this workgroup takes of row `row`, in the order of the recurrence.
__device__ __forceinline__ uint32_t link_draw(const ScanArgs& a, uint32_t row) {
  __shared__ uint32_t drawn;
  if (threadIdx.x == 0)
    drawn = (uint32_t)__hip_atomic_fetch_add(a.links + 2 * a.R * a.nseg + (int64_t)row * kLinkStride, (uint64_t)1,
                                             __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(drawn);
}

// By one wavefront: the state that enters segment `i` (in the order of the
// recurrence) of a row whose words begin at `row`; the row starts from `start`.
__device__ __forceinline__ float link_enter(uint64_t* row, uint32_t i, Span mine, float start, int lane) {
  float x = start;
  if (i > 0) {
    if (lane == 0) {
      link_store(row + 2 * i, link_word(kSpan, mine.s));
      link_store(row + 2 * i + 1, link_word(kSpan, mine.u));
    }
    // lane l looks at segment i - 1 - l
    const bool there = (uint32_t)lane < i;
    const uint64_t* at = row + 2 * (there ? i - 1 - lane : 0);
    uint64_t w = 0;
    int from = -1;
    for (int polls = 0; polls < kMostPolls; ++polls) {
      if (there && w >> 32 != kState) w = link_load(at + 1);
      const uint64_t done = __ballot(there && w >> 32 == kState), known = __ballot(there && w >> 32 != 0);
      if (done) {
        const int nearest = __builtin_ctzll(done);
        const uint64_t between = (uint64_t(1) << nearest) - 1;
        if ((known & between) == between) {
          from = nearest;
          break;
        }
      }
      __builtin_amdgcn_s_sleep(4);
    }
    uint64_t ws = link_word(kSpan, 0.f);
    if (lane < from) {
      ws = link_load(at);
      for (int polls = 0; ws >> 32 != kSpan && polls < kMostPolls; ++polls) {
        __builtin_amdgcn_s_sleep(1);
        ws = link_load(at);
      }
    }
    x = from < 0 ? __builtin_nanf("") : read_lane(link_value(w), from < 0 ? 0 : from);
    const float a = pow2f(link_value(ws));
    const uint64_t starts = __ballot(link_value(ws) == neg_inf());
    for (int l = from - 1; l >= 0; --l) {
      const float u = read_lane(link_value(w), l), r = fmaf(read_lane(a, l), x, u);
      x = (starts >> l) & 1 ? u : r;
    }
  }
  if (lane == 0) link_store(row + 2 * i + 1, link_word(kState, through(mine, x)));
  return x;
}

// Where a lane works: its row and the tile of a wavefront.
template <int G, int W>
struct Place {
  int lane, wave;
  int64_t row;
  bool live;  // false: a lane beyond the last row, which computes on the last one and writes nothing
  __device__ __forceinline__ explicit Place(int64_t R, uint32_t group = blockIdx.x) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if constexpr (W > 1) {
      row = group;
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
