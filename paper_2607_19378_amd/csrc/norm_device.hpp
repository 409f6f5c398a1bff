// Device parts of the norms around a block, shared by forward and backward.
//
// The norms run over the channels of a point, whose stride is a row.  A workgroup
// takes a tile of 2^lp * V consecutive points of all channels: the lanes of a
// wavefront lie 2^lp over the points (V consecutive ones each) and the others
// over channels, so that a tile's rows are read in whole cache lines where the
// channels fit.  The tile stays in registers between the sums.
#pragma once

#include "norm.hpp"
#include "row_access.hpp"

namespace hyenand {
namespace norm_dev {

using rows::keep_packed;
using rows::Raw;

constexpr int kMaxNT = 1024;
constexpr int kMaxLanes = 8;  // over a channel's points

// sigmoid(g) as the bits of the smaller of it and 1 - sigmoid(g), with the sign bit
// set where that is the latter: both follow from it to an fp32 rounding of their own.
// Bits and no float: the smaller one is 0 for gates far from 0, and the library is
// compiled with -fno-signed-zeros, which lets the sign of a float 0 be lost.
__device__ __forceinline__ uint32_t gate(float g) {
  const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(g));
  const float m = e * __builtin_amdgcn_rcpf(1.f + e);
  return __float_as_uint(m) | (~__float_as_uint(g) & 0x80000000u);
}
constexpr uint32_t kNoGate = 0x80000000u;  // of sigmoid 1
__device__ __forceinline__ float sigmoid_of(uint32_t m) { return m >> 31 ? 1.f + __uint_as_float(m) : __uint_as_float(m); }
__device__ __forceinline__ float rest_of(uint32_t m) { return m >> 31 ? -__uint_as_float(m) : 1.f - __uint_as_float(m); }

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as
// 1, 2, 3", 2011): four 32-bit words from a 128-bit counter and a 64-bit key.
__device__ __forceinline__ void philox(uint64_t index, uint64_t offset, uint64_t seed, uint32_t (&w)[4]) {
  uint32_t c0 = (uint32_t)index, c1 = (uint32_t)(index >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
  asm volatile("" : "+s"(k0), "+s"(k1));  // or the keys of all rounds are kept in registers, of which there are too few
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = __builtin_amdgcn_bitop3_b32((uint32_t)(p1 >> 32), c1, k0, 0x96);  // a ^ b ^ c
    c1 = (uint32_t)p1;
    c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(p0 >> 32), c3, k1, 0x96);
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  w[0] = c0;
  w[1] = c1;
  w[2] = c2;
  w[3] = c3;
}

// The draws of a call: eight points of a row, from a multiple of eight on, take the
// eight halves of one output of the generator.
struct Draws {
  uint64_t seed, offset;
  int64_t groups;  // of a row
  uint32_t drop;
  static __device__ __forceinline__ uint64_t uniform(uint64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
    return (uint64_t)hi << 32 | lo;
  }
  __device__ __forceinline__ explicit Draws(const NormArgs& a) {
    seed = uniform(a.drop ? a.rng[0] : 0);
    offset = uniform(a.drop ? a.rng[1] : 0);
    groups = (a.P + 7) / 8;
    drop = a.drop;
  }
  // The draws of V points of row `row`, p the first one, a multiple of V; place j
  // has that of point j - shift.
  template <int V, bool TAIL>
  __device__ __forceinline__ void words(int64_t row, int64_t p, int shift, uint32_t (&w)[4]) const {
    philox((uint64_t)(row * groups + (p >> 3)), offset, seed, w);
    if constexpr (V == 1) {
      const int i = (int)(p & 7);
      uint32_t x = w[0];
#pragma unroll
      for (int j = 1; j < 4; ++j) x = i / 2 == j ? w[j] : x;
      w[0] = (i & 1) ? x >> 16 : x;
    }
    if (V == 4 && (p & 4)) {
      w[0] = w[2];
      w[1] = w[3];
    }
    if (V > 1 && TAIL && shift) {  // the row's last points
      if (V == 8 && (shift & 4)) {
        w[3] = w[1];
        w[2] = w[0];
      }
      if (shift & 2) {
        if (V == 8) {
          w[3] = w[2];
          w[2] = w[1];
        }
        w[1] = w[0];
      }
      if (shift & 1) {
        if (V == 8) {
          w[3] = w[3] << 16 | w[2] >> 16;
          w[2] = w[2] << 16 | w[1] >> 16;
        }
        w[1] = w[1] << 16 | w[0] >> 16;
        w[0] <<= 16;
      }
    }
  }
  __device__ __forceinline__ bool keeps(const uint32_t (&w)[4], int j) const {
    return ((j & 1) ? w[j / 2] >> 16 : w[j / 2] & 0xffffu) >= drop;
  }
};

// The tile of turn `w` (a workgroup's index, then that and the launch's number of
// workgroups, ...).  Workgroups go round the 8 XCDs; neighbouring tiles, which
// share cache lines where they are narrower than one, go to the same XCD, whose L2
// then reads the lines once: runs of 2^log_run tiles for each XCD in turn.
__device__ __forceinline__ uint32_t tile_of(const NormArgs& a, uint32_t w) {
  const uint32_t q = w >> 3;
  return (((q >> a.log_run) * 8 + (w & 7)) << a.log_run) + (q & ((1u << a.log_run) - 1));
}

// Where a thread of a tile works, tile by tile: its group of points, its first
// channel and the distance to its next one.
template <int V>
struct Spot {
  int pg, cl, CL;
  int64_t b, p;  // sample and first point
  __device__ __forceinline__ Spot(const NormArgs& a, uint32_t tile) {
    pg = threadIdx.x & ((1 << a.lp) - 1);
    cl = threadIdx.x >> a.lp;
    CL = blockDim.x >> a.lp;
    const uint32_t q = tile / a.row_tiles;
    b = q;
    p = ((int64_t)(tile - q * a.row_tiles) * V << a.lp) + pg * V;
  }
};

// The same for a thread whose tile stays in registers.  With TAIL (rows that are
// no whole number of V points) a lane at a row's end takes the row's last V points, so
// that each load is a whole one; its own are those from `shift` on, the others are
// computed and not written.  Offsets are of 32 bits from the sample's tensors.
template <typename TS, int V, bool TAIL>
struct Held : Spot<V> {
  int shift;           // V: no point of the row
  uint32_t off, step;  // of the first channel's points, and to the next channel's, in bytes
  int64_t sample;      // of the sample's tensors
  __device__ __forceinline__ Held(const NormArgs& a, uint32_t tile) : Spot<V>(a, tile) {
    const int64_t over = this->p + V - a.P;
    shift = over > 0 ? (over < V ? (int)over : V) : 0;
    off = (uint32_t)(((int64_t)this->cl * a.P + (TAIL && over > 0 ? a.P - V : this->p)) * (int)sizeof(TS));
    step = (uint32_t)((int64_t)this->CL * a.P * (int)sizeof(TS));
    sample = this->b * a.C * a.P * (int)sizeof(TS);
  }
  // whether it has points to load: with TAIL also lanes that have none of their own
  __device__ __forceinline__ bool any() const { return TAIL || shift < V; }
  // a tensor's part of this sample, computed for each access: kept for all eight
  // tensors, the addresses would take the scalar registers
  __device__ __forceinline__ char* part(const void* t) const {
    int64_t s = sample;
    asm volatile("" : "+s"(s));
    return reinterpret_cast<char*>(const_cast<void*>(t)) + s;
  }
  __device__ __forceinline__ Raw<TS, V> load(const void* t, int k) const {
    return rows::load_at<TS, V>(part(t), off + k * step);
  }
  // the same with zeros in the points that are not this lane's
  __device__ __forceinline__ Raw<TS, V> load_own(const void* t, int k) const {
    Raw<TS, V> r = load(t, k);
    if (TAIL && shift) {
      int first = shift;
      asm volatile("" : "+v"(first));  // or a mask for each point is kept, here and in store()
      if constexpr (sizeof(TS) == 2 && V > 1) {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (j < first) r.w[j / 2] &= (j & 1) ? 0xffffu : 0xffff0000u;
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (j < first) r.w[j] = 0u;
      }
    }
    return r;
  }
  __device__ __forceinline__ void store(void* t, int k, const float (&y)[V]) const {
    char* base = part(t);
    if (!TAIL || shift == 0) {
      rows::store_at<TS, V>(base, off + k * step, y);
    } else {
      int first = shift;
      asm volatile("" : "+v"(first));
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j >= first) st1(reinterpret_cast<TS*>(base + off + k * step) + j, y[j]);
    }
  }
};

// x + its value in the lanes D apart of a row of 16, the sum so far having that period
template <int D>
__device__ __forceinline__ float add_across(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + D, 0xf, 0xf, false));
}

// a + its other half in the lower lanes, b + its other half in the upper ones
// (halves of a wavefront, or of each of its two halves): two sums in one swap
template <int D>
__device__ __forceinline__ float add_halves(float a, float b) {
  const auto r = D == 32 ? __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false)
                         : __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// M sums over the channels of each point of the tile.  all[m] is what finish(m,
// sum, point) makes of them; it may ask for another one of the point's sums.
template <int M, int V>
struct Joint {
  float part[kMaxNT / 64][M * V][kMaxLanes];
  alignas(16) float all[M][kMaxLanes * V];
};

// The lanes of a wavefront are joined with their values halved at each of the
// first steps, so that N values take about 2 N instructions; the wavefronts in LDS.
template <int M, int V, typename F>
__device__ __forceinline__ void over_channels(const float (&acc)[M][V], Joint<M, V>& lds, int lp, int pg, F finish) {
  constexpr int N = M * V, N1 = N % 2 ? N : N / 2, N2 = N1 % 2 ? N1 : N1 / 2;
  constexpr bool halves = N1 < N, quarters = N2 < N1;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, LP = 1 << lp;
  float x[N], y[N1], z[N2];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = acc[i / V][i % V];
#pragma unroll
  for (int i = 0; i < N1; ++i) y[i] = add_halves<32>(x[i], x[halves ? i + N1 : i]);
#pragma unroll
  for (int i = 0; i < N2; ++i) z[i] = add_across<8>(add_halves<16>(y[i], y[quarters ? i + N2 : i]));
  if (lp < 3)
#pragma unroll
    for (int i = 0; i < N2; ++i) z[i] = add_across<4>(z[i]);
  if (lp < 2)
#pragma unroll
    for (int i = 0; i < N2; ++i) z[i] = add_across<2>(z[i]);
  if (lp < 1)
#pragma unroll
    for (int i = 0; i < N2; ++i) z[i] = add_across<1>(z[i]);
  if ((lane & 15) < LP && (halves || lane < 32) && (quarters || !(lane & 16))) {
    const int from = (halves && lane >= 32 ? N1 : 0) + (quarters && (lane & 16) ? N2 : 0);
#pragma unroll
    for (int i = 0; i < N2; ++i) lds.part[wave][from + i][pg] = z[i];
  }
  __syncthreads();
  for (int t = threadIdx.x; t < N << lp; t += blockDim.x) {
    const int i = t >> lp, g = t & (LP - 1);
    auto sum = [&](int m) {
      float x = 0.f;
#pragma unroll 4
      for (int w = 0; w < waves; ++w) x += lds.part[w][m * V + i % V][g];
      return x;
    };
    const int m = i / V, point = g * V + i % V;
    lds.all[m][point] = finish(m, sum, point);
  }
  __syncthreads();
}

// sum m of a lane's points.  Read where it is used: held, the sums would push the
// tile out of the registers, so the compiler may not carry them over next_channel().
template <int M, int V, int N>
__device__ __forceinline__ void read_sums(const Joint<M, V>& lds, int m, int pg, float (&x)[N], int from = 0) {
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] = lds.all[m][pg * V + from + j];
}
__device__ __forceinline__ void next_channel() { asm volatile("" ::: "memory"); }

// What a call has: known beforehand for a block with its branch and both norms
// (KNOWN), looked up for the others.  TAIL: see Held.
template <bool KNOWN, bool GATE, bool DROP, bool TAIL_>
struct Parts {
  static constexpr bool TAIL = TAIL_;
  static __device__ __forceinline__ bool z(const NormArgs& a) { return KNOWN || a.z; }
  static __device__ __forceinline__ bool g(const NormArgs& a) { return KNOWN ? GATE : a.g != nullptr; }
  static __device__ __forceinline__ bool drop(const NormArgs& a) { return KNOWN ? DROP : a.drop != 0; }
  static __device__ __forceinline__ bool n(const NormArgs& a) { return KNOWN || a.n; }
  static __device__ __forceinline__ bool gn(const NormArgs& a) { return KNOWN || a.gn; }
  static __device__ __forceinline__ bool gx_out(const NormArgs& a) { return KNOWN || a.gx_out; }
};

// 1 / rms of C channels whose squares sum to s; 0 for a point of zeros without an eps
__device__ __forceinline__ float inverse_rms(float s, int C, float eps) {
  const float r = sqrtf(s / (float)C + eps);
  return r > 0.f || r != r ? 1.f / r : 0.f;
}

template <typename TS>
__device__ __forceinline__ float weight(const void* w, int c) {
  return w ? ld1(reinterpret_cast<const TS*>(w) + c) : 1.f;
}

}  // namespace norm_dev

// How a call's tiles are cut: points a lane (16 bytes of them, or 1 for rows of
// one), log2 of the lanes over points, channels a thread (0: more than its
// registers hold, the tile is read again instead), threads.
struct NormShape {
  int V, lp, K, NT;
};
// threads of a workgroup at most, so that K channels a thread stay in registers
constexpr int norm_threads(int K) { return K > 2 ? 512 : 1024; }
NormShape norm_shape(int64_t C, int64_t P, int64_t B, bool bf16, bool backward);
uint32_t norm_log_run(int64_t sample_bytes, int64_t tiles, int64_t row_tiles, int lp, bool backward);
void norm_tiles(NormArgs& a, const NormShape& s, bool backward);

}  // namespace hyenand
