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

constexpr int kMaxNT = 1024;
constexpr int kMaxPoints = 64;  // of a tile

// sigmoid(g) and 1 - sigmoid(g), neither as a difference
__device__ __forceinline__ void gates(float g, float* sig, float* rest) {
  const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(g));
  const float s = __builtin_amdgcn_rcpf(1.f + e);
  const float t = e * s;
  *sig = g >= 0.f ? s : t;
  *rest = g >= 0.f ? t : s;
  if (g != g) *sig = *rest = g;
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as
// 1, 2, 3", 2011): four 32-bit words from a 128-bit counter and a 64-bit key.
__device__ __forceinline__ void philox(uint64_t index, uint64_t offset, uint64_t seed, uint32_t (&w)[4]) {
  uint32_t c0 = (uint32_t)index, c1 = (uint32_t)(index >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)p1;
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  w[0] = c0;
  w[1] = c1;
  w[2] = c2;
  w[3] = c3;
}

// The factors (0 or a.kept) of the V points from p on (a multiple of eight) of
// row `row`: eight points take the eight halves of one output of the generator.
template <int V>
__device__ __forceinline__ void keep_factors(const NormArgs& a, uint64_t seed, uint64_t offset, int64_t row, int64_t p,
                                             float (&f)[V]) {
  uint32_t w[4];
  philox((uint64_t)row * (uint64_t)((a.P + 7) / 8) + (uint64_t)(p / 8), offset, seed, w);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const uint32_t bits = (j & 1) ? w[j / 2] >> 16 : w[j / 2] & 0xffffu;
    f[j] = bits >= a.drop ? a.kept : 0.f;
  }
}

// Where a thread of a tile works.
template <int V>
struct Spot {
  int pg, cl, CL;   // group of points, first channel, and the distance to its next one
  int64_t b, p;     // sample and first point
  int n;            // points there
  __device__ __forceinline__ Spot(const NormArgs& a, int64_t tile) {
    pg = threadIdx.x & ((1 << a.lp) - 1);
    cl = threadIdx.x >> a.lp;
    CL = blockDim.x >> a.lp;
    // a 32-bit quotient where it is one
    b = a.tiles <= 0xffffffffll ? (int64_t)((uint32_t)tile / (uint32_t)a.row_tiles) : tile / a.row_tiles;
    p = ((tile - b * a.row_tiles) << a.lp) * V + pg * V;
    n = rows::clamp_count<V>(a.P - p);
  }
};

// M sums over the channels of each point of the tile, S(sum, m) of which every
// lane of the point gets: over the lanes of a wavefront, then in LDS.
template <int M>
struct Joint {
  float part[M][kMaxNT / 64][kMaxPoints];
  float all[M][kMaxPoints];
};

template <int M, int V, typename F>
__device__ __forceinline__ void over_channels(float (&acc)[M][V], Joint<M>& lds, int lp, int pg, F finish) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, LP = 1 << lp;
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int j = 0; j < V; ++j)
      for (int d = LP; d < 64; d *= 2) acc[m][j] += __shfl_xor(acc[m][j], d);
  if (lane < LP)
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int j = 0; j < V; ++j) lds.part[m][wave][pg * V + j] = acc[m][j];
  __syncthreads();
  if (threadIdx.x < (unsigned)(LP * V)) {
    float sum[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      sum[m] = 0.f;
      for (int w = 0; w < waves; ++w) sum[m] += lds.part[m][w][threadIdx.x];
    }
    finish(sum);
#pragma unroll
    for (int m = 0; m < M; ++m) lds.all[m][threadIdx.x] = sum[m];
  }
  __syncthreads();
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int j = 0; j < V; ++j) acc[m][j] = lds.all[m][pg * V + j];
}

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

// How a call's tiles are cut: V points a lane (1 for rows of one point), log2 of
// the lanes over points, channels a thread (0: more than its registers hold, the
// tile is read again instead), threads.
struct NormShape {
  int V, lp, K, NT;
};
NormShape norm_shape(int64_t C, int64_t P, bool bf16, bool backward);
void norm_tiles(NormArgs& a, const NormShape& s);

}  // namespace hyenand
