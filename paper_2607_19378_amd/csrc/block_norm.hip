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
template <typename TS, int V, int K, typename Has>
__global__ void __launch_bounds__(V == 1 ? kMaxNT : norm_threads(K)) norm_forward(NormArgs a) {
  __shared__ Joint<1, V> lds;
  const Draws draws(a);
  const int first = threadIdx.x >> a.lp, CL = blockDim.x >> a.lp;
  float w_post[K], w_pre[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = first + k * CL;
    w_post[k] = Has::z(a) && c < a.C ? weight<TS>(a.w_post, c) * weight<TS>(a.scale, c) * a.kept : 0.f;
    w_pre[k] = Has::n(a) && c < a.C ? weight<TS>(a.w_pre, c) : 0.f;
  }
  for (uint32_t turn = blockIdx.x; turn < a.turns; turn += gridDim.x) {
    const uint32_t tile = tile_of(a, turn);
    if (tile >= a.tiles) continue;
    const Held<TS, V, Has::TAIL> at(a, tile);
    Raw<TS, V> x[K], z[K], g[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (first + k * CL < a.C && at.any()) {
        if (Has::z(a)) z[k] = at.load(a.z, k);
        if (Has::g(a)) g[k] = at.load(a.g, k);
        x[k] = at.load(a.x, k);
      } else {
        x[k] = Raw<TS, V>{};
        z[k] = Raw<TS, V>{};
        g[k] = Raw<TS, V>{};
      }
    }
    float y[K][V];  // the branch, then the sum
    float acc[1][V], post[V];
    if (Has::z(a)) {
#pragma unroll
      for (int j = 0; j < V; ++j) acc[0][j] = 0.f;
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          y[k][j] = get(z[k], j);
          if (Has::g(a)) y[k][j] *= sigmoid_of(gate(get(g[k], j)));
          acc[0][j] = fmaf(y[k][j], y[k][j], acc[0][j]);
        }
      over_channels(acc, lds, a.lp, at.pg, [&](int, auto sum, int) { return inverse_rms(sum(0), a.C, a.eps_post); });
      read_sums(lds, 0, at.pg, post);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) acc[0][j] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = first + k * CL;
      if (Has::z(a)) {
        uint32_t drawn[4];
        if (Has::drop(a)) draws.words<V, Has::TAIL>(at.b * a.C + c, at.p, at.shift, drawn);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float w = !Has::drop(a) || draws.keeps(drawn, j) ? w_post[k] : 0.f;
          y[k][j] = fmaf(w, y[k][j] * post[j], get(x[k], j));
        }
        if (c < a.C && at.any()) at.store(a.x_out, k, y[k]);
        __builtin_amdgcn_sched_barrier(0);  // one channel's generator at a time: interleaved, they spill
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) y[k][j] = get(x[k], j);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) acc[0][j] = fmaf(y[k][j], y[k][j], acc[0][j]);
    }
    if (!Has::n(a)) continue;
    over_channels(acc, lds, a.lp, at.pg, [&](int, auto sum, int) { return inverse_rms(sum(0), a.C, a.eps_pre); });
    read_sums(lds, 0, at.pg, post);
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j) y[k][j] *= post[j] * w_pre[k];
      if (first + k * CL < a.C && at.any()) at.store(a.n, k, y[k]);
    }
  }
}

// More channels than registers hold: the tile is read again for each sum.
template <typename TS, int V>
__global__ void __launch_bounds__(kMaxNT) norm_forward_reread(NormArgs a) {
  __shared__ Joint<1, V> lds;
  for (uint32_t turn = blockIdx.x; turn < a.turns; turn += gridDim.x) {
    const uint32_t tile = tile_of(a, turn);
    if (tile >= a.tiles) continue;
    const Spot<V> at(a, tile);
    const int n = clamp_count<V>(a.P - at.p);
    const Draws draws(a);
    float post[1][V], pre[1][V];
    auto branch = [&](int c, float (&t)[V]) {
      const int64_t o = (at.b * a.C + c) * a.P + at.p;
      const Raw<TS, V> z = load<TS, V>(reinterpret_cast<const TS*>(a.z) + o, n);
      Raw<TS, V> g;
      if (a.g) g = load<TS, V>(reinterpret_cast<const TS*>(a.g) + o, n);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        t[j] = get(z, j);
        if (a.g) t[j] *= sigmoid_of(gate(get(g, j)));
      }
    };
    auto sum = [&](int c, float (&y)[V]) {
      const Raw<TS, V> x = load<TS, V>(reinterpret_cast<const TS*>(a.x) + (at.b * a.C + c) * a.P + at.p, n);
      if (!a.z) {
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = get(x, j);
        return;
      }
      branch(c, y);
      const float w = weight<TS>(a.w_post, c) * weight<TS>(a.scale, c) * a.kept;
      uint32_t drawn[4];
      if (a.drop) draws.words<V, false>(at.b * a.C + c, at.p, 0, drawn);
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] = fmaf(!a.drop || draws.keeps(drawn, j) ? w : 0.f, y[j] * post[0][j], get(x, j));
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
      over_channels(post, lds, a.lp, at.pg, [&](int, auto sum, int) { return inverse_rms(sum(0), a.C, a.eps_post); });
      read_sums(lds, 0, at.pg, post[0]);
    }
    for (int c = at.cl; c < a.C; c += at.CL) {
      float y[V];
      sum(c, y);
      if (a.z) store<TS, V>(reinterpret_cast<TS*>(a.x_out) + (at.b * a.C + c) * a.P + at.p, y, n);
#pragma unroll
      for (int j = 0; j < V; ++j) pre[0][j] = fmaf(y[j], y[j], pre[0][j]);
    }
    if (!a.n) continue;
    over_channels(pre, lds, a.lp, at.pg, [&](int, auto sum, int) { return inverse_rms(sum(0), a.C, a.eps_pre); });
    read_sums(lds, 0, at.pg, pre[0]);
    for (int c = at.cl; c < a.C; c += at.CL) {
      float y[V];
      sum(c, y);
      const float w = weight<TS>(a.w_pre, c);
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] *= pre[0][j] * w;
      store<TS, V>(reinterpret_cast<TS*>(a.n) + (at.b * a.C + c) * a.P + at.p, y, n);
    }
  }
}

constexpr uint32_t kMaxGrid = 1u << 20;  // workgroups of a launch (fewer than 2^32 work-items)

template <typename TS, typename Has>
hipError_t forward_held(const NormArgs& a, const NormShape& s, hipStream_t st) {
  const dim3 grid((unsigned)(a.turns < kMaxGrid ? a.turns : kMaxGrid)), block((unsigned)s.NT);
  constexpr int V = 16 / sizeof(TS);
#define HY_CASE(v, k) \
  if (s.V == v && s.K == k) hipLaunchKernelGGL((norm_forward<TS, v, k, Has>), grid, block, 0, st, a);
  if constexpr (!Has::TAIL) {
    HY_CASE(1, 1) HY_CASE(1, 4) HY_CASE(1, 8)
  }
  HY_CASE(V, 1) HY_CASE(V, 2) HY_CASE(V, 4) HY_CASE(V, 8)
#undef HY_CASE
  return hipGetLastError();
}

template <typename TS, bool TAIL>
hipError_t forward_parts(const NormArgs& a, const NormShape& s, hipStream_t st) {
  if (!a.z || !a.n) return forward_held<TS, Parts<false, false, false, TAIL>>(a, s, st);
  if (a.drop)
    return a.g ? forward_held<TS, Parts<true, true, true, TAIL>>(a, s, st)
               : forward_held<TS, Parts<true, false, true, TAIL>>(a, s, st);
  return a.g ? forward_held<TS, Parts<true, true, false, TAIL>>(a, s, st)
             : forward_held<TS, Parts<true, false, false, TAIL>>(a, s, st);
}

template <typename TS>
hipError_t forward(const NormArgs& a, const NormShape& s, hipStream_t st) {
  if (s.K > 0) return a.P % s.V == 0 ? forward_parts<TS, false>(a, s, st) : forward_parts<TS, true>(a, s, st);
  const dim3 grid((unsigned)(a.turns < kMaxGrid ? a.turns : kMaxGrid)), block((unsigned)s.NT);
  constexpr int V = 16 / sizeof(TS);
  if (s.V == 1) hipLaunchKernelGGL((norm_forward_reread<TS, 1>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((norm_forward_reread<TS, V>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace

// A row's accesses are as wide as 8 lanes make them (128 bytes), since narrower
// ones cost most (8 x 256 x 64 x 64 fp32 forward: 40 us at 128 bytes, 45, 48 and 61 us
// at 64, 32 and 16; backward of 2 x 512 x 8192 bf16: 47 us at 64 bytes, 56 and 73 us
// at 32 and 16), as far as the channels then fit.  The forward takes four channels a
// thread in 512 threads where two would need 1024 (2 x 512 x 8192 bf16: 21 against
// 24 us, two workgroups a CU), unless that leaves CUs without a tile; eight only
// where four would halve the width to 16 bytes (2 x 2048 x 2048 bf16: 30 against
// 34 us; 2 x 512 x 8192: 27 against 21 us for 128 bytes in place of 64).  The backward
// takes as few channels a thread as fit (2 x 512 x 8192 bf16: 47 us with two, 50 us
// with four), and gives up tiles of 16 bytes for two sweeps (norm_sums).
// Rows shorter than a lane's 16 bytes are one point a lane; four channels a thread where
// threads of one would fill the chip (2^19 of them; 4096 x 1024 x 1 bf16: forward 21 against 53
// us, at 256 samples 5.8 against 4.7) or, backward, fill it twice (43 against 66 us, at 512
// samples 15.0 against 14.2), as long as more than a wavefront is left of a tile (8192 x 64 x 3
// fp32: 37 against 32 us, forward 11 against 15).
NormShape norm_shape(int64_t C, int64_t P, int64_t B, bool bf16, bool backward) {
  NormShape s;
  const int V = bf16 ? 8 : 4;
  s.V = P < V ? 1 : V;
  auto threads = [&](int K, int lp) { return (((C + K - 1) / K << lp) + 63) / 64 * 64; };
  auto take = [&](int K, int lp, int most) {
    if (threads(K, lp) > most) return false;
    s.K = K;
    s.lp = lp;
    s.NT = (int)threads(K, lp);
    return true;
  };
  const int64_t groups = (P + s.V - 1) / s.V;
  int lp = 0;
  while (lp < 3 && (int64_t(1) << lp) < groups) ++lp;
  const int widest = lp;
  // 32-bit offsets in a sample's tensors
  if (C * P <= (int64_t(1) << 32) / (bf16 ? 2 : 4) - 4096) {
    for (; lp >= 0; --lp) {
      if (s.V == 1) {
        const int64_t fill = threads(1, lp) < (backward ? 512 : 256) ? 0 : B * threads(1, lp) >> 19;
        if (fill >= (backward ? 2 : 1) && take(4, lp, kMaxNT)) return s;
        if (take(1, lp, kMaxNT) || take(4, lp, kMaxNT) || (!backward && take(8, lp, kMaxNT))) return s;
        continue;
      }
      if (backward && lp == 0 && widest > 0) break;
      const bool many = (groups >> lp) * B >= 512;
      if (!backward && many && (take(1, lp, 512) || take(2, lp, 512) || take(4, lp, 512))) return s;
      if (take(1, lp, kMaxNT) || take(2, lp, kMaxNT)) return s;
      if (!backward && lp <= 1 && take(8, lp, norm_threads(8))) return s;
    }
  }
  s.lp = widest;
  s.K = 0;
  if (!backward) s.lp = 0;
  s.NT = (int)(C < kMaxNT ? threads(1, 0) : kMaxNT);
  return s;
}

// log2 of the consecutive tiles of an XCD's turn: 32 lanes' points, 512 bytes of a row, but
// every XCD has a turn (1 x 2048 x 256 fp32: 12 against 17 us forward, 14 against 24 backward).
// Samples of one tile share no lines.  Forward, up to 32 of them stay together all the same, as
// each XCD that has one fetches the weights (32 x 1024 x 1 bf16: 3.6 us against 4.2 for one
// after the other; 128 x 2048 x 1: 5.1 against 5.3), but no more than 256 KB of a tensor, or one
// XCD moves too much (32 x 8192 x 1 bf16: 8.3 us against 13.1 for 32 together and 8.4 for one
// after the other; 32 x 4096 x 1 fp32: 5.1, 6.4 and 5.2).  Backward every workgroup less is one
// less to add up (64 x 6000 x 1 bf16: 16 against 37 us).
uint32_t norm_log_run(int64_t sample_bytes, int64_t tiles, int64_t row_tiles, int lp, bool backward) {
  if (row_tiles == 1 && backward) return 0;
  int run = 5 - lp;
  if (row_tiles == 1)
    while (run > 0 && sample_bytes << run > 256 * 1024) --run;
  else
    while (run > 0 && tiles < int64_t(8) << run) --run;
  return (uint32_t)run;
}

void norm_tiles(NormArgs& a, const NormShape& s, bool backward) {
  const int64_t points = (int64_t)s.V << s.lp, row_tiles = (a.P + points - 1) / points;
  a.lp = s.lp;
  a.row_tiles = (uint32_t)row_tiles;
  a.tiles = (uint32_t)(row_tiles * a.B);  // fewer than 2^31 + 2^26: kMaxNormPoints points, of which a tile has 4 or a row's
  a.log_run = norm_log_run(a.C * a.P * (a.bf16 ? 2 : 4), a.tiles, row_tiles, s.lp, backward);
  const uint32_t round = a.log_run > 0 ? 8u << a.log_run : 1;
  a.turns = (a.tiles + round - 1) / round * round;
}

hipError_t launch_norm(const NormArgs& args, hipStream_t st) {
  NormArgs a = args;
  const NormShape s = norm_shape(a.C, a.P, a.B, a.bf16, false);
  norm_tiles(a, s, false);
  return a.bf16 ? forward<uint16_t>(a, s, st) : forward<float>(a, s, st);
}

}  // namespace hyenand
