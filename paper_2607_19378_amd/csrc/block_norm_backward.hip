// Gradients of the norms around a block (block_norm.hip).  With q = 1 / rms(x),
// r = 1 / rms(t), means over the C channels of a point, x the forward's x_out:
//
//   gx = gx_out + q (gn w_pre - x q^2 mean(gn w_pre x))
//   gm = scale drop(gx),  gt = r (gm w_post - t r^2 mean(gm w_post t))
//   gz = gt sigmoid(g),   gg = gt t (1 - sigmoid(g))
//   gw_pre = sum gn x q,  gw_post = scale S, gscale = w_post S,
//   S = sum drop(gx) t r  (over samples and points)
//
// Bound by HBM: five tensors read and three written.  The dropped points are drawn
// again from the counter.  A workgroup takes tile after tile and adds its weight
// sums up in registers; a second kernel adds those of the workgroups, in order.
#include "norm_device.hpp"

namespace hyenand {

using namespace rows;
using namespace norm_dev;

namespace {

// The raw inputs of V points of a channel.
template <typename TS, int V>
struct BwdRow {
  Raw<TS, V> x, gn, gxo, z, g;
};

template <typename Has, typename TS, int V>
__device__ __forceinline__ void load_row(BwdRow<TS, V>& r, const NormArgs& a, const Held<TS, V, Has::TAIL>& at, int k) {
  r.x = at.load(a.x, k);
  if (Has::gn(a)) r.gn = at.load_own(a.gn, k);
  if (Has::z(a)) {
    r.z = at.load(a.z, k);
    if (Has::g(a)) r.g = at.load(a.g, k);
  }
  if (Has::gx_out(a)) r.gxo = at.load_own(a.gx_out, k);
}

template <typename TS, int V>
__device__ __forceinline__ void load_row(BwdRow<TS, V>& r, const NormArgs& a, int64_t o, int n) {
  r.x = load<TS, V>(reinterpret_cast<const TS*>(a.x) + o, n);
  if (a.gn) r.gn = load<TS, V>(reinterpret_cast<const TS*>(a.gn) + o, n);
  if (a.z) {
    r.z = load<TS, V>(reinterpret_cast<const TS*>(a.z) + o, n);
    if (a.g) r.g = load<TS, V>(reinterpret_cast<const TS*>(a.g) + o, n);
  }
  if (a.gx_out) r.gxo = load<TS, V>(reinterpret_cast<const TS*>(a.gx_out) + o, n);
}

// What is left of the sums of the first kind: q = 1 / rms(x), mean(gn w_pre x), r = 1 / rms(t)
__device__ __forceinline__ float first_kind(const NormArgs& a, int m, float s) {
  return m == 1 ? s / (float)a.C : inverse_rms(s, a.C, m == 0 ? a.eps_pre : a.eps_post);
}

// The gates (see gate()) of a channel's points, from the first sums on in LDS: in
// registers, they would push the tile out of them.  A thread reads what it wrote.
extern __shared__ float gate_lds[];
template <int V>
struct Gates {
  static constexpr int N = V < 4 ? V : 4;  // points at a time
  float* at;
  __device__ __forceinline__ explicit Gates(int k) : at(gate_lds + ((size_t)k * V * blockDim.x + N * threadIdx.x)) {}
  __device__ __forceinline__ void write(int from, const float (&x)[N]) const { __builtin_memcpy(place(from), x, sizeof x); }
  __device__ __forceinline__ void read(int from, float (&x)[N]) const { __builtin_memcpy(x, place(from), sizeof x); }
  __device__ __forceinline__ float* place(int from) const {
    return reinterpret_cast<float*>(__builtin_assume_aligned(at + (size_t)from * blockDim.x, N * 4));
  }
};

// The gates of V points, and the sums of the first kind: squares of x, gn w_pre x,
// squares of t
template <typename Has, typename TS, int V>
__device__ __forceinline__ void first_sums(const BwdRow<TS, V>& r, const NormArgs& a, float w_pre, const Gates<V>& gates,
                                           float (&acc)[3][V]) {
  constexpr int N = Gates<V>::N;
#pragma unroll
  for (int from = 0; from < V; from += N) {
    float half[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int j = from + i;
      if (Has::gn(a)) {
        const float x = get(r.x, j);
        acc[0][j] = fmaf(x, x, acc[0][j]);
        acc[1][j] = fmaf(get(r.gn, j) * w_pre, x, acc[1][j]);
      }
      if (Has::z(a)) {
        float t = get(r.z, j);
        if (Has::g(a)) {
          half[i] = gate(get(r.g, j));
          t *= sigmoid_of(half[i]);
        }
        acc[2][j] = fmaf(t, t, acc[2][j]);
      }
    }
    if (Has::z(a) && Has::g(a)) gates.write(from, half);
    next_channel();
    __builtin_amdgcn_sched_barrier(0);
  }
}

// gx of V points; what reaches the branch's norm (gmw), and its sum with t (the
// second kind); wp = w_post scale.  Points that are not the lane's own come with
// zeros for gn and gx_out and add nothing to the weights' sums.
template <typename Has, typename TS, int V>
__device__ __forceinline__ void second_sums(const BwdRow<TS, V>& r, const NormArgs& a, const Draws& draws, int64_t row,
                                            int64_t p, int shift, float w_pre, float wp, const Joint<3, V>& lds, int pg,
                                            const Gates<V>& gates, float (&gx)[V], float (&gmw)[V], float (&sum)[1][V],
                                            float2* weights) {
  constexpr int N = Gates<V>::N;
  uint32_t drawn[4];
  if (Has::z(a) && Has::drop(a)) draws.words<V, Has::TAIL>(row, p, shift, drawn);
#pragma unroll
  for (int from = 0; from < V; from += N) {
    float q[N], mean[N], rinv[N], half[N];
    if (Has::z(a) && Has::g(a)) gates.read(from, half);
    if (Has::gn(a)) {
      read_sums(lds, 0, pg, q, from);
      read_sums(lds, 1, pg, mean, from);
    }
    if (Has::z(a)) read_sums(lds, 2, pg, rinv, from);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int j = from + i;
      gx[j] = Has::gx_out(a) ? get(r.gxo, j) : 0.f;
      if (Has::gn(a)) {
        const float gn = get(r.gn, j), xq = get(r.x, j) * q[i];
        gx[j] = fmaf(q[i], fmaf(-xq, mean[i] * q[i], gn * w_pre), gx[j]);
        weights->x = fmaf(gn, xq, weights->x);
      }
      if (Has::z(a)) {
        const float kept = Has::drop(a) ? draws.factor(drawn, j) * gx[j] : gx[j];
        float t = get(r.z, j);
        if (Has::g(a)) t *= sigmoid_of(half[i]);
        gmw[j] = kept * wp;
        sum[0][j] = fmaf(gmw[j], t, sum[0][j]);
        weights->y = fmaf(kept, t * rinv[i], weights->y);
      }
    }
    // here, or the sums are put off to the next tile, with all that they take
    asm volatile("" : "+v"(weights->x), "+v"(weights->y));
    next_channel();
  }
}

// gz and gg of V points
template <typename Has, typename TS, int V>
__device__ __forceinline__ void last_row(const Raw<TS, V>& z, const NormArgs& a, const Joint<3, V>& lds,
                                         const Joint<1, V>& lds1, int pg, const Gates<V>& gates, const float (&gmw)[V],
                                         float (&gz)[V], float (&gg)[V]) {
  constexpr int N = Gates<V>::N;
#pragma unroll
  for (int from = 0; from < V; from += N) {
    float rinv[N], mean[N], half[N];
    if (Has::g(a)) gates.read(from, half);
    read_sums(lds, 2, pg, rinv, from);
    read_sums(lds1, 0, pg, mean, from);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int j = from + i;
      const float sig = Has::g(a) ? sigmoid_of(half[i]) : 1.f;
      const float t = get(z, j) * sig;
      const float gt = rinv[i] * fmaf(-t * rinv[i], mean[i] * rinv[i], gmw[j]);
      gz[j] = gt * sig;
      gg[j] = Has::g(a) ? gt * t * rest_of(half[i]) : 0.f;
    }
    next_channel();
  }
}

template <typename TS, int V, int K, typename Has>
__global__ void __launch_bounds__(V == 1 ? kMaxNT : norm_threads(K)) norm_backward(NormArgs a) {
  __shared__ Joint<3, V> lds;
  __shared__ Joint<1, V> lds1;
  const Draws draws(a);
  const int first = threadIdx.x >> a.lp, CL = blockDim.x >> a.lp;
  float2 weights[K];
  float wp[K], w_pre[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = first + k * CL;
    weights[k] = make_float2(0.f, 0.f);
    wp[k] = Has::z(a) && c < a.C ? weight<TS>(a.w_post, c) * weight<TS>(a.scale, c) : 0.f;
    w_pre[k] = Has::gn(a) && c < a.C ? weight<TS>(a.w_pre, c) : 0.f;
  }
  // this workgroup's next tile, from turn `turn` on (a.tiles: none)
  uint32_t turn = blockIdx.x;
  auto next_tile = [&]() {
    for (; turn < a.turns; turn += gridDim.x) {
      const uint32_t tile = tile_of(a, turn);
      if (tile < a.tiles) {
        turn += gridDim.x;
        return tile;
      }
    }
    return a.tiles;
  };
  BwdRow<TS, V> r[K];
  auto fetch = [&](const Held<TS, V, Has::TAIL>& at) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      r[k] = BwdRow<TS, V>{};
      if (first + k * CL < a.C && at.any()) load_row<Has>(r[k], a, at, k);
    }
  };
  uint32_t tile = next_tile();
  if (tile < a.tiles) fetch(Held<TS, V, Has::TAIL>(a, tile));
  while (tile < a.tiles) {
    const Held<TS, V, Has::TAIL> at(a, tile);
    float acc[3][V], sum[1][V], gmw[K][V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[0][j] = acc[1][j] = acc[2][j] = sum[0][j] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) first_sums<Has>(r[k], a, w_pre[k], Gates<V>(k), acc);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      keep_packed(r[k].x);
      keep_packed(r[k].gn);
      keep_packed(r[k].gxo);
      keep_packed(r[k].z);
    }
    over_channels(acc, lds, a.lp, at.pg, [&](int m, float s) { return first_kind(a, m, s); });
    Raw<TS, V> z[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float gx[V];
      second_sums<Has>(r[k], a, draws, at.b * a.C + first + k * CL, at.p, at.shift, w_pre[k], wp[k], lds, at.pg, Gates<V>(k),
                       gx, gmw[k], sum, &weights[k]);
      if (first + k * CL < a.C && at.any()) at.store(a.gx, k, gx);
      keep_packed(r[k].z);
      z[k] = r[k].z;
      next_channel();
    }
    // the next tile's inputs come while this one's branch is finished
    tile = next_tile();
    if (tile < a.tiles) fetch(Held<TS, V, Has::TAIL>(a, tile));
    if (!Has::z(a)) continue;
    over_channels(sum, lds1, a.lp, at.pg, [&](int, float s) { return s / (float)a.C; });
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float gz[V], gg[V];
      last_row<Has>(z[k], a, lds, lds1, at.pg, Gates<V>(k), gmw[k], gz, gg);
      if (first + k * CL < a.C && at.any()) {
        at.store(a.gz, k, gz);
        if (Has::g(a)) at.store(a.gg, k, gg);
      }
      next_channel();
    }
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    for (int d = 1; d < (1 << a.lp); d *= 2) {
      weights[k].x += __shfl_xor(weights[k].x, d);
      weights[k].y += __shfl_xor(weights[k].y, d);
    }
    const int c = first + k * CL;
    if ((threadIdx.x & ((1 << a.lp) - 1)) == 0 && c < a.C) a.partial[(int64_t)blockIdx.x * a.C + c] = weights[k];
  }
}

// More channels than registers hold: the tile is read again for each sum, and
// the weight sums are added up in the workspace, each by its own thread.
template <typename TS, int V>
__global__ void __launch_bounds__(kMaxNT) norm_backward_reread(NormArgs a) {
  using Has = Parts<false, false, false, false>;
  __shared__ Joint<3, V> lds;
  __shared__ Joint<1, V> lds1;
  const Draws draws(a);
  float2* partial = a.partial + (int64_t)blockIdx.x * a.C;  // lp = 0: a channel is one thread's
  for (int c = threadIdx.x; c < a.C; c += blockDim.x) partial[c] = make_float2(0.f, 0.f);
  for (uint32_t turn = blockIdx.x; turn < a.turns; turn += gridDim.x) {
    const uint32_t tile = tile_of(a, turn);
    if (tile >= a.tiles) continue;
    const Spot<V> at(a, tile);
    const int n = clamp_count<V>(a.P - at.p);
    auto where = [&](int c) { return (at.b * a.C + c) * a.P + at.p; };
    BwdRow<TS, V> r;
    float acc[3][V], sum[1][V], gx[V], gmw[V];
    const Gates<V> gates(0);
#pragma unroll
    for (int j = 0; j < V; ++j) acc[0][j] = acc[1][j] = acc[2][j] = sum[0][j] = 0.f;
    for (int c = at.cl; c < a.C; c += at.CL) {
      load_row(r, a, where(c), n);
      first_sums<Has>(r, a, a.gn ? weight<TS>(a.w_pre, c) : 0.f, gates, acc);
    }
    over_channels(acc, lds, a.lp, at.pg, [&](int m, float s) { return first_kind(a, m, s); });
    // the second sums of a channel, and with them all that its last row takes
    auto row = [&](int c, float (&to)[1][V], float2* w) {
      float none[3][V];
      load_row(r, a, where(c), n);
      const float w_pre = a.gn ? weight<TS>(a.w_pre, c) : 0.f, wp = a.z ? weight<TS>(a.w_post, c) * weight<TS>(a.scale, c) : 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) none[0][j] = none[1][j] = none[2][j] = 0.f;
      first_sums<Has>(r, a, w_pre, gates, none);
      second_sums<Has>(r, a, draws, at.b * a.C + c, at.p, 0, w_pre, wp, lds, at.pg, gates, gx, gmw, to, w);
    };
    for (int c = at.cl; c < a.C; c += at.CL) {
      float2 w = partial[c];
      row(c, sum, &w);
      partial[c] = w;
      if (!a.z) store<TS, V>(reinterpret_cast<TS*>(a.gx) + where(c), gx, n);
    }
    if (!a.z) continue;
    over_channels(sum, lds1, a.lp, at.pg, [&](int, float s) { return s / (float)a.C; });
    for (int c = at.cl; c < a.C; c += at.CL) {
      float unused[1][V];
      float2 none = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < V; ++j) unused[0][j] = 0.f;
      row(c, unused, &none);
      store<TS, V>(reinterpret_cast<TS*>(a.gx) + where(c), gx, n);
      float gz[V], gg[V];
      last_row<Has>(r.z, a, lds, lds1, at.pg, gates, gmw, gz, gg);
      store<TS, V>(reinterpret_cast<TS*>(a.gz) + where(c), gz, n);
      if (a.gg) store<TS, V>(reinterpret_cast<TS*>(a.gg) + where(c), gg, n);
    }
  }
}

// The weights' gradients: the workgroups' sums, 32 channels a workgroup, every
// 32nd of them a thread.
template <typename TS>
__global__ void __launch_bounds__(1024) norm_weights(NormArgs a) {
  __shared__ double sx[32][33], sy[32][33];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  double x = 0.0, y = 0.0;
  if (c < a.C)
#pragma unroll 8
    for (int i = part; i < a.groups; i += 32) {
      const float2 w = a.partial[(int64_t)i * a.C + c];
      x += w.x;
      y += w.y;
    }
  sx[part][lane] = x;
  sy[part][lane] = y;
  __syncthreads();
  if (part == 0 && c < a.C) {
    for (int i = 1; i < 32; ++i) {
      x += sx[i][lane];
      y += sy[i][lane];
    }
    if (a.gw_pre) st1(reinterpret_cast<TS*>(a.gw_pre) + c, (float)x);
    if (a.gw_post) st1(reinterpret_cast<TS*>(a.gw_post) + c, (float)(y * weight<TS>(a.scale, c)));
    if (a.gscale) st1(reinterpret_cast<TS*>(a.gscale) + c, (float)(y * weight<TS>(a.w_post, c)));
  }
}

// The workgroups that the chip holds at once (16 wavefronts a CU of the registers that
// a tile takes): each goes through its share of the tiles.
int groups_of(uint32_t turns, int NT) {
  const uint32_t most = 256u * (NT >= 1024 ? 1 : 1024 / NT);
  return (int)(turns < most ? turns : most);
}

template <typename TS, typename Has>
void backward_held(const NormArgs& a, const NormShape& s, hipStream_t st) {
  const dim3 grid((unsigned)a.groups), block((unsigned)s.NT);
  constexpr int V = 16 / sizeof(TS);
  const unsigned lds = a.g ? (unsigned)(s.K * s.V * s.NT * 4) : 0u;  // at most 64 KB
#define HY_CASE(v, k) \
  if (s.V == v && s.K == k) hipLaunchKernelGGL((norm_backward<TS, v, k, Has>), grid, block, lds, st, a);
  if constexpr (!Has::TAIL) {
    HY_CASE(1, 1) HY_CASE(1, 4) HY_CASE(1, 8)
  }
  HY_CASE(V, 1) HY_CASE(V, 2) HY_CASE(V, 4)
#undef HY_CASE
}

template <typename TS, bool TAIL>
void backward_parts(const NormArgs& a, const NormShape& s, hipStream_t st) {
  if (!a.z || !a.gn || !a.gx_out)
    backward_held<TS, Parts<false, false, false, TAIL>>(a, s, st);
  else if (a.drop)
    a.g ? backward_held<TS, Parts<true, true, true, TAIL>>(a, s, st) : backward_held<TS, Parts<true, false, true, TAIL>>(a, s, st);
  else
    a.g ? backward_held<TS, Parts<true, true, false, TAIL>>(a, s, st) : backward_held<TS, Parts<true, false, false, TAIL>>(a, s, st);
}

template <typename TS>
hipError_t backward(const NormArgs& a, const NormShape& s, hipStream_t st) {
  if (s.K > 0) {
    a.P % s.V == 0 ? backward_parts<TS, false>(a, s, st) : backward_parts<TS, true>(a, s, st);
  } else {
    const dim3 grid((unsigned)a.groups), block((unsigned)s.NT);
    constexpr int V = 16 / sizeof(TS);
    if (s.V == 1) hipLaunchKernelGGL((norm_backward_reread<TS, 1>), grid, block, 4 * s.NT, st, a);
    else hipLaunchKernelGGL((norm_backward_reread<TS, V>), grid, block, 4 * V * s.NT, st, a);
  }
  hipLaunchKernelGGL((norm_weights<TS>), dim3((unsigned)((a.C + 31) / 32)), dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t norm_backward_workspace_bytes(int64_t B, int64_t C, int64_t P, bool bf16) {
  NormArgs a;
  a.B = B;
  a.C = (int)C;
  a.P = P;
  const NormShape s = norm_shape(C, P, B, bf16, true);
  norm_tiles(a, s);
  return (size_t)groups_of(a.turns, s.NT) * (size_t)C * sizeof(float2);
}

hipError_t launch_norm_backward(const NormArgs& args, hipStream_t st) {
  NormArgs a = args;
  const NormShape s = norm_shape(a.C, a.P, a.B, a.bf16, true);
  norm_tiles(a, s);
  a.groups = groups_of(a.turns, s.NT);
  return a.bf16 ? backward<uint16_t>(a, s, st) : backward<float>(a, s, st);
}

}  // namespace hyenand
