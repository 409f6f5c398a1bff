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
#include <mutex>

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

// What is left of the sums of the first kind: q = 1 / rms(x), q^3 mean(gn w_pre x), r = 1 / rms(t)
template <typename F>
__device__ __forceinline__ float first_kind(const NormArgs& a, int m, F sum) {
  if (m == 2) return inverse_rms(sum(2), a.C, a.eps_post);
  const float q = inverse_rms(sum(0), a.C, a.eps_pre);
  return m == 0 ? q : sum(1) / (float)a.C * q * q * q;
}

// The gates (see gate()) and t of a channel's points, from the first sums on in LDS:
// in registers, they would push the tile out of them.  A thread reads what it wrote.
extern __shared__ float branch_lds[];
template <int V>
struct Branch {
  static constexpr int N = V < 4 ? V : 4;  // points at a time
  static constexpr int kWords = 2 * V;     // of a channel and thread
  float* at;
  __device__ __forceinline__ explicit Branch(int k) : at(branch_lds + ((size_t)k * kWords * blockDim.x + N * threadIdx.x)) {}
  __device__ __forceinline__ void write(int what, int from, const float (&x)[N]) const { __builtin_memcpy(place(what, from), x, sizeof x); }
  __device__ __forceinline__ void read(int what, int from, float (&x)[N]) const { __builtin_memcpy(x, place(what, from), sizeof x); }
  __device__ __forceinline__ float* place(int what, int from) const {
    return reinterpret_cast<float*>(__builtin_assume_aligned(at + (size_t)(what * V + from) * blockDim.x, N * 4));
  }
};
constexpr int kT = 0, kGate = 1;

// t and the gates of V points, and the sums of the first kind: squares of x, gn w_pre x,
// squares of t
template <typename Has, typename TS, int V>
__device__ __forceinline__ void first_sums(const BwdRow<TS, V>& r, const NormArgs& a, float w_pre, const Branch<V>& branch,
                                           float (&acc)[3][V]) {
  constexpr int N = Branch<V>::N;
#pragma unroll
  for (int from = 0; from < V; from += N) {
    float half[N], t[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int j = from + i;
      if (Has::gn(a)) {
        const float x = get(r.x, j);
        acc[0][j] = fmaf(x, x, acc[0][j]);
        acc[1][j] = fmaf(get(r.gn, j) * w_pre, x, acc[1][j]);
      }
      if (Has::z(a)) {
        t[i] = get(r.z, j);
        if (Has::g(a)) {
          half[i] = gate(get(r.g, j));
          t[i] *= sigmoid_of(half[i]);
        }
        acc[2][j] = fmaf(t[i], t[i], acc[2][j]);
      }
    }
    if (Has::z(a)) branch.write(kT, from, t);
    if (Has::z(a) && Has::g(a)) branch.write(kGate, from, half);
    next_channel();
    __builtin_amdgcn_sched_barrier(0);
  }
}

// gx of V points; what reaches the branch's norm (gmw), and its sum with t (the
// second kind); wp = w_post scale / (1 - p).  Points that are not the lane's own come
// with zeros for gn and gx_out and add nothing to the weights' sums (weights->y without
// its 1 / (1 - p)).
template <typename Has, typename TS, int V>
__device__ __forceinline__ void second_sums(const BwdRow<TS, V>& r, const NormArgs& a, const Draws& draws, int64_t row,
                                            int64_t p, int shift, float w_pre, float wp, const Joint<3, V>& lds, int pg,
                                            const Branch<V>& branch, float (&gx)[V], float (&gmw)[V], float (&sum)[1][V],
                                            float2* weights) {
  constexpr int N = Branch<V>::N;
  uint32_t drawn[4];
  if (Has::z(a) && Has::drop(a)) draws.words<V, Has::TAIL>(row, p, shift, drawn);
#pragma unroll
  for (int from = 0; from < V; from += N) {
    float q[N], mean[N], rinv[N], t[N];
    if (Has::z(a)) branch.read(kT, from, t);
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
        const float gnq = get(r.gn, j) * q[i], x = get(r.x, j);
        gx[j] = fmaf(-x, mean[i], fmaf(gnq, w_pre, gx[j]));
        weights->x = fmaf(gnq, x, weights->x);
      }
      if (Has::z(a)) {
        const float kept = !Has::drop(a) || draws.keeps(drawn, j) ? gx[j] : 0.f;
        gmw[j] = kept * wp;
        sum[0][j] = fmaf(gmw[j], t[i], sum[0][j]);
        weights->y = fmaf(kept, t[i] * rinv[i], weights->y);
      }
    }
    // here, or the sums are put off to the next tile, with all that they take
    asm volatile("" : "+v"(weights->x), "+v"(weights->y));
    next_channel();
  }
}

// gz and gg of V points; lds1 holds r^3 mean(gmw t)
template <typename Has, int V>
__device__ __forceinline__ void last_row(const NormArgs& a, const Joint<3, V>& lds, const Joint<1, V>& lds1, int pg,
                                         const Branch<V>& branch, const float (&gmw)[V], float (&gz)[V], float (&gg)[V]) {
  constexpr int N = Branch<V>::N;
#pragma unroll
  for (int from = 0; from < V; from += N) {
    float rinv[N], mean[N], half[N], t[N];
    branch.read(kT, from, t);
    if (Has::g(a)) branch.read(kGate, from, half);
    read_sums(lds, 2, pg, rinv, from);
    read_sums(lds1, 0, pg, mean, from);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int j = from + i;
      const float gt = fmaf(-t[i], mean[i], rinv[i] * gmw[j]);
      gz[j] = Has::g(a) ? gt * sigmoid_of(half[i]) : gt;
      gg[j] = Has::g(a) ? gt * t[i] * rest_of(half[i]) : 0.f;
    }
    next_channel();
  }
}

// r^3 mean(gmw t)
template <int V>
__device__ __forceinline__ float second_kind(const NormArgs& a, const Joint<3, V>& lds, int point, float sum) {
  const float r = lds.all[2][point];
  return sum / (float)a.C * r * r * r;
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
    wp[k] = Has::z(a) && c < a.C ? weight<TS>(a.w_post, c) * weight<TS>(a.scale, c) * a.kept : 0.f;
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
  // the inputs of a tile: of the branch, and of the stream
  auto fetch_branch = [&](const Held<TS, V, Has::TAIL>& at) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (first + k * CL < a.C && at.any()) {
        if (Has::z(a)) r[k].z = at.load(a.z, k);
        if (Has::g(a)) r[k].g = at.load(a.g, k);
      } else {
        if (Has::z(a)) r[k].z = Raw<TS, V>{};
        if (Has::g(a)) r[k].g = Raw<TS, V>{};
      }
    }
  };
  auto fetch_stream = [&](const Held<TS, V, Has::TAIL>& at) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (first + k * CL < a.C && at.any()) {
        r[k].x = at.load(a.x, k);
        if (Has::gn(a)) r[k].gn = at.load_own(a.gn, k);
        if (Has::gx_out(a)) r[k].gxo = at.load_own(a.gx_out, k);
      } else {
        r[k].x = Raw<TS, V>{};
        if (Has::gn(a)) r[k].gn = Raw<TS, V>{};
        if (Has::gx_out(a)) r[k].gxo = Raw<TS, V>{};
      }
    }
  };
  uint32_t tile = next_tile();
  if (tile < a.tiles) {
    const Held<TS, V, Has::TAIL> at(a, tile);
    fetch_branch(at);
    fetch_stream(at);
  }
  while (tile < a.tiles) {
    const Held<TS, V, Has::TAIL> at(a, tile);
    float acc[3][V], sum[1][V], gmw[K][V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[0][j] = acc[1][j] = acc[2][j] = sum[0][j] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) first_sums<Has>(r[k], a, w_pre[k], Branch<V>(k), acc);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      keep_packed(r[k].x);
      keep_packed(r[k].gn);
      keep_packed(r[k].gxo);
    }
    // the next tile's inputs come as soon as this one's have been used
    const uint32_t next = next_tile();
    if (next < a.tiles) fetch_branch(Held<TS, V, Has::TAIL>(a, next));
    over_channels(acc, lds, a.lp, at.pg, [&](int m, auto sum, int) { return first_kind(a, m, sum); });
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float gx[V];
      second_sums<Has>(r[k], a, draws, at.b * a.C + first + k * CL, at.p, at.shift, w_pre[k], wp[k], lds, at.pg, Branch<V>(k),
                       gx, gmw[k], sum, &weights[k]);
      if (first + k * CL < a.C && at.any()) at.store(a.gx, k, gx);
      next_channel();
    }
    if (next < a.tiles) fetch_stream(Held<TS, V, Has::TAIL>(a, next));
    tile = next;
    if (!Has::z(a)) continue;
    over_channels(sum, lds1, a.lp, at.pg, [&](int, auto sum, int point) { return second_kind(a, lds, point, sum(0)); });
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float gz[V], gg[V];
      last_row<Has>(a, lds, lds1, at.pg, Branch<V>(k), gmw[k], gz, gg);
      // the next inputs are there by now, or else they would be waited for behind these
      // stores, and with them
      if (k == 0) __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
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
    if ((threadIdx.x & ((1 << a.lp) - 1)) == 0 && c < a.C) a.partial[(int64_t)blockIdx.x * a.C + c] = make_float2(weights[k].x, weights[k].y * a.kept);
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
    const Branch<V> branch(0);
#pragma unroll
    for (int j = 0; j < V; ++j) acc[0][j] = acc[1][j] = acc[2][j] = sum[0][j] = 0.f;
    for (int c = at.cl; c < a.C; c += at.CL) {
      load_row(r, a, where(c), n);
      first_sums<Has>(r, a, a.gn ? weight<TS>(a.w_pre, c) : 0.f, branch, acc);
    }
    over_channels(acc, lds, a.lp, at.pg, [&](int m, auto sum, int) { return first_kind(a, m, sum); });
    // the second sums of a channel, and with them all that its last row takes
    auto row = [&](int c, float (&to)[1][V], float2* w) {
      float none[3][V];
      load_row(r, a, where(c), n);
      const float w_pre = a.gn ? weight<TS>(a.w_pre, c) : 0.f, wp = a.z ? weight<TS>(a.w_post, c) * weight<TS>(a.scale, c) * a.kept : 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) none[0][j] = none[1][j] = none[2][j] = 0.f;
      first_sums<Has>(r, a, w_pre, branch, none);
      second_sums<Has>(r, a, draws, at.b * a.C + c, at.p, 0, w_pre, wp, lds, at.pg, branch, gx, gmw, to, w);
    };
    for (int c = at.cl; c < a.C; c += at.CL) {
      float2 w = make_float2(0.f, 0.f);
      row(c, sum, &w);
      partial[c] = make_float2(partial[c].x + w.x, fmaf(w.y, a.kept, partial[c].y));
      if (!a.z) store<TS, V>(reinterpret_cast<TS*>(a.gx) + where(c), gx, n);
    }
    if (!a.z) continue;
    over_channels(sum, lds1, a.lp, at.pg, [&](int, auto sum, int point) { return second_kind(a, lds, point, sum(0)); });
    for (int c = at.cl; c < a.C; c += at.CL) {
      float unused[1][V];
      float2 none = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < V; ++j) unused[0][j] = 0.f;
      row(c, unused, &none);
      store<TS, V>(reinterpret_cast<TS*>(a.gx) + where(c), gx, n);
      float gz[V], gg[V];
      last_row<Has>(a, lds, lds1, at.pg, branch, gmw, gz, gg);
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

// A kernel's dynamic LDS limit is raised beyond the default 64 KB once.
template <auto Kernel>
hipError_t launch(const NormArgs& a, int NT, size_t lds, hipStream_t st) {
  static std::once_flag once;
  static hipError_t attr = hipSuccess;
  std::call_once(once, [] {
    attr = hipFuncSetAttribute(reinterpret_cast<const void*>(Kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024);
  });
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL(Kernel, dim3((unsigned)a.groups), dim3((unsigned)NT), lds, st, a);
  return hipGetLastError();
}

template <typename TS, typename Has>
hipError_t backward_held(const NormArgs& a, const NormShape& s, hipStream_t st) {
  constexpr int V = 16 / sizeof(TS);
  const size_t lds = a.z ? (size_t)s.K * 2 * s.V * s.NT * sizeof(float) : 0;  // at most 128 KB (norm_threads)
#define HY_CASE(v, k) \
  if (s.V == v && s.K == k) return launch<norm_backward<TS, v, k, Has>>(a, s.NT, lds, st);
  if constexpr (!Has::TAIL) {
    HY_CASE(1, 1) HY_CASE(1, 4)
  }
  HY_CASE(V, 1) HY_CASE(V, 2) HY_CASE(V, 4)
#undef HY_CASE
  return hipErrorInvalidValue;
}

template <typename TS, bool TAIL>
hipError_t backward_parts(const NormArgs& a, const NormShape& s, hipStream_t st) {
  if (!a.z || !a.gn || !a.gx_out) return backward_held<TS, Parts<false, false, false, TAIL>>(a, s, st);
  if (a.drop)
    return a.g ? backward_held<TS, Parts<true, true, true, TAIL>>(a, s, st)
               : backward_held<TS, Parts<true, false, true, TAIL>>(a, s, st);
  return a.g ? backward_held<TS, Parts<true, true, false, TAIL>>(a, s, st)
             : backward_held<TS, Parts<true, false, false, TAIL>>(a, s, st);
}

template <typename TS>
hipError_t backward(const NormArgs& a, const NormShape& s, hipStream_t st) {
  constexpr int V = 16 / sizeof(TS);
  const size_t lds = (size_t)2 * s.V * s.NT * sizeof(float);
  hipError_t err;
  if (s.K > 0)
    err = a.P % s.V == 0 ? backward_parts<TS, false>(a, s, st) : backward_parts<TS, true>(a, s, st);
  else
    err = s.V == 1 ? launch<norm_backward_reread<TS, 1>>(a, s.NT, lds, st) : launch<norm_backward_reread<TS, V>>(a, s.NT, lds, st);
  if (err != hipSuccess) return err;
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
