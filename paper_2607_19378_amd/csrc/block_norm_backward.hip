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
// sums up in registers, in fp32 over at most kSumTiles tiles; those of the next ones
// are a row of their own, and a second kernel adds all rows in 64 bits, in order.  So
// a weight's gradient carries the roundings of 64 tiles, whatever the number of points
// (2^30 equal terms of a channel: exact, against 4e-4 off in one fp32 sum a workgroup).
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
  template <typename T>
  __device__ __forceinline__ void write(int what, int from, const T (&x)[N]) const { __builtin_memcpy(place(what, from), x, sizeof x); }
  template <typename T>
  __device__ __forceinline__ void read(int what, int from, T (&x)[N]) const { __builtin_memcpy(x, place(what, from), sizeof x); }
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
    float t[N];
    uint32_t half[N];
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
    float rinv[N], mean[N], t[N];
    uint32_t half[N];
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

constexpr int kSumTiles = 64;

template <typename TS, int V, int K, typename Has>
__global__ void __launch_bounds__(kMaxNT) norm_backward(NormArgs a) {
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
  for (int row = 0; row < a.rows; ++row) {
    for (int left = kSumTiles; left > 0 && tile < a.tiles; --left) {
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
      if ((threadIdx.x & ((1 << a.lp) - 1)) == 0 && c < a.C)
        a.partial[((int64_t)row * gridDim.x + blockIdx.x) * a.C + c] = make_float2(weights[k].x, weights[k].y * a.kept);
      weights[k] = make_float2(0.f, 0.f);
    }
  }
}

// Where a tile of 32 bytes or more of a row does not fit in registers, the tensors
// are read twice in place of once: norm_sums leaves each point's sums over a part of
// the channels, norm_apply joins them and does the rest.  (2 x 2048 x 2048 bf16: 59 us
// against 78 us for tiles of 16 bytes in registers; 2 x 1024 x 4095 bf16: 97 us against 75 us
// for tiles of 32 bytes in registers, so only tiles of 16 bytes are given up.)  gmw is linear in gx_out, gn and
// x, so its sum with t follows from three more sums of the first sweep:
//   sum gmw t = sum w t gx_out + q sum w t gn w_pre - q^3 mean(gn w_pre x) sum w t x,
// w = drop's factor w_post scale.
constexpr int kSplitNT = 256;
constexpr int kSums = 6;  // x x, gn w_pre x, t t, and w t with gx_out, gn w_pre, x

// The raw inputs, t and w of V points of a channel
template <typename TS, int V>
struct SplitRow {
  BwdRow<TS, V> r;
  float t[V];
  uint32_t half[V], drawn[4];
  float w_pre, wp;
  __device__ __forceinline__ SplitRow(const NormArgs& a, const Draws& draws, int64_t b, int c, int64_t p, int n) {
    const int64_t o = (b * a.C + c) * a.P + p;
    r = BwdRow<TS, V>{};
    w_pre = wp = 0.f;
    if (a.gn) {  // without it x has no part in anything, be it an infinity or a NaN
      r.x = load<TS, V>(reinterpret_cast<const TS*>(a.x) + o, n);
      r.gn = load<TS, V>(reinterpret_cast<const TS*>(a.gn) + o, n);
      w_pre = weight<TS>(a.w_pre, c);
    }
    if (a.gx_out) r.gxo = load<TS, V>(reinterpret_cast<const TS*>(a.gx_out) + o, n);
    if (!a.z) return;
    wp = weight<TS>(a.w_post, c) * weight<TS>(a.scale, c) * a.kept;
    r.z = load<TS, V>(reinterpret_cast<const TS*>(a.z) + o, n);
    if (a.g) r.g = load<TS, V>(reinterpret_cast<const TS*>(a.g) + o, n);
    if (a.drop) draws.words<V, false>(b * a.C + c, p, 0, drawn);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      half[j] = a.g ? gate(get(r.g, j)) : kNoGate;
      t[j] = get(r.z, j) * sigmoid_of(half[j]);
    }
  }
};

// A workgroup's part of the channels of a tile.
struct Part {
  uint32_t index;
  int from, to;
  __device__ __forceinline__ Part(const NormArgs& a, uint32_t i) {
    index = i;
    from = i * a.part;
    to = from + a.part < a.C ? from + a.part : a.C;
  }
};

template <typename TS, int V>
__global__ void __launch_bounds__(kSplitNT) norm_sums(NormArgs a) {
  __shared__ Joint<kSums, V> lds;
  const Draws draws(a);
  const int points = V << a.lp;
  for (uint32_t turn = blockIdx.x; turn < a.turns; turn += gridDim.x) {
    const uint32_t tile = tile_of(a, turn);
    if (tile >= a.tiles) continue;
    const Spot<V> at(a, tile);
    const int n = clamp_count<V>(a.P - at.p);
    const Part part(a, blockIdx.y);
    float acc[kSums][V];
#pragma unroll
    for (int m = 0; m < kSums; ++m)
#pragma unroll
      for (int j = 0; j < V; ++j) acc[m][j] = 0.f;
    if (n > 0)
      for (int c = part.from + at.cl; c < part.to; c += at.CL) {
        const SplitRow<TS, V> s(a, draws, at.b, c, at.p, n);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float x = get(s.r.x, j), g = get(s.r.gn, j) * s.w_pre;
          acc[0][j] = fmaf(x, x, acc[0][j]);
          acc[1][j] = fmaf(g, x, acc[1][j]);
          if (a.z) {
            const float wt = !a.drop || draws.keeps(s.drawn, j) ? s.wp * s.t[j] : 0.f;
            acc[2][j] = fmaf(s.t[j], s.t[j], acc[2][j]);
            acc[3][j] = fmaf(wt, get(s.r.gxo, j), acc[3][j]);
            acc[4][j] = fmaf(wt, g, acc[4][j]);
            acc[5][j] = fmaf(wt, x, acc[5][j]);
          }
        }
      }
    over_channels(acc, lds, a.lp, at.pg, [](int m, auto sum, int) { return sum(m); });
    float* to = a.sums + ((int64_t)tile * gridDim.y + part.index) * kSums * points;
    for (int i = threadIdx.x; i < kSums * points; i += kSplitNT) to[i] = lds.all[i / points][i % points];
    __syncthreads();  // read before the next tile's
  }
}

template <typename TS, int V>
__global__ void __launch_bounds__(kSplitNT) norm_apply(NormArgs a) {
  __shared__ float sum[kSums][kMaxLanes * V];
  // of each point: q, q^3 mean(gn w_pre x), r, r^3 mean(gmw t)
  __shared__ float of[4][kMaxLanes * V];
  const Draws draws(a);
  const int points = V << a.lp;
  const Part part(a, blockIdx.y);
  uint32_t turn = blockIdx.x;
  for (int row = 0; row < a.rows; ++row) {
    float2* partial = a.partial + ((int64_t)row * gridDim.x + blockIdx.x) * a.C;
    // a channel's weight sums are kept by the first lane over its points
    for (int c = part.from + (threadIdx.x >> a.lp); c < part.to; c += kSplitNT >> a.lp)
      if ((threadIdx.x & ((1 << a.lp) - 1)) == 0) partial[c] = make_float2(0.f, 0.f);
    for (int left = kSumTiles; left > 0 && turn < a.turns; --left, turn += gridDim.x) {
      const uint32_t tile = tile_of(a, turn);
      if (tile >= a.tiles) continue;
      const Spot<V> at(a, tile);
      const int n = clamp_count<V>(a.P - at.p);
      const float* from = a.sums + (int64_t)tile * gridDim.y * kSums * points;
      for (int i = threadIdx.x; i < kSums * points; i += kSplitNT) {
        float x = 0.f;
#pragma unroll 8
        for (uint32_t k = 0; k < gridDim.y; ++k) x += from[(int64_t)k * kSums * points + i];
        sum[i / points][i % points] = x;
      }
      __syncthreads();
      if ((int)threadIdx.x < points) {
        const int i = threadIdx.x;
        const float C = (float)a.C, q = inverse_rms(sum[0][i], a.C, a.eps_pre), r = inverse_rms(sum[2][i], a.C, a.eps_post);
        const float mean = a.gn ? sum[1][i] / C * q * q * q : 0.f;
        of[0][i] = q;
        of[1][i] = mean;
        of[2][i] = r;
        of[3][i] = (fmaf(q, sum[4][i], sum[3][i]) - mean * sum[5][i]) / C * r * r * r;
      }
      __syncthreads();
      for (int c = part.from + at.cl; c < part.to; c += at.CL) {
        const SplitRow<TS, V> s(a, draws, at.b, c, at.p, n);
        float gx[V], gz[V], gg[V];
        float2 w = make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int i = at.pg * V + j;
          const float q = of[0][i], r = of[2][i], x = get(s.r.x, j), gnq = get(s.r.gn, j) * q;
          gx[j] = fmaf(-x, of[1][i], fmaf(gnq, s.w_pre, get(s.r.gxo, j)));
          if (j < n) w.x = fmaf(gnq, x, w.x);
          if (a.z) {
            const float kept = !a.drop || draws.keeps(s.drawn, j) ? gx[j] : 0.f;
            const float gt = fmaf(-s.t[j], of[3][i], r * (kept * s.wp));
            if (j < n) w.y = fmaf(kept, s.t[j] * r, w.y);
            gz[j] = gt * sigmoid_of(s.half[j]);
            gg[j] = gt * s.t[j] * rest_of(s.half[j]);
          }
        }
        const int64_t o = (at.b * a.C + c) * a.P + at.p;
        store<TS, V>(reinterpret_cast<TS*>(a.gx) + o, gx, n);
        if (a.z) store<TS, V>(reinterpret_cast<TS*>(a.gz) + o, gz, n);
        if (a.g) store<TS, V>(reinterpret_cast<TS*>(a.gg) + o, gg, n);
        for (int d = 1; d < (1 << a.lp); d *= 2) {
          w.x += __shfl_xor(w.x, d);
          w.y += __shfl_xor(w.y, d);
        }
        if (at.pg == 0) partial[c] = make_float2(partial[c].x + w.x, fmaf(w.y, a.kept, partial[c].y));
      }
      __syncthreads();  // `of` is read before the next tile's
    }
  }
}

// The weights' gradients: the rows' sums, 32 channels a workgroup, every 32nd row a
// thread.
template <typename TS>
__global__ void __launch_bounds__(1024) norm_weights(NormArgs a) {
  __shared__ double sx[32][33], sy[32][33];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  double x = 0.0, y = 0.0;
  if (c < a.C)
#pragma unroll 8
    for (int i = part; i < a.all_rows; i += 32) {
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

// The workgroups of the whole chip (16 wavefronts a CU of the registers that a tile takes):
// each goes through its share of the tiles.  Of a split call at most 1024.
int groups_of(const NormArgs& a, const NormShape& s) {
  const uint32_t most = s.K == 0 ? 1024u : 256u * (s.NT >= 1024 ? 1 : 1024 / s.NT);
  return (int)(a.turns < most ? a.turns : most);
}

// A split call's channels in parts: four workgroups a CU with those of all tiles, but few
// enough that the joining of a tile's sums, which each of them does, stays small.
void split_parts(NormArgs& a, const NormShape& s) {
  const int CL = kSplitNT >> s.lp, rows = (a.C + CL - 1) / CL;
  const uint32_t enough = (1024 + a.tiles - 1) / a.tiles, wanted = enough < 32 ? enough : 32;
  const int parts = wanted < (uint32_t)rows ? (int)wanted : rows, each = (rows + parts - 1) / parts;
  a.part = each * CL;
  a.parts = (rows + each - 1) / each;
}

template <auto Kernel>
hipError_t launch(const NormArgs& a, int NT, size_t lds, hipStream_t st) {
  const hipError_t e = raise_lds_limit<Kernel>(128 * 1024);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(Kernel, dim3((unsigned)a.groups), dim3((unsigned)NT), lds, st, a);
  return hipGetLastError();
}

template <typename TS, typename Has>
hipError_t backward_held(const NormArgs& a, const NormShape& s, hipStream_t st) {
  constexpr int V = 16 / sizeof(TS);
  const size_t lds = a.z ? (size_t)s.K * 2 * s.V * s.NT * sizeof(float) : 0;  // at most 128 KB: two channels of eight points a thread
#define HY_CASE(v, k) \
  if (s.V == v && s.K == k) return launch<norm_backward<TS, v, k, Has>>(a, s.NT, lds, st);
  if constexpr (!Has::TAIL) {
    HY_CASE(1, 1) HY_CASE(1, 4)
  }
  HY_CASE(V, 1) HY_CASE(V, 2)
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

template <typename TS, int V>
hipError_t backward_split(const NormArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.groups, (unsigned)a.parts);
  hipLaunchKernelGGL((norm_sums<TS, V>), grid, dim3(kSplitNT), 0, st, a);
  hipLaunchKernelGGL((norm_apply<TS, V>), grid, dim3(kSplitNT), 0, st, a);
  return hipGetLastError();
}

template <typename TS>
hipError_t backward(const NormArgs& a, const NormShape& s, hipStream_t st) {
  hipError_t err;
  if (s.K > 0)
    err = a.P % s.V == 0 ? backward_parts<TS, false>(a, s, st) : backward_parts<TS, true>(a, s, st);
  else
    err = s.V == 1 ? backward_split<TS, 1>(a, st) : backward_split<TS, 16 / sizeof(TS)>(a, st);
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL((norm_weights<TS>), dim3((unsigned)((a.C + 31) / 32)), dim3(1024), 0, st, a);
  return hipGetLastError();
}

// Everything of a call's shape.
NormShape plan(NormArgs& a) {
  const NormShape s = norm_shape(a.C, a.P, a.B, a.bf16, true);
  norm_tiles(a, s, true);
  a.groups = groups_of(a, s);
  const uint32_t each = (a.turns + a.groups - 1) / a.groups;
  a.rows = (int)((each + kSumTiles - 1) / kSumTiles);
  a.all_rows = a.groups * a.rows;  // fewer than 2^26
  a.parts = 0;
  if (s.K == 0) split_parts(a, s);
  return s;
}

size_t partial_bytes(const NormArgs& a) { return (size_t)a.all_rows * (size_t)a.C * sizeof(float2); }

}  // namespace

size_t norm_backward_workspace_bytes(int64_t B, int64_t C, int64_t P, bool bf16) {
  NormArgs a;
  a.B = B;
  a.C = (int)C;
  a.P = P;
  a.bf16 = bf16;
  const NormShape s = plan(a);
  return partial_bytes(a) + (size_t)a.tiles * a.parts * kSums * ((size_t)s.V << s.lp) * sizeof(float);
}

hipError_t launch_norm_backward(const NormArgs& args, hipStream_t st) {
  NormArgs a = args;
  const NormShape s = plan(a);
  a.sums = reinterpret_cast<float*>(reinterpret_cast<char*>(a.partial) + partial_bytes(a));
  return a.bf16 ? backward<uint16_t>(a, s, st) : backward<float>(a, s, st);
}

}  // namespace hyenand
