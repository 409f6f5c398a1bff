// Accesses of a few consecutive elements of a row that may begin and end anywhere.
#pragma once

#include "kernels.hpp"

namespace hyenand {
namespace rows {

// V = 8, 4 or 1 consecutive elements as they lie in memory.  A row begins wherever
// the one before it ends, so that an access is aligned to its element only;
// gfx950 takes 16-byte accesses at such addresses.
template <typename TS, int V = 8>
struct Raw {
  uint32_t w[V * sizeof(TS) >= 4 ? V * sizeof(TS) / 4 : 1];
};

// n <= V elements from p on, zeros behind them
template <typename TS, int V = 8>
__device__ __forceinline__ Raw<TS, V> load(const TS* p, int n) {
  Raw<TS, V> r;
  if constexpr (V == 1) {
    r.w[0] = n > 0 ? __float_as_uint(ld1(p)) : 0u;
  } else if (n >= V) {
    __builtin_memcpy(&r, p, sizeof r);
  } else {
    if constexpr (sizeof(TS) == 2) {
#pragma unroll
      for (int j = 0; j < V / 2; ++j)
        r.w[j] = (2 * j < n ? (uint32_t)p[2 * j] : 0u) | (2 * j + 1 < n ? (uint32_t)p[2 * j + 1] << 16 : 0u);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) r.w[j] = j < n ? __float_as_uint(p[j]) : 0u;
    }
  }
  return r;
}

template <typename TS, int V>
__device__ __forceinline__ float get(const Raw<TS, V>& r, int j) {
  if constexpr (sizeof(TS) == 2 && V > 1)
    return __uint_as_float((j & 1) ? r.w[j / 2] & 0xffff0000u : r.w[j / 2] << 16);
  else
    return __uint_as_float(r.w[j]);
}

// the first n <= V of y to p on
template <typename TS, int V>
__device__ __forceinline__ void store(TS* p, const float (&y)[V], int n) {
  if (V > 1 && n >= V) {
    Raw<TS, V> r;
    if constexpr (sizeof(TS) == 2) {
#pragma unroll
      for (int j = 0; j < V / 2; ++j) r.w[j] = bf16_pack(y[2 * j], y[2 * j + 1]);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) r.w[j] = __float_as_uint(y[j]);
    }
    __builtin_memcpy(p, &r, sizeof r);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j < n) st1(p + j, y[j]);
  }
}

// V elements at a byte offset from an address that is the same for all lanes
template <typename TS, int V>
__device__ __forceinline__ Raw<TS, V> load_at(const void* base, uint32_t off) {
  Raw<TS, V> r;
  if constexpr (V == 1)
    r.w[0] = __float_as_uint(ld1(reinterpret_cast<const TS*>(reinterpret_cast<const char*>(base) + off)));
  else
    __builtin_memcpy(&r, reinterpret_cast<const char*>(base) + off, sizeof r);
  return r;
}
template <typename TS, int V>
__device__ __forceinline__ void store_at(void* base, uint32_t off, const float (&y)[V]) {
  store<TS, V>(reinterpret_cast<TS*>(reinterpret_cast<char*>(base) + off), y, V);
}

// Values that come from x are computed from it again after this, instead of being
// kept beside it: a row of bf16 takes half the registers of what it unpacks to.
template <typename TS, int V>
__device__ __forceinline__ void keep_packed(Raw<TS, V>& x) {
#pragma unroll
  for (uint32_t& w : x.w) asm volatile("" : "+v"(w));
}

template <int V>
__device__ __forceinline__ int clamp_count(int64_t n) {
  return n >= V ? V : (n > 0 ? (int)n : 0);
}

}  // namespace rows
}  // namespace hyenand
