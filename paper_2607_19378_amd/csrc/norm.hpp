// Internal interface of the norms around a block (block_norm.hip).
#pragma once

#include "kernels.hpp"

namespace hyenand {

// One validated call on [B, C, P] tensors; see include/hyenand.h for the formulas.
struct NormArgs {
  const void *x, *z, *g;            // z null: no branch; g null: no gate.  Backward: x is the forward's x_out
  const void *w_post, *scale, *w_pre;  // scale null: 1
  const uint64_t* rng;              // {seed, offset} on the device, read where drop > 0
  void *x_out, *n;                  // n null: no norm behind the sum
  int64_t B, P;
  int C;
  float eps_post, eps_pre;
  uint32_t drop;                    // a point is dropped where its 16 random bits are below this
  float kept;                       // what a kept one is multiplied by, 65536 / (65536 - drop); 1 without dropout
  bool bf16;
  // backward: null where there is none
  const void *gx_out, *gn;
  void *gx, *gz, *gg, *gw_post, *gscale, *gw_pre;
  float2* partial;                  // [rows, groups, C] a workgroup's sums for the weights, of 64 tiles a row
  // set by the launchers
  int lp;                           // log2 of the lanes over a channel's positions
  uint32_t tiles, row_tiles;        // tiles of points in all, and of a sample
  uint32_t log_run;                 // log2 of the consecutive tiles of an XCD's turn
  uint32_t turns;                   // tiles, and the turns that fall behind the last one
  int groups;                       // workgroups of the backward (of a part of the channels)
  int rows, all_rows;               // rows of sums of each workgroup, and of all
  int part, parts;                  // split calls: channels of a part, and parts
  float* sums;                      // [tiles, parts, sums of a point, points]
};

constexpr int64_t kMaxNormPoints = int64_t(1) << 33;  // B * P: tiles are counted in 32 bits

size_t norm_backward_workspace_bytes(int64_t B, int64_t C, int64_t P, bool bf16);
hipError_t launch_norm(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s);

}  // namespace hyenand
