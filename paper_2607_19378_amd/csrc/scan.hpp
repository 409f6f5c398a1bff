// Internal interface of the gated linear recurrence (scan.hip, scan_backward.hip).
#pragma once

#include "kernels.hpp"

namespace hyenand {

constexpr int kScanV = 8;                // consecutive positions of a lane
constexpr int kScanTile = 64 * kScanV;   // positions of a wavefront's tile, and between two kept states

// One validated call.  R = B * C rows of L positions; row r belongs to sample r / C and channel r % C.
struct ScanArgs {
  const void *x1, *x2, *v, *la, *D;
  const float* h0;       // [R] or null (zeros)
  const int64_t* len;    // [B] or null (L)
  void* y;
  float* h_last;         // [R] or null
  float* states;         // [R, nst]: written by the forward if not null, read by the backward
  int64_t R, L, nst;
  int C;
  bool bf16;
  // backward
  const void* gy;
  const float* gh_last;  // [R] or null (zeros)
  void *gx1, *gx2, *gv, *gla, *gD;
  float* gh0;            // [R] or null
  double* partial;       // [R * nseg] sums of gz u, then added over b and segments into gD
  // set by the launchers: where rows are split, into nseg segments of one tile a wavefront
  int nseg;
  uint64_t* links;       // 2 words a segment (see scan_device.hpp), then each row's next segment to take
};

constexpr int64_t kLinkStride = 16;  // words between the rows' counters: a cache line each
constexpr int kLinkedWaves = 8;  // wavefronts, and tiles, of a segment

// How a call's rows are spread: lanes of a row (under 64: the row is one tile of lanes * kScanV positions), wavefronts
// of a row, segments of a row (1: the wavefronts go through the whole row).
struct ScanShape {
  int lanes, waves, nseg;
};
ScanShape scan_shape(int64_t R, int64_t L);
size_t scan_link_bytes(const ScanShape& p, int64_t R);  // workspace of a split call's segments
hipError_t launch_scan_links(const ScanArgs& a, hipStream_t s);  // clears them
size_t scan_workspace_bytes(int64_t R, int64_t L, bool backward);
hipError_t launch_scan(const ScanArgs& a, void* ws, hipStream_t s);
hipError_t launch_scan_backward(const ScanArgs& a, void* ws, hipStream_t s);

struct ScanStepArgs {
  const void *x1, *x2, *v, *la, *D;
  const int64_t* slots;  // [B] or null
  float* state;          // [nslots, C]
  void* y;
  int64_t B, nslots;
  int C;
  bool bf16;
};
hipError_t launch_scan_step(const ScanStepArgs& a, hipStream_t s);

}  // namespace hyenand
