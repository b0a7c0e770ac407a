// Norms around a block: what the entry point hands to the kernels.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "tsd.h"

namespace tsd {

constexpr int kMaxWidth = 16384;

struct NormArgs {
  int n, d;
  const void *x, *y, *gate;
  void *r, *h;
  int64_t x_row, y_row, gate_row, r_row, h_row;
  float scale;
  tsd_norm post, norm;
  int base, stride;  // rows in groups of eight: how far row 0 begins into one, and how it grows from row to row, mod 8
  int depth, slot;   // rows on their way per thread group, bytes of one
};

// How rows stand in memory: each array anywhere; in groups of eight elements that begin at a multiple of eight, the row's first element
// equally far into its first group in all row arrays; or in whole groups, weights too.
enum class NormHow { kApart, kShifted, kWhole };

// XT, YT: types of the residual stream and of the block's output.
template <int XT, int YT>
cudaError_t norm_launch(const NormArgs& a, NormHow how, int sms, cudaStream_t s);

}  // namespace tsd
