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
  // even rows: all row arrays stand equally off a multiple of eight elements
  int base, stride;  // that, of row 0, and how it grows from row to row, mod 8
  int depth, slot;   // rows on their way per thread group, bytes of one
};

// XT, YT: types of the residual stream and of the block's output.
template <int XT, int YT>
cudaError_t norm_launch(const NormArgs& a, bool even, int sms, cudaStream_t s);

}  // namespace tsd
