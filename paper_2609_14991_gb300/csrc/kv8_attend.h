// Attention over the 8-bit paged cache: what its kernels share.
#pragma once

#include "kv8.h"

namespace tsd {

struct Kv8Attend {
  tsd_kv8 c;
  tsd_kv8_batch b;
  const uint16_t* q;  // 16-bit floats of the cache's dtype
  uint16_t* out;
  int64_t q_row, q_head, out_row, out_head;
  int heads, group, window, sinks;
  float scale;
  float* part;      // [splits][rows][heads][dim] partial results
  float2* part_ml;  // [splits][rows][heads] their maximum and sum
};

// A pair of integers placed (offset by 128) in the mantissas of two fp16 1024s: their values.
__device__ __forceinline__ uint32_t int_half2(uint32_t x) {
  const uint32_t off = 0xe480e480u;  // -1152, twice
  uint32_t r;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(off));
  return r;
}

// Few rows per key head (kv8_rows.cu): row tiles of 16 x mw, the keys over `splits` CTAs.
struct Kv8RowsPlan {
  int mw = 1, mtiles = 1, splits = 1;
  int64_t bytes = 0;  // workspace
};
Kv8RowsPlan kv8_rows_plan(const tsd_kv8& c, const tsd_kv8_batch& b, int heads, int window, int sinks, int sms);
cudaError_t kv8_rows_launch(Kv8Attend a, const Kv8RowsPlan& p, void* workspace, cudaStream_t s);

}  // namespace tsd
