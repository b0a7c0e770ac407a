// Attention over the 8-bit paged cache: what its kernels share.
#pragma once

#include "kv8.h"
#include "kv8_keys.h"

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

template <bool BF16>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
  if (BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ float lg2_approx(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The power of two that brings a row's largest magnitude into [2^14, 2^15) (2^126 at
// most); fine: false for NaN and infinity.
struct QueryScale {
  float f;
  bool fine;
};
__device__ __forceinline__ QueryScale query_scale(float top) {
  const int ex = (int)(__float_as_uint(top) >> 23);
  const bool fine = ex < 255;
  return {__uint_as_float((uint32_t)(fine ? min(127 + 126, 127 + 14 - (ex - 127)) : 127) << 23), fine};
}

// Few rows per key head (kv8_rows.cu): row tiles of 8, 16 (two or four warps) or 32, the
// keys over `splits` CTAs.
struct Kv8RowsPlan {
  int rows = 8, warps = 4, mtiles = 1, splits = 1;
  int64_t bytes = 0;  // workspace
};
Kv8RowsPlan kv8_rows_plan(const tsd_kv8& c, const tsd_kv8_batch& b, int heads, int window, int sinks, int sms);
cudaError_t kv8_rows_launch(const Kv8Attend& a, const Kv8RowsPlan& p, cudaStream_t s);

// Many (kv8_tiles.cu): row tiles of 256.  false: kv8_rows.cu is the better one.
struct Kv8TilesPlan {
  int mtiles = 0, splits = 1;
  int64_t bytes = 0;
};
bool kv8_tiles_plan(const tsd_kv8& c, const tsd_kv8_batch& b, int heads, int window, int sinks, int sms, Kv8TilesPlan* p);
cudaError_t kv8_tiles_launch(const Kv8Attend& a, const Kv8TilesPlan& p, cudaStream_t s);

// Joins the splits' partial results (kv8_rows.cu).
cudaError_t kv8_join_launch(const Kv8Attend& a, int splits, cudaStream_t s);

}  // namespace tsd
