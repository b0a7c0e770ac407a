// Attention over an encoder's states: what its kernels share (tsd.h: tsd_cross_attend).
#pragma once

#include "elem.cuh"
#include "internal.h"
#include "tc_common.cuh"

namespace tsd {

// Two weights go into the values' product as the sum of two pairs of 16-bit floats, `first`, a little less than they, and what is left: within
// 2^-16 of them.  Neither is negative or (but of a weight of 0) 0: that would make a value's infinity a NaN.
// bf16: cut off, and 2^-20 more is left; fp16: 31/32 rounded.  (The cut part's numbers from its pair, not by masks: 195 us where
// those take 200, 6 x 1100 over 9000.)
template <bool BF16>
__device__ __forceinline__ void weight_parts(float a, float b, uint32_t& first, uint32_t& rest) {
  const float scale = BF16 ? 1.f + 0x1p-20f : 31.f / 32;
  const uint64_t w = tc::pair_of(a, b), scaled = tc::mul2(w, tc::pair_of(scale, scale));
  float x, y;
  tc::unpair(scaled, x, y);
  first = BF16 ? __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632) : narrow2<BF16>(x, y);
  tc::unpair(tc::fma2(tc::pair_of(wide16<BF16>(first & 0xffffu), wide16<BF16>(first >> 16)), tc::pair_of(-1.f, -1.f), BF16 ? scaled : w), x, y);
  rest = narrow2<BF16>(x, y);
}

struct CrossAttend {
  tsd_states s;
  tsd_cross_batch b;
  const uint16_t* q;  // 16-bit floats of the states' dtype
  uint16_t* out;
  int64_t q_row, q_head, out_row, out_head;
  int heads, group;
  float scale;
};

// A sequence of a call as the kernels see it; see tsd_cross_batch.
struct CrossSeq {
  int source, len, row0, count;
  bool ok;  // false: rows row0 .. row0 + count - 1 (inside the call's) get NaN
};

__device__ __forceinline__ CrossSeq cross_seq(const tsd_states& s, const tsd_cross_batch& b, int i) {
  CrossSeq q;
  q.source = b.sources ? __ldg(b.sources + i) : i;
  int r0 = b.starts ? __ldg(b.starts + i) : i, r1 = b.starts ? __ldg(b.starts + i + 1) : i + 1;
  q.ok = q.source >= 0 && q.source < s.n_sources && r0 >= 0 && r1 >= r0 && r1 <= b.rows;
  q.len = q.ok ? (s.lens ? __ldg(s.lens + q.source) : s.frames) : 0;
  if (q.len < 0 || q.len > s.frames) q.ok = false, q.len = 0;
  r0 = min(max(r0, 0), b.rows);
  r1 = min(max(r1, r0), b.rows);
  q.row0 = r0;
  q.count = r1 - r0;
  return q;
}

// Few rows per key head (cross_rows.cu): row tiles of 16, the frames of one over a cluster.
struct CrossRowsPlan {
  int mtiles = 1, splits = 1, warps = 4;  // of a CTA
};
CrossRowsPlan cross_rows_plan(const tsd_states& s, const tsd_cross_batch& b, int heads, int sms);
cudaError_t cross_rows_launch(const CrossAttend& a, const CrossRowsPlan& p, cudaStream_t s);

// Many (cross_tiles.cu); false: they are few.  bytes of workspace.
struct CrossTilesPlan {
  int ctas = 1;
  int64_t bytes = 0;
};
bool cross_tiles_plan(const tsd_states& s, const tsd_cross_batch& b, int heads, int sms, CrossTilesPlan* p);
cudaError_t cross_tiles_launch(const CrossAttend& a, const CrossTilesPlan& p, void* workspace, cudaStream_t s);

}  // namespace tsd
