// Attention over an encoder's states: what its kernels share (tsd.h: tsd_cross_attend).
#pragma once

#include "elem.cuh"
#include "internal.h"

namespace tsd {

// A weight goes into the values' product as the sum of two 16-bit floats, hi = round(w f) and round(w - hi): half a step of the
// second is at most 2^-16 w.  f is below 1, so neither is negative or (a rest of 0) makes a value's infinity a NaN.
template <bool BF16>
constexpr float kFirstPart = BF16 ? 255.f / 256 : 31.f / 32;

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
