// The 8-bit paged cache (tsd.h: tsd_kv8): internal declarations shared by its
// append, read and attention kernels.
#pragma once

#include "elem.cuh"
#include "internal.h"

namespace tsd {

constexpr float kKv8Least = 0x1p-32f;  // smallest magnitude that a block's scale covers
constexpr float kKv8Most = 0x1p60f;    // largest: scales of one sequence then differ by less than 2^93, so that
                                       // a softmax kept relative to them stays inside fp32's exponents

// A sequence of a call as the kernels see it; see tsd_kv8_batch.
struct Kv8Seq {
  int slot, len, row0, count;  // count rows from row0 are its last tokens
  bool ok;                     // false: rows row0 .. row0 + count - 1 (inside the call's) get NaN
};

__device__ __forceinline__ Kv8Seq kv8_seq(const tsd_kv8& c, const tsd_kv8_batch& b, int i) {
  Kv8Seq s;
  s.slot = b.slots ? __ldg(b.slots + i) : i;
  int r0 = b.starts ? __ldg(b.starts + i) : i, r1 = b.starts ? __ldg(b.starts + i + 1) : i + 1;
  s.ok = s.slot >= 0 && s.slot < c.n_slots && r0 >= 0 && r1 >= r0 && r1 <= b.rows;
  s.len = s.ok ? __ldg(b.lens + s.slot) : 0;
  s.ok = s.ok && s.len >= 0 && s.len <= b.table_width * c.block && r1 - r0 <= s.len;
  if (!s.ok) {
    r0 = min(max(r0, 0), b.rows);
    r1 = min(max(r1, r0), b.rows);
    s.len = 0;
  }
  s.row0 = r0;
  s.count = r1 - r0;
  return s;
}

// Checks shared by the entry points (before any device work).
tsd_status kv8_check(const char* who, const tsd_kv8* c, const tsd_kv8_batch* b);
tsd_status kv8_check_rows(const char* who, const char* what, const void* p, int64_t row, int64_t head);

}  // namespace tsd
