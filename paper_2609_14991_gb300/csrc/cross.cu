// Attention over an encoder's states: the entry point (tsd.h: tsd_cross_attend).
#include <cmath>

#include "cross.h"
#include "launch.h"

using namespace tsd;

namespace {

tsd_status check_rows(const char* who, const char* what, const void* p, int64_t row, int64_t head) {
  if (!p) return fail(TSD_EINVAL, "%s: NULL %s", who, what);
  if (reinterpret_cast<uintptr_t>(p) % 16 || row % 8 || head % 8)
    return fail(TSD_EINVAL, "%s: %s must be 16-byte aligned with strides a multiple of 8 elements", who, what);
  if (row < 0 || head < 0 || row > (1ll << 36) || head > (1ll << 36)) return fail(TSD_EINVAL, "%s: %s strides out of range", who, what);
  return TSD_OK;
}

// What can be said of a call without its queries.
tsd_status call_check(const char* who, const tsd_states* states, const tsd_cross_batch* batch, int32_t heads) {
  if (!states || !batch) return fail(TSD_EINVAL, "%s: NULL argument", who);
  const tsd_states& s = *states;
  const tsd_cross_batch& b = *batch;
  if (s.dtype != TSD_BF16 && s.dtype != TSD_F16) return fail(TSD_EINVAL, "%s: dtype %d is not bf16 or fp16", who, s.dtype);
  if (s.dim != 64 && s.dim != 128) return fail(TSD_EINVAL, "%s: dim=%d is not 64 or 128", who, s.dim);
  if (s.kv_heads < 1 || s.kv_heads > 1024) return fail(TSD_EINVAL, "%s: kv_heads=%d outside [1, 1024]", who, s.kv_heads);
  if (s.n_sources < 1) return fail(TSD_EINVAL, "%s: n_sources=%d must be positive", who, s.n_sources);
  if (s.frames < 1 || s.frames > (1 << 30)) return fail(TSD_EINVAL, "%s: frames=%d outside [1, 2^30]", who, s.frames);
  if (tsd_status st = check_rows(who, "k", s.k, s.k_frame, s.k_head)) return st;
  if (tsd_status st = check_rows(who, "v", s.v, s.v_frame, s.v_head)) return st;
  if (tsd_status st = check_rows(who, "k", s.k, s.k_source, 0)) return st;
  if (tsd_status st = check_rows(who, "v", s.v, s.v_source, 0)) return st;
  if (heads < 1 || heads > 1024 || heads % s.kv_heads || heads / s.kv_heads > 64)
    return fail(TSD_EINVAL, "%s: heads=%d must be 1..64 times kv_heads=%d, at most 1024", who, heads, s.kv_heads);
  if (b.n < 1 || b.n > 65535) return fail(TSD_EINVAL, "%s: n=%d outside [1, 65535]", who, b.n);
  if (b.rows < 1 || b.rows > (1 << 22)) return fail(TSD_EINVAL, "%s: rows=%d outside [1, 2^22]", who, b.rows);
  if (!b.starts && b.rows != b.n) return fail(TSD_EINVAL, "%s: starts is NULL: rows=%d must be n=%d", who, b.rows, b.n);
  if (!b.sources && b.n > s.n_sources) return fail(TSD_EINVAL, "%s: sources is NULL: n=%d is above n_sources=%d", who, b.n, s.n_sources);
  if (b.max_rows < 0) return fail(TSD_EINVAL, "%s: negative max_rows", who);
  return TSD_OK;
}

}  // namespace

extern "C" tsd_status tsd_cross_attend_workspace(const tsd_states* states, const tsd_cross_batch* batch, int32_t heads, int64_t* bytes) {
  clear_error();
  if (!bytes) return fail(TSD_EINVAL, "tsd_cross_attend_workspace: NULL argument");
  if (tsd_status st = call_check("tsd_cross_attend_workspace", states, batch, heads)) return st;
  int sms = 0;
  TSD_CUDA(device_sms(&sms));
  CrossTilesPlan p;
  *bytes = cross_tiles_plan(*states, *batch, heads, sms, &p) ? p.bytes : 0;
  return TSD_OK;
}

extern "C" tsd_status tsd_cross_attend(const tsd_states* states, const tsd_cross_batch* batch, int32_t heads, const void* q, int64_t q_row,
                                       int64_t q_head, float scale, void* out, int64_t out_row, int64_t out_head, void* workspace, int64_t workspace_bytes,
                                       void* cuda_stream) {
  clear_error();
  const char* who = "tsd_cross_attend";
  if (tsd_status st = call_check(who, states, batch, heads)) return st;
  const tsd_states& s = *states;
  const tsd_cross_batch& b = *batch;
  if (!std::isfinite(scale)) return fail(TSD_EINVAL, "tsd_cross_attend: scale is not finite");
  if (tsd_status st = check_rows(who, "q", q, q_row, q_head)) return st;
  if (tsd_status st = check_rows(who, "out", out, out_row, out_head)) return st;
  if ((b.rows > 1 && out_row < s.dim) || (heads > 1 && out_head < s.dim)) return fail(TSD_EINVAL, "tsd_cross_attend: rows or heads of out overlap");
  int sms = 0;
  TSD_CUDA(device_sms(&sms));
  CrossAttend a{};
  a.s = s;
  a.b = b;
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.q_row = q_row, a.q_head = q_head, a.out_row = out_row, a.out_head = out_head;
  a.heads = heads;
  a.group = heads / s.kv_heads;
  a.scale = scale;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  CrossTilesPlan p;
  // (queries that share memory are no tensor that TMA takes)
  if ((heads == 1 || q_head > 0) && (b.rows == 1 || q_row > 0) && cross_tiles_plan(s, b, heads, sms, &p)) {
    if (p.bytes > 0 && (!workspace || workspace_bytes < p.bytes || reinterpret_cast<uintptr_t>(workspace) % 16))
      return fail(TSD_EINVAL, "tsd_cross_attend: workspace of %lld bytes, %lld needed (16-byte aligned)", (long long)workspace_bytes, (long long)p.bytes);
    TSD_CUDA(cross_tiles_launch(a, p, workspace, stream));
    return TSD_OK;
  }
  TSD_CUDA(cross_rows_launch(a, cross_rows_plan(s, b, heads, sms), stream));
  return TSD_OK;
}
