// Attention over the 8-bit paged cache: the entry points (tsd.h: tsd_kv8_attend).
#include "kv8_attend.h"
#include "launch.h"

using namespace tsd;

namespace {

struct Plan {
  bool tiled = false;
  Kv8TilesPlan tiles;
  Kv8RowsPlan rows;
  int64_t bytes() const { return tiled ? tiles.bytes : rows.bytes; }
  int splits() const { return tiled ? tiles.splits : rows.splits; }
};

Plan plan_of(const tsd_kv8& c, const tsd_kv8_batch& b, int heads, int window, int sinks, int sms) {
  Plan p;
  p.tiled = kv8_tiles_plan(c, b, heads, window, sinks, sms, &p.tiles);
  if (!p.tiled) p.rows = kv8_rows_plan(c, b, heads, window, sinks, sms);
  return p;
}

tsd_status attend_check(const char* who, const tsd_kv8* cache, const tsd_kv8_batch* batch, int32_t heads, int32_t window, int32_t sinks) {
  if (tsd_status st = kv8_check(who, cache, batch)) return st;
  if (heads < 1 || heads % cache->kv_heads || heads / cache->kv_heads > 64)
    return fail(TSD_EINVAL, "%s: heads=%d must be 1..64 times kv_heads=%d", who, heads, cache->kv_heads);
  if (heads > 1024) return fail(TSD_EINVAL, "%s: heads=%d above 1024", who, heads);
  if (window < 0 || sinks < 0) return fail(TSD_EINVAL, "%s: negative window=%d or sinks=%d", who, window, sinks);
  return TSD_OK;
}

}  // namespace

extern "C" tsd_status tsd_kv8_attend_workspace(const tsd_kv8* cache, const tsd_kv8_batch* batch, int32_t heads,
                                               int32_t window, int32_t sinks, int64_t* bytes) {
  clear_error();
  if (!bytes) return fail(TSD_EINVAL, "tsd_kv8_attend_workspace: NULL argument");
  if (tsd_status st = attend_check("tsd_kv8_attend_workspace", cache, batch, heads, window, sinks)) return st;
  int sms = 0;
  TSD_CUDA(device_sms(&sms));
  *bytes = plan_of(*cache, *batch, heads, window, sinks, sms).bytes();
  return TSD_OK;
}

extern "C" tsd_status tsd_kv8_attend(const tsd_kv8* cache, const tsd_kv8_batch* batch, int32_t heads, const void* q,
                                     int64_t q_row, int64_t q_head, float scale, int32_t window, int32_t sinks, void* out,
                                     int64_t out_row, int64_t out_head, void* workspace, int64_t workspace_bytes,
                                     void* cuda_stream) {
  clear_error();
  if (tsd_status st = attend_check("tsd_kv8_attend", cache, batch, heads, window, sinks)) return st;
  if (tsd_status st = kv8_check_rows("tsd_kv8_attend", "q", q, q_row, q_head)) return st;
  if (tsd_status st = kv8_check_rows("tsd_kv8_attend", "out", out, out_row, out_head)) return st;
  int sms = 0;
  TSD_CUDA(device_sms(&sms));
  const Plan p = plan_of(*cache, *batch, heads, window, sinks, sms);
  if (p.bytes() > 0 && (!workspace || workspace_bytes < p.bytes() || reinterpret_cast<uintptr_t>(workspace) % 16))
    return fail(TSD_EINVAL, "tsd_kv8_attend: workspace of %lld bytes, %lld needed (16-byte aligned)", (long long)workspace_bytes, (long long)p.bytes());
  Kv8Attend a{};
  a.c = *cache;
  a.b = *batch;
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.q_row = q_row, a.q_head = q_head, a.out_row = out_row, a.out_head = out_head;
  a.heads = heads;
  a.group = heads / cache->kv_heads;
  a.window = window;
  a.sinks = sinks;
  a.scale = scale;
  a.part = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float2*>(a.part + (p.splits() > 1 ? (size_t)p.splits() * a.b.rows * heads * a.c.dim : 0));
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  TSD_CUDA(p.tiled ? kv8_tiles_launch(a, p.tiles, s) : kv8_rows_launch(a, p.rows, s));
  return TSD_OK;
}
