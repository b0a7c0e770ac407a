// The entry point of norms around a block (tsd.h: tsd_residual_norm); norm.cuh has the kernel.
#include <algorithm>
#include <cmath>

#include "internal.h"
#include "launch.h"
#include "norm.h"

namespace tsd {

namespace {

tsd_status check_rows(const char* what, const void* p, int64_t row, int d, int n, int size) {
  if (!p) return fail(TSD_EINVAL, "tsd_residual_norm: NULL %s", what);
  if (reinterpret_cast<uintptr_t>(p) % size) return fail(TSD_EINVAL, "tsd_residual_norm: %s is not aligned to its elements", what);
  if (row < 0 || row > (1ll << 40) || (row < d && n > 1)) return fail(TSD_EINVAL, "tsd_residual_norm: rows of %s overlap or are out of range", what);
  return TSD_OK;
}

tsd_status check_norm(const char* what, const tsd_norm* k) {
  if (!k || k->kind == TSD_NORM_NONE) return TSD_OK;
  if (k->kind != TSD_NORM_RMS && k->kind != TSD_NORM_LAYER) return fail(TSD_EINVAL, "tsd_residual_norm: %s has kind %d", what, k->kind);
  if (!(k->eps >= 0.f && std::isfinite(k->eps))) return fail(TSD_EINVAL, "tsd_residual_norm: %s needs a finite eps of 0 or more", what);
  if (reinterpret_cast<uintptr_t>(k->weight) % 4 || reinterpret_cast<uintptr_t>(k->bias) % 4)
    return fail(TSD_EINVAL, "tsd_residual_norm: %s's weight or bias is not aligned", what);
  return TSD_OK;
}

// Whether `bytes` at p lie in one of n rows of `width` bytes, `row` apart from `base` on (at least `width`, or there is one).
bool in_rows(const void* p, int64_t bytes, const void* base, int64_t row, int64_t width, int n) {
  const int64_t at = reinterpret_cast<intptr_t>(p) - reinterpret_cast<intptr_t>(base);
  if (at + bytes <= 0) return false;
  if (at < 0 || n == 1) return at < width;
  const int64_t i = std::min<int64_t>(at / row, n - 1);  // the last row that begins at p or before it
  return at < i * row + width || (i + 1 < n && at + bytes > (i + 1) * row);
}

// Results (NULL: none) over the gate or over a norm's weight or bias.
tsd_status check_vectors(const char* what, const void* to, int64_t row, int64_t width, int n, int d, const NormArgs& a, const void* gate, int64_t gate_row,
                         int size) {
  if (!to) return TSD_OK;
  if (gate && (gate_row ? gate == to : in_rows(gate, (int64_t)d * size, to, row, width, n))) return fail(TSD_EINVAL, "tsd_residual_norm: %s and the gate overlap", what);
  for (const tsd_norm* k : {&a.post, &a.norm}) {
    if (k->weight && in_rows(k->weight, 4ll * d, to, row, width, n)) return fail(TSD_EINVAL, "tsd_residual_norm: %s and a weight overlap", what);
    if (k->bias && in_rows(k->bias, 4ll * d, to, row, width, n)) return fail(TSD_EINVAL, "tsd_residual_norm: %s and a bias overlap", what);
  }
  return TSD_OK;
}

}  // namespace

}  // namespace tsd

using namespace tsd;

extern "C" tsd_status tsd_residual_norm(int32_t n, int32_t d, const void* x, int32_t x_dtype, int64_t x_row, const void* y, int32_t dtype,
                                        int64_t y_row, const tsd_norm* post, const void* gate, int64_t gate_row, float scale,
                                        const tsd_norm* norm, void* r, int64_t r_row, void* h, int64_t h_row, void* cuda_stream) {
  clear_error();
  if (n < 1 || n > (1 << 27)) return fail(TSD_EINVAL, "tsd_residual_norm: n=%d outside [1, 2^27]", n);
  if (d < 1 || d > kMaxWidth) return fail(TSD_EINVAL, "tsd_residual_norm: d=%d outside [1, %d]", d, kMaxWidth);
  if (dtype < TSD_F32 || dtype > TSD_F16 || (x_dtype != dtype && x_dtype != TSD_F32))
    return fail(TSD_EINVAL, "tsd_residual_norm: dtype %d must be fp32, bf16 or fp16 and x's %d the same or fp32", dtype, x_dtype);
  const void* src = y ? y : x;  // what h may replace
  const int64_t src_row = y ? y_row : x_row;
  const int size = dtype == TSD_F32 ? 4 : 2, x_size = x_dtype == TSD_F32 ? 4 : 2;
  if (tsd_status st = check_norm("post", post)) return st;
  if (tsd_status st = check_norm("norm", norm)) return st;
  NormArgs a{};
  if (post) a.post = *post;
  if (norm) a.norm = *norm;
  if (a.post.kind == TSD_NORM_NONE) a.post = tsd_norm{};
  if (a.norm.kind == TSD_NORM_NONE) a.norm = tsd_norm{};
  if (tsd_status st = check_rows("x", x, x_row, d, n, x_size)) return st;
  if (y) {
    if (tsd_status st = check_rows("y", y, y_row, d, n, size)) return st;
    if (tsd_status st = check_rows("r", r, r_row, d, n, x_size)) return st;
    if (!std::isfinite(scale)) return fail(TSD_EINVAL, "tsd_residual_norm: scale is not finite");
    if (gate && gate_row)
      if (tsd_status st = check_rows("gate", gate, gate_row, d, n, size)) return st;
    if (gate && reinterpret_cast<uintptr_t>(gate) % size) return fail(TSD_EINVAL, "tsd_residual_norm: gate is not aligned to its elements");
  } else if (gate || a.post.kind != TSD_NORM_NONE || a.norm.kind == TSD_NORM_NONE) {
    return fail(TSD_EINVAL, "tsd_residual_norm: without y there is a norm, and no gate or post");
  }
  if (a.norm.kind != TSD_NORM_NONE)
    if (tsd_status st = check_rows("h", h, h_row, d, n, size)) return st;
  // in place a thread writes what it has read: the same elements
  const auto moved = [&](const void* in, int64_t in_row, const void* to, int64_t to_row) { return in == to && in_row != to_row && n > 1; };
  if ((y && a.norm.kind != TSD_NORM_NONE && (h == r || h == x)) || (y && r == y) || (y && moved(x, x_row, r, r_row)) ||
      (a.norm.kind != TSD_NORM_NONE && moved(src, src_row, h, h_row)))
    return fail(TSD_EINVAL, "tsd_residual_norm: results overlap each other or another input");
  // what other rows read, or read later, is not written
  if (tsd_status st = check_vectors("r", y ? r : nullptr, r_row * x_size, (int64_t)d * x_size, n, d, a, gate, gate_row, size)) return st;
  if (tsd_status st = check_vectors("h", a.norm.kind != TSD_NORM_NONE ? h : nullptr, h_row * size, (int64_t)d * size, n, d, a, gate, gate_row, size)) return st;
  a.n = n, a.d = d, a.x = x, a.x_row = x_row, a.scale = scale;
  if (y) a.y = y, a.y_row = y_row, a.gate = gate, a.gate_row = gate ? gate_row : 0, a.r = r, a.r_row = r_row;
  if (a.norm.kind != TSD_NORM_NONE) a.h = h, a.h_row = h_row;
  // rows in groups of eight elements at 16-byte boundaries, where they stand alike in all arrays
  const auto off = [&](const void* p, int bytes) { return (int)(reinterpret_cast<uintptr_t>(p) / bytes % 8); };
  a.base = off(a.x, x_size);
  a.stride = (int)(x_row % 8);
  const auto alike = [&](const void* p, int64_t row, int bytes) { return !p || (off(p, bytes) == a.base && (n == 1 || row % 8 == a.stride)); };
  const bool even = alike(a.y, a.y_row, size) && alike(a.r, a.r_row, x_size) && alike(a.h, a.h_row, size) && (!a.gate_row || alike(a.gate, a.gate_row, size));
  const auto aligned = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  NormHow how = NormHow::kApart;
  if (even && a.base == 0 && (n == 1 || a.stride == 0) && d % 8 == 0 && aligned(a.post.weight) && aligned(a.post.bias) && aligned(a.norm.weight) &&
      aligned(a.norm.bias) && aligned(a.gate))
    how = NormHow::kWhole;
  else if (even && d + 7 <= kMaxWidth)
    how = NormHow::kShifted;
  int sms = 0;
  TSD_CUDA(device_sms(&sms));
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (dtype == TSD_F32) TSD_CUDA((norm_launch<TSD_F32, TSD_F32>(a, how, sms, s)));
  else if (dtype == TSD_BF16) TSD_CUDA((x_dtype == TSD_F32 ? norm_launch<TSD_F32, TSD_BF16>(a, how, sms, s) : norm_launch<TSD_BF16, TSD_BF16>(a, how, sms, s)));
  else TSD_CUDA((x_dtype == TSD_F32 ? norm_launch<TSD_F32, TSD_F16>(a, how, sms, s) : norm_launch<TSD_F16, TSD_F16>(a, how, sms, s)));
  return TSD_OK;
}
