// A block's output normed, gated and added to the residual stream, and the next
// block's norm (tsd.h: tsd_residual_norm):
//   r = x + scale g (.) post(y),   h = norm(r)
// in one pass: a row stays in registers from its loads to its stores, statistics
// are fp32 sums over deviations from a mean known before (layer) or squares (rms),
// and h is computed from r before r is rounded.  Reads x, y (and g), writes r and h:
// bound by memory.
#include <cmath>
#include <type_traits>

#include "elem.cuh"
#include "internal.h"

namespace tsd {

namespace {

constexpr int kMaxWidth = 16384;

struct NormArgs {
  int n, d;
  const void *x, *y, *gate;
  void *r, *h;
  int64_t x_row, y_row, gate_row, r_row, h_row;
  float scale;
  tsd_norm post, norm;
};

// Sum over the row's THREADS threads (a power of two; above a warp: the whole CTA).
template <int THREADS>
__device__ __forceinline__ float row_sum(float v, float* s_part) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if constexpr (THREADS > 32) {
    __syncthreads();  // the last sum's parts have been read
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = s_part[threadIdx.x & (THREADS / 32 - 1)];
#pragma unroll
    for (int o = THREADS / 64; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  }
  return v;
}

// Where a thread's elements stand: WIDE, eight adjacent ones per chunk, else every THREADS-th.
template <int THREADS, bool WIDE>
__device__ __forceinline__ int place(int t, int c, int j) {
  return WIDE ? (c * THREADS + t) * 8 + j : (c * 8 + j) * THREADS + t;
}

template <int DT, int THREADS, int CHUNKS, bool WIDE>
__device__ __forceinline__ void load_row(const void* base, int64_t at, int t, int d, float* v) {
  using Raw = typename Elem<DT>::Raw;
  const Raw* p = static_cast<const Raw*>(base) + at;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    if constexpr (WIDE) {
      const int e = place<THREADS, true>(t, c, 0);
      Eight<DT> x;
#pragma unroll
      for (int i = 0; i < Eight<DT>::kWords; ++i) x.w[i] = 0;
      if (e < d) x.load(p + e);
      x.get(v + 8 * c);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int e = place<THREADS, false>(t, c, j);
        v[8 * c + j] = e < d ? Elem<DT>::wide(p[e]) : 0.f;
      }
    }
  }
}

template <int DT, int THREADS, int CHUNKS, bool WIDE>
__device__ __forceinline__ void store_row(void* base, int64_t at, int t, int d, const float* v) {
  using Raw = typename Elem<DT>::Raw;
  Raw* p = static_cast<Raw*>(base) + at;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    if constexpr (WIDE) {
      const int e = place<THREADS, true>(t, c, 0);
      Eight<DT> x;
      x.put(v + 8 * c);
      if (e < d) x.store(p + e);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int e = place<THREADS, false>(t, c, j);
        if (e < d) p[e] = Elem<DT>::narrow(v[8 * c + j]);
      }
    }
  }
}

// v <- norm(v); elements past d are 0 (weights and biases are read as 0 there) and stay out of the sums.
template <int THREADS, int CHUNKS, bool WIDE>
__device__ __forceinline__ void normalise(const tsd_norm& k, int t, int d, float* v, float* s_part) {
  constexpr int N = 8 * CHUNKS;
  if (k.kind == TSD_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s += v[i];
    const float mean = row_sum<THREADS>(s, s_part) / d;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = place<THREADS, WIDE>(t, i / 8, i % 8) < d ? v[i] - mean : 0.f;
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) s = fmaf(v[i], v[i], s);
  const float inv = 1.f / sqrtf(row_sum<THREADS>(s, s_part) / d + k.eps);
  float w[N];
  if (k.weight) {
    load_row<TSD_F32, THREADS, CHUNKS, WIDE>(k.weight, 0, t, d, w);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= inv * w[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= inv;
  }
  if (k.bias) {
    load_row<TSD_F32, THREADS, CHUNKS, WIDE>(k.bias, 0, t, d, w);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += w[i];
  }
}

constexpr int cta_threads(int per_row) { return per_row > 128 ? per_row : 128; }

template <int XT, int YT, int THREADS, int CHUNKS, bool WIDE>
__global__ void __launch_bounds__(cta_threads(THREADS)) k_residual_norm(const __grid_constant__ NormArgs a) {
  constexpr int kRows = cta_threads(THREADS) / THREADS, N = 8 * CHUNKS;
  static_assert(kRows == 1 || THREADS == 32, "several rows per CTA: a warp each");
  __shared__ float s_part[32];
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / THREADS;
  const int t = threadIdx.x % THREADS;
  if (row >= a.n) return;  // a whole warp (one row per CTA: none)
  float v[N], x[N];
  load_row<XT, THREADS, CHUNKS, WIDE>(a.x, row * a.x_row, t, a.d, x);
  if (a.y) {
    load_row<YT, THREADS, CHUNKS, WIDE>(a.y, row * a.y_row, t, a.d, v);
    if (a.post.kind != TSD_NORM_NONE) normalise<THREADS, CHUNKS, WIDE>(a.post, t, a.d, v, s_part);
    if (a.gate) {
      float g[N];
      load_row<YT, THREADS, CHUNKS, WIDE>(a.gate, row * a.gate_row, t, a.d, g);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] *= g[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = fmaf(a.scale, v[i], x[i]);
    store_row<XT, THREADS, CHUNKS, WIDE>(a.r, row * a.r_row, t, a.d, x);
  }
  if (a.norm.kind != TSD_NORM_NONE) {
    normalise<THREADS, CHUNKS, WIDE>(a.norm, t, a.d, x, s_part);
    store_row<YT, THREADS, CHUNKS, WIDE>(a.h, row * a.h_row, t, a.d, x);
  }
}

template <int XT, int YT, bool WIDE>
void launch(const NormArgs& a, cudaStream_t s) {
  // the fewest registers that hold a row: up to 1024 a warp's, else a CTA's
  const auto go = [&](auto threads, auto chunks) {
    constexpr int T = decltype(threads)::value, C = decltype(chunks)::value;
    constexpr int kRows = cta_threads(T) / T;
    k_residual_norm<XT, YT, T, C, WIDE><<<(unsigned)((a.n + kRows - 1) / kRows), cta_threads(T), 0, s>>>(a);
  };
  using std::integral_constant;
  if (a.d <= 256) go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  else if (a.d <= 512) go(integral_constant<int, 32>{}, integral_constant<int, 2>{});
  else if (a.d <= 1024) go(integral_constant<int, 32>{}, integral_constant<int, 4>{});
  else if (a.d <= 2048) go(integral_constant<int, 128>{}, integral_constant<int, 2>{});
  else if (a.d <= 4096) go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (a.d <= 8192) go(integral_constant<int, 512>{}, integral_constant<int, 2>{});
  else go(integral_constant<int, 512>{}, integral_constant<int, 4>{});
}

template <int XT, int YT>
void launch_wide(const NormArgs& a, bool wide, cudaStream_t s) {
  if (wide) launch<XT, YT, true>(a, s);
  else launch<XT, YT, false>(a, s);
}

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
  a.n = n, a.d = d, a.x = x, a.x_row = x_row, a.scale = scale;
  if (y) a.y = y, a.y_row = y_row, a.gate = gate, a.gate_row = gate ? gate_row : 0, a.r = r, a.r_row = r_row;
  if (a.norm.kind != TSD_NORM_NONE) a.h = h, a.h_row = h_row;
  // sixteen-byte accesses, where every row allows them
  const auto even = [&](const void* p, int64_t row) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && row % 8 == 0; };
  const bool wide = d % 8 == 0 && even(a.x, x_row) && even(a.y, a.y_row) && even(a.gate, a.gate_row) && even(a.r, a.r_row) && even(a.h, a.h_row) &&
                    even(a.post.weight, 0) && even(a.post.bias, 0) && even(a.norm.weight, 0) && even(a.norm.bias, 0);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (dtype == TSD_F32) launch_wide<TSD_F32, TSD_F32>(a, wide, s);
  else if (dtype == TSD_BF16) x_dtype == TSD_F32 ? launch_wide<TSD_F32, TSD_BF16>(a, wide, s) : launch_wide<TSD_BF16, TSD_BF16>(a, wide, s);
  else x_dtype == TSD_F32 ? launch_wide<TSD_F32, TSD_F16>(a, wide, s) : launch_wide<TSD_F16, TSD_F16>(a, wide, s);
  TSD_CUDA(cudaGetLastError());
  return TSD_OK;
}
