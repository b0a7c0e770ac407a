// A block's output normed, gated and added to the residual stream, and the next
// block's norm (tsd.h: tsd_residual_norm):
//   r = x + scale g (.) post(y),   h = norm(r)
// in one pass: a row stays in registers from its loads to its stores, statistics
// are fp32 sums over deviations from a mean known before (layer) or squares (rms),
// and h is computed from r before r is rounded.  Reads x, y (and g), writes r and h:
// bound by memory.  16384 x 4096, bf16, norms on both sides and a gate: 89 us, 0.89 of the copy rate; 7000 x 8192, one norm:
// 69 us, 0.97; 60000 x 256: 22 us, 0.81 (what a row takes besides its elements); 16384 x 3001: 84 us, 0.69 (weights from
// the 16 bytes around them).  One array of a row is in registers at a time, in pairs: the others come from shared
// memory or the L1 cache group by group, so that six CTAs of 128 rows' threads fit an SM.
#pragma once

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "elem.cuh"
#include "launch.h"
#include "norm.h"
#include "tc_common.cuh"

namespace tsd {

namespace {

using tc::add2;
using tc::fma2;
using tc::mul2;
using tc::pair_of;
using tc::unpair;

constexpr int kMaxSmem = 227 * 1024 - 512;  // of a CTA, dynamic
constexpr int kRingBytes = 128 * 1024;      // of an SM for rows on their way; the rest caches weights

// Sum over a row of its groups' sums v (group c * THREADS + t is thread t's c-th; THREADS a power of two; above a warp: the whole CTA;
// the warp's lanes are all here).  Always in the same order, so that a row's bits do not depend on how many threads the call's size
// gives it: 32 groups that follow each other by halves, then those sums by halves; groups that a row does not have are 0.
// s_part: two places that sums take in turn, so that one barrier serves for each.
template <int THREADS, int CHUNKS>
__device__ __forceinline__ float row_sum(const float (&v)[CHUNKS], float (*s_part)[32], int& turn) {
  static_assert(CHUNKS <= 2 || (CHUNKS == 4 && THREADS >= 32), "");
  const auto swap = [](float x, int o) { return __shfl_xor_sync(0xffffffffu, x, o); };
  float s;
  if constexpr (CHUNKS == 1 || THREADS < 32) {  // (two groups of fewer lanes than a warp's: halves of 32)
    s = v[0];
    if constexpr (CHUNKS == 2) s += v[1];
#pragma unroll
    for (int o = THREADS < 32 ? THREADS / 2 : 16; o; o >>= 1) s += swap(s, o);
  } else {
    // a lane goes on with half of the sums: the other half's of its partner for its own
    const int lane = threadIdx.x & 31;
    const bool high = lane & 16;
    s = (high ? v[CHUNKS / 2] : v[0]) + swap(high ? v[0] : v[CHUNKS / 2], 16);
    if constexpr (CHUNKS == 4) {
      const float z = (high ? v[3] : v[1]) + swap(high ? v[1] : v[3], 16);
      s = (lane & 8 ? z : s) + swap(lane & 8 ? s : z, 8);
    } else {
      s += swap(s, 8);
    }
#pragma unroll
    for (int o = 4; o; o >>= 1) s += swap(s, o);
    s += swap(s, 16);
    if constexpr (CHUNKS == 4) s += swap(s, 8);
  }
  if constexpr (THREADS > 32) {
    float* part = s_part[turn ^= 1];
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    s = part[threadIdx.x & (THREADS / 32 - 1)];
#pragma unroll
    for (int o = THREADS / 64; o; o >>= 1) s += swap(s, o);
  }
  return s;
}

// A thread's elements of a row: groups of eight, THREADS of them apart, or (apart) every THREADS-th element.
template <int THREADS, int CHUNKS, NormHow HOW>
struct Places {
  static constexpr bool EVEN = HOW != NormHow::kApart;
  int t, d, shift;
  __device__ __forceinline__ int first(int c) const { return (c * THREADS + t) * 8 - (HOW == NormHow::kShifted ? shift : 0); }  // a group's first element
  __device__ __forceinline__ int at(int i) const { return EVEN ? first(i / 8) + i % 8 : i * THREADS + t; }
  __device__ __forceinline__ bool some(int c) const { return first(c) < d; }  // (the first group always has some)
  __device__ __forceinline__ bool whole(int c) const { return HOW == NormHow::kWhole ? some(c) : first(c) >= 0 && first(c) + 8 <= d; }
  __device__ __forceinline__ bool has(int i) const { return HOW == NormHow::kWhole ? some(i / 8) : (unsigned)at(i) < (unsigned)d; }

  // Eight elements (group c's), as pairs, of an array that stands anywhere; 0 past the row
  template <int DT>
  __device__ __forceinline__ void load(const void* base, int c, uint64_t* v) const {
    const typename Elem<DT>::Raw* p = static_cast<const typename Elem<DT>::Raw*>(base);
    float x[8];
    if (HOW == NormHow::kWhole) {
      Eight<DT> y;
#pragma unroll
      for (int i = 0; i < Eight<DT>::kWords; ++i) y.w[i] = 0;
      if (some(c)) y.load(p + first(c));
      y.get(x);
    } else if (EVEN && reinterpret_cast<uintptr_t>(base) % 16 == 0) {
      // 16 bytes at a time: the group lies in them from element `over` on, alike for all groups of the row
      constexpr int kPer = DT == TSD_F32 ? 4 : 8, kPieces = 8 / kPer + 1;
      const int over = -shift & (kPer - 1), begin = first(c) - over;
      uint32_t w[4 * kPieces];
#pragma unroll
      for (int u = 0; u < kPieces; ++u) {
        const int e = begin + u * kPer;
        uint4 y = make_uint4(0, 0, 0, 0);
        if (e >= 0 && e < d && (u + 1 < kPieces || over)) y = __ldg(reinterpret_cast<const uint4*>(p + e));
        w[4 * u] = y.x, w[4 * u + 1] = y.y, w[4 * u + 2] = y.z, w[4 * u + 3] = y.w;
      }
      if constexpr (DT == TSD_F32) {
#pragma unroll
        for (int m = 0; m < 4; ++m)
          if (over == m)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[m + i]);
      } else {
        uint32_t y[5] = {0, 0, 0, 0, 0}, z[4];
#pragma unroll
        for (int m = 0; m < 4; ++m)
          if (over / 2 == m)
#pragma unroll
            for (int i = 0; i < 5; ++i) y[i] = m + i < 8 ? w[m + i] : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = over & 1 ? __funnelshift_r(y[i], y[i + 1], 16) : y[i];
        Elem<DT>::wide4(z, x);
      }
      if (!whole(c))
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!has(8 * c + i)) x[i] = 0.f;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = has(8 * c + i) ? Elem<DT>::wide(p[at(8 * c + i)]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pair_of(x[2 * i], x[2 * i + 1]);
  }
  template <int DT>
  __device__ __forceinline__ void store(void* base, int64_t row, int c, const uint64_t* v) const {
    typename Elem<DT>::Raw* p = static_cast<typename Elem<DT>::Raw*>(base) + row;
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpair(v[i], x[2 * i], x[2 * i + 1]);
    if (EVEN && whole(c)) {
      Eight<DT> y;
      y.put(x);
      y.store_even(p + first(c));
    } else if (HOW != NormHow::kWhole && (!EVEN || some(c))) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (has(8 * c + j)) p[at(8 * c + j)] = Elem<DT>::narrow(x[j]);
    }
  }
  // group c's elements past the row become 0
  __device__ __forceinline__ void trim(int c, uint64_t* v) const {
    if (EVEN && whole(c)) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      unpair(v[i], a, b);
      v[i] = pair_of(has(8 * c + 2 * i) ? a : 0.f, has(8 * c + 2 * i + 1) ? b : 0.f);
    }
  }
};

__device__ __forceinline__ float both(uint64_t v) {
  float a, b;
  unpair(v, a, b);
  return a + b;
}

// The first half of a norm: v <- v or (layer) its deviations from the mean, and the factor 1 / sqrt(mean square + eps);
// elements past the row are 0 and stay out of the sums.
template <int THREADS, int CHUNKS, NormHow HOW>
__device__ __forceinline__ float statistics(const tsd_norm& k, const Places<THREADS, CHUNKS, HOW>& pl, uint64_t* v, float (*s_part)[32], int& turn) {
  constexpr int N = 4 * CHUNKS;
  float sum[CHUNKS];  // of groups of eight
  if (k.kind == TSD_NORM_LAYER) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) sum[c] = both(add2(add2(v[4 * c], v[4 * c + 1]), add2(v[4 * c + 2], v[4 * c + 3])));
    const float mean = row_sum<THREADS, CHUNKS>(sum, s_part, turn) / pl.d;
    const uint64_t m2 = pair_of(-mean, -mean);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = add2(v[i], m2);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) pl.trim(c, v + 4 * c);
  }
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    uint64_t s = mul2(v[4 * c], v[4 * c]);
#pragma unroll
    for (int i = 1; i < 4; ++i) s = fma2(v[4 * c + i], v[4 * c + i], s);
    sum[c] = both(s);
  }
  return 1.f / sqrtf(row_sum<THREADS, CHUNKS>(sum, s_part, turn) / pl.d + k.eps);
}
// The second, for group c, but for that factor: v <- v * weight
template <int THREADS, int CHUNKS, NormHow HOW>
__device__ __forceinline__ void weighed(const tsd_norm& k, const Places<THREADS, CHUNKS, HOW>& pl, int c, uint64_t* v) {
  if (!k.weight) return;
  uint64_t w[4];
  pl.template load<TSD_F32>(k.weight, c, w);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], w[i]);
}
// ... and v <- v * factor + bias
template <int THREADS, int CHUNKS, NormHow HOW>
__device__ __forceinline__ void scaled(const tsd_norm& k, const Places<THREADS, CHUNKS, HOW>& pl, int c, uint64_t factor, uint64_t* v) {
  if (k.bias) {
    uint64_t b[4];
    pl.template load<TSD_F32>(k.bias, c, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = fma2(v[i], factor, b[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], factor);
  }
}

// A row array's groups of eight in shared memory, copied there asynchronously, 16 bytes at a time by neighbouring
// lanes: a thread's own, or (fp32, whose groups take two) its warp's.
template <int DT, int THREADS, int CHUNKS>
struct Staged {
  static constexpr int kUnits = DT == TSD_F32 ? 2 : 1;  // 16 bytes each
  static constexpr int kBytes = kUnits * CHUNKS * THREADS * 16;
  static constexpr int kLanes = THREADS < 32 ? THREADS : 32;  // of a row
  template <class P>
  static __device__ __forceinline__ void begin(unsigned char* to, const void* base, int64_t row, const P& pl) {
    const typename Elem<DT>::Raw* p = static_cast<const typename Elem<DT>::Raw*>(base) + row;
    constexpr int kPer = 8 / kUnits;
    const int lane = pl.t % kLanes;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const int unit = (c * THREADS + pl.t - lane) * kUnits + u * kLanes + lane, e = unit * kPer - pl.shift;
        if (e > -kPer && e < pl.d)  // at least one of the row's elements: the 16 bytes around them
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to + unit * 16)), "l"(p + e) : "memory");
      }
  }
  template <class P>
  static __device__ __forceinline__ void get(const unsigned char* from, const P& pl, int c, uint64_t* v) {
    Eight<DT> x;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const uint4 w = *reinterpret_cast<const uint4*>(from + ((c * THREADS + pl.t) * kUnits + u) * 16);
      x.w[4 * u] = w.x, x.w[4 * u + 1] = w.y, x.w[4 * u + 2] = w.z, x.w[4 * u + 3] = w.w;
    }
    float y[8];
    x.get(y);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pair_of(y[2 * i], y[2 * i + 1]);
    pl.trim(c, v);
  }
};

// Rows per CTA and CTAs per SM: those of a warp's lanes or part of them in CTAs of 128, wider ones a CTA's.
constexpr int cta_threads(int per_row) { return per_row <= 32 ? 128 : per_row; }
constexpr int ctas_per_sm(int per_row, int chunks) { return (chunks == 1 ? 1024 : per_row < 512 ? 768 : per_row) / cta_threads(per_row); }

// A CTA goes from row to row.  Where they stand in groups of eight the next rows are on their way to shared memory, each warp's elements to its own
// place, so no barrier guards them.
template <int XT, int YT, int THREADS, int CHUNKS, NormHow HOW>
__global__ void __launch_bounds__(cta_threads(THREADS), ctas_per_sm(THREADS, CHUNKS)) k_residual_norm(const __grid_constant__ NormArgs a) {
  constexpr int kRows = cta_threads(THREADS) / THREADS;
  constexpr bool EVEN = HOW != NormHow::kApart;
  static_assert(kRows == 1 || THREADS <= 32, "several rows per CTA: a warp's lanes each, or part of them");
  using X = Staged<XT, THREADS, CHUNKS>;
  using Y = Staged<YT, THREADS, CHUNKS>;
  extern __shared__ __align__(16) unsigned char s_ring[];
  __shared__ float s_part[2][32];
  int turn = 0;
  Places<THREADS, CHUNKS, HOW> pl{(int)threadIdx.x % THREADS, a.d, 0};
  const int64_t step = (int64_t)gridDim.x * kRows;
  constexpr int kOfWarp = THREADS < 32 ? 32 / THREADS : 1;  // a warp's rows go together
  const int sub = threadIdx.x / THREADS % kOfWarp;
  int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / THREADS;
  unsigned char* ring = s_ring + threadIdx.x / THREADS * a.depth * a.slot;
  const auto shift_of = [&](int64_t r) { return HOW == NormHow::kShifted ? (int)((a.base + r * a.stride) & 7) : 0; };
  const auto fetch = [&](int slot, int64_t r) {
    if constexpr (EVEN) {
      if (r < a.n) {
        const Places<THREADS, CHUNKS, HOW> at{pl.t, a.d, shift_of(r)};
        unsigned char* to = ring + slot * a.slot;
        X::begin(to, a.x, r * a.x_row, at);
        if (a.y) Y::begin(to + X::kBytes, a.y, r * a.y_row, at);
        if (a.gate && a.gate_row) Y::begin(to + X::kBytes + Y::kBytes, a.gate, r * a.gate_row, at);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
  };
  if constexpr (EVEN)
    for (int i = 0; i < a.depth; ++i) fetch(i, row + i * step);
  for (int slot = 0; row - sub < a.n; row += step) {  // (all lanes of a warp, all warps of a row)
    const bool live = kOfWarp == 1 || row < a.n;
    // One array of the row's values at a time stays in registers; what each group of eight takes besides comes when it is
    // its turn.
    uint64_t v[4 * CHUNKS];
    const bool gate_rows = a.gate && a.gate_row;
    pl.shift = shift_of(row);
    const unsigned char* from = ring + slot * a.slot;
    if constexpr (EVEN) {
      if (a.depth >= 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
      else if (a.depth == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
      else if (a.depth == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
      else asm volatile("cp.async.wait_group 0;" ::: "memory");
      __syncwarp();
    }
    const auto get_x = [&](int c, uint64_t* to) {
      if constexpr (EVEN) X::get(from, pl, c, to);
      else if (live) pl.template load<XT>(static_cast<const typename Elem<XT>::Raw*>(a.x) + row * a.x_row, c, to);
    };
    if (a.y) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        if constexpr (EVEN) Y::get(from + X::kBytes, pl, c, v + 4 * c);
        else if (live) pl.template load<YT>(static_cast<const typename Elem<YT>::Raw*>(a.y) + row * a.y_row, c, v + 4 * c);
      }
      float factor = a.scale;  // what a gated output takes besides: scale, and the norm's factor where no bias comes between
      uint64_t inv = 0;
      const bool post = a.post.kind != TSD_NORM_NONE;
      if (post) {
        const float f = statistics(a.post, pl, v, s_part, turn);
        if (a.post.bias) inv = pair_of(f, f);
        else factor *= f;
      }
      const uint64_t factor2 = pair_of(factor, factor);
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        uint64_t* z = v + 4 * c;
        if (post) {
          weighed(a.post, pl, c, z);
          if (a.post.bias) scaled(a.post, pl, c, inv, z);
        }
        uint64_t x[4];
        if (a.gate) {
          if (!gate_rows) pl.template load<YT>(a.gate, c, x);
          else if constexpr (EVEN) Y::get(from + X::kBytes + Y::kBytes, pl, c, x);
          else if (live) pl.template load<YT>(static_cast<const typename Elem<YT>::Raw*>(a.gate) + row * a.gate_row, c, x);
#pragma unroll
          for (int i = 0; i < 4; ++i) z[i] = mul2(z[i], x[i]);
        }
        get_x(c, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = fma2(z[i], factor2, x[i]);
        if (live) pl.template store<XT>(a.r, row * a.r_row, c, z);
      }
    } else {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) get_x(c, v + 4 * c);
    }
    if constexpr (EVEN) {
      __syncwarp();  // the slot has been read
      fetch(slot, row + a.depth * step);
      slot = slot + 1 == a.depth ? 0 : slot + 1;
    }
    if (a.norm.kind != TSD_NORM_NONE) {
      const float f = statistics(a.norm, pl, v, s_part, turn);
      const uint64_t inv = pair_of(f, f);
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        weighed(a.norm, pl, c, v + 4 * c);
        scaled(a.norm, pl, c, inv, v + 4 * c);
        if (live) pl.template store<YT>(a.h, row * a.h_row, c, v + 4 * c);
      }
    }
  }
}

template <int XT, int YT, NormHow HOW>
cudaError_t launch(NormArgs a, int sms, cudaStream_t s) {
  constexpr bool EVEN = HOW != NormHow::kApart;
  const auto go = [&](auto threads, auto chunks) {
    constexpr int T = decltype(threads)::value, C = decltype(chunks)::value;
    constexpr int kRows = cta_threads(T) / T;
    int per_sm = ctas_per_sm(T, C);
    if (EVEN) {
      a.slot = Staged<XT, T, C>::kBytes + ((a.y ? 1 : 0) + (a.gate && a.gate_row ? 1 : 0)) * Staged<YT, T, C>::kBytes;
      a.depth = std::min(std::max(kRingBytes / (per_sm * kRows * a.slot), 1), 4);
      per_sm = std::max(1, std::min(per_sm, kMaxSmem / (a.depth * kRows * a.slot)));
      const cudaError_t e = smem_opt_in<k_residual_norm<XT, YT, T, C, HOW>>(kMaxSmem);
      if (e != cudaSuccess) return e;
    }
    // Many rows: two per CTA and as many CTAs as that takes, which reads and writes memory more evenly than CTAs that stay (16384 x
    // 2048: 43 us, 47), but for one or two wide ones per SM (4000 x 12000 with norms on both sides: 173 us, 155).
    const int groups = (a.n + kRows - 1) / kRows, stay = sms * per_sm;
    const int ctas = per_sm > 2 && groups > 2 * stay ? (groups + 1) / 2 : std::min(groups, stay);
    k_residual_norm<XT, YT, T, C, HOW><<<(unsigned)ctas, cta_threads(T), (size_t)a.depth * kRows * a.slot, s>>>(a);
    return cudaGetLastError();
  };
  using std::integral_constant;
  const int d = a.d + (HOW == NormHow::kShifted ? 7 : 0);  // (with the elements that a row's first group may begin before it)
  // Up to 32 elements per thread: what each thread does besides (the sums' joins, the root) then weighs little.  Few rows:
  // as many threads as a row has groups.  With norms on both sides, us, so and with the threads of many rows: 152 rows of 512 2.5 and 2.8, of
  // 1537 3.4 and 6.1, of 4096 3.4 and 3.9, of 8192 4.5 and 4.4; 608 rows: 2.7 and 2.8, 4.2 and 6.4, 6.4 and 5.1, 10.9 and 9.0; 912 rows: 3.0
  // and 3.1, 6.2 and 6.7, 8.4 and 5.9, 15.2 and 10.3 (above 2048 elements many rows' threads are the better ones from some 300 rows on).
  if constexpr (EVEN)
    if (a.n <= 6 * sms && d > 256) {
      if (d <= 512) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
      if (d <= 1024) return go(integral_constant<int, 128>{}, integral_constant<int, 1>{});
      if (d <= 2048) return go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
      if (d <= 4096) return go(integral_constant<int, 512>{}, integral_constant<int, 1>{});
      if (d <= 8192) return go(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
    }
  if (d <= 64) return go(integral_constant<int, 8>{}, integral_constant<int, 1>{});
  if (d <= 128) return go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  if (d <= 256) return go(integral_constant<int, 16>{}, integral_constant<int, 2>{});
  if (d <= 512) return go(integral_constant<int, 32>{}, integral_constant<int, 2>{});
  if (d <= 1024) return go(integral_constant<int, 32>{}, integral_constant<int, 4>{});
  if (d <= 2048) return go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  if (d <= 4096) return go(integral_constant<int, 128>{}, integral_constant<int, 4>{});
  if (d <= 8192) return go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  return go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

}  // namespace

template <int XT, int YT>
cudaError_t norm_launch(const NormArgs& a, NormHow how, int sms, cudaStream_t s) {
  return how == NormHow::kWhole ? launch<XT, YT, NormHow::kWhole>(a, sms, s) : how == NormHow::kShifted ? launch<XT, YT, NormHow::kShifted>(a, sms, s) : launch<XT, YT, NormHow::kApart>(a, sms, s);
}

}  // namespace tsd
