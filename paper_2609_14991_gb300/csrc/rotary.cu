// Rotary positions (tsd.h: tsd_rotary_apply).
//
// Pair i of a head at position p is turned by the angle p f_i.  The product is
// taken in turns as a 64-bit fraction: with t_i = frac(f_i / 2 pi) 2^64 it is p t_i
// mod 2^64, exact for every 32-bit position, so far positions lose nothing (in
// fp32 p f_i is off by 0.06 rad at p = 10^6).  What is left of an eighth of a turn
// goes through sincospif in fp32, its quarter turns are swaps and signs.
//
// Reads and writes each element once: bound by memory.  A CTA takes a few rows: one
// sine and cosine per row and pair, kept in shared memory for all query and key
// heads, which follow 16 bytes (of each half) at a time.
#include <algorithm>
#include <cmath>

#include "elem.cuh"
#include "internal.h"
#include "launch.h"
#include "seq.h"

namespace tsd {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 8;        // rows of a CTA
constexpr int kMaxAngles = 2048;   // ... and their angles

struct HeadRows {
  const void* x;
  void* out;
  int64_t row, head, out_row, out_head;
};

struct RotaryArgs {
  const unsigned long long* turns;
  const int32_t *positions, *slots, *lens, *starts;
  int n, n_slots, rows;
  int rot, dim, heads_q, heads;  // heads: of queries and keys
  int per_cta;                   // rows of a CTA
  float magnitude;
  HeadRows q, k;
};

// (cos, sin) of p t / 2^64 turns, times m
__device__ __forceinline__ float2 turn_of(int p, unsigned long long t, float m) {
  const unsigned long long ph = (unsigned long long)(long long)p * t;
  const unsigned quarter = (unsigned)((ph + (1ull << 61)) >> 62);
  const long long rest = (long long)(ph - ((unsigned long long)quarter << 62));  // within an eighth of a turn
  float s, c;
  sincospif((float)rest * 0x1p-63f, &s, &c);
  s *= m, c *= m;
  const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
  return make_float2((quarter + 1) & 2 ? -x : x, quarter & 2 ? -y : y);
}

// V adjacent elements; WIDE: by one access
template <int DT, int V, bool WIDE>
struct Some {
  using Raw = typename Elem<DT>::Raw;
  Raw x[V];
  __device__ __forceinline__ void load(const Raw* p) {
    if constexpr (WIDE) {
      static_assert(sizeof(x) == 16);
      *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = p[i];
    }
  }
  __device__ __forceinline__ void store(Raw* p) const {
    if constexpr (WIDE) {
      *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(x);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = x[i];
    }
  }
};

template <int DT, bool PAIRS, bool WIDE>  // PAIRS: neighbours are a pair
__global__ void __launch_bounds__(kThreads) k_rotary(const __grid_constant__ RotaryArgs a) {
  using Raw = typename Elem<DT>::Raw;
  constexpr int kWide = 16 / (int)sizeof(Raw);
  constexpr int kTurn = WIDE ? kWide : PAIRS ? 2 : 1;  // elements (of each half) of a turned item
  constexpr int kPass = WIDE ? kWide : 1;              // ... of one that stays as it is
  constexpr int kAtOnce = PAIRS ? 4 : 2;               // items of a thread on their way together
  __shared__ alignas(16) float2 s_turn[kMaxAngles];
  __shared__ int s_pos[kMaxRows], s_state[kMaxRows];  // state: 0 a row of no sequence, 1 turned, 2 NaN
  const int half = a.rot / 2, row0 = blockIdx.x * a.per_cta, rows = min(a.per_cta, a.rows - row0);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned turned = (PAIRS ? a.rot : half) / kTurn, per_head = turned + (a.dim - a.rot) / kPass, per_row = per_head * a.heads;
  const unsigned total = per_row * rows;
  // a thread's items, kThreads apart: row, head (queries', then keys') and place in the head
  struct Item {
    unsigned r, h, at;
  };
  unsigned i = threadIdx.x;
  Item next{i / per_row, 0, 0};
  next.h = (i - next.r * per_row) / per_head;
  next.at = i - next.r * per_row - next.h * per_head;
  const unsigned step_h = kThreads / per_head, step_at = kThreads % per_head;
  const auto advance = [&] {
    next.at += step_at;
    next.h += step_h;
    if (next.at >= per_head) next.at -= per_head, ++next.h;
    while (next.h >= (unsigned)a.heads) next.h -= a.heads, ++next.r;
  };
  const auto place = [&](const Item& t, bool out) {
    const bool key = t.h >= (unsigned)a.heads_q;
    const HeadRows& x = key ? a.k : a.q;
    const int64_t row = row0 + (int)t.r, head = key ? t.h - a.heads_q : t.h;
    return out ? row * x.out_row + head * x.out_head : row * x.row + head * x.head;
  };
  const auto base = [&](const Item& t, bool out) {
    const HeadRows& x = t.h >= (unsigned)a.heads_q ? a.k : a.q;
    return (out ? static_cast<Raw*>(x.out) : static_cast<Raw*>(const_cast<void*>(x.x))) + place(t, out);
  };
  Item items[kAtOnce];
  Some<DT, kTurn, WIDE> v[kAtOnce], z[PAIRS ? 1 : kAtOnce];
  static_assert(kPass <= kTurn, "");
  const auto fetch = [&] {
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      items[u] = next;
      if (i + u * kThreads < total) {
        const Raw* x = base(next, false);
        if (next.at >= turned) {
          Some<DT, kPass, WIDE> w;
          w.load(x + a.rot + (next.at - turned) * kPass);
#pragma unroll
          for (int j = 0; j < kPass; ++j) v[u].x[j] = w.x[j];
        } else {
          v[u].load(x + next.at * kTurn);
          if constexpr (!PAIRS) z[u].load(x + half + next.at * kTurn);
        }
      }
      advance();
    }
  };
  fetch();  // the first items are on their way while positions and angles are found
  if (warp < rows) {
    const int r = row0 + warp;
    int pos = 0, state = 1;
    if (a.positions) {
      pos = __ldg(a.positions + r);
    } else {
      const int i = seq_of(a.starts, a.n, r, lane);
      state = 0;
      if (i >= 0) {
        const int r0 = a.starts ? __ldg(a.starts + i) : i, r1 = a.starts ? __ldg(a.starts + i + 1) : i + 1;
        const int slot = a.slots ? __ldg(a.slots + i) : i;
        if (r >= r0 && r < r1) {
          const int len = slot >= 0 && slot < a.n_slots ? __ldg(a.lens + slot) : -1;
          state = r0 >= 0 && r1 <= a.rows && r1 - r0 <= len ? 1 : 2;
          pos = len - (r1 - r);
        }
      }
    }
    if (lane == 0) s_pos[warp] = pos, s_state[warp] = state;
  }
  __syncthreads();
  for (int j = threadIdx.x; j < rows * half; j += kThreads) {
    const int r = j / half;
    if (s_state[r] == 1) s_turn[j] = turn_of(s_pos[r], __ldg(a.turns + (j - r * half)), a.magnitude);
  }
  __syncthreads();
  const Raw nan = Elem<DT>::narrow(__uint_as_float(0x7fc00000u));
  for (; i < total; i += kAtOnce * kThreads) {
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const Item& t = items[u];
      if (i + u * kThreads >= total) break;
      const int state = s_state[t.r];
      if (state == 0) continue;
      Raw* out = base(t, true);
      if (t.at >= turned) {
        const unsigned at = a.rot + (t.at - turned) * kPass;
        if (state == 1 && out == base(t, false)) continue;
        Some<DT, kPass, WIDE> w;
#pragma unroll
        for (int j = 0; j < kPass; ++j) w.x[j] = state == 2 ? nan : v[u].x[j];
        w.store(out + at);
      } else if constexpr (PAIRS) {
        const float2* turn = s_turn + t.r * half + t.at * (kTurn / 2);
#pragma unroll
        for (int j = 0; j < kTurn; j += 2) {
          const float2 cs = turn[j / 2];
          const float x = Elem<DT>::wide(v[u].x[j]), y = Elem<DT>::wide(v[u].x[j + 1]);
          v[u].x[j] = state == 2 ? nan : Elem<DT>::narrow(x * cs.x - y * cs.y);
          v[u].x[j + 1] = state == 2 ? nan : Elem<DT>::narrow(y * cs.x + x * cs.y);
        }
        v[u].store(out + t.at * kTurn);
      } else {
        const float2* turn = s_turn + t.r * half + t.at * kTurn;
#pragma unroll
        for (int j = 0; j < kTurn; ++j) {
          const float2 cs = turn[j];
          const float x = Elem<DT>::wide(v[u].x[j]), y = Elem<DT>::wide(z[u].x[j]);
          v[u].x[j] = state == 2 ? nan : Elem<DT>::narrow(x * cs.x - y * cs.y);
          z[u].x[j] = state == 2 ? nan : Elem<DT>::narrow(y * cs.x + x * cs.y);
        }
        v[u].store(out + t.at * kTurn);
        z[u].store(out + half + t.at * kTurn);
      }
    }
    i += kAtOnce * kThreads;
    fetch();
    i -= kAtOnce * kThreads;
  }
}

template <int DT>
void launch(const RotaryArgs& a, bool pairs, bool wide, cudaStream_t s) {
  const unsigned grid = (unsigned)((a.rows + a.per_cta - 1) / a.per_cta);
  if (pairs) {
    if (wide) k_rotary<DT, true, true><<<grid, kThreads, 0, s>>>(a);
    else k_rotary<DT, true, false><<<grid, kThreads, 0, s>>>(a);
  } else {
    if (wide) k_rotary<DT, false, true><<<grid, kThreads, 0, s>>>(a);
    else k_rotary<DT, false, false><<<grid, kThreads, 0, s>>>(a);
  }
}

tsd_status check_heads(const char* what, const tsd_rotary_heads& t, int size, int rows, int dim) {
  if (!t.x || !t.out) return fail(TSD_EINVAL, "tsd_rotary_apply: NULL %s", what);
  if (t.heads < 1 || t.heads > 1024) return fail(TSD_EINVAL, "tsd_rotary_apply: %s has heads=%d outside [1, 1024]", what, t.heads);
  if (reinterpret_cast<uintptr_t>(t.x) % size || reinterpret_cast<uintptr_t>(t.out) % size)
    return fail(TSD_EINVAL, "tsd_rotary_apply: %s is not aligned to its elements", what);
  for (int64_t x : {t.row, t.head, t.out_row, t.out_head})
    if (x < 0 || x > (1ll << 40)) return fail(TSD_EINVAL, "tsd_rotary_apply: %s strides out of range", what);
  if ((rows > 1 && t.out_row < dim) || (t.heads > 1 && t.out_head < dim)) return fail(TSD_EINVAL, "tsd_rotary_apply: rows or heads of %s's result overlap", what);
  if (t.x == t.out && ((rows > 1 && t.row != t.out_row) || (t.heads > 1 && t.head != t.out_head)))
    return fail(TSD_EINVAL, "tsd_rotary_apply: %s is turned in place, but with other strides", what);
  return TSD_OK;
}

bool is_wide(const tsd_rotary_heads& t, int v) {
  return reinterpret_cast<uintptr_t>(t.x) % 16 == 0 && reinterpret_cast<uintptr_t>(t.out) % 16 == 0 && t.row % v == 0 && t.head % v == 0 &&
         t.out_row % v == 0 && t.out_head % v == 0;
}

}  // namespace

}  // namespace tsd

using namespace tsd;

extern "C" tsd_status tsd_rotary_turns(const tsd_rotary_cfg* cfg, uint64_t* turns) {
  clear_error();
  if (!cfg || !turns) return fail(TSD_EINVAL, "tsd_rotary_turns: NULL argument");
  const tsd_rotary_cfg& c = *cfg;
  if (c.rot < 2 || c.rot > 1024 || c.rot % 2) return fail(TSD_EINVAL, "tsd_rotary_turns: rot=%d is not even in [2, 1024]", c.rot);
  if (!(c.base > 0 && std::isfinite(c.base))) return fail(TSD_EINVAL, "tsd_rotary_turns: base must be positive and finite");
  if (c.scaling < TSD_ROTARY_PLAIN || c.scaling > TSD_ROTARY_RAMP) return fail(TSD_EINVAL, "tsd_rotary_turns: scaling %d is none of them", c.scaling);
  if (c.scaling != TSD_ROTARY_PLAIN && !(c.factor > 0 && std::isfinite(c.factor)))
    return fail(TSD_EINVAL, "tsd_rotary_turns: factor must be positive and finite");
  if (c.scaling == TSD_ROTARY_RAMP && !(c.original > 0 && std::isfinite(c.original) && std::isfinite(c.low) && c.high > c.low && std::isfinite(c.high)))
    return fail(TSD_EINVAL, "tsd_rotary_turns: a ramp needs original > 0 and high > low, all finite");
  const int half = c.rot / 2;
  constexpr double kHi = 0x1.45f306dc9c883p-3, kLo = -0x1.6b01ec5417056p-57;  // 1 / (2 pi)
  double base = c.base;
  if (c.scaling == TSD_ROTARY_BASE && half > 1) base *= std::pow(c.factor, (double)half / (half - 1));
  for (int i = 0; i < half; ++i) {
    double f = std::pow(base, -(double)i / half);
    if (c.scaling == TSD_ROTARY_LINEAR) f /= c.factor;
    if (c.scaling == TSD_ROTARY_RAMP) {
      const double keep = std::min(1.0, std::max(0.0, (c.original * f * kHi - c.low) / (c.high - c.low)));
      f = f * keep + f / c.factor * (1 - keep);
    }
    if (!(f <= 0x1p52)) return fail(TSD_EINVAL, "tsd_rotary_turns: the frequency of pair %d is above 2^52", i);
    const double t = f * kHi, lo = std::fma(f, kHi, -t) + f * kLo;  // t + lo turns per position
    turns[i] = (uint64_t)((t - std::floor(t)) * 0x1p64) + (uint64_t)std::llrint(lo * 0x1p64);
  }
  return TSD_OK;
}

extern "C" tsd_status tsd_rotary_apply(const tsd_rotary* rotary, const tsd_rotary_rows* rows, const tsd_rotary_heads* q, const tsd_rotary_heads* k,
                                       void* cuda_stream) {
  clear_error();
  if (!rotary || !rows || !q) return fail(TSD_EINVAL, "tsd_rotary_apply: NULL argument");
  const tsd_rotary& c = *rotary;
  if (!c.turns || reinterpret_cast<uintptr_t>(c.turns) % 8) return fail(TSD_EINVAL, "tsd_rotary_apply: NULL or unaligned turns");
  if (c.dtype < TSD_F32 || c.dtype > TSD_F16) return fail(TSD_EINVAL, "tsd_rotary_apply: dtype %d is not fp32, bf16 or fp16", c.dtype);
  if (c.dim < 2 || c.dim > 1024 || c.rot < 2 || c.rot > c.dim || c.rot % 2)
    return fail(TSD_EINVAL, "tsd_rotary_apply: dim=%d and rot=%d must have 2 <= rot <= dim <= 1024 and rot even", c.dim, c.rot);
  if (!std::isfinite(c.magnitude)) return fail(TSD_EINVAL, "tsd_rotary_apply: magnitude is not finite");
  if (rows->rows < 1 || rows->rows > (1 << 22)) return fail(TSD_EINVAL, "tsd_rotary_apply: rows=%d outside [1, 2^22]", rows->rows);
  const int size = c.dtype == TSD_F32 ? 4 : 2;
  if (tsd_status st = check_heads("q", *q, size, rows->rows, c.dim)) return st;
  if (k)
    if (tsd_status st = check_heads("k", *k, size, rows->rows, c.dim)) return st;
  if (k && (q->out == k->out || q->out == k->x || k->out == q->x)) return fail(TSD_EINVAL, "tsd_rotary_apply: queries and keys overlap");
  if (rows->positions) {
    if (rows->lens || rows->starts || rows->slots) return fail(TSD_EINVAL, "tsd_rotary_apply: positions, or lens, starts and slots");
  } else {
    if (!rows->lens) return fail(TSD_EINVAL, "tsd_rotary_apply: NULL positions and lens");
    if (rows->n < 1 || rows->n > 65535 || rows->n_slots < 1) return fail(TSD_EINVAL, "tsd_rotary_apply: n=%d outside [1, 65535] or n_slots=%d below 1", rows->n, rows->n_slots);
    if (!rows->starts && rows->rows != rows->n) return fail(TSD_EINVAL, "tsd_rotary_apply: starts is NULL: rows=%d must be n=%d", rows->rows, rows->n);
  }
  RotaryArgs a{};
  a.turns = reinterpret_cast<const unsigned long long*>(c.turns);
  a.positions = rows->positions, a.slots = rows->slots, a.lens = rows->lens, a.starts = rows->starts;
  a.n = rows->n, a.n_slots = rows->n_slots, a.rows = rows->rows;
  a.rot = c.rot, a.dim = c.dim, a.heads_q = q->heads, a.heads = q->heads + (k ? k->heads : 0);
  a.magnitude = c.magnitude;
  a.q = {q->x, q->out, q->row, q->head, q->out_row, q->out_head};
  if (k) a.k = {k->x, k->out, k->row, k->head, k->out_row, k->out_head};
  int sms = 0;
  TSD_CUDA(device_sms(&sms));
  // rows of a CTA: enough for its threads, but no fewer CTAs than twelve per SM
  const int64_t per_row = (int64_t)a.heads * c.dim;
  a.per_cta = (int)std::max<int64_t>(1, std::min<int64_t>({kMaxRows, kMaxAngles / (c.rot / 2), 16384 / per_row, a.rows / (12 * sms)}));
  const int v = 16 / size;
  const bool wide = is_wide(*q, v) && (!k || is_wide(*k, v)) && (c.interleaved ? c.rot : c.rot / 2) % v == 0 && c.dim % v == 0;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (c.dtype == TSD_F32) launch<TSD_F32>(a, c.interleaved, wide, s);
  else if (c.dtype == TSD_BF16) launch<TSD_BF16>(a, c.interleaved, wide, s);
  else launch<TSD_F16>(a, c.interleaved, wide, s);
  TSD_CUDA(cudaGetLastError());
  return TSD_OK;
}
