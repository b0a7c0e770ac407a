// Rotary positions (tsd.h: tsd_rotary_apply).
//
// Pair i of a head at position p is turned by the angle p f_i.  The product is
// taken in turns as a 64-bit fraction: with t_i = frac(f_i / 2 pi) 2^64 it is p t_i
// mod 2^64, exact for every 32-bit position, so far positions lose nothing (in
// fp32 p f_i is off by 0.06 rad at p = 10^6).  What is left of an eighth of a turn
// goes through sincospif in fp32, its quarter turns are swaps and signs.
//
// Reads and writes each element once: bound by memory, and by the instructions of half-words.  A CTA takes a few rows: one
// sine and cosine per row and pair, kept in shared memory for all query and key
// heads, which follow 16 bytes (of each half) at a time.  16500 rows of 18 heads (128 wide, bf16, half layout): 28 us, 0.80 of the
// copy rate; CTAs of 256 threads and twice the rows 31, of 64 and half 35; half of the head turned, interleaved, fp16: 29.  Parts of a
// head that 16 bytes do not divide go through shared memory: 26 of 80, 16500 rows: 24 us, 0.59.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "elem.cuh"
#include "internal.h"
#include "launch.h"
#include "seq.h"

namespace tsd {

namespace {

constexpr int kDirect = 128, kThreads = 256;  // of a CTA: 16 bytes at a time straight through, staged
constexpr int kMaxRows = 8;        // rows of a CTA
constexpr int kMaxAngles = 512;    // ... and their angles
constexpr int kStaged = 24 * 1024; // bytes of heads that a CTA stages

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
  int per_cta, heads_cta;        // rows of a CTA, and (staged) heads
  bool pairs;                    // neighbours are a pair
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

// Rows row0 .. row0 + rows - 1 of a CTA: positions, states and angles in shared memory.
struct Turns {
  alignas(16) float2 cs[kMaxAngles];   // [rows][rot / 2] (cosine, sine), in an order of the kernel's
  int pos[kMaxRows], state[kMaxRows];  // state: 0 a row of no sequence, 1 turned, 2 NaN
};

// PLACE: where the cosine and the sine of pair i of a row stand among the row's floats
template <int THREADS, class PLACE>
__device__ __forceinline__ void find_turns(const RotaryArgs& a, int row0, int rows, Turns& s, PLACE place) {
  const int half = a.rot / 2, lane = threadIdx.x & 31;
  for (int w = threadIdx.x >> 5; w < rows; w += THREADS / 32) {
    const int r = row0 + w;
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
    if (lane == 0) s.pos[w] = pos, s.state[w] = state;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * half; i += THREADS) {
    const int r = i / half;
    if (s.state[r] == 1) {
      const float2 cs = turn_of(s.pos[r], __ldg(a.turns + (i - r * half)), a.magnitude);
      const int2 at = place(i - r * half);
      float* to = reinterpret_cast<float*>(s.cs) + 2 * r * half;
      to[at.x] = cs.x, to[at.y] = cs.y;
    }
  }
  __syncthreads();
}

// A thread's items, THREADS apart, of rows x heads x per_head: row, head (queries', then keys') and place in the head.
template <int THREADS>
struct Items {
  unsigned heads, per_head, r, h, at, step_h, step_at;
  __device__ __forceinline__ Items(unsigned hs, unsigned per) : heads(hs), per_head(per) {
    const unsigned i = threadIdx.x, per_row = heads * per_head;
    r = i / per_row;
    h = (i - r * per_row) / per_head;
    at = i - r * per_row - h * per_head;
    step_h = THREADS / per_head;
    step_at = THREADS - step_h * per_head;
  }
  __device__ __forceinline__ void advance() {
    at += step_at;
    h += step_h;
    if (at >= per_head) at -= per_head, ++h;
    while (h >= heads) h -= heads, ++r;
  }
};

template <class Raw>
__device__ __forceinline__ Raw* head_at(const RotaryArgs& a, int row, unsigned h, bool out) {
  const bool key = h >= (unsigned)a.heads_q;
  const HeadRows& x = key ? a.k : a.q;
  const int64_t head = key ? h - a.heads_q : h;
  return out ? static_cast<Raw*>(x.out) + row * x.out_row + head * x.out_head : static_cast<Raw*>(const_cast<void*>(x.x)) + row * x.row + head * x.head;
}

// (a, b) turned
__device__ __forceinline__ float2 turn(float a, float b, float2 cs) { return make_float2(a * cs.x - b * cs.y, b * cs.x + a * cs.y); }

// Twice 16 bytes at a time: halves of a head's turned dimensions begin at 16-byte boundaries.  An item is 16 bytes of
// the first half and those of the second (PAIRS: neighbours are pairs, in each of both), or such of the other dimensions.
template <int DT, bool PAIRS>
__global__ void __launch_bounds__(kDirect) k_rotary(const __grid_constant__ RotaryArgs a) {
  using Raw = typename Elem<DT>::Raw;
  constexpr int kPer = 16 / (int)sizeof(Raw);  // elements of 16 bytes
  constexpr int kAtOnce = 2;                   // items of a thread on their way together
  __shared__ Turns s;
  const int half = a.rot / 2, row0 = blockIdx.x * a.per_cta, rows = min(a.per_cta, a.rows - row0);
  const unsigned turned = half / kPer, rest = (a.dim - a.rot) / kPer, twice = rest % 2 ? 0 : rest / 2;  // (an odd rest: one by one)
  const unsigned per_head = turned + (twice ? twice : rest), total = per_head * a.heads * rows;
  Items<kDirect> next(a.heads, per_head);
  struct Item {
    unsigned r, h, at;
    uint4 v, z;
  } items[kAtOnce];
  unsigned i = threadIdx.x;
  const auto fetch = [&](unsigned first) {
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      Item& t = items[u];
      t.r = next.r, t.h = next.h, t.at = next.at;
      if (first + u * kDirect < total) {
        const Raw* x = head_at<Raw>(a, row0 + (int)t.r, t.h, false);
        if (t.at >= turned) x += a.rot - half;  // (turned * kPer is half)
        t.v = *reinterpret_cast<const uint4*>(x + t.at * kPer);
        if (t.at < turned || twice) t.z = *reinterpret_cast<const uint4*>(x + (t.at < turned ? turned : twice) * kPer + t.at * kPer);
      }
      next.advance();
    }
  };
  fetch(i);  // the first items are on their way while positions and angles are found
  // Four floats (of two pairs) of an item stand among those of the others of the head, so that neighbouring lanes read
  // neighbouring ones: (c0, c1, s0, s1), PAIRS (c0, s0, c1, s1).
  constexpr int kPairs = PAIRS ? kPer / 2 : kPer;  // of 16 bytes
  find_turns<kDirect>(a, row0, rows, s, [&](int i) {
    const int second = PAIRS && i >= half / 2, k = second ? i - half / 2 : i;
    const int item = k / kPairs, j = k % kPairs, at = 4 * ((second * (kPairs / 2) + j / 2) * (int)turned + item);
    return PAIRS ? make_int2(at + 2 * (j & 1), at + 2 * (j & 1) + 1) : make_int2(at + (j & 1), at + 2 + (j & 1));
  });
  const uint32_t nan = DT == TSD_F32 ? 0x7fc00000u : DT == TSD_BF16 ? 0x7fc07fc0u : 0x7e007e00u;
  for (; i < total; i += kAtOnce * kDirect) {
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      Item& t = items[u];
      if (i + u * kDirect >= total) break;
      const int state = s.state[t.r];
      if (state == 0) continue;
      Raw* out = head_at<Raw>(a, row0 + (int)t.r, t.h, true);
      if (state == 2) t.v = t.z = make_uint4(nan, nan, nan, nan);
      if (t.at >= turned) {
        if (state == 1 && out == head_at<Raw>(a, row0 + (int)t.r, t.h, false)) continue;  // in place
        out += a.rot - half + t.at * kPer;
        *reinterpret_cast<uint4*>(out) = t.v;
        if (twice) *reinterpret_cast<uint4*>(out + twice * kPer) = t.z;
        continue;
      }
      const float4* cs = reinterpret_cast<const float4*>(s.cs + t.r * half) + t.at;
      if (state == 1) {
        uint32_t v[4] = {t.v.x, t.v.y, t.v.z, t.v.w}, z[4] = {t.z.x, t.z.y, t.z.z, t.z.w};
        if constexpr (PAIRS) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint32_t(&w)[4] = k ? z : v;
            float x[kPer];
            Elem<DT>::wide4(w, x);
#pragma unroll
            for (int j = 0; j < kPer; j += 4) {
              const float4 c = cs[(k * (kPairs / 2) + j / 4) * turned];
              const float2 p = turn(x[j], x[j + 1], make_float2(c.x, c.y)), q = turn(x[j + 2], x[j + 3], make_float2(c.z, c.w));
              x[j] = p.x, x[j + 1] = p.y, x[j + 2] = q.x, x[j + 3] = q.y;
            }
            Elem<DT>::narrow4(x, w);
          }
        } else {
          float x[kPer], y[kPer];
          Elem<DT>::wide4(v, x);
          Elem<DT>::wide4(z, y);
#pragma unroll
          for (int j = 0; j < kPer; j += 2) {
            const float4 c = cs[j / 2 * turned];
            const float2 p = turn(x[j], y[j], make_float2(c.x, c.z)), q = turn(x[j + 1], y[j + 1], make_float2(c.y, c.w));
            x[j] = p.x, y[j] = p.y, x[j + 1] = q.x, y[j + 1] = q.y;
          }
          Elem<DT>::narrow4(x, v);
          Elem<DT>::narrow4(y, z);
        }
        t.v = make_uint4(v[0], v[1], v[2], v[3]), t.z = make_uint4(z[0], z[1], z[2], z[3]);
      }
      *reinterpret_cast<uint4*>(out + t.at * kPer) = t.v;
      *reinterpret_cast<uint4*>(out + half + t.at * kPer) = t.z;
    }
    fetch(i + kAtOnce * kDirect);
  }
}

// Any number of turned dimensions: heads through shared memory, where neighbouring lanes turn neighbouring pairs.  WIDE: heads begin
// and end at 16-byte boundaries, and come and leave by them; else element by element.
template <int DT, bool WIDE>
__global__ void __launch_bounds__(kThreads) k_rotary_staged(const __grid_constant__ RotaryArgs a) {
  using Raw = typename Elem<DT>::Raw;
  constexpr int kPer = WIDE ? 16 / (int)sizeof(Raw) : 1;
  using Unit = typename std::conditional<WIDE, uint4, Raw>::type;
  __shared__ Turns s;
  extern __shared__ __align__(16) unsigned char s_raw[];
  Raw* const data = reinterpret_cast<Raw*>(s_raw);
  const int half = a.rot / 2, row0 = blockIdx.x * a.per_cta, rows = min(a.per_cta, a.rows - row0);
  const unsigned head0 = blockIdx.y * a.heads_cta, heads = min(a.heads_cta, a.heads - (int)head0), per_head = a.dim / kPer, total = per_head * heads * rows;
  {
    Items<kThreads> t(heads, per_head);
    for (unsigned i = threadIdx.x; i < total; i += kThreads, t.advance()) {
      const Raw* x = head_at<Raw>(a, row0 + (int)t.r, head0 + t.h, false) + t.at * kPer;
      if constexpr (WIDE)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(data + i * kPer)), "l"(x) : "memory");
      else
        data[i] = *x;
    }
    if constexpr (WIDE) asm volatile("cp.async.wait_all;" ::: "memory");
  }
  find_turns<kThreads>(a, row0, rows, s, [](int i) { return make_int2(2 * i, 2 * i + 1); });
  {
    Items<kThreads> t(heads, half);
    for (unsigned i = threadIdx.x; i < half * heads * rows; i += kThreads, t.advance()) {
      if (s.state[t.r] != 1) continue;
      Raw* x = data + (t.r * heads + t.h) * a.dim;
      Raw &u = x[a.pairs ? 2 * t.at : t.at], &w = x[a.pairs ? 2 * t.at + 1 : half + t.at];
      const float2 y = turn(Elem<DT>::wide(u), Elem<DT>::wide(w), s.cs[t.r * half + t.at]);
      u = Elem<DT>::narrow(y.x), w = Elem<DT>::narrow(y.y);
    }
  }
  __syncthreads();
  Items<kThreads> t(heads, per_head);
  for (unsigned i = threadIdx.x; i < total; i += kThreads, t.advance()) {
    const int state = s.state[t.r];
    if (state == 0) continue;
    Unit v = reinterpret_cast<const Unit*>(data)[i];
    if (state == 2) {
      const Raw nan = Elem<DT>::narrow(__uint_as_float(0x7fc00000u));
#pragma unroll
      for (int j = 0; j < kPer; ++j) reinterpret_cast<Raw*>(&v)[j] = nan;
    }
    *reinterpret_cast<Unit*>(head_at<Raw>(a, row0 + (int)t.r, head0 + t.h, true) + t.at * kPer) = v;
  }
}

template <int DT>
void launch(const RotaryArgs& a, bool direct, bool wide, cudaStream_t s) {
  const unsigned grid = (unsigned)((a.rows + a.per_cta - 1) / a.per_cta);
  if (direct) {
    if (a.pairs) k_rotary<DT, true><<<grid, kDirect, 0, s>>>(a);
    else k_rotary<DT, false><<<grid, kDirect, 0, s>>>(a);
    return;
  }
  const dim3 g(grid, (unsigned)((a.heads + a.heads_cta - 1) / a.heads_cta));
  const size_t bytes = (size_t)a.per_cta * a.heads_cta * a.dim * sizeof(typename Elem<DT>::Raw);
  if (wide) k_rotary_staged<DT, true><<<g, kThreads, bytes, s>>>(a);
  else k_rotary_staged<DT, false><<<g, kThreads, bytes, s>>>(a);
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
  a.pairs = c.interleaved;
  const int v = 16 / size;
  const bool wide = is_wide(*q, v) && (!k || is_wide(*k, v)) && c.dim % v == 0, direct = wide && c.rot / 2 % v == 0;
  // rows of a CTA: a few items for each of its threads, but no fewer CTAs than four per SM
  const int64_t per_row = (int64_t)a.heads * c.dim, most = direct ? 8192 : kStaged / size;
  a.per_cta = (int)std::max<int64_t>(1, std::min<int64_t>({kMaxRows, kMaxAngles / (c.rot / 2), most / per_row, a.rows / (4 * sms)}));
  a.heads_cta = (int)std::min<int64_t>(a.heads, std::max<int64_t>(1, most / c.dim));
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (c.dtype == TSD_F32) launch<TSD_F32>(a, direct, wide, s);
  else if (c.dtype == TSD_BF16) launch<TSD_BF16>(a, direct, wide, s);
  else launch<TSD_F16>(a, direct, wide, s);
  TSD_CUDA(cudaGetLastError());
  return TSD_OK;
}
