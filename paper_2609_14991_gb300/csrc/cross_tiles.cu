// Attention over an encoder's states with many query rows per key head: whole
// transcripts, n-best lists (tsd.h: tsd_cross_attend).
//
// The mathematics is cross_rows.cu's; the products run on tcgen05 (16-bit in, fp32 accumulate in
// TMEM).  A unit is 256 rows of a sequence and key head (row = token * group + head of the
// group), two row tiles of 128, over the frames of its source, 128 at a time:
//   warps 0-7   softmax: a thread is a row (warps 0-3 tile 0, 4-7 tile 1), so its maximum
//               and sum need no exchange.  Reads its 128 scores from TMEM and leaves the weights
//               in their place, as the values' product's A operands: the product wants the states'
//               type, 8 or 11 bits of a weight, so a weight is a sum of two (cross.h), 16 bits, whose products
//               run one after the other;
//   warp 8      copies keys and values, a ring of tiles by TMA (128-byte swizzle);
//   warp 9      issues the MMAs;
//   warp 10     zeroes what stands behind a source's length in its last tile of values: a
//               weight of 0 does not make a NaN or infinity 0;
//   warp 11     says which parts of the work are this CTA's.
// While one row tile's scores are with the softmax, the other's products run.  Keys are the K-major B
// operand of the scores; the same layout of the values is read as an MN-major B
// operand, so neither is transposed.  The maximum is looked for, and the accumulator rescaled in
// TMEM, only in steps whose weights outgrow fp16 relative to the one so far.
//
// Work: every unit has its tiles of frames in one line of all sequences, weighted by what they
// cost, and each CTA takes an equal share of that line, so ragged sequences and few
// long ones fill the device alike.  A unit that several CTAs share leaves its parts in the workspace, which a
// second kernel joins in their order.
//
// A step of two row tiles and 128 frames takes 1.80 us at dim 128, its three products (scores, values with both parts of the weights)
// at 2.1 PFLOP/s, above the library's rate: they bound it (with weights of 8 bits, two products, 1.39 us).  Dim 64: 1.66 us, a values' product whose
// weights come from TMEM takes 65 clocks at any width, and the softmax 1300 a row tile.  6 ragged texts of up to 1100 tokens, 16 heads, over up to 9000 frames,
// 4 key heads of 128: 194 us.  What a unit takes besides its tiles, 3.0 us: first maximum, last products, results (64 KB at 64 bytes per
// clock, 128 where it is shared).
#include <algorithm>
#include <type_traits>

#include "cross.h"
#include "launch.h"
#include "tc_attend.cuh"

namespace tsd {

namespace {

using namespace tc;

constexpr int kFrames = 128;  // per tile
constexpr int kUnitRows = 256;  // of which a row tile takes whole tokens' heads: 128 / group tokens
constexpr int kSoftWarps = 8, kTmaWarp = 8, kMmaWarp = 9, kFixWarp = 10;
constexpr int kPlanWarp = 11, kReaders = 11;  // the warps that follow its parts
constexpr int kThreads = 384, kPlanned = 4;
constexpr int kSoftRegs = 192, kOtherRegs = 120, kLaunchRegs = 168;
static_assert(32 * kSoftWarps * kSoftRegs + 128 * kOtherRegs <= kThreads * kLaunchRegs, "register split");

template <int DIM>
struct TilesShape {
  static constexpr int kHalf = 128 * 128;                // 128 rows of 64 elements
  static constexpr int kTileBytes = kHalf * (DIM / 64);  // a row tile's queries, or a tile of keys or values
  static constexpr int kStages = DIM == 128 ? 4 : 8;
  static constexpr int kQ = 0;
  static constexpr int kRing = 2 * kTileBytes;
  static constexpr int kKnown = kRing + kStages * kTileBytes;  // sequences of a small call
  static constexpr int kParts = kKnown + kThreads * (int)sizeof(CrossSeq);
  static constexpr int kBar = kParts + kPlanned * 48;
  static constexpr int kSmem = kBar + 512 + 1024;
  static constexpr int kO = 256;  // TMEM: the row tiles' scores at 0 and 128; accumulators from here
};

static_assert(TilesShape<64>::kStages % 2 == 0 && TilesShape<128>::kStages % 2 == 0, "keys in even stages, values in odd ones");

// What a unit and its tiles cost, in sixteenths of a tile of two row tiles: 3.0 us, 1.80 and (one row tile) 1.60 at dim 128.  (A unit
// of one row tile: 2.1 us; dim 64: 2.0, 1.66 and 1.38, 1.1.)
constexpr int kPad = 27, kTwo = 16, kOne = 14, kLeast = 64;

struct TilesArgs {
  CrossAttend a;
  float* part;      // [2 * CTAs][kUnitRows][DIM]: a unit begun by an earlier CTA; one that the next CTAs go on with
  float2* part_ml;  // (maximum, sum) of those rows
  int4* joins;      // [2 * CTAs]: the second one's place
  int k_heads, k_sources, v_heads, v_sources;  // 0: the coordinate is 0 (stride 0)
  int tokens;       // of a row tile
  bool wide;        // results allow 32-byte stores
};

// a / b; mostly small numbers
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (uint64_t)(a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

struct Line {
  int kv, tokens;  // key heads; tokens of a row tile
  __device__ __forceinline__ int units(const CrossSeq& q) const { return (q.count + 2 * tokens - 1) / (2 * tokens); }
  static __device__ __forceinline__ int tiles(const CrossSeq& q) { return max(1, (q.len + kFrames - 1) / kFrames); }
  __device__ __forceinline__ bool two(const CrossSeq& q, int u) const { return q.count - 2 * u * tokens > tokens; }
  static __device__ __forceinline__ int64_t unit(int tiles, bool two) { return kPad + (int64_t)tiles * (two ? kTwo : kOne); }
  __device__ __forceinline__ int64_t head(const CrossSeq& q) const {
    const int n = units(q), t = tiles(q);
    return n ? (n - 1) * unit(t, true) + unit(t, two(q, n - 1)) : 0;
  }
  __device__ __forceinline__ int64_t seq(const CrossSeq& q) const { return kv * head(q); }
};

// One CTA's share of a unit.
struct alignas(16) Part {
  int row0, count, head, tok0;  // the sequence's rows; the key head; the unit's first token
  int source, len, lo, hi;      // tiles of frames lo .. hi - 1 ...
  int all, n, what, last;       // ... of all; those to compute (0: a row sees nothing; -1: no part, the last one was); the CTA of the unit's last tile
  static constexpr int kTwo = 1, kOk = 2;  // `what`: two row tiles; the sequence is in range
  __device__ __forceinline__ bool two() const { return what & kTwo; }
  __device__ __forceinline__ bool ok() const { return what & kOk; }
};
static_assert(sizeof(Part) == 48, "");

// The parts of a CTA in order: places lo .. hi - 1 of the line, from sequence i (which begins at place `at`)
// on.  A warp holds 32 sequences at a time.
struct Walk {
  const CrossAttend& a;
  const CrossSeq* known;  // [n], or NULL: in the call's arrays
  Line line;
  int64_t at, lo, hi;
  int lane, base, i, head, u, units, tiles;
  CrossSeq w, q;
  __device__ __forceinline__ Walk(const CrossAttend& args, const Line& l, const CrossSeq* sequences, int64_t place, int64_t from, int64_t to, int seq)
      : a(args), known(sequences), line(l), at(place), lo(from), hi(to), lane(threadIdx.x & 31), base(seq), i(seq) {
    window();
    take();
    if (units == 0) return;  // (a share begins inside a sequence)
    const int64_t per = line.head(q);
    head = (int)min(quotient(lo - at, per), (int64_t)line.kv - 1);
    at += head * per;
    u = (int)min(quotient(lo - at, Line::unit(tiles, true)), (int64_t)units - 1);
    at += u * Line::unit(tiles, true);
  }
  __device__ __forceinline__ void window() {
    w.source = w.len = w.row0 = w.count = 0, w.ok = false;
    if (base + lane < a.b.n) w = known ? known[base + lane] : cross_seq(a.s, a.b, base + lane);
  }
  __device__ __forceinline__ void take() {
    const int l = i - base;
    q.source = __shfl_sync(0xffffffffu, w.source, l);
    q.len = __shfl_sync(0xffffffffu, w.len, l);
    q.row0 = __shfl_sync(0xffffffffu, w.row0, l);
    q.count = __shfl_sync(0xffffffffu, w.count, l);
    q.ok = __shfl_sync(0xffffffffu, (int)w.ok, l);
    units = line.units(q), tiles = Line::tiles(q), head = 0, u = 0;
  }
  __device__ __forceinline__ bool sequence() {  // the next one with rows
    while (true) {
      const unsigned some = __ballot_sync(0xffffffffu, w.count > 0 && base + lane > i);
      if (some) {
        i = base + __ffs(some) - 1;
        take();
        return true;
      }
      base += 32;
      i = base - 1;
      if (base >= a.b.n) return false;
      window();
    }
  }
  __device__ __forceinline__ bool next(Part& p, int64_t share, int ctas) {
    while (at < hi) {
      if (u >= units) {
        u = 0;
        if (++head >= line.kv && !sequence()) return false;
      }
      if (units == 0) return false;
      const bool two = line.two(q, u);
      const auto first = [&](int64_t place) {  // the first tile that begins there or later
        const int64_t x = place - at - kPad;
        if (x <= 0) return 0;
        if (x >= (int64_t)tiles * (two ? kTwo : kOne)) return tiles;
        const uint32_t y = (uint32_t)x;
        return (int)(two ? (y + kTwo - 1) / kTwo : (y + kOne - 1) / kOne);
      };
      p.row0 = q.row0, p.count = q.count, p.head = head, p.tok0 = 2 * u * line.tokens;
      p.source = q.source, p.len = q.len, p.lo = first(lo), p.hi = first(hi);
      p.all = tiles, p.n = q.ok && q.len > 0 ? p.hi - p.lo : 0, p.what = (two ? Part::kTwo : 0) | (q.ok ? Part::kOk : 0);
      p.last = 0;
      if (p.lo == 0 && p.hi > 0 && p.hi < tiles) p.last = (int)min(quotient(at + kPad + (int64_t)(tiles - 1) * (two ? kTwo : kOne), share), (int64_t)ctas - 1);
      at += Line::unit(tiles, two);
      ++u;
      if (p.hi > p.lo) return true;
    }
    return false;
  }
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
               : "memory");
}

// Eight words at a 16-byte, or (wide) 32-byte boundary: the lanes' rows lie apart, and a whole sector goes out at once.
__device__ __forceinline__ void store32(uint16_t* to, const uint32_t (&z)[8], bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(z[0]), "r"(z[1]), "r"(z[2]), "r"(z[3]), "r"(z[4]), "r"(z[5]),
                 "r"(z[6]), "r"(z[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(to)[0] = make_uint4(z[0], z[1], z[2], z[3]);
    reinterpret_cast<uint4*>(to)[1] = make_uint4(z[4], z[5], z[6], z[7]);
  }
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z, int w) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
               : "memory");
}

template <bool BF16, int DIM>
__global__ void __launch_bounds__(kThreads, 1) k_cross_tiles(const __grid_constant__ TilesArgs args, const __grid_constant__ CUtensorMap q_map,
                                                             const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using S = TilesShape<DIM>;
  constexpr int ST = S::kStages;
  extern __shared__ unsigned char smem_raw[];
  __shared__ int64_t s_sums[kThreads / 32], s_upto[kThreads];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::kBar);
  uint64_t *full = bars, *empty = bars + ST, *v_ready = bars + 2 * ST;  // the ring's stages; those of values past warp 10
  uint64_t *s_full = v_ready + ST / 2, *o_half = s_full + 2, *o_full = s_full + 4, *p_full = s_full + 6;  // [2] row tiles; [2][2] and halves of a step
  uint64_t *q_full = s_full + 10, *q_empty = s_full + 11, *drain = s_full + 12;
  uint64_t *part_full = s_full + 13, *part_empty = part_full + kPlanned;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(part_empty + kPlanned);
  Part* plan = reinterpret_cast<Part*>(smem + S::kParts);
  const CrossAttend& a = args.a;
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const Line line{a.s.kv_heads, args.tokens};

  // The line's length and this CTA's share: a thread's run of sequences, then the threads'.
  const int run = (a.b.n + kThreads - 1) / kThreads, run0 = min((int)threadIdx.x * run, a.b.n), run1 = min(run0 + run, a.b.n);
  CrossSeq* known = run == 1 ? reinterpret_cast<CrossSeq*>(smem + S::kKnown) : nullptr;
  int64_t mine = 0;
  for (int i = run0; i < run1; ++i) {
    const CrossSeq q = cross_seq(a.s, a.b, i);
    if (known) known[i] = q;
    mine += line.seq(q);
  }
  int64_t upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  s_upto[threadIdx.x] = upto;
  if (lane == 31) s_sums[warp] = upto;
  if (warp == kTmaWarp && lane < 3)
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(lane == 0 ? &q_map : lane == 1 ? &k_map : &v_map)) : "memory");
  if (threadIdx.x == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, 1);
    }
    for (int i = 0; i < ST / 2; ++i) mbar_init(v_ready + i, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + i, 1);
      mbar_init(o_half + i, 1);
      mbar_init(o_full + i, 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(p_full + i, 4);
    for (int i = 0; i < kPlanned; ++i) {
      mbar_init(part_full + i, 1);
      mbar_init(part_empty + i, kReaders);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *tmem_slot;
  int64_t total = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) total += s_sums[i];
  const int64_t share = max(quotient(total + gridDim.x - 1, gridDim.x), (int64_t)kLeast);
  const int64_t lo = share * blockIdx.x, hi = min(lo + share, total);
  if (lo >= hi) {
    if (args.joins && threadIdx.x == 0) args.joins[2 * blockIdx.x + 1].x = -1;
    if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    return;
  }
  Part p;
  int seen = 0;
  const auto next = [&] {  // the next part; false: there is none
    const int s = seen % kPlanned;
    if (!__all_sync(0xffffffffu, mbar_wait(part_full + s, (uint32_t)(seen / kPlanned) & 1u, 16 * kWaitNs))) return false;
    p = plan[s];
    __syncwarp();
    if (lane == 0) mbar_arrive(part_empty + s);
    ++seen;
    return p.n >= 0;
  };
  // A wait that runs out ends what its role does (it goes on to follow the parts); the others' waits on it
  // run out in turn, and the rows from there on say NaN.
  if (warp < kSoftWarps) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    const int tile = warp >> 2;
    const int row = threadIdx.x % 128, row_tok = tile * args.tokens + row / a.group, row_h = row % a.group;  // the thread's, of a unit
    const bool used = row < args.tokens * a.group;
    const uint32_t st = tmem + (uint32_t)(tile * 128) + ((uint32_t)((warp & 3) * 32) << 16);  // scores, then weights
    const uint32_t ot = tmem + (uint32_t)(S::kO + tile * DIM) + ((uint32_t)((warp & 3) * 32) << 16);
    // (not 0: what no row may see is an infinite score; the least factor leaves the others 0)
    const float c = a.scale * kLog2e == 0.f ? 0x1p-120f : a.scale * kLog2e;
    const float sign = c < 0.f ? -1.f : 1.f;
    // A score is the product times c less the maximum's, rounded once: off by half a step of that maximum, above 2^26 (or below -2^26)
    // more than an exponent should be.  There c is the next power of two, so that the maximum's own is 0: of such scores
    // any two that differ do so by so much that the lower weighs nothing (by 4 at least, times c's change).
    constexpr float kFar = 0x1p26f;
    const float c_far = sign * __uint_as_float((__float_as_uint(fabsf(c)) + 0x7fffffu) & 0x7f800000u);
    const float nan = __uint_as_float(0x7fc00000u);
    int at0 = 0, done = 0;  // steps and parts of this row tile so far
    bool fine = true, join = false;
    while (next()) {
      const int tok = p.tok0 + row_tok;
      const bool live = used && tok < p.count;
      uint16_t* const dst = a.out + (int64_t)(p.row0 + tok) * a.out_row + (int64_t)(p.head * a.group + row_h) * a.out_head;
      const bool whole_unit = p.lo == 0 && p.hi == p.all;
      const int slot = 2 * (int)blockIdx.x + (p.lo == 0 ? 1 : 0);
      if (!whole_unit && p.lo == 0) {
        join = true;
        if (threadIdx.x == 0) {
          args.joins[slot - 1] = make_int4(p.row0, p.count, p.tok0, p.head);
          args.joins[slot].x = p.last;
        }
      }
      if (p.n == 0 || !fine) {
        if (live) {
          const uint32_t x = p.ok() && fine ? 0u : BF16 ? 0x7fc07fc0u : 0x7e007e00u;
          if (whole_unit) {
            for (int i = 0; i < DIM / 8; ++i) reinterpret_cast<uint4*>(dst)[i] = make_uint4(x, x, x, x);
          } else {
            args.part_ml[(size_t)slot * kUnitRows + threadIdx.x] = make_float2(0.f, nan);
          }
        }
        continue;
      }
      bool dead = false;
      if (tile == 0 || p.two()) {
        float m = -INFINITY, l = 0.f, factor = c;  // (of the row: c, or c_far as its maximum is)
#pragma unroll 1
        for (int j = 0; j < p.n; ++j) {
          if (!__all_sync(0xffffffffu, mbar_wait(s_full + tile, (uint32_t)(at0 + j) & 1u))) {
            dead = true;
            break;
          }
          fence_after();
          const int left = p.len - (p.lo + j) * kFrames;  // frames from here on
          if (left < kFrames) {  // the last tile: what lies behind the length becomes a score that gives weight 0
            const float none = sign * -INFINITY;
#pragma unroll 1
            for (int b = left / 16; b < kFrames / 16; ++b) {
              float v[16];
              tmem_ld16(st + 16 * b, v);
              uint32_t z[16];
#pragma unroll
              for (int e = 0; e < 16; ++e) z[e] = __float_as_uint(16 * b + e < left ? v[e] : none);
              tmem_st16(st + 16 * b, z);
            }
            tmem_st_wait();
          }
          // 64 frames, then 64: the first ones' values' product runs while the others' weights are
          // made.  Weights are relative to the maximum so far, without looking for that of these 64: one
          // that a score has outgrown shows in the sum, and they are taken again from their
          // scores, which the weights have not replaced yet.  (Sums up to 2^15: no weight then
          // reaches fp16's largest.)
          uint32_t raw[2][32];  // 32 scores are on their way while the ones before are worked on
          tmem_ld32_begin(st, raw[0]);
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {
            if (h == 1 && left <= 64) {  // nothing to see: no product reads these weights
              tmem_ld32_wait(raw[0]);
              __syncwarp();
              if (lane == 0) mbar_arrive(p_full + 2 * tile + 1);
              break;
            }
            uint32_t y[32], rest[32];  // the weights' two parts
            float sum;
            bool look = h == 0 && j == 0;
#pragma unroll 1
            while (true) {
              if (look) {
                float top = -INFINITY;
                tmem_ld32_wait(raw[0]);
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                  float v[32];
                  tmem_ld32(st + 64 * h + 32 * b, v);
#pragma unroll
                  for (int e = 0; e < 32; ++e) top = fmaxf(top, v[e] * sign);
                }
                const float near = top * fabsf(c);
                top = fabsf(near) < kFar ? near : top * fabsf(c_far);
                float w = 1.f;
                if (top > m) {
                  w = ex2_approx(m - top);
                  m = top;
                  factor = fabsf(near) < kFar ? c : c_far;
                }
                l *= w;
                if (j > 0 || h > 0) {
                  // the last step's values are in the accumulator (this one's scores came after them); the first 64's
                  if (h == 1 && !__all_sync(0xffffffffu, mbar_wait(o_half + tile, (uint32_t)(at0 + j) & 1u))) {
                    dead = true;
                    break;
                  }
                  fence_after();
#pragma unroll 1
                  for (int ch = 0; ch < DIM / 16; ++ch) {
                    float o[16];
                    tmem_ld16(ot + 16 * ch, o);
                    uint32_t z[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) z[e] = __float_as_uint(o[e] * w);
                    tmem_st16(ot + 16 * ch, z);
                  }
                }
                tmem_ld32_begin(st + 64 * h, raw[0]);
              }
              // (no maximum yet, every score so far -inf: any other has outgrown the least number)
              const float ref = m > -INFINITY ? m - 7.f : look ? 0.f : -3.4e38f;
              const uint64_t ref2 = pair_of(-ref, -ref), c2 = pair_of(factor, factor);
              uint64_t sums[2] = {0, 0};  // (four take registers that there are not: 205 us where two take 200, 6 x 1100 over 9000, fp16)
#pragma unroll
              for (int b = 0; b < 2; ++b) {
                tmem_ld32_wait(raw[b]);
                if (b == 0) tmem_ld32_begin(st + 64 * h + 32, raw[1]);
                else if (h == 0) tmem_ld32_begin(st + 64, raw[0]);
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                  float x0, x1;
                  unpair(fma2(pair_of(__uint_as_float(raw[b][e]), __uint_as_float(raw[b][e + 1])), c2, ref2), x0, x1);
                  const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
                  sums[e / 2 & 1] = add2(sums[e / 2 & 1], pair_of(p0, p1));
                  weight_parts<BF16>(p0, p1, y[16 * b + e / 2], rest[16 * b + e / 2]);
                }
              }
              float s0, s1;
              unpair(add2(sums[0], sums[1]), s0, s1);
              sum = s0 + s1;
              if (look || !__any_sync(0xffffffffu, live && sum > 32768.f)) break;
              look = true;
            }
            if (dead) break;
            l += sum;
            tmem_st32(st + 64 * h, y);
            tmem_st32(st + 64 * h + 32, rest);
            tmem_st_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full + 2 * tile + h);
          }
          if (dead) break;
        }
        if (!dead && !mbar_wait(o_full + tile, (uint32_t)done & 1u)) dead = true;
        fence_after();
        dead = __any_sync(0xffffffffu, dead);
        if (dead) l = nan;
        // results: a thread its row
        if (whole_unit) {
          const float inv = 1.f / l;
#pragma unroll
          for (int ch = 0; ch < DIM / 32; ++ch) {
            float v[32];
            tmem_ld32(ot + 32 * ch, v);
            if (live)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                uint32_t z[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = narrow2<BF16>(v[16 * i + 2 * e] * inv, v[16 * i + 2 * e + 1] * inv);
                store32(dst + 32 * ch + 16 * i, z, args.wide);
              }
          }
        } else {  // [DIM / 4][rows] of four: neighbouring lanes write a column
          float4* to = reinterpret_cast<float4*>(args.part) + (size_t)slot * (DIM / 4) * kUnitRows + threadIdx.x;
#pragma unroll
          for (int ch = 0; ch < DIM / 32; ++ch) {
            float v[32];
            tmem_ld32(ot + 32 * ch, v);
            if (live)
#pragma unroll
              for (int i = 0; i < 8; ++i) to[(8 * ch + i) * kUnitRows] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
          }
          if (live) args.part_ml[(size_t)slot * kUnitRows + threadIdx.x] = make_float2(m, l);
        }
        at0 += p.n;
        ++done;
      }
      fence_before();
      fine = !dead;
    }
    if (threadIdx.x == 0 && args.joins && !join) args.joins[2 * blockIdx.x + 1].x = -1;
    asm volatile("bar.arrive 2, %0;" ::"n"(32 * (kSoftWarps + 1)) : "memory");
    return;
  }
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));  // one instruction for the whole warpgroup
  if (warp == kTmaWarp) {
    uint32_t at = 0, parts = 0;  // tiles through the ring, keys and values; parts with any
    bool dead = false;
    while (next()) {
      if (!dead && elect()) {
        bool asked = false;
        for (int j = 0; j < p.n && !dead; ++j) {
#pragma unroll
          for (int kind = 0; kind < 2 && !dead; ++kind, ++at) {
            const int s = at % ST;
            if (at >= ST && !mbar_wait(empty + s, (at / ST - 1) & 1u)) {
              dead = true;
              break;
            }
            mbar_expect_tx(full + s, S::kTileBytes);
#pragma unroll
            for (int h = 0; h < DIM / 64; ++h)
              tma_load_4d(smem_u32(smem + S::kRing + s * S::kTileBytes + h * S::kHalf), kind ? &v_map : &k_map, full + s, 64 * h, (p.lo + j) * kFrames,
                          kind ? p.head * args.v_heads : p.head * args.k_heads, kind ? p.source * args.v_sources : p.source * args.k_sources);
            if (j == 0 && kind == 0) {  // the queries, once the last part's have been used
              if (parts > 0 && !mbar_wait(q_empty, (parts - 1) & 1u)) {
                dead = true;
                ++at;
                break;
              }
              const int tiles = p.two() ? 2 : 1;
              mbar_expect_tx(q_full, tiles * (DIM / 64) * args.tokens * a.group * 128);
              for (int t = 0; t < tiles; ++t)
#pragma unroll
                for (int h = 0; h < DIM / 64; ++h)
                  tma_load_3d(smem_u32(smem + S::kQ + t * S::kTileBytes + h * S::kHalf), &q_map, q_full, 64 * h, p.head * a.group,
                              p.row0 + p.tok0 + t * args.tokens);
              asked = true;
            }
          }
        }
        if (dead) {  // what is on its way ends first
          for (uint32_t i = at - min(at, (uint32_t)ST); i < at; ++i) mbar_wait(full + i % ST, (i / ST) & 1u);
          if (asked) mbar_wait(q_full, parts & 1u);
        }
      }
      parts += p.n > 0;
      dead = __any_sync(0xffffffffu, dead);
      at = __reduce_max_sync(0xffffffffu, at);
    }
  } else if (warp == kFixWarp) {
    uint32_t at = 0;
    bool dead = false;
    while (next()) {
      const bool fix = p.hi == p.all && p.len % 16;
      for (int j = 0; j < p.n && !dead; ++j, at += 2) {
        const uint32_t v = at + 1;
        if (!__all_sync(0xffffffffu, mbar_wait(full + v % ST, (v / ST) & 1u))) {
          dead = true;
          break;
        }
        if (fix && j == p.n - 1) {
          const int from = p.len - (p.all - 1) * kFrames, to = (from + 15) & ~15;
          unsigned char* tile = smem + S::kRing + (v % ST) * S::kTileBytes;
          for (int i = lane; i < (to - from) * (DIM / 8); i += 32) {
            const int f = from + i / (DIM / 8), c = i % (DIM / 8);
            *reinterpret_cast<uint4*>(tile + (c >> 3) * S::kHalf + f * 128 + ((c & 7) << 4)) = make_uint4(0, 0, 0, 0);
          }
          fence_async_smem();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(v_ready + v % ST / 2);
      }
    }
  } else if (warp == kMmaWarp) {
    uint32_t at0 = 0, parts = 0, tile_at[2] = {0, 0};
    bool dead = false;
    while (next()) {
      if (p.n == 0 || dead) continue;
      const int n = p.n, tiles = p.two() ? 2 : 1;
      const bool ends = p.hi == p.all;
      const int rest = p.len - (p.all - 1) * kFrames;  // of the last tile
      if (elect()) {
        const uint32_t sq = smem_u32(smem + S::kQ), ring = smem_u32(smem + S::kRing);
        bool ok = mbar_wait(q_full, parts & 1u);
        const auto have = [&](uint32_t at) {
          const bool there = mbar_wait(full + at % ST, (at / ST) & 1u);
          fence_after();
          return there;
        };
        const auto scores = [&](int t, int j) {
          const uint32_t at = at0 + 2 * (uint32_t)j, qa = sq + t * S::kTileBytes, kb = ring + (at % ST) * S::kTileBytes;
#pragma unroll
          for (int kk = 0; kk < DIM / 16; ++kk)
            mma_f16_ss(tmem + t * 128, sw128_desc(qa + (kk >> 2) * S::kHalf) + 2 * (kk & 3), sw128_desc(kb + (kk >> 2) * S::kHalf) + 2 * (kk & 3),
                       idesc_f16(128, kFrames, false, BF16), kk > 0);
          mma_commit(s_full + t);
          if (t == tiles - 1) mma_commit(empty + at % ST);
          if (t == tiles - 1 && j == n - 1) mma_commit(q_empty);
        };
        const auto values = [&](int t, int j, int h) {
          const uint32_t at = at0 + 2 * (uint32_t)j + 1, vb = ring + (at % ST) * S::kTileBytes;
          const int steps = ends && j == n - 1 ? (rest + 15) / 16 : kFrames / 16;  // frames behind the length stay out
#pragma unroll
          for (int k = 0; k < kFrames / 32; ++k) {
            const int kk = h * (kFrames / 32) + k;
            if (kk < steps) {
              const uint32_t w = tmem + t * 128 + 64 * h + 8 * k;
              const uint64_t v = sw128_mn_desc(vb + kk * 2048, S::kHalf);
              mma_f16_ts(tmem + S::kO + t * DIM, w, v, idesc_f16(128, DIM, true, BF16), j > 0 || kk > 0);
              mma_f16_ts(tmem + S::kO + t * DIM, w + 32, v, idesc_f16(128, DIM, true, BF16), true);
            }
          }
          if (h == 0) {
            mma_commit(o_half + t);
            return;
          }
          if (j == n - 1) mma_commit(o_full + t);
          if (t == tiles - 1) mma_commit(empty + at % ST);
        };
        if (ok) ok = have(at0);
        for (int t = 0; t < tiles && ok; ++t) scores(t, 0);
        for (int j = 0; j < n && ok; ++j) {
          for (int t = 0; t < tiles && ok; ++t) {
            ok = mbar_wait(p_full + 2 * t, (tile_at[t] + j) & 1u);
            if (ok && t == 0) ok = have(at0 + 2 * j + 1);
            if (ok && t == 0) ok = mbar_wait(v_ready + (at0 + 2 * j + 1) % ST / 2, ((at0 + 2 * j + 1) / ST) & 1u);
            if (!ok) break;
            fence_after();
            values(t, j, 0);
            ok = mbar_wait(p_full + 2 * t + 1, (tile_at[t] + j) & 1u);
            if (!ok) break;
            fence_after();
            values(t, j, 1);
            if (j + 1 < n) {
              if (t == 0) ok = have(at0 + 2 * j + 2);
              if (ok) scores(t, j + 1);
            }
          }
        }
        if (!ok) {  // the rows say NaN, once their own waits have run out; what was issued ends first
          mma_commit(drain);
          mbar_wait(drain, 0);
          dead = true;
        }
      }
      __syncwarp();
      ++parts;
      at0 += 2 * (uint32_t)n;
      tile_at[0] += n;
      if (p.two()) tile_at[1] += n;
      dead = __any_sync(0xffffffffu, dead);
    }
    asm volatile("bar.sync 2, %0;" ::"n"(32 * (kSoftWarps + 1)) : "memory");  // the accumulators have been read
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  } else if (warp == kPlanWarp) {
    // the thread whose run of sequences holds place lo, among the warps' sums, then among a warp's threads
    int64_t place = 0, sum = s_sums[0];
    int w = 0;
    while (place + sum <= lo) place += sum, sum = s_sums[++w];
    const int first = __ffs(__ballot_sync(0xffffffffu, place + s_upto[32 * w + lane] > lo)) - 1;
    if (first > 0) place += s_upto[32 * w + first - 1];
    int i = (32 * w + first) * run;
    if (run > 1)
      while (true) {
        const int64_t x = line.seq(cross_seq(a.s, a.b, i));
        if (lo < place + x || i + 1 >= a.b.n) break;
        place += x, ++i;
      }
    Walk walk(a, line, known, place, lo, hi, i);
    bool more = true;
    for (int n = 0; more; ++n) {
      const int s = n % kPlanned;
      more = walk.next(p, share, gridDim.x);
      if (!more) p.n = -1;
      if (n >= kPlanned && !__all_sync(0xffffffffu, mbar_wait(part_empty + s, (uint32_t)(n / kPlanned - 1) & 1u, 8 * kWaitNs))) break;
      if (lane == 0) {
        plan[s] = p;
        mbar_arrive(part_full + s);
      }
      __syncwarp();
    }
  }
}

// The units that several CTAs share: blocks (c, ..) take the one that CTA c began.
// A warp takes 32 rows and 16 of their dimensions.
template <bool BF16, int DIM>
__global__ void __launch_bounds__(DIM) k_cross_join(const __grid_constant__ TilesArgs args) {
  const int c = blockIdx.x, warp = blockIdx.z * (DIM / 32) + (threadIdx.x >> 5), rr = blockIdx.y * 32 + (threadIdx.x & 31), row = rr % 128;
  const CrossAttend& a = args.a;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int4 place = args.joins[2 * c];  // the sequence's first row and its tokens, the unit's first token, the key head
  const int parts = args.joins[2 * c + 1].x - c + 1, tok = place.z + rr / 128 * args.tokens + row / a.group;
  if (parts < 2 || row >= args.tokens * a.group || tok >= place.y) return;
  const auto slot = [&](int k) { return (size_t)(k == 0 ? 2 * c + 1 : 2 * (c + k)); };
  // (kAtOnce parts' loads are on their way together; one that is not there has weight 0)
  constexpr int kAtOnce = 4;
  float top = -INFINITY;
  for (int k0 = 0; k0 < parts; k0 += 2 * kAtOnce) {
    float x[2 * kAtOnce];
#pragma unroll
    for (int k = 0; k < 2 * kAtOnce; ++k) x[k] = k0 + k < parts ? args.part_ml[slot(k0 + k) * kUnitRows + rr].x : -INFINITY;
#pragma unroll
    for (int k = 0; k < 2 * kAtOnce; ++k) top = fmaxf(top, x[k]);
  }
  float acc[16], sum = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
  for (int k0 = 0; k0 < parts; k0 += kAtOnce) {
    float2 x[kAtOnce];
    float4 v[kAtOnce][4];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      x[k] = make_float2(0.f, 0.f);
      if (k0 + k < parts) {
        const size_t at = slot(k0 + k);
        x[k] = args.part_ml[at * kUnitRows + rr];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[k][i] = reinterpret_cast<const float4*>(args.part)[(at * (DIM / 4) + 4 * warp + i) * kUnitRows + rr];
      }
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      if (k0 + k < parts) {
        const float f = x[k].x == top ? 1.f : ex2_approx(x[k].x - top);  // (top -inf: every score is, and 0 / 0 is the result)
        sum = fmaf(f, x[k].y, sum);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[4 * i] = fmaf(f, v[k][i].x, acc[4 * i]), acc[4 * i + 1] = fmaf(f, v[k][i].y, acc[4 * i + 1]);
          acc[4 * i + 2] = fmaf(f, v[k][i].z, acc[4 * i + 2]), acc[4 * i + 3] = fmaf(f, v[k][i].w, acc[4 * i + 3]);
        }
      }
  }
  const float inv = 1.f / sum;
  uint32_t z[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = narrow2<BF16>(acc[2 * e] * inv, acc[2 * e + 1] * inv);
  store32(a.out + (int64_t)(place.x + tok) * a.out_row + (int64_t)(place.w * a.group + row % a.group) * a.out_head + 16 * warp, z, args.wide);
}

// Keys or values as [sources][heads][frames][dim], a dimension of stride 0 as one of size 1.
bool make_states_map(CUtensorMap* m, const tsd_states& s, const void* base, int64_t source, int64_t frame, int64_t head) {
  const EncodeTiledFn fn = encode_fn();
  if (!fn || frame < s.dim) return false;
  const auto stride = [&](int64_t x, int64_t size) { return (cuuint64_t)(size > 1 && x ? x : s.dim) * 2; };
  const cuuint64_t dims[4] = {(cuuint64_t)s.dim, (cuuint64_t)s.frames, (cuuint64_t)(head ? s.kv_heads : 1), (cuuint64_t)(source ? s.n_sources : 1)};
  const cuuint64_t strides[3] = {stride(frame, s.frames), stride(head, s.kv_heads), stride(source, s.n_sources)};
  const cuuint32_t box[4] = {64, kFrames, 1, 1}, es[4] = {1, 1, 1, 1};
  return fn(m, s.dtype == TSD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Queries as [rows][heads][dim], in boxes of a row tile's tokens and a key head's heads.
bool make_queries_map(CUtensorMap* m, const CrossAttend& a, int tokens) {
  const EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)a.s.dim, (cuuint64_t)a.heads, (cuuint64_t)a.b.rows};
  const cuuint64_t strides[2] = {(cuuint64_t)(a.heads > 1 ? a.q_head : a.s.dim) * 2, (cuuint64_t)(a.b.rows > 1 ? a.q_row : a.s.dim) * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)a.group, (cuuint32_t)tokens}, es[3] = {1, 1, 1};
  return fn(m, a.s.dtype == TSD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<uint16_t*>(a.q), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool BF16, int DIM>
cudaError_t launch(const TilesArgs& args, const CrossTilesPlan& p, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t s) {
  using S = TilesShape<DIM>;
  static const bool enough = [] {  // setmaxnreg waits for registers that the launch did not bring
    cudaFuncAttributes at{};
    return cudaFuncGetAttributes(&at, k_cross_tiles<BF16, DIM>) == cudaSuccess && at.numRegs >= kLaunchRegs;
  }();
  if (!enough) return cudaErrorLaunchOutOfResources;
  const cudaError_t e = smem_opt_in<k_cross_tiles<BF16, DIM>>(S::kSmem);
  if (e != cudaSuccess) return e;
  k_cross_tiles<BF16, DIM><<<p.ctas, kThreads, S::kSmem, s>>>(args, q, k, v);
  const cudaError_t launched = cudaGetLastError();
  if (launched != cudaSuccess || p.bytes == 0) return launched;
  cudaLaunchConfig_t c{};
  c.gridDim = dim3((unsigned)p.ctas, kUnitRows / 32, 2);
  c.blockDim = DIM;
  c.stream = s;
  cudaLaunchAttribute at{};  // its blocks come while the last CTAs end, and wait for them
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  c.attrs = &at;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, k_cross_join<BF16, DIM>, args);
}

}  // namespace

bool cross_tiles_plan(const tsd_states& s, const tsd_cross_batch& b, int heads, int sms, CrossTilesPlan* p) {
  const int group = heads / s.kv_heads;
  const int64_t most = std::max<int64_t>(1, b.max_rows ? std::min(b.max_rows, b.rows) : !b.starts ? 1 : ((int64_t)b.rows + b.n - 1) / b.n);
  if (s.k_frame < s.dim || s.v_frame < s.dim) return false;
  // cross_rows.cu's time grows with its units of 16 rows, each of which reads the frames again (0.016 us + 0.047 us per 1000 frames at dim 128,
  // half of that at 64), this kernel's starts at 9 to 15 us.  Here and there, us, ragged (from 0.4 of the sizes on), dim 128: 64 sources of 100 frames,
  // 8 key heads: 20 rows 15 and 15, 64 rows 16 and 23; 4 of 300, 4 key heads: 64 rows 14 and 7, 500 rows 18 and 12; 24 of 500, 8: 24 rows 18 and
  // 20; one of 9000, 4: 64 rows 20 and 23; one of 20000, 8: 17 rows 30 and 44.  Dim 64, 8 key heads, 64 of 400: 20 rows 24 and 16, 40 rows 24 and 21;
  // 24 of 900: 48 rows 20 and 20; 2 of 15000: 40 rows 26 and 27; 32 of 300: 40 rows 16 and 11.  (From the bounds on to twice them
  // the other kernel is often the faster one still.)
  const int64_t sixteens = (most * group + 15) / 16;
  if (sixteens < 2) return false;
  const bool much = sixteens > (s.dim == 64 ? 2 : 1) && (double)b.n * s.kv_heads * sixteens * (s.frames + 330.0) >= (s.dim == 64 ? 350e3 : 200e3);
  if (!much && s.frames <= 8000) return false;
  const int64_t tiles = ((int64_t)s.frames + kFrames - 1) / kFrames;
  const int64_t units = s.kv_heads * ((int64_t)b.rows / (2 * (128 / group)) + b.n);  // at most
  const double line = (double)units * (double)(kPad + tiles * kTwo);
  p->ctas = (int)std::max(1.0, std::min((double)sms, std::ceil(line / kLeast)));
  // one tile of frames is never shared
  p->bytes = tiles > 1 && p->ctas > 1 ? (int64_t)p->ctas * 2 * (kUnitRows * (s.dim * 4 + 8) + 16) : 0;
  return true;
}

cudaError_t cross_tiles_launch(const CrossAttend& a, const CrossTilesPlan& p, void* workspace, cudaStream_t s) {
  const bool bf = a.s.dtype == TSD_BF16;
  const int tokens = 128 / a.group;
  CUtensorMap q, k, v;
  if (!make_queries_map(&q, a, tokens) || !make_states_map(&k, a.s, a.s.k, a.s.k_source, a.s.k_frame, a.s.k_head) || !make_states_map(&v, a.s, a.s.v, a.s.v_source, a.s.v_frame, a.s.v_head))
    return cudaErrorInvalidValue;
  TilesArgs t{};
  t.a = a;
  if (p.bytes > 0) {
    t.part = static_cast<float*>(workspace);
    t.part_ml = reinterpret_cast<float2*>(t.part + (size_t)2 * p.ctas * kUnitRows * a.s.dim);
    t.joins = reinterpret_cast<int4*>(t.part_ml + (size_t)2 * p.ctas * kUnitRows);
  }
  t.tokens = tokens;
  t.wide = reinterpret_cast<uintptr_t>(a.out) % 32 == 0 && a.out_row % 16 == 0 && a.out_head % 16 == 0;
  t.k_heads = a.s.k_head != 0, t.k_sources = a.s.k_source != 0, t.v_heads = a.s.v_head != 0, t.v_sources = a.s.v_source != 0;
  return a.s.dim == 64 ? (bf ? launch<true, 64>(t, p, q, k, v, s) : launch<false, 64>(t, p, q, k, v, s))
                       : (bf ? launch<true, 128>(t, p, q, k, v, s) : launch<false, 128>(t, p, q, k, v, s));
}

}  // namespace tsd
