// Attention over the 8-bit paged cache with many query rows per key head:
// prompts (tsd.h: tsd_kv8_attend).
//
// The mathematics is kv8_rows.cu's, but for when the maximum follows (below); the products run on tcgen05 (fp16 in, fp32
// accumulate in TMEM).  A CTA takes 256 rows of a sequence and key head (row =
// token * group + head of the group) as two tiles of 128, and the keys they see in
// tiles of 128, 64 at a time:
//   warps 0-7   softmax: a thread is a row (warps 0-3 tile 0, 4-7 tile 1), so its
//               maximum, sum and masks need no exchange.  Reads its 64 scores from TMEM,
//               leaves probabilities (fp16) in their place as the values'
//               product's A operand;
//   warps 8-15  turn the integers of the next key tile into fp16 in shared memory
//               (128-byte swizzle; warps 8-11 keys, 12-15 values), once for both row
//               tiles and all heads of a group;
//   warp 16     issues the MMAs;
//   warp 17     puts each key tile's scales, and the value scales' logarithms and reciprocals,
//               into shared memory for the softmax.
// Registers go to where they are used (setmaxnreg): 144 for softmax, 72 for conversion.
// Queries come and results leave through shared memory, a row's bytes by neighbouring
// lanes; a CTA's first queries are on their way while it sets up.
// Each row tile has two score buffers of 64 keys: the scores of step i + 2 are computed
// as soon as the values' product of step i has read its probabilities, so the softmax
// never waits for a product that waits for it.  (With one buffer of 128 keys a tile's
// softmax, 3700 clocks, and its products, 1600, took turns.)  Keys are the K-major B
// operand of the scores; the same layout of the values is read as an MN-major B
// operand, so neither is transposed.  The maximum is looked for, and the accumulator rescaled in
// TMEM, only in steps whose probabilities outgrow fp16, and in which a row sees its first key.
//
// Measured (16 query and 4 key heads of 128, bf16): 2000 clocks per step of 64 keys and 256
// rows, of which the MMAs are 1300 (49 for 128 x 64 x 16, whose operands come from shared
// memory at 128 bytes per clock, 65 for 128 x 128 x 16 with A in TMEM), and 16000 per CTA
// before the first step and after the last: 4 ragged sequences of 4000 new tokens past 2000
// take 248 us (0.50 of the MMAs' floor at the library's rate), one of 2432 past 16000 292
// us (0.61).  A step's 2000 are the softmax's at dim 64 too (1930): two of its warps per scheduler
// wait for scores, for TMEM and for one another's 2^x in turn, at half of the issue slots.
#include <algorithm>
#include <climits>

#include "kv8_attend.h"
#include "launch.h"
#include "tc_common.cuh"

namespace tsd {

namespace {

using namespace tc;

constexpr int kUnit = kKv8Unit;
constexpr int kKeys = 128;            // keys per tile
constexpr int kUnits = kKeys / kUnit;
constexpr int kStep = 64;             // keys per step
constexpr int kStepUnits = kStep / kUnit;
constexpr int kSoftWarps = 8, kConvWarps = 4;  // softmax; conversion of keys, and as many of values
constexpr int kMmaWarp = kSoftWarps + 2 * kConvWarps;
constexpr int kScaleWarp = kMmaWarp + 1;
constexpr int kThreads = 32 * (kMmaWarp + 4);  // whole warpgroups: two warps of the last have no work
constexpr int kSoftRegs = 144, kConvRegs = 72, kMmaRegs = 48;
constexpr int kLaunchRegs = 96;  // per thread, what the launch has to bring
static_assert(32 * kSoftWarps * kSoftRegs + 64 * kConvWarps * kConvRegs + 128 * kMmaRegs <= kThreads * kLaunchRegs, "register split");

template <int DIM>
struct TilesShape {
  static constexpr int kHalf = 128 * 128;              // 128 rows of 64 fp16
  static constexpr int kTileBytes = kHalf * (DIM / 64);  // a row tile's queries, or a key tile's keys or values
  static constexpr int kQ = 0;
  static constexpr int kK = 2 * kTileBytes;             // two stages
  static constexpr int kV = 4 * kTileBytes;             // two stages
  static constexpr int kBar = 6 * kTileBytes;
  static constexpr int kScales = kBar + 256;  // [stage][3][kUnits]: a key tile's key scales, log2 and reciprocal of its value scales
  static constexpr int kSmem = kScales + 2 * 3 * kUnits * 4 + 1024;
  static constexpr int kO = 256;  // TMEM: the row tiles' two score buffers at 0, 64 and 128, 192; accumulators from here
};

// fp16 operands, fp32 accumulate; bTrans: B is MN-major
constexpr uint32_t idesc_f16(int M, int N, bool b_mn) {
  return (1u << 4) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// Descriptor of an MN-major tile in the 128-byte swizzle: 64 consecutive elements of
// the N axis per 128-byte row, rows along K; eight-row groups 1024 bytes apart, the next 64
// elements of N kHalf bytes on.
__device__ __forceinline__ uint64_t sw128_mn_desc(uint32_t saddr, int next_n) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(next_n >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc)
      : "memory");
}
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc)
      : "memory");
}

// 16 columns, on their way until tmem_ld16_wait (which waits for all of the thread's loads).
__device__ __forceinline__ void tmem_ld16_begin(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld16_wait(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
      : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
        "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
      :
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
      "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]),
      "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <bool BF16, int DIM>
__global__ void __launch_bounds__(kThreads, 1) k_kv8_tiles(const __grid_constant__ Kv8Attend a) {
  using S = TilesShape<DIM>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::kBar);
  uint64_t *k_full = bars, *k_empty = bars + 2, *v_full = bars + 4, *v_empty = bars + 6;  // [2] stages
  uint64_t *s_full = bars + 8, *p_full = bars + 12;  // [row tile][buffer]
  uint64_t *o_done = bars + 16, *o_full = bars + 18;  // [2] row tiles: a step's values' product, the last one's
  uint64_t *q_full = bars + 20, *drain = bars + 21;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 22);

  float* scales = reinterpret_cast<float*>(smem + S::kScales);
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const Kv8Seq q = kv8_seq(a.c, a.b, blockIdx.y);
  const int head = blockIdx.x % a.c.kv_heads, split = blockIdx.x / a.c.kv_heads, splits = gridDim.x / a.c.kv_heads;
  const int rows = q.count * a.group;
  const int mts = (rows + 255) / 256;
  if ((int)blockIdx.z >= mts) return;

  // row r says NaN
  const auto say_nan = [&](int r) {
    if (r >= rows) return;
    const int tok = q.row0 + r / a.group, h = head * a.group + r % a.group;
    const uint32_t nan2 = BF16 ? 0x7fc07fc0u : 0x7e007e00u;
    if (splits == 1) {
      uint4* dst = reinterpret_cast<uint4*>(a.out + (int64_t)tok * a.out_row + (int64_t)h * a.out_head);
      for (int i = 0; i < DIM / 8; ++i) dst[i] = make_uint4(nan2, nan2, nan2, nan2);
    } else {
      a.part_ml[((size_t)split * a.b.rows + tok) * a.heads + h] = make_float2(0.f, __uint_as_float(0x7fc00000u));
    }
  };
  if (!q.ok) {
    if (threadIdx.x < 256)
      for (int mt = blockIdx.z; mt < mts; mt += gridDim.z) say_nan(mt * 256 + threadIdx.x);
    return;
  }

  // The softmax warps' queries and results pass through shared memory row by row, kRowLanes
  // lanes each: 16 bytes of a row of the warp's, in the 128-byte swizzle
  constexpr int kRowLanes = DIM / 8, kRowsPer = 32 / kRowLanes;
  const auto chunk = [&](int row, int c) {
    return reinterpret_cast<uint4*>(smem + S::kQ + (warp >> 2) * S::kTileBytes + (c >> 3) * S::kHalf + ((warp & 3) * 32 + row) * 128 + (((c ^ row) & 7) << 4));
  };
  const int step_tok = kRowsPer / a.group, step_h = kRowsPer % a.group;
  const auto next_row = [&](int& t, int& h) {
    t += step_tok;
    h += step_h;
    if (h >= (head + 1) * a.group) h -= a.group, ++t;
  };
  // Starts the copies of the warp's queries to where their fp16 will stand, and gives the token and
  // head of the lane's first row.  (The products have read the last row tile's: its accumulators were waited for.)
  const auto load_q = [&](int row0, int& own_tok, int& own_h) {
    const int wr = row0 + (threadIdx.x & ~31), r = wr + lane / kRowLanes;
    own_tok = r / a.group;
    own_h = head * a.group + r - own_tok * a.group;
    int t = own_tok, h = own_h;
#pragma unroll
    for (int i = 0; i < kRowLanes; ++i) {
      const int rw = i * kRowsPer + lane / kRowLanes;
      const uint16_t* src = a.q + (int64_t)(q.row0 + t) * a.q_row + (int64_t)h * a.q_head + 8 * (lane % kRowLanes);
      if (wr + rw < rows)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(chunk(rw, lane % kRowLanes))), "l"(src) : "memory");
      else
        *chunk(rw, lane % kRowLanes) = make_uint4(0, 0, 0, 0);
      next_row(t, h);
    }
  };
  int first_tok = 0, first_h = 0;
  if (warp < kSoftWarps) load_q((mts - 1 - (int)blockIdx.z) * 256, first_tok, first_h);

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(k_full + i, kConvWarps);
      mbar_init(v_full + i, kConvWarps + 1);
      mbar_init(k_empty + i, 1);
      mbar_init(v_empty + i, 1);
      mbar_init(o_done + i, 1);
      mbar_init(o_full + i, 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(s_full + i, 1);
      mbar_init(p_full + i, 4);
    }
    mbar_init(q_full, kSoftWarps);
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
  const int32_t* table = a.b.table + (size_t)q.slot * a.b.table_width;
  const int before = q.len - q.count;
  const int shift = __ffs(a.c.block) - 1;  // tokens per block: 16, 32 or 64
  // a row tile of 256 and its share of the keys
  struct Part {
    int row0, lo, n, steps;  // first row; first key tile, key tiles and steps
    bool two;
    KeyTiles units;
  };
  const auto part_of = [&](int mt) {
    Part p;
    p.row0 = (mts - 1 - mt) * 256;  // the later rows see the most keys: they go first, of all heads and sequences
    p.two = rows - p.row0 > 128;
    p.units = key_tiles(before + p.row0 / a.group, before + (min(rows, p.row0 + 256) - 1) / a.group, a.window, a.sinks);
    const KeyShare share = key_share(p.units.total, kUnits, kStepUnits, split, splits);
    p.lo = share.lo, p.n = share.n, p.steps = share.steps;
    return p;
  };
  // Every role walks the row tiles by itself (each has registers of its own number), so the
  // next one's keys and values are converted while the softmax ends this one.  A wait
  // that runs out ends its role; the others' waits on it run out in turn, and the rows from
  // there on say NaN.
  if (warp < kSoftWarps) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    const int tile = warp >> 2;
    int at0 = 0, kt0 = 0, done = 0;  // the barriers' positions: steps, key tiles and row tiles with steps so far
    int mt = (int)blockIdx.z;
    // (a warp of a row tile that has no rows must not arrive for the next one's queries early)
    const auto row_tile_end = [] { asm volatile("bar.sync 1, %0;" ::"n"(32 * kSoftWarps) : "memory"); };
    for (bool fine = true; mt < mts; mt += gridDim.z) {
      const Part pt = part_of(mt);
      const int row0 = pt.row0, lo = pt.lo, n = pt.n, steps = pt.steps;
      const KeyTiles& units = pt.units;
      const int r = row0 + threadIdx.x;
      if (!fine) {
        say_nan(r);
        row_tile_end();
        continue;
      }
      bool dead = false;
      const bool live = r < rows;
      const int wr = row0 + (threadIdx.x & ~31);  // the warp's first row
      const int tok = min(r, rows - 1) / a.group, pos = before + tok;
      int own_tok, own_h;
      if (mt == (int)blockIdx.z) own_tok = first_tok, own_h = first_h;
      else load_q(row0, own_tok, own_h);
      // the row's queries as fp16, scaled by f into [2^14, 2^15)
      float rc = 0.f;
      asm volatile("cp.async.wait_all;" ::: "memory");  // (before the next row tile's, also where nothing is to be done)
      if (steps > 0) {
        __syncwarp();
        uint32_t top2 = 0;  // magnitudes compare as integers
#pragma unroll
        for (int i = 0; i < DIM / 8; ++i) {
          const uint4 w = *chunk(lane, i);
          top2 = __vmaxu2(__vmaxu2(top2, __vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu)), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
        }
        const float top = wide16<BF16>(max(top2 & 0xffffu, top2 >> 16));
        // (a negative scale's sign too, so that a larger product is a larger score)
        const QueryScale qs = query_scale(top);
        rc = qs.fine ? fabsf(a.scale) * kLog2e / qs.f : __uint_as_float(0x7fc00000u);
        const float f = a.scale < 0.f ? -qs.f : qs.f;
#pragma unroll
        for (int i = 0; i < DIM / 8; ++i) {
          const uint4 w = *chunk(lane, i);
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
          uint32_t y[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] = narrow2<false>(wide16<BF16>(u[j] & 0xffffu) * f, wide16<BF16>(u[j] >> 16) * f);
          *chunk(lane, i) = make_uint4(y[0], y[1], y[2], y[3]);
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full);
      }
      if (tile == 0 || pt.two) {
        const uint32_t st = tmem + (uint32_t)(tile * 128) + ((uint32_t)((warp & 3) * 32) << 16);  // scores, then probabilities
        const uint32_t ot = tmem + (uint32_t)(S::kO + tile * DIM) + ((uint32_t)((warp & 3) * 32) << 16);
        // positions that every row of the warp sees
        const int all_to = before + min(wr, rows - 1) / a.group;
        const int all_from = a.window > 0 ? before + min(wr + 31, rows - 1) / a.group - a.window + 1 : 0;
        // ... and the units of the list, past the sinks, that hold nothing else
        const int seen_from = max(units.sink, (max(all_from, 0) + kUnit - 1) / kUnit - units.from + units.sink);
        const int seen_to = min(units.total, (all_to + 1) / kUnit - units.from + units.sink);
        float m = -INFINITY, l = 0.f;
        const float nan = __uint_as_float(0x7fc00000u);
#pragma unroll 1
        for (int i = 0; i < steps; ++i) {
          const int at = at0 + i, buf = at & 1, kt = kt0 + (i >> 1);
          // a key tile's scales, with its values
          if ((i & 1) == 0 && !__all_sync(0xffffffffu, mbar_wait(v_full + (kt & 1), (uint32_t)(kt >> 1) & 1u))) {
            dead = true;
            break;
          }
          if (!__all_sync(0xffffffffu, mbar_wait(s_full + 2 * tile + buf, (uint32_t)(at >> 1) & 1u))) {
            dead = true;
            break;
          }
          fence_after();
          const uint32_t sb = st + (uint32_t)(buf * kStep);
          float c[kStepUnits], lc[kStepUnits], ic[kStepUnits];
          {
            const float* from = scales + 3 * kUnits * (kt & 1) + kStepUnits * (i & 1);
            const float4 x = *reinterpret_cast<const float4*>(from), y = *reinterpret_cast<const float4*>(from + kUnits), z = *reinterpret_cast<const float4*>(from + 2 * kUnits);
            c[0] = rc * x.x, c[1] = rc * x.y, c[2] = rc * x.z, c[3] = rc * x.w;
            lc[0] = y.x, lc[1] = y.y, lc[2] = y.z, lc[3] = y.w;
            ic[0] = z.x, ic[1] = z.y, ic[2] = z.z, ic[3] = z.w;
          }
          const int u0 = lo * kUnits + i * kStepUnits;  // the step's first unit
          const bool whole = u0 >= seen_from && u0 + kStepUnits <= seen_to;
          // a unit's products, masked where a row does not see all of the step
          const auto mask = [&](float* x, int u) {
            const int t0 = units.token(u0 + u);
            const int lim = u0 + u < units.total ? pos - t0 : -1;  // the row sees the unit's keys up to here
            const int from = a.window > 0 && lim >= 0 ? lim - a.window : INT_MIN, sk = a.sinks - t0;
#pragma unroll
            for (int e = 0; e < kUnit; ++e)
              if (!(e <= lim && (e > from || e < sk))) x[e] = -INFINITY;
          };
          // Probabilities relative to the maximum so far, without looking for this step's:
          // one that a score has outgrown shows in the sum, and the step is taken again from
          // its scores, which the probabilities have not replaced yet.  (Sums up to 2^15:
          // no probability then reaches fp16's largest.)  A row that has seen nothing (its
          // window begins later) has no maximum: relative to -1e30 a key that it sees now
          // has outgrown anything, and a masked one still adds 0.
          uint32_t y[kStep / 2];
          float more;
          bool look = i == 0;
#pragma unroll 1
          while (true) {
            if (look) {
              float top = -INFINITY;
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                float v[32];
                tmem_ld32(sb + 32 * h, v);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                  if (!whole) mask(v + kUnit * u, 2 * h + u);
                  float x = v[kUnit * u];
#pragma unroll
                  for (int e = 1; e < kUnit; ++e) x = fmaxf(x, v[kUnit * u + e]);
                  if (x > -INFINITY) top = fmaxf(top, fmaf(x, c[2 * h + u], lc[2 * h + u]));  // c >= 0: the largest product has the largest score
                }
              }
              const float x = fmaxf(m, top);
              const float w = x == m ? 1.f : ex2_approx(m - x);
              m = x;
              l *= w;
              if (i > 0) {  // the accumulator, once the last step's values are in it (those before are: this step's scores came after them)
                if (!__all_sync(0xffffffffu, mbar_wait(o_done + tile, (uint32_t)(at - 1) & 1u))) {
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
            }
            const float ref = m > -INFINITY ? m - 7.f : look ? 0.f : -1e30f;
            more = 0.f;
            float whole_sum = 0.f;
            const auto unit = [&](const uint32_t (&raw)[kUnit], int u) {
                float x[kUnit];
                const float lr = lc[u] - ref;
                const uint64_t c2 = pair_of(c[u], c[u]), l2 = pair_of(lr, lr);
#pragma unroll
                for (int e = 0; e < kUnit; e += 2)
                  unpair(fma2(pair_of(__uint_as_float(raw[e]), __uint_as_float(raw[e + 1])), c2, l2), x[e], x[e + 1]);
                if (!whole) mask(x, u);
                uint64_t sum = 0;
#pragma unroll
                for (int e = 0; e < kUnit; e += 2) {
                  const float p0 = ex2_approx(x[e]), p1 = ex2_approx(x[e + 1]);
                  sum = add2(sum, pair_of(p0, p1));
                  y[8 * u + e / 2] = narrow2<false>(p0, p1);
                }
                float s0, s1;
                unpair(sum, s0, s1);
                s0 += s1;
                whole_sum += s0;
                if (s0 != 0.f) more = fmaf(s0, ic[u], more);  // a unit that the row does not see may have a NaN scale
            };
            uint32_t raw[2][kUnit];  // a unit's scores are on their way while the one before is worked on
            tmem_ld16_begin(sb, raw[0]);
#pragma unroll
            for (int u = 0; u < kStepUnits; ++u) {
              tmem_ld16_wait(raw[u & 1]);
              if (u + 1 < kStepUnits) tmem_ld16_begin(sb + kUnit * (u + 1), raw[(u + 1) & 1]);
              unit(raw[u & 1], u);
            }
            if (look || !__any_sync(0xffffffffu, whole_sum > 32768.f)) break;
            look = true;
          }
          if (dead) break;
          l += more;
          tmem_st32(sb, y);
          tmem_st_wait();
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full + 2 * tile + buf);
        }
        if (steps > 0 && !dead && !mbar_wait(o_full + tile, (uint32_t)done & 1u)) dead = true;
        fence_after();
        if (__any_sync(0xffffffffu, dead)) l = nan;
        // results, through shared memory: neighbouring lanes write a row
        const int h = head * a.group + min(r, rows - 1) % a.group;
        const size_t item = ((size_t)split * a.b.rows + q.row0 + tok) * a.heads + h;
        const float inv = 1.f / l;
        if (splits == 1) {
#pragma unroll
          for (int ch = 0; ch < DIM / 32; ++ch) {
            float v[32];
            tmem_ld32(ot + 32 * ch, v);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *chunk(lane, 4 * ch + i) = make_uint4(narrow2<BF16>(v[8 * i] * inv, v[8 * i + 1] * inv), narrow2<BF16>(v[8 * i + 2] * inv, v[8 * i + 3] * inv),
                                                    narrow2<BF16>(v[8 * i + 4] * inv, v[8 * i + 5] * inv), narrow2<BF16>(v[8 * i + 6] * inv, v[8 * i + 7] * inv));
          }
          __syncwarp();
          int ct = own_tok, ch = own_h;
#pragma unroll 8
          for (int i = 0; i < kRowLanes; ++i) {
            const int rw = i * kRowsPer + lane / kRowLanes;
            if (wr + rw < rows)
              *reinterpret_cast<uint4*>(a.out + (int64_t)(q.row0 + ct) * a.out_row + (int64_t)ch * a.out_head + 8 * (lane % kRowLanes)) = *chunk(rw, lane % kRowLanes);
            next_row(ct, ch);
          }
        } else if (steps > 0) {
#pragma unroll
          for (int part = 0; part < 2; ++part) {  // half of the dimensions, fp32
#pragma unroll
            for (int ch = 0; ch < DIM / 64; ++ch) {
              float v[32];
              tmem_ld32(ot + part * (DIM / 2) + 32 * ch, v);
#pragma unroll
              for (int i = 0; i < 8; ++i)
                *chunk(lane, 8 * ch + i) = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
            }
            __syncwarp();
            int ct = own_tok, ch = own_h;
#pragma unroll 8
            for (int i = 0; i < kRowLanes; ++i) {
              const int rw = i * kRowsPer + lane / kRowLanes;
              if (wr + rw < rows)
                *reinterpret_cast<uint4*>(a.part + (((size_t)split * a.b.rows + q.row0 + ct) * a.heads + ch) * DIM + part * (DIM / 2) + 4 * (lane % kRowLanes)) =
                    *chunk(rw, lane % kRowLanes);
              next_row(ct, ch);
            }
            __syncwarp();
          }
        }
        if (splits > 1 && live) a.part_ml[item] = make_float2(m, l);
        at0 += steps;
        done += steps > 0;
      }
      kt0 += n;
      fence_before();
      fine = !__any_sync(0xffffffffu, dead);
      row_tile_end();
    }
    asm volatile("bar.arrive 2, %0;" ::"n"(32 * (kSoftWarps + 1)) : "memory");
  } else if (warp < kMmaWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kConvRegs));
    int at0 = 0;
    for (int mt = blockIdx.z; mt < mts; mt += gridDim.z) {
      const Part pt = part_of(mt);
      const int lo = pt.lo, n = pt.n;
      const KeyTiles& units = pt.units;
      bool dead = false;
      // integers to fp16: instruction i of a tile takes 16 keys, four per warp, eight (four) lanes each
      constexpr int kLanes = DIM / 16, kPer = 32 / kLanes;  // lanes per key, keys per warp and instruction
      constexpr int kInst = kKeys / (kConvWarps * kPer);
      const bool vals = warp >= kSoftWarps + kConvWarps;
      const int cw = (warp - kSoftWarps) % kConvWarps, key = cw * kPer + lane / kLanes, part = lane % kLanes;
      // lane u < 8: the block of tile j's unit u (-1: none), and its first row in the pool (kNone)
      constexpr uint32_t kNone = 0xffffffffu;
      const auto block_of = [&](int j) {
        const int u = (lo + j) * kUnits + lane;
        return lane < kUnits && u < units.total && j < n ? __ldg(table + (units.token(u) >> shift)) : -1;
      };
      const auto row_of = [&](int j, int id) {
        return id >= 0 && id < a.c.n_blocks ? ((uint32_t)id * a.c.kv_heads + head) * a.c.block + (units.token((lo + j) * kUnits + lane) & (a.c.block - 1)) : kNone;
      };
      const uint32_t in_unit = key % kUnit;
      const unsigned char* base = static_cast<const unsigned char*>(vals ? a.c.v : a.c.k) + 16 * part;  // this lane's 16 bytes of row 0
      const auto load = [&](uint32_t where, int i) {
        const uint32_t row = __shfl_sync(0xffffffffu, where, (i * kConvWarps * kPer + key) / kUnit);
        return row != kNone ? __ldg(reinterpret_cast<const uint4*>(base + (size_t)(row + in_unit) * DIM)) : make_uint4(0, 0, 0, 0);
      };
      uint64_t *full = vals ? v_full : k_full, *empty = vals ? v_empty : k_empty;
      unsigned char* stages = smem + (vals ? S::kV : S::kK) + (part >> 2) * S::kHalf;
      const int c0 = 2 * (part & 3);
      const bool swap = part >> 2;  // these lanes write their two chunks in the other order (bank conflicts)
      uint4 x[kInst];  // a tile's loads take the registers of the tile before it as they are freed
      uint32_t next = row_of(0, block_of(0));
#pragma unroll
      for (int i = 0; i < kInst; ++i) x[i] = load(next, i);
      next = row_of(1, block_of(1));
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const int at = at0 + j, id = block_of(j + 2);
        if (at >= 2 && !__all_sync(0xffffffffu, mbar_wait(empty + (at & 1), (uint32_t)((at >> 1) - 1) & 1u))) {
          dead = true;
          break;
        }
        unsigned char* dst = stages + (at & 1) * S::kTileBytes;
#pragma unroll
        for (int i = 0; i < kInst; ++i) {
          const int r = i * kConvWarps * kPer + key;
          const uint32_t w[4] = {x[i].x ^ 0x80808080u, x[i].y ^ 0x80808080u, x[i].z ^ 0x80808080u, x[i].w ^ 0x80808080u};
          x[i] = load(next, i);
          // chunks of eight: the first and the second half of the 16 bytes
          const uint32_t a0 = swap ? w[2] : w[0], a1 = swap ? w[3] : w[1], b0 = swap ? w[0] : w[2], b1 = swap ? w[1] : w[3];
          const auto lo2 = [](uint32_t v) { return int_half2(__byte_perm(v, 0x64646464u, 0x4140)); };
          const auto hi2 = [](uint32_t v) { return int_half2(__byte_perm(v, 0x64646464u, 0x4342)); };
          *reinterpret_cast<uint4*>(dst + r * 128 + (((c0 + (swap ? 1 : 0)) ^ (r & 7)) << 4)) = make_uint4(lo2(a0), hi2(a0), lo2(a1), hi2(a1));
          *reinterpret_cast<uint4*>(dst + r * 128 + (((c0 + (swap ? 0 : 1)) ^ (r & 7)) << 4)) = make_uint4(lo2(b0), hi2(b0), lo2(b1), hi2(b1));
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(full + (at & 1));
        next = row_of(j + 2, id);
      }
      at0 += n;
      if (__any_sync(0xffffffffu, dead)) break;
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kMmaRegs));  // one instruction for the whole warpgroup
    if (warp > kScaleWarp) return;
    if (warp == kScaleWarp) {
      int at0 = 0;
      for (int mt = blockIdx.z; mt < mts; mt += gridDim.z) {
        const Part pt = part_of(mt);
        const int lo = pt.lo, n = pt.n;
        bool dead = false;
        // lane u < 8: unit u of the tile: its scales, loaded a tile ahead, from the block read two ahead
        const auto block_of = [&](int j) {
          const int u = (lo + j) * kUnits + lane;
          return lane < kUnits && u < pt.units.total && j < n ? __ldg(table + (pt.units.token(u) >> shift)) : -1;
        };
        float ka, vc;
        const auto fetch = [&](int id) {
          ka = vc = __uint_as_float(0x7fc00000u);
          if (id >= 0 && id < a.c.n_blocks) {
            ka = __ldg(a.c.k_scale + (size_t)id * a.c.kv_heads + head);
            vc = __ldg(a.c.v_scale + (size_t)id * a.c.kv_heads + head);
          }
        };
        fetch(block_of(0));
        int id1 = block_of(1);
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
          const int at = at0 + j;
          if (at >= 2 && !__all_sync(0xffffffffu, mbar_wait(v_empty + (at & 1), (uint32_t)((at >> 1) - 1) & 1u))) {
            dead = true;
            break;
          }
          const float y = vc == 0.f ? 0x1p-80f : vc;
          float* to = scales + 3 * kUnits * (at & 1) + lane;
          if (lane < kUnits) {
            to[0] = ka;
            to[kUnits] = lg2_approx(y);  // 2^-22 of the value: 2^-17 at a scale of 2^-32, an fp16 weight rounds by 2^-11
            to[2 * kUnits] = rcp_approx(y);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(v_full + (at & 1));
          fetch(id1);
          id1 = block_of(j + 2);
        }
        at0 += n;
        if (__any_sync(0xffffffffu, dead)) break;
      }
    } else {
      int at0 = 0, tile_at[2] = {0, 0}, mi = 0;  // key tiles, steps of the row tiles, row tiles with steps
      for (int mt = blockIdx.z; mt < mts; mt += gridDim.z) {
        const Part pt = part_of(mt);
        const int steps = pt.steps, tiles = pt.two ? 2 : 1;
        if (steps == 0) continue;
        bool dead = false;
        if (elect()) {
          bool ok = mbar_wait(q_full, (uint32_t)mi & 1u);
          const uint32_t sq = smem_u32(smem + S::kQ), sk = smem_u32(smem + S::kK), sv = smem_u32(smem + S::kV);
          // step i's products; a key tile's stage is free once its last step's of all row tiles are done
          const auto scores = [&](int t, int i) {
            const int stage = (at0 + (i >> 1)) & 1, buf = (tile_at[t] + i) & 1;
            const uint32_t qa = sq + t * S::kTileBytes, kb = sk + stage * S::kTileBytes + (i & 1) * (kStep * 128);
#pragma unroll
            for (int kk = 0; kk < DIM / 16; ++kk)
              mma_f16_ss(tmem + t * 128 + buf * kStep, sw128_desc(qa + (kk >> 2) * S::kHalf) + 2 * (kk & 3), sw128_desc(kb + (kk >> 2) * S::kHalf) + 2 * (kk & 3),
                         idesc_f16(128, kStep, false), kk > 0);
            mma_commit(s_full + 2 * t + buf);
            if (t == tiles - 1 && ((i & 1) || i == steps - 1)) mma_commit(k_empty + stage);
          };
          const auto values = [&](int t, int i) {
            const int stage = (at0 + (i >> 1)) & 1, buf = (tile_at[t] + i) & 1;
            const uint32_t vb = sv + stage * S::kTileBytes + (i & 1) * (kStep * 128);
#pragma unroll
            for (int kk = 0; kk < kStep / 16; ++kk)
              mma_f16_ts(tmem + S::kO + t * DIM, tmem + t * 128 + buf * kStep + 8 * kk, sw128_mn_desc(vb + kk * 2048, S::kHalf), idesc_f16(128, DIM, true),
                         i > 0 || kk > 0);
            mma_commit(o_done + t);
            if (i == steps - 1) mma_commit(o_full + t);
            if (t == tiles - 1 && ((i & 1) || i == steps - 1)) mma_commit(v_empty + stage);
          };
          const auto have = [&](uint64_t* full, int i) {
            const int at = at0 + (i >> 1);
            const bool there = mbar_wait(full + (at & 1), (uint32_t)(at >> 1) & 1u);
            fence_after();
            return there;
          };
          if (ok) ok = have(k_full, 0);
          for (int i = 0; i < min(2, steps) && ok; ++i)
            for (int t = 0; t < tiles; ++t) scores(t, i);
          for (int i = 0; i < steps && ok; ++i) {
            if ((i & 1) == 0) ok = have(v_full, i);
            for (int t = 0; t < tiles && ok; ++t) {
              const int at = tile_at[t] + i;
              ok = mbar_wait(p_full + 2 * t + (at & 1), (uint32_t)(at >> 1) & 1u);
              if (!ok) break;
              fence_after();
              values(t, i);
              if (i + 2 < steps) {
                if (t == 0 && (i & 1) == 0) ok = have(k_full, i + 2);
                if (ok) scores(t, i + 2);
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
        ++mi;
        at0 += pt.n;
        tile_at[0] += steps;
        if (pt.two) tile_at[1] += steps;
        if (__any_sync(0xffffffffu, dead)) break;
      }
      asm volatile("bar.sync 2, %0;" ::"n"(32 * (kSoftWarps + 1)) : "memory");  // the accumulators have been read
      fence_after();
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
  }
}

template <bool BF16, int DIM>
cudaError_t launch(const Kv8Attend& a, const Kv8TilesPlan& p, cudaStream_t s) {
  using S = TilesShape<DIM>;
  static const bool enough = [] {  // setmaxnreg waits for registers that the launch did not bring
    cudaFuncAttributes at{};
    return cudaFuncGetAttributes(&at, k_kv8_tiles<BF16, DIM>) == cudaSuccess && at.numRegs >= kLaunchRegs;
  }();
  if (!enough) return cudaErrorLaunchOutOfResources;
  const cudaError_t e = smem_opt_in<k_kv8_tiles<BF16, DIM>>(S::kSmem);
  if (e != cudaSuccess) return e;
  k_kv8_tiles<BF16, DIM><<<dim3(a.c.kv_heads * p.splits, a.b.n, p.mtiles), kThreads, S::kSmem, s>>>(a);
  return cudaGetLastError();
}

}  // namespace

bool kv8_tiles_plan(const tsd_kv8& c, const tsd_kv8_batch& b, int heads, int window, int sinks, int sms, Kv8TilesPlan* p) {
  const int group = heads / c.kv_heads;
  const int most = std::max(1, b.max_new ? std::min(b.max_new, b.rows) : (b.rows + b.n - 1) / b.n);
  // Rows from which a tile of 256 pays although most of it is empty; here and with kv8_rows.cu, dim 128, us: 4 sequences of 4
  // key heads past 2000 tokens 21 and 20 at 48 rows, 23 and 23 at 64, 21 and 29 at 96; 60 past 300 27 and 22, 27 and 26, 29 and
  // 37; 64 past 2000 64 and 82, 65 and 105, 64 and 140.  (Dim 64: 60 past 300 22 and 16, 23 and 17, 25 and 24.)
  if ((int64_t)most * group <= 48) return false;
  p->mtiles = (int)std::min<int64_t>(((int64_t)most * group + 255) / 256, 65535);
  const int64_t cap = std::min<int64_t>(b.max_len ? b.max_len : INT64_MAX, (int64_t)b.table_width * c.block);
  const int64_t keys = window > 0 ? std::min<int64_t>(cap, (int64_t)window + sinks + most) : cap;
  // few row tiles: the keys over several CTAs too, four key tiles each at least
  const int64_t units = (int64_t)b.n * c.kv_heads * p->mtiles;
  p->splits = (int)std::max<int64_t>(1, std::min<int64_t>({sms / units, keys / kKeys / 4, 64, 65535 / c.kv_heads}));
  p->bytes = p->splits > 1 ? (int64_t)p->splits * b.rows * heads * (c.dim + 2) * 4 : 0;
  return true;
}

cudaError_t kv8_tiles_launch(const Kv8Attend& a, const Kv8TilesPlan& p, cudaStream_t s) {
  const bool bf = a.c.dtype == TSD_BF16;
  const cudaError_t e = a.c.dim == 64 ? (bf ? launch<true, 64>(a, p, s) : launch<false, 64>(a, p, s))
                                      : (bf ? launch<true, 128>(a, p, s) : launch<false, 128>(a, p, s));
  return e == cudaSuccess && p.splits > 1 ? kv8_join_launch(a, p.splits, s) : e;
}

}  // namespace tsd
