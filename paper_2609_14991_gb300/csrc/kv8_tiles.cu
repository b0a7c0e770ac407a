// Attention over the 8-bit paged cache with many query rows per key head:
// prompts (tsd.h: tsd_kv8_attend).
//
// The mathematics is kv8_rows.cu's; the products run on tcgen05 (fp16 in, fp32
// accumulate in TMEM).  A CTA takes 256 rows of a sequence and key head (row =
// token * group + head of the group) as two tiles of 128, and the keys they see in
// tiles of 128:
//   warps 0-7   softmax: a thread is a row (warps 0-3 tile 0, 4-7 tile 1), so its
//               maximum, sum and masks need no exchange.  Reads its scores from TMEM,
//               leaves probabilities (fp16) in their place as the values'
//               product's A operand;
//   warps 8-11  turn the integers of the next key tile into fp16 in shared memory
//               (128-byte swizzle), once for both row tiles and all heads of a group;
//   warp 12     issues the MMAs: while one tile's softmax runs, the other tile's
//               products do.
// Keys are the K-major B operand of the scores; the same layout of the values is read as
// an MN-major B operand, so neither is transposed.  A tile's accumulator is rescaled in
// TMEM only when a row's maximum grows by more than 2^8.
//
// What bounds it at dim 128: per key tile and CTA the MMAs take 2080 clocks, the
// hardware's 2^x 2048 (256 x 128 of them at 16 per clock), beside 1400 issue slots per
// scheduler for scores, probabilities and conversions.
#include <algorithm>
#include <climits>

#include "kv8_attend.h"
#include "tc_common.cuh"

namespace tsd {

namespace {

using namespace tc;

constexpr int kUnit = kKv8Unit;
constexpr int kKeys = 128;            // keys per tile
constexpr int kUnits = kKeys / kUnit;
constexpr int kSoftWarps = 8, kConvWarps = 4;
constexpr int kThreads = 32 * (kSoftWarps + kConvWarps + 1);

template <int DIM>
struct TilesShape {
  static constexpr int kHalf = 128 * 128;              // 128 rows of 64 fp16
  static constexpr int kTileBytes = kHalf * (DIM / 64);  // a row tile's queries, or a key tile's keys or values
  static constexpr int kQ = 0;
  static constexpr int kK = 2 * kTileBytes;             // two stages
  static constexpr int kV = 4 * kTileBytes;             // two stages
  static constexpr int kBar = 6 * kTileBytes;
  static constexpr int kSmem = kBar + 256 + 1024;
  static constexpr int kO = 256;  // TMEM: scores of the tiles at 0 and 128, accumulators from here
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
  uint64_t *s_full = bars + 8, *p_full = bars + 10, *o_full = bars + 12;                    // [2] row tiles
  uint64_t *q_full = bars + 14, *drain = bars + 15;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 16);

  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const Kv8Seq q = kv8_seq(a.c, a.b, blockIdx.z);
  const int head = blockIdx.y % a.c.kv_heads, split = blockIdx.y / a.c.kv_heads, splits = gridDim.y / a.c.kv_heads;
  const int rows = q.count * a.group;
  const int mts = (rows + 255) / 256;
  if ((int)blockIdx.x >= mts) return;

  const auto say_nan = [&](int row0) {
    for (int e = threadIdx.x; e < 256 * (DIM / 8); e += kThreads) {
      const int r = row0 + e / (DIM / 8), col = 8 * (e % (DIM / 8));
      if (r >= rows) break;
      const int tok = q.row0 + r / a.group, h = head * a.group + r % a.group;
      const uint32_t nan2 = BF16 ? 0x7fc07fc0u : 0x7e007e00u;
      if (splits == 1)
        *reinterpret_cast<uint4*>(a.out + (int64_t)tok * a.out_row + (int64_t)h * a.out_head + col) = make_uint4(nan2, nan2, nan2, nan2);
      else if (col == 0)
        a.part_ml[((size_t)split * a.b.rows + tok) * a.heads + h] = make_float2(0.f, __uint_as_float(0x7fc00000u));
    }
  };
  if (!q.ok) {
    for (int mt = blockIdx.x; mt < mts; mt += gridDim.x) say_nan(mt * 256);
    return;
  }

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(k_full + i, kConvWarps);
      mbar_init(v_full + i, kConvWarps);
      mbar_init(k_empty + i, 1);
      mbar_init(v_empty + i, 1);
      mbar_init(s_full + i, 1);
      mbar_init(p_full + i, 4);
      mbar_init(o_full + i, 1);
    }
    mbar_init(q_full, kSoftWarps);
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kSoftWarps + kConvWarps) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *tmem_slot;

  const int32_t* table = a.b.table + (size_t)q.slot * a.b.table_width;
  const int before = q.len - q.count;
  // the barriers' positions: key tiles so far (of row tile 0, of row tile 1), row tiles, and those with keys
  int at0 = 0, at1 = 0, mi = 0, done0 = 0, done1 = 0;
  bool dead = false;  // a wait ran out: NaN from there on
  for (int mt = blockIdx.x; mt < mts; mt += gridDim.x, ++mi) {
    // the later rows see the most keys: they go first
    const int row0 = (mts - 1 - mt) * 256;
    const bool two = rows - row0 > 128;
    const KeyTiles units = key_tiles(before + row0 / a.group, before + (min(rows, row0 + 256) - 1) / a.group, a.window, a.sinks);
    const int all = (units.total + kUnits - 1) / kUnits;
    const int lo = (int)((int64_t)all * split / splits), n = (int)((int64_t)all * (split + 1) / splits) - lo;

    if (dead) {
      say_nan(row0);
    } else if (warp < kSoftWarps) {
      const int tile = warp >> 2, r = row0 + threadIdx.x;
      const bool live = r < rows;
      const int tok = min(r, rows - 1) / a.group, pos = before + tok;
      // the row's queries as fp16, scaled by f into [2^14, 2^15)
      float rc;
      {
        float top = 0.f;
        bool odd = false;
        const uint16_t* src = a.q + (int64_t)(q.row0 + tok) * a.q_row + (int64_t)(head * a.group + min(r, rows - 1) % a.group) * a.q_head;
#pragma unroll 8
        for (int i = 0; i < DIM / 8; ++i) {
          const uint4 w = live ? __ldg(reinterpret_cast<const uint4*>(src) + i) : make_uint4(0, 0, 0, 0);
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float x = fabsf(wide16<BF16>(u[j] & 0xffffu)), y = fabsf(wide16<BF16>(u[j] >> 16));
            top = fmaxf(top, fmaxf(x, y));
            odd = odd || !(x + y <= INFINITY);
          }
        }
        const QueryScale qs = query_scale(odd ? INFINITY : top);
        rc = qs.fine ? a.scale * kLog2e / qs.f : __uint_as_float(0x7fc00000u);
        // the last row tile's products have read the rows before these: its accumulators were waited for
        const int rr = threadIdx.x & 127;
        unsigned char* dst = smem + S::kQ + tile * S::kTileBytes + rr * 128;
#pragma unroll 4
        for (int i = 0; i < DIM / 8; ++i) {
          const uint4 w = live ? __ldg(reinterpret_cast<const uint4*>(src) + i) : make_uint4(0, 0, 0, 0);
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
          uint32_t y[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] = narrow2<false>(wide16<BF16>(u[j] & 0xffffu) * qs.f, wide16<BF16>(u[j] >> 16) * qs.f);
          *reinterpret_cast<uint4*>(dst + (i >> 3) * S::kHalf + (((i & 7) ^ (rr & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full);
      }
      if (tile == 0 || two) {
        const uint32_t st = tmem + (uint32_t)(tile * 128) + ((uint32_t)((warp & 3) * 32) << 16);  // scores, then probabilities
        const uint32_t ot = tmem + (uint32_t)(S::kO + tile * DIM) + ((uint32_t)((warp & 3) * 32) << 16);
        // positions that every row of the warp sees
        const int wr = row0 + (threadIdx.x & ~31);
        const int all_to = before + min(wr, rows - 1) / a.group;
        const int all_from = a.window > 0 ? before + min(wr + 31, rows - 1) / a.group - a.window + 1 : 0;
        float m = -INFINITY, l = 0.f;
        // lane u < 8: scales of the next key tile's unit u
        const float nan = __uint_as_float(0x7fc00000u);
        float na = nan, nc = nan;
        const auto fetch = [&](int j) {
          const int u = (lo + j) * kUnits + lane;
          na = nc = nan;
          if (lane < kUnits && u < units.total) {
            const int id = __ldg(table + units.token(u) / a.c.block);
            if (id >= 0 && id < a.c.n_blocks) {
              na = __ldg(a.c.k_scale + (size_t)id * a.c.kv_heads + head);
              nc = __ldg(a.c.v_scale + (size_t)id * a.c.kv_heads + head);
            }
          }
        };
        if (n > 0) fetch(0);
        for (int j = 0; j < n; ++j) {
          const float ua = na, uc = nc == 0.f ? 0x1p-80f : nc;
          const float ul = log2f(uc), ui = 1.f / uc;
          if (j + 1 < n) fetch(j + 1);
          if (!mbar_wait(s_full + tile, (uint32_t)((tile ? at1 : at0) + j) & 1u)) {
            dead = true;
            break;
          }
          fence_after();
          const int u0 = (lo + j) * kUnits;
          const int t_lo = units.token(u0), t_hi = units.token(min(u0 + kUnits, units.total) - 1) + kUnit - 1;
          const bool whole = u0 + kUnits <= units.total && t_hi <= all_to && (t_lo >= all_from || t_hi < a.sinks);
          // s' of a unit's 16 scores, masked
          const auto scores = [&](const float* v, int u, float* s) {
            const float c = rc * __shfl_sync(0xffffffffu, ua, u), lc = __shfl_sync(0xffffffffu, ul, u);
#pragma unroll
            for (int i = 0; i < kUnit; ++i) s[i] = fmaf(v[i], c, lc);
            if (!whole) {
              const int t0 = units.token(u0 + u);
              const int lim = u0 + u < units.total ? pos - t0 : -1;  // the row sees the unit's keys up to here
              const int from = a.window > 0 && lim >= 0 ? lim - a.window : INT_MIN, sk = a.sinks - t0;
#pragma unroll
              for (int i = 0; i < kUnit; ++i)
                if (!(i <= lim && (i > from || i < sk))) s[i] = -INFINITY;
            }
          };
          float top = -INFINITY;
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) {
            float v[32], s[16];
            tmem_ld32(st + 32 * ch, v);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              scores(v + 16 * h, 2 * ch + h, s);
#pragma unroll
              for (int i = 0; i < kUnit; ++i) top = fmaxf(top, s[i]);
            }
          }
          if (__any_sync(0xffffffffu, top > m + 8.f)) {
            const float x = fmaxf(m, top);
            const float w = x == m ? 1.f : ex2_approx(m - x);
            m = x;
            l *= w;
            if (j > 0) {  // the values' products so far are done: the scores came after them
#pragma unroll
              for (int ch = 0; ch < DIM / 32; ++ch) {
                float v[32];
                tmem_ld32(ot + 32 * ch, v);
                uint32_t y[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) y[i] = __float_as_uint(v[i] * w);
                tmem_st16(ot + 32 * ch, y);
                tmem_st16(ot + 32 * ch + 16, y + 16);
              }
            }
          }
          const float ref = m == -INFINITY ? 0.f : m - 7.f;
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) {
            float v[32];
            tmem_ld32(st + 32 * ch, v);
            uint32_t y[16];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float s[16];
              scores(v + 16 * h, 2 * ch + h, s);
              const float ic = __shfl_sync(0xffffffffu, ui, 2 * ch + h);
              float sum = 0.f;
#pragma unroll
              for (int i = 0; i < kUnit; i += 2) {
                const float p0 = ex2_approx(s[i] - ref), p1 = ex2_approx(s[i + 1] - ref);
                sum += p0 + p1;
                y[8 * h + i / 2] = narrow2<false>(p0, p1);
              }
              if (sum != 0.f) l = fmaf(sum, ic, l);  // a unit that the row does not see may have a NaN scale
            }
            tmem_st16(st + 16 * ch, y);
          }
          tmem_st_wait();
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full + tile);
        }
        if (n > 0 && !dead && !mbar_wait(o_full + tile, (uint32_t)(tile ? done1 : done0) & 1u)) dead = true;
        fence_after();
        if (__any_sync(0xffffffffu, dead)) l = nan;
        // a row's results: its own contiguous DIM values
        const int h = head * a.group + min(r, rows - 1) % a.group;
        const size_t at = ((size_t)split * a.b.rows + q.row0 + tok) * a.heads + h;
        const float inv = 1.f / l;
#pragma unroll
        for (int ch = 0; ch < DIM / 32; ++ch) {
          float v[32];
          __syncwarp();
          if (n > 0) tmem_ld32(ot + 32 * ch, v);
          if (!live) continue;
          if (splits == 1) {
            uint4* dst = reinterpret_cast<uint4*>(a.out + (int64_t)(q.row0 + tok) * a.out_row + (int64_t)h * a.out_head + 32 * ch);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              dst[i] = make_uint4(narrow2<BF16>(v[8 * i] * inv, v[8 * i + 1] * inv), narrow2<BF16>(v[8 * i + 2] * inv, v[8 * i + 3] * inv),
                                  narrow2<BF16>(v[8 * i + 4] * inv, v[8 * i + 5] * inv), narrow2<BF16>(v[8 * i + 6] * inv, v[8 * i + 7] * inv));
          } else if (n > 0) {
            float4* dst = reinterpret_cast<float4*>(a.part + at * DIM + 32 * ch);
#pragma unroll
            for (int i = 0; i < 8; ++i) dst[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
          }
        }
        if (splits > 1 && live) a.part_ml[at] = make_float2(m, l);
        fence_before();
      }
    } else if (warp < kSoftWarps + kConvWarps) {
      // integers to fp16: instruction i of a tile takes 16 keys, four per warp, eight (four) lanes each
      constexpr int kLanes = DIM / 16, kPer = 32 / kLanes;  // lanes per key, keys per warp and instruction
      constexpr int kInst = kKeys / (kConvWarps * kPer);
      const int cw = warp - kSoftWarps, key = cw * kPer + lane / kLanes, part = lane % kLanes;
      for (int j = 0; j < n && !dead; ++j) {
        const int at = at0 + j, s = at & 1;
        // lane u < 8: unit u's block and first row in it
        int id = -1, row = 0;
        const int u = (lo + j) * kUnits + lane;
        if (lane < kUnits && u < units.total) {
          const int t0 = units.token(u);
          id = __ldg(table + t0 / a.c.block);
          if (id >= a.c.n_blocks) id = -1;
          row = t0 % a.c.block;
        }
#pragma unroll
        for (int which = 0; which < 2; ++which) {
          const int8_t* base = static_cast<const int8_t*>(which ? a.c.v : a.c.k);
          uint4 x[kInst];
#pragma unroll
          for (int i = 0; i < kInst; ++i) {
            const int r = i * kConvWarps * kPer + key;
            const int rid = __shfl_sync(0xffffffffu, id, r / kUnit), rrow = __shfl_sync(0xffffffffu, row, r / kUnit);
            x[i] = make_uint4(0, 0, 0, 0);
            if (rid >= 0)
              x[i] = __ldg(reinterpret_cast<const uint4*>(base + (((size_t)rid * a.c.kv_heads + head) * a.c.block + rrow + r % kUnit) * DIM) + part);
          }
          uint64_t* empty = (which ? v_empty : k_empty) + s;
          if (at >= 2 && !mbar_wait(empty, (uint32_t)((at >> 1) - 1) & 1u)) {
            dead = true;
            break;
          }
          unsigned char* dst = smem + (which ? S::kV : S::kK) + s * S::kTileBytes + (part >> 2) * S::kHalf;
#pragma unroll
          for (int i = 0; i < kInst; ++i) {
            const int r = i * kConvWarps * kPer + key;
            const uint32_t w[4] = {x[i].x ^ 0x80808080u, x[i].y ^ 0x80808080u, x[i].z ^ 0x80808080u, x[i].w ^ 0x80808080u};
            uint32_t y[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              y[2 * e] = int_half2(__byte_perm(w[e], 0x64646464u, 0x4140));
              y[2 * e + 1] = int_half2(__byte_perm(w[e], 0x64646464u, 0x4342));
            }
            // two 16-byte chunks; the lanes of the second half of a key write theirs in the other order (bank conflicts)
            const int c0 = 2 * (part & 3);
            const uint4 y0 = make_uint4(y[0], y[1], y[2], y[3]), y1 = make_uint4(y[4], y[5], y[6], y[7]);
            const bool swap = part >> 2;
            *reinterpret_cast<uint4*>(dst + r * 128 + (((c0 + (swap ? 1 : 0)) ^ (r & 7)) << 4)) = swap ? y1 : y0;
            *reinterpret_cast<uint4*>(dst + r * 128 + (((c0 + (swap ? 0 : 1)) ^ (r & 7)) << 4)) = swap ? y0 : y1;
          }
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive((which ? v_full : k_full) + s);
        }
      }
    } else {
     if (elect()) {
      bool ok = mbar_wait(q_full, (uint32_t)mi & 1u);
      const uint32_t sq = smem_u32(smem + S::kQ), sk = smem_u32(smem + S::kK), sv = smem_u32(smem + S::kV);
      const auto scores = [&](int tile, int at) {
        const uint32_t qa = sq + tile * S::kTileBytes, kb = sk + (at & 1) * S::kTileBytes;
#pragma unroll
        for (int kk = 0; kk < DIM / 16; ++kk)
          mma_f16_ss(tmem + tile * 128, sw128_desc(qa + (kk >> 2) * S::kHalf) + 2 * (kk & 3), sw128_desc(kb + (kk >> 2) * S::kHalf) + 2 * (kk & 3),
                     idesc_f16(128, kKeys, false), kk > 0);
        mma_commit(s_full + tile);
      };
      const auto values = [&](int tile, int at, bool acc) {
        const uint32_t vb = sv + (at & 1) * S::kTileBytes;
#pragma unroll
        for (int kk = 0; kk < kKeys / 16; ++kk)
          mma_f16_ts(tmem + S::kO + tile * DIM, tmem + tile * 128 + 8 * kk, sw128_mn_desc(vb + kk * 2048, S::kHalf), idesc_f16(128, DIM, true),
                     acc || kk > 0);
      };
      const int tiles = two ? 2 : 1;
      if (ok && n > 0) {
        ok = mbar_wait(k_full + (at0 & 1), (uint32_t)(at0 >> 1) & 1u);
        if (ok) {
          fence_after();
          for (int t = 0; t < tiles; ++t) scores(t, at0);
          mma_commit(k_empty + (at0 & 1));
        }
      }
      for (int j = 0; j < n && ok; ++j) {
        const int at = at0 + j;
        ok = mbar_wait(v_full + (at & 1), (uint32_t)(at >> 1) & 1u);
        for (int t = 0; t < tiles && ok; ++t) {
          ok = mbar_wait(p_full + t, (uint32_t)((t ? at1 : at0) + j) & 1u);
          if (!ok) break;
          fence_after();
          values(t, at, j > 0);
          if (t == tiles - 1) mma_commit(v_empty + (at & 1));
          if (j + 1 < n) {
            ok = t > 0 || mbar_wait(k_full + ((at + 1) & 1), (uint32_t)((at + 1) >> 1) & 1u);
            if (!ok) break;
            fence_after();
            scores(t, at + 1);
            if (t == tiles - 1) mma_commit(k_empty + ((at + 1) & 1));
          } else {
            mma_commit(o_full + t);
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
    }
    at0 += n;
    done0 += n > 0;
    if (two) at1 += n, done1 += n > 0;
    // every role is done with this row tile before the next one's queries
    fence_before();
    dead = __syncthreads_or(dead);
    fence_after();
  }
  if (warp == kSoftWarps + kConvWarps)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

template <bool BF16, int DIM>
cudaError_t launch(const Kv8Attend& a, const Kv8TilesPlan& p, cudaStream_t s) {
  using S = TilesShape<DIM>;
  const cudaError_t e = smem_opt_in<k_kv8_tiles<BF16, DIM>>(S::kSmem);
  if (e != cudaSuccess) return e;
  k_kv8_tiles<BF16, DIM><<<dim3(p.mtiles, a.c.kv_heads * p.splits, a.b.n), kThreads, S::kSmem, s>>>(a);
  return cudaGetLastError();
}

}  // namespace

bool kv8_tiles_plan(const tsd_kv8& c, const tsd_kv8_batch& b, int heads, int window, int sinks, int sms, Kv8TilesPlan* p) {
  const int group = heads / c.kv_heads;
  const int most = std::max(1, b.max_new ? std::min(b.max_new, b.rows) : (b.rows + b.n - 1) / b.n);
  if ((int64_t)most * group < 96) return false;
  p->mtiles = (int)(((int64_t)most * group + 255) / 256);
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
