// Attention over the 8-bit paged cache with few query rows per key head: single
// tokens and short chunks (tsd.h: tsd_kv8_attend).
//
// The rows of a sequence and key head are its new tokens times the query heads
// that share the head (row = token * group + head of the group).  The products are
// mma.sync.m16n8k16 (fp16 in, fp32 out): tcgen05 takes 64 or 128 rows, and these are
// few.  Up to 16 rows (k_kv8_eight) are one or two column tiles of eight: scores are
// keys x rows, results dimensions x rows, so few products are spent on rows that are
// not there.  More (k_kv8_rows) are two row tiles of 16 per CTA (four, with one key group, took 133
// us where two take 82: 48 rows, 64 sequences past 2000 tokens).  The keys and values are read once
// for all rows of a CTA, whose four warps share the work as two row tiles x two key groups; a
// long context is split over CTAs too (partial results in the workspace, joined by
// k_kv8_join).
//
// Mathematics, per row: with integers k_j, v_j, scales a_b, c_b of key j's block b and
// the row's factor f (queries are scaled by f, a power of two, into fp16),
//   s_j = (q f . k_j) (scale log2(e) a_b / f) + log2(c_b),   m = max_j s_j,
//   out = sum_j 2^(s_j - m) v_j  /  sum_j 2^(s_j - m) / c_b,
// so a value's scale is an addend of the exponent and the integers go into the
// products as they are (exact in fp16, as is every query within 2^28 of its
// row's largest).  The weights 2^(s_j - m), with their value's scale in them, are rounded to fp16
// (half a step 2^-11) as multiples of 2^(m - 7): below 2^-21 of the largest to multiples of 2^-31
// of it, so a block whose values are 2^21 times smaller than another's counts more coarsely.  The maximum
// follows only when a score passes it by more than 2^8, which fp16 still holds:
// most tiles need no exchange between lanes.
//
// Layout: a tile is 16 tokens of one block and head, 16 x dim contiguous
// bytes: one untiled bulk copy for its keys and one for its values into a ring of
// stages per key group.  A product over the head dimension may take the
// dimensions in any order, and so may one over keys: lane (g, t) of a warp takes 16
// consecutive bytes of key g as its part of four k-steps, and 16 consecutive
// dimensions of keys 2t, 2t+1, 2t+8, 2t+9 as its part of 16 column tiles, so
// nothing is transposed.  Integers become fp16 by placing the byte (offset by 128)
// in the mantissa of 1024 and subtracting 1152: both exact.
#include <algorithm>

#include "kv8_attend.h"
#include "launch.h"
#include "tc_common.cuh"

namespace tsd {

namespace {

using namespace tc;

constexpr int kTile = kKv8Unit;  // keys per tile
constexpr int kRowTiles = 2;     // row tiles of 16 in a CTA of k_kv8_rows

template <int DIM>
struct RowsShape {
  static constexpr int kKeyGroups = 4 / kRowTiles;
  static constexpr int kStages = 8;
  static constexpr int kStageBytes = 2 * kTile * DIM;
  static constexpr int kRing = kKeyGroups * kStages * kStageBytes;
  static constexpr int kOutStride = DIM + 4;
  static constexpr int kOut = 64 * kOutStride * 4;  // four warps' 16 rows
  static constexpr int kBarOff = kRing > kOut ? kRing : kOut;
  static constexpr int kSmem = kBarOff + kKeyGroups * kStages * 16 + 64 * 8;
};

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Joins a row's results of the CTA's `parts` key groups (maximum and sum ml_step apart,
// eight of its dimensions from col on acc_step apart) and writes them, or this
// split's share.
template <bool BF16, int DIM>
__device__ __forceinline__ void emit_row(const Kv8Attend& a, const Kv8Seq& q, int r, int head, int col, const float2* ml, int ml_step, const float* src,
                                         int acc_step, int parts) {
  float top = -INFINITY;
  for (int k = 0; k < parts; ++k) top = fmaxf(top, ml[k * ml_step].x);
  float acc[8] = {}, sum = 0.f;
  for (int k = 0; k < parts; ++k) {
    const float2 x = ml[k * ml_step];
    if (x.x == -INFINITY && x.y == 0.f) continue;
    const float w = x.x == -INFINITY ? 1.f : ex2_approx(x.x - top);
    sum = fmaf(w, x.y, sum);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = fmaf(w, src[k * acc_step + j], acc[j]);
  }
  const int tok = q.row0 + r / a.group, h = head * a.group + r % a.group;
  if (gridDim.x == 1) {
    const float inv = 1.f / sum;
    uint4 y;
    y.x = narrow2<BF16>(acc[0] * inv, acc[1] * inv);
    y.y = narrow2<BF16>(acc[2] * inv, acc[3] * inv);
    y.z = narrow2<BF16>(acc[4] * inv, acc[5] * inv);
    y.w = narrow2<BF16>(acc[6] * inv, acc[7] * inv);
    *reinterpret_cast<uint4*>(a.out + (int64_t)tok * a.out_row + (int64_t)h * a.out_head + col) = y;
  } else {
    const size_t at = ((size_t)blockIdx.x * a.b.rows + tok) * a.heads + h;
    float4* dst = reinterpret_cast<float4*>(a.part + at * DIM + col);
    dst[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    dst[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
    if (col == 0) a.part_ml[at] = make_float2(top, sum);
  }
}

template <bool BF16, int DIM>
__global__ void __launch_bounds__(128) k_kv8_rows(const __grid_constant__ Kv8Attend a) {
  using S = RowsShape<DIM>;
  constexpr int KW = S::kKeyGroups, ST = S::kStages;
  constexpr int kSteps = DIM / 16;  // k-steps of the scores' product
  constexpr int kCols = DIM / 8;    // column tiles of the values' product
  extern __shared__ __align__(128) unsigned char smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::kBarOff);
  float2* s_ml = reinterpret_cast<float2*>(bars + 2 * KW * ST);  // [64] (max, sum) of the warps' rows
  float* s_out = reinterpret_cast<float*>(smem);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int mw = warp % kRowTiles, kg = warp / kRowTiles;
  const int head = blockIdx.y % a.c.kv_heads, mt0 = blockIdx.y / a.c.kv_heads, mts = gridDim.y / a.c.kv_heads;
  const Kv8Seq q = kv8_seq(a.c, a.b, blockIdx.z);
  const int rows = q.count * a.group;
  if (mt0 * 16 * kRowTiles >= rows) return;
  uint64_t* full = bars + kg * ST;
  uint64_t* empty = bars + KW * ST + kg * ST;
  unsigned char* ring = smem + kg * ST * S::kStageBytes;

  if (threadIdx.x == 0) {
    for (int i = 0; i < KW * ST; ++i) {
      mbar_init(bars + i, 1);
      mbar_init(bars + KW * ST + i, kRowTiles);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  int it0 = 0;  // tiles that this key group has taken so far (the ring's position)
  bool dead = false;  // a wait of this CTA ran out: NaN for its rows from there on

  for (int mt = mt0; mt * 16 * kRowTiles < rows; mt += mts) {
    const int r0 = mt * 16 * kRowTiles + mw * 16;  // this warp's first row
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    float o[kCols][4];
#pragma unroll
    for (int j = 0; j < kCols; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;

    if (q.ok && !dead) {
      const int before = q.len - q.count;
      const int last_row = min(rows, (mt + 1) * 16 * kRowTiles) - 1;
      const KeyTiles tiles = key_tiles(before + mt * 16 * kRowTiles / a.group, before + last_row / a.group, a.window, a.sinks);
      const int lo = share_from(tiles.total, blockIdx.x, gridDim.x), hi = share_from(tiles.total, blockIdx.x + 1, gridDim.x);
      const int n = hi - lo > kg ? (hi - lo - kg + KW - 1) / KW : 0;  // this key group's tiles lo + kg + i KW
      // the queries' fragments
      uint32_t qf[kSteps][4];
      float rc[2];
      int pos[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = r0 + g + 8 * h, tok = r / a.group;
        pos[h] = before + min(tok, q.count - 1);
        uint2 w[kSteps];
        float top = 0.f;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
          w[kk] = make_uint2(0, 0);
          if (r < rows)
            w[kk] = __ldg(reinterpret_cast<const uint2*>(a.q + (int64_t)(q.row0 + tok) * a.q_row + (int64_t)(head * a.group + r % a.group) * a.q_head +
                                                         64 * (kk >> 2) + 16 * t + 4 * (kk & 3)));
        }
        bool odd = false;  // a NaN, which the maximum would pass over
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
          const float x0 = fabsf(wide16<BF16>(w[kk].x & 0xffffu)), x1 = fabsf(wide16<BF16>(w[kk].x >> 16));
          const float x2 = fabsf(wide16<BF16>(w[kk].y & 0xffffu)), x3 = fabsf(wide16<BF16>(w[kk].y >> 16));
          top = fmaxf(fmaxf(top, fmaxf(x0, x1)), fmaxf(x2, x3));
          odd = odd || !(x0 + x1 + x2 + x3 <= INFINITY);
        }
        top = odd ? INFINITY : top;
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const QueryScale qs = query_scale(top);
        const float f = qs.f;
        rc[h] = qs.fine ? a.scale * kLog2e / f : __uint_as_float(0x7fc00000u);
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
          qf[kk][h] = narrow2<false>(wide16<BF16>(w[kk].x & 0xffffu) * f, wide16<BF16>(w[kk].x >> 16) * f);
          qf[kk][2 + h] = narrow2<false>(wide16<BF16>(w[kk].y & 0xffffu) * f, wide16<BF16>(w[kk].y >> 16) * f);
        }
      }
      // positions that every row of this warp sees
      const int all_to = before + min(r0, rows - 1) / a.group;                                             // the first row's
      const int all_from = a.window > 0 ? before + min(r0 + 15, rows - 1) / a.group - a.window + 1 : 0;  // the last row's window

      const int32_t* table = a.b.table + (size_t)q.slot * a.b.table_width;
      const int shift = __ffs(a.c.block) - 1;
      const auto block_of = [&](int i) {  // of the key group's tile i; -1 outside the pool
        const int id = __ldg(table + (tiles.token(lo + kg + i * KW) >> shift));
        return id < a.c.n_blocks ? id : -1;
      };
      int ids = 0;  // lane j: the block of issued tile (i & ~31) + j
      const auto issue = [&](int i) {
        if ((i & 31) == 0) ids = i + lane < n ? block_of(i + lane) : -1;
        const int id = __shfl_sync(0xffffffffu, ids, i & 31);
        if (lane == 0) {
          const int at = it0 + i, st = at % ST;
          // a wait that runs out leaves a stage that nothing is copied into: its consumers' waits run out too
          if (at < ST || mbar_wait(empty + st, (uint32_t)(at / ST - 1) & 1u)) {
            if (id >= 0) {
              const size_t off = (((size_t)id * a.c.kv_heads + head) * a.c.block + (tiles.token(lo + kg + i * KW) & (a.c.block - 1))) * DIM;
              mbar_expect_tx(full + st, S::kStageBytes);
              bulk_g2s(ring + st * S::kStageBytes, static_cast<const int8_t*>(a.c.k) + off, kTile * DIM, full + st);
              bulk_g2s(ring + st * S::kStageBytes + kTile * DIM, static_cast<const int8_t*>(a.c.v) + off, kTile * DIM, full + st);
            } else {
              mbar_arrive(full + st);
            }
          }
        }
        __syncwarp();
      };
      if (mw == 0)
        for (int i = 0; i < min(n, ST - 1); ++i) issue(i);
      float a_b = 0.f, lc_b = 0.f, ic_b = 0.f;  // lane j: scales of tile (i & ~31) + j
      bool expired = false;
      for (int i = 0; i < n; ++i) {
        if ((i & 31) == 0) {
          const int id = i + lane < n ? block_of(i + lane) : -1;
          const float nan = __uint_as_float(0x7fc00000u);
          a_b = id >= 0 ? __ldg(a.c.k_scale + (size_t)id * a.c.kv_heads + head) : nan;
          const float c = id >= 0 ? __ldg(a.c.v_scale + (size_t)id * a.c.kv_heads + head) : nan;
          const float cs = c == 0.f ? 0x1p-80f : c;  // a scale of 0 stands for values of 0, of their weight all the same
          // (approximate: 2^-22 of the logarithm is 2^-17 at a scale of 2^-32, where a weight in fp16 rounds by
          // 2^-11; 2^-23 of the reciprocal)
          lc_b = lg2_approx(cs);
          ic_b = rcp_approx(cs);
        }
        if (mw == 0 && i + ST - 1 < n) issue(i + ST - 1);
        const int at = it0 + i, st = at % ST;
        if (!__all_sync(0xffffffffu, mbar_wait(full + st, (uint32_t)(at / ST) & 1u))) {
          // what is still in flight lands before anything reuses the ring
          for (int j = at + 1; j < min(it0 + n, at + ST); ++j) mbar_wait(full + j % ST, (uint32_t)(j / ST) & 1u);
          expired = true;
          break;
        }
        const unsigned char* kt = ring + st * S::kStageBytes;
        const unsigned char* vt = kt + kTile * DIM;
        // scores: two column tiles of eight keys
        float s[2][4];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
          for (int u = 0; u < DIM / 64; ++u) {
            const uint4 x = *reinterpret_cast<const uint4*>(kt + (nt * 8 + g) * DIM + 64 * u + 16 * t);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t y = w[j] ^ 0x80808080u;
              mma16816(s[nt], qf[4 * u + j], int_half2(__byte_perm(y, 0x64646464u, 0x4140)), int_half2(__byte_perm(y, 0x64646464u, 0x4342)));
            }
          }
        }
        const int tok0 = tiles.token(lo + kg + i * KW);
        const float ab = __shfl_sync(0xffffffffu, a_b, i & 31), lc = __shfl_sync(0xffffffffu, lc_b, i & 31), ic = __shfl_sync(0xffffffffu, ic_b, i & 31);
        float top[2] = {-INFINITY, -INFINITY};
        const bool whole = tok0 + kTile - 1 <= all_to && (tok0 >= all_from || tok0 + kTile <= a.sinks);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float c = rc[h] * ab;
#pragma unroll
          for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float v = fmaf(s[nt][2 * h + e], c, lc);
              if (!whole) {
                const int key = tok0 + nt * 8 + 2 * t + e;
                const bool see = key <= pos[h] && (a.window <= 0 || key > pos[h] - a.window || key < a.sinks);
                v = see ? v : -INFINITY;
              }
              s[nt][2 * h + e] = v;
              top[h] = fmaxf(top[h], v);
            }
        }
        if (__any_sync(0xffffffffu, top[0] > m[0] + 8.f || top[1] > m[1] + 8.f)) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float x = fmaxf(m[h], top[h]);
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
            const float w = x == m[h] ? 1.f : ex2_approx(m[h] - x);
            m[h] = x;
            l[h] *= w;
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
              o[j][2 * h] *= w;
              o[j][2 * h + 1] *= w;
            }
          }
        }
        uint32_t p[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float ref = m[h] == -INFINITY ? 0.f : m[h] - 7.f;
          float sum = 0.f;
#pragma unroll
          for (int nt = 0; nt < 2; ++nt) {
            const float x = ex2_approx(s[nt][2 * h] - ref), y = ex2_approx(s[nt][2 * h + 1] - ref);
            sum += x + y;
            p[2 * nt + h] = narrow2<false>(x, y);
          }
          if (sum != 0.f) l[h] = fmaf(sum, ic, l[h]);  // a block that the row does not see may have a NaN scale
        }
        // values: keys 2t, 2t+1, 2t+8, 2t+9 of 16 (8) dimensions
        constexpr int kW = DIM / 32;  // words per key
        uint32_t v[4][kW];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const unsigned char* src = vt + (2 * t + (j & 1) + 8 * (j >> 1)) * DIM + (DIM / 8) * g;
          if constexpr (DIM == 128) {
            const uint4 x = *reinterpret_cast<const uint4*>(src);
            v[j][0] = x.x, v[j][1] = x.y, v[j][2] = x.z, v[j][3] = x.w;
          } else {
            const uint2 x = *reinterpret_cast<const uint2*>(src);
            v[j][0] = x.x, v[j][1] = x.y;
          }
        }
        // the stage has been read
        __syncwarp();
        if (lane == 0) mbar_arrive(empty + st);
#pragma unroll
        for (int w = 0; w < kW; ++w) {
          const uint32_t x0 = v[0][w] ^ 0x80808080u, x1 = v[1][w] ^ 0x80808080u, y0 = v[2][w] ^ 0x80808080u, y1 = v[3][w] ^ 0x80808080u;
          const uint32_t xl = __byte_perm(x0, x1, 0x5140), xh = __byte_perm(x0, x1, 0x7362);
          const uint32_t yl = __byte_perm(y0, y1, 0x5140), yh = __byte_perm(y0, y1, 0x7362);
          mma16816(o[4 * w], p, int_half2(__byte_perm(xl, 0x64646464u, 0x4140)), int_half2(__byte_perm(yl, 0x64646464u, 0x4140)));
          mma16816(o[4 * w + 1], p, int_half2(__byte_perm(xl, 0x64646464u, 0x4342)), int_half2(__byte_perm(yl, 0x64646464u, 0x4342)));
          mma16816(o[4 * w + 2], p, int_half2(__byte_perm(xh, 0x64646464u, 0x4140)), int_half2(__byte_perm(yh, 0x64646464u, 0x4140)));
          mma16816(o[4 * w + 3], p, int_half2(__byte_perm(xh, 0x64646464u, 0x4342)), int_half2(__byte_perm(yh, 0x64646464u, 0x4342)));
        }
      }
      dead = __any_sync(0xffffffffu, expired);
      if (dead) {  // the rows say NaN
        l[0] = l[1] = __uint_as_float(0x7fc00000u);
        m[0] = m[1] = 0.f;
      }
      it0 += n;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
      }
    } else if (kg == 0 && (dead || blockIdx.x == 0)) {
      m[0] = m[1] = 0.f;
      l[0] = l[1] = __uint_as_float(0x7fc00000u);
    }

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // join the key groups through shared memory (the ring's: every stage has been read)
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = warp * 16 + g + 8 * h;
      if (t == 0) s_ml[r] = make_float2(m[h], l[h]);
      // column tile j, column c: dimension c (DIM / 8) + j; this lane has columns 2t and 2t + 1
      float* dst = s_out + r * S::kOutStride + (DIM / 4) * t;
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int j = 0; j < kCols; j += 4)
          *reinterpret_cast<float4*>(dst + e * kCols + j) = make_float4(o[j][2 * h + e], o[j + 1][2 * h + e], o[j + 2][2 * h + e], o[j + 3][2 * h + e]);
    }
    __syncthreads();
    constexpr int kOct = DIM / 8;
    for (int e = threadIdx.x; e < 16 * kRowTiles * kOct; e += 128) {
      const int row = e / kOct, col = 8 * (e % kOct), r = mt * 16 * kRowTiles + row;
      if (r >= rows) break;
      emit_row<BF16, DIM>(a, q, r, head, col, s_ml + row, 16 * kRowTiles, s_out + row * S::kOutStride + col, 16 * kRowTiles * S::kOutStride, KW);
    }
    fence_async_smem();
    dead = __syncthreads_or(dead);  // then the ring is written again
  }
}

// Up to 8 NT rows per CTA of W warps (more rows: in turns).  Each warp takes every W-th
// stage of two 16-key units, which it copies into a ring of its own.
template <int DIM, int NT, int W>
struct EightShape {
  static constexpr int kStages = 2;
  static constexpr int kUnitBytes = 2 * kTile * DIM;       // keys, then values
  static constexpr int kRing = W * kStages * 2 * kUnitBytes;
  static constexpr int kOutStride = DIM + 4;
  static constexpr int kQStride = DIM + 8;  // fp16 queries, padded
  static constexpr int kQOff = kRing;
  static constexpr int kBarOff = kQOff + 8 * NT * (kQStride * 2 + 8);
  static constexpr int kSmem = kBarOff + W * kStages * 8 + W * 8 * NT * 8;
  static_assert(W * 8 * NT * kOutStride * 4 <= kRing, "the warps' results pass through the ring");
};

// The transpose of an 8 x 8 matrix of 16-bit elements spread over a warp.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

template <bool BF16, int DIM, int NT, int W>
__global__ void __launch_bounds__(32 * W, 12 / W) k_kv8_eight(const __grid_constant__ Kv8Attend a) {
  using S = EightShape<DIM, NT, W>;
  constexpr int ST = S::kStages;
  constexpr int kSteps = DIM / 16, kTiles = DIM / 16, kRows = 8 * NT;  // k-steps of the scores; 16-dimension tiles of the results
  extern __shared__ __align__(128) unsigned char smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kBarOff) + warp * ST;
  float2* s_ml = reinterpret_cast<float2*>(smem + S::kBarOff + W * ST * 8);  // [warp][row] maximum, sum
  float* s_out = reinterpret_cast<float*>(smem);
  unsigned char* ring = smem + warp * ST * 2 * S::kUnitBytes;
  uint16_t* s_q = reinterpret_cast<uint16_t*>(smem + S::kQOff);               // [rows][kQStride]
  float* s_rc = reinterpret_cast<float*>(smem + S::kQOff + kRows * S::kQStride * 2);  // [rows]
  const int head = blockIdx.y % a.c.kv_heads, mt0 = blockIdx.y / a.c.kv_heads, mts = gridDim.y / a.c.kv_heads;
  const Kv8Seq q = kv8_seq(a.c, a.b, blockIdx.z);
  const int rows = q.count * a.group;
  if (mt0 * kRows >= rows) return;
  if (lane < ST) mbar_init(full + lane, 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncwarp();
  const int shift = __ffs(a.c.block) - 1;
  int it0 = 0;        // stages of this warp so far
  bool dead = false;  // a wait of this CTA ran out: NaN for its rows from there on

  for (int mt = mt0; mt * kRows < rows; mt += mts) {
    const int r0 = mt * kRows;
    float m[NT][2], l[NT][2];  // rows 8 c + 2t, 8 c + 2t + 1
    float o[NT][kTiles][4];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      m[c][0] = m[c][1] = -INFINITY;
      l[c][0] = l[c][1] = 0.f;
#pragma unroll
      for (int j = 0; j < kTiles; ++j) o[c][j][0] = o[c][j][1] = o[c][j][2] = o[c][j][3] = 0.f;
    }
    if (q.ok && !dead) {
      const int before = q.len - q.count;
      const KeyTiles units = key_tiles(before + r0 / a.group, before + (min(rows, r0 + kRows) - 1) / a.group, a.window, a.sinks);
      const int all = (units.total + 1) / 2;
      const int lo = share_from(all, blockIdx.x, gridDim.x), hi = share_from(all, blockIdx.x + 1, gridDim.x);
      const int n = hi - lo > warp ? (hi - lo - warp + W - 1) / W : 0;  // this warp's stages lo + warp + W i
      const int32_t* table = a.b.table + (size_t)q.slot * a.b.table_width;
      // unit u of stage i in the list of units
      const auto unit_at = [&](int i, int u) { return 2 * (lo + warp + W * i) + u; };
      const auto block_of = [&](int v) {
        const int id = v < units.total ? __ldg(table + (units.token(v) >> shift)) : -1;
        return id < a.c.n_blocks ? id : -1;
      };
      int ids = -1;  // lane 2 j + u: the block of unit u of stage (i & ~15) + j
      const auto issue = [&](int i) {
        if ((i & 15) == 0) ids = i + (lane >> 1) < n ? block_of(unit_at(i + (lane >> 1), lane & 1)) : -1;
        const int id0 = __shfl_sync(0xffffffffu, ids, 2 * (i & 15)), id1 = __shfl_sync(0xffffffffu, ids, 2 * (i & 15) + 1);
        const int st = (it0 + i) % ST;
        if (lane == 0) {
          const uint32_t bytes = ((id0 >= 0) + (id1 >= 0)) * S::kUnitBytes;
          if (bytes) mbar_expect_tx(full + st, bytes);
          else mbar_arrive(full + st);
        }
        __syncwarp();
        // lanes 0 .. 3: keys and values of the two units
        const int id = lane & 2 ? id1 : id0;
        if (lane < 4 && id >= 0) {
          const size_t off = (((size_t)id * a.c.kv_heads + head) * a.c.block + (units.token(unit_at(i, lane >> 1)) & (a.c.block - 1))) * DIM;
          bulk_g2s(ring + st * 2 * S::kUnitBytes + (lane >> 1) * S::kUnitBytes + (lane & 1) * kTile * DIM,
                   static_cast<const int8_t*>(lane & 1 ? a.c.v : a.c.k) + off, kTile * DIM, full + st);
        }
        __syncwarp();
      };
      for (int i = 0; i < min(n, ST); ++i) issue(i);

      // the queries as fp16, scaled by f: each thread its part of a row, then the warps' fragments
      {
        constexpr int kPer = 32 * W / kRows, kQuads = DIM / kPer / 4;  // threads per row, groups of four elements per thread
        const int row = threadIdx.x / kPer, part = threadIdx.x % kPer, r = r0 + row, tok = r / a.group;
        uint2 w[kQuads];
        float top = 0.f;
        bool odd = false;
        const uint16_t* src = a.q + (int64_t)(q.row0 + tok) * a.q_row + (int64_t)(head * a.group + r - tok * a.group) * a.q_head + 4 * part;
#pragma unroll
        for (int k = 0; k < kQuads; ++k) w[k] = r < rows ? __ldg(reinterpret_cast<const uint2*>(src + 4 * kPer * k)) : make_uint2(0, 0);
#pragma unroll
        for (int k = 0; k < kQuads; ++k) {
          const float x0 = fabsf(wide16<BF16>(w[k].x & 0xffffu)), x1 = fabsf(wide16<BF16>(w[k].x >> 16));
          const float x2 = fabsf(wide16<BF16>(w[k].y & 0xffffu)), x3 = fabsf(wide16<BF16>(w[k].y >> 16));
          top = fmaxf(fmaxf(top, fmaxf(x0, x1)), fmaxf(x2, x3));
          odd = odd || !(x0 + x1 + x2 + x3 <= INFINITY);
        }
        top = odd ? INFINITY : top;
#pragma unroll
        for (int d = 1; d < kPer; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const QueryScale qs = query_scale(top);
        if (part == 0) s_rc[row] = qs.fine ? a.scale * kLog2e / qs.f : __uint_as_float(0x7fc00000u);
#pragma unroll
        for (int k = 0; k < kQuads; ++k)
          *reinterpret_cast<uint2*>(s_q + row * S::kQStride + 4 * (part + kPer * k)) =
              make_uint2(narrow2<false>(wide16<BF16>(w[k].x & 0xffffu) * qs.f, wide16<BF16>(w[k].x >> 16) * qs.f),
                         narrow2<false>(wide16<BF16>(w[k].y & 0xffffu) * qs.f, wide16<BF16>(w[k].y >> 16) * qs.f));
      }
      __syncthreads();
      uint32_t qf[NT][kSteps][2];  // rows 8 c + g
      float rc[NT][2];
      int pos[NT][2];
#pragma unroll
      for (int c = 0; c < NT; ++c) {
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
          const uint2 w = *reinterpret_cast<const uint2*>(s_q + (8 * c + g) * S::kQStride + 64 * (kk >> 2) + 16 * t + 4 * (kk & 3));
          qf[c][kk][0] = w.x;
          qf[c][kk][1] = w.y;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          rc[c][h] = s_rc[8 * c + 2 * t + h];
          pos[c][h] = before + min(r0 + 8 * c + 2 * t + h, rows - 1) / a.group;
        }
      }
      // positions that every row sees
      const int all_to = before + r0 / a.group;
      const int all_from = a.window > 0 ? before + (min(rows, r0 + kRows) - 1) / a.group - a.window + 1 : 0;

      float a_b = 0.f, lc_b = 0.f, ic_b = 0.f;  // lane 2 j + u: scales of unit u of stage (i & ~15) + j
      bool expired = false;
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        if ((i & 15) == 0) {
          const int id = i + (lane >> 1) < n ? block_of(unit_at(i + (lane >> 1), lane & 1)) : -1;
          const float nan = __uint_as_float(0x7fc00000u);
          a_b = id >= 0 ? __ldg(a.c.k_scale + (size_t)id * a.c.kv_heads + head) : nan;
          const float c = id >= 0 ? __ldg(a.c.v_scale + (size_t)id * a.c.kv_heads + head) : nan;
          const float cs = c == 0.f ? 0x1p-80f : c;  // a scale of 0 stands for values of 0, of their weight all the same
          lc_b = lg2_approx(cs);
          ic_b = rcp_approx(cs);
        }
        const int at = it0 + i, st = at % ST;
        if (!__all_sync(0xffffffffu, mbar_wait(full + st, (uint32_t)(at / ST) & 1u))) {
          for (int j = at + 1; j < min(it0 + n, at + ST); ++j) mbar_wait(full + j % ST, (uint32_t)(j / ST) & 1u);
          expired = true;
          break;
        }
        const unsigned char* stage = ring + st * 2 * S::kUnitBytes;
        float s[NT][2][4];  // unit u's keys g, g + 8 x rows 2t, 2t + 1
        float top[NT][2], ic[2];
#pragma unroll
        for (int c = 0; c < NT; ++c) top[c][0] = top[c][1] = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int c = 0; c < NT; ++c) s[c][u][0] = s[c][u][1] = s[c][u][2] = s[c][u][3] = 0.f;
          const unsigned char* kt = stage + u * S::kUnitBytes + g * DIM + 16 * t;
#pragma unroll
          for (int v = 0; v < DIM / 64; ++v) {
            const uint4 x = *reinterpret_cast<const uint4*>(kt + 64 * v), y = *reinterpret_cast<const uint4*>(kt + 8 * DIM + 64 * v);
            const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const uint32_t xx = xw[w] ^ 0x80808080u, yy = yw[w] ^ 0x80808080u;
              const uint32_t f[4] = {int_half2(__byte_perm(xx, 0x64646464u, 0x4140)), int_half2(__byte_perm(yy, 0x64646464u, 0x4140)),
                                     int_half2(__byte_perm(xx, 0x64646464u, 0x4342)), int_half2(__byte_perm(yy, 0x64646464u, 0x4342))};
#pragma unroll
              for (int c = 0; c < NT; ++c) mma16816(s[c][u], f, qf[c][4 * v + w][0], qf[c][4 * v + w][1]);
            }
          }
          const int from = 2 * (i & 15) + u;
          const float ab = __shfl_sync(0xffffffffu, a_b, from), lc = __shfl_sync(0xffffffffu, lc_b, from);
          ic[u] = __shfl_sync(0xffffffffu, ic_b, from);
          const int vu = unit_at(i, u), tok0 = units.token(vu);
          const bool whole = vu < units.total && tok0 + kTile - 1 <= all_to && (tok0 >= all_from || tok0 + kTile <= a.sinks);
#pragma unroll
          for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int h = e & 1;
              float x = fmaf(s[c][u][e], rc[c][h] * ab, lc);
              if (!whole) {
                const int key = tok0 + g + 8 * (e >> 1);
                const bool see = vu < units.total && key <= pos[c][h] && (a.window <= 0 || key > pos[c][h] - a.window || key < a.sinks);
                x = see ? x : -INFINITY;
              }
              s[c][u][e] = x;
              top[c][h] = fmaxf(top[c][h], x);
            }
        }
        bool grows = false;
#pragma unroll
        for (int c = 0; c < NT; ++c) grows = grows || top[c][0] > m[c][0] + 8.f || top[c][1] > m[c][1] + 8.f;
        if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
          for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float x = fmaxf(m[c][h], top[c][h]);
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
              const float w = x == m[c][h] ? 1.f : ex2_approx(m[c][h] - x);
              m[c][h] = x;
              l[c][h] *= w;
#pragma unroll
              for (int j = 0; j < kTiles; ++j) {
                o[c][j][h] *= w;
                o[c][j][2 + h] *= w;
              }
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          uint32_t b[NT][2];
#pragma unroll
          for (int c = 0; c < NT; ++c) {
            float p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = ex2_approx(s[c][u][e] - (m[c][e & 1] == -INFINITY ? 0.f : m[c][e & 1] - 7.f));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float sum = p[h] + p[2 + h];
              if (sum != 0.f) l[c][h] = fmaf(sum, ic[u], l[c][h]);  // a unit that the row does not see may have a NaN scale
            }
            b[c][0] = transpose8(narrow2<false>(p[0], p[1]));
            b[c][1] = transpose8(narrow2<false>(p[2], p[3]));
          }
          // values: keys 2t, 2t+1, 2t+8, 2t+9 of 16 (8) dimensions
          constexpr int kW = DIM / 32;  // words per key
          const unsigned char* vt = stage + u * S::kUnitBytes + kTile * DIM + 2 * t * DIM + (DIM / 8) * g;
          uint32_t v[4][kW];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const unsigned char* src = vt + ((j & 1) + 8 * (j >> 1)) * DIM;
            if constexpr (DIM == 128) {
              const uint4 x = *reinterpret_cast<const uint4*>(src);
              v[j][0] = x.x, v[j][1] = x.y, v[j][2] = x.z, v[j][3] = x.w;
            } else {
              const uint2 x = *reinterpret_cast<const uint2*>(src);
              v[j][0] = x.x, v[j][1] = x.y;
            }
          }
#pragma unroll
          for (int w = 0; w < kW; ++w) {
            const uint32_t x0 = v[0][w] ^ 0x80808080u, x1 = v[1][w] ^ 0x80808080u, y0 = v[2][w] ^ 0x80808080u, y1 = v[3][w] ^ 0x80808080u;
#pragma unroll
            for (int half = 0; half < 2; ++half) {  // dimensions 4 w + 2 half, and the next
              const uint32_t x = __byte_perm(x0, x1, half ? 0x7362 : 0x5140), y = __byte_perm(y0, y1, half ? 0x7362 : 0x5140);
              const uint32_t f[4] = {int_half2(__byte_perm(x, 0x64646464u, 0x4140)), int_half2(__byte_perm(x, 0x64646464u, 0x4342)),
                                     int_half2(__byte_perm(y, 0x64646464u, 0x4140)), int_half2(__byte_perm(y, 0x64646464u, 0x4342))};
#pragma unroll
              for (int c = 0; c < NT; ++c) mma16816(o[c][2 * w + half], f, b[c][0], b[c][1]);
            }
          }
        }
        __syncwarp();  // the stage has been read
        if (i + ST < n) issue(i + ST);
      }
      dead = expired;
      it0 += n;
#pragma unroll
      for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) l[c][h] += __shfl_xor_sync(0xffffffffu, l[c][h], d);
        }
    }
    if (dead || (!q.ok && warp == 0 && blockIdx.x == 0)) {
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        m[c][0] = m[c][1] = 0.f;
        l[c][0] = l[c][1] = __uint_as_float(0x7fc00000u);
      }
    }

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // join the warps through shared memory (the rings': every stage has been read)
    __syncthreads();
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = warp * kRows + 8 * c + 2 * t + h;
        if (g == 0) s_ml[row] = make_float2(m[c][h], l[c][h]);
        float* dst = s_out + row * S::kOutStride + (DIM / 8) * g;
#pragma unroll
        for (int j = 0; j < kTiles; j += 2)
          *reinterpret_cast<float4*>(dst + 2 * j) = make_float4(o[c][j][h], o[c][j][2 + h], o[c][j + 1][h], o[c][j + 1][2 + h]);
      }
    __syncthreads();
    constexpr int kOct = DIM / 8;
    for (int e = threadIdx.x; e < kRows * kOct; e += 32 * W) {
      const int row = e / kOct, col = 8 * (e % kOct), r = r0 + row;
      if (r >= rows) break;
      emit_row<BF16, DIM>(a, q, r, head, col, s_ml + row, kRows, s_out + row * S::kOutStride + col, kRows * S::kOutStride, W);
    }
    fence_async_smem();
    dead = __syncthreads_or(dead);  // then the rings are written again
  }
}

// Joins the splits' partial results: one warp per row and query head, lane = DIM / 32 dimensions.
template <bool BF16, int DIM>
__global__ void __launch_bounds__(128) k_kv8_join(const __grid_constant__ Kv8Attend a, int splits) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const size_t at = (size_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  const size_t items = (size_t)a.b.rows * a.heads;
  if (at >= items) return;
  const int tok = (int)(at / a.heads), h = (int)(at % a.heads);
  if (a.b.starts && (tok < __ldg(a.b.starts) || tok >= __ldg(a.b.starts + a.b.n))) return;
  float top = -INFINITY;
  for (int s = lane; s < splits; s += 32) top = fmaxf(top, a.part_ml[s * items + at].x);
#pragma unroll
  for (int i = 16; i; i >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i));
  constexpr int kN = DIM / 32;
  float acc[kN] = {}, sum = 0.f;
  for (int s = 0; s < splits; ++s) {
    const float2 ml = a.part_ml[s * items + at];
    if (ml.x == -INFINITY && ml.y == 0.f) continue;
    const float w = ml.x == -INFINITY ? 1.f : ex2_approx(ml.x - top);
    sum = fmaf(w, ml.y, sum);
    const float* src = a.part + (s * items + at) * DIM + kN * lane;
#pragma unroll
    for (int j = 0; j < kN; ++j) acc[j] = fmaf(w, src[j], acc[j]);
  }
  const float inv = 1.f / sum;
  uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + (int64_t)tok * a.out_row + (int64_t)h * a.out_head + kN * lane);
#pragma unroll
  for (int j = 0; j < kN; j += 2) dst[j / 2] = narrow2<BF16>(acc[j] * inv, acc[j + 1] * inv);
}

template <bool BF16, int DIM>
cudaError_t launch_rows(const Kv8Attend& a, int splits, int mtiles, cudaStream_t s) {
  using S = RowsShape<DIM>;
  const cudaError_t e = smem_opt_in<k_kv8_rows<BF16, DIM>>(S::kSmem);
  if (e != cudaSuccess) return e;
  k_kv8_rows<BF16, DIM><<<dim3(splits, mtiles * a.c.kv_heads, a.b.n), 128, S::kSmem, s>>>(a);
  return cudaGetLastError();
}

template <bool BF16, int DIM, int NT, int W>
cudaError_t launch_eight(const Kv8Attend& a, int splits, int mtiles, cudaStream_t s) {
  using S = EightShape<DIM, NT, W>;
  const cudaError_t e = smem_opt_in<k_kv8_eight<BF16, DIM, NT, W>>(S::kSmem);
  if (e != cudaSuccess) return e;
  k_kv8_eight<BF16, DIM, NT, W><<<dim3(splits, mtiles * a.c.kv_heads, a.b.n), 32 * W, S::kSmem, s>>>(a);
  return cudaGetLastError();
}

template <bool BF16, int DIM>
cudaError_t launch_dim(const Kv8Attend& a, const Kv8RowsPlan& p, cudaStream_t s) {
  if (p.rows <= 16 && p.warps == 2)
    return p.rows == 8 ? launch_eight<BF16, DIM, 1, 2>(a, p.splits, p.mtiles, s) : launch_eight<BF16, DIM, 2, 2>(a, p.splits, p.mtiles, s);
  return p.rows == 8    ? launch_eight<BF16, DIM, 1, 4>(a, p.splits, p.mtiles, s)
         : p.rows == 16 ? launch_eight<BF16, DIM, 2, 4>(a, p.splits, p.mtiles, s)
                        : launch_rows<BF16, DIM>(a, p.splits, p.mtiles, s);
}

template <bool BF16, int DIM>
cudaError_t launch_join(const Kv8Attend& a, int splits, cudaStream_t s) {
  const size_t items = (size_t)a.b.rows * a.heads;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((items + 3) / 4));
  cfg.blockDim = dim3(128);
  cfg.stream = s;
  cudaLaunchAttribute pdl{};
  pdl.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &pdl;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_kv8_join<BF16, DIM>, a, splits);
}

}  // namespace

Kv8RowsPlan kv8_rows_plan(const tsd_kv8& c, const tsd_kv8_batch& b, int heads, int window, int sinks, int sms) {
  Kv8RowsPlan p;
  const int group = heads / c.kv_heads;
  const int most = std::max(1, b.max_new ? std::min(b.max_new, b.rows) : (b.rows + b.n - 1) / b.n);
  const int64_t rows = (int64_t)most * group;
  p.rows = rows <= 8 ? 8 : rows <= 16 ? 16 : 32;
  const int64_t mtiles = (rows + p.rows - 1) / p.rows;
  p.mtiles = (int)std::min<int64_t>(mtiles, std::max(1, 65535 / c.kv_heads));
  const int64_t cap = std::min<int64_t>(b.max_len ? b.max_len : INT64_MAX, (int64_t)b.table_width * c.block);
  const int64_t keys = window > 0 ? std::min<int64_t>(cap, (int64_t)window + sinks + most) : cap;
  // CTAs wanted: four rounds of three per SM, so that ragged lengths even out (64 x 16000: 221 us; 239 with two rounds), in shares of at
  // least 1024 keys; where there are fewer sequences and heads than SMs, of 128
  const int64_t units = (int64_t)b.n * c.kv_heads * p.mtiles;
  const int64_t want = ((int64_t)sms * 12 + units - 1) / units;
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({want, keys / (units < sms ? 128 : 1024), 64}));
  // short shares in more CTAs than fit at once: two warps each, so that all start together (544 keys and 13
  // rows, 768 CTAs: 35.7 us, with four warps 44.8; 1200 keys, 1 row: 40.9 and 41.4; 2400: 73.7 and 70.9)
  p.warps = units * p.splits > 3 * sms && keys / p.splits <= 1024 ? 2 : 4;
  p.bytes = p.splits > 1 ? (int64_t)p.splits * b.rows * heads * (c.dim + 2) * 4 : 0;
  return p;
}

cudaError_t kv8_join_launch(const Kv8Attend& a, int splits, cudaStream_t s) {
  const bool bf = a.c.dtype == TSD_BF16;
  if (a.c.dim == 64) return bf ? launch_join<true, 64>(a, splits, s) : launch_join<false, 64>(a, splits, s);
  return bf ? launch_join<true, 128>(a, splits, s) : launch_join<false, 128>(a, splits, s);
}

cudaError_t kv8_rows_launch(const Kv8Attend& a, const Kv8RowsPlan& p, cudaStream_t s) {
  const bool bf = a.c.dtype == TSD_BF16;
  const cudaError_t e = a.c.dim == 64 ? (bf ? launch_dim<true, 64>(a, p, s) : launch_dim<false, 64>(a, p, s))
                                      : (bf ? launch_dim<true, 128>(a, p, s) : launch_dim<false, 128>(a, p, s));
  return e == cudaSuccess && p.splits > 1 ? kv8_join_launch(a, p.splits, s) : e;
}

}  // namespace tsd
