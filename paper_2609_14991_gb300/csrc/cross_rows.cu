// Attention over an encoder's states with few query rows per key head: a token of
// each hypothesis of an utterance (tsd.h: tsd_cross_attend).
//
// Mathematics, per row: s_j = (scale log2 e) q . k_j, m >= max_j s_j - 8 (fp16 states: 1),
//   out = sum_j 2^(s_j - m) v_j / sum_j 2^(s_j - m)
// in one pass over the frames; the maximum follows when a score passes it by more.
// Rows (row = token * group + head of the group) are taken 16 at a time, as the
// rows of mma.sync.m16n8k16 (fp32 accumulate).  A weight goes into the values'
// product as a sum of two 16-bit floats (cross.h), so it keeps 16 bits: the products
// are not what bounds this kernel.  fp16's end at 2^-24, and many frames far below a row's largest may be its result
// (where that one's values are 0): fp16 weights are taken relative to m - 14.
//
// Layout: a warp has frames of its own, 16 at a time, in a ring of its own that it
// fills with 16-byte asynchronous copies (frames past the length arrive as zeros), so
// its loop meets no barrier.  Both products may take their inner dimension in any
// order: lane (g, t) takes 16 consecutive bytes of key g as its part of two k-steps,
// and 16 consecutive bytes of values 2t, 2t+1, 2t+8, 2t+9 as its part of eight column
// tiles, so nothing is transposed.  The 16-byte chunks of a frame are permuted so that
// eight neighbouring lanes read all banks.
// Warps, then the CTAs of a cluster (a long source's frames are dealt out to up to
// eight), join their maxima, sums and results through shared memory.
//
// Bound by memory: 4 sources of 45000 frames, one row each, 8 key heads of 128: 88 us, 0.88 of the copy rate; 64 of 1500, 8
// rows, 16 heads of 64: 48.5 us, 0.82.  Rings of three steps (dim 64: four): with one more per warp fewer CTAs fit an SM (139 and 52
// us), with one less 102 and 49.  One row over 375 frames: 5.2 us, launch, length, frames and join one after the other.
#include <cooperative_groups.h>

#include <algorithm>

#include "cross.h"
#include "launch.h"
#include "tc_common.cuh"

namespace tsd {

namespace {

using namespace tc;
namespace cg = cooperative_groups;

constexpr int kTile = 16;  // frames per step of a warp
constexpr int kRows = 16;  // rows per CTA
constexpr int kMaxSplits = 8;

template <int DIM, int WARPS>
struct RowsShape {
  static constexpr int kStages = DIM == 128 ? 3 : 4;
  static constexpr int kHalf = kTile * DIM * 2;     // a step's keys, or its values
  static constexpr int kStageBytes = 2 * kHalf;
  static constexpr int kRing = WARPS * kStages * kStageBytes;
  static constexpr int kOutStride = DIM + 4;
  static constexpr int kOut = WARPS * kRows * kOutStride * 4;
  static constexpr int kMl = kRing > kOut ? kRing : kOut;  // [warps + 1][rows] (maximum, sum): the warps', the CTA's
  static constexpr int kSmem = kMl + (WARPS + 1) * kRows * 8;
};

template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 16 bytes to shared memory; zeros where there is nothing to read
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool have) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(have ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <bool BF16, int DIM, int kWarps>
__global__ void __launch_bounds__(32 * kWarps, (DIM == 128 ? 8 : 12) / kWarps) k_cross_rows(const __grid_constant__ CrossAttend a) {
  using S = RowsShape<DIM, kWarps>;
  constexpr int ST = S::kStages, kChunks = DIM / 8;  // 16-byte chunks of a frame
  constexpr int kSteps = DIM / 16, kCols = DIM / 8;
  // (weights up to 2^(kUp + kLag), fp16's largest is below 2^16; one is good to 2^-25, 2^-39 of the row's largest)
  constexpr float kUp = BF16 ? 0.f : 14.f, kLag = BF16 ? 8.f : 1.f;
  extern __shared__ __align__(128) unsigned char smem[];
  float* s_out = reinterpret_cast<float*>(smem);
  float2* s_ml = reinterpret_cast<float2*>(smem + S::kMl);
  const cg::cluster_group cluster = cg::this_cluster();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int splits = (int)cluster.num_blocks(), split = (int)cluster.block_rank();
  const int unit = blockIdx.x / splits, head = unit % a.s.kv_heads, mts = gridDim.x / splits / a.s.kv_heads;
  const CrossSeq q = cross_seq(a.s, a.b, blockIdx.y);
  const int rows = q.count * a.group;
  const int parts = splits * kWarps;
  const unsigned char* ring = smem + warp * ST * S::kStageBytes;
  const uint32_t ring32 = smem_u32(ring);
  const uint16_t* kbase = static_cast<const uint16_t*>(a.s.k) + (int64_t)q.source * a.s.k_source + (int64_t)head * a.s.k_head;
  const uint16_t* vbase = static_cast<const uint16_t*>(a.s.v) + (int64_t)q.source * a.s.v_source + (int64_t)head * a.s.v_head;
  const int tiles = (q.len + kTile - 1) / kTile;
  // this warp's tiles: lo .. lo + n - 1
  const int part = split * kWarps + warp;
  const int lo = (int)((int64_t)tiles * part / parts), n = (int)((int64_t)tiles * (part + 1) / parts) - lo;

  for (int mt = unit / a.s.kv_heads; mt * kRows < rows; mt += mts) {
    const int r0 = mt * kRows;
    if (q.ok) {
      const auto issue = [&](int i) {
        if (i < n) {
          const int f0 = (lo + i) * kTile;
          const uint32_t dst = ring32 + (i % ST) * S::kStageBytes;
#pragma unroll
          for (int j = 0; j < kTile * kChunks / 32; ++j) {
            const int f = (j * 32 + lane) / kChunks, c = (j * 32 + lane) % kChunks;
            const bool have = f0 + f < q.len;
            const int64_t at = have ? f0 + f : 0;
            copy16(dst + f * (DIM * 2) + ((c ^ ((f & 1) << 2)) << 4), kbase + at * a.s.k_frame + 8 * c, have);
            copy16(dst + S::kHalf + f * (DIM * 2) + ((c ^ (f & 6)) << 4), vbase + at * a.s.v_frame + 8 * c, have);
          }
        }
        copy_commit();
      };
#pragma unroll
      for (int i = 0; i < ST - 1; ++i) issue(i);
      // the queries' fragments
      uint32_t qf[kSteps][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = r0 + g + 8 * h, tok = q.row0 + r / a.group, hd = head * a.group + r % a.group;
#pragma unroll
        for (int u = 0; u < DIM / 32; ++u) {
          uint4 w = make_uint4(0, 0, 0, 0);
          if (r < rows) w = __ldg(reinterpret_cast<const uint4*>(a.q + (int64_t)tok * a.q_row + (int64_t)hd * a.q_head + 32 * u + 8 * t));
          qf[2 * u][h] = w.x, qf[2 * u][2 + h] = w.y, qf[2 * u + 1][h] = w.z, qf[2 * u + 1][2 + h] = w.w;
        }
      }
      const float c = a.scale * kLog2e;
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
      float o[kCols][4];
#pragma unroll
      for (int j = 0; j < kCols; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
      for (int i = 0; i < n; ++i) {
        copy_wait<ST - 2>();
        __syncwarp();
        issue(i + ST - 1);  // (its stage was read in the step before)
        const unsigned char* kt = ring + (i % ST) * S::kStageBytes;
        const unsigned char* vt = kt + S::kHalf;
        float s[2][4];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
          for (int u = 0; u < DIM / 32; ++u) {
            const uint4 w = *reinterpret_cast<const uint4*>(kt + (nt * 8 + g) * (DIM * 2) + (((4 * u + t) ^ ((g & 1) << 2)) << 4));
            mma<BF16>(s[nt], qf[2 * u], w.x, w.y);
            mma<BF16>(s[nt], qf[2 * u + 1], w.z, w.w);
          }
        }
        const int left = q.len - (lo + i) * kTile;  // frames from here on
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float v = s[nt][2 * h + e] * c;
              if (nt * 8 + 2 * t + e >= left) v = -INFINITY;
              s[nt][2 * h + e] = v;
              top[h] = fmaxf(top[h], v);
            }
        if (__any_sync(0xffffffffu, top[0] > m[0] + kLag || top[1] > m[1] + kLag)) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float x = fmaxf(m[h], top[h]);
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
            const float w = x == m[h] ? 1.f : ex2_approx(m[h] - x);
            m[h] = x;
            l[h] *= w;
#pragma unroll
            for (int j = 0; j < kCols; ++j) o[j][2 * h] *= w, o[j][2 * h + 1] *= w;
          }
        }
        uint32_t p[4], rest[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float ref = m[h] == -INFINITY ? 0.f : m[h] - kUp;
#pragma unroll
          for (int nt = 0; nt < 2; ++nt) {
            const float x = ex2_approx(s[nt][2 * h] - ref), y = ex2_approx(s[nt][2 * h + 1] - ref);
            l[h] += x + y;
            weight_parts<BF16>(x, y, p[2 * nt + h], rest[2 * nt + h]);
          }
        }
        // values: frames 2t, 2t+1, 2t+8, 2t+9; eight dimensions from 64 u + 8 g
#pragma unroll
        for (int u = 0; u < DIM / 64; ++u) {
          uint32_t x[4][4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int f = 2 * t + (j & 1) + 8 * (j >> 1);
            const uint4 w = *reinterpret_cast<const uint4*>(vt + f * (DIM * 2) + (((8 * u + g) ^ (f & 6)) << 4));
            x[j][0] = w.x, x[j][1] = w.y, x[j][2] = w.z, x[j][3] = w.w;
          }
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t b0 = __byte_perm(x[0][w], x[1][w], 0x5410), b1 = __byte_perm(x[2][w], x[3][w], 0x5410);
            const uint32_t d0 = __byte_perm(x[0][w], x[1][w], 0x7632), d1 = __byte_perm(x[2][w], x[3][w], 0x7632);
            mma<BF16>(o[8 * u + 2 * w], p, b0, b1);
            mma<BF16>(o[8 * u + 2 * w + 1], p, d0, d1);
            mma<BF16>(o[8 * u + 2 * w], rest, b0, b1);
            mma<BF16>(o[8 * u + 2 * w + 1], rest, d0, d1);
          }
        }
        __syncwarp();  // all lanes have read the stage
      }
      copy_wait<0>();
      // the warps' shares: (maximum, sum) and results
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        if (t == 0) s_ml[warp * kRows + g + 8 * h] = make_float2(m[h], l[h]);
      }
      __syncthreads();  // every warp is done with its ring, where the results go
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int u = 0; u < DIM / 64; ++u)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float* dst = s_out + (warp * kRows + g + 8 * h) * S::kOutStride + 64 * u + 8 * (2 * t + e);
            *reinterpret_cast<float4*>(dst) = make_float4(o[8 * u][2 * h + e], o[8 * u + 1][2 * h + e], o[8 * u + 2][2 * h + e], o[8 * u + 3][2 * h + e]);
            *reinterpret_cast<float4*>(dst + 4) = make_float4(o[8 * u + 4][2 * h + e], o[8 * u + 5][2 * h + e], o[8 * u + 6][2 * h + e], o[8 * u + 7][2 * h + e]);
          }
    }
    // The warps' shares are joined in place of the first's, then (splits) the CTAs' by the CTA of the cluster that takes the row's
    // dimensions, all of them read at once.
    __syncthreads();
    const int vecs = min(kRows, rows - r0) * (DIM / 4);
    const bool seen = q.ok && q.len > 0;
    struct Share {
      float top, sum;
      float4 acc;
      __device__ __forceinline__ void add(float2 ml, float4 v) {  // (top is known; -inf: every score is, and 0 / 0 is the result)
        const float f = ml.x == top ? 1.f : ex2_approx(ml.x - top);
        sum = fmaf(f, ml.y, sum);
        acc.x = fmaf(f, v.x, acc.x), acc.y = fmaf(f, v.y, acc.y), acc.z = fmaf(f, v.z, acc.z), acc.w = fmaf(f, v.w, acc.w);
      }
    };
    const auto own = [&](int rr, int col) {
      Share x{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll
      for (int w = 0; w < kWarps; ++w) x.top = fmaxf(x.top, s_ml[w * kRows + rr].x);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) x.add(s_ml[w * kRows + rr], *reinterpret_cast<const float4*>(s_out + (w * kRows + rr) * S::kOutStride + col));
      return x;
    };
    if (splits > 1) {
      if (seen)
        for (int i = threadIdx.x; i < vecs; i += 32 * kWarps) {
          const int rr = i / (DIM / 4), col = 4 * (i % (DIM / 4));
          const Share x = own(rr, col);
          *reinterpret_cast<float4*>(s_out + rr * S::kOutStride + col) = x.acc;
          if (col == 0) s_ml[kWarps * kRows + rr] = make_float2(x.top, x.sum);
        }
      cluster.sync();
    }
    for (int i = split * 32 * kWarps + threadIdx.x; i < vecs; i += splits * 32 * kWarps) {
      const int rr = i / (DIM / 4), col = 4 * (i % (DIM / 4)), r = r0 + rr;
      Share x{0.f, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
      if (!q.ok) {
        x.sum = __uint_as_float(0x7fc00000u);
      } else if (!seen) {
        x.sum = 1.f;
      } else if (splits == 1) {
        x = own(rr, col);
      } else {
        float2 ml[kMaxSplits];
        float4 v[kMaxSplits];
#pragma unroll
        for (int k = 0; k < kMaxSplits; ++k)
          if (k < splits) {
            ml[k] = cluster.map_shared_rank(s_ml, k)[kWarps * kRows + rr];
            v[k] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(s_out, k) + rr * S::kOutStride + col);
          }
        x.top = -INFINITY;
#pragma unroll
        for (int k = 0; k < kMaxSplits; ++k)
          if (k < splits) x.top = fmaxf(x.top, ml[k].x);
#pragma unroll
        for (int k = 0; k < kMaxSplits; ++k)
          if (k < splits) x.add(ml[k], v[k]);
      }
      const float inv = 1.f / x.sum;
      const int tok = q.row0 + r / a.group, hd = head * a.group + r % a.group;
      *reinterpret_cast<uint2*>(a.out + (int64_t)tok * a.out_row + (int64_t)hd * a.out_head + col) =
          make_uint2(narrow2<BF16>(x.acc.x * inv, x.acc.y * inv), narrow2<BF16>(x.acc.z * inv, x.acc.w * inv));
    }
    if (splits > 1) cluster.sync();  // the others have read this CTA's shares
    else __syncthreads();
  }
}

template <bool BF16, int DIM, int kWarps>
cudaError_t launch(const CrossAttend& a, const CrossRowsPlan& p, cudaStream_t s) {
  using S = RowsShape<DIM, kWarps>;
  const cudaError_t e = smem_opt_in<k_cross_rows<BF16, DIM, kWarps>>(S::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t c{};
  c.gridDim = dim3((unsigned)(a.s.kv_heads * p.mtiles * p.splits), (unsigned)a.b.n);
  c.blockDim = 32 * kWarps;
  c.dynamicSmemBytes = S::kSmem;
  c.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = (unsigned)p.splits, at.val.clusterDim.y = 1, at.val.clusterDim.z = 1;
  c.attrs = &at;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, k_cross_rows<BF16, DIM, kWarps>, a);
}

template <bool BF16, int DIM>
cudaError_t launch_warps(const CrossAttend& a, const CrossRowsPlan& p, cudaStream_t s) {
  return p.warps == 2 ? launch<BF16, DIM, 2>(a, p, s) : launch<BF16, DIM, 4>(a, p, s);
}

}  // namespace

CrossRowsPlan cross_rows_plan(const tsd_states& s, const tsd_cross_batch& b, int heads, int sms) {
  CrossRowsPlan p;
  const int group = heads / s.kv_heads;
  const int64_t most = std::max<int64_t>(1, b.max_rows ? std::min(b.max_rows, b.rows) : !b.starts ? 1 : ((int64_t)b.rows + b.n - 1) / b.n);
  p.mtiles = (int)std::min<int64_t>((most * group + kRows - 1) / kRows, 65535);
  // Few row tiles: a source's frames over up to eight CTAs, two steps for each warp at least (one row, 8 key heads, dim 64, us: over 375
  // frames 5.2 with two steps or more, over 750 5.6 with two, 6.4 with four, over 3000 6.7 and 8.7 with six).
  const int64_t units = (int64_t)b.n * s.kv_heads * p.mtiles, slots = (s.dim == 128 ? 2 : 3) * (int64_t)sms;
  while (p.splits < kMaxSplits && units * p.splits * 2 <= slots && (int64_t)p.splits * 2 * 4 * kTile * 2 <= s.frames) p.splits *= 2;
  // More than the device holds at once, of four warps each, but not of two: one turn instead of one and a part, in which few would
  // read (64 sources of 1500 frames, 8 rows, 8 key heads, dim 64: 35 us, 44; 128: 62, 65.  Two turns of two are worse than more of
  // four where sources are long: 16 heads, ragged: 58, 48; 160 of 1500, 8 heads: 93, 76.)  Of short sources a CTA's start, join and
  // end are a good part, and more of them at once hide it (300 sources, 8 heads, dim 64, of 60 frames: 12.8 us, 18.6; 200: 27.4, 32.5;
  // 375: 42.6, 45.2; 500: 53.2, 55.3.  Dim 128, 60: 18.4, 27.6; 375: 73, 78.  160 sources, dim 128: 375: 48.5, 46.8; 500: 60.6, 59.4;
  // 750: 87.8, 83.7.)
  if (units > slots && (units <= 2 * slots || s.frames <= 400)) p.warps = 2;
  return p;
}

cudaError_t cross_rows_launch(const CrossAttend& a, const CrossRowsPlan& p, cudaStream_t s) {
  const bool bf = a.s.dtype == TSD_BF16;
  return a.s.dim == 64 ? (bf ? launch_warps<true, 64>(a, p, s) : launch_warps<false, 64>(a, p, s)) : (bf ? launch_warps<true, 128>(a, p, s) : launch_warps<false, 128>(a, p, s));
}

}  // namespace tsd
