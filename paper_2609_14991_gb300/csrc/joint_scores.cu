// Scores of labels from a joint network's input rows (tsd.h:
// tsd_joint_label_scores): the product A . Wt^T on the tensor cores.  From two
// 256 x 256 tiles per pair of SMs on, the scores' sums, the given labels' logits
// and the best labels are taken in its epilogue and no logit leaves the SM.
// Smaller calls store their logits (at most 40 MB, which stay in L2) and scores.cu's kernel
// follows: the epilogue's code runs once per tile there, and fetching it takes longer
// than running it (1001 x 640 x 1025 with 4 alternatives: 23.4 us fused, 13.0 stored).
//
// Mathematics: scores.cu's, with a running maximum m per row: when it grows to m',
// w = 2^((m - m') c), S := w S, E := w (E + (m - m') c S).
//
// Persistent: the tiles, label tiles of a row tile adjacent, are dealt out as one
// contiguous range per CTA (or CTA pair), so a row's sums and best labels stay in
// the registers of its threads over many label tiles; a row tile that two CTAs
// share leaves one partial result each, joined by k_joint_scores_join.  Warp 0
// streams operands by TMA, warp 1 issues the MMAs of tile i into accumulator i
// mod 2, warps 2-17 take tile i - 1 (thread = row; the four warps of a TMEM
// lane quadrant take a quarter of the columns each).
//
// The best labels: a thread keeps the K largest maxima of its groups of eight
// logits (two min/max instructions per place and group, no branch).  After
// each tile the four threads of a row show one another theirs: the K-th
// largest of all is a bound that K of the row's logits reach and hardly more.
// Only then are the tile's logits read again, and those that reach the bound put
// with their labels into a buffer in shared memory, unordered; a full buffer
// drops what the bound has passed since.  The row tile's end orders what is left.
#include <cuda.h>

#include <algorithm>

#include "internal.h"
#include "label_scores.h"
#include "launch.h"
#include "tc_pair.cuh"

namespace tsd {

namespace {

using namespace tc;

constexpr int kEpiWarps = 16;
constexpr int kThreads = 64 + 32 * kEpiWarps;
// Candidates per thread: what an ordering leaves, four more, and as much again as
// keeps a full buffer rare (K 8: 9059 orderings a call with 12, hardly any with 16).
template <int K>
constexpr int kBufOf = K <= 0 ? 0 : K + 8;

struct JointScoreArgs {
  LabelArgs o;
  int n, H, C;
  int Nt;          // label tiles
  int tiles;       // row tiles x label tiles
  int workers;     // CTAs or pairs
  int segs;        // most partial results per row
  float* logits;   // small calls: [n][ld]
  int ld;
  float* given;    // [n][m] the given labels' logits
  float4* part;    // [n][segs] partial results: m, S, E and the number of candidates
  float2* cand;    // [n][segs][4 K] logits and labels that may be among the row's best
};

// the worker whose range of tiles holds tile t (worker p has tiles p T / P .. (p + 1) T / P)
__host__ __device__ __forceinline__ int worker_of(int64_t t, int64_t tiles, int64_t workers) {
  return (int)(((t + 1) * workers - 1) / tiles);
}

// K: the most alternatives, or kStore: logits are stored
constexpr int kStore = -1;

template <int BN, bool PAIR, int K>
struct ScoreShape {
  static constexpr int kABytes = kBM * kBK * 2;
  static constexpr int kBRows = PAIR ? BN / 2 : BN;
  static constexpr int kStageBytes = kABytes + kBRows * kBK * 2;
  static constexpr int kParts = BN / 32 < 4 ? BN / 32 : 4;  // warps of a lane quadrant with work
  static constexpr int kCols = BN / kParts;                 // columns of a warp
  static constexpr int kBuf = kBufOf<K>;
  static constexpr int kBufBytes = kEpiWarps * 32 * kBuf * 8;
  static constexpr int kShownBytes = K < 0 ? 0 : 4 * 128 * (K > 4 ? K : 4) * 4;  // per part and row of the CTA
  static constexpr int kFit = (227 * 1024 - 1024 - 512 - kBufBytes - kShownBytes) / kStageBytes;
  static constexpr int kStages = kFit < 12 ? kFit : 12;
  static constexpr int kBufOff = kStages * kStageBytes;
  static constexpr int kShownOff = kBufOff + kBufBytes;
  static constexpr int kBarOff = kShownOff + kShownBytes;
  static constexpr int kSmem = kBarOff + 512 + 1024;
  static_assert((2 * kStages + 5) * 8 + 4 <= 512, "barrier area");
  static_assert(kSmem <= 227 * 1024 && kStages >= 4, "shared memory per CTA");
  static_assert(K <= 0 || (kParts == 4 && kCols == 64), "lists of four parts, of eight groups of eight each");
};

constexpr float kLowest = -3.402823466e38f;  // finite: masked logits (-inf) stay below it

// the next float above a finite one
__device__ __forceinline__ float above(float x) {
  int o = __float_as_int(x + 0.f);
  o = (o ^ ((o >> 31) & 0x7fffffff)) + 1;
  return __int_as_float(o ^ ((o >> 31) & 0x7fffffff));
}

// Makes room in a warp's buffers: what the bound has passed goes; where that
// leaves more than `full` (many logits reach it), all but the K best of this part, and the
// gate rises above the last of them.  A part's labels ascend in its buffer, so of equal
// logits the first are the better ones, and a later one is not among its best.
// Not inlined: rare, and called from many places.
struct Room {
  int cnt;
  float gate;
};
template <int K>
__device__ __noinline__ Room make_room(float2* buf, int cnt, float bound, float gate, int full) {
  const auto keep = [&](auto stays) {
    int to = 0;
    const int most = __reduce_max_sync(0xffffffffu, cnt);
#pragma unroll 1
    for (int j = 0; j < most; ++j) {
      const float2 y = buf[j * 32];
      if (j < cnt && stays(y.x)) {
        buf[to * 32] = y;
        ++to;
      }
    }
    cnt = to;
  };
  keep([&](float y) { return y >= bound; });
  if (__any_sync(0xffffffffu, cnt > full)) {
    float best[K];
#pragma unroll
    for (int i = 0; i < K; ++i) best[i] = -INFINITY;
    int most = __reduce_max_sync(0xffffffffu, cnt);
#pragma unroll 1
    for (int j = 0; j < most; ++j) {
      float y = j < cnt ? buf[j * 32].x : -INFINITY;
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const float hi = fmaxf(best[i], y);
        y = fminf(best[i], y);
        best[i] = hi;
      }
    }
    const float last = best[K - 1];  // -inf in a lane with fewer: all stay
    int equal = 0;                   // places for logits equal to the last
#pragma unroll
    for (int i = 0; i < K; ++i) equal += best[i] == last;
    keep([&](float y) { return y > last || (y == last && equal-- > 0); });
    if (last > -INFINITY) gate = fmaxf(gate, above(last));
  }
  return {cnt, gate};
}

// Puts those of 32 logits (labels from c0 on; maxima of eight each in top) that
// reach the gate into the buffers.
template <int K>
__device__ __forceinline__ void push32(const float (&v)[32], const float* top, int c0, float2* buf, int& cnt, float bound, float& gate) {
  constexpr int kBuf = kBufOf<K>;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    if (__any_sync(0xffffffffu, top[g] >= gate)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j % 4 == 0 && __any_sync(0xffffffffu, cnt > kBuf - 4)) {
          const Room r = make_room<K>(buf, cnt, bound, gate, kBuf - 4);
          cnt = r.cnt;
          gate = r.gate;
        }
        if (v[8 * g + j] >= gate) {
          buf[cnt * 32] = make_float2(v[8 * g + j], __int_as_float(c0 + 8 * g + j));
          ++cnt;
        }
      }
    }
  }
}

// The larger half of two lists in descending order (a[i] against b[K-1-i]), in order again.
template <int K>
__device__ __forceinline__ void merge_top(float (&a)[K], const float (&b)[K]) {
#pragma unroll
  for (int i = 0; i < K; ++i) a[i] = fmaxf(a[i], b[K - 1 - i]);
#pragma unroll
  for (int d = K / 2; d > 0; d >>= 1)
#pragma unroll
    for (int i = 0; i < K; ++i)
      if (!(i & d)) {
        const float hi = fmaxf(a[i], a[i + d]), lo = fminf(a[i], a[i + d]);
        a[i] = hi;
        a[i + d] = lo;
      }
}

// Enters eight group maxima into the list of the K largest (K 4 or 8).
template <int K>
__device__ __forceinline__ void enter(float (&kept)[K], const float (&groups)[8]) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = groups[i];
  // bitonic sort, descending
#pragma unroll
  for (int w = 2; w <= 8; w <<= 1)
#pragma unroll
    for (int d = w / 2; d > 0; d >>= 1)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (!(i & d)) {
          const float hi = fmaxf(x[i], x[i + d]), lo = fminf(x[i], x[i + d]);
          const bool down = (i & w) == 0;
          x[i] = down ? hi : lo;
          x[i + d] = down ? lo : hi;
        }
  float b[K];
#pragma unroll
  for (int i = 0; i < K; ++i) b[i] = x[i];
  merge_top<K>(kept, b);
}

// The K-th largest of the four parts' lists ([part][K / 4][128], this thread's row).
template <int K>
__device__ __forceinline__ float row_bound(const float4* shown) {
  float a[4][K];
#pragma unroll
  for (int p = 0; p < 4; ++p)
#pragma unroll
    for (int j = 0; j < K; j += 4) {
      float4 x;  // another warp may be writing it
      asm volatile("ld.volatile.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(smem_u32(shown + (p * (K / 4) + j / 4) * 128)));
      a[p][j] = x.x, a[p][j + 1] = x.y, a[p][j + 2] = x.z, a[p][j + 3] = x.w;
    }
  merge_top<K>(a[0], a[1]);
  merge_top<K>(a[2], a[3]);
  float least = INFINITY;
#pragma unroll
  for (int i = 0; i < K; ++i) least = fminf(least, fmaxf(a[0][i], a[2][K - 1 - i]));
  return least;
}

template <int BN, bool PAIR, int K>
__global__ void __launch_bounds__(kThreads, 1)
    k_joint_scores(const __grid_constant__ JointScoreArgs a, const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB) {
  using S = ScoreShape<BN, PAIR, K>;
  constexpr int kStages = S::kStages, kBuf = S::kBuf;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kBarOff);
  uint64_t* empty = full + kStages;
  uint64_t* accf = empty + kStages;  // [2] accumulator holds a finished tile
  uint64_t* acce = accf + 2;         // [2] accumulator read out by the epilogue (of both CTAs)
  uint64_t* drain = acce + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);

  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int rank = PAIR ? (int)(blockIdx.x & 1) : 0;
  const int worker = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x;
  const int KB = a.H / kBK;
  constexpr int kTM = PAIR ? 2 * kBM : kBM;  // rows per tile
  const int first = (int)((int64_t)a.tiles * worker / a.workers), last = (int)((int64_t)a.tiles * (worker + 1) / a.workers);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(accf + b, 1);
      mbar_init(acce + b, kEpiWarps * (PAIR ? 2 : 1));  // one arrival per epilogue warp
    }
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(2 * BN) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(2 * BN) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  fence_before();
  if constexpr (PAIR)  // the pair's barriers and accumulators exist before either CTA uses them
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  __syncthreads();
  fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == 0) {
    if (elect()) {
      int it = 0;
      bool ok = true;
      for (int t = first; t < last && ok; ++t) {
        const int m0 = t / a.Nt * kTM + rank * kBM, n0 = t % a.Nt * BN + rank * S::kBRows;
        for (int kb = 0; kb < KB; ++kb, ++it) {
          const int s = it % kStages;
          if (it >= kStages && !mbar_wait(empty + s, (uint32_t)(it / kStages - 1) & 1u)) {
            ok = false;
            break;
          }
          const uint32_t bar = PAIR ? map_rank(smem_u32(full + s), 0) : smem_u32(full + s);
          if (rank == 0) mbar_expect_tx(full + s, (PAIR ? 2 : 1) * S::kStageBytes);
          load_2d<PAIR>(smem + s * S::kStageBytes, &tmA, bar, kb * kBK, m0);
          load_2d<PAIR>(smem + s * S::kStageBytes + S::kABytes, &tmB, bar, kb * kBK, n0);
        }
      }
      if (!ok && rank == 0)  // the copies in flight land before the CTA goes (the leader's barriers count the pair's)
        for (int j = std::max(0, it - kStages); j < it; ++j) mbar_wait(full + j % kStages, (uint32_t)(j / kStages) & 1u);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && elect()) {
      const uint32_t idesc = idesc_bf16(kTM, BN);
      int tl = 0, s = 0;
      uint32_t ph = 0;
      bool ok = true, ready = mbar_test(full, 0);
      for (int t = first; t < last && ok; ++t, ++tl) {
        const int buf = tl & 1, use = tl >> 1;
        if (tl >= 2 && !mbar_wait(acce + buf, (uint32_t)(use - 1) & 1u)) {
          ok = false;
          break;
        }
        fence_after();
        const uint32_t acc = tmem + (uint32_t)(buf * BN);
        for (int kb = 0; kb < KB; ++kb) {
          if (!ready && !mbar_wait(full + s, ph)) {
            ok = false;
            break;
          }
          // the next stage's barrier is read while this stage's MMAs are issued
          const int s1 = s + 1 == kStages ? 0 : s + 1;
          const uint32_t ph1 = s1 == 0 ? ph ^ 1u : ph;
          ready = mbar_test(full + s1, ph1);
          fence_after();
          const uint32_t sa = smem_u32(smem + s * S::kStageBytes);
          const uint64_t ad = sw128_desc(sa), bd = sw128_desc(sa + S::kABytes);
#pragma unroll
          for (int k = 0; k < kBK / 16; ++k) mma<PAIR>(acc, ad + (uint64_t)(2 * k), bd + (uint64_t)(2 * k), idesc, (kb | k) ? 1u : 0u);
          commit<PAIR>(empty + s);
          s = s1;
          ph = ph1;
        }
        if (ok) commit<PAIR>(accf + buf);
      }
      if (!ok) {  // no tile is announced: the epilogue's wait runs out and its rows say NaN
        commit<PAIR>(drain);
        mbar_wait(drain, 0);
      }
    }
    __syncwarp();
  } else {
    const int q = warp & 3;            // TMEM lane quadrant this warp may access
    const int part = (warp - 2) >> 2;  // this warp among the quadrant's
    // the quadrant's share of the buffers: [part][kBuf][32]
    float2* quadrant = reinterpret_cast<float2*>(smem + S::kBufOff) + q * 4 * 32 * kBuf;
    float2* buf = quadrant + part * 32 * kBuf + lane;
    const float c = a.o.inv_temp * kLog2e;
    const uint64_t cc = pair_of(c, c);
    float m = -INFINITY, s = 0.f, e = 0.f;
    float bound = kLowest;  // K logits of the row reach it
    float gate = kLowest;   // what a later logit of this part has to reach: the bound, or more after a full ordering
    // the K largest of each part's group maxima so far, in order: [part][K / 4][128]
    float4* shown = reinterpret_cast<float4*>(smem + S::kShownOff) + q * 32 + lane;
    const auto bar = [&]() { asm volatile("bar.sync %0, 128;" ::"r"(1 + q) : "memory"); };  // the quadrant's four warps
    int cnt = 0, tl = 0;
    bool ok = true, opening = true;
    if constexpr (K > 0) {
#pragma unroll
      for (int j = 0; j < K; j += 4) shown[(part * (K / 4) + j / 4) * 128] = make_float4(kLowest, kLowest, kLowest, kLowest);
    }
    for (int t = first; t < last; ++t, ++tl) {
      const int ab = tl & 1;
      const int mt = t / a.Nt, row = mt * kTM + rank * kBM + q * 32 + lane, n0 = t % a.Nt * BN;
      // also the warps without columns: none hands a tile back before it is there
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait(accf + ab, (uint32_t)(tl >> 1) & 1u));
      const bool live = ok && part < S::kParts && row - lane < a.n;
      float groups[S::kCols / 8];  // maxima of eight logits each
#pragma unroll
      for (int g = 0; g < S::kCols / 8; ++g) groups[g] = -INFINITY;
      if (live) {
        fence_after();
#pragma unroll
        for (int h = 0; h < S::kCols / 32; ++h) {
          const int c0 = n0 + part * S::kCols + 32 * h;
          if (c0 >= a.C) break;
          float v[32];
          __syncwarp();
          tmem_ld32(tmem + (uint32_t)(ab * BN + part * S::kCols + 32 * h) + ((uint32_t)(q * 32) << 16), v);
          if constexpr (K == kStore) {  // past the last label too: rows are padded to whole 32s
            float4* to = reinterpret_cast<float4*>(a.logits + (int64_t)row * a.ld + c0);
            if (row < a.n) {
#pragma unroll
              for (int j = 0; j < 8; ++j) to[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            }
            continue;
          }
          if (c0 + 32 > a.C) {  // past the last label
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (c0 + j >= a.C) v[j] = -INFINITY;
          }
          // given labels among these
          for (int j = 0; j < a.o.m; ++j) {
            const int at = (row < a.n ? __ldg(a.o.labels + (int64_t)row * a.o.m + j) : -1) - c0;
            const bool here = at >= 0 && at < 32;
            if (__any_sync(0xffffffffu, here)) {
              float x = 0.f;
#pragma unroll
              for (int i = 0; i < 32; ++i) x = at == i ? v[i] : x;
              if (here) a.given[(int64_t)row * a.o.m + j] = x;
            }
          }
          // the groups' and the whole's maxima
          float* top = groups + 4 * h;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            top[g] = fmaxf(fmaxf(fmaxf(v[8 * g], v[8 * g + 1]), fmaxf(v[8 * g + 2], v[8 * g + 3])),
                           fmaxf(fmaxf(v[8 * g + 4], v[8 * g + 5]), fmaxf(v[8 * g + 6], v[8 * g + 7])));
          }
          const float all = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
          if (__any_sync(0xffffffffu, all > m)) {
            const float to = fmaxf(m, all);
            const float d = growth(m, to, c), w = ex2_approx(d);
            e = w * fmaf(d, s, e);
            s *= w;
            m = to;
          }
          const float ms = m == -INFINITY ? 0.f : m;
          uint64_t s2 = 0, e2 = 0;
          const uint64_t nm = pair_of(-ms, -ms);
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const uint64_t d = mul2(add2(pair_of(v[j], v[j + 1]), nm), cc);
            float d0, d1;
            unpair(d, d0, d1);
            d0 = max_nan(d0, -1e30f);
            d1 = max_nan(d1, -1e30f);
            const uint64_t p = pair_of(ex2_approx(d0), ex2_approx(d1));
            s2 = add2(s2, p);
            e2 = fma2(p, pair_of(d0, d1), e2);
          }
          float x0, x1;
          unpair(s2, x0, x1);
          s += x0 + x1;
          unpair(e2, x0, x1);
          e += x0 + x1;
          if constexpr (K > 0) {
            if (!opening) push32<K>(v, top, c0, buf, cnt, bound, gate);
          }
        }
      }
      if constexpr (K > 0) {
        // the part's maxima, the row's bound, and the logits that reach it
        float widest = groups[0];
#pragma unroll
        for (int g = 1; g < S::kCols / 8; ++g) widest = fmaxf(widest, groups[g]);
        if (__any_sync(0xffffffffu, widest > bound)) {
          float kept[K];
#pragma unroll
          for (int j = 0; j < K; j += 4) {
            const float4 x = shown[(part * (K / 4) + j / 4) * 128];
            kept[j] = x.x, kept[j + 1] = x.y, kept[j + 2] = x.z, kept[j + 3] = x.w;
          }
          enter<K>(kept, groups);
#pragma unroll
          for (int j = 0; j < K; j += 4) shown[(part * (K / 4) + j / 4) * 128] = make_float4(kept[j], kept[j + 1], kept[j + 2], kept[j + 3]);
        }
        // in step on a row tile's first tile; later the others' lists may be a tile old, or half
        // of each: every entry only grows, so the bound, which serves the next tile, holds all the same
        if (opening) bar();
        bound = fmaxf(bound, row_bound<K>(shown));
        gate = fmaxf(gate, bound);
        if (live && opening) {  // the first tile's logits again, now that there is a bound
#pragma unroll
          for (int h = 0; h < S::kCols / 32; ++h) {
            const int c0 = n0 + part * S::kCols + 32 * h;
            if (c0 >= a.C) break;
            float v[32];
            __syncwarp();
            tmem_ld32(tmem + (uint32_t)(ab * BN + part * S::kCols + 32 * h) + ((uint32_t)(q * 32) << 16), v);
            if (c0 + 32 > a.C) {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (c0 + j >= a.C) v[j] = -INFINITY;
            }
            push32<K>(v, groups + 4 * h, c0, buf, cnt, bound, gate);
          }
        }
        opening = false;
      }
      // this warp's reads of the accumulator are done: hand it back
      fence_before();
      __syncwarp();
      if (ok && lane == 0) {
        if (rank == 0) mbar_arrive(acce + ab);
        else
          asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(map_rank(smem_u32(acce + ab), 0)) : "memory");
      }
      if (K == kStore) {
        if (!ok && part == 0 && row < a.n) a.logits[(int64_t)row * a.ld + n0] = __uint_as_float(0x7fc00000u);
        continue;
      }
      if (t + 1 == last || (t + 1) / a.Nt != mt) {
        // the row tile's last tile here: join the parts of each row and leave the result
        if (!ok) s = __uint_as_float(0x7fc00000u);
        const int seg = worker - worker_of((int64_t)mt * a.Nt, a.tiles, a.workers);
        const int64_t at = (int64_t)row * a.segs + seg;
        if constexpr (K > 0) {
          bar();  // every part's last list is there
          bound = row_bound<K>(shown);
          cnt = make_room<K>(buf, cnt, bound, gate, 4 * K / S::kParts).cnt;
          bar();  // the lists have been read: the sums take their place
        }
        float4* sums = reinterpret_cast<float4*>(smem + S::kShownOff) + q * 32 + lane;  // [part][128] m, S, E, candidates
        sums[part * 128] = make_float4(m, s, e, __int_as_float(cnt));
        bar();
        float4 of[S::kParts];
        int all = 0, mine = 0;  // candidates of the row, and of the parts before this one
#pragma unroll
        for (int p = 0; p < S::kParts; ++p) {
          of[p] = sums[p * 128];
          if (p < part) mine += __float_as_int(of[p].w);
          all += __float_as_int(of[p].w);
        }
        if constexpr (K > 0) {
          if (row < a.n)
            for (int i = 0; i < cnt; ++i) a.cand[at * (4 * K) + mine + i] = buf[i * 32];
        }
        if (part == 0 && row < a.n) {
#pragma unroll
          for (int p = 1; p < S::kParts; ++p) {
            const float to = fmaxf(m, of[p].x);
            const float d0 = growth(m, to, c), w0 = ex2_approx(d0);
            const float d1 = growth(of[p].x, to, c), w1 = ex2_approx(d1);
            e = w0 * fmaf(d0, s, e) + w1 * fmaf(d1, of[p].y, of[p].z);
            s = w0 * s + w1 * of[p].y;
            m = to;
          }
          a.part[at] = make_float4(m, s, e, __int_as_float(all));
        }
        bar();  // before the buffers and the lists are written again
        m = -INFINITY, s = 0.f, e = 0.f;
        cnt = 0;
        bound = gate = kLowest;
        opening = true;
        if constexpr (K > 0) {
#pragma unroll
          for (int j = 0; j < K; j += 4) shown[(part * (K / 4) + j / 4) * 128] = make_float4(kLowest, kLowest, kLowest, kLowest);
        }
      }
    }
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  fence_before();
  __syncthreads();
  if constexpr (PAIR)  // neither CTA leaves while the other may still signal it or read its operands
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (warp == 1) {
    fence_after();
    if constexpr (PAIR)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * BN) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * BN) : "memory");
  }
}

// L lanes per row (8 or 32) join its partial results and write the scores.  A
// lane takes every fourth candidate of its partial results, with no load
// waiting for another but where a result has more than eight.  The K largest
// values come from lists in registers, as above; the candidates that reach
// the last of them, hardly more than K, are placed by counting better ones.
constexpr int kJoinCap = 32;
template <int K, int L>
__global__ void __launch_bounds__(128) k_joint_scores_join(const __grid_constant__ JointScoreArgs a, int rows_per_tile, int cap) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr int kRows = 128 / L;
  __shared__ float2 s_list[kRows][K > 0 ? kJoinCap : 1];
  __shared__ int s_count[kRows];
  const int slot = threadIdx.x / L;
  const int64_t row = (int64_t)blockIdx.x * kRows + slot;
  const int l = threadIdx.x & (L - 1);
  const bool live = row < a.n;
  const int mt = (int)((live ? row : 0) / rows_per_tile);
  const int w0 = worker_of((int64_t)mt * a.Nt, a.tiles, a.workers), w1 = worker_of((int64_t)(mt + 1) * a.Nt - 1, a.tiles, a.workers);
  const int segs = live ? w1 - w0 + 1 : 0;
  const float4* part = a.part + row * a.segs;
  const float2* cand = a.cand + row * a.segs * cap;
  const float c = a.o.inv_temp * kLog2e;
  if (l == 0) s_count[slot] = 0;
  // the given labels and their logits
  const int label = live && l < a.o.m ? __ldg(a.o.labels + row * a.o.m + l) : -1;
  const float x = label >= 0 && label < a.C ? a.given[row * a.o.m + l] : 0.f;
  // sums, of each partial result by one lane; values, by all
  float m = -INFINITY, s = 0.f, e = 0.f;
  float best[K > 0 ? K : 1];
#pragma unroll
  for (int i = 0; i < K; ++i) best[i] = kLowest;
  const auto enter_one = [&](float y) {
#pragma unroll
    for (int i = 0; i < K; ++i) {
      const float hi = fmaxf(best[i], y);
      y = fminf(best[i], y);
      best[i] = hi;
    }
  };
  const auto join = [&](float om, float os, float oe) {
    const float to = fmaxf(m, om);
    const float d0 = growth(m, to, c), x0 = ex2_approx(d0);
    const float d1 = growth(om, to, c), x1 = ex2_approx(d1);
    e = x0 * fmaf(d0, s, e) + x1 * fmaf(d1, os, oe);
    s = x0 * s + x1 * os;
    m = to;
  };
  // f(candidate) for each of this lane's
  const auto each = [&](auto f) {
    for (int u = l; u < segs * 4; u += L) {
      const float4 p = part[u >> 2];
      const float2* x = cand + (int64_t)(u >> 2) * cap;
      float2 y0, y1;
      if (K > 0) y0 = x[u & 3], y1 = x[(u & 3) + 4];  // within the result's places, filled or not
      f(p, u, true);
      if constexpr (K > 0) {
        const int n = __float_as_int(p.w);
        if ((u & 3) < n) f(y0);
        if ((u & 3) + 4 < n) f(y1);
        for (int j = (u & 3) + 8; j < n; j += 4) f(x[j]);
      }
    }
  };
  struct First {
    decltype(join)& add;
    decltype(enter_one)& enter;
    __device__ void operator()(const float4& p, int u, bool) {
      if ((u & 3) == 0) add(p.x, p.y, p.z);
    }
    __device__ void operator()(const float2& y) { enter(y.x); }
  };
  each(First{join, enter_one});
#pragma unroll
  for (int o = 1; o < L; o <<= 1) {
    const float om = __shfl_xor_sync(0xffffffffu, m, o), os = __shfl_xor_sync(0xffffffffu, s, o), oe = __shfl_xor_sync(0xffffffffu, e, o);
    // in the same order in both lanes: one result for the row
    if (l & o) {
      const float tm = m, ts = s, te = e;
      m = om, s = os, e = oe;
      join(tm, ts, te);
    } else {
      join(om, os, oe);
    }
    if constexpr (K > 0) {
      float b[K];
#pragma unroll
      for (int i = 0; i < K; ++i) b[i] = __shfl_xor_sync(0xffffffffu, best[i], o);
      merge_top<K>(best, b);
    }
  }
  const RowScore sums(RowSums{m, s, e});
  if (live) {
    if (l < a.o.m) a.o.logp[row * a.o.m + l] = label_given(a.o, sums, label, label < a.C ? x : __uint_as_float(0x7fc00000u));
    if (l == 0 && a.o.entropy) a.o.entropy[row] = sums.entropy;
  }
  if constexpr (K > 0) {
    const float bound = best[K - 1];
    struct Second {
      float bound;
      int* count;
      float2* list;
      __device__ void operator()(const float4&, int, bool) {}
      __device__ void operator()(const float2& y) {
        if (y.x >= bound) {
          const int at = atomicAdd(count, 1);
          if (at < kJoinCap) list[at] = y;
        }
      }
    };
    __syncwarp();
    each(Second{bound, &s_count[slot], s_list[slot]});
    __syncwarp();
    const int n = s_count[slot];
    if (!live) return;
    if (n <= kJoinCap) {
      for (int i = l; i < n; i += L) {
        const float2 y = s_list[slot][i];
        const int label = __float_as_int(y.y);
        int place = 0;
        for (int j = 0; j < n; ++j) {
          const float2 z = s_list[slot][j];
          place += z.x > y.x || (z.x == y.x && __float_as_int(z.y) < label) ? 1 : 0;
        }
        if (place < a.o.k) label_alternative(a.o, row, place, sums, y.x, label);
      }
      for (int j = n + l; j < a.o.k; j += L) label_alternative(a.o, row, j, sums, -INFINITY, -1);
    } else if (l == 0) {  // many equal logits: one lane looks for the next one k times
      float pv = INFINITY;
      int pi = -1;
      for (int r = 0; r < a.o.k; ++r) {
        float bv = -INFINITY;
        int bi = 0x7fffffff;
        for (int u = 0; u < segs; ++u)
          for (int j = 0; j < __float_as_int(part[u].w); ++j) {
            const float2 y = cand[(int64_t)u * cap + j];
            const int label = __float_as_int(y.y);
            const bool after = y.x < pv || (y.x == pv && label > pi);
            if (after && (y.x > bv || (y.x == bv && label < bi))) bv = y.x, bi = label;
          }
        label_alternative(a.o, row, r, sums, bv, bi);
        pv = bv;
        pi = bi;
      }
    }
  }
}

struct ScorePlan {
  bool store, pair;  // logits stored; pairs of CTAs
  int bn, tm, Nt, tiles, workers, segs, K, ld;
  int64_t given, bytes;  // offset of the partial results, size of the workspace
};

ScorePlan score_plan(int n, int H, int C, int m, int k, int sms) {
  ScorePlan p{};
  const auto tiles_of = [&](int tm, int bn) { return (int64_t)((n + tm - 1) / tm) * ((C + bn - 1) / bn); };
  p.store = tiles_of(256, 256) < 2 * (sms / 2);
  p.pair = !p.store;
  p.bn = 256;
  if (p.store) {
    // rounds of tiles times a k-block's clocks: its MMAs, or its operands at 64 bytes
    // per clock and SM
    const auto cost = [&](int tm, int bn, int slots, double mma, double rows) {
      const int64_t t = tiles_of(tm, bn);
      return (double)((t + slots - 1) / slots) * (H / kBK) * std::max(mma, rows * 128 / 64) + 12 * bn;
    };
    double best = cost(256, 256, sms / 2, 516, 256);
    p.pair = true;
    for (int bn : {128, 64}) {
      const double x = cost(128, bn, sms, bn == 128 ? 260 : 196, 128 + bn);
      if (x < best) best = x, p.bn = bn, p.pair = false;
    }
  }
  p.tm = p.pair ? 256 : 128;
  p.Nt = (C + p.bn - 1) / p.bn;
  p.tiles = (int)tiles_of(p.tm, p.bn);
  p.workers = std::min(p.tiles, p.pair ? sms / 2 : sms);
  if (p.store) {
    p.ld = (C + 31) / 32 * 32;
    p.bytes = (int64_t)n * p.ld * 4;
    return p;
  }
  const int each = p.tiles / p.workers;  // fewest tiles of a worker
  p.segs = std::min(p.Nt, (p.Nt - 2 + each) / each + 1);
  p.K = k == 0 ? 0 : k <= 4 ? 4 : kMaxAlt;
  p.given = ((int64_t)n * m * 4 + 15) / 16 * 16;
  p.bytes = p.given + (int64_t)n * p.segs * (16 + 4 * p.K * 8);
  return p;
}

template <int BN, bool PAIR, int K>
cudaError_t launch_tiles(const ScorePlan& p, const JointScoreArgs& a, const CUtensorMap& tmA, const CUtensorMap& tmB, cudaStream_t s) {
  using S = ScoreShape<BN, PAIR, K>;
  cudaError_t e = smem_opt_in<k_joint_scores<BN, PAIR, K>>(S::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(PAIR ? 2 * p.workers : p.workers));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = S::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = 2;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = PAIR ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, k_joint_scores<BN, PAIR, K>, a, tmA, tmB);
}

template <int K>
cudaError_t launch_fused(const ScorePlan& p, const JointScoreArgs& a, const CUtensorMap& tmA, const CUtensorMap& tmB, cudaStream_t s) {
  const cudaError_t e = launch_tiles<256, true, K>(p, a, tmA, tmB, s);
  if (e != cudaSuccess) return e;
  // few partial results per row: eight lanes; more (few rows, many labels): a warp
  const bool wide = p.segs > 4;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(wide ? (a.n + 3) / 4 : (a.n + 15) / 16));
  cfg.blockDim = dim3(128);
  cfg.stream = s;
  cudaLaunchAttribute pdl{};
  pdl.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &pdl;
  cfg.numAttrs = 1;
  return wide ? cudaLaunchKernelEx(&cfg, k_joint_scores_join<K, 32>, a, p.tm, 4 * K) : cudaLaunchKernelEx(&cfg, k_joint_scores_join<K, 8>, a, p.tm, 4 * K);
}

cudaError_t launch_stored(const ScorePlan& p, const JointScoreArgs& a, const CUtensorMap& tmA, const CUtensorMap& tmB, cudaStream_t s) {
  const cudaError_t e = p.pair        ? launch_tiles<256, true, kStore>(p, a, tmA, tmB, s)
                        : p.bn == 128 ? launch_tiles<128, false, kStore>(p, a, tmA, tmB, s)
                                      : launch_tiles<64, false, kStore>(p, a, tmA, tmB, s);
  return e == cudaSuccess ? label_rows_launch(a.o, a.logits, TSD_F32, a.ld, a.n, a.C, true, s) : e;
}

tsd_status check(const char* who, int32_t n, int32_t H, int32_t C) {
  if (n < 1 || n > (1 << 24)) return fail(TSD_EINVAL, "%s: n=%d outside [1, 2^24]", who, n);
  if (H < 64 || H > 8192 || H % 64) return fail(TSD_EINVAL, "%s: H=%d must be a multiple of 64 in [64, 8192]", who, H);
  if (C < 1 || C > 262144) return fail(TSD_EINVAL, "%s: C=%d outside [1, 262144]", who, C);
  if ((int64_t)((n + 255) / 256) * ((C + 255) / 256) > (1 << 24)) return fail(TSD_EINVAL, "%s: n=%d x C=%d is more than 2^40 logits", who, n, C);
  return TSD_OK;
}

}  // namespace

}  // namespace tsd

using namespace tsd;

extern "C" tsd_status tsd_joint_label_scores_workspace(int32_t n, int32_t H, int32_t C, int32_t m, int32_t k, int64_t* bytes) {
  clear_error();
  const char* who = "tsd_joint_label_scores_workspace";
  if (!bytes) return fail(TSD_EINVAL, "%s: NULL argument", who);
  if (tsd_status st = check(who, n, H, C)) return st;
  if (m < 0 || m > kMaxGiven || k < 0 || k > kMaxAlt) return fail(TSD_EINVAL, "%s: m=%d or k=%d outside [0, 8]", who, m, k);
  int sms = 0;
  TSD_CUDA(device_sms(&sms));
  *bytes = score_plan(n, H, C, m, k, sms).bytes;
  return TSD_OK;
}

extern "C" tsd_status tsd_joint_label_scores(int32_t n, int32_t H, int32_t C, const void* A_bf16, int64_t a_stride,
                                             const void* Wt_bf16, int64_t w_stride, float temperature, int32_t m,
                                             const int32_t* labels, int32_t k, float* logp, float* entropy,
                                             int32_t* alt_labels, float* alt_logp, void* workspace,
                                             int64_t workspace_bytes, void* cuda_stream) {
  clear_error();
  const char* who = "tsd_joint_label_scores";
  if (!A_bf16 || !Wt_bf16) return fail(TSD_EINVAL, "%s: NULL argument", who);
  if (tsd_status st = check(who, n, H, C)) return st;
  if (tsd_status st = label_check(who, n, 1 << 24, C, temperature, m, labels, k, logp, alt_labels, alt_logp)) return st;
  if (n == 1) a_stride = H;
  if (C == 1) w_stride = H;
  if (a_stride < H || w_stride < H || a_stride % 8 || w_stride % 8 || a_stride > (1ll << 36) || w_stride > (1ll << 36))
    return fail(TSD_EINVAL, "%s: strides %lld, %lld must be multiples of 8, at least H=%d", who, (long long)a_stride, (long long)w_stride, H);
  if (reinterpret_cast<uintptr_t>(A_bf16) % 16 || reinterpret_cast<uintptr_t>(Wt_bf16) % 16)
    return fail(TSD_EINVAL, "%s: A and Wt must be 16-byte aligned", who);
  int sms = 0;
  TSD_CUDA(device_sms(&sms));
  const ScorePlan p = score_plan(n, H, C, m, k, sms);
  if (!workspace || workspace_bytes < p.bytes || reinterpret_cast<uintptr_t>(workspace) % 16)
    return fail(TSD_EINVAL, "%s: workspace of %lld bytes, %lld needed (16-byte aligned)", who, (long long)workspace_bytes, (long long)p.bytes);
  CUtensorMap tmA, tmB;
  if (!make_strided_map(&tmA, A_bf16, H, n, a_stride, kBK, kBM) ||
      !make_strided_map(&tmB, Wt_bf16, H, C, w_stride, kBK, p.pair ? p.bn / 2 : p.bn))
    return fail(TSD_ECUDA, "%s: cuTensorMapEncodeTiled failed", who);
  JointScoreArgs a{};
  a.o = {m, k, labels, logp, entropy, alt_labels, alt_logp, 1.f / temperature};
  a.n = n, a.H = H, a.C = C;
  a.Nt = p.Nt, a.tiles = p.tiles, a.workers = p.workers, a.segs = p.segs;
  a.logits = static_cast<float*>(workspace);
  a.ld = p.ld;
  a.given = static_cast<float*>(workspace);
  a.part = reinterpret_cast<float4*>(static_cast<unsigned char*>(workspace) + p.given);
  a.cand = reinterpret_cast<float2*>(a.part + (int64_t)n * p.segs);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  TSD_CUDA(p.store ? launch_stored(p, a, tmA, tmB, s)
           : p.K == 0 ? launch_fused<0>(p, a, tmA, tmB, s)
           : p.K == 4 ? launch_fused<4>(p, a, tmA, tmB, s)
                      : launch_fused<kMaxAlt>(p, a, tmA, tmB, s));
  return TSD_OK;
}
