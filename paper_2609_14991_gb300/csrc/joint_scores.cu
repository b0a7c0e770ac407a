// Scores of labels from a joint network's input rows (tsd.h:
// tsd_joint_label_scores): the product A . Wt^T on the tensor cores with the
// scores' sums, the given labels' logits and the best labels taken in its
// epilogue; logits never leave the SM.
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
// The best labels: a thread keeps its best in order in registers, and logits
// above its last one go to a small buffer in shared memory first (three
// instructions each, only where one of eight neighbours passes in some
// lane); the buffer is sorted in when one of the warp's fills.
#include <cuda.h>

#include <algorithm>

#include "internal.h"
#include "label_scores.h"
#include "tc_common.cuh"

namespace tsd {

namespace {

using namespace tc;

constexpr int kEpiWarps = 16;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kBuf = 16;  // candidates per thread between sorts

struct JointScoreArgs {
  LabelArgs o;
  int n, H, C;
  int Nt;          // label tiles
  int tiles;       // row tiles x label tiles
  int workers;     // CTAs or pairs
  int segs;        // most partial results per row
  float* given;    // [n][m] the given labels' logits
  float* part;     // [n][segs][3 + 2 K]: m, S, E, logits, labels
};

// the worker whose range of tiles holds tile t (worker p has tiles p T / P .. (p + 1) T / P)
__host__ __device__ __forceinline__ int worker_of(int64_t t, int64_t tiles, int64_t workers) {
  return (int)(((t + 1) * workers - 1) / tiles);
}

template <int BN, bool PAIR>
struct ScoreShape {
  static constexpr int kABytes = kBM * kBK * 2;
  static constexpr int kBRows = PAIR ? BN / 2 : BN;
  static constexpr int kStageBytes = kABytes + kBRows * kBK * 2;
  static constexpr int kParts = BN / 32 < 4 ? BN / 32 : 4;  // warps of a lane quadrant with work
  static constexpr int kCols = BN / kParts;                 // columns of a warp
  static constexpr int kBufBytes = kEpiWarps * 32 * kBuf * 8;
  static constexpr int kFit = (227 * 1024 - 1024 - 512 - kBufBytes) / kStageBytes;
  static constexpr int kStages = kFit < 12 ? kFit : 12;
  static constexpr int kBufOff = kStages * kStageBytes;
  static constexpr int kBarOff = kBufOff + kBufBytes;
  static constexpr int kSmem = kBarOff + 512 + 1024;
  static_assert((2 * kStages + 5) * 8 + 4 <= 512, "barrier area");
  static_assert(kSmem <= 227 * 1024 && kStages >= 4, "shared memory per CTA");
  static_assert(kBufBytes >= kEpiWarps * 32 * (3 + 2 * kMaxAlt) * 4, "the parts' results pass through the buffer");
};

template <int K>
struct Best {
  float v[K > 0 ? K : 1];
  int i[K > 0 ? K : 1];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < K; ++j) {
      v[j] = -INFINITY;
      i[j] = 0x7fffffff;
    }
  }
  // in descending order, equal logits by label
  __device__ __forceinline__ void insert(float y, int label) {
#pragma unroll
    for (int j = K - 1; j >= 0; --j) {
      const bool here = y > v[j] || (y == v[j] && label < i[j]);
      const bool above = j > 0 && (y > v[j - 1] || (y == v[j - 1] && label < i[j - 1]));
      v[j] = here ? (above ? v[j - 1] : y) : v[j];
      i[j] = here ? (above ? i[j - 1] : label) : i[j];
    }
  }
};

template <int BN, bool PAIR, int K>
__global__ void __launch_bounds__(kThreads, 1)
    k_joint_scores(const __grid_constant__ JointScoreArgs a, const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB) {
  using S = ScoreShape<BN, PAIR>;
  constexpr int kStages = S::kStages;
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
    Best<K> best;
    best.clear();
    int cnt = 0, tl = 0;
    bool ok = true;
    const auto sort_in = [&]() {
      const int most = __reduce_max_sync(0xffffffffu, cnt);
      for (int j = 0; j < most; ++j)
        if (j < cnt) {
          const float2 y = buf[j * 32];
          best.insert(y.x, __float_as_int(y.y));
        }
      cnt = 0;
    };
    for (int t = first; t < last; ++t, ++tl) {
      const int ab = tl & 1;
      const int mt = t / a.Nt, row = mt * kTM + rank * kBM + q * 32 + lane, n0 = t % a.Nt * BN;
      // also the warps without columns: none hands a tile back before it is there
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait(accf + ab, (uint32_t)(tl >> 1) & 1u));
      if (ok && part < S::kParts && row - lane < a.n) {
        fence_after();
        int given[kMaxGiven];
#pragma unroll
        for (int j = 0; j < kMaxGiven; ++j) given[j] = j < a.o.m && row < a.n ? __ldg(a.o.labels + (int64_t)row * a.o.m + j) : -1;
#pragma unroll 1
        for (int h = 0; h < S::kCols / 32; ++h) {
          const int c0 = n0 + part * S::kCols + 32 * h;
          if (c0 >= a.C) break;
          float v[32];
          __syncwarp();
          tmem_ld32(tmem + (uint32_t)(ab * BN + part * S::kCols + 32 * h) + ((uint32_t)(q * 32) << 16), v);
          if (c0 + 32 > a.C) {  // past the last label
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (c0 + j >= a.C) v[j] = -INFINITY;
          }
          // given labels among these
#pragma unroll
          for (int j = 0; j < kMaxGiven; ++j) {
            if (j >= a.o.m) break;
            const int at = given[j] - c0;
            const bool here = at >= 0 && at < 32;
            if (__any_sync(0xffffffffu, here)) {
              float x = 0.f;
#pragma unroll
              for (int i = 0; i < 32; ++i) x = at == i ? v[i] : x;
              if (here) a.given[(int64_t)row * a.o.m + j] = x;
            }
          }
          // eighths' and the whole's maxima
          float top[4];
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            top[g] = fmaxf(fmaxf(fmaxf(v[8 * g], v[8 * g + 1]), fmaxf(v[8 * g + 2], v[8 * g + 3])),
                           fmaxf(fmaxf(v[8 * g + 4], v[8 * g + 5]), fmaxf(v[8 * g + 6], v[8 * g + 7])));
          }
          const float all = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
          if (__any_sync(0xffffffffu, all > m)) {
            const float to = fmaxf(m, all);
            const float d = m == -INFINITY ? 0.f : (m - to) * c, w = ex2_approx(d);
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
            float bound = best.v[K - 1];
            if (__any_sync(0xffffffffu, all > bound)) {
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                if (__any_sync(0xffffffffu, top[g] > bound)) {
                  if (__any_sync(0xffffffffu, cnt > kBuf - 8)) {
                    sort_in();
                    bound = best.v[K - 1];
                  }
#pragma unroll
                  for (int j = 0; j < 8; ++j)
                    if (v[8 * g + j] > bound) {
                      buf[cnt * 32] = make_float2(v[8 * g + j], __int_as_float(c0 + 8 * g + j));
                      ++cnt;
                    }
                }
              }
            }
          }
        }
      }
      // this warp's reads of the accumulator are done: hand it back
      fence_before();
      __syncwarp();
      if (ok && lane == 0) {
        if (rank == 0) mbar_arrive(acce + ab);
        else
          asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(map_rank(smem_u32(acce + ab), 0)) : "memory");
      }
      if (t + 1 == last || (t + 1) / a.Nt != mt) {
        // the row tile's last tile here: join the parts of each row and leave the result
        if constexpr (K > 0) {
          sort_in();
        }
        if (!ok) s = __uint_as_float(0x7fc00000u);
        constexpr int kF = 3 + 2 * K;
        float* parts = reinterpret_cast<float*>(quadrant) + lane;  // [part][kF][32]
        const auto bar = [&]() { asm volatile("bar.sync %0, 128;" ::"r"(1 + q) : "memory"); };
        bar();  // the quadrant's four warps: every buffer has been read ...
        if constexpr (S::kParts > 1) {
          if (part > 0 && part < S::kParts) {
            float* f = parts + part * kF * 32;
            f[0] = m, f[32] = s, f[64] = e;
#pragma unroll
            for (int j = 0; j < K; ++j) {
              f[(3 + j) * 32] = best.v[j];
              f[(3 + K + j) * 32] = __int_as_float(best.i[j]);
            }
          }
        }
        bar();
        if (part == 0) {
#pragma unroll 1
          for (int p = 1; p < S::kParts; ++p) {
            const float* f = parts + p * kF * 32;
            const float om = f[0];
            float os = f[32], oe = f[64];
            const float to = fmaxf(m, om);
            const float d0 = m == -INFINITY ? 0.f : (m - to) * c, w0 = ex2_approx(d0);
            const float d1 = om == -INFINITY ? 0.f : (om - to) * c, w1 = ex2_approx(d1);
            e = w0 * fmaf(d0, s, e) + w1 * fmaf(d1, os, oe);
            s = w0 * s + w1 * os;
            m = to;
#pragma unroll 1
            for (int j = 0; j < K; ++j) best.insert(f[(3 + j) * 32], __float_as_int(f[(3 + K + j) * 32]));
          }
          if (row < a.n) {
            const int seg = worker - worker_of((int64_t)mt * a.Nt, a.tiles, a.workers);
            float* f = a.part + ((int64_t)row * a.segs + seg) * kF;
            f[0] = m, f[1] = s, f[2] = e;
#pragma unroll
            for (int j = 0; j < K; ++j) {
              f[3 + j] = best.v[j];
              f[3 + K + j] = __int_as_float(best.i[j]);
            }
          }
        }
        bar();  // ... and the results, before the buffers are written again
        m = -INFINITY, s = 0.f, e = 0.f;
        best.clear();
      }
    }
  }
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

// Eight lanes per row join its partial results and write the scores.
template <int K>
__global__ void __launch_bounds__(128) k_joint_scores_join(const __grid_constant__ JointScoreArgs a, int rows_per_tile) {
  const int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 8;
  const int l = threadIdx.x & 7;
  const bool live = row < a.n;
  constexpr int kF = 3 + 2 * K;
  const int mt = (int)((live ? row : 0) / rows_per_tile);
  const int w0 = worker_of((int64_t)mt * a.Nt, a.tiles, a.workers), w1 = worker_of((int64_t)(mt + 1) * a.Nt - 1, a.tiles, a.workers);
  const int segs = live ? w1 - w0 + 1 : 0;
  const float* part = a.part + row * a.segs * kF;
  const auto widest = [](float x) {
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
  };
  const auto total = [](float x) {
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
  };
  const float c = a.o.inv_temp * kLog2e;
  float m = -INFINITY;
  for (int i = l; i < segs; i += 8) m = fmaxf(m, part[i * kF]);
  m = widest(m);
  float s = 0.f, e = 0.f;
  for (int i = l; i < segs; i += 8) {
    const float pm = part[i * kF], ps = part[i * kF + 1], pe = part[i * kF + 2];
    const float d = pm == -INFINITY ? 0.f : (pm - m) * c, w = ex2_approx(d);
    s += w * ps;
    e += w * fmaf(d, ps, pe);
  }
  const RowSums sums{m, total(s), total(e)};
  if (live) {
    label_finish(a.o, row, sums, l, [&](int label) {
      if (label >= a.C) return __uint_as_float(0x7fc00000u);
      return a.given[row * a.o.m + l];
    });
  }
  if constexpr (K > 0) {
    float pv = INFINITY;
    int pi = -1;
    for (int r = 0; r < a.o.k; ++r) {
      float bv = -INFINITY;
      int bi = 0x7fffffff;
      for (int i = l; i < segs * K; i += 8) {
        const float* f = part + (i / K) * kF + 3 + i % K;
        const float y = f[0];
        const int label = __float_as_int(f[K]);
        const bool after = y < pv || (y == pv && label > pi);
        if (after && (y > bv || (y == bv && label < bi))) bv = y, bi = label;
      }
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) {
        const float y = __shfl_xor_sync(0xffffffffu, bv, o);
        const int label = __shfl_xor_sync(0xffffffffu, bi, o);
        if (y > bv || (y == bv && label < bi)) bv = y, bi = label;
      }
      if (live && l == 0) label_alternative(a.o, row, r, sums, bv, bi);
      pv = bv;
      pi = bi;
    }
  }
}

struct ScorePlan {
  bool pair;
  int bn, tm, Nt, tiles, workers, segs, K;
  int64_t given, bytes;  // offset of the partial results, size of the workspace
};

// The tile shape: pairs of 256 x 256 once they fill the SMs; below, 128 x 128 and 128 x 64
// tiles put more SMs on the operands.
ScorePlan score_plan(int n, int H, int C, int m, int k, int sms) {
  ScorePlan p;
  const auto tiles_of = [&](int tm, int bn) { return (int64_t)((n + tm - 1) / tm) * ((C + bn - 1) / bn); };
  p.pair = tiles_of(256, 256) >= sms / 2;
  p.bn = p.pair ? 256 : tiles_of(128, 128) >= sms ? 128 : 64;
  p.tm = p.pair ? 256 : 128;
  p.Nt = (C + p.bn - 1) / p.bn;
  p.tiles = (int)tiles_of(p.tm, p.bn);
  p.workers = std::min(p.tiles, p.pair ? sms / 2 : sms);
  const int each = p.tiles / p.workers;  // fewest tiles of a worker
  p.segs = std::min(p.Nt, (p.Nt - 2 + each) / each + 1);
  p.K = k == 0 ? 0 : k <= 4 ? 4 : kMaxAlt;
  p.given = ((int64_t)n * m * 4 + 15) / 16 * 16;
  p.bytes = p.given + (int64_t)n * p.segs * (3 + 2 * p.K) * 4;
  return p;
}

template <int BN, bool PAIR, int K>
cudaError_t launch_shape(const ScorePlan& p, const JointScoreArgs& a, const CUtensorMap& tmA, const CUtensorMap& tmB, cudaStream_t s) {
  using S = ScoreShape<BN, PAIR>;
  cudaError_t e = cudaFuncSetAttribute(k_joint_scores<BN, PAIR, K>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
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
  e = cudaLaunchKernelEx(&cfg, k_joint_scores<BN, PAIR, K>, a, tmA, tmB);
  if (e != cudaSuccess) return e;
  k_joint_scores_join<K><<<(unsigned)((a.n + 15) / 16), 128, 0, s>>>(a, p.tm);
  return cudaGetLastError();
}

template <int K>
cudaError_t launch_k(const ScorePlan& p, const JointScoreArgs& a, const CUtensorMap& tmA, const CUtensorMap& tmB, cudaStream_t s) {
  if (p.pair) return launch_shape<256, true, K>(p, a, tmA, tmB, s);
  if (p.bn == 128) return launch_shape<128, false, K>(p, a, tmA, tmB, s);
  return launch_shape<64, false, K>(p, a, tmA, tmB, s);
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
  int dev = 0, sms = 0;
  TSD_CUDA(cudaGetDevice(&dev));
  TSD_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
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
  int dev = 0, sms = 0;
  TSD_CUDA(cudaGetDevice(&dev));
  TSD_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  const ScorePlan p = score_plan(n, H, C, m, k, sms);
  if (!workspace || workspace_bytes < p.bytes || reinterpret_cast<uintptr_t>(workspace) % 16)
    return fail(TSD_EINVAL, "%s: workspace of %lld bytes, %lld needed (16-byte aligned)", who, (long long)workspace_bytes, (long long)p.bytes);
  CUtensorMap tmA, tmB;
  if (!make_map(&tmA, A_bf16, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, H, n, kBK, kBM, CU_TENSOR_MAP_SWIZZLE_128B, a_stride) ||
      !make_map(&tmB, Wt_bf16, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, H, C, kBK, p.pair ? p.bn / 2 : p.bn, CU_TENSOR_MAP_SWIZZLE_128B, w_stride))
    return fail(TSD_ECUDA, "%s: cuTensorMapEncodeTiled failed", who);
  JointScoreArgs a{{m, k, labels, logp, entropy, alt_labels, alt_logp, 1.f / temperature}, n, H, C, p.Nt, p.tiles, p.workers, p.segs,
                   static_cast<float*>(workspace), reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + p.given)};
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  TSD_CUDA(p.K == 0 ? launch_k<0>(p, a, tmA, tmB, s) : p.K == 4 ? launch_k<4>(p, a, tmA, tmB, s) : launch_k<8>(p, a, tmA, tmB, s));
  return TSD_OK;
}
