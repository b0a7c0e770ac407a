// Scores of labels from logits in memory (tsd.h: tsd_label_scores): log
// probabilities of given labels, entropy, top alternatives, in one pass over
// the logits.
//
// Mathematics, per row with m the largest logit, c = log2(e) / T, d_i = (x_i - m) c:
//   S = sum 2^d_i,  E = sum 2^d_i d_i,
//   log p(l) = (x_l - m) / T - ln S,   entropy = ln S - ln 2 E / S.
// x_i - m is formed first (exact or rounded once), so a row's offset costs no
// precision.  A row stays in registers as it came (32 logits per thread, 64 of long 16-bit rows): 32 to 512
// threads per row, above 16384 logits (32768 of 16 bits) a cluster of 2 to 8 CTAs of 512 that exchange
// through distributed shared memory.  The k largest: the threads form 16 groups (per CTA); the
// k-th largest of the groups' maxima is a bound that at least k logits reach and few pass
// (about 11 of random ones for 8; the least of eight classes' maxima let 22 pass, which took 1.4 times as long in all).  Threads that hold one
// leave it with its seven neighbours; one warp picks and orders, in k rounds of a
// maximum where more than 32 reach it.  If the gathering has no room for them (many equal
// logits), those rounds go over the whole row, by all threads of its CTA.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.h"
#include "label_scores.h"
#include "tc_common.cuh"

namespace tsd {

namespace {

namespace cg = cooperative_groups;
using namespace tc;

struct RowsArgs {
  LabelArgs o;
  const void* x;
  int64_t ld;
  int n, C;
};

constexpr int kCap = 64;     // logits that the last step takes
constexpr int kGroups = 16;  // groups of a CTA's threads (of a row's, where a warp takes one)

// A row's shared memory.  In a cluster every CTA writes its groups' maxima
// into each CTA's and its sums into the first CTA's; the first one fetches the
// eights gathered by the others.
template <int CS>
struct RowShared {
  static constexpr int kEights = CS == 1 ? 64 : 128;  // gathered per row
  float top[kGroups * CS];                            // groups' maxima
  float2 sums[16 * CS];                               // warps' S and E
  float4 eight[kEights][2];                           // eight logits of a thread, one of which reaches the bound
  int code[kEights];                                  // whose and which; below 0: a single logit's label, ~label
  float cv[kCap];                                     // the logits that reach it, and their labels
  int ci[kCap];
  int count;         // this CTA's eights
  float best_v[16];  // warps' best of a round over the whole row
  int best_i[16];
};

template <typename T>
__device__ __forceinline__ float to_float(T v) {
  return (float)v;
}

// eight consecutive logits from their words
template <typename T>
__device__ __forceinline__ void unpack(const uint32_t* w, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
      }
    }
  }
}
// -inf in every place of a word
template <typename T>
constexpr uint32_t kNoneWord = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, __nv_bfloat16>::value ? 0xff80ff80u : 0xfc00fc00u;

// order-preserving int of a float (-0 and 0 alike, no NaN)
__device__ __forceinline__ int order_of(float x) {
  const int i = __float_as_int(x + 0.f);
  return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float value_of(int o) { return __int_as_float(o ^ ((o >> 31) & 0x7fffffff)); }

__device__ __forceinline__ bool before(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

// the best (largest, then lowest label) of a warp's lanes
__device__ __forceinline__ void warp_best(float& v, int& i) {
  const int o = order_of(v), top = __reduce_max_sync(0xffffffffu, o);
  i = __reduce_min_sync(0xffffffffu, o == top ? i : 0x7fffffff);
  v = value_of(top);
}

template <typename T, int G, int CS, int E>
__global__ void __launch_bounds__(G == 32 ? 128 : G, E * sizeof(T) > 128 ? 1 : 1024 / (G == 32 ? 128 : G)) k_label_rows(const __grid_constant__ RowsArgs a) {
  constexpr int VE = 16 / sizeof(T), NV = E / VE;
  constexpr int kWarps = G / 32;
  constexpr int kLanes = G / kGroups;  // threads of a group
  constexpr int kRows = G == 32 ? 4 : 1;
  constexpr int kEights = E / 8;  // a thread's logits in eights
  __shared__ RowShared<CS> s_rows[kRows];
  const int warp_in_cta = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int slot = G == 32 ? warp_in_cta : 0, warp = G == 32 ? 0 : warp_in_cta;
  const int64_t row = (int64_t)(blockIdx.x / CS) * kRows + slot;
  asm volatile("griddepcontrol.wait;" ::: "memory");  // stored logits of joint rows: the product before
  if (row >= a.n) return;  // a whole warp (G 32) or none: the grid has n CTAs or clusters
  const int rank = CS > 1 ? (int)(blockIdx.x % CS) : 0;
  RowShared<CS>& sh = s_rows[slot];
  const auto peer = [&](int r) -> RowShared<CS>* {
    if constexpr (CS > 1) return cg::this_cluster().map_shared_rank(&sh, r);
    else return &sh;
  };
  const auto sync_cta = [&]() {
    if constexpr (G == 32) __syncwarp();
    else __syncthreads();
  };
  const auto sync_row = [&]() {
    if constexpr (CS > 1) cg::this_cluster().sync();
    else sync_cta();
  };
  // the cluster's CTAs have started before one writes to another (waited for below)
  if constexpr (CS > 1) cg::this_cluster().barrier_arrive();
  const int t = warp * 32 + lane, rt = rank * G + t;
  const T* x = static_cast<const T*>(a.x) + row * a.ld;
  const int C = a.C, k = a.o.k;

  // the given labels, on their way before the logits, and theirs after
  const int given = rt < a.o.m ? __ldg(a.o.labels + row * a.o.m + rt) : -1;
  float given_x = __uint_as_float(0x7fc00000u);

  // the logits: whole aligned vectors, and the ends one by one
  const int lead = min(C, (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(T));
  const int nvec = (C - lead) / VE, tail = C - lead - nvec * VE;
  constexpr int kWords = 2 * sizeof(T);  // of eight logits
  uint32_t held[E / 8 * kWords];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int j = rt + i * G * CS;
    uint4 w = make_uint4(kNoneWord<T>, kNoneWord<T>, kNoneWord<T>, kNoneWord<T>);
    if (j < nvec) w = __ldcs(reinterpret_cast<const uint4*>(x + lead) + j);
    held[4 * i] = w.x, held[4 * i + 1] = w.y, held[4 * i + 2] = w.z, held[4 * i + 3] = w.w;
  }
  if (given >= 0 && given < C) given_x = to_float(x[given]);
  const int xi = rt < lead ? rt : rt < lead + tail ? nvec * VE + rt : -1;
  const float xv = xi >= 0 ? to_float(x[xi]) : -INFINITY;
  const auto label_of = [&](int e) { return lead + (rt + e / VE * G * CS) * VE + e % VE; };

  // maxima: the thread's, the groups'
  const auto largest = [](const float (&v)[8]) { return fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7]))); };
  float mine = xv;
#pragma unroll
  for (int i = 0; i < kEights; ++i) {
    float v[8];
    unpack<T>(held + i * kWords, v);
    mine = fmaxf(mine, largest(v));
  }
  if (!(mine >= -INFINITY)) mine = INFINITY;  // NaN alone: the sums say so
  float gm = mine;
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) gm = fmaxf(gm, __shfl_xor_sync(0xffffffffu, gm, o));
  constexpr int kHeld = 32 / kLanes;  // groups of a warp
  if constexpr (CS == 1) {
    if (lane % kLanes == 0) sh.top[warp * kHeld + lane / kLanes] = gm;
  } else {
    // lane r of the warp (one group) writes to CTA r
    static_assert(CS == 1 || kLanes == 32, "a warp is a group");
    cg::this_cluster().barrier_wait();
    if (lane < CS) peer(lane)->top[rank * kGroups + warp] = gm;
  }
  if (t == 0) sh.count = 0;
  sync_row();
  // The row's maximum, and the k-th largest of the groups' maxima: a lane's place is the
  // number of larger ones (in a cluster of 32 classes of groups).
  constexpr int kClasses = CS > 1 ? 32 : kGroups;
  int key = order_of(sh.top[lane % (kGroups * CS)]);
#pragma unroll
  for (int i = 1; i < kGroups * CS / 32; ++i) key = max(key, order_of(sh.top[lane + 32 * i]));
  const float m = value_of(__reduce_max_sync(0xffffffffu, key));
  float bound = -INFINITY;
  if (k > 0) {
    // the class's number in the lowest bits: no two are equal, and the bound is lower by a few steps at most
    const int own = (key & -kClasses) | (lane & (kClasses - 1));
    int place = 0;
#pragma unroll
    for (int d = 1; d < kClasses; ++d) place += __shfl_xor_sync(0xffffffffu, own, d) > own ? 1 : 0;
    const int kth = __shfl_sync(0xffffffffu, own, __ffs(__ballot_sync(0xffffffffu, place == k - 1)) - 1) & -kClasses;
    bound = fmaxf(value_of(kth), -INFINITY);  // (a few steps below -inf is a NaN)
  }

  // (unpacked anew each time, not kept unpacked since the maxima: that took registers there are not)
  const auto forget = [&]() {
    if constexpr (E > 32 && sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < E / 8 * kWords; ++i) asm volatile("" : "+r"(held[i]));
    }
  };
  forget();

  // sums: in pairs, a masked logit's exponent held finite (its term is 0 all the same)
  const float ms = m == -INFINITY ? 0.f : m, c = a.o.inv_temp * kLog2e;
  uint64_t s2 = 0, e2 = 0;
  const uint64_t nm = pair_of(-ms, -ms), cc = pair_of(c, c);
#pragma unroll
  for (int i = 0; i < kEights; ++i) {
    float v[8];
    unpack<T>(held + i * kWords, v);
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const uint64_t d = mul2(add2(pair_of(v[e], v[e + 1]), nm), cc);
      float d0, d1;
      unpair(d, d0, d1);
      d0 = max_nan(d0, -1e30f);
      d1 = max_nan(d1, -1e30f);
      const uint64_t p = pair_of(ex2_approx(d0), ex2_approx(d1));
      s2 = add2(s2, p);
      e2 = fma2(p, pair_of(d0, d1), e2);
    }
  }
  float S, E2;
  {
    const float d = max_nan((xv - ms) * c, -1e30f), p = ex2_approx(d);
    float s0, s1, e0, e1;
    unpair(s2, s0, s1);
    unpair(e2, e0, e1);
    S = s0 + s1 + p;
    E2 = fmaf(p, d, e0 + e1);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    S += __shfl_xor_sync(0xffffffffu, S, o);
    E2 += __shfl_xor_sync(0xffffffffu, E2, o);
  }
  if (lane == 0) peer(0)->sums[rank * kWarps + warp] = make_float2(S, E2);

  // gather the eights with a logit that reaches the bound
  forget();
  constexpr int kMine = RowShared<CS>::kEights / CS;
  if (k > 0 && mine >= bound && mine > -INFINITY) {
#pragma unroll
    for (int i = 0; i < kEights; ++i) {
      float v[8];
      unpack<T>(held + i * kWords, v);
      if (largest(v) >= bound) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < kMine) {
          sh.eight[at][0] = make_float4(v[0], v[1], v[2], v[3]);
          sh.eight[at][1] = make_float4(v[4], v[5], v[6], v[7]);
          sh.code[at] = rt * kEights + i;
        }
      }
    }
    if (xv >= bound && xi >= 0) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < kMine) {
        sh.eight[at][0] = make_float4(xv, -INFINITY, -INFINITY, -INFINITY);
        sh.eight[at][1] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        sh.code[at] = ~xi;
      }
    }
  }
  sync_row();

  int count = sh.count;
  bool over = count > kMine;
  if constexpr (CS > 1) {
    if (rank == 0) {
      int theirs[CS];
#pragma unroll
      for (int r = 1; r < CS; ++r) theirs[r] = peer(r)->count;
#pragma unroll
      for (int r = 1; r < CS; ++r) over = over || theirs[r] > kMine;
      if (!over) {
        static_assert(kMine <= G, "a thread per gathered eight");
#pragma unroll
        for (int r = 1; r < CS; ++r) {
          if (t < theirs[r]) {
            sh.eight[count + t][0] = peer(r)->eight[t][0];
            sh.eight[count + t][1] = peer(r)->eight[t][1];
            sh.code[count + t] = peer(r)->code[t];
          }
          count += theirs[r];
        }
      }
    }
    cg::this_cluster().sync();  // the others' memory has been read
    if (rank != 0) return;
  }
  if (!over && warp != 0) return;
  RowSums total{m, 0.f, 0.f};
  if constexpr (kWarps == 1) {
    total.S = S;
    total.E = E2;
  } else if (warp == 0) {
#pragma unroll
    for (int i = 0; i < (kWarps * CS + 31) / 32; ++i) {
      const float2 y = lane + 32 * i < kWarps * CS ? sh.sums[lane + 32 * i] : make_float2(0.f, 0.f);
      total.S += y.x;
      total.E += y.y;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      total.S += __shfl_xor_sync(0xffffffffu, total.S, o);
      total.E += __shfl_xor_sync(0xffffffffu, total.E, o);
    }
  }
  const RowScore sums(total);
  if (t < a.o.m) a.o.logp[row * a.o.m + t] = label_given(a.o, sums, given, given_x);
  if (t == 0 && a.o.entropy) a.o.entropy[row] = sums.entropy;

  // the k best in order
  if (!over) {  // the first warp alone: all that reach the bound are in the gathered eights
    if (k == 0) return;
    const auto label_at = [&](int at, int j) {
      const int code = sh.code[at], e = code % kEights * 8 + j;
      return code < 0 ? ~code : lead + (code / kEights + e / VE * G * CS) * VE + e % VE;
    };
    const auto logit_at = [&](int at, int j) { return reinterpret_cast<const float*>(sh.eight[at])[j]; };
    // those logits, with their labels
    int found = 0;
    for (int base = 0; base < count; base += 4) {  // eight lanes per eight
      const int at = base + (lane >> 3), j = lane & 7;
      const float y = at < count ? logit_at(at, j) : -INFINITY;
      const bool in = y >= bound && y > -INFINITY;
      const unsigned who = __ballot_sync(0xffffffffu, in);
      const int to = found + __popc(who & ((1u << lane) - 1));
      if (in && to < kCap) {
        sh.cv[to] = y;
        sh.ci[to] = label_at(at, j);
      }
      found += __popc(who);
    }
    __syncwarp();
    if (found <= 32) {  // a logit's place is the number of better ones
      const float y0 = lane < found ? sh.cv[lane] : -INFINITY;
      const int i0 = lane < found ? sh.ci[lane] : 0x7fffffff;
      int place = 0;
#pragma unroll 4
      for (int j = 0; j < found; ++j) place += before(__shfl_sync(0xffffffffu, y0, j), __shfl_sync(0xffffffffu, i0, j), y0, i0) ? 1 : 0;
      if (lane < found && place < k) label_alternative(a.o, row, place, sums, y0, i0);
      if (lane >= found && lane < k) label_alternative(a.o, row, lane, sums, -INFINITY, -1);  // fewer than k
      return;
    }
    // more: k rounds of the best one after the last, in the list or, where it has no room, in the eights
    float pv = INFINITY;
    int pi = -1;
    for (int r = 0; r < k; ++r) {
      float bv = -INFINITY;
      int bi = 0x7fffffff;
      const auto look = [&](float y, int l) {
        if (y > -INFINITY && before(pv, pi, y, l) && before(y, l, bv, bi)) bv = y, bi = l;
      };
      if (found <= kCap) {
        for (int i = lane; i < found; i += 32) look(sh.cv[i], sh.ci[i]);
      } else {
        for (int i = lane; i < 8 * count; i += 32) look(logit_at(i >> 3, i & 7), label_at(i >> 3, i & 7));
      }
      warp_best(bv, bi);
      if (lane == 0) label_alternative(a.o, row, r, sums, bv, bi);
      pv = bv;
      pi = bi;
    }
    return;
  }
  // Many equal logits, for whose eights there was no room: a maximum over the whole row per
  // round, by all threads of the (first) CTA; a cluster's from memory.
  float pv = INFINITY;
  int pi = -1;
  for (int r = 0; r < k; ++r) {
    float bv = -INFINITY;
    int bi = 0x7fffffff;
    const auto look = [&](float y, int i) {
      if (y > -INFINITY && before(pv, pi, y, i) && before(y, i, bv, bi)) {
        bv = y;
        bi = i;
      }
    };
    if constexpr (CS > 1) {
      for (int i = t; i < C; i += G) look(to_float(x[i]), i);
    } else {
      forget();
#pragma unroll
      for (int i = 0; i < kEights; ++i) {
        float v[8];
        unpack<T>(held + i * kWords, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) look(v[j], label_of(8 * i + j));
      }
      if (xi >= 0) look(xv, xi);
    }
    warp_best(bv, bi);
    if constexpr (kWarps > 1) {
      if (lane == 0) {
        sh.best_v[warp] = bv;
        sh.best_i[warp] = bi;
      }
      sync_cta();
      bv = lane < kWarps ? sh.best_v[lane] : -INFINITY;
      bi = lane < kWarps ? sh.best_i[lane] : 0x7fffffff;
      warp_best(bv, bi);
      sync_cta();  // before the next round's are written
    }
    if (t == 0) label_alternative(a.o, row, r, sums, bv, bi);
    pv = bv;
    pi = bi;
  }
}

template <typename T, int G, int CS, int E>
cudaError_t launch(const RowsArgs& a, bool after, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  constexpr int kRows = G == 32 ? 4 : 1;
  cfg.gridDim = dim3((unsigned)(((int64_t)a.n + kRows - 1) / kRows * CS));
  cfg.blockDim = dim3(G == 32 ? 128 : G);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  int n = 0;
  if (CS > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = CS;
    at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
    ++n;
  }
  if (after) {
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.attrs = at;
  cfg.numAttrs = (unsigned)n;
  return cudaLaunchKernelEx(&cfg, k_label_rows<T, G, CS, E>, a);
}

// The fewest threads that hold a row in 32 registers each: with twice as many, half of which
// idle, 16384 rows of 4097 take 94 us and not 51, of 1500 44 and not 31 (200 rows of 4097, a
// wave at most: 4.9 and 4.7).  64 registers above 8 x 512 x 32; 8 for rows of at most a warp's worth of
// them (16384 x 120: 11 us, with 32 15).  Rows of 16 bits above 16384 pack 64 logits into 32 registers, half as many
// CTAs: 96 x 131073 20 us and 24, 300 x 60000 21 and 30, 2000 x 20000 60 and 79; where all fit at once anyway
// they wait longer for each other's sums, 1 x 131073 8.2 and 7.2.
template <typename T>
cudaError_t launch_type(const RowsArgs& a, bool after, cudaStream_t s) {
  const int vecs = a.C / (16 / (int)sizeof(T)) + 1;  // most whole vectors, with one of the ends
  const int per = 32 / (16 / (int)sizeof(T));        // vectors per thread
  if (vecs <= 32 * per / 4) return launch<T, 32, 1, 8>(a, after, s);
  if (a.C / (16 / (int)sizeof(T)) <= 32 * per) return launch<T, 32, 1, 32>(a, after, s);
  const int v = a.C / (16 / (int)sizeof(T));
  if (v <= 64 * per) return launch<T, 64, 1, 32>(a, after, s);
  if (v <= 128 * per) return launch<T, 128, 1, 32>(a, after, s);
  if (v <= 256 * per) return launch<T, 256, 1, 32>(a, after, s);
  if (v <= 512 * per) return launch<T, 512, 1, 32>(a, after, s);
  constexpr int kE = sizeof(T) == 4 ? 32 : 64;  // 16-bit logits stay packed: as many registers for twice as many
  constexpr int kPer = kE / (16 / (int)sizeof(T));  // whole vectors per thread
  if (kE > 32 && v <= 512 * kPer) return launch<T, 512, 1, kE>(a, after, s);
  if (v <= 2 * 512 * kPer) return launch<T, 512, 2, kE>(a, after, s);
  if (v <= 4 * 512 * kPer) return launch<T, 512, 4, kE>(a, after, s);
  if (v <= 8 * 512 * kPer) return launch<T, 512, 8, kE>(a, after, s);
  return launch<T, 512, 8, 64>(a, after, s);
}

}  // namespace

cudaError_t label_rows_launch(const LabelArgs& o, const void* x, int dtype, int64_t ld, int n, int C, bool after, cudaStream_t s) {
  const RowsArgs a{o, x, n > 1 ? ld : 0, n, C};
  return dtype == TSD_F32    ? launch_type<float>(a, after, s)
         : dtype == TSD_BF16 ? launch_type<__nv_bfloat16>(a, after, s)
                             : launch_type<__half>(a, after, s);
}

tsd_status label_check(const char* who, int32_t n, int32_t most_n, int32_t C, float temperature, int32_t m,
                       const int32_t* labels, int32_t k, const float* logp, const int32_t* alt_labels, const float* alt_logp) {
  if (n < 1 || n > most_n) return fail(TSD_EINVAL, "%s: n=%d outside [1, %d]", who, n, most_n);
  if (C < 1 || C > 262144) return fail(TSD_EINVAL, "%s: C=%d outside [1, 262144]", who, C);
  if (!(temperature > 0.f) || temperature > 3.4e38f || !(1.f / temperature * kLog2e <= 3.4e38f))  // the exponents' factor
    return fail(TSD_EINVAL, "%s: temperature=%g must be positive and finite, as log2(e) over it", who, (double)temperature);
  if (m < 0 || m > kMaxGiven) return fail(TSD_EINVAL, "%s: m=%d outside [0, %d]", who, m, kMaxGiven);
  if (k < 0 || k > kMaxAlt) return fail(TSD_EINVAL, "%s: k=%d outside [0, %d]", who, k, kMaxAlt);
  if (m > 0 && (!labels || !logp)) return fail(TSD_EINVAL, "%s: NULL labels or logp with m=%d", who, m);
  if (k > 0 && (!alt_labels || !alt_logp)) return fail(TSD_EINVAL, "%s: NULL alt_labels or alt_logp with k=%d", who, k);
  return TSD_OK;
}

}  // namespace tsd

using namespace tsd;

extern "C" tsd_status tsd_label_scores(int32_t n, int32_t C, const void* logits, int32_t dtype, int64_t row_stride,
                                       float temperature, int32_t m, const int32_t* labels, int32_t k, float* logp,
                                       float* entropy, int32_t* alt_labels, float* alt_logp, void* cuda_stream) {
  clear_error();
  const char* who = "tsd_label_scores";
  if (!logits) return fail(TSD_EINVAL, "%s: NULL logits", who);
  if (tsd_status st = label_check(who, n, 1 << 27, C, temperature, m, labels, k, logp, alt_labels, alt_logp)) return st;
  if (dtype != TSD_F32 && dtype != TSD_BF16 && dtype != TSD_F16) return fail(TSD_EINVAL, "%s: unknown dtype %d", who, dtype);
  if (n > 1 && row_stride < C) return fail(TSD_EINVAL, "%s: row_stride=%lld below C=%d", who, (long long)row_stride, C);
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == TSD_F32 ? 4 : 2)) return fail(TSD_EINVAL, "%s: logits not aligned to their type", who);
  const LabelArgs o{m, k, labels, logp, entropy, alt_labels, alt_logp, 1.f / temperature};
  TSD_CUDA(label_rows_launch(o, logits, dtype, row_stride, n, C, false, static_cast<cudaStream_t>(cuda_stream)));
  return TSD_OK;
}
