// Scores of labels from logits in memory (tsd.h: tsd_label_scores): log
// probabilities of given labels, entropy, top alternatives, in one pass over
// the logits.
//
// Mathematics, per row with m the largest logit, c = log2(e) / T, d_i = (x_i - m) c:
//   S = sum 2^d_i,  E = sum 2^d_i d_i,
//   log p(l) = (x_l - m) / T - ln S,   entropy = ln S - ln 2 E / S.
// x_i - m is formed first (exact or rounded once), so a row's offset costs no
// precision.  A row stays in registers (32 or 64 logits per thread): 32 to 512 threads
// per row, above 16384 logits a cluster of 2 to 8 CTAs of 512 that exchange
// through distributed shared memory.  The k largest: the threads form groups (8 to 128 of
// them); the k-th largest of the groups' maxima is a bound that at least
// k logits reach and few pass, so only those few are gathered and ordered.  If more
// than the gathering holds reach it (many equal logits), k rounds of a maximum over
// the whole row take its place.
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

constexpr int kCap = 256;       // logits gathered per row (and CTA)
constexpr int kGroupsMax = 16;  // groups per CTA

// What the CTAs of a row's cluster show one another.
struct RowShared {
  float top[kGroupsMax];  // groups' maxima
  float2 sums[16];        // warps' S and E
  float cv[kCap];         // gathered logits and their labels
  int ci[kCap];
  int count;
  float best_v[16];  // warps' best of a round over the whole row
  int best_i[16];
  float pick_v;
  int pick_i;
};

template <typename T>
__device__ __forceinline__ float to_float(T v) {
  return (float)v;
}

// eight (16-bit) or four (fp32) consecutive logits
template <typename T>
__device__ __forceinline__ void unpack(uint4 w, float* v) {
  if constexpr (sizeof(T) == 4) {
    v[0] = __uint_as_float(w.x), v[1] = __uint_as_float(w.y), v[2] = __uint_as_float(w.z), v[3] = __uint_as_float(w.w);
  } else {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
      }
    }
  }
}

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
__global__ void __launch_bounds__(G == 32 ? 128 : G) k_label_rows(const __grid_constant__ RowsArgs a) {
  constexpr int VE = 16 / sizeof(T), NV = E / VE;
  constexpr int kWarps = G / 32;
  constexpr int kPerWarp = kWarps >= 16 ? 1 : (16 / kWarps < 8 ? 16 / kWarps : 8);  // groups in a warp
  constexpr int kGroups = kPerWarp * kWarps;
  constexpr int kRows = G == 32 ? 4 : 1;
  constexpr int kKeys = (kGroups * CS + 31) / 32;  // groups' maxima per lane
  __shared__ RowShared s_rows[kRows];
  const int warp_in_cta = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int slot = G == 32 ? warp_in_cta : 0, warp = G == 32 ? 0 : warp_in_cta;
  const int64_t row = (int64_t)(blockIdx.x / CS) * kRows + slot;
  if (row >= a.n) return;  // a whole warp (G 32) or none: the grid has n CTAs or clusters
  const int rank = CS > 1 ? (int)(blockIdx.x % CS) : 0;
  RowShared& sh = s_rows[slot];
  const auto peer = [&](int r) -> RowShared* {
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
  const int t = warp * 32 + lane, rt = rank * G + t;
  const T* x = static_cast<const T*>(a.x) + row * a.ld;
  const int C = a.C, k = a.o.k;

  // the logits: whole aligned vectors, and the ends one by one
  const int lead = min(C, (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(T));
  const int nvec = (C - lead) / VE, tail = C - lead - nvec * VE;
  float v[E];
  {
    uint4 w[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = rt + i * G * CS;
      if (j < nvec) w[i] = __ldcs(reinterpret_cast<const uint4*>(x + lead) + j);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      unpack<T>(w[i], v + i * VE);
      if (rt + i * G * CS >= nvec) {
#pragma unroll
        for (int j = 0; j < VE; ++j) v[i * VE + j] = -INFINITY;
      }
    }
  }
  const int xi = rt < lead ? rt : rt < lead + tail ? nvec * VE + rt : -1;
  const float xv = xi >= 0 ? to_float(x[xi]) : -INFINITY;
  const auto label_of = [&](int e) { return lead + (rt + e / VE * G * CS) * VE + e % VE; };

  // the groups' maxima, the row's, and the bound of the k largest
  float mine = xv;
#pragma unroll
  for (int e = 0; e < E; ++e) mine = fmaxf(mine, v[e]);
  float gm = mine;
#pragma unroll
  for (int o = 1; o < 32 / kPerWarp; o <<= 1) gm = fmaxf(gm, __shfl_xor_sync(0xffffffffu, gm, o));
  if (lane % (32 / kPerWarp) == 0) sh.top[warp * kPerWarp + lane / (32 / kPerWarp)] = gm;
  if (t == 0) sh.count = 0;
  sync_row();
  int keys[kKeys];
#pragma unroll
  for (int i = 0; i < kKeys; ++i) {
    const int j = lane + 32 * i;
    keys[i] = j < kGroups * CS ? order_of(peer(j / kGroups)->top[j % kGroups]) : INT32_MIN;
  }
  float m = 0.f, bound = 0.f;
  for (int r = 0; r < max(k, 1); ++r) {
    int best = keys[0];
#pragma unroll
    for (int i = 1; i < kKeys; ++i) best = max(best, keys[i]);
    const int top = __reduce_max_sync(0xffffffffu, best);
    bound = value_of(top);
    if (r == 0) m = bound;
    // one holder gives it up
    const bool holder = lane == __ffs(__ballot_sync(0xffffffffu, best == top)) - 1;
    bool open = holder;
#pragma unroll
    for (int i = 0; i < kKeys; ++i)
      if (open && keys[i] == top) {
        keys[i] = INT32_MIN;
        open = false;
      }
    if (top == INT32_MIN) break;
  }
  if (!(bound >= -INFINITY)) bound = -INFINITY;  // fewer groups than k

  // sums: in pairs, a masked logit's exponent held finite (its term is 0 all the same)
  const float ms = m == -INFINITY ? 0.f : m, c = a.o.inv_temp * kLog2e;
  uint64_t s2 = 0, e2 = 0;
  const uint64_t nm = pair_of(-ms, -ms), cc = pair_of(c, c);
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    const uint64_t d = mul2(add2(pair_of(v[e], v[e + 1]), nm), cc);
    float d0, d1;
    unpair(d, d0, d1);
    d0 = max_nan(d0, -1e30f);
    d1 = max_nan(d1, -1e30f);
    const uint64_t p = pair_of(ex2_approx(d0), ex2_approx(d1));
    s2 = add2(s2, p);
    e2 = fma2(p, pair_of(d0, d1), e2);
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
  if (lane == 0) sh.sums[warp] = make_float2(S, E2);

  // gather what reaches the bound
  if (k > 0 && mine >= bound && mine > -INFINITY) {
    const auto take = [&](float y, int label) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < kCap) {
        sh.cv[at] = y;
        sh.ci[at] = label;
      }
    };
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (v[e] >= bound && v[e] > -INFINITY) take(v[e], label_of(e));
    if (xv >= bound && xv > -INFINITY) take(xv, xi);
  }
  sync_row();

  S = E2 = 0.f;
  bool over = false;
  for (int r = 0; r < CS; ++r) {
    const RowShared* p = peer(r);
    const float2 y = lane < kWarps ? p->sums[lane] : make_float2(0.f, 0.f);
    S += y.x;
    E2 += y.y;
    over = over || p->count > kCap;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    S += __shfl_xor_sync(0xffffffffu, S, o);
    E2 += __shfl_xor_sync(0xffffffffu, E2, o);
  }
  const RowSums sums{m, S, E2};
  if (rank == 0 && warp == 0) {
    label_finish(a.o, row, sums, lane, [&](int l) { return l < C ? to_float(x[l]) : __uint_as_float(0x7fc00000u); });
  }

  // the k best in order
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
    if (!over) {
      if (rank != 0 || warp != 0) break;
      for (int q = 0; q < CS; ++q) {
        const RowShared* p = peer(q);
        for (int i = lane; i < p->count; i += 32) look(p->cv[i], p->ci[i]);
      }
      warp_best(bv, bi);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) look(v[e], label_of(e));
      if (xi >= 0) look(xv, xi);
      warp_best(bv, bi);
      if (lane == 0) {
        sh.best_v[warp] = bv;
        sh.best_i[warp] = bi;
      }
      sync_row();
      bv = -INFINITY;
      bi = 0x7fffffff;
      for (int q = 0; q < CS; ++q) {
        const RowShared* p = peer(q);
        const float y = lane < kWarps ? p->best_v[lane] : -INFINITY;
        const int i = lane < kWarps ? p->best_i[lane] : 0x7fffffff;
        if (before(y, i, bv, bi)) {
          bv = y;
          bi = i;
        }
      }
      warp_best(bv, bi);
      sync_row();  // before the next round's are written
    }
    if (rank == 0 && warp == 0 && lane == 0) label_alternative(a.o, row, r, sums, bv, bi);
    pv = bv;
    pi = bi;
  }
  if constexpr (CS > 1) cg::this_cluster().sync();  // no CTA leaves while its memory is read
}

template <typename T, int G, int CS, int E>
cudaError_t launch(const RowsArgs& a, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  constexpr int kRows = G == 32 ? 4 : 1;
  cfg.gridDim = dim3((unsigned)(((int64_t)a.n + kRows - 1) / kRows * CS));
  cfg.blockDim = dim3(G == 32 ? 128 : G);
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = CS;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = CS > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, k_label_rows<T, G, CS, E>, a);
}

// The fewest threads that hold a row in 32 registers each (64 above 8 x 512 x 32; 8 for
// rows of a few vectors, where 32 would be mostly empty).
template <typename T>
cudaError_t launch_type(const RowsArgs& a, cudaStream_t s) {
  const int vecs = a.C / (16 / (int)sizeof(T)) + 1;  // most whole vectors, with one of the ends
  const int per = 32 / (16 / (int)sizeof(T));        // vectors per thread
  if (vecs <= 32 * per / 4) return launch<T, 32, 1, 8>(a, s);
  if (a.C / (16 / (int)sizeof(T)) <= 32 * per) return launch<T, 32, 1, 32>(a, s);
  const int v = a.C / (16 / (int)sizeof(T));
  if (v <= 64 * per) return launch<T, 64, 1, 32>(a, s);
  if (v <= 128 * per) return launch<T, 128, 1, 32>(a, s);
  if (v <= 256 * per) return launch<T, 256, 1, 32>(a, s);
  if (v <= 512 * per) return launch<T, 512, 1, 32>(a, s);
  if (v <= 1024 * per) return launch<T, 512, 2, 32>(a, s);
  if (v <= 2048 * per) return launch<T, 512, 4, 32>(a, s);
  if (v <= 4096 * per) return launch<T, 512, 8, 32>(a, s);
  return launch<T, 512, 8, 64>(a, s);
}

}  // namespace

tsd_status label_check(const char* who, int32_t n, int32_t most_n, int32_t C, float temperature, int32_t m,
                       const int32_t* labels, int32_t k, const float* logp, const int32_t* alt_labels, const float* alt_logp) {
  if (n < 1 || n > most_n) return fail(TSD_EINVAL, "%s: n=%d outside [1, %d]", who, n, most_n);
  if (C < 1 || C > 262144) return fail(TSD_EINVAL, "%s: C=%d outside [1, 262144]", who, C);
  if (!(temperature > 0.f) || temperature > 3.4e38f || !(1.f / temperature <= 3.4e38f))
    return fail(TSD_EINVAL, "%s: temperature=%g must be positive and finite, as its reciprocal", who, (double)temperature);
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
  if (tsd_status st = label_check(who, n, 1 << 28, C, temperature, m, labels, k, logp, alt_labels, alt_logp)) return st;
  if (dtype != TSD_F32 && dtype != TSD_BF16 && dtype != TSD_F16) return fail(TSD_EINVAL, "%s: unknown dtype %d", who, dtype);
  if (n > 1 && row_stride < C) return fail(TSD_EINVAL, "%s: row_stride=%lld below C=%d", who, (long long)row_stride, C);
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == TSD_F32 ? 4 : 2)) return fail(TSD_EINVAL, "%s: logits not aligned to their type", who);
  RowsArgs a{{m, k, labels, logp, entropy, alt_labels, alt_logp, 1.f / temperature}, logits, n > 1 ? row_stride : 0, n, C};
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  TSD_CUDA(dtype == TSD_F32 ? launch_type<float>(a, s) : dtype == TSD_BF16 ? launch_type<__nv_bfloat16>(a, s) : launch_type<__half>(a, s));
  return TSD_OK;
}
