// Scores of labels: what its two operators (scores.cu, joint_scores.cu) share.
#pragma once

#include "internal.h"

namespace tsd {

constexpr int kMaxGiven = 8;  // given labels per row
constexpr int kMaxAlt = 8;    // alternatives per row

struct LabelArgs {
  int m, k;
  const int32_t* labels;
  float *logp, *entropy;
  int32_t* alt_labels;
  float* alt_logp;
  float inv_temp;
};

// A row's sums: m its largest logit, S = sum 2^d, E = sum 2^d d with d =
// (x - m) log2(e) / T (m = 0 in the exponents of a row without finite logits).
struct RowSums {
  float m, S, E;
};

// max that keeps NaN
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// The exponent of a running sum whose maximum grows from m to `to`.  Held finite: the
// weight 2^d of a far lower maximum (labels masked by the type's lowest value) is 0, and E's
// share, d S times it, is not to be infinity times 0.
__device__ __forceinline__ float growth(float m, float to, float c) { return m == -INFINITY ? 0.f : max_nan((m - to) * c, -1e30f); }

// What a row's scores are made of.
struct RowScore {
  float m, ln_s, entropy;
  bool odd;  // NaN or +inf among the logits: the sums are NaN, as inf - inf is
  __device__ __forceinline__ explicit RowScore(const RowSums& r) {
    m = r.m;
    ln_s = logf(r.S);
    odd = !(r.S >= 0.f) || r.m == INFINITY;
    entropy = odd ? __uint_as_float(0x7fc00000u) : m == -INFINITY ? 0.f : fmaxf(0.f, ln_s - 0.693147180559945f * (r.E / r.S));
  }
  // y - lse of a logit of the row
  __device__ __forceinline__ float logp(float inv_temp, float x) const {
    if (odd) return __uint_as_float(0x7fc00000u);
    if (m == -INFINITY) return x == -INFINITY ? x : __uint_as_float(0x7fc00000u);
    return (x - m) * inv_temp - ln_s;
  }
};

// The score of given label l with logit x (NaN outside the row).
__device__ __forceinline__ float label_given(const LabelArgs& a, const RowScore& r, int l, float x) {
  return l == -1 ? 0.f : l >= 0 ? r.logp(a.inv_temp, x) : __uint_as_float(0x7fc00000u);
}

// Alternative j: the logit and label found (-inf: none).
__device__ __forceinline__ void label_alternative(const LabelArgs& a, int64_t row, int j, const RowScore& r, float x, int label) {
  const bool none = r.odd || !(x > -INFINITY);
  a.alt_labels[row * a.k + j] = none ? -1 : label;
  a.alt_logp[row * a.k + j] = r.odd ? __uint_as_float(0x7fc00000u) : none ? -INFINITY : r.logp(a.inv_temp, x);
}

// The scores of n rows of logits in memory (scores.cu), ld elements apart; after: once
// the kernel before it in the stream, launched to allow that, is done.
cudaError_t label_rows_launch(const LabelArgs& o, const void* x, int dtype, int64_t ld, int n, int C, bool after, cudaStream_t s);

tsd_status label_check(const char* who, int32_t n, int32_t most_n, int32_t C, float temperature, int32_t m,
                       const int32_t* labels, int32_t k, const float* logp, const int32_t* alt_labels, const float* alt_logp);

}  // namespace tsd
