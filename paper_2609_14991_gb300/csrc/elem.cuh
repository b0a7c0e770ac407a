// Element types of the operators on device memory: 16-bit floats and fp32, by the
// library's numbers (tsd.h: TSD_F32, TSD_BF16, TSD_F16).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "tsd.h"

namespace tsd {

// 16-bit float pattern (bf16 or fp16) to fp32
template <bool BF16>
__device__ __forceinline__ float wide16(uint32_t u) {
  if (BF16) return __uint_as_float(u << 16);
  return __half2float(__ushort_as_half((unsigned short)u));
}

// Two fp32 values rounded to a pair of 16-bit floats.
template <bool BF16>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
  if (BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <int DT>
struct Elem {  // 16-bit floats
  using Raw = uint16_t;
  static constexpr bool kBf16 = DT == TSD_BF16;
  static __device__ __forceinline__ float wide(Raw x) { return wide16<kBf16>(x); }
  static __device__ __forceinline__ Raw narrow(float x) { return (Raw)narrow2<kBf16>(x, 0.f); }
  // two elements as they lie in a 32-bit word
  static __device__ __forceinline__ float2 wide_pair(uint32_t w) { return make_float2(wide16<kBf16>(w & 0xffffu), wide16<kBf16>(w >> 16)); }
  // the eight of four words
  static __device__ __forceinline__ void wide4(const uint32_t (&w)[4], float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = wide_pair(w[i]);
      x[2 * i] = v.x, x[2 * i + 1] = v.y;
    }
  }
  static __device__ __forceinline__ void narrow4(const float (&x)[8], uint32_t (&w)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = narrow2<kBf16>(x[2 * i], x[2 * i + 1]);
  }
};
template <>
struct Elem<TSD_F32> {
  using Raw = float;
  static __device__ __forceinline__ float wide(Raw x) { return x; }
  static __device__ __forceinline__ Raw narrow(float x) { return x; }
  static __device__ __forceinline__ void wide4(const uint32_t (&w)[4], float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
  }
  static __device__ __forceinline__ void narrow4(const float (&x)[4], uint32_t (&w)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
  }
};

// Eight adjacent elements, 16-byte aligned, as they came from memory.
template <int DT>
struct Eight {
  static constexpr int kWords = DT == TSD_F32 ? 8 : 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const typename Elem<DT>::Raw* p) {
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) {
      const uint4 v = reinterpret_cast<const uint4*>(p)[i];
      w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
    }
  }
  __device__ __forceinline__ void store(typename Elem<DT>::Raw* p) const {
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
  // at a 32-byte boundary where there are 32 bytes: whole sectors at once
  __device__ __forceinline__ void store_even(typename Elem<DT>::Raw* p) const {
    if constexpr (DT == TSD_F32)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
                   "r"(w[6]), "r"(w[7])
                   : "memory");
    else
      store(p);
  }
  __device__ __forceinline__ void get(float* x) const {
    if constexpr (DT == TSD_F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 v = Elem<DT>::wide_pair(w[i]);
        x[2 * i] = v.x, x[2 * i + 1] = v.y;
      }
    }
  }
  __device__ __forceinline__ void put(const float* x) {
    if constexpr (DT == TSD_F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = narrow2<Elem<DT>::kBf16>(x[2 * i], x[2 * i + 1]);
    }
  }
};

}  // namespace tsd
