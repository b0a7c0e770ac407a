// The 8-bit paged cache: appending (quantisation) and reading back.
//
// A block of tokens and head has one scale, a / 127 with a the largest
// magnitude, so a block can only be rounded once all of its tokens are known.
// A filling block is therefore rounded again at each append, from unrounded
// copies of its tokens (the tail) and the new ones: what the cache holds then
// does not depend on the calls' splits, and the attention kernels read one
// format.  Two blocks of originals per slot cost 2 x block tokens of 16 bits
// per head and let a caller take tokens back into the block before the last.
#include <climits>

#include "kv8.h"
#include "kv8_keys.h"
#include "seq.h"
#include "tc_common.cuh"

namespace tsd {

namespace {

constexpr int kThreads = 128;

struct AppendArgs {
  tsd_kv8 c;
  tsd_kv8_batch b;
  const uint16_t* src[2];  // keys, values
  int64_t row[2], head[2];
};

// Eight quotients x / s rounded to nearest even, as bytes (|x / s| below 127.5, s >
// 2^-40).  r = x (1 / s) is off by less than 2^-15; adding 1.5 * 2^23 leaves its nearest
// integer in the low bits.  Only a quotient that near to a half needs more: the exact side
// is the sign of x - h s, which a fused multiply-add has right.
constexpr float kMagic = 12582912.f;
__device__ __forceinline__ float beside_half(float x, float s, float r) {
  float q = rintf(r);
  const float d = r - q;
  if (fabsf(d) > 0.5f - 0x1p-14f) {
    const float h = d > 0.f ? q + 0.5f : q - 0.5f;
    const float rem = fmaf(-h, s, x);
    q = rem > 0.f ? h + 0.5f : rem < 0.f ? h - 0.5f : rintf(h);
  }
  return q + kMagic;
}
__device__ __forceinline__ uint2 round8(const float (&x)[8], float s, float inv) {
  const uint64_t v2 = tc::pair_of(inv, inv), up = tc::pair_of(kMagic, kMagic), down = tc::pair_of(-kMagic, -kMagic);
  float m[8], far = 0.f;
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const uint64_t r = tc::mul2(tc::pair_of(x[j], x[j + 1]), v2), t = tc::add2(r, up);
    float q0, q1, r0, r1;
    tc::unpair(t, m[j], m[j + 1]);
    tc::unpair(tc::add2(t, down), q0, q1);
    tc::unpair(r, r0, r1);
    far = fmaxf(far, fmaxf(fabsf(r0 - q0), fabsf(r1 - q1)));
  }
  if (far > 0.5f - 0x1p-14f) {
#pragma unroll
    for (int j = 0; j < 8; ++j) m[j] = beside_half(x[j], s, x[j] * inv);
  }
  const auto bytes = [](float a, float b, float c, float d) {
    return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040), __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
  };
  return make_uint2(bytes(m[0], m[1], m[2], m[3]), bytes(m[4], m[5], m[6], m[7]));
}

// A touched block, head, and keys or values is one unit: 64 elements per thread
// (32 in the smallest blocks), so a unit is a warp, two or four, and CTAs of 128 threads hold 4, 2 or 1.  A
// thread holds its elements as packed 16-bit vectors: one read, the largest
// magnitude from the patterns (they order as integers without the sign, NaN
// and infinity above every number), one write.  Bound by the rounding's instructions in
// prompts (66% of issue slots; 6 ragged ones of 4000, 8 heads of 128: 26.5 us, where 2 bytes in and 1 out
// per element take 15), by its dependent loads in single tokens (256: 10 us).
template <bool BF16, int BLOCK, int DIM>
__global__ void __launch_bounds__(kThreads, 8) k_kv8_append(const __grid_constant__ AppendArgs a) {
  constexpr int T = BLOCK * DIM / 64 < 32 ? 32 : BLOCK * DIM / 64;  // threads per unit
  constexpr int kVecs = BLOCK * DIM / 8 / T;                        // 8-element vectors per thread
  constexpr int kCols = DIM / 8;
  __shared__ uint32_t s_top[kThreads / 32];
  const int u = threadIdx.x / T, t = threadIdx.x % T, unit = blockIdx.y * (kThreads / T) + u;
  const Kv8Seq q = kv8_seq(a.c, a.b, blockIdx.z);
  if (!q.ok || q.count == 0 || unit >= 2 * a.c.kv_heads) return;  // whole units
  const auto sync = [&]() {
    if constexpr (T == 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + u), "n"(T) : "memory");
  };
  const int head = unit >> 1, which = unit & 1;
  const int start = q.len - q.count;  // first new token
  const int b0 = start / BLOCK, b1 = (q.len - 1) / BLOCK;
  const uint16_t* src = (which ? a.src[1] : a.src[0]) + head * (which ? a.head[1] : a.head[0]);
  const int64_t stride = which ? a.row[1] : a.row[0];
  uint16_t* tail = static_cast<uint16_t*>(which ? a.c.v_tail : a.c.k_tail);
  const auto tail_at = [&](int b, int tok, int col) {
    return tail + ((((size_t)q.slot * 2 + (b & 1)) * a.c.kv_heads + head) * BLOCK + tok) * DIM + col * 8;
  };
  for (int b = b0 + (int)blockIdx.x; b <= b1; b += gridDim.x) {
    const int id = __ldg(a.b.table + (size_t)q.slot * a.b.table_width + b);
    uint4 x[kVecs];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int e = t + i * T, tok = e / kCols, col = e % kCols;
      const int pos = b * BLOCK + tok;
      x[i] = make_uint4(0, 0, 0, 0);
      if (pos < start) x[i] = *reinterpret_cast<const uint4*>(tail_at(b, tok, col));
      else if (pos < q.len)
        x[i] = __ldcs(reinterpret_cast<const uint4*>(src + (int64_t)(q.row0 + pos - start) * stride + col * 8));
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const uint32_t m = 0x7fff7fffu;
      top = __vmaxu2(top, __vmaxu2(__vmaxu2(x[i].x & m, x[i].y & m), __vmaxu2(x[i].z & m, x[i].w & m)));
    }
    top = __reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16));
    sync();  // the last block's use of s_top, and (first block) its reads of the tail
    if constexpr (T > 32) {
      if ((t & 31) == 0) s_top[threadIdx.x >> 5] = top;
      sync();
      const uint32_t* mine = s_top + u * (T / 32);
#pragma unroll
      for (int i = 0; i < T / 32; ++i) top = max(top, mine[i]);
    }
    const float big = wide16<BF16>(top);
    const bool fine = big <= kKv8Most;  // false for NaN and infinity
    const float s = fmaxf(big, kKv8Least) * (1.f / 127.f), inv = 1.f / s;
    if (id >= 0 && id < a.c.n_blocks) {
      int8_t* out = static_cast<int8_t*>(which ? a.c.v : a.c.k) + ((size_t)id * a.c.kv_heads + head) * BLOCK * DIM;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        if (b * BLOCK + (t + i * T) / kCols >= q.len) break;  // not yet tokens: left as they are
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        uint2 y = make_uint2(0, 0);
        if (fine) {
          float v[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[2 * j] = wide16<BF16>(w[j] & 0xffffu), v[2 * j + 1] = BF16 ? __uint_as_float(w[j] & 0xffff0000u) : wide16<BF16>(w[j] >> 16);
          y = round8(v, s, inv);
        }
        *reinterpret_cast<uint2*>(out + (size_t)(t + i * T) * 8) = y;
      }
      if (t == 0) (which ? a.c.v_scale : a.c.k_scale)[(size_t)id * a.c.kv_heads + head] = fine ? s : __uint_as_float(0x7fc00000u);
    }
    if (b == b0) {
      // originals of the new tokens in the last two blocks: written by the unit that has
      // read the old ones (all of its threads have, above), in rows that no other reads
      const int from = max(start, (b1 - 1) * BLOCK);
      for (int e = t; e < (q.len - from) * kCols; e += T) {
        const int pos = from + e / kCols, col = e % kCols;
        *reinterpret_cast<uint4*>(tail_at(pos / BLOCK, pos % BLOCK, col)) =
            __ldg(reinterpret_cast<const uint4*>(src + (int64_t)(q.row0 + pos - start) * stride + col * 8));
      }
    }
  }
}

// One warp per row: its keys or its values, all heads.  Bound by the writes (4 bytes an
// element): 134 MB of them and 34 read, 31 us.  All keys, then all values, written past the caches, with two loads
// ahead: both by one warp 33.6, without the hint 34.4, with eight loads ahead 53.
template <int DIM>
__global__ void __launch_bounds__(256) k_kv8_read(const __grid_constant__ tsd_kv8 c, const __grid_constant__ tsd_kv8_batch b,
                                                  float* k_out, float* v_out) {
  const int r = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (r >= b.rows) return;
  const int i = seq_of(b.starts, b.n, r, lane);
  if (i < 0) return;  // behind the last sequence
  const Kv8Seq q = kv8_seq(c, b, i);
  if (r < q.row0 || r >= q.row0 + q.count) return;
  int id = -1, tok = 0;
  if (q.ok) {
    const int pos = q.len - q.count + r - q.row0;
    id = __ldg(b.table + (size_t)q.slot * b.table_width + pos / c.block);
    tok = pos % c.block;
  }
  const bool have = id >= 0 && id < c.n_blocks;
  constexpr int kQuads = DIM / 4;
  const int quads = c.kv_heads * kQuads;
  const size_t out0 = (size_t)r * quads;
  const size_t head0 = (size_t)(have ? id : 0) * c.kv_heads;
  const int w = blockIdx.y;
  const int8_t* src = static_cast<const int8_t*>(w ? c.v : c.k);
  const float* sc = w ? c.v_scale : c.k_scale;
  float4* out = reinterpret_cast<float4*>(w ? v_out : k_out) + out0;
#pragma unroll 2
  for (int e = lane; e < quads; e += 32) {
    const int h = e / kQuads, col = e % kQuads;
    float4 y;
    if (have) {
      const float s = __ldg(sc + head0 + h);
      const char4 x = __ldg(reinterpret_cast<const char4*>(src + ((head0 + h) * c.block + tok) * DIM) + col);
      y = make_float4(x.x * s, x.y * s, x.z * s, x.w * s);
    } else {
      y.x = y.y = y.z = y.w = __uint_as_float(0x7fc00000u);
    }
    __stcs(out + e, y);
  }
}

template <bool BF16, int BLOCK, int DIM>
void launch_append(const AppendArgs& a, dim3 grid, cudaStream_t s) {
  constexpr int T = BLOCK * DIM / 64 < 32 ? 32 : BLOCK * DIM / 64, kUnits = kThreads / T;
  grid.y = (2 * a.c.kv_heads + kUnits - 1) / kUnits;
  k_kv8_append<BF16, BLOCK, DIM><<<grid, kThreads, 0, s>>>(a);
}

template <bool BF16, int BLOCK>
void launch_append_dim(const AppendArgs& a, dim3 grid, cudaStream_t s) {
  if (a.c.dim == 64) launch_append<BF16, BLOCK, 64>(a, grid, s);
  else launch_append<BF16, BLOCK, 128>(a, grid, s);
}

template <bool BF16>
void launch_append_type(const AppendArgs& a, dim3 grid, cudaStream_t s) {
  if (a.c.block == 16) launch_append_dim<BF16, 16>(a, grid, s);
  else if (a.c.block == 32) launch_append_dim<BF16, 32>(a, grid, s);
  else launch_append_dim<BF16, 64>(a, grid, s);
}

}  // namespace

tsd_status kv8_check(const char* who, const tsd_kv8* c, const tsd_kv8_batch* b) {
  if (!c || !b) return fail(TSD_EINVAL, "%s: NULL argument", who);
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->k_tail || !c->v_tail)
    return fail(TSD_EINVAL, "%s: NULL cache array", who);
  for (const void* p : {(const void*)c->k, (const void*)c->v, (const void*)c->k_tail, (const void*)c->v_tail})
    if (reinterpret_cast<uintptr_t>(p) % 16) return fail(TSD_EINVAL, "%s: cache arrays must be 16-byte aligned", who);
  if (c->dtype != TSD_BF16 && c->dtype != TSD_F16) return fail(TSD_EINVAL, "%s: dtype %d is not bf16 or fp16", who, c->dtype);
  if (c->block != 16 && c->block != 32 && c->block != 64) return fail(TSD_EINVAL, "%s: block=%d is not 16, 32 or 64", who, c->block);
  if (c->dim != 64 && c->dim != 128) return fail(TSD_EINVAL, "%s: dim=%d is not 64 or 128", who, c->dim);
  if (c->kv_heads < 1 || c->kv_heads > 1024) return fail(TSD_EINVAL, "%s: kv_heads=%d outside [1, 1024]", who, c->kv_heads);
  if (c->n_blocks < 1 || c->n_slots < 1) return fail(TSD_EINVAL, "%s: n_blocks=%d and n_slots=%d must be positive", who, c->n_blocks, c->n_slots);
  if ((int64_t)c->n_blocks * c->kv_heads * c->block > UINT32_MAX - 64)
    return fail(TSD_EINVAL, "%s: n_blocks=%d x kv_heads=%d x block=%d above 2^32 rows", who, c->n_blocks, c->kv_heads, c->block);
  if (!b->lens || !b->table) return fail(TSD_EINVAL, "%s: NULL lens or table", who);
  if (b->n < 1 || b->n > 65535) return fail(TSD_EINVAL, "%s: n=%d outside [1, 65535]", who, b->n);
  if (b->table_width < 1 || (int64_t)b->table_width * c->block > INT32_MAX - 64)
    return fail(TSD_EINVAL, "%s: table_width=%d x block %d outside [1, 2^31 - 65] tokens", who, b->table_width, c->block);
  if (b->rows < 1 || b->rows > (1 << 22)) return fail(TSD_EINVAL, "%s: rows=%d outside [1, 2^22]", who, b->rows);
  if (!b->starts && b->rows != b->n) return fail(TSD_EINVAL, "%s: starts is NULL: rows=%d must be n=%d", who, b->rows, b->n);
  if (b->max_new < 0 || b->max_len < 0) return fail(TSD_EINVAL, "%s: negative max_new or max_len", who);
  return TSD_OK;
}

tsd_status kv8_check_rows(const char* who, const char* what, const void* p, int64_t row, int64_t head) {
  if (!p) return fail(TSD_EINVAL, "%s: NULL %s", who, what);
  if (reinterpret_cast<uintptr_t>(p) % 16 || row % 8 || head % 8)
    return fail(TSD_EINVAL, "%s: %s must be 16-byte aligned with strides a multiple of 8 elements", who, what);
  if (row < 0 || head < 0 || row > (1ll << 40) || head > (1ll << 40))
    return fail(TSD_EINVAL, "%s: %s strides out of range", who, what);
  return TSD_OK;
}

}  // namespace tsd

using namespace tsd;

extern "C" tsd_status tsd_kv8_append(const tsd_kv8* cache, const tsd_kv8_batch* batch, const void* k, int64_t k_row,
                                     int64_t k_head, const void* v, int64_t v_row, int64_t v_head, void* cuda_stream) {
  clear_error();
  if (tsd_status st = kv8_check("tsd_kv8_append", cache, batch)) return st;
  if (tsd_status st = kv8_check_rows("tsd_kv8_append", "k", k, k_row, k_head)) return st;
  if (tsd_status st = kv8_check_rows("tsd_kv8_append", "v", v, v_row, v_head)) return st;
  AppendArgs a{*cache, *batch, {static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v)}, {k_row, v_row}, {k_head, v_head}};
  const int64_t blocks = append_blocks(batch->n, batch->rows, batch->starts != nullptr, batch->max_new, cache->block);
  const dim3 grid((unsigned)blocks, 1, batch->n);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (cache->dtype == TSD_BF16) launch_append_type<true>(a, grid, s);
  else launch_append_type<false>(a, grid, s);
  TSD_CUDA(cudaGetLastError());
  return TSD_OK;
}

extern "C" tsd_status tsd_kv8_read(const tsd_kv8* cache, const tsd_kv8_batch* batch, float* k_out, float* v_out, void* cuda_stream) {
  clear_error();
  if (tsd_status st = kv8_check("tsd_kv8_read", cache, batch)) return st;
  if (!k_out || !v_out) return fail(TSD_EINVAL, "tsd_kv8_read: NULL output");
  if (reinterpret_cast<uintptr_t>(k_out) % 16 || reinterpret_cast<uintptr_t>(v_out) % 16)
    return fail(TSD_EINVAL, "tsd_kv8_read: outputs must be 16-byte aligned");
  const unsigned grid = (unsigned)((batch->rows + 7) / 8);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (cache->dim == 64) k_kv8_read<64><<<dim3(grid, 2), 256, 0, s>>>(*cache, *batch, k_out, v_out);
  else k_kv8_read<128><<<dim3(grid, 2), 256, 0, s>>>(*cache, *batch, k_out, v_out);
  TSD_CUDA(cudaGetLastError());
  return TSD_OK;
}
