// Device code that the paged cache's gfx950 kernels share: number formats, where a
// row's token lies, storing a row, and what the attention kernels have in common.
#pragma once
#include <hip/hip_runtime.h>

#include "ss_cache.h"

#include <math.h>

namespace ss {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x2_t __attribute__((ext_vector_type(2)));

constexpr float kNegInf = -__builtin_huge_valf();
constexpr int kBufferFlags = 0x00020000;   // buffer resource word 3: 32-bit data format, raw offsets
constexpr int kStreamLoad = 2;             // non-temporal: the cache is read once per call
constexpr int kThreads = 256;
constexpr int kWaves = 4;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Max / sum across the GROUPS (4 or 2) equal groups of lanes of a wave.
template <int GROUPS>
__device__ __forceinline__ float xgroup_max(float x) {
  if constexpr (GROUPS == 4) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <int GROUPS>
__device__ __forceinline__ float xgroup_sum(float x) {
  if constexpr (GROUPS == 4) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ s16x4_t lds_read_tr16(uint32_t at) {   // an LDS address
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(uintptr_t)at);
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// By value: __builtin_bit_cast of a vector's element takes its first one.
__device__ __forceinline__ bf16x2_t as_bf16x2(uint32_t w) { return __builtin_bit_cast(bf16x2_t, w); }

// The four (e4m3) or eight (e2m1) values of a dword, times scale, as bf16.
__device__ __forceinline__ u32x2_t widen8(uint32_t w, float scale) {
  return {__builtin_bit_cast(uint32_t, (bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
          __builtin_bit_cast(uint32_t, (bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))};
}
__device__ __forceinline__ u32x4_t widen4(uint32_t w, float scale) {
  return {__builtin_bit_cast(uint32_t, (bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
          __builtin_bit_cast(uint32_t, (bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
          __builtin_bit_cast(uint32_t, (bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
          __builtin_bit_cast(uint32_t, (bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}

constexpr int kGroupRows = 16;

// Where row t lives: its page block of KV head 0 and its slot there.
struct Place {
  uint8_t *page;   // null: nowhere
  int slot;
  bool row;        // whether t is a row of some request
  int64_t pos;     // its token's position (of a row)
};

// starts, ends: LDS, B + 1 and B words (none without row_start).
__device__ __forceinline__ Place place_of(const CacheArgs &p, int64_t t, int tx, int32_t *starts, int32_t *ends) {
  int b, e;
  int64_t i, n;
  if (p.row_start == nullptr) {
    if (t >= p.num_rows) return {nullptr, 0, false, 0};
    b = (int)((uint32_t)t / (uint32_t)p.max_rows);
    i = t - (int64_t)b * p.max_rows;
    n = p.max_rows;
    e = p.end[b];
  } else {
    for (int j = tx; j <= p.B; j += kThreads) {
      starts[j] = p.row_start[j];
      if (j < p.B) ends[j] = p.end[j];
    }
    __syncthreads();
    // the last request that starts at or before t: an empty one's start is
    // also the next one's, so it is never the last
    int lo = 0, hi = p.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (starts[mid] <= t)
        lo = mid;
      else
        hi = mid;
    }
    b = lo;
    i = t - starts[b];
    n = (int64_t)starts[b + 1] - starts[b];
    if (t >= p.num_rows || i < 0 || i >= n) return {nullptr, 0, false, 0};
    e = ends[b];
  }
  const int64_t pos = e - n + i;
  if (pos < 0 || pos >= p.capacity) return {nullptr, 0, true, pos};
  const int page = p.table[(int64_t)b * p.table_stride + (pos >> p.page_shift)];
  if (page < 0 || page >= p.num_pages) return {nullptr, 0, true, pos};
  return {p.pages + (uint64_t)page * p.page_stride, (int)(pos & ((1 << p.page_shift) - 1)), true, pos};
}

__device__ __forceinline__ uint32_t pack_max(uint32_t a, uint32_t b) {   // of two halves below 2^15 each
  const uint32_t hi = (a & 0xffff0000u) > (b & 0xffff0000u) ? a & 0xffff0000u : b & 0xffff0000u;
  const uint32_t lo = (a & 0xffffu) > (b & 0xffffu) ? a & 0xffffu : b & 0xffffu;
  return hi | lo;
}

// Store a lane's 8 channels x (lane c of the row's 16) into row `slot` of the
// rows at `rows` and the block's scale at `scales`.
template <int FMT>
__device__ __forceinline__ void store_row(uint8_t *rows, uint8_t *scales, int slot, int c, u32x4_t x) {
  if constexpr (FMT == kCacheBf16) {
    *reinterpret_cast<u32x4_t *>(rows + slot * 256 + 16 * c) = x;
  } else {
    // largest magnitude of the block, as bf16 bits, over the lane and its quad
    uint32_t m = pack_max(pack_max(x[0] & 0x7fff7fffu, x[1] & 0x7fff7fffu), pack_max(x[2] & 0x7fff7fffu, x[3] & 0x7fff7fffu));
    m = (m >> 16) > (m & 0xffffu) ? m >> 16 : m & 0xffffu;
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, false);   // quad_perm [1,0,3,2]
    m = o > m ? o : m;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, false);            // quad_perm [2,3,0,1]
    m = o > m ? o : m;
    // the smallest e with m <= F 2^e: F = 448 = 1.75 x 2^8 or 6 = 1.5 x 2^2.
    // Adding what carries a fraction above F's into the exponent rounds up.
    // Below 2^-111 a code's value would leave bf16's normal numbers.
    constexpr uint32_t kCarry = FMT == kCacheMx8 ? 0x1f : 0x3f;
    constexpr int kTop = FMT == kCacheMx8 ? 8 : 2;
    const bool finite = m < 0x7f80u;
    int e = (int)((m + kCarry) >> 7) - kTop;
    e = e < 16 ? 16 : e;
    const float scale = scale_of((uint32_t)e);
    // round to nearest even, exact otherwise: a power of two divides.  bf16's
    // largest numbers round up to 2^128 (header)
    if constexpr (FMT == kCacheMx8) {
      u32x2_t code;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        s16x2_t w = {0, 0};
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, as_bf16x2(x[2 * j]), scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, as_bf16x2(x[2 * j + 1]), scale, true);
        code[j] = finite ? __builtin_bit_cast(uint32_t, w) : 0u;
      }
      *reinterpret_cast<u32x2_t *>(rows + slot * 128 + 8 * c) = code;
    } else {
      uint32_t code = 0;
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_bf16x2(x[0]), scale, 0);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_bf16x2(x[1]), scale, 1);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_bf16x2(x[2]), scale, 2);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_bf16x2(x[3]), scale, 3);
      *reinterpret_cast<uint32_t *>(rows + slot * 64 + 4 * c) = finite ? code : 0u;
    }
    // the row's four scale bytes as one word
    uint32_t word = (finite ? (uint32_t)e : 255u) << (8 * (c >> 2));
    word |= (uint32_t)__builtin_amdgcn_mov_dpp((int)word, 0x124, 0xf, 0xf, false);    // row_ror:4
    word |= (uint32_t)__builtin_amdgcn_mov_dpp((int)word, 0x128, 0xf, 0xf, false);    // row_ror:8
    if (c == 0) *reinterpret_cast<uint32_t *>(scales + 4 * slot) = word;
  }
}

}  // namespace
}  // namespace ss
