// gfx950 (MI355X) kernels of the paged cache: tokens written into pages as
// bf16 or in 8 or 4 bits with a power-of-two scale per 32 channels, read back
// as bf16, and attended in place.
//
// Numbers.  A scaled block stands for code * 2^(byte - 127), code an OCP e4m3
// or e2m1 number: v_cvt_scalef32 converts two of them with their scale in one
// instruction, and every value of a finite block is a normal bf16 number, so
// nothing is lost between the cache and the matrix instructions.  A scale byte
// of 255 makes the conversion give NaN.
//
// Rows.  Request b's row i of n_b stands for position end_b - n_b + i.  What a
// table, an end or a row start could make unsafe is checked here: a page number
// outside [0, num_pages) is a page without tokens, a position outside the table
// is no token, a row outside [0, num_rows) is no row.
#include <hip/hip_runtime.h>

#include "ss_cache.h"

#include <math.h>

namespace ss {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
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

// Max / sum across the four 16-lane groups of a wave (lanes l, l^16, l^32, l^48).
__device__ __forceinline__ float xgroup_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float xgroup_sum(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ s16x4_t lds_read_tr16(const unsigned char *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4_t *)(reinterpret_cast<uintptr_t>(p)));
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

// Rows of request b for the attention: more than max_rows, or fewer than none, count as none.
__device__ __forceinline__ int rows_of(const CacheArgs &p, int b) {
  if (p.row_start == nullptr) return p.max_rows;
  const int n = p.row_start[b + 1] - p.row_start[b];
  return n < 0 || n > p.max_rows ? 0 : n;
}

// ---------------------------------------------------------------------------
// Writing and reading rows.  A workgroup takes 16 rows and HEADS KV heads, 16
// lanes to a row's 128 channels: a lane holds 8 channels, four lanes a scaled
// block.  Both directions are bound by memory; the rows' loads go out before
// their places in the cache are looked up, which takes two round trips (starts
// and ends, then the table).  Few rows take one head per workgroup, so that
// the chip fills: see launch_rows.
// ---------------------------------------------------------------------------
constexpr int kGroupRows = 16;

// Where row t lives: its page block of KV head 0 and its slot there.
struct Place {
  uint8_t *page;   // null: nowhere
  int slot;
  bool row;        // whether t is a row of some request
};

// starts, ends: LDS, kCacheMaxRequests + 1 and kCacheMaxRequests words.
__device__ __forceinline__ Place place_of(const CacheArgs &p, int t, int tx, int32_t *starts, int32_t *ends) {
  int b, i, n, e;
  if (p.row_start == nullptr) {
    b = t / p.max_rows;
    i = t - b * p.max_rows;
    n = p.max_rows;
    if (t >= p.num_rows) return {nullptr, 0, false};
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
    n = starts[b + 1] - starts[b];
    if (t >= p.num_rows || i < 0 || i >= n) return {nullptr, 0, false};
    e = ends[b];
  }
  const int64_t pos = (int64_t)e - n + i;
  if (pos < 0 || pos >= p.capacity) return {nullptr, 0, true};
  const int page = p.table[(int64_t)b * p.table_stride + (pos >> p.page_shift)];
  if (page < 0 || page >= p.num_pages) return {nullptr, 0, true};
  return {p.pages + (uint64_t)page * p.page_stride, (int)(pos & ((1 << p.page_shift) - 1)), true};
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
    // round to nearest even, exact otherwise: a power of two divides
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

template <int FMT, int HEADS>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(CacheRowsArgs p) {
  __shared__ int32_t starts[kCacheMaxRequests + 1], ends[kCacheMaxRequests];
  const int tx = threadIdx.x, c = tx & 15;
  const int64_t t = (int64_t)blockIdx.x * kGroupRows + (tx >> 4);
  const int h0 = blockIdx.y * HEADS;
  u32x4_t kx[HEADS], vx[HEADS];
  const int64_t tl = t < p.num_rows ? t : p.num_rows - 1;
#pragma unroll
  for (int j = 0; j < HEADS; ++j) {
    const int h = h0 + j < p.Hkv ? h0 + j : p.Hkv - 1;
    const int64_t at = tl * p.row_stride + h * p.head_stride + 8 * c;
    kx[j] = *reinterpret_cast<const u32x4_t *>(p.k + at);
    vx[j] = *reinterpret_cast<const u32x4_t *>(p.v + at);
  }
  const Place pl = place_of(p, (int)t, tx, starts, ends);
  if (pl.page == nullptr) return;
  constexpr int kRow = cache_row_bytes(FMT);
  const int tokens = 1 << p.page_shift;
#pragma unroll
  for (int j = 0; j < HEADS; ++j) {
    if (h0 + j >= p.Hkv) break;
    uint8_t *block = pl.page + (uint64_t)(h0 + j) * p.head_bytes;
    uint8_t *scales = block + 2 * tokens * kRow;
    store_row<FMT>(block, scales, pl.slot, c, kx[j]);
    store_row<FMT>(block + tokens * kRow, scales + 4 * tokens, pl.slot, c, vx[j]);
  }
}

template <int FMT, int HEADS>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CacheRowsArgs p) {
  __shared__ int32_t starts[kCacheMaxRequests + 1], ends[kCacheMaxRequests];
  const int tx = threadIdx.x, c = tx & 15;
  const int64_t t = (int64_t)blockIdx.x * kGroupRows + (tx >> 4);
  const int h0 = blockIdx.y * HEADS;
  const Place pl = place_of(p, (int)t, tx, starts, ends);
  if (!pl.row) return;
  constexpr int kRow = cache_row_bytes(FMT);
  const int tokens = 1 << p.page_shift;
  u32x4_t x[HEADS][2];
#pragma unroll
  for (int j = 0; j < HEADS; ++j) x[j][0] = x[j][1] = u32x4_t{0u, 0u, 0u, 0u};   // a token outside the cache reads zero
  if (pl.page != nullptr) {
    u32x4_t w[HEADS][2];
    uint32_t sc[HEADS][2];
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
      const int h = h0 + j < p.Hkv ? h0 + j : p.Hkv - 1;
      const uint8_t *block = pl.page + (uint64_t)h * p.head_bytes;
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const uint8_t *row = block + a * tokens * kRow + pl.slot * kRow;
        if constexpr (FMT == kCacheBf16) w[j][a] = *reinterpret_cast<const u32x4_t *>(row + 16 * c);
        if constexpr (FMT == kCacheMx8) {
          const u32x2_t r = *reinterpret_cast<const u32x2_t *>(row + 8 * c);
          w[j][a][0] = r[0];
          w[j][a][1] = r[1];
        }
        if constexpr (FMT == kCacheMx4) w[j][a][0] = *reinterpret_cast<const uint32_t *>(row + 4 * c);
        if constexpr (FMT != kCacheBf16)
          sc[j][a] = *reinterpret_cast<const uint32_t *>(block + 2 * tokens * kRow + 4 * (a * tokens + pl.slot));
      }
    }
#pragma unroll
    for (int j = 0; j < HEADS; ++j)
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        if constexpr (FMT == kCacheBf16) {
          x[j][a] = w[j][a];
        } else {
          const float scale = scale_of((sc[j][a] >> (8 * (c >> 2))) & 0xffu);
          if constexpr (FMT == kCacheMx8) {
            const u32x2_t lo = widen8(w[j][a][0], scale), hi = widen8(w[j][a][1], scale);
            x[j][a] = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
          } else {
            x[j][a] = widen4(w[j][a][0], scale);
          }
        }
      }
  }
#pragma unroll
  for (int j = 0; j < HEADS; ++j) {
    if (h0 + j >= p.Hkv) break;
    const int64_t at = t * p.row_stride + (h0 + j) * p.head_stride + 8 * c;
    *reinterpret_cast<u32x4_t *>(p.k + at) = x[j][0];
    *reinterpret_cast<u32x4_t *>(p.v + at) = x[j][1];
  }
}

// ---------------------------------------------------------------------------
// Attention.  The call's tiles of 32 tokens, of every request and KV head, head
// by head, are one sequence that is cut into equal shares, one per workgroup,
// however long the requests are.  The lengths are device data, so every
// workgroup finds its share itself from the ends (a prefix sum over the
// requests).  A share's part of one (request, head) is a piece; its waves
// attend the piece's tiles w, w + 4, ... and merge through LDS.  A piece that is
// all of its pair writes the result; the others leave their state (m, l, a) in
// the workspace, at most two per workgroup, and cache_join_kernel merges them.
//
// Per tile: S^T = K Q^T with v_mfma_f32_16x16x32_bf16, K straight from memory
// in the operand's layout (lane (lr, lq) holds 16 bytes of token lr; the
// channels of a k-step are permuted alike in Q); softmax with one running
// maximum and sum per row; O^T += V^T P^T, V through LDS and its transpose
// read, P straight from the score registers.  In a score tile lane (lr, lq)
// holds tokens 16 u + 4 lq + r of row lr, in O channels 16 db + 4 lq + r.
//
// Precision: P enters as three bf16 parts, 24 bits, so that it is as good as
// fp32 (two parts leave 1.7e-6 of relative error in the result, three 2e-7);
// sums and accumulators are fp32.  The running maximum moves only where a score
// passes it by more than 2^8, which keeps a cross-lane maximum and the
// rescaling out of most tiles; weights up to 2^8 cost no precision.
// ---------------------------------------------------------------------------
constexpr int kLdsRow = 256;                        // a staged V row, bf16
constexpr int kVTile = kCacheTile * kLdsRow;
constexpr int kKept = 7;                            // rows that only some of a request's candidates see
constexpr int kAwPitch = 132;                       // floats per row of a wave's partial accumulator
constexpr float kSlack = 8.f;                       // log2 by which weights may pass 1
constexpr int kMinShare = 4;                        // tiles: one per wave

// LDS: the queries where they do not stay in registers, then the waves' V tiles
// and kept rows, whose place the waves' states take at a piece's end.
template <int RB>
struct AttendLds {
  static constexpr bool kQueries = RB > 1;
  static constexpr int kQ = kQueries ? RB * 16 * kLdsRow : 0;
  static constexpr int kWave = kVTile + kKept * kLdsRow;
  static constexpr int kMerge = kWaves * RB * 16 * (kAwPitch + 2) * 4;
  static constexpr int kBytes = kQ + (kWaves * kWave > kMerge ? kWaves * kWave : kMerge);
};

__device__ __forceinline__ int clamped_end(const CacheArgs &p, int b) {
  const int e = p.end[b];
  return e < 0 ? 0 : e > p.capacity ? p.capacity : e;
}
__device__ __forceinline__ int tiles_of(const CacheArgs &p, int b) {
  return rows_of(p, b) == 0 ? 0 : (clamped_end(p, b) + kCacheTile - 1) / kCacheTile;
}

// Tiles of the requests before mine (my requests: tx per, tx per + 1, ...) and of all; every thread of the workgroup.
struct Count {
  int before, mine, all, per;
};
__device__ __forceinline__ Count count_tiles(const CacheArgs &p, int tx, int *wave_sums) {
  Count c;
  c.per = (p.B + kThreads - 1) / kThreads;
  c.mine = 0;
  for (int j = 0; j < c.per; ++j) {
    const int b = tx * c.per + j;
    if (b < p.B) c.mine += tiles_of(p, b);
  }
  int s = c.mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(s, d);
    if ((tx & 63) >= d) s += o;
  }
  if ((tx & 63) == 63) wave_sums[tx >> 6] = s;
  __syncthreads();
  int base = 0;
  c.all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int v = wave_sums[w];
    base += w < (tx >> 6) ? v : 0;
    c.all += v;
  }
  c.before = base + s - c.mine;
  return c;
}

__device__ __forceinline__ int share_of(int total, int wgs) {
  const int s = (total + wgs - 1) / wgs;
  return s < kMinShare ? kMinShare : s;
}

// The result of one row: (m, l) of its state in the log2 domain, a / l and what came before it.  v: four channels.
struct RowEnd {
  float inv, lse, own, prev;   // 1 / l; of all; weights of this and of the earlier part
};
__device__ __forceinline__ RowEnd row_end(const CacheAttendArgs &p, int64_t row, float m, float l) {
  RowEnd r;
  r.inv = l == 0.f ? 0.f : 1.f / l;
  r.lse = l == 0.f ? kNegInf : __builtin_fmaf(m, 0.69314718055994531f, logf(l));
  r.own = 1.f;
  r.prev = 0.f;
  if (p.prev_lse != nullptr) {
    const float q = p.prev_lse[row];
    const float top = fmaxf(q, r.lse);
    if (top == kNegInf) {        // neither part has a token
      r.own = 0.f;
    } else {
      const float a = expf(r.lse - top), b = expf(q - top);
      r.own = a / (a + b);
      r.prev = b / (a + b);
      r.lse = top + logf(a + b);
    }
  }
  return r;
}
__device__ __forceinline__ f32x4_t row_value(const CacheAttendArgs &p, const RowEnd &r, int64_t at, f32x4_t a) {
  f32x4_t v = (r.inv * a) * r.own;
  // a part without tokens does not count, whatever its values
  if (r.own == 0.f) v = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (p.prev_lse != nullptr && r.prev != 0.f) v += r.prev * *reinterpret_cast<const f32x4_t *>(p.prev_out + at);
  return v;
}

template <int FMT>
struct Tile {   // a wave's loads of one tile
  static constexpr int kKLoads = FMT == kCacheBf16 ? 4 : FMT == kCacheMx8 ? 2 : 1;   // per 16 tokens
  static constexpr int kVLoads = 2 * kKLoads;
  u32x4_t k[2][kKLoads], v[kVLoads];
  uint32_t ks[2], vs[kVLoads];
};

template <int FMT, int RB>
__global__ __launch_bounds__(kThreads, RB == 4 || (RB == 2 && FMT == kCacheBf16) ? 1 : 2) void cache_attend_kernel(CacheAttendArgs p) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[AttendLds<RB>::kBytes];
  __shared__ int wave_sums[kWaves], found[2];
  constexpr int kRow = cache_row_bytes(FMT);
  constexpr int kRows = RB * 16;
  const int thread = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(thread >> 6);
  int tx = thread;

  // this workgroup's share and where it starts
  const Count cnt = count_tiles(p, tx, wave_sums);
  const int total = cnt.all * p.Hkv;
  const int share = share_of(total, p.wgs);
  const int64_t first = (int64_t)blockIdx.x * share;
  if (first >= total) return;
  int left = total - (int)first < share ? total - (int)first : share;
  int h = (int)first / cnt.all;
  const int at = (int)first - h * cnt.all;
  if (at >= cnt.before && at < cnt.before + cnt.mine) {
    int t = at - cnt.before, b = tx * cnt.per;
    for (int n = tiles_of(p, b); t >= n; n = tiles_of(p, b)) {
      t -= n;
      ++b;
    }
    found[0] = b;
    found[1] = t;
  }
  __syncthreads();
  int b = __builtin_amdgcn_readfirstlane(found[0]);
  int t0 = __builtin_amdgcn_readfirstlane(found[1]);

  const int page_tokens = 1 << p.page_shift;
  const uint32_t v_off = (uint32_t)(page_tokens * kRow), ks_off = 2 * v_off, vs_off = ks_off + 4u * (uint32_t)page_tokens;
  unsigned char *qs = smem, *vs_lds = smem + AttendLds<RB>::kQ + w * AttendLds<RB>::kWave;
  while (left > 0) {
    const int tiles = tiles_of(p, b);
    if (tiles - t0 <= 0) {            // a request without tokens or rows
      t0 = 0;
      if (++b == p.B) {
        b = 0;
        ++h;
      }
      continue;
    }
    const int piece = tiles - t0 < left ? tiles - t0 : left;
    // from here on, and again per tile and behind them, the thread's index is
    // one that the compiler has not seen: else it keeps every address of the
    // piece, the tile and the merge in a register of its own all the way
    tx = thread;
    asm volatile("" : "+v"(tx));
    const int lane = tx & 63, lr = lane & 15, lq = lane >> 4;
    const int n = rows_of(p, b), M = n * p.G;
    const int len = clamped_end(p, b);
    const int row0 = p.row_start == nullptr ? b * p.max_rows : p.row_start[b];
    const int raw_end = p.end[b];     // a causal row's last token counts from the uncut end
    const int32_t *table = p.table + (int64_t)b * p.table_stride;

    // queries: B operand of k-step s, row 16 rb + lr, the chunk of 8 channels
    // that K's lanes hold there; from LDS (chunk c of row r at c ^ (r & 15))
    // where they would take too many registers
    auto chunk_of = [](int s, int lq) { return FMT == kCacheBf16 ? 4 * s + lq : FMT == kCacheMx8 ? 2 * (4 * (s >> 1) + lq) + (s & 1) : 4 * lq + s; };
    bf16x8_t qop[4];
    if constexpr (!AttendLds<RB>::kQueries) {
      const int i = lr / p.G;
      const int64_t row = row0 + i;
      const bool ok = lr < M && row >= 0 && row < p.num_rows;
      const uint16_t *src = p.q + (ok ? row * p.q_row_stride + (int64_t)(h * p.G + lr - i * p.G) * kCacheDim : 0);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t *>(src + 8 * chunk_of(s, lq));
        qop[s] = __builtin_bit_cast(bf16x8_t, ok ? x : u32x4_t{0u, 0u, 0u, 0u});
      }
    } else {
#pragma unroll
      for (int e = 0; e < RB; ++e) {
        const int r = 16 * e + (tx >> 4), c = tx & 15;
        const int i = r / p.G;
        const int64_t row = row0 + i;
        const bool ok = r < M && row >= 0 && row < p.num_rows;
        const uint16_t *src = p.q + (ok ? row * p.q_row_stride + (int64_t)(h * p.G + r - i * p.G) * kCacheDim : 0);
        const u32x4_t x = *reinterpret_cast<const u32x4_t *>(src + 8 * c);
        *reinterpret_cast<u32x4_t *>(qs + r * kLdsRow + 16 * (c ^ (r & 15))) = ok ? x : u32x4_t{0u, 0u, 0u, 0u};
      }
      __syncthreads();
    }
    // tokens that each of the lane's rows sees
    int limit[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int i = (16 * rb + lr) / p.G;
      const int64_t last = (int64_t)raw_end - n + i + 1;
      limit[rb] = p.causal && last < len ? (last < 0 ? 0 : (int)last) : len;
    }
    const int64_t first_last = (int64_t)raw_end - n + 1;
    const int all_see = p.causal && first_last < len ? (first_last < 0 ? 0 : (int)first_last) : len;   // tokens that every row sees

    float m_run[RB], l_run[RB];
    f32x4_t acc[RB][8];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      m_run[rb] = kNegInf;
      l_run[rb] = 0.f;
#pragma unroll
      for (int db = 0; db < 8; ++db) acc[rb][db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    // page of half tile j of this wave's tiles: one load for 32 tiles, lane j
    // for half tile j; -1 for what is no page
    const int mine = (piece - w + kWaves - 1) / kWaves;     // this wave's tiles (may be 0 or less)
    auto pages_of = [&](int k0) {
      const int k = k0 + (lane >> 1);
      const int64_t tok = (int64_t)(t0 + w + kWaves * k) * kCacheTile + 16 * (lane & 1);
      int id = -1;
      if (k < mine && tok < len) id = table[tok >> p.page_shift];
      return id >= 0 && id < p.num_pages ? id : -1;
    };
    int ids = pages_of(0), ids_next = -1;

    Tile<FMT> cur;
    uint32_t gone = 0;     // halves of the loaded tile without a page
    auto load = [&](int k, Tile<FMT> &d) {
      const int tok = (t0 + w + kWaves * k) * kCacheTile;
      __amdgpu_buffer_rsrc_t krs[2], vrs[2], srs[2];
      uint32_t slot[2];
      gone = 0;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int id = __builtin_amdgcn_readlane(ids, 2 * (k & 31) + u);
        const int tu = tok + 16 * u;
        int ok = len - tu;
        ok = ok < 0 || id < 0 ? 0 : ok > 16 ? 16 : ok;
        gone |= (id < 0 ? 1u : 0u) << u;
        slot[u] = (uint32_t)(tu & (page_tokens - 1));
        uint8_t *base = p.pages + (uint64_t)(id < 0 ? 0 : id) * p.page_stride + (uint64_t)h * p.head_bytes;
        krs[u] = __builtin_amdgcn_make_buffer_rsrc(base, (short)0, ok > 0 ? (int)p.head_bytes : 0, kBufferFlags);
        // rows past the request's tokens read zero: a weight of zero must meet no leftover NaN
        vrs[u] = __builtin_amdgcn_make_buffer_rsrc(base, (short)0, ok > 0 ? (int)(v_off + (slot[u] + ok) * kRow) : 0, kBufferFlags);
        srs[u] = __builtin_amdgcn_make_buffer_rsrc(base, (short)0, ok > 0 ? (int)(vs_off + (slot[u] + ok) * 4) : 0, kBufferFlags);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t o = (slot[u] + lr) * kRow + 16 * lq;
#pragma unroll
        for (int s = 0; s < Tile<FMT>::kKLoads; ++s)
          d.k[u][s] = __builtin_amdgcn_raw_buffer_load_b128(krs[u], o + 64 * s, 0, kStreamLoad);
        if constexpr (FMT != kCacheBf16) d.ks[u] = __builtin_amdgcn_raw_buffer_load_b32(krs[u], ks_off + (slot[u] + lr) * 4, 0, kStreamLoad);
      }
      // V: 16-byte chunks of whole rows, kLanes lanes to a row
      constexpr int kLanes = kRow / 16, kStep = 64 / kLanes;   // rows per load: 4, 8, 16
#pragma unroll
      for (int i = 0; i < Tile<FMT>::kVLoads; ++i) {
        const int u = i * kStep / 16;
        const uint32_t row = slot[u] + (i * kStep) % 16 + lane / kLanes;
        d.v[i] = __builtin_amdgcn_raw_buffer_load_b128(vrs[u], v_off + row * kRow + 16 * (lane % kLanes), 0, kStreamLoad);
        if constexpr (FMT != kCacheBf16)
          d.vs[i] = __builtin_amdgcn_raw_buffer_load_b8(srs[u], vs_off + row * 4 + (lane % kLanes) * 4 / kLanes, 0, kStreamLoad);
      }
    };

    auto tile = [&](int k, int lane) {
      const int lr = lane & 15, lq = lane >> 4;
      // V's transpose read: row 4 lq + lr / 4 (+ 16), chunk 2 db + (lr & 3) / 2, half lr & 1
      const int vrow = 4 * lq + (lr >> 2);
      const int vrd = vrow * kLdsRow + 8 * (lr & 1);
      const int vsw = 2 * (vrow & 7);
      const int vc0 = (lr & 3) >> 1;
      const int tok = (t0 + w + kWaves * k) * kCacheTile;
      const uint32_t hole = gone;
      // V to LDS as bf16: 16-byte chunk c of row t at c ^ 2 (t & 7)
      constexpr int kLanes = kRow / 16, kStep = 64 / kLanes;
      bool odd = false;      // a value that is no number, where that matters
      const bool mixed = p.causal && tok + kCacheTile > all_see;
#pragma unroll
      for (int i = 0; i < Tile<FMT>::kVLoads; ++i) {
        const int t = i * kStep + lane / kLanes, c = lane % kLanes;
        unsigned char *row = vs_lds + t * kLdsRow;
        u32x4_t x[kLdsRow / kRow];
        if constexpr (FMT == kCacheBf16) {
          x[0] = cur.v[i];
        } else if constexpr (FMT == kCacheMx8) {
          const float s = scale_of(cur.vs[i]);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const u32x2_t a = widen8(cur.v[i][2 * j], s), d = widen8(cur.v[i][2 * j + 1], s);
            x[j] = u32x4_t{a[0], a[1], d[0], d[1]};
          }
        } else {
          const float s = scale_of(cur.vs[i]);
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = widen4(cur.v[i][j], s);
        }
#pragma unroll
        for (int j = 0; j < kLdsRow / kRow; ++j)
          *reinterpret_cast<u32x4_t *>(row + 16 * ((c * (kLdsRow / kRow) + j) ^ (2 * (t & 7)))) = x[j];
        if (mixed) {
#pragma unroll
          for (int j = 0; j < kLdsRow / kRow; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              odd |= (x[j][e] & 0x7f80u) == 0x7f80u || (x[j][e] & 0x7f800000u) == 0x7f800000u;
        }
      }

      // S^T = K Q^T
      f32x4_t sacc[2][RB];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        bf16x8_t kop[4];
        if constexpr (FMT == kCacheBf16) {
#pragma unroll
          for (int s = 0; s < 4; ++s) kop[s] = __builtin_bit_cast(bf16x8_t, cur.k[u][s]);
        } else if constexpr (FMT == kCacheMx8) {
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const float f = scale_of((cur.ks[u] >> (16 * (s >> 1) + 8 * (lq >> 1))) & 0xffu);
            const u32x2_t a = widen8(cur.k[u][s >> 1][2 * (s & 1)], f), d = widen8(cur.k[u][s >> 1][2 * (s & 1) + 1], f);
            kop[s] = __builtin_bit_cast(bf16x8_t, u32x4_t{a[0], a[1], d[0], d[1]});
          }
        } else {
          const float f = scale_of((cur.ks[u] >> (8 * lq)) & 0xffu);
#pragma unroll
          for (int s = 0; s < 4; ++s) kop[s] = __builtin_bit_cast(bf16x8_t, widen4(cur.k[u][0][s], f));
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            bf16x8_t qv;
            if constexpr (AttendLds<RB>::kQueries)
              qv = *reinterpret_cast<const bf16x8_t *>(qs + (16 * rb + lr) * kLdsRow + 16 * (chunk_of(s, lq) ^ lr));
            else
              qv = qop[s];
            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[s], qv, x, 0, 0, 0);
          }
          sacc[u][rb] = x;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      load(k + 1, cur);     // behind the last tile there are no pages: such loads touch no memory
      __builtin_amdgcn_sched_barrier(0);

      const bool masked = hole != 0 || tok + kCacheTile > all_see;
      const int odd_first = all_see > tok ? all_see - tok : 0, odd_end = len - tok < kCacheTile ? len - tok : kCacheTile;
      const bool apart = mixed && __builtin_amdgcn_ballot_w64(odd) != 0;
      if (apart) {
        // A value that is no number stands at a token that some rows see and
        // others do not, where a weight of zero would spread it.  Such tokens'
        // V rows (kKept at most) are set aside and cleared here, and added one
        // by one to the rows that see them.
        for (int t = odd_first; t < odd_end; ++t)
          if (lane < 16) {
            u32x4_t *row = reinterpret_cast<u32x4_t *>(vs_lds + t * kLdsRow + 16 * lane);
            *reinterpret_cast<u32x4_t *>(vs_lds + kVTile + (t - odd_first) * kLdsRow + 16 * (lane ^ (2 * (t & 7)))) = *row;
            *row = u32x4_t{0u, 0u, 0u, 0u};
          }
        asm volatile("" ::: "memory");
      }
      constexpr int RP = RB < 2 ? RB : 2;     // row blocks at once: what P's parts take of the registers
#pragma unroll
      for (int r0 = 0; r0 < RB; r0 += RP) {
      bf16x8_t part[RP][3];
#pragma unroll
      for (int rp = 0; rp < RP; ++rp) {
        const int rb = r0 + rp;
        float x[8], mx = kNegInf;
        if (!masked) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] = sacc[e >> 2][rb][e & 3];
            mx = fmaxf(mx, x[e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int t = tok + 16 * (e >> 2) + 4 * lq + (e & 3);
            const bool sees = t < limit[rb] && !((hole >> (e >> 2)) & 1u);
            x[e] = sees ? sacc[e >> 2][rb][e & 3] : kNegInf;
            mx = fmaxf(mx, x[e]);
          }
        }
        mx *= p.scale_log2;
        if (__builtin_amdgcn_ballot_w64(mx > m_run[rb] + kSlack)) {
          const float mn = fmaxf(m_run[rb], xgroup_max(mx));
          const float alpha = mn == kNegInf ? 1.f : exp2_fast(m_run[rb] - mn);
          l_run[rb] *= alpha;
#pragma unroll
          for (int db = 0; db < 8; ++db) acc[rb][db] *= alpha;
          m_run[rb] = mn;
        }
        const float ms = m_run[rb] == kNegInf ? 0.f : m_run[rb];
        float ls = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float pe = exp2_fast(__builtin_fmaf(x[e], p.scale_log2, -ms));
          ls += pe;
          const __bf16 a = (__bf16)pe;
          const float r1 = pe - (float)a;
          const __bf16 m = (__bf16)r1;
          part[rp][0][e] = a;
          part[rp][1][e] = m;
          part[rp][2][e] = (__bf16)(r1 - (float)m);
        }
        l_run[rb] += ls;
      }
      __builtin_amdgcn_sched_barrier(0);

      if (apart) {
        for (int t = odd_first; t < odd_end; ++t) {
          const unsigned char *row = vs_lds + kVTile + (t - odd_first) * kLdsRow + 8 * lq;
          const int e = 4 * (t >> 4) + (t & 3);
#pragma unroll
          for (int rp = 0; rp < RP; ++rp) {
            const int rb = r0 + rp;
            float pe = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) pe = j == e ? (float)part[rp][0][j] + (float)part[rp][1][j] + (float)part[rp][2][j] : pe;
            pe = __shfl(pe, lr + 16 * ((t >> 2) & 3));
            if (tok + t >= limit[rb]) continue;
#pragma unroll
            for (int db = 0; db < 8; ++db) {
              const u32x2_t x = *reinterpret_cast<const u32x2_t *>(row + 32 * db);
#pragma unroll
              for (int j = 0; j < 4; ++j)
                acc[rb][db][j] += pe * __uint_as_float(j & 1 ? x[j >> 1] & 0xffff0000u : x[j >> 1] << 16);
            }
          }
        }
      }

      // O^T += V^T P^T
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        if (db == 4) __builtin_amdgcn_sched_barrier(0);
        const int off = vrd + 16 * ((2 * db + vc0) ^ vsw);
        const s16x4_t v0 = lds_read_tr16(vs_lds + off);
        const s16x4_t v1 = lds_read_tr16(vs_lds + off + 16 * kLdsRow);
        const bf16x8_t vop = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int rp = 0; rp < RP; ++rp)
#pragma unroll
          for (int j = 0; j < 3; ++j)
            acc[r0 + rp][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop, part[rp][j], acc[r0 + rp][db], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      }
    };

    if (mine > 0) {
      load(0, cur);
      for (int k = 0; k < mine; ++k) {
        if ((k & 31) == 0) ids_next = pages_of(k + 32);
        // tile k is in flight; the loads of tile k + 1 take its pages from the next word
        if ((k & 31) == 31) ids = ids_next;
        int l = lane;
        asm volatile("" : "+v"(l));
        tile(k, l);
      }
    }

    // the waves' states -> LDS, merged by kSegs threads per row
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) l_run[rb] = xgroup_sum(l_run[rb]);
    __syncthreads();
    tx = thread;
    asm volatile("" : "+v"(tx));
    float *aw = reinterpret_cast<float *>(smem + AttendLds<RB>::kQ);
    float *mw = aw + kWaves * kRows * kAwPitch;
    float *lw = mw + kWaves * kRows;
    {
    const int lr = tx & 15, lq = (tx >> 4) & 3;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float *row = aw + (w * kRows + rb * 16 + lr) * kAwPitch + 4 * lq;
#pragma unroll
      for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4_t *>(row + 16 * db) = acc[rb][db];
      if (lq == 0) {
        mw[w * kRows + rb * 16 + lr] = m_run[rb];
        lw[w * kRows + rb * 16 + lr] = l_run[rb];
      }
    }
    }
    __syncthreads();
    constexpr int kSegs = kThreads / kRows, kPieces = kCacheDim / 4 / kSegs;   // 16, 8 or 4 threads a row
    const int r = tx / kSegs, seg = tx % kSegs;
    if (r < M) {
      float mv[kWaves], top = kNegInf;
#pragma unroll
      for (int j = 0; j < kWaves; ++j) {
        mv[j] = mw[j * kRows + r];
        top = fmaxf(top, mv[j]);
      }
      float f[kWaves], l = 0.f;
#pragma unroll
      for (int j = 0; j < kWaves; ++j) {
        f[j] = top == kNegInf ? 1.f : exp2_fast(mv[j] - top);   // without a maximum every state is zero, or no number
        l += f[j] * lw[j * kRows + r];
      }
      f32x4_t a[kPieces];
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        a[k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kWaves; ++j)
          a[k] += f[j] * *reinterpret_cast<const f32x4_t *>(aw + (j * kRows + r) * kAwPitch + 4 * (seg + kSegs * k));
      }
      if (piece == tiles) {
        const int i = r / p.G;
        const int64_t row = ((int64_t)row0 + i) * p.Hq + h * p.G + r - i * p.G;
        if (row0 + i >= 0 && row0 + i < p.num_rows) {
          const RowEnd end = row_end(p, row, top, l);
#pragma unroll
          for (int k = 0; k < kPieces; ++k) {
            const int64_t o = row * kCacheDim + 4 * (seg + kSegs * k);
            *reinterpret_cast<f32x4_t *>(p.out + o) = row_value(p, end, o, a[k]);
          }
          if (seg == 0 && p.lse != nullptr) p.lse[row] = end.lse;
        }
      } else {
        // two states per workgroup at most: of a pair that starts before the share, and of one that ends behind it
        const int64_t o = (int64_t)(2 * blockIdx.x + (t0 == 0 ? 1 : 0)) * p.M + r;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) *reinterpret_cast<f32x4_t *>(p.part_a + o * kCacheDim + 4 * (seg + kSegs * k)) = a[k];
        if (seg == 0) *reinterpret_cast<f32x2_t *>(p.part_ml + 2 * o) = f32x2_t{top, l};
      }
    }
    left -= piece;
    t0 = 0;
    if (++b == p.B) {
      b = 0;
      ++h;
    }
    if (left > 0) __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Merge the pieces' states of each (request, KV head) that more than one
// workgroup attended, and write the rows of requests without tokens.  A half
// wave holds a row's 128 channels; SPLIT half waves of the workgroup share a
// row's states (8 where a pair has many), else each takes a row of its own.
// ---------------------------------------------------------------------------
template <int SPLIT>
__global__ __launch_bounds__(kThreads) void cache_join_kernel(CacheAttendArgs p) {
  __shared__ int wave_sums[kWaves], found;
  constexpr int kRowsPer = 8 / SPLIT;
  const int tx = threadIdx.x, lane = tx & 31;
  const int part = (tx >> 5) % SPLIT;
  const int b = blockIdx.x / p.Hkv, h = blockIdx.x % p.Hkv;
  const int r = blockIdx.y * kRowsPer + (tx >> 5) / SPLIT;
  const Count cnt = count_tiles(p, tx, wave_sums);
  if (b >= tx * cnt.per && b < (tx + 1) * cnt.per) {
    int s = cnt.before;
    for (int j = tx * cnt.per; j < b; ++j) s += tiles_of(p, j);
    found = s;
  }
  __syncthreads();
  const int tiles = tiles_of(p, b), n = rows_of(p, b);
  const int row0 = p.row_start == nullptr ? b * p.max_rows : p.row_start[b];
  const int i = r / p.G;
  const bool mine = r < n * p.G && row0 + i >= 0 && row0 + i < p.num_rows;
  const int64_t row = ((int64_t)row0 + i) * p.Hq + h * p.G + r - i * p.G;
  float m = kNegInf, l = 0.f;
  f32x4_t a = {0.f, 0.f, 0.f, 0.f};
  if (tiles > 0) {
    const int share = share_of(cnt.all * p.Hkv, p.wgs);
    const int start = h * cnt.all + found;
    const int w0 = start / share, w1 = (start + tiles - 1) / share;
    if (w0 == w1) return;           // one workgroup attended all of it
    if (mine)
      for (int w = w0 + part; w <= w1; w += SPLIT) {
        const int64_t o = (int64_t)(2 * w + (w == w0 ? 1 : 0)) * p.M + r;
        const f32x2_t ml = *reinterpret_cast<const f32x2_t *>(p.part_ml + 2 * o);
        const f32x4_t x = *reinterpret_cast<const f32x4_t *>(p.part_a + o * kCacheDim + 4 * lane);
        const float mn = fmaxf(m, ml[0]);
        const float fa = mn == kNegInf ? 1.f : exp2_fast(m - mn), fb = mn == kNegInf ? 1.f : exp2_fast(ml[0] - mn);
        a = fa * a + fb * x;
        l = fa * l + fb * ml[1];
        m = mn;
      }
  }
  if constexpr (SPLIT > 1) {
    __shared__ __attribute__((aligned(16))) float sa[8][kCacheDim];
    __shared__ float sm[8], sl[8];
    *reinterpret_cast<f32x4_t *>(&sa[tx >> 5][4 * lane]) = a;
    if (lane == 0) {
      sm[tx >> 5] = m;
      sl[tx >> 5] = l;
    }
    __syncthreads();
    if (part != 0) return;
    float top = kNegInf;
#pragma unroll
    for (int j = 0; j < SPLIT; ++j) top = fmaxf(top, sm[(tx >> 5) + j]);
    a = f32x4_t{0.f, 0.f, 0.f, 0.f};
    l = 0.f;
#pragma unroll
    for (int j = 0; j < SPLIT; ++j) {
      const float f = top == kNegInf ? 1.f : exp2_fast(sm[(tx >> 5) + j] - top);
      l += f * sl[(tx >> 5) + j];
      a += f * *reinterpret_cast<const f32x4_t *>(&sa[(tx >> 5) + j][4 * lane]);
    }
    m = top;
  }
  if (!mine) return;
  const RowEnd end = row_end(p, row, m, l);
  const int64_t o = row * kCacheDim + 4 * lane;
  *reinterpret_cast<f32x4_t *>(p.out + o) = row_value(p, end, o, a);
  if (lane == 0 && p.lse != nullptr) p.lse[row] = end.lse;
}

// One head per workgroup up to this many rows x heads, four above.
constexpr int64_t kFewRows = 1 << 14;

template <int FMT, typename F1, typename F4>
hipError_t launch_rows(const CacheRowsArgs &p, F1 one, F4 four, hipStream_t s) {
  const unsigned groups = (unsigned)((p.num_rows + (int64_t)kGroupRows - 1) / kGroupRows);
  if ((int64_t)p.num_rows * p.Hkv <= kFewRows)
    hipLaunchKernelGGL(one, dim3(groups, p.Hkv), dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL(four, dim3(groups, (p.Hkv + 3) / 4), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

template <int FMT>
hipError_t attend(const CacheAttendArgs &p, hipStream_t s) {
  if (p.M <= 16)
    hipLaunchKernelGGL((cache_attend_kernel<FMT, 1>), dim3(p.wgs), dim3(kThreads), 0, s, p);
  else if (p.M <= 32)
    hipLaunchKernelGGL((cache_attend_kernel<FMT, 2>), dim3(p.wgs), dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL((cache_attend_kernel<FMT, 4>), dim3(p.wgs), dim3(kThreads), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t pairs = (int64_t)p.B * p.Hkv;
  if (pairs * 8 <= p.wgs)
    hipLaunchKernelGGL((cache_join_kernel<8>), dim3((unsigned)pairs, p.M), dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL((cache_join_kernel<1>), dim3((unsigned)pairs, (p.M + 7) / 8), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

int cache_attend_wgs(int fmt, int B, int Hkv, int capacity, int M) {
  (void)fmt;
  const int64_t most = M <= 32 ? 512 : 256;
  const int64_t tiles = (int64_t)B * Hkv * ((capacity + kCacheTile - 1) / kCacheTile);
  const int64_t need = (tiles + kMinShare - 1) / kMinShare;
  return (int)(need < most ? need : most);
}

hipError_t launch_cache_write(const CacheRowsArgs &p, int fmt, hipStream_t s) {
  if (fmt == kCacheBf16) return launch_rows<kCacheBf16>(p, cache_write_kernel<kCacheBf16, 1>, cache_write_kernel<kCacheBf16, 4>, s);
  if (fmt == kCacheMx8) return launch_rows<kCacheMx8>(p, cache_write_kernel<kCacheMx8, 1>, cache_write_kernel<kCacheMx8, 4>, s);
  return launch_rows<kCacheMx4>(p, cache_write_kernel<kCacheMx4, 1>, cache_write_kernel<kCacheMx4, 4>, s);
}

hipError_t launch_cache_read(const CacheRowsArgs &p, int fmt, hipStream_t s) {
  if (fmt == kCacheBf16) return launch_rows<kCacheBf16>(p, cache_read_kernel<kCacheBf16, 1>, cache_read_kernel<kCacheBf16, 4>, s);
  if (fmt == kCacheMx8) return launch_rows<kCacheMx8>(p, cache_read_kernel<kCacheMx8, 1>, cache_read_kernel<kCacheMx8, 4>, s);
  return launch_rows<kCacheMx4>(p, cache_read_kernel<kCacheMx4, 1>, cache_read_kernel<kCacheMx4, 4>, s);
}

hipError_t launch_cache_attend(const CacheAttendArgs &p, int fmt, hipStream_t s) {
  if (fmt == kCacheBf16) return attend<kCacheBf16>(p, s);
  if (fmt == kCacheMx8) return attend<kCacheMx8>(p, s);
  return attend<kCacheMx4>(p, s);
}

}  // namespace ss
