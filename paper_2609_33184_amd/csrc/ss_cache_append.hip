// gfx950 (MI355X) kernels of the paged cache's drafted rows: K, V and Q rows that
// enter with the position rotation applied, and the rows of an accepted path that
// move to the places behind the history.
#include <hip/hip_runtime.h>

#include "ss_cache.h"
#include "ss_cache_device.h"
#include "ss_turn.h"

namespace ss {
namespace {

// ---------------------------------------------------------------------------
// Appending rows.  A pair of channels (x1, x2) of a row at position p turns by the
// angle a = p f, f the pair's frequency: y1 = s (x1 cos a - x2 sin a), y2 = s (x2 cos
// a + x1 sin a).  Lanes and rows as in cache_write_kernel: 16 lanes to a row's 128
// channels, 8 each; a workgroup takes 16 rows and HEADS KV heads, or 2 HEADS query
// heads of them.  A lane turns the same channels in all its heads, so its angles'
// sines are computed once.  Pairs half a rotated head apart lie in lanes half of
// its lanes apart and are exchanged, neighbouring pairs lie in a lane.
//
// Precision.  All of it is in 64 bits, whose products cost what those of 32 do here:
// the angle, which grows with the position; its rest of a quarter turn, taken off in
// two steps; sine and cosine, Taylor series over an eighth of a turn either way, off
// by 7e-12; the turned pair.  That is rounded to fp32 and then to bf16, as a
// reference in 64 bits rounds it; K is quantised from there, so that a cache is bit
// for bit the one that the rotated rows' ss_cache_write gives.
//
// What bounds it: filling prompts, memory (16 of 2048 to 8191 rows, 32 + 8 heads, 8 bits: 1.7 GB read and
// written, 389 us, 4.3 TB/s; a large copy 4.9); drafted rows a launch and the angles' 30 products of 64 bits each, which the 40 workgroups
// of 16 rows repeat (16 requests of 16 to 48 rows, 64 + 8 heads in bf16 8.4 us; every lane its own eight angles 10.3).
// ---------------------------------------------------------------------------

__device__ __forceinline__ float low_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)lo, (__bf16)hi});
}

__device__ __forceinline__ double from_lane(double x, int lane) {
  const uint64_t w = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * lane, (int)w), hi = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * lane, (int)(w >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// To fp32 and no further: the compiler would join this rounding and that to bf16, which costs nine instructions more.
__device__ __forceinline__ float rounded(double x) {
  float y = (float)x;
  asm("" : "+v"(y));
  return y;
}

struct Turn {
  double c[8], s[8];     // of the lane's channels: y = c x + s partner; of its neighbouring pairs: the first four
  int partner;           // the lane that holds the partners; itself: neighbouring pairs
  bool turns;            // whether the lane's channels turn at all
};
__device__ __forceinline__ Turn turn_at(const CacheAppendArgs &p, int64_t pos, int c) {
  Turn r;
  const int half = p.rotary_dim / 2, lanes = half / 8;      // of a half of the rotated channels
  r.turns = 8 * c < p.rotary_dim;
  const int me = threadIdx.x & 63;
  r.partner = p.interleaved || !r.turns ? me : c < lanes ? me + lanes : me - lanes;
  // A lane's four neighbouring pairs, or half of the eight that it has with its partner, who brings the others.
  const bool lower = c < lanes;
  const int first = p.interleaved ? 4 * c : lower ? 8 * c : 8 * (c - lanes) + 4;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    double cj, sj;
    turn_of((double)pos, p.inv_freq[r.turns ? first + j : 0], p.scale, cj, sj);
    const double co = from_lane(cj, r.partner), so = from_lane(sj, r.partner);
    r.c[j] = p.interleaved || lower ? cj : co;
    r.s[j] = p.interleaved ? sj : lower ? -sj : so;
    r.c[4 + j] = lower ? co : cj;
    r.s[4 + j] = lower ? -so : sj;
  }
  return r;
}
__device__ __forceinline__ u32x4_t turned(const CacheAppendArgs &p, const Turn &r, u32x4_t x) {
  u32x4_t y;
  if (p.interleaved) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const double a = low_of(x[j]), b = high_of(x[j]), c = r.c[j], s = r.s[j];
      y[j] = pack_bf16(rounded(__builtin_fma(a, c, -(b * s))), rounded(__builtin_fma(b, c, a * s)));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t o = (uint32_t)__shfl((int)x[j], r.partner);
      y[j] = pack_bf16(rounded(__builtin_fma((double)low_of(x[j]), r.c[2 * j], (double)low_of(o) * r.s[2 * j])),
                       rounded(__builtin_fma((double)high_of(x[j]), r.c[2 * j + 1], (double)high_of(o) * r.s[2 * j + 1])));
    }
  }
  return r.turns ? y : x;
}

template <int FMT, int HEADS>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(CacheAppendArgs p) {
  extern __shared__ int32_t starts[];
  int32_t *ends = starts + p.B + 1;
  const int tx = threadIdx.x, c = tx & 15;
  const int64_t t = (int64_t)blockIdx.x * kGroupRows + (tx >> 4);
  const int64_t tl = t < p.num_rows ? t : p.num_rows - 1;
  const int kv_parts = (p.Hkv + HEADS - 1) / HEADS;
  const bool is_q = (int)blockIdx.y >= kv_parts;
  const int h0 = is_q ? ((int)blockIdx.y - kv_parts) * 2 * HEADS : (int)blockIdx.y * HEADS;
  const int heads = is_q ? p.Hq : p.Hkv;
  u32x4_t x[2 * HEADS];      // query heads, or K and V of KV heads
#pragma unroll
  for (int j = 0; j < 2 * HEADS; ++j) {
    const int hj = is_q ? h0 + j : h0 + (j >> 1), h = hj < heads ? hj : heads - 1;
    const uint16_t *row = is_q ? p.q + tl * p.q_row_stride : (j & 1 ? p.v : p.k) + tl * p.row_stride;
    x[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(row + h * kCacheDim + 8 * c));
  }
  const Place pl = place_of(p, t, tx, starts, ends);
  const Turn turn = turn_at(p, p.positions != nullptr ? p.positions[tl] : pl.pos, c);
  if (is_q) {
#pragma unroll
    for (int j = 0; j < 2 * HEADS; ++j) x[j] = turned(p, turn, x[j]);
    if (!pl.row) return;
#pragma unroll
    for (int j = 0; j < 2 * HEADS; ++j) {
      if (h0 + j >= heads) break;
      *reinterpret_cast<u32x4_t *>(p.q_out + t * p.q_out_row_stride + (h0 + j) * kCacheDim + 8 * c) = x[j];
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < HEADS; ++j) x[2 * j] = turned(p, turn, x[2 * j]);
  if (pl.page == nullptr) return;
  constexpr int kRow = cache_row_bytes(FMT);
  const int tokens = 1 << p.page_shift;
#pragma unroll
  for (int j = 0; j < HEADS; ++j) {
    if (h0 + j >= heads) break;
    uint8_t *block = pl.page + (uint64_t)(h0 + j) * p.head_bytes;
    uint8_t *scales = block + 2 * tokens * kRow;
    store_row<FMT>(block, scales, pl.slot, c, x[2 * j]);
    store_row<FMT>(block + tokens * kRow, scales + 4 * tokens, pl.slot, c, x[2 * j + 1]);
  }
}

// Rows x KV heads up to which a workgroup takes one KV head or two query heads, beyond four and eight, since all of a row's
// workgroups compute the same sines: with 8 KV heads one and four, in the kernel, 64 rows 4.2 and 5.2 us, 256 rows 5.3 and 6.1, 480 rows
// with 64 query heads 8.1 and 8.5; 1024 rows 9.4 and 8.8, 2048 rows 16.6 and 11.8.
constexpr int64_t kFewRows = 1 << 12;

template <int FMT>
hipError_t append(const CacheAppendArgs &p, hipStream_t s) {
  const unsigned groups = (unsigned)((p.num_rows + (int64_t)kGroupRows - 1) / kGroupRows);
  const size_t lds = p.row_start == nullptr ? 0 : (2 * (size_t)p.B + 1) * sizeof(int32_t);
  const int hq = p.q != nullptr ? p.Hq : 0;
  if ((int64_t)p.num_rows * p.Hkv <= kFewRows)
    hipLaunchKernelGGL((cache_append_kernel<FMT, 1>), dim3(groups, p.Hkv + (hq + 1) / 2), dim3(kThreads), lds, s, p);
  else
    hipLaunchKernelGGL((cache_append_kernel<FMT, 4>), dim3(groups, (p.Hkv + 3) / 4 + (hq + 7) / 8), dim3(kThreads), lds, s, p);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Keeping a path.  Of a request's last n tokens the kept ones move to the first
// places, whole rows with their scales, so nothing is rounded.  A workgroup takes
// one request and KV head and has read all of them (at most kCacheMaxTree, 16 lanes
// a row) before it writes one, whatever order they are given in.  Its time is one round
// trip to memory behind the table's and the list's: 256 requests, up to 12 rows each of 8 heads in bf16 (7 MB) 6.1 us, one request 3.2.
// ---------------------------------------------------------------------------
template <int BYTES>
struct Bytes;
template <>
struct Bytes<16> { using T = u32x4_t; };
template <>
struct Bytes<8> { using T = u32x2_t; };
template <>
struct Bytes<4> { using T = uint32_t; };

template <int FMT>
__global__ __launch_bounds__(kThreads) void cache_keep_kernel(CacheKeepArgs p) {
  constexpr int kRow = cache_row_bytes(FMT), kEach = kCacheMaxTree / kGroupRows;
  using T = typename Bytes<kRow / 16>::T;
  const int tx = threadIdx.x, c = tx & 15, b = blockIdx.x, h = blockIdx.y;
  const int64_t first = p.row_start == nullptr ? (int64_t)b * p.max_rows : p.row_start[b];
  const int64_t n = p.row_start == nullptr ? p.max_rows : p.row_start[b + 1] - first;
  if (n < 1 || n > p.max_rows) return;
  const int most = p.num_kept[b], m = most < n ? most : (int)n;
  const int64_t base = p.end[b] - n;
  const int tokens = 1 << p.page_shift;
  const auto at = [&](int64_t pos, int &slot) -> uint8_t * {      // the head's block and the slot there of the token at pos
    if (pos < 0 || pos >= p.capacity) return nullptr;
    const int page = p.table[(int64_t)b * p.table_stride + (pos >> p.page_shift)];
    slot = (int)(pos & (tokens - 1));
    return page < 0 || page >= p.num_pages ? nullptr : p.pages + (uint64_t)page * p.page_stride + (uint64_t)h * p.head_bytes;
  };
  T k[kEach], v[kEach];
  uint32_t ks[kEach], vs[kEach];
  uint8_t *to[kEach];
  int to_slot[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int j = (tx >> 4) + kGroupRows * i;
    const int64_t row = first + j;
    to[i] = nullptr;
    to_slot[i] = 0;
    k[i] = v[i] = T{};
    ks[i] = vs[i] = 0;
    const int node = j < m && row >= 0 && row < p.num_rows ? p.kept[row] : -1;
    if (node < 0 || node >= n || node == j) continue;
    int slot = 0;
    const uint8_t *from = at(base + node, slot);
    if (from == nullptr) continue;
    to[i] = at(base + j, to_slot[i]);
    k[i] = *reinterpret_cast<const T *>(from + slot * kRow + c * (kRow / 16));
    v[i] = *reinterpret_cast<const T *>(from + (tokens + slot) * kRow + c * (kRow / 16));
    if constexpr (FMT != kCacheBf16) {
      ks[i] = *reinterpret_cast<const uint32_t *>(from + 2 * tokens * kRow + 4 * slot);
      vs[i] = *reinterpret_cast<const uint32_t *>(from + 2 * tokens * kRow + 4 * (tokens + slot));
    }
  }
  // the rows are in registers, not only asked for, when the first one is overwritten
#pragma unroll
  for (int i = 0; i < kEach; ++i) asm volatile("" : "+v"(k[i]), "+v"(v[i]), "+v"(ks[i]), "+v"(vs[i])::"memory");
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (to[i] == nullptr) continue;
    *reinterpret_cast<T *>(to[i] + to_slot[i] * kRow + c * (kRow / 16)) = k[i];
    *reinterpret_cast<T *>(to[i] + (tokens + to_slot[i]) * kRow + c * (kRow / 16)) = v[i];
    if constexpr (FMT != kCacheBf16) {
      if (c == 0) {
        *reinterpret_cast<uint32_t *>(to[i] + 2 * tokens * kRow + 4 * to_slot[i]) = ks[i];
        *reinterpret_cast<uint32_t *>(to[i] + 2 * tokens * kRow + 4 * (tokens + to_slot[i])) = vs[i];
      }
    }
  }
}

}  // namespace

hipError_t launch_cache_append(const CacheAppendArgs &p, int fmt, hipStream_t s) {
  if (fmt == kCacheBf16) return append<kCacheBf16>(p, s);
  if (fmt == kCacheMx8) return append<kCacheMx8>(p, s);
  return append<kCacheMx4>(p, s);
}

hipError_t launch_cache_keep(const CacheKeepArgs &p, int fmt, hipStream_t s) {
  const dim3 grid(p.B, p.Hkv);
  if (fmt == kCacheBf16)
    hipLaunchKernelGGL(cache_keep_kernel<kCacheBf16>, grid, dim3(kThreads), 0, s, p);
  else if (fmt == kCacheMx8)
    hipLaunchKernelGGL(cache_keep_kernel<kCacheMx8>, grid, dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL(cache_keep_kernel<kCacheMx4>, grid, dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace ss
