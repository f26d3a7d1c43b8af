// What the paged cache's attention kernels share: how the work is cut into shares,
// which tokens a row sees, a row's end, and the merge of the pieces' states.
#pragma once
#include "ss_cache_device.h"

#include <type_traits>

namespace ss {
namespace {

constexpr float kSlack = 8.f;                       // log2 by which weights may pass 1
constexpr int kMinShare = 4;                        // units: 300 tokens 7.5 us, with 8 and 12 units 7.9 and 10.4

// What the rows of a request see (SeenArgs).  With a window no row sees the tokens
// between the sinks and the first row's window: of the request's tiles the first
// `sinks` and those behind them and the gap are attended.
template <typename Args>
constexpr bool kSeen = std::is_base_of_v<CacheSeenArgs, Args>;
// Tokens of a tile, and rows of one KV head that a piece holds at most.
template <typename Args>
constexpr int kTileOf = std::is_same_v<Args, CacheGroupArgs> ? kCacheGroupTile : kCacheTile;
template <typename Args>
constexpr int kBlockOf = std::is_same_v<Args, CacheGroupArgs> ? kCacheGroupBlock : kCacheMaxRows;
struct Sight {
  int sinks, gap;
};
template <typename Args>
__device__ __forceinline__ Sight sight_of(const Args &p, int rows, int end, int len) {
  Sight s = {0, 0};
  if constexpr (kSeen<Args>) {
    if (p.window > 0) {
      constexpr int kTile = kTileOf<Args>;
      const int all = (len + kTile - 1) / kTile;
      const int64_t low = (int64_t)end - rows - p.window;      // below every row's window (a row of a tree that sees no node stands before it)
      const int from = low <= 0 ? 0 : low >= len ? all : (int)low / kTile;
      s.sinks = ((p.sinks < len ? p.sinks : len) + kTile - 1) / kTile;
      s.gap = from > s.sinks ? from - s.sinks : 0;
    }
  }
  return s;
}
// Blocks that a request's rows of one KV head are attended in.
template <typename Args>
__device__ __forceinline__ int row_blocks(const Args &p, int rows) {
  if constexpr (std::is_same_v<Args, CacheGroupArgs>) return (rows * p.G + kCacheGroupBlock - 1) / kCacheGroupBlock;
  return 1;
}
// Rows of a piece's state.
template <typename Args>
__device__ __forceinline__ int part_rows(const Args &p) {
  return p.M < kBlockOf<Args> ? p.M : kBlockOf<Args>;
}

// A request as the attention needs it; in a window, lane i holds request base + i.
struct Request {
  int rows;      // n_b: 0 if there are more than max_rows or fewer than none
  int row0;      // its first row
  int end;       // as given: positions count from it
  int len;       // tokens that its table reaches
  int tiles;
  int units;     // what the shares count: the tiles and the cost of a piece
};
template <typename Args>
__device__ __forceinline__ Request request_at(const Args &p, int b) {
  Request r;
  const int c = b < p.B ? b : p.B - 1;     // loads without a branch, so that several calls' overlap
  r.end = p.end[c];
  if (p.row_start == nullptr) {
    r.row0 = c * p.max_rows;
    r.rows = p.max_rows;
  } else {
    const int first = p.row_start[c], behind = p.row_start[c + 1];
    r.row0 = first;
    r.rows = behind >= first && (int64_t)behind - first <= p.max_rows ? behind - first : 0;
  }
  r.rows = b < p.B ? r.rows : 0;
  r.len = r.end < 0 ? 0 : r.end > p.capacity ? p.capacity : r.end;
  r.tiles = r.rows == 0 ? 0 : (r.len + kTileOf<Args> - 1) / kTileOf<Args>;
  if constexpr (kSeen<Args>) r.tiles = r.rows == 0 ? 0 : r.tiles - sight_of(p, r.rows, r.end, r.len).gap;
  r.units = r.tiles == 0 ? 0 : row_blocks(p, r.rows) * (r.tiles + p.piece_units);
  return r;
}

// Which tokens a row sees: those before the request's rows, from `low` on or below
// `sinks`, and of its n last tokens, from `first` on, those whose bit is set.
struct Seen {
  uint64_t bits;
  int64_t first;      // position of the request's first row
  int low, sinks;     // no window: 0, 0
  int len;
  int all_from, all_to;     // between these every row sees every token
  __device__ __forceinline__ bool whole(int tok) const {
    return tok + kCacheTile <= all_to && (tok >= all_from || tok + kCacheTile <= sinks);
  }
  static __device__ __forceinline__ uint32_t below(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }
  __device__ __forceinline__ uint32_t word(int tok) const {
    const int64_t far = tok - first;
    const int rel = far > 64 ? 64 : far < -32 ? -32 : (int)far;
    const uint32_t before = below(-rel) & (~below(low - tok) | below(sinks - tok));
    const uint32_t tree = rel >= 64 ? 0u : rel >= 0 ? (uint32_t)(bits >> rel) : (uint32_t)(bits << -rel);
    return (before | tree) & below(len - tok);
  }
};
// Of row i of a request's n, the row0 + i-th of the call.
__device__ __forceinline__ Seen seen_by(const CacheSeenArgs &p, int n, int row0, int end, int len, int i) {
  const int64_t row = (int64_t)row0 + i;
  Seen s;
  s.first = (int64_t)end - n;
  s.len = len;
  s.sinks = p.sinks;
  uint64_t bits = i < n && row >= 0 && row < p.num_rows ? p.tree != nullptr ? p.tree[row] : (2ull << i) - 1 : 0;
  bits &= n >= 64 ? ~0ull : (1ull << n) - 1;
  const auto clamp = [](int64_t x) { return x < 0 ? 0 : x > 0x7fffffff ? 0x7fffffff : (int)x; };
  const int64_t low = s.first + __popcll(bits) - p.window;      // the row's position is first + its nodes - 1
  s.low = p.window > 0 ? clamp(low) : 0;
  if (p.tree == nullptr && p.window > 0) {      // a chain's window may reach into it; a tree's word says all
    const int hides = clamp(s.low - s.first), sink = clamp(s.sinks - s.first);
    const uint64_t sinks = sink >= 64 ? ~0ull : (1ull << sink) - 1;
    bits &= (hides >= 64 ? 0ull : ~0ull << hides) | sinks;
  }
  s.bits = bits;
  const int to = clamp(s.first);
  s.all_to = to < len ? to : len;
  s.all_from = p.window > 0 ? clamp(s.first + n - p.window) : 0;
  return s;
}

// What a worker of a call that is cut into parts attends: part `part` of its (request, KV head, block of rows).
struct Whole {
  int b, h, block, part;
  // of the request's units: the first one, and how many (none where no tile is left)
  __device__ __forceinline__ void units(const CacheSeenArgs &p, int tiles, int &skip, int &left) const {
    const int each = (int)((uint32_t)(tiles + p.parts - 1) / (uint32_t)p.parts), from = part * each;
    const int there = tiles - from < each ? tiles - from : each;
    skip = block * (tiles + p.piece_units) + (part == 0 ? 0 : p.piece_units + from);
    left = there <= 0 ? 0 : there + (part == 0 ? p.piece_units : 0);
  }
};
__device__ __forceinline__ Whole whole_of(const CacheSeenArgs &p, int worker) {
  const int whole = (int)((uint32_t)worker / (uint32_t)p.parts);
  const int pair = (int)((uint32_t)whole / (uint32_t)p.B), block = (int)((uint32_t)pair / (uint32_t)p.Hkv);
  return {whole - pair * p.B, pair - block * p.Hkv, block, worker - whole * p.parts};
}
// x as a value that the compiler has not seen: of the thread's index, so that it
// does not keep every address of a piece, a tile and a merge in a register of
// its own all the way.
__device__ __forceinline__ int hidden(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Inclusive prefix sum over the wave's lanes.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast:31 into rows 2 and 3
  return x;
}
__device__ __forceinline__ int lane_of(int x, int i) { return __builtin_amdgcn_readlane(x, i); }

__device__ __forceinline__ int share_of(int total, int wgs) {
  const int s = (int)(((uint32_t)total + (uint32_t)wgs - 1) / (uint32_t)wgs);
  return s < kMinShare ? kMinShare : s;
}

// The result of one row: (m, l) of its state in the log2 domain, a / l and what came before it.
struct RowEnd {
  float inv, lse, own, prev;   // 1 / l; of all; weights of this and of the earlier part
  bool counts, before;         // whether this and the earlier part count: all do whose lse is not -inf, NaN among them
                               // (no token, or every score -inf, leaves l = 0)
};
__device__ __forceinline__ RowEnd row_end(const CacheAttendArgs &p, int64_t row, float m, float l) {
  RowEnd r;
  r.counts = l != 0.f;
  r.inv = r.counts ? 1.f / l : 0.f;
  r.lse = r.counts ? __builtin_fmaf(m, 0.69314718055994531f, logf(l)) : kNegInf;
  r.own = r.prev = 1.f;
  r.before = false;
  if (p.prev_lse != nullptr) {
    const float q = p.prev_lse[row];
    r.before = q != kNegInf;
    if (!r.counts) {
      r.lse = q;
    } else if (r.before) {
      const float top = fmaxf(q, r.lse);         // of a number and a NaN the number: the NaN's weight is one
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
  // a part that does not count may have any values; one whose weight underflows still brings a NaN
  if (!r.counts) v = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (r.before) v += r.prev * *reinterpret_cast<const f32x4_t *>(p.prev_out + at);
  return v;
}

// The rows of a block of a request without tokens, by the workgroup.
template <typename Args>
__device__ __forceinline__ void write_empty(const Args &p, int rows, int row0, const Whole &at) {
  const int first = kBlockOf<Args> * at.block, behind = rows * p.G < first + kBlockOf<Args> ? rows * p.G : first + kBlockOf<Args>;
  for (int j = threadIdx.x; j < (behind - first) * (kCacheDim / 4); j += kThreads) {
    const int r = first + j / (kCacheDim / 4), c = j % (kCacheDim / 4), i = (int)((uint32_t)r * p.g_inv >> 16);
    const int64_t row = (int64_t)row0 + i;
    if (row < 0 || row >= p.num_rows) continue;
    const int64_t o = row * p.Hq + at.h * p.G + r - i * p.G;
    const RowEnd end = row_end(p, o, kNegInf, 0.f);
    *reinterpret_cast<f32x4_t *>(p.out + o * kCacheDim + 4 * c) = row_value(p, end, o * kCacheDim + 4 * c, f32x4_t{0.f, 0.f, 0.f, 0.f});
    if (c == 0 && p.lse != nullptr) p.lse[o] = end.lse;
  }
}

// Staged V: 16-byte chunk c of row t lies at c ^ swizzle(t), so that neither the
// rows' stores (whole rows of 16, 2 x 8 or 4 x 4 chunks) nor the transpose reads
// (8 rows of two chunks, or 4 rows of four) meet in a bank.
template <int FMT, int NR>
__device__ __forceinline__ int swizzle(int t) {
  if constexpr (NR == 32) return FMT == kCacheBf16 ? 4 * (t & 3) + 2 * ((t >> 2) & 1) : 5 * (t & 3);
  return 2 * (t & 7) ^ (FMT == kCacheMx8 ? t & 1 : FMT == kCacheMx4 ? (t >> 1) & 1 : 0);
}

// p0, p1 as pairs of bf16 whose sum they are: the 24 bits of a fraction in three cuts of eight.
__device__ __forceinline__ void cut3(float p0, float p1, uint32_t &a, uint32_t &b, uint32_t &c) {
  const uint32_t w0 = __float_as_uint(p0), w1 = __float_as_uint(p1);
  a = __builtin_amdgcn_perm(w1, w0, 0x07060302u);                     // the high halves
  const float r0 = p0 - __uint_as_float(w0 & 0xffff0000u), r1 = p1 - __uint_as_float(w1 & 0xffff0000u);
  const uint32_t x0 = __float_as_uint(r0), x1 = __float_as_uint(r1);
  b = __builtin_amdgcn_perm(x1, x0, 0x07060302u);
  const float s0 = r0 - __uint_as_float(x0 & 0xffff0000u), s1 = r1 - __uint_as_float(x1 & 0xffff0000u);
  c = __builtin_amdgcn_perm(__float_as_uint(s1), __float_as_uint(s0), 0x07060302u);
}

// ---------------------------------------------------------------------------
// Merge the pieces' states of each (request, KV head) that more than one worker
// attended, and write the rows of requests without tokens.  A half wave holds a
// row's 128 channels; SPLIT half waves of the workgroup share a row's states (32 or
// 8 where a pair may have that many: 32768 tokens with 4 heads, 128 states a pair,
// 8.8 us with 8 and 6.3 with 32), else each takes a row of its own.
// ---------------------------------------------------------------------------
template <int SPLIT>
__global__ __launch_bounds__(SPLIT > 8 ? 32 * SPLIT : kThreads) void cache_join_kernel(CacheAttendArgs p) {
  constexpr int kHalves = SPLIT > 8 ? SPLIT : 8, kRowsPer = kHalves / SPLIT;
  const int tx = threadIdx.x, lane = tx & 31;
  const int part = (tx >> 5) % SPLIT;
  const int b = blockIdx.x;
  const int item = blockIdx.y * kRowsPer + (tx >> 5) / SPLIT;     // of the request's heads and rows
  const int h = item / p.M, r = item - h * p.M;
  // units (tiles and pieces' cost) of the requests before b, and of all, by every wave
  int before = 0, all = 0;
  for (int j = tx & 63; j < p.B; j += 64) {
    const int t = request_at(p, j).units;
    all += t;
    before += j < b ? t : 0;
  }
  before = lane_of(wave_scan(before), 63);
  all = lane_of(wave_scan(all), 63);
  const Request q = request_at(p, b);
  const int i = (int)((uint32_t)r * p.g_inv >> 16);
  bool mine = h < p.Hkv && r < q.rows * p.G && q.row0 + i >= 0 && q.row0 + i < p.num_rows;
  const int64_t row = ((int64_t)q.row0 + i) * p.Hq + h * p.G + r - i * p.G;
  float m = kNegInf, l = 0.f;
  f32x4_t a = {0.f, 0.f, 0.f, 0.f};
  if (q.tiles > 0) {
    const int share = share_of(all * p.Hkv, p.workers);
    const int start = h * all + before;
    const int w0 = (int)((uint32_t)(start + p.piece_units) / (uint32_t)share), w1 = (int)((uint32_t)(start + q.units - 1) / (uint32_t)share);
    mine &= w0 != w1;               // else one worker attended all of it
    if (mine) {
      constexpr int kAhead = SPLIT > 8 ? 4 : 8;     // states in flight
      for (int w = w0 + part; w <= w1; w += kAhead * SPLIT) {
        f32x2_t ml[kAhead];
        f32x4_t x[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int v = w + j * SPLIT <= w1 ? w + j * SPLIT : w1;
          const int64_t o = (int64_t)(2 * v + (v == w0 ? 1 : 0)) * p.M + r;
          ml[j] = *reinterpret_cast<const f32x2_t *>(p.part_ml + 2 * o);
          x[j] = *reinterpret_cast<const f32x4_t *>(p.part_a + o * kCacheDim + 4 * lane);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          if (w + j * SPLIT > w1) break;
          const float mn = fmaxf(m, ml[j][0]);
          const float fa = mn == kNegInf ? 1.f : exp2_fast(m - mn), fb = mn == kNegInf ? 1.f : exp2_fast(ml[j][0] - mn);
          a = fa * a + fb * x[j];
          l = fa * l + fb * ml[j][1];
          m = mn;
        }
      }
    }
  }
  if constexpr (SPLIT > 1) {
    __shared__ __attribute__((aligned(16))) float sa[kHalves][kCacheDim];
    __shared__ float sm[kHalves], sl[kHalves];
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
#pragma unroll 8
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

// The same for rows that see a tree or a window, which may be many more, in blocks: a workgroup goes over the request's own
// heads and rows, gridDim.y workgroups a request (24 requests of 6 to 384 rows on 8 heads: a workgroup for every eight that there
// may be 14.6 us, gone over 12.2).
template <int SPLIT, typename Args>
__global__ __launch_bounds__(SPLIT > 8 ? 32 * SPLIT : kThreads) void cache_join_seen_kernel(Args p) {
  constexpr int kHalves = SPLIT > 8 ? SPLIT : 8, kRowsPer = kHalves / SPLIT;
  __shared__ __attribute__((aligned(16))) float sa[SPLIT > 1 ? kHalves : 1][kCacheDim];
  __shared__ float sm[kHalves], sl[kHalves];
  const int tx = threadIdx.x, lane = tx & 31;
  const int part = (tx >> 5) % SPLIT;
  const int b = blockIdx.x;
  int before = 0, all = 0;
  for (int j = p.parts > 0 ? p.B : tx & 63; j < p.B; j += 64) {
    const int t = request_at(p, j).units;
    all += t;
    before += j < b ? t : 0;
  }
  const Request q = request_at(p, b);
  before = lane_of(wave_scan(before), 63);
  all = lane_of(wave_scan(all), 63);
  const int share = share_of(all * p.Hkv, p.workers), units = q.tiles + p.piece_units;
  const int rows = q.rows * p.G;
  for (int first = blockIdx.y * kRowsPer; first < p.Hkv * rows; first += gridDim.y * kRowsPer) {
    const int item = first + (tx >> 5) / SPLIT;
    const int h = (int)((uint32_t)item / (uint32_t)rows), r = item - h * rows;
    const int i = (int)((uint32_t)r * p.g_inv >> 16), block = r / kBlockOf<Args>;
    bool mine = h < p.Hkv && q.row0 + i >= 0 && q.row0 + i < p.num_rows;
    const int64_t row = ((int64_t)q.row0 + i) * p.Hq + h * p.G + r - i * p.G;
    float m = kNegInf, l = 0.f;
    f32x4_t a = {0.f, 0.f, 0.f, 0.f};
    if (q.tiles > 0) {
      int w0, w1;
      if (p.parts > 0) {
        const int each = (int)((uint32_t)(q.tiles + p.parts - 1) / (uint32_t)p.parts);
        w0 = ((block * p.Hkv + h) * p.B + b) * p.parts;
        w1 = w0 + (int)((uint32_t)(q.tiles - 1) / (uint32_t)each);
      } else {
        const int start = h * all + before + block * units;
        w0 = (int)((uint32_t)(start + p.piece_units) / (uint32_t)share);
        w1 = (int)((uint32_t)(start + units - 1) / (uint32_t)share);
      }
      mine &= w0 != w1;               // else one worker attended all of it
      if (mine) {
        constexpr int kAhead = 4;     // states in flight
        for (int w = w0 + part; w <= w1; w += kAhead * SPLIT) {
          f32x2_t ml[kAhead];
          f32x4_t x[kAhead];
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
            const int v = w + j * SPLIT <= w1 ? w + j * SPLIT : w1;
            const int64_t o = (int64_t)(2 * v + (v == w0 ? 1 : 0)) * part_rows(p) + r - block * kBlockOf<Args>;
            ml[j] = *reinterpret_cast<const f32x2_t *>(p.part_ml + 2 * o);
            x[j] = *reinterpret_cast<const f32x4_t *>(p.part_a + o * kCacheDim + 4 * lane);
          }
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
            if (w + j * SPLIT > w1) break;
            const float mn = fmaxf(m, ml[j][0]);
            const float fa = mn == kNegInf ? 1.f : exp2_fast(m - mn), fb = mn == kNegInf ? 1.f : exp2_fast(ml[j][0] - mn);
            a = fa * a + fb * x[j];
            l = fa * l + fb * ml[j][1];
            m = mn;
          }
        }
      }
    }
    if constexpr (SPLIT > 1) {
      __syncthreads();
      *reinterpret_cast<f32x4_t *>(&sa[tx >> 5][4 * lane]) = a;
      if (lane == 0) {
        sm[tx >> 5] = m;
        sl[tx >> 5] = l;
      }
      __syncthreads();
      if (part != 0) continue;
      float top = kNegInf;
#pragma unroll
      for (int j = 0; j < SPLIT; ++j) top = fmaxf(top, sm[(tx >> 5) + j]);
      a = f32x4_t{0.f, 0.f, 0.f, 0.f};
      l = 0.f;
#pragma unroll 8
      for (int j = 0; j < SPLIT; ++j) {
        const float f = top == kNegInf ? 1.f : exp2_fast(sm[(tx >> 5) + j] - top);
        l += f * sl[(tx >> 5) + j];
        a += f * *reinterpret_cast<const f32x4_t *>(&sa[(tx >> 5) + j][4 * lane]);
      }
      m = top;
    }
    if (!mine) continue;
    const RowEnd end = row_end(p, row, m, l);
    const int64_t o = row * kCacheDim + 4 * lane;
    *reinterpret_cast<f32x4_t *>(p.out + o) = row_value(p, end, o, a);
    if (lane == 0 && p.lse != nullptr) p.lse[row] = end.lse;
  }
}

// Merge what an attention over p left: 32 or 8 half waves a row where a (request, KV head, block of rows) may have that many states.
template <typename Args>
hipError_t launch_join(const Args &p, hipStream_t s) {
  if constexpr (kSeen<Args>) {
    const int64_t pairs = (int64_t)p.B * p.Hkv * ((p.M + kBlockOf<Args> - 1) / kBlockOf<Args>);
    // more threads than the chip holds at once only wait: one request, 2048 rows of 32 states 22.4 us with 32 half waves each, 9.0 with 8
    const bool few = (int64_t)p.B * p.Hkv * p.M <= 512;
    const auto groups = [&](int rows_per) {
      const int64_t most = ((int64_t)p.Hkv * p.M + rows_per - 1) / rows_per, some = 2048 / p.B;
      return dim3(p.B, (unsigned)(most < some ? most : some > 1 ? some : 1));
    };
    if (pairs * 32 <= p.workers && few)
      hipLaunchKernelGGL((cache_join_seen_kernel<32, Args>), groups(1), dim3(1024), 0, s, p);
    else if (pairs * 8 <= p.workers)
      hipLaunchKernelGGL((cache_join_seen_kernel<8, Args>), groups(1), dim3(kThreads), 0, s, p);
    else
      hipLaunchKernelGGL((cache_join_seen_kernel<1, Args>), groups(8), dim3(kThreads), 0, s, p);
  } else {
    const int64_t pairs = (int64_t)p.B * p.Hkv;
    if (pairs * 32 <= p.workers)
      hipLaunchKernelGGL((cache_join_kernel<32>), dim3(p.B, p.Hkv * p.M), dim3(1024), 0, s, p);
    else if (pairs * 8 <= p.workers)
      hipLaunchKernelGGL((cache_join_kernel<8>), dim3(p.B, p.Hkv * p.M), dim3(kThreads), 0, s, p);
    else
      hipLaunchKernelGGL((cache_join_kernel<1>), dim3(p.B, (p.Hkv * p.M + 7) / 8), dim3(kThreads), 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace
}  // namespace ss
