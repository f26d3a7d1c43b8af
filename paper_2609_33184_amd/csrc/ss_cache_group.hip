// gfx950 (MI355X) attention of many query rows per KV head over the paged cache:
// trees of drafted tokens.
//
// o = sum_t softmax(s)_t v_t over the tokens that a row sees, s_t = scale q k_t; one pass over the tiles with a
// running maximum and sum per row.  In cache_attend_kernel each wave brings, decodes
// and stages its own tiles for 32 rows; with more rows the decoding of K and V and the bytes are
// paid again and again.  Here a workgroup's four waves hold 128 rows of a KV head (32
// each; up to 64 rows: two waves for either half of the tiles) and share each
// tile of 32 tokens: it is decoded once into LDS, 16 bits a value, K in the rows' order and V
// for its transpose read, four tiles deep, with one barrier a tile.  More than 128 rows are attended
// in blocks of 128, each of which reads K and V again (16 x 12000..16384 tokens, 256 rows: 1.8 GB of 0.9).  The work is
// cut as in cache_attend_kernel.
//
// Per wave and tile: 8 v_mfma_f32_32x32x16 for S^T = K Q^T of the next tile, beside this tile's
// softmax, and 16 (V in 8 or 4 bits) or 24 (bf16) for O^T += V^T P^T, interleaved with
// the vector work by hand.
//
// Precision.  bf16: P in three parts of bf16, exact, as in cache_attend_kernel.  8 and 4 bits: V's code times
// scale times 2^6 or 2^2 is an exact f16 number while the scale lies in [2^-21, 2] (e4m3) or
// [2^-25, 2^11] (e2m1), and P, at most 2^3 and times 2^12, is cut into two f16 numbers, 22 bits or all but 2^-25 of it: a
// third less matrix work than three parts (16 x 32768 tokens, 96 rows: 550 us, in three parts 707
// by waves for themselves).  The running maximum is followed closer for it, from 2^3 on instead of 2^8.  Each weight is held to
// 2^-18 of itself: where a row sees one below 2^-19 of the largest, the wave attends the tile in two or three steps, each over a
// range of weights and with a reference 2^20 or 2^40 lower, where it stays while the tiles go on so.  Left in one range, thousands of
// weights of 2^-37 before large values would be lost, 1.5e-3 of a result where the values are 2^16 times the largest weight's.
// A tile with other
// scales, or values that are no numbers, is attended token by token in fp32.  Against 64 bits 9e-7, the plain form in fp32 3.2e-6.
//
// bf16 rows go from memory to LDS without passing registers.  What a wave needs next is waited for by
// count, so that the loads behind it stay in flight.
//
// What bounds it.  bf16, 16 x 12000..16384 tokens, 256 rows: 520 us; the SIMDs issue vector work 45% and
// matrix work 47% of the cycles, one after the other, at 1.65 GHz; the matrix work alone would take 185 us of the formula and
// twice that in three parts.  8 bits, 16 x 32768 tokens, 96 rows: 530 us, 155 for the bytes; vector work 37%,
// matrix work 31% on three SIMDs of four (96 rows leave a wave without), the rest waits at the barrier and for LDS.  One
// request of 32768 tokens, 256 rows: 92 us and 10.5 for the join of its 32 states a row.
#include <hip/hip_runtime.h>

#include "ss_cache.h"
#include "ss_cache_attend.h"

namespace ss {
namespace {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

constexpr int kTokens = kCacheGroupTile;        // of a tile
constexpr int kRows = 32;                       // of a wave
constexpr int kTileBytes = kTokens * 256;       // K or V of a tile, 16 bits a value
constexpr int kBuffers = 4;                     // tiles in LDS
constexpr int kSteps = kCacheDim / 16;          // of a product over the channels
constexpr int kAccs = kCacheDim / 32;           // accumulators of 32 channels

// What a piece costs beside its tiles, in tiles: 24 ragged requests with 4, 8 and 16 52.7, 53.4 and 63.6 us.
constexpr int kPieceGroupTiles = 8;

// Half precision for P and V.  V's values times 2^kVShift are exact numbers of it if
// their blocks' scale bytes lie in [kLeast, kMost]: blocks of e4m3 whose largest value lies between 2^-13 and 896, and of e2m1
// between 2^-23 and 12288.  P's maximum is 2^kPShift times 2^kHalfSlack.
constexpr int kPShift = 12;
constexpr float kHalfSlack = 3.f;
// log2 of the least weight, of the largest, that two parts hold well: they leave 2^-25 of P, so 2^-18 of it.  And by how much the
// reference is lowered for smaller ones: once, or twice, which does for weights of 2^-59.
constexpr float kHalfLeast = -19.f;
constexpr int kHalfStep = 20;
template <int FMT>
struct Half {
  // least and largest magnitude of a code but 0: 2^-9 and 448, 1/2 and 6; of an f16 number 2^-24 and 65504
  static constexpr int kVShift = FMT == kCacheMx8 ? 6 : 2;
  static constexpr uint32_t kLeast = 127 - (FMT == kCacheMx8 ? 15 : 23) - kVShift, kMost = 127 + (FMT == kCacheMx8 ? 7 : 13) - kVShift;
};

// Scale bytes beyond which V's sums might pass the largest number with these factors: from such a tile on a piece goes without.
// Below, 2^21 tokens' sums are below 2^(15 + 6 + 9 + 20 + 21), and 2^40 times that while small weights are added.
constexpr uint32_t kHuge = 127 + 20;

template <int I>
using Int = std::integral_constant<int, I>;

// Values 2 I and 2 I + 1 of a dword, times scale, as f16.
template <int FMT, int I>
__device__ __forceinline__ uint32_t half_of(uint32_t w, float scale) {
  if constexpr (FMT == kCacheMx8)
    return __builtin_bit_cast(uint32_t, (f16x2_t)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, I != 0));
  else
    return __builtin_bit_cast(uint32_t, (f16x2_t)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, I));
}

// p0, p1 as pairs of f16 whose sums they are, to 22 bits or 2^-25.
__device__ __forceinline__ void cut2(float p0, float p1, uint32_t &a, uint32_t &b) {
  const f16x2_t h = __builtin_convertvector(f32x2_t{p0, p1}, f16x2_t);
  a = __builtin_bit_cast(uint32_t, h);
  float r0, r1;      // p - h, h's halves widened on the way
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r0) : "v"(a), "v"(p0));
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r1) : "v"(a), "v"(p1));
  const f16x2_t l = __builtin_convertvector((f32x2_t{r0, r1}), f16x2_t);
  b = __builtin_bit_cast(uint32_t, l);
}

// A wave's 64 x 16 bytes, at `from` + its lanes' offsets, straight into LDS, lane by lane from `to` on (a byte address there,
// the wave's).  In assembly, since with the builtin every read of LDS waits for all of them; it has no output register,
// and what reads the bytes is behind a wait and a barrier.  The compiler keeps no distances inside assembly: the load needs one
// wait state behind M0's write, and five behind a vector instruction that may have written its scalar address.
__device__ __forceinline__ void load_to_lds(const uint8_t *from, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(from) : "memory", "m0");
}

__device__ __forceinline__ void workgroup_barrier() {      // of what lies in LDS; loads to registers go on
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// A piece: tiles t0 .. t0 + tiles - 1 of a request's `whole`, for head h and a block of rows.  tiles = 0: none.
struct Piece {
  int b, rows, row0, end, len, whole, h, t0, tiles, block;
  Sight sight;
};
__device__ __forceinline__ int token_of(const Piece &q, int k) {       // first one of the piece's k-th tile
  const int t = q.t0 + k;
  return (t < q.sight.sinks ? t : t + q.sight.gap) * kTokens;
}

template <int FMT>
__global__ __launch_bounds__(kThreads, 2) void cache_attend_group_kernel(CacheGroupArgs p) {
  constexpr int kRow = cache_row_bytes(FMT);
  constexpr bool kHalf = FMT != kCacheBf16;                // P and V in half precision, where V fits
  constexpr bool kDirect = FMT == kCacheBf16;              // rows go to LDS as they are
  constexpr int kLanes = kRow / 16;                        // lanes of a stored row
  __shared__ __attribute__((aligned(256))) unsigned char smem[kBuffers][2][kTileBytes];     // tiles' K, V
  __shared__ float merge_m[2][64], merge_l[2][64];
  __shared__ int wide[kBuffers], huge[kBuffers];           // the tile's number if some of its V is beyond half precision, or beyond kHuge
  __shared__ int spoilt[kBuffers];                         // its number if some is no number at tokens that not all rows see:
  __shared__ __attribute__((aligned(16))) uint8_t no_number[kBuffers][kTokens][kCacheDim / 8];      // which, a bit each
  __shared__ Request window[kWaves][64];                   // requests base .. base + 63, each wave its own copy: the registers are full
  __shared__ Piece ring[kWaves][8];                        // the pieces on their way
  const int thread = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(thread >> 6);
  const int worker = blockIdx.x;
  auto one = [](int x) { return __builtin_amdgcn_readfirstlane(x); };

  // This worker's share and where it starts, as in cache_attend_kernel.
  int base = 0, idx, skip, h, left;
  if (p.parts > 0) {
    const Whole at = whole_of(p, worker);
    base = at.b & ~63;
    idx = at.b & 63;
    h = at.h;
    const Request win = request_at(p, base + (thread & 63));
    at.units(p, lane_of(win.tiles, idx), skip, left);
    if (lane_of(win.tiles, idx) == 0 && p.parts == 1) write_empty(p, lane_of(win.rows, idx), lane_of(win.row0, idx), at);
    if (left == 0 || skip >= lane_of(win.units, idx)) return;      // without tokens, or fewer rows
    window[w][thread & 63] = win;
  } else {
    Request win;
    const int lane = thread & 63;
    const int chunks = (p.B + 63) / 64;
    int before = 0, scan, all;
    if (chunks == 1) {
      win = request_at(p, lane);
      scan = wave_scan(win.units);
      all = lane_of(scan, 63);
    } else {
      int sums = 0;
      for (int j = 0; j < chunks; ++j) {
        const int sum = lane_of(wave_scan(request_at(p, 64 * j + lane).units), 63);
        sums = lane == j ? sum : sums;
      }
      scan = wave_scan(sums);
      all = lane_of(scan, 63);
    }
    const int total = all * p.Hkv;
    const int share = share_of(total, p.workers);
    const int64_t first = (int64_t)worker * share;
    if (first >= total) return;
    left = total - (int)first < share ? total - (int)first : share;
    h = (int)((uint32_t)first / (uint32_t)all);
    const int at = (int)first - h * all;
    if (chunks > 1) {
      const int owner = __builtin_popcountll(__builtin_amdgcn_ballot_w64(scan <= at));
      before = owner == 0 ? 0 : lane_of(scan, owner - 1);
      base = 64 * owner;
      win = request_at(p, base + lane);
      scan = before + wave_scan(win.units);
    }
    idx = __builtin_popcountll(__builtin_amdgcn_ballot_w64(scan <= at));
    skip = at - (idx == 0 ? before : lane_of(scan, idx - 1));
    window[w][lane] = win;
  }
  const int page_tokens = 1 << p.page_shift;
  const uint32_t v_off = (uint32_t)(page_tokens * kRow), ks_off = 2 * v_off, vs_off = ks_off + 4u * (uint32_t)page_tokens;

  auto uniform = [&](const Piece &q) {     // the wave's, in scalar registers
    return Piece{one(q.b), one(q.rows), one(q.row0), one(q.end), one(q.len), one(q.whole), one(q.h), one(q.t0), one(q.tiles), one(q.block),
                 {one(q.sight.sinks), one(q.sight.gap)}};
  };
  auto next_piece = [&]() {
    Piece q = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, {0, 0}};
    while (left > 0) {
      const int lane = hidden(thread & 63);
      const uint64_t more = idx < 64 ? __builtin_amdgcn_ballot_w64(window[w][lane].units > 0) & (~0ull << idx) : 0;
      if (more == 0) {
        base += 64;
        idx = 0;
        if (base >= p.B) {
          base = 0;
          if (++h >= p.Hkv) left = 0;     // not reached while nobody changes the lengths under a call
        }
        window[w][lane] = request_at(p, base + lane);
        continue;
      }
      idx = __builtin_ctzll(more);
      const Request &r = window[w][idx];
      const int units = one(r.units), cost = p.piece_units, per = one(r.tiles) + cost;
      const int block = units > per ? skip / per : 0, off = skip - block * per;
      const int take = per - off < left ? per - off : left;
      const int t0 = off > cost ? off - cost : 0, t1 = off + take > cost ? off + take - cost : 0;
      const int b = base + idx;
      left -= take;
      skip += take;
      if (skip >= units) {
        skip = 0;
        ++idx;
      }
      if (t1 > t0) {
        q = Piece{b, one(r.rows), one(r.row0), one(r.end), one(r.len), one(r.tiles), h, t0, t1 - t0, block, {0, 0}};
        q.sight = sight_of(p, q.rows, q.end, q.len);
        break;
      }
    }
    left = one(left);
    idx = one(idx);
    base = one(base);
    skip = one(skip);
    h = one(h);
    return uniform(q);
  };
  // Pages of the 32 tiles from the piece's k-th on, lanes 2 j and 2 j + 1 those of the j-th's runs of 16; -1 for what is none.
  auto pages_of = [&](const Piece &q, int k) {
    const int lane = hidden(thread & 63), j = k + (lane >> 1);
    const int64_t tok = (int64_t)token_of(q, j) + 16 * (lane & 1);
    int id = -1;
    if (j < q.tiles && tok < q.len) id = p.table[(int64_t)q.b * p.table_stride + (tok >> p.page_shift)];
    return id >= 0 && id < p.num_pages ? id : -1;
  };

  // The loads.  A run of 16 tokens lies in one page, of which every slot may be read; what is behind the request's tokens,
  // or stands in for a page that is none, is masked, and its V replaced by zeros, when the tile is staged or attended.
  Piece lp;                            // of the next tile to load
  int lk = 0, lplace = 0, issued = 0;  // which one of it; its place in the ring; tiles so far
  uint64_t head = 0;                   // its KV head in page 0
  int ids = -1, ids_next = -1;         // pages of the piece's tiles lk & ~31 .. and the 32 behind them
  uint32_t holes = 0;                  // two bits a tile, eight tiles: its runs without a page
  u32x4_t kr[2], vr[2];                // two tiles on their way, by parity of their number (4 bits: K in half of the lanes, V in the others)
  uint32_t ks[2], vs[2];
  uint64_t gone[2] = {0, 0};           // lanes whose row is no token
  auto enter = [&]() {                 // the next piece to load
    lp = next_piece();
    lk = 0;
    if (lp.tiles == 0) return;
    lplace = (lplace + 1) & 7;
    ring[w][lplace] = lp;
    ids = pages_of(lp, 0);
    ids_next = pages_of(lp, 32);
    head = (uint64_t)p.pages + (uint64_t)lp.h * p.head_bytes;
  };
  auto one64 = [&](uint64_t x) { return (uint64_t)(uint32_t)one((int)(x >> 32)) << 32 | (uint32_t)one((int)x); };
  // Issue the loads of the next tile, if there is one: into LDS, or into registers `set`.
  auto load = [&](auto parity) {
    constexpr int set = decltype(parity)::value;
    if (lk == lp.tiles) {            // none is left once there is no next piece
      if (lp.tiles != 0) enter();
      if (lp.tiles == 0) return;
    } else if (lk != 0 && (lk & 31) == 0) {
      ids = ids_next;
      ids_next = pages_of(lp, lk + 32);
    }
    lk = one(lk);
    const int tok = one(token_of(lp, lk)), len = one(lp.len);
    const uint32_t hole = (uint32_t)(__builtin_amdgcn_ballot_w64(ids < 0) >> (2 * (lk & 31))) & 3u;
    holes = (holes & ~(3u << 2 * (issued & 7))) | hole << 2 * (issued & 7);
    const uint64_t from = one64(head);
    // K rows of run `run`, from its first token on
    auto run_at = [&](int run) {
      const int page = lane_of(ids, 2 * (lk & 31) + run);
      return from + (uint64_t)(page < 0 ? 0 : page) * p.page_stride + (uint32_t)((tok + 16 * run) & (page_tokens - 1)) * kRow;
    };
    const int tx = hidden(thread);
    if constexpr (FMT == kCacheBf16) {
      const int c = tx & 15, r = tx >> 4;      // lane i brings chunk i of the row's 16 in LDS
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint64_t run = run_at(u);
        const uint32_t to = (uint32_t)(uintptr_t)smem[issued & (kBuffers - 1)][0] + (16 * u + 4 * w) * 256;
        load_to_lds((const uint8_t *)run, r * kRow + 16 * (c ^ r), one((int)to));
        load_to_lds((const uint8_t *)(run + v_off), r * kRow + 16 * (c ^ swizzle<FMT, 32>(r)), one((int)to + kTileBytes));
      }
    } else {
      const int mine = FMT == kCacheMx8 ? w >> 1 : w & 1;                       // the wave's run
      const int r = FMT == kCacheMx8 ? (tx >> 3) & 15 : (tx >> 2) & 15;
      const uint64_t run = run_at(mine);
      const uint64_t scales = run + ks_off - (uint32_t)((tok + 16 * mine) & (page_tokens - 1)) * (kRow - 4);
      gone[set] = tok + kTokens > len || hole != 0 ? __builtin_amdgcn_ballot_w64(tok + 16 * mine + r >= len || ((hole >> mine) & 1u) != 0) : 0;
      // said to be global: a load that might be of LDS is waited for at every barrier
      using Bytes = const __attribute__((address_space(1))) uint8_t *;
      auto rows = [&](uint64_t at) { return *(const __attribute__((address_space(1))) u32x4_t *)((Bytes)at + (uint32_t)(r * kRow + 16 * (tx % kLanes))); };
      auto scale = [&](uint64_t at) { return (uint32_t)*((Bytes)at + (uint32_t)(4 * r + tx % kLanes * 4 / kLanes)); };
      if constexpr (FMT == kCacheMx8) {
        kr[set] = rows(run);
        vr[set] = rows(run + v_off);
        ks[set] = scale(scales);
        vs[set] = scale(scales + (vs_off - ks_off));
      } else {
        kr[set] = rows(run + (w >= 2 ? v_off : 0));
        vs[set] = scale(scales + (w >= 2 ? vs_off - ks_off : 0));
      }
    }
    ++lk;
    ++issued;
  };
  // Where the lane's part of a tile goes in LDS; the other chunks of it lie a flip of bits away.
  const int own = FMT == kCacheMx8 ? thread >> 3 : (thread >> 2) & 31;      // its row
  const uint32_t k_to = own * 256 + 16 * ((thread % kLanes * (256 / kRow)) ^ (own & 15));
  const uint32_t v_to = kTileBytes + own * 256 + 16 * ((thread % kLanes * (256 / kRow)) ^ swizzle<FMT, 32>(own));
  auto put = [&](uint32_t at, u32x4_t y) { *(__attribute__((address_space(3))) u32x4_t *)(uintptr_t)at = y; };
  // The tile in the registers into LDS, its V in half precision or, `exact`, in bf16.
  auto stage = [&](auto parity, int number, bool exact) {
    constexpr int set = decltype(parity)::value;
    const uint32_t to = (uint32_t)(uintptr_t)smem[number & (kBuffers - 1)][0];
    if constexpr (FMT == kCacheMx8) {
      const float kf = scale_of(ks[set]), vf = scale_of(vs[set] + (exact ? 0 : Half<FMT>::kVShift));
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const u32x2_t a = widen8(kr[set][2 * j], kf), d = widen8(kr[set][2 * j + 1], kf);
        put(to + (k_to ^ (16 * j)), u32x4_t{a[0], a[1], d[0], d[1]});
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        u32x4_t y;
        if (exact) {
          const u32x2_t a = widen8(vr[set][2 * j], vf), d = widen8(vr[set][2 * j + 1], vf);
          y = u32x4_t{a[0], a[1], d[0], d[1]};
        } else {
          y = u32x4_t{half_of<FMT, 0>(vr[set][2 * j], vf), half_of<FMT, 1>(vr[set][2 * j], vf), half_of<FMT, 0>(vr[set][2 * j + 1], vf),
                      half_of<FMT, 1>(vr[set][2 * j + 1], vf)};
        }
        put(to + (v_to ^ (16 * j)), y);
      }
    } else if constexpr (FMT == kCacheMx4) {
      const bool half = w >= 2 && !exact;
      const float f = scale_of(vs[set] + (half ? Half<FMT>::kVShift : 0));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t x = kr[set][j];
        put(to + ((w >= 2 ? v_to : k_to) ^ (16 * j)),
            half ? u32x4_t{half_of<FMT, 0>(x, f), half_of<FMT, 1>(x, f), half_of<FMT, 2>(x, f), half_of<FMT, 3>(x, f)} : widen4(x, f));
      }
    }
  };
  // Whether the V in the registers is beyond half precision: told to the others, who see it behind a barrier.
  auto tell = [&](auto parity, int number) {
    constexpr int set = decltype(parity)::value;
    if (FMT == kCacheMx4 && w < 2) return;
    u32x4_t &y = FMT == kCacheMx8 ? vr[set] : kr[set];
    if (gone[set] != 0) {      // a weight of zero must meet no leftover NaN
      const bool none = (gone[set] >> hidden(thread & 63)) & 1u;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = none ? 0u : y[j];
      vs[set] = none ? 127 : vs[set];
    }
    bool beyond = vs[set] - Half<FMT>::kLeast > Half<FMT>::kMost - Half<FMT>::kLeast;
    if constexpr (FMT == kCacheMx8) {      // a value that is no number by itself, which the writes make none of
      uint32_t none = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) none |= (y[j] & 0x7f7f7f7fu) + 0x01010101u;
      beyond |= (none & 0x80808080u) != 0;
    }
    if (__builtin_amdgcn_ballot_w64(beyond) != 0) {
      const uint32_t any = (y[0] | y[1] | y[2] | y[3]) & (FMT == kCacheMx8 ? 0x7f7f7f7fu : 0x77777777u);      // zeros fit with any scale but NaN's
      if (beyond && (any != 0 || vs[set] == 255)) wide[number & (kBuffers - 1)] = number;
      if (vs[set] > kHuge && any != 0) huge[number & (kBuffers - 1)] = number;
    }
  };
  // In a tile in LDS that some rows see a part of, V's values that are no numbers become zeros: a weight of zero would
  // spread them.  Where they were is kept for the rows that see them.
  auto clear = [&](int number, int there, uint32_t hole) {      // there: tokens of the request from the tile's first on
    const int tx = hidden(thread), buf = number & (kBuffers - 1);
    bool any = false;
#pragma unroll 1
    for (int u = 0; u < kTokens / 16; ++u) {
      const int t = 16 * u + tx / 16, c = tx & 15;
      u32x4_t *at = reinterpret_cast<u32x4_t *>(smem[buf][1] + t * 256 + 16 * (c ^ swizzle<FMT, 32>(t)));
      u32x4_t y = *at;
      const bool none = t >= there || ((hole >> u) & 1u) != 0;
      uint32_t bad = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool lo = (y[e] & 0x7f80u) == 0x7f80u, hi = (y[e] & 0x7f800000u) == 0x7f800000u;
        bad |= ((lo ? 1u : 0u) | (hi ? 2u : 0u)) << (2 * e);
        y[e] = none ? 0u : y[e] & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u));
      }
      no_number[buf][t][c] = (uint8_t)bad;
      if (bad != 0 || none) *at = y;
      any |= bad != 0 && !none;
    }
    if (any) spoilt[buf] = number;
  };

  // Before tile i is attended, tiles i + 1 and i + 2 are in LDS; beside it tile i + 3 gets there, and i + 4 and i + 5 are on
  // their way to registers.
  enter();
  if (lp.tiles == 0) return;
  if (thread < kBuffers) wide[thread] = huge[thread] = spoilt[thread] = -1;
  workgroup_barrier();
  int exacts = kHalf ? 0 : -1;      // bit i % kBuffers: tile i's V is bf16; kBuffers bits on: beyond kHuge (what was told is gone by then)
  auto bring = [&](auto parity, int number) {      // tile `number` from registers into LDS, behind the barrier that follows its tell
    if (number < issued) {
      const bool exact = one(wide[number & (kBuffers - 1)]) == number;
      const bool far = exact && one(huge[number & (kBuffers - 1)]) == number;
      exacts = (exacts & ~((1 << kBuffers | 1) << (number & (kBuffers - 1)))) | (exact ? (far ? 1 << kBuffers | 1 : 1) << (number & (kBuffers - 1)) : 0);
      if (__builtin_expect(exact, 0))
        stage(parity, number, true);
      else
        stage(parity, number, false);
    }
    load(parity);
  };
  load(Int<0>{});
  load(Int<1>{});
  if constexpr (kDirect) {
    load(Int<0>{});
  } else {
    if (0 < issued) tell(Int<0>{}, 0);
    workgroup_barrier();
    bring(Int<0>{}, 0);
    if (1 < issued) tell(Int<1>{}, 1);
    workgroup_barrier();
    bring(Int<1>{}, 1);
    if (2 < issued) tell(Int<0>{}, 2);
    workgroup_barrier();
    bring(Int<0>{}, 2);
  }

  bf16x8_t qop[kSteps];
  uint64_t bits = 0;         // of the row's word
  int low = 0;               // its window's first token
  float m_run = kNegInf, l_run = 0.f;
  f32x16_t acc[kAccs], x = f32x16_t{};      // x: the scores of the tile that this wave attends next
  int M = 0, first_row = 0, groups = 1, mine = 0, turn = 0;      // rows of the block; of all, its first; waves per 32 rows; this wave's rows, its tiles
  bool works = false, plain = false;      // whether it has rows; its state goes without the factors of half precision
  // Half precision: how far m_run, log2 of what the weights are relative to, lies below the largest score, for the sake of
  // small weights (not if plain).
  int lift = 0;
  // S^T = K Q^T of a tile: K's rows read, and multiplied.
  auto read_k = [&](int number, int lane, u32x4_t (&kw)[kSteps]) {
    // chunk 2 s + lq of row lr, at (2 s + lq) ^ (lr & 15): s flips bits of the first one's place
    const int lr = lane & 31, lq = lane >> 5;
    const uint32_t from = (uint32_t)(uintptr_t)smem[number & (kBuffers - 1)][0] + lr * 256 + 16 * (lq ^ (lr & 15));
#pragma unroll
    for (int s = 0; s < kSteps; ++s) kw[s] = *(const __attribute__((address_space(3))) u32x4_t *)(uintptr_t)(from ^ (32 * s));
  };
  auto scores = [&](const u32x4_t (&kw)[kSteps]) {
    f32x16_t s_acc = f32x16_t{};
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      s_acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kw[s]), qop[s], s_acc, 0, 0, 0);
    return s_acc;
  };

  int place = 0, k = 0, tiles = 0, t0 = 0;      // the attended piece's place in the ring, which tile of it, how many, the first
  int sinks_to = 0, gap = 0, len = 0;           // of its sight; its request's tokens
  int sees_from = 0, sees_to = 0;               // tokens that all its rows see
  int to_come = 0;                              // ranges of the tile's weights that are still to come, a bit each
  for (int number = 0; number < issued; ++number, ++k) {      // of the tile attended
    const int buf = number & (kBuffers - 1);
    const bool begins = k == tiles;
    if (begins) {
      place = (place + 1) & 7;
      k = 0;
      const Piece q = uniform(ring[w][place]);
      tiles = q.tiles;
      t0 = q.t0;
      sinks_to = q.sight.sinks;
      gap = q.sight.gap;
      len = q.len;
      const auto clamp = [](int64_t x) { return x < 0 ? 0 : x > 0x7fffffff ? 0x7fffffff : (int)x; };
      const int64_t first = (int64_t)q.end - q.rows;
      sees_to = clamp(first) < len ? clamp(first) : len;
      sees_from = p.window > 0 ? clamp(first + q.rows - p.window) : 0;
      first_row = kCacheGroupBlock * q.block;
      M = q.rows * p.G - first_row < kCacheGroupBlock ? q.rows * p.G - first_row : kCacheGroupBlock;
      groups = M <= 2 * kRows ? 2 : 1;
      mine = groups == 2 ? (w & 1) * kRows : w * kRows;
      turn = groups == 2 ? w >> 1 : 0;
      works = mine < M;
      const int lane = hidden(thread & 63), lr = lane & 31, lq = lane >> 5;
      const int rb = first_row + mine + lr, i = (int)((uint32_t)rb * p.g_inv >> 16);
      const int64_t row = (int64_t)q.row0 + i;
      const bool ok = mine + lr < M && row >= 0 && row < p.num_rows;
      const uint16_t *src = p.q + (ok ? row * p.q_row_stride + (int64_t)(q.h * p.G + rb - i * p.G) * kCacheDim : 0);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const u32x4_t y = *reinterpret_cast<const u32x4_t *>(src + 16 * s + 8 * lq);
        qop[s] = __builtin_bit_cast(bf16x8_t, ok ? y : u32x4_t{0u, 0u, 0u, 0u});
      }
      // here, not at their first use, where the next tiles' loads would be waited for too
#pragma unroll
      for (int s = 0; s < kSteps; ++s) asm volatile("" : "+v"(qop[s]));
      const Seen seen = seen_by(p, q.rows, q.row0, q.end, q.len, i);
      bits = ok ? seen.bits : 0;
      low = seen.low;
      m_run = kNegInf;
      l_run = 0.f;
      plain = false;
      lift = 0;
#pragma unroll
      for (int a = 0; a < kAccs; ++a) acc[a] = f32x16_t{};
    }
    const int tok = kTokens * (t0 + k + (t0 + k < sinks_to ? 0 : gap));
    const uint32_t hole = (holes >> 2 * (number & 7)) & 3u;
    const bool cut = hole != 0 || tok + kTokens > sees_to || (tok < sees_from && tok + kTokens > p.sinks);      // some rows do not see some of it
    const int pending = to_come;      // not 0: the tile was attended, but for these
    to_come = 0;
    if (!kHalf || pending == 0) {
      // in flight stay, straight to LDS, tile i + 2's four loads where tile i + 1 is needed next, else none; to registers all
      if constexpr (kDirect) {
        if (groups == 1 && number + 2 < issued)
          asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
        else
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      } else if (number + 3 < issued) {
        if (number & 1)
          tell(Int<0>{}, number + 3);
        else
          tell(Int<1>{}, number + 3);
      }
      workgroup_barrier();
      if (kDirect && __builtin_expect(cut, 0)) {
        clear(number, len - tok, hole);
        workgroup_barrier();
      }
      if constexpr (kDirect) {
        load(Int<0>{});
      } else {
        if (number & 1)
          bring(Int<0>{}, number + 3);
        else
          bring(Int<1>{}, number + 3);
      }
    }

    const bool exact = (exacts >> buf) & 1;
    if (begins && works) {      // the first scores of the piece: of its tile 0 or 1
      u32x4_t kw[kSteps];
      read_k(number + turn, hidden(thread & 63), kw);
      x = scores(kw);
    }
    // This tile's softmax and products, and the scores of the wave's next tile (of whatever lies there, if that is none)
    if (works && (groups == 1 || (k & 1) == turn)) {
      uint32_t word = ~0u;       // the tile's tokens that the lane's row sees
      const int lane = hidden(thread & 63), lq = lane >> 5;
      float least = -kNegInf;    // the smallest score that is seen
      if (__builtin_expect(cut, 0)) {
        const Piece q = uniform(ring[w][place]);
        const Seen seen = {bits, (int64_t)q.end - q.rows, low, p.sinks, q.len, 0, 0};
        word = seen.word(tok) & (hole & 1u ? 0xffff0000u : ~0u) & (hole & 2u ? 0xffffu : ~0u);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const bool sees = (word >> (8 * (e >> 2) + 4 * lq + (e & 3))) & 1u;
          if constexpr (kHalf) least = fminf(least, sees ? x[e] : -kNegInf);
          x[e] = sees ? x[e] : kNegInf;
        }
      } else if constexpr (kHalf) {
#pragma unroll
        for (int e = 0; e < 16; ++e) least = fminf(least, x[e]);
      }
      float mx = kNegInf;
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, x[e]);
      mx *= p.scale_log2;
      int then = number + groups;      // the tile whose scores are next
      const float small = least * p.scale_log2;
      uint64_t moves = __builtin_amdgcn_ballot_w64(mx > m_run + (kHalf ? kHalfSlack : kSlack));
      if constexpr (kHalf) moves |= __builtin_amdgcn_ballot_w64(small < m_run + kHalfLeast) | (uint64_t)pending;
      if (__builtin_expect(moves != 0, 0)) {
        float mn = xgroup_max<2>(mx), lower = 0.f;
        if constexpr (kHalf) {
          // a whole number, so that nothing is rounded where lift is added or taken off and a tile's ranges meet
          mn = fmaxf(plain ? m_run : m_run + (float)lift, ceilf(mn));
          if (one(exact || plain ? 1 : 0) == 0 && (lift != 0 || pending != 0 || __builtin_amdgcn_ballot_w64(small < mn + kHalfLeast) != 0)) {
            // Ranges of weights: from 2^kHalfLeast of the largest on, the 2^kHalfStep below, what is still smaller.  Those that the
            // tile may have are attended one after the other, m_run as far below the largest score, and the tile's scores computed
            // again in between.
            const float a = mn + kHalfLeast, b = a - kHalfStep;
            const int all = pending != 0 ? pending
                                         : (__builtin_amdgcn_ballot_w64(mx >= a) != 0 ? 1 : 0) | (__builtin_amdgcn_ballot_w64(small < a && mx >= b) != 0 ? 2 : 0) |
                                               (__builtin_amdgcn_ballot_w64(small < b) != 0 ? 4 : 0);
            const int range = all == 0 ? 0 : __builtin_ctz(all);
            to_come = all & (all - 1);
            if (to_come != 0) {      // the loop comes to the same tile again
              then = number--;
              --k;
            }
            lift = kHalfStep * range;
            const float from = range == 0 ? a : range == 1 ? b : kNegInf, to = range == 0 ? __builtin_nanf("") : range == 1 ? a : b;
#pragma unroll
            for (int e = 0; e < 16; ++e) {      // a NaN stays
              const float y = x[e] * p.scale_log2;
              x[e] = y < from || y >= to ? kNegInf : x[e];
            }
          }
          lower = plain ? 0.f : (float)lift;
        } else {
          mn = fmaxf(m_run, mn);
        }
        const float alpha = mn - lower == m_run ? 1.f : exp2_fast(m_run - (mn - lower));
        l_run *= alpha;
#pragma unroll
        for (int a = 0; a < kAccs; ++a) acc[a] *= alpha;
        m_run = mn - lower;
      }
      if (kHalf && __builtin_expect(exact, 0)) {
        if (!plain && ((exacts >> (kBuffers + buf)) & 1) != 0) {
          plain = true;
          const float to = m_run + (float)lift, f = to == m_run ? 1.f : exp2_fast(m_run - to);
          m_run = to;
          l_run *= f / (1 << kPShift);
#pragma unroll
          for (int a = 0; a < kAccs; ++a) acc[a] *= f / (1 << (kPShift + Half<FMT>::kVShift));
        }
      }
      const float ms = m_run == kNegInf ? 0.f : kHalf && !plain ? m_run - kPShift : m_run;

      if (kHalf && __builtin_expect(exact || plain, 0)) {
        // V beyond half precision, which may be no number: each token is added to the rows that see it
        const float factor = exact ? plain ? 1.f : (float)(1 << Half<FMT>::kVShift) : 1.f / (1 << Half<FMT>::kVShift);
#pragma unroll 1
        for (int t = 0; t < 32; ++t) {
          const int e = 4 * (t >> 3) + (t & 3);
          float xe = 0.f;
#pragma unroll
          for (int j = 0; j < 16; ++j) xe = j == e ? x[j] : xe;
          xe = __shfl(xe, (lane & 31) + 32 * ((t >> 2) & 1));
          const float pe = exp2_fast(__builtin_fmaf(xe, p.scale_log2, -ms));
          if (lq == 0) l_run += pe;        // the row's lanes are summed at the end
          if (!((word >> t) & 1u)) continue;
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const u32x2_t y = *reinterpret_cast<const u32x2_t *>(smem[buf][1] + t * 256 + 16 * (c ^ swizzle<FMT, 32>(t)) + 8 * lq);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t v = j & 1 ? y[j >> 1] >> 16 : y[j >> 1] & 0xffffu;
              acc[c >> 2][4 * (c & 3) + j] += pe * factor * (exact ? __uint_as_float(v << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)v));
            }
          }
        }
        u32x4_t kw[kSteps];
        read_k(number + groups, lane, kw);
        x = scores(kw);
      } else {
        u32x4_t kw[kSteps];
        read_k(then, lane, kw);
        // O^T += V^T P^T, V's transpose read as in cache_attend_kernel with 32 rows
        const int li = lane & 15;
        const int vrow = 4 * lq + (li >> 2), chunk = 2 * ((lane >> 4) & 1) + ((li & 3) >> 1);
        const uint32_t vat = (uint32_t)(uintptr_t)smem[buf][1] + vrow * 256 + 16 * (chunk ^ swizzle<FMT, 32>(vrow)) + 8 * (li & 1);
        constexpr int kParts = kHalf ? 2 : 3;
        s16x8_t v[2][kAccs];
        u32x4_t part[2][kParts];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
          for (int a = 0; a < kAccs; ++a) {
            const uint32_t from = (vat ^ (64 * a)) + 16 * 256 * t;
            const s16x4_t v0 = lds_read_tr16(from), v1 = lds_read_tr16(from + 8 * 256);
            v[t][a] = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p0 = exp2_fast(__builtin_fmaf(x[8 * t + 2 * e], p.scale_log2, -ms));
            const float p1 = exp2_fast(__builtin_fmaf(x[8 * t + 2 * e + 1], p.scale_log2, -ms));
            l_run += p0;
            l_run += p1;
            uint32_t a, b, c;
            if constexpr (kHalf) {
              cut2(p0, p1, a, b);
            } else {
              cut3(p0, p1, a, b, c);
              part[t][2][e] = c;
            }
            part[t][0][e] = a;
            part[t][1][e] = b;
          }
        }
        const f32x16_t next = scores(kw);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int j = 0; j < kParts; ++j)
#pragma unroll
            for (int a = 0; a < kAccs; ++a) {
              if constexpr (kHalf)
                acc[a] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, v[t][a]), __builtin_bit_cast(f16x8_t, part[t][j]), acc[a], 0, 0, 0);
              else
                acc[a] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v[t][a]), __builtin_bit_cast(bf16x8_t, part[t][j]), acc[a], 0, 0, 0);
            }
        // The reads first; then each product with the vector work that fits beside it: the first half's weights beside the
        // scores, the second's beside the first's products.
        __builtin_amdgcn_sched_group_barrier(0x100, kHalf ? 17 : 16, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, 24, 0);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x2, kHalf ? 4 : 7, 0);
        }
        
#pragma unroll
        for (int i = 0; i < kParts * kAccs; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x2, kHalf ? 5 : 7, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, kParts * kAccs, 0);
        x = next;
      }
      if (kDirect && __builtin_expect(cut && one(spoilt[buf]) == number, 0)) {
        // values that are no numbers, left out of the products, make none of the rows' that see them
#pragma unroll 1
        for (int t = 0; t < 32; ++t) {
          const uint32_t *bad = reinterpret_cast<const uint32_t *>(no_number[buf][t]);
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const uint32_t which = (word >> t) & 1u ? bad[c >> 2] >> (8 * (c & 3) + 4 * lq) : 0u;
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[c >> 2][4 * (c & 3) + j] = (which >> j) & 1u ? __builtin_nanf("") : acc[c >> 2][4 * (c & 3) + j];
          }
        }
      }
    }

    if (k + 1 == tiles) {      // the piece ends: its states, or its result
      const int lane = hidden(thread & 63), lr = lane & 31, lq = lane >> 5;
      float m = m_run, l = xgroup_sum<2>(l_run);
      if constexpr (kHalf) {      // without the factors, which are powers of two
        const int up = plain ? 0 : kPShift + lift;
        const float f = __uint_as_float((uint32_t)(127 - up) << 23);
        m += plain ? 0.f : (float)lift;
        l *= f;
#pragma unroll
        for (int a = 0; a < kAccs; ++a) acc[a] *= plain ? 1.f : f / (1 << Half<FMT>::kVShift);
      }
      auto piece_of = [&](int c) {
        return f32x4_t{acc[c >> 2][4 * (c & 3)], acc[c >> 2][4 * (c & 3) + 1], acc[c >> 2][4 * (c & 3) + 2], acc[c >> 2][4 * (c & 3) + 3]};
      };
      if (groups == 2) {
        // the two waves of the same rows meet in the tile that was attended, lane by lane, half of the channels at a time
        float f = 1.f, fo = 0.f;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          workgroup_barrier();
          f32x4_t *there = reinterpret_cast<f32x4_t *>(smem[buf]) + (w & 1) * 8 * 64 + lane;
          if (w >= 2) {
#pragma unroll
            for (int c = 0; c < 8; ++c) there[64 * c] = piece_of(8 * g + c);
            merge_m[w & 1][lane] = m;
            merge_l[w & 1][lane] = l;
          }
          workgroup_barrier();
          if (w < 2) {
            if (g == 0) {
              const float mo = merge_m[w & 1][lane], top = fmaxf(m, mo);
              f = top == kNegInf ? 1.f : exp2_fast(m - top), fo = top == kNegInf ? 1.f : exp2_fast(mo - top);
              l = f * l + fo * merge_l[w & 1][lane];
              m = top;
            }
#pragma unroll
            for (int c = 8 * g; c < 8 * g + 8; ++c) {
              const f32x4_t o = there[64 * (c - 8 * g)];
#pragma unroll
              for (int j = 0; j < 4; ++j) acc[c >> 2][4 * (c & 3) + j] = f * acc[c >> 2][4 * (c & 3) + j] + fo * o[j];
            }
          }
        }
      }
      const int r = mine + lr;
      if (r < M && (groups == 1 || w < 2)) {
        const Piece q = uniform(ring[w][place]);
        if (q.tiles == q.whole) {
          const int rb = first_row + r, i = (int)((uint32_t)rb * p.g_inv >> 16);
          const int64_t row = ((int64_t)q.row0 + i) * p.Hq + q.h * p.G + rb - i * p.G;
          if (q.row0 + i >= 0 && q.row0 + i < p.num_rows) {
            const RowEnd end = row_end(p, row, m, l);
#pragma unroll
            for (int c = 0; c < 16; ++c) {
              const int64_t o = row * kCacheDim + 8 * c + 4 * lq;
              *reinterpret_cast<f32x4_t *>(p.out + o) = row_value(p, end, o, piece_of(c));
            }
            if (lq == 0 && p.lse != nullptr) p.lse[row] = end.lse;
          }
        } else {
          const int64_t o = (int64_t)(2 * worker + (q.t0 == 0 ? 1 : 0)) * part_rows(p) + r;
#pragma unroll
          for (int c = 0; c < 16; ++c) *reinterpret_cast<f32x4_t *>(p.part_a + o * kCacheDim + 8 * c + 4 * lq) = piece_of(c);
          if (lq == 0) *reinterpret_cast<f32x2_t *>(p.part_ml + 2 * o) = f32x2_t{m, l};
        }
      }
    }
  }
}

template <int FMT>
hipError_t attend_group(const CacheGroupArgs &p, hipStream_t s) {
  hipLaunchKernelGGL((cache_attend_group_kernel<FMT>), dim3(p.workers), dim3(kThreads), 0, s, p);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess && p.parts != 1 ? launch_join(p, s) : e;
}

}  // namespace

CacheSplit cache_group_split(int fmt, int B, int Hkv, int capacity, int M) {
  (void)fmt;
  const int64_t pairs = (int64_t)B * Hkv * ((M + kCacheGroupBlock - 1) / kCacheGroupBlock);
  CacheSplit r;
  r.alone = false;
  r.piece_units = kPieceGroupTiles;
  const int64_t units = pairs * ((capacity + kTokens - 1) / kTokens + r.piece_units);
  const int64_t need = (units + kMinShare - 1) / kMinShare, most = 512;      // two workgroups per CU
  r.workers = (int)(need < most ? need : most);
  return r;
}

hipError_t launch_cache_attend_group(const CacheGroupArgs &p, int fmt, hipStream_t s) {
  if (fmt == kCacheBf16) return attend_group<kCacheBf16>(p, s);
  if (fmt == kCacheMx8) return attend_group<kCacheMx8>(p, s);
  return attend_group<kCacheMx4>(p, s);
}

}  // namespace ss
