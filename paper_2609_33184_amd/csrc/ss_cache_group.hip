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
// Per wave and tile: 8 v_mfma_f32_32x32x16_bf16 for S^T = K Q^T of the next tile, beside this tile's
// softmax, and 24 for O^T += V^T P^T, in the compiler's order (held to one with the vector work between the products, 16 x 32768
// tokens with 96 rows took 638 us instead of 621, 16 x 12000..16384 with 256 rows in bf16 535 instead of 522).
//
// Precision.  P in three parts of bf16, exact, as in cache_attend_kernel, and V as bf16, which the values of all formats are:
// against 64 bits 1e-7 to 2e-7 in the 2-norm, the plain form in fp32 1e-7 to 7e-7.  P in two parts of f16 and V as f16, in 8 and 4 bits, took 530
// us where this takes 621, and was off by 1.5e-3 behind a first token that outweighs thousands of others by e^26 whose values are 2^16 times
// its own, since f16 ends 2^-37 below the largest weight; by 4.9e-5 where V's f16 were subnormal, which the matrix unit adds with fewer
// bits; and needed a way around for larger values that took 20 times as long.  Two parts of bf16: 565 us and 2e-6 throughout.
//
// bf16 rows go from memory to LDS without passing registers.  What a wave needs next is waited for by
// count, so that the loads behind it stay in flight.
//
// What bounds it (whole calls, the join in them; shares of the cycles from a trace of the kernel alone).  bf16, 16 x 12000..16384
// tokens, 256 rows: 503 to 522 us; the SIMDs issue vector work 48% and matrix work 47% of the cycles, one after the other; the
// matrix work alone would take 382.  8 bits, 16 x 32768 tokens, 96 rows: 617 us, 155 for the bytes, 344 for the matrix work, all of it on
// three SIMDs of four (96 rows leave a wave without): vector work 35%, matrix work 27% of all four's cycles, and the rest waits at the
// barrier and for LDS.  One request of 32768 tokens, 256 rows: 99 us, 57 for the matrix work, 10 for the join of its 32 states a
// row.  None of it depends on the scores or the values.
#include <hip/hip_runtime.h>

#include "ss_cache.h"
#include "ss_cache_attend.h"

namespace ss {
namespace {

typedef short s16x8_t __attribute__((ext_vector_type(8)));

constexpr int kTokens = kCacheGroupTile;        // of a tile
constexpr int kRows = 32;                       // of a wave
constexpr int kTileBytes = kTokens * 256;       // K or V of a tile, 16 bits a value
constexpr int kBuffers = 4;                     // tiles in LDS
constexpr int kSteps = kCacheDim / 16;          // of a product over the channels
constexpr int kAccs = kCacheDim / 32;           // accumulators of 32 channels

// What a piece costs beside its tiles, in tiles: 24 ragged requests with 4, 8 and 16 54.0, 55.9 and 62.8 us.
constexpr int kPieceGroupTiles = 8;

template <int I>
using Int = std::integral_constant<int, I>;

// A wave's 64 x 16 bytes, at `from` + its lanes' offsets, straight into LDS, lane by lane from `to` on (a byte address there,
// the wave's).  In assembly, since with the builtin every read of LDS waits for all of them; it has no output register,
// and what reads the bytes is behind a wait and a barrier.  The compiler keeps no distances inside assembly: the load needs one
// wait state behind M0's write, and five behind a vector instruction that may have written its scalar address.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"      // that M0 is a reserved register
__device__ __forceinline__ void load_to_lds(const uint8_t *from, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(from) : "memory", "m0");
}
#pragma clang diagnostic pop

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
  constexpr bool kDirect = FMT == kCacheBf16;              // rows go to LDS as they are
  constexpr int kLanes = kRow / 16;                        // lanes of a stored row
  __shared__ __attribute__((aligned(256))) unsigned char smem[kBuffers][2][kTileBytes];     // tiles' K, V
  __shared__ float merge_m[2][64], merge_l[2][64];
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
  // The tile in the registers into LDS.
  auto stage = [&](auto parity, int number) {
    constexpr int set = decltype(parity)::value;
    const uint32_t to = (uint32_t)(uintptr_t)smem[number & (kBuffers - 1)][0];
    if constexpr (FMT == kCacheMx8) {
      const float kf = scale_of(ks[set]), vf = scale_of(vs[set]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const u32x2_t a = widen8(kr[set][2 * j], kf), d = widen8(kr[set][2 * j + 1], kf);
        put(to + (k_to ^ (16 * j)), u32x4_t{a[0], a[1], d[0], d[1]});
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const u32x2_t a = widen8(vr[set][2 * j], vf), d = widen8(vr[set][2 * j + 1], vf);
        put(to + (v_to ^ (16 * j)), u32x4_t{a[0], a[1], d[0], d[1]});
      }
    } else if constexpr (FMT == kCacheMx4) {
      const float f = scale_of(vs[set]);
#pragma unroll
      for (int j = 0; j < 4; ++j) put(to + ((w >= 2 ? v_to : k_to) ^ (16 * j)), widen4(kr[set][j], f));
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
  if (thread < kBuffers) spoilt[thread] = -1;
  workgroup_barrier();
  auto bring = [&](auto parity, int number) {      // tile `number` from registers into LDS, the second next one into them
    if (number < issued) stage(parity, number);
    load(parity);
  };
  load(Int<0>{});
  load(Int<1>{});
  if constexpr (kDirect) {
    load(Int<0>{});
  } else {
    bring(Int<0>{}, 0);
    bring(Int<1>{}, 1);
    bring(Int<0>{}, 2);
  }

  bf16x8_t qop[kSteps];
  uint64_t bits = 0;         // of the row's word
  int low = 0;               // its window's first token
  float m_run = kNegInf, l_run = 0.f;
  f32x16_t acc[kAccs], x = f32x16_t{};      // x: the scores of the tile that this wave attends next
  int M = 0, first_row = 0, groups = 1, mine = 0, turn = 0;      // rows of the block; of all, its first; waves per 32 rows; this wave's rows, its tiles
  bool works = false;        // whether it has rows
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
#pragma unroll
      for (int a = 0; a < kAccs; ++a) acc[a] = f32x16_t{};
    }
    const int tok = kTokens * (t0 + k + (t0 + k < sinks_to ? 0 : gap));
    const uint32_t hole = (holes >> 2 * (number & 7)) & 3u;
    const bool cut = hole != 0 || tok + kTokens > sees_to || (tok < sees_from && tok + kTokens > p.sinks);      // some rows do not see some of it
    // in flight stay, straight to LDS, tile i + 2's four loads where tile i + 1 is needed next, else none; to registers all
    if constexpr (kDirect) {
      if (groups == 1 && number + 2 < issued)
        asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
      else
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    workgroup_barrier();
    if (__builtin_expect(cut, 0)) {
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

    if (begins && works) {      // the first scores of the piece: of its tile 0 or 1
      u32x4_t kw[kSteps];
      read_k(number + turn, hidden(thread & 63), kw);
      x = scores(kw);
    }
    // This tile's softmax and products, and the scores of the wave's next tile (of whatever lies there, if that is none)
    if (works && (groups == 1 || (k & 1) == turn)) {
      const int lane = hidden(thread & 63), lq = lane >> 5;
      uint32_t word = ~0u;       // the tile's tokens that the lane's row sees
      if (__builtin_expect(cut, 0)) {
        const Piece q = uniform(ring[w][place]);
        const Seen seen = {bits, (int64_t)q.end - q.rows, low, p.sinks, q.len, 0, 0};
        word = seen.word(tok) & (hole & 1u ? 0xffff0000u : ~0u) & (hole & 2u ? 0xffffu : ~0u);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = (word >> (8 * (e >> 2) + 4 * lq + (e & 3))) & 1u ? x[e] : kNegInf;
      }
      float mx = kNegInf;
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, x[e]);
      mx *= p.scale_log2;
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(mx > m_run + kSlack) != 0, 0)) {
        const float mn = fmaxf(m_run, xgroup_max<2>(mx));
        const float alpha = mn == kNegInf ? 1.f : exp2_fast(m_run - mn);
        l_run *= alpha;
#pragma unroll
        for (int a = 0; a < kAccs; ++a) acc[a] *= alpha;
        m_run = mn;
      }
      const float ms = m_run == kNegInf ? 0.f : m_run;

      u32x4_t kw[kSteps];
      read_k(number + groups, lane, kw);
      // O^T += V^T P^T, V's transpose read as in cache_attend_kernel with 32 rows
      const int li = lane & 15;
      const int vrow = 4 * lq + (li >> 2), chunk = 2 * ((lane >> 4) & 1) + ((li & 3) >> 1);
      const uint32_t vat = (uint32_t)(uintptr_t)smem[buf][1] + vrow * 256 + 16 * (chunk ^ swizzle<FMT, 32>(vrow)) + 8 * (li & 1);
      s16x8_t v[2][kAccs];
      u32x4_t part[2][3];
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
          cut3(p0, p1, a, b, c);
          part[t][0][e] = a;
          part[t][1][e] = b;
          part[t][2][e] = c;
        }
      }
      const f32x16_t next = scores(kw);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 3; ++j)
#pragma unroll
          for (int a = 0; a < kAccs; ++a)
            acc[a] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v[t][a]), __builtin_bit_cast(bf16x8_t, part[t][j]), acc[a], 0, 0, 0);
      x = next;
      if (__builtin_expect(cut && one(spoilt[buf]) == number, 0)) {
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
