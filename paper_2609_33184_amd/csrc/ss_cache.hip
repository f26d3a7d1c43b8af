// gfx950 (MI355X) kernels of the paged cache: tokens written into pages as
// bf16 or in 8 or 4 bits with a power-of-two scale per 32 channels, read back
// as bf16, and attended in place.
//
// Numbers.  A scaled block stands for code * 2^(byte - 127), code an OCP e4m3
// or e2m1 number: v_cvt_scalef32 converts two of them with their scale in one
// instruction, and every value of a finite block is zero or a normal bf16 number,
// so nothing is lost between the cache and the matrix instructions (but 2^128, to
// which the largest bf16 numbers round, is an infinity from there on).  A scale
// byte of 255 makes the conversion give NaN.
//
// Rows.  Request b's row i of n_b stands for position end_b - n_b + i.  What a
// table, an end or a row start could make unsafe is checked here: a page number
// outside [0, num_pages) is a page without tokens, a position outside the table
// is no token, a row outside [0, num_rows) is no row.
#include <hip/hip_runtime.h>

#include "ss_cache.h"
#include "ss_cache_attend.h"
#include "ss_cache_device.h"

#include <type_traits>

namespace ss {
namespace {

// ---------------------------------------------------------------------------
// Writing and reading rows.  A workgroup takes 16 rows and HEADS KV heads, 16
// lanes to a row's 128 channels: a lane holds 8 channels, four lanes a scaled
// block.  Both directions are bound by memory; the rows' loads go out before
// their places in the cache are looked up, which takes two round trips (starts
// and ends, then the table).  The bf16 rows stream past the caches, the pages do
// not: what is written is attended next (32000 tokens with 8 heads written in 4
// bits 43.5 us through the caches, 32 past them; 65536 tokens read from 8 bits 80
// and 68, a copy's rate and a quarter more).
// ---------------------------------------------------------------------------
template <int FMT, int HEADS>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(CacheRowsArgs p) {
  extern __shared__ int32_t starts[];
  int32_t *ends = starts + p.B + 1;
  const int tx = threadIdx.x, c = tx & 15;
  const int64_t t = (int64_t)blockIdx.x * kGroupRows + (tx >> 4);
  const int h0 = blockIdx.y * HEADS;
  u32x4_t kx[HEADS], vx[HEADS];
  const int64_t tl = t < p.num_rows ? t : p.num_rows - 1;
#pragma unroll
  for (int j = 0; j < HEADS; ++j) {
    const int h = h0 + j < p.Hkv ? h0 + j : p.Hkv - 1;
    const int64_t at = tl * p.row_stride + h * p.head_stride + 8 * c;
    kx[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p.k + at));
    vx[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p.v + at));
  }
  const Place pl = place_of(p, t, tx, starts, ends);
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
  extern __shared__ int32_t starts[];
  int32_t *ends = starts + p.B + 1;
  const int tx = threadIdx.x, c = tx & 15;
  const int64_t t = (int64_t)blockIdx.x * kGroupRows + (tx >> 4);
  const int h0 = blockIdx.y * HEADS;
  const Place pl = place_of(p, t, tx, starts, ends);
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
    __builtin_nontemporal_store(x[j][0], reinterpret_cast<u32x4_t *>(p.k + at));
    __builtin_nontemporal_store(x[j][1], reinterpret_cast<u32x4_t *>(p.v + at));
  }
}

// ---------------------------------------------------------------------------
// Attention.  The call's tiles of 32 tokens, of every request and KV head, head
// by head, are one sequence that is cut into equal shares, one per worker, however
// long the requests are.  The lengths are device data, so every worker finds its
// share itself from the ends (a prefix sum over the requests).  A share's part of
// one (request, head) is a piece.  A worker is a workgroup, whose waves attend a
// piece's tiles w, w + 4, ... and merge through LDS, or, where there are (request,
// head) pairs enough, a wave.  A piece that is all of its pair writes the result;
// the others leave their state (m, l, a) in the workspace, at most two per worker,
// and cache_join_kernel merges them in the workers' order.  A worker that finds
// itself the last of a pair could do that in the same launch; the release and
// acquire between the XCDs' caches cost far more than the second launch (256
// short requests 100 us with fences and 28.5 with coherent accesses alone, 27
// with two launches).
//
// Per tile: S^T = K Q^T, K straight from memory in the operand's layout (a lane
// holds 16 bytes at a time of one token; the channels of a k-step are permuted
// alike in Q); softmax with one running maximum and sum per row; O^T += V^T P^T, V
// through LDS and its transpose read, P straight from the score registers.  Up
// to 16 rows per KV head use v_mfma_f32_16x16x32_bf16, more v_mfma_f32_32x32x16_bf16
// (NR rows), beside which more vector work fits: two waves of a SIMD take 12.0 ns
// for one of the small products (7.7 ns by itself) with 4 independent FMAs (7.8),
// 10.3 for half a large one with them.  Lane l: lr = l % NR, lq = l / NR, kGroups =
// 64 / NR.  In a score tile lane (lr, lq) holds, as score e, token 4 kGroups (e / 4)
// + 4 lq + e % 4 of row lr; in O, as piece c, channels 4 kGroups c + 4 lq .. + 3.
// The matrix instructions that take e4m3 and e2m1 operands with their scales are
// not used for S: their sums were off by up to 2^-12 of the sum of the products'
// magnitudes.
//
// A wave has the loads of its next tile in flight while it works on one, and
// computes that tile's scores and stages its V beside this one's products, over
// the end of a piece too, so that a short piece does not wait for memory.
// Requests of more than 32 rows per KV head are attended by two waves a tile, 32
// rows each (HALVES): 64 rows in one wave leave one wave per SIMD (16 x 32768
// tokens in 8 bits 413 us, 400 with two waves, 320 to 390 since).
//
// What bounds it: bf16 is read at 6.7 TB/s (64 requests of 2048 to 65536 tokens,
// 4.5 GB: 675 us, 664 with the arithmetic taken out); 8 and 4 bits with up to 16
// rows at 6.4 and 5.2 (16 x 32768 tokens: 174 and 110 us); with 24 to 64 rows the
// vector and matrix instructions, which the SIMD issues one after the other (16 x
// 32768 tokens in 4 bits with 24 rows: 155 to 185 us, 130 without its loads, 94
// without its arithmetic); short requests the latency of a piece's first loads and
// of its merge.
//
// Precision: P enters as three bf16 parts cut from its 24 bits, so that it is
// exact (two parts would leave 1.7e-6 of relative error in the result, against
// 1e-7 to 7e-7); sums and accumulators are fp32.  The running maximum moves only
// where a score passes it by more than 2^8, which keeps a cross-lane maximum
// and the rescaling out of most tiles; weights up to 2^8 cost no precision.
//
// SeenArgs: rows that see a tree, or a window and the first tokens.  Of a request's
// tiles only those are counted and read of which some row may see a token: the
// sinks' and, behind the gap, the windows' (Sight); a tile that all rows see whole
// needs no mask, of the others a word of 32 bits says which tokens a row sees.
// Where a window makes the lengths alike the call is cut into equal parts of each
// request instead of equal shares while they are short (cache_attend_parts).  64 requests
// of one row in a window of 4096 in bf16 (1.03 GB) 170 us, 6.0 TB/s; 16 requests of 8
// rows, 64 per KV head, in a window of 1024 in 4 bits 27.0 us, in a trace 25.5 and 5.0 for
// the join: nine steps of two tiles, of which the SIMDs issue a third and the rest is latency.
// ---------------------------------------------------------------------------
constexpr int kLdsRow = 256;                        // a staged V row, bf16
constexpr int kVTile = kCacheTile * kLdsRow;
constexpr int kAwPitch = 132;                       // floats per row of a wave's partial accumulator
// What a piece costs beside its tiles, in tiles: its first loads, its merge.  A
// workgroup's at 4, 8, 12 and 16: 24 ragged requests 22.2, 20.3, 18.9 and 19.0 us,
// 16 chunks of 4096 tokens 34.2, 34.1, 32.5 and 32.0; a wave's at 1, 2, 3 and 4: 256
// short requests 22.7, 20.4, 21.4 and 21.4.
constexpr int kPieceGroup = 16, kPieceAlone = 2;

// LDS: the waves' V tiles, and where the states of two waves meet at a piece's end.
template <int NR, int STREAMS>
struct AttendLds {
  static constexpr int kMerge = STREAMS == 1 ? 0 : 2 * NR * (kAwPitch + 2) * 4;
  static constexpr int kBytes = kWaves * kVTile + kMerge;
};

template <int FMT, int NR>
struct Tile {   // a wave's loads of one tile
  static constexpr int kBlocks = kCacheTile / NR;                                    // of NR tokens
  static constexpr int kKLoads = cache_row_bytes(FMT) / 16 / (64 / NR);              // 16 bytes each, per block
  static constexpr int kVLoads = cache_row_bytes(FMT) / 32;
  u32x4_t k[kBlocks][kKLoads], v[kVLoads];
  uint32_t ks[kBlocks], vs[kVLoads];
};

template <int NR>
struct Mfma;
template <>
struct Mfma<16> {
  using Acc = f32x4_t;
  static constexpr int kDepth = 32;    // of a product
  static __device__ __forceinline__ Acc run(bf16x8_t a, bf16x8_t b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mfma<32> {
  using Acc = f32x16_t;
  static constexpr int kDepth = 16;
  static __device__ __forceinline__ Acc run(bf16x8_t a, bf16x8_t b, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

// Waves per SIMD that the registers are held to.  Up to 16 rows: 8 bits with one
// and two 8 x 6000 tokens 29.1 and 24.7 us, 4 bits with two and three 16 x 32768
// tokens 120 and 111; more rows: 8 and 4 bits with one and two 242 and 207, 209 and
// 166 (24 rows).  bf16 with more rows takes 312 registers and does not fit two: 16 x
// 32768 tokens with 24 and 64 rows 338 and 498 us, 299 of them for the bytes.
constexpr int attend_waves(int fmt, int nr) {
  if (nr == 32) return fmt == kCacheBf16 ? 1 : 2;
  return fmt == kCacheMx4 ? 3 : 2;
}

template <int FMT, int NR, int HALVES, int STREAMS, typename Args>
__global__ __launch_bounds__(kThreads, attend_waves(FMT, NR)) void cache_attend_kernel(Args p) {
  using Lds = AttendLds<NR, STREAMS>;
  static_assert(STREAMS * HALVES == kWaves || (STREAMS == 1 && HALVES == 1), "a workgroup's waves, or each for itself");
  using Acc = typename Mfma<NR>::Acc;
  __shared__ __attribute__((aligned(256))) unsigned char smem[Lds::kBytes];
  constexpr int kRow = cache_row_bytes(FMT);
  constexpr int kGroups = 64 / NR;
  constexpr int kScores = kCacheTile / kGroups;            // of a tile, per lane
  constexpr int kRegs = NR / kGroups;                      // of an accumulator: scores of NR tokens, or channels
  constexpr int kAccs = kCacheDim / NR, kChans = kCacheDim / kGroups / 4;   // accumulators of NR channels; 4-channel pieces
  constexpr int kSteps = kCacheDim / Mfma<NR>::kDepth, kVSteps = kCacheTile / Mfma<NR>::kDepth;
  constexpr int kPer = 256 / kRow;                         // k-steps that a lane's 16 bytes of K serve
  constexpr int kLanes = kRow / 16, kStep = 64 / kLanes;   // V: lanes per row, rows per load
  constexpr bool kAlone = STREAMS == 1;                    // each wave is a worker
  const int thread = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(thread >> 6);
  const int half = HALVES == 2 ? w & 1 : 0, ws = kAlone ? 0 : HALVES == 2 ? w >> 1 : w;   // its rows, its tiles
  const int worker = kAlone ? blockIdx.x * kWaves + w : blockIdx.x;

  // This worker's share and where it starts; every wave finds it by itself.  The
  // requests are counted 64 at a time, lane j keeping the units of chunk j.
  Request win;            // requests base .. base + 63
  int base = 0, idx, skip, h, left;   // the next request, its units that are not ours, its head; our units
  bool even = false;
  if constexpr (kSeen<Args>) even = p.parts > 0;
  if (even) {
    if constexpr (kSeen<Args>) {
      const Whole at = whole_of(p, worker);
      base = at.b & ~63;
      idx = at.b & 63;
      h = at.h;
      win = request_at(p, base + (thread & 63));
      at.units(p, lane_of(win.tiles, idx), skip, left);
      if (lane_of(win.tiles, idx) == 0 && p.parts == 1) write_empty(p, lane_of(win.rows, idx), lane_of(win.row0, idx), at);
      if (left == 0 || skip >= lane_of(win.units, idx)) return;      // without tokens, or fewer rows
    }
  } else {
    const int lane = thread & 63;
    const int chunks = (p.B + 63) / 64;
    int before = 0, scan, all;
    if (chunks == 1) {
      win = request_at(p, lane);
      scan = wave_scan(win.units);
      all = lane_of(scan, 63);
    } else {
      int sums = 0;
      for (int j = 0; j < chunks; j += 4) {
        int t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = request_at(p, 64 * (j + i) + lane).units;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int sum = lane_of(wave_scan(t[i]), 63);
          sums = lane == j + i ? sum : sums;
        }
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
  }

  const int page_tokens = 1 << p.page_shift;
  const uint32_t v_off = (uint32_t)(page_tokens * kRow), ks_off = 2 * v_off, vs_off = ks_off + 4u * (uint32_t)page_tokens;
  unsigned char *vs_lds = smem + w * kVTile;

  // A piece: tiles t0 .. t0 + tiles - 1 of a request's `whole`, for head h.  tiles = 0: none.
  struct Piece {
    int b, rows, row0, end, len, whole;
    int h, t0, tiles;
    int count;     // this wave's tiles: t0 + ws, + STREAMS, ...
    int ids;       // lane j: page of half tile j of them, -1 for what is none
    Sight sight;
  };
  // The request's tile that is the t-th attended one.
  auto tile_at = [&](const Piece &q, int t) {
    if constexpr (kSeen<Args>) return t < q.sight.sinks ? t : t + q.sight.gap;
    return t;
  };
  // Pages of the wave's tiles k0 .. k0 + 31 of a piece.
  auto pages_of = [&](const Piece &q, int k0) {
    const int lane = hidden(thread & 63);
    const int k = k0 + (lane >> 1);
    const int64_t tok = (int64_t)tile_at(q, q.t0 + ws + STREAMS * k) * kCacheTile + 16 * (lane & 1);
    int id = -1;
    if (k < q.count && tok < q.len) id = p.table[(int64_t)q.b * p.table_stride + (tok >> p.page_shift)];
    return id >= 0 && id < p.num_pages ? id : -1;
  };
  auto one = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  auto uniform = [&](const Piece &q) {     // the wave's, in scalar registers
    return Piece{one(q.b), one(q.rows), one(q.row0), one(q.end), one(q.len), one(q.whole), one(q.h), one(q.t0), one(q.tiles), one(q.count), q.ids,
                 {one(q.sight.sinks), one(q.sight.gap)}};
  };
  // The share's next piece.  Its units are the piece's cost, then the tiles: a
  // share that ends within the cost leaves the tiles to the next one.
  auto next_piece = [&]() {
    Piece q = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, -1, {0, 0}};
    while (left > 0) {
      const uint64_t more = idx < 64 ? __builtin_amdgcn_ballot_w64(win.units > 0) & (~0ull << idx) : 0;
      if (more == 0) {
        base += 64;
        idx = 0;
        if (base >= p.B) {
          base = 0;
          if (++h >= p.Hkv) left = 0;     // not reached while nobody changes the lengths under a call
        }
        win = request_at(p, base + hidden(thread & 63));
        continue;
      }
      idx = __builtin_ctzll(more);
      const int units = lane_of(win.units, idx), cost = p.piece_units;
      const int take = units - skip < left ? units - skip : left;
      const int t0 = skip > cost ? skip - cost : 0, t1 = skip + take > cost ? skip + take - cost : 0;
      left -= take;
      skip = 0;
      if (t1 > t0) {
        q.b = base + idx;
        q.rows = lane_of(win.rows, idx);
        q.row0 = lane_of(win.row0, idx);
        q.end = lane_of(win.end, idx);
        q.len = lane_of(win.len, idx);
        q.whole = lane_of(win.tiles, idx);
        q.h = h;
        q.t0 = t0;
        q.tiles = t1 - t0;
        q.count = q.tiles <= ws ? 0 : (q.tiles - ws + STREAMS - 1) / STREAMS;
        q.sight = sight_of(p, q.rows, q.end, q.len);
        q.ids = pages_of(q, 0);
        ++idx;
        break;
      }
      ++idx;
    }
    left = one(left);
    idx = one(idx);
    base = one(base);
    skip = one(skip);
    h = one(h);
    return uniform(q);
  };

  Tile<FMT, NR> cur;
  uint32_t gone = 0;     // halves of the loaded tile without a page
  // Where the tile at token tok of head h lies, its pages in lanes j and j + 1 of ids.
  struct Where {
    uint8_t *block[2];
    uint32_t slot[2];
    int ok[2];           // tokens of each half
  };
  auto find = [&](int tok, int len, int h, int ids, int j) {
    Where at;
    gone = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int id = lane_of(ids, j + u);
      const int tu = tok + 16 * u;
      const int ok = len - tu;
      at.ok[u] = ok < 0 || id < 0 ? 0 : ok > 16 ? 16 : ok;
      gone |= (id < 0 ? 1u : 0u) << u;
      at.slot[u] = (uint32_t)(tu & (page_tokens - 1));
      at.block[u] = p.pages + (uint64_t)(id < 0 ? 0 : id) * p.page_stride + (uint64_t)h * p.head_bytes;
    }
    return at;
  };
  // Issue the loads of its K.  Rows past the request's tokens are whatever the
  // page holds (page 0 stands in for none): their scores are masked.  A row's
  // bytes are spread over several loads, so K's go through the caches; V's are
  // whole lines and stream past them (64 requests in bf16: 665 us, all through
  // the caches 742; K streamed costs 64 rows in 8 bits 435 -> 530 us).
  auto load_k = [&](const Where &at) {
    const int lane = hidden(thread & 63), lr = lane % NR, lq = lane / NR;
#pragma unroll
    for (int u = 0; u < Tile<FMT, NR>::kBlocks; ++u) {
      if constexpr (NR == 16) {
        const __amdgpu_buffer_rsrc_t krs = __builtin_amdgcn_make_buffer_rsrc(at.block[u], (short)0, at.ok[u] > 0 ? (int)p.head_bytes : 0, kBufferFlags);
        const uint32_t o = (at.slot[u] + lr) * kRow + 16 * lq;
#pragma unroll
        for (int s = 0; s < Tile<FMT, NR>::kKLoads; ++s) cur.k[u][s] = __builtin_amdgcn_raw_buffer_load_b128(krs, o + 16 * kGroups * s, 0, 0);
        if constexpr (FMT != kCacheBf16) cur.ks[u] = __builtin_amdgcn_raw_buffer_load_b32(krs, ks_off + (at.slot[u] + lr) * 4, 0, 0);
      } else {
        // the block's two halves may lie in different pages
        const uint8_t *block = lr < 16 ? at.block[0] : at.block[1];
        const uint32_t row = (lr < 16 ? at.slot[0] : at.slot[1]) + (lr & 15);
        const u32x4_t *src = reinterpret_cast<const u32x4_t *>(block + row * kRow + 16 * lq);
#pragma unroll
        for (int s = 0; s < Tile<FMT, NR>::kKLoads; ++s) cur.k[u][s] = src[kGroups * s];
        if constexpr (FMT != kCacheBf16) cur.ks[u] = *reinterpret_cast<const uint32_t *>(block + ks_off + row * 4);
      }
    }
  };
  // Issue the loads of its V.  Rows past the request's tokens touch no memory and
  // read zero: a weight of zero must meet no leftover NaN.
  auto load_v = [&](const Where &at) {
    const int lane = hidden(thread & 63);
    __amdgpu_buffer_rsrc_t vrs[2], srs[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      vrs[u] = __builtin_amdgcn_make_buffer_rsrc(at.block[u], (short)0, at.ok[u] > 0 ? (int)(v_off + (at.slot[u] + at.ok[u]) * kRow) : 0, kBufferFlags);
      srs[u] = __builtin_amdgcn_make_buffer_rsrc(at.block[u], (short)0, at.ok[u] > 0 ? (int)(vs_off + (at.slot[u] + at.ok[u]) * 4) : 0, kBufferFlags);
    }
#pragma unroll
    for (int i = 0; i < Tile<FMT, NR>::kVLoads; ++i) {
      const int u = i * kStep / 16;
      const uint32_t row = at.slot[u] + (i * kStep) % 16 + lane / kLanes;
      cur.v[i] = __builtin_amdgcn_raw_buffer_load_b128(vrs[u], v_off + row * kRow + 16 * (lane % kLanes), 0, kStreamLoad);
      if constexpr (FMT != kCacheBf16)
        cur.vs[i] = __builtin_amdgcn_raw_buffer_load_b8(srs[u], vs_off + row * 4 + (lane % kLanes) * 4 / kLanes, 0, kStreamLoad);
    }
  };
  // Queries of a piece: B operand of k-step s, row lr, the chunk of 8 channels that K's lanes hold there
  bf16x8_t qop[kSteps];
  auto load_q = [&](const Piece &q) {
    const int lane = hidden(thread & 63), r = NR * half + lane % NR, lq = lane / NR;
    const int i = (int)((uint32_t)r * p.g_inv >> 16);      // r / G
    const int64_t row = (int64_t)q.row0 + i;
    const bool ok = r < q.rows * p.G && row >= 0 && row < p.num_rows;
    const uint16_t *src = p.q + (ok ? row * p.q_row_stride + (int64_t)(q.h * p.G + r - i * p.G) * kCacheDim : 0);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const u32x4_t y = *reinterpret_cast<const u32x4_t *>(src + 8 * (kPer * (kGroups * (s / kPer) + lq) + s % kPer));
      qop[s] = __builtin_bit_cast(bf16x8_t, ok ? y : u32x4_t{0u, 0u, 0u, 0u});
    }
  };
  // The scores of the tile whose K is in cur, and its V into LDS as bf16.
  auto scores = [&](float (&x)[kScores], int lane) {
    const int lq = lane / NR;
#pragma unroll
    for (int u = 0; u < Tile<FMT, NR>::kBlocks; ++u) {
      Acc s_acc = Acc{};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        bf16x8_t kop;
        const u32x4_t kw = cur.k[u][s / kPer];
        if constexpr (FMT == kCacheBf16) {
          kop = __builtin_bit_cast(bf16x8_t, kw);
        } else if constexpr (FMT == kCacheMx8) {
          const float f = scale_of((cur.ks[u] >> (8 * ((kGroups * (s / kPer) + lq) / 2))) & 0xffu);
          const u32x2_t a = widen8(kw[2 * (s % kPer)], f), d = widen8(kw[2 * (s % kPer) + 1], f);
          kop = __builtin_bit_cast(bf16x8_t, u32x4_t{a[0], a[1], d[0], d[1]});
        } else {
          const float f = scale_of((cur.ks[u] >> (8 * (kGroups * (s / kPer) + lq))) & 0xffu);
          kop = __builtin_bit_cast(bf16x8_t, widen4(kw[s % kPer], f));
        }
        s_acc = Mfma<NR>::run(kop, qop[s], s_acc);
      }
#pragma unroll
      for (int e = 0; e < kRegs; ++e) x[kRegs * u + e] = s_acc[e];
    }
  };
  auto stage = [&](int lane) {
#pragma unroll
    for (int i = 0; i < Tile<FMT, NR>::kVLoads; ++i) {
      const int t = i * kStep + lane / kLanes, c = lane % kLanes;
      unsigned char *row = vs_lds + t * kLdsRow;
      u32x4_t y[kPer];
      if constexpr (FMT == kCacheBf16) {
        y[0] = cur.v[i];
      } else if constexpr (FMT == kCacheMx8) {
        const float s = scale_of(cur.vs[i]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const u32x2_t a = widen8(cur.v[i][2 * j], s), d = widen8(cur.v[i][2 * j + 1], s);
          y[j] = u32x4_t{a[0], a[1], d[0], d[1]};
        }
      } else {
        const float s = scale_of(cur.vs[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = widen4(cur.v[i][j], s);
      }
#pragma unroll
      for (int j = 0; j < kPer; ++j) *reinterpret_cast<u32x4_t *>(row + 16 * ((c * kPer + j) ^ swizzle<FMT, NR>(t))) = y[j];
    }
  };
  // A wave without a tile in a piece attends one without tokens.
  Piece cp = next_piece();        // attended now
  if (cp.tiles == 0) return;
  Piece np = next_piece();        // the one behind it
  Piece ahead = np;               // and the one behind that
  int ids_next = -1, ids = cp.ids;
  // Issue the loads of tile k of this piece, or of the next piece's first with its queries.
  auto load_tile = [&](int k) {
    const bool here = k < cp.count;
    if (!here && np.tiles == 0) return;
    asm volatile("" : "+s"(k));      // or the loop keeps copies of what depends on it, 40 registers of them
    const Where at = find((here ? tile_at(cp, cp.t0 + ws + STREAMS * k) : tile_at(np, np.t0 + ws)) * kCacheTile, here ? cp.len : np.len, here ? cp.h : np.h,
                          here ? ids : np.ids, here ? 2 * (k & 31) : 0);
    if (!here) load_q(np);
    load_k(at);
    load_v(at);
    if (!here) ahead = next_piece();
  };
  float x[kScores];
  {
    const Where at = find(tile_at(cp, cp.t0 + ws) * kCacheTile, cp.len, cp.h, cp.ids, 0);
    load_q(cp);
    load_k(at);
    load_v(at);
    scores(x, hidden(thread & 63));
    stage(hidden(thread & 63));
  }

  while (true) {
    const int n = cp.rows, M = n * p.G, len = cp.len, row0 = cp.row0, end = cp.end, h = cp.h, t0 = cp.t0;
    int tx = hidden(thread);
    const int lane = tx & 63, lr = lane % NR;
    uint32_t hole = gone;      // of the tile that x belongs to
    ids_next = pages_of(cp, 32);
    load_tile(1);

    Seen seen;
    if constexpr (kSeen<Args>) seen = seen_by(p, n, row0, end, len, (int)((uint32_t)(NR * half + lr) * p.g_inv >> 16));
    // tokens that the lane's row sees, and that every row sees
    const int64_t last = (int64_t)end - n + 1 + (int)((uint32_t)(NR * half + lr) * p.g_inv >> 16);
    const int limit = p.causal && last < len ? (last < 0 ? 0 : (int)last) : len;
    const int64_t first_last = (int64_t)end - n + 1;
    const int all_see = p.causal && first_last < len ? (first_last < 0 ? 0 : (int)first_last) : len;

    float m_run = kNegInf, l_run = 0.f;
    Acc acc[kAccs];
#pragma unroll
    for (int a = 0; a < kAccs; ++a) acc[a] = Acc{};

    int k = 0;
    do {
      const int lane = hidden(tx & 63);
      const int lr = lane % NR, lq = lane / NR;
      const int tok = tile_at(cp, t0 + ws + STREAMS * k) * kCacheTile;
      const bool mixed = kSeen<Args> ? !seen.whole(tok) : p.causal && tok + kCacheTile > all_see;
      uint32_t word = 0;         // tokens of the tile that the lane's row sees
      if constexpr (kSeen<Args>) {
        if (hole != 0 || mixed) {
          word = seen.word(tok) & ((hole & 1u ? 0u : 0xffffu) | (hole & 2u ? 0u : 0xffff0000u));
#pragma unroll
          for (int e = 0; e < kScores; ++e) {
            const int t = 4 * kGroups * (e >> 2) + 4 * lq + (e & 3);
            x[e] = (word >> t) & 1u ? x[e] : kNegInf;
          }
        }
      } else if (hole != 0 || tok + kCacheTile > all_see) {
#pragma unroll
        for (int e = 0; e < kScores; ++e) {
          const int t = 4 * kGroups * (e >> 2) + 4 * lq + (e & 3);
          x[e] = tok + t >= limit || ((hole >> (t >> 4)) & 1u) ? kNegInf : x[e];
        }
      }
      float mx = kNegInf;
#pragma unroll
      for (int e = 0; e < kScores; ++e) mx = fmaxf(mx, x[e]);
      mx *= p.scale_log2;
      if (__builtin_amdgcn_ballot_w64(mx > m_run + kSlack)) {
        const float mn = fmaxf(m_run, xgroup_max<kGroups>(mx));
        const float alpha = mn == kNegInf ? 1.f : exp2_fast(m_run - mn);
        l_run *= alpha;
#pragma unroll
        for (int a = 0; a < kAccs; ++a) acc[a] *= alpha;
        m_run = mn;
      }
      const float ms = m_run == kNegInf ? 0.f : m_run;
      if (mixed) {
        // Values that are no numbers at tokens that some rows see and others do
        // not: a weight of zero would spread them.  Such tokens, SS_MAX_CANDIDATES -
        // 1 at most (all of a tile that a window or a tree cuts), are then added one by one to the rows that see them, and
        // their V rows are cleared for the others.
        bool odd = false;
#pragma unroll
        for (int i = 0; i < kVTile / 1024; ++i) {
          const u32x4_t y = *reinterpret_cast<const u32x4_t *>(vs_lds + 1024 * i + 16 * lane);
#pragma unroll
          for (int e = 0; e < 4; ++e) odd |= (y[e] & 0x7f80u) == 0x7f80u || (y[e] & 0x7f800000u) == 0x7f800000u;
        }
        const int stop = __builtin_amdgcn_ballot_w64(odd) == 0 ? 0 : len - tok < kCacheTile ? len - tok : kCacheTile;
        for (int t = !kSeen<Args> && all_see > tok ? all_see - tok : 0; t < stop; ++t) {
          if (kSeen<Args> && __builtin_amdgcn_ballot_w64((word >> t) & 1u) == ~0ull) continue;
          unsigned char *row = vs_lds + t * kLdsRow;
          const int e = 4 * (t / (4 * kGroups)) + (t & 3);
          float xe = 0.f;
#pragma unroll
          for (int j = 0; j < kScores; ++j) xe = j == e ? x[j] : xe;
          xe = __shfl(xe, lr + NR * ((t >> 2) % kGroups));
          const float pe = exp2_fast(__builtin_fmaf(xe, p.scale_log2, -ms));
          if (kSeen<Args> ? (word >> t) & 1u : tok + t < limit) {
#pragma unroll
            for (int c = 0; c < kChans; ++c) {
              const int at = 4 * kGroups * c + 4 * lq;     // the piece's first channel
              const u32x2_t y = *reinterpret_cast<const u32x2_t *>(row + 16 * ((at >> 3) ^ swizzle<FMT, NR>(t)) + 8 * (lq & 1));
#pragma unroll
              for (int j = 0; j < 4; ++j)
                acc[4 * c / kRegs][4 * c % kRegs + j] += pe * __uint_as_float(j & 1 ? y[j >> 1] & 0xffff0000u : y[j >> 1] << 16);
            }
          }
          asm volatile("" ::: "memory");
          if (lane < 16) *reinterpret_cast<u32x4_t *>(row + 16 * lane) = u32x4_t{0u, 0u, 0u, 0u};
          asm volatile("" ::: "memory");
        }
      }

      // O^T += V^T P^T.  V's transpose read for k-step t: a 16-lane group's 4 rows
      // from 16 t + 4 lq on (and 4 kGroups further), 16 channels of the NR from
      // NR a on; lane i of the group addresses row i / 4, 4 channels from 4 (i % 4) on.
      // The swizzle leaves a row's 256 bytes aligned, so the accumulator's part of
      // the address is a flip of bits.
      const int li = lane & 15;
      const int vrow = 4 * lq + (li >> 2), chunk = (NR == 32 ? 2 * ((lane >> 4) & 1) : 0) + ((li & 3) >> 1);
      const uint32_t vat = (uint32_t)(uintptr_t)vs_lds + vrow * kLdsRow + 16 * (chunk ^ swizzle<FMT, NR>(vrow)) + 8 * (li & 1);
      bf16x8_t vop[kVSteps][kAccs];
#pragma unroll
      for (int t = 0; t < kVSteps; ++t)
#pragma unroll
        for (int a = 0; a < kAccs; ++a) {
          const uint32_t at = (vat ^ (NR * 2 * a)) + 16 * t * kLdsRow;
          const s16x4_t v0 = lds_read_tr16(at), v1 = lds_read_tr16(at + 4 * kGroups * kLdsRow);
          vop[t][a] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        }
#pragma unroll
      for (int t = 0; t < kVSteps; ++t) {
        u32x4_t part[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p0 = exp2_fast(__builtin_fmaf(x[8 * t + 2 * e], p.scale_log2, -ms));
          const float p1 = exp2_fast(__builtin_fmaf(x[8 * t + 2 * e + 1], p.scale_log2, -ms));
          l_run += p0;
          l_run += p1;
          uint32_t a, b, c;
          cut3(p0, p1, a, b, c);
          part[0][e] = a;
          part[1][e] = b;
          part[2][e] = c;
        }
#pragma unroll
        for (int j = 0; j < 3; ++j)
#pragma unroll
          for (int a = 0; a < kAccs; ++a) acc[a] = Mfma<NR>::run(vop[t][a], __builtin_bit_cast(bf16x8_t, part[j]), acc[a]);
      }
      // the next tile, maybe the next piece's first, in the shade of these products
      hole = gone;
      scores(x, lane);
      stage(lane);
      if (++k < cp.count) {
        if ((k & 31) == 31) {
          ids = ids_next;
          ids_next = pages_of(cp, k + 33);
        }
        load_tile(k + 1);
      }
    } while (k < cp.count);

    l_run = xgroup_sum<kGroups>(l_run);
    auto piece_of = [&](int c) {
      return f32x4_t{acc[4 * c / kRegs][4 * c % kRegs], acc[4 * c / kRegs][4 * c % kRegs + 1], acc[4 * c / kRegs][4 * c % kRegs + 2],
                     acc[4 * c / kRegs][4 * c % kRegs + 3]};
    };
    // Row r's state (m, l) with pieces a[k] of 4 channels, at every kSegs-th 4 channels from the seg-th on
    auto finish = [&](int r, int seg, auto segs, float m, float l, auto piece_at) {
      constexpr int kSegs = decltype(segs)::value, kPieces = kCacheDim / 4 / kSegs;
      if (cp.tiles == cp.whole) {
        const int i = (int)((uint32_t)r * p.g_inv >> 16);
        const int64_t row = ((int64_t)row0 + i) * p.Hq + h * p.G + r - i * p.G;
        if (row0 + i >= 0 && row0 + i < p.num_rows) {
          const RowEnd end = row_end(p, row, m, l);
#pragma unroll
          for (int k = 0; k < kPieces; ++k) {
            const int64_t o = row * kCacheDim + 4 * (seg + kSegs * k);
            *reinterpret_cast<f32x4_t *>(p.out + o) = row_value(p, end, o, piece_at(k));
          }
          if (seg == 0 && p.lse != nullptr) p.lse[row] = end.lse;
        }
      } else {
        // two states per worker at most: of a pair that starts before the share, and of one that ends behind it
        const int64_t o = (int64_t)(2 * worker + (t0 == 0 ? 1 : 0)) * p.M + r;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) *reinterpret_cast<f32x4_t *>(p.part_a + o * kCacheDim + 4 * (seg + kSegs * k)) = piece_at(k);
        if (seg == 0) *reinterpret_cast<f32x2_t *>(p.part_ml + 2 * o) = f32x2_t{m, l};
      }
    };
    if constexpr (kAlone) {
      const int lx = hidden(lane);
      const int r = lx % NR;
      if (r < M) finish(r, lx / NR, std::integral_constant<int, kGroups>{}, m_run, l_run, piece_of);
    } else {
    // The waves' states, first of waves 2 and 3 into those of waves 0 and 1 (of
    // the same rows), then what is left through LDS, kSegs threads to a row.
    __syncthreads();
    tx = hidden(thread);
    float *aw = reinterpret_cast<float *>(smem + kWaves * kVTile);
    float *mw = aw + 2 * NR * kAwPitch;
    float *lw = mw + 2 * NR;
    {
      const int lr = tx & (NR - 1), lq = (tx & 63) / NR;
      const int slot = (w & 1) * NR + lr;
      float *row = aw + slot * kAwPitch + 4 * lq;
      if (w >= 2) {
#pragma unroll
        for (int c = 0; c < kChans; ++c) *reinterpret_cast<f32x4_t *>(row + 4 * kGroups * c) = piece_of(c);
        if (lq == 0) {
          mw[slot] = m_run;
          lw[slot] = l_run;
        }
      }
      __syncthreads();
      if (w < 2) {
        const float mo = mw[slot], top = fmaxf(m_run, mo);
        // without a maximum both states are zero, or no number
        const float f = top == kNegInf ? 1.f : exp2_fast(m_run - top), fo = top == kNegInf ? 1.f : exp2_fast(mo - top);
        const float l = f * l_run + fo * lw[slot];
#pragma unroll
        for (int c = 0; c < kChans; ++c) {
          f32x4_t *at = reinterpret_cast<f32x4_t *>(row + 4 * kGroups * c);
          *at = f * piece_of(c) + fo * *at;
        }
        if (lq == 0) {       // the row's other lanes have read them: a wave runs in step
          mw[slot] = top;
          lw[slot] = l;
        }
      }
      __syncthreads();
    }
    constexpr int kAll = NR * HALVES, kSlots = 2 / HALVES;                 // rows of the piece; states of each
    constexpr int kSegs = kThreads / kAll;   // 16, 8 or 4 threads a row
    const int r = tx / kSegs, seg = tx % kSegs;
    if (r < M) {
      float mv[kSlots], top = kNegInf;
#pragma unroll
      for (int j = 0; j < kSlots; ++j) {
        mv[j] = mw[j * NR + r];
        top = fmaxf(top, mv[j]);
      }
      float f[kSlots], l = 0.f;
#pragma unroll
      for (int j = 0; j < kSlots; ++j) {
        f[j] = top == kNegInf ? 1.f : exp2_fast(mv[j] - top);
        l += f[j] * lw[j * NR + r];
      }
      finish(r, seg, std::integral_constant<int, kSegs>{}, top, l, [&](int k) {
        const float *at = aw + r * kAwPitch + 4 * (seg + kSegs * k);
        f32x4_t a = f[0] * *reinterpret_cast<const f32x4_t *>(at);
        if constexpr (kSlots == 2) a += f[1] * *reinterpret_cast<const f32x4_t *>(at + NR * kAwPitch);
        return a;
      });
    }
    }
    if (np.tiles == 0) break;
    cp = uniform(np);
    np = uniform(ahead);
    ids = cp.ids;
  }
}

// One head per workgroup up to this many rows x heads, so that the chip fills,
// four above.  Writes of 64 x 1, 32, 64 and 128 rows with 8 heads, one and four:
// 4.1 and 4.6 us, 4.7 and 4.9, 7.2 and 6.8, 12.9 and 10.9.
constexpr int64_t kFewRows = 1 << 14;

template <int FMT, typename F1, typename F4>
hipError_t launch_rows(const CacheRowsArgs &p, F1 one, F4 four, hipStream_t s) {
  const unsigned groups = (unsigned)((p.num_rows + (int64_t)kGroupRows - 1) / kGroupRows);
  const size_t lds = p.row_start == nullptr ? 0 : (2 * (size_t)p.B + 1) * sizeof(int32_t);
  if ((int64_t)p.num_rows * p.Hkv <= kFewRows)
    hipLaunchKernelGGL(one, dim3(groups, p.Hkv), dim3(kThreads), lds, s, p);
  else
    hipLaunchKernelGGL(four, dim3(groups, (p.Hkv + 3) / 4), dim3(kThreads), lds, s, p);
  return hipGetLastError();
}

template <int FMT, typename Args>
hipError_t attend(const Args &p, hipStream_t s) {
  if (p.alone) {
    const dim3 grid((p.workers + kWaves - 1) / kWaves);
    if (p.M <= 16)
      hipLaunchKernelGGL((cache_attend_kernel<FMT, 16, 1, 1, Args>), grid, dim3(kThreads), 0, s, p);
    else
      hipLaunchKernelGGL((cache_attend_kernel<FMT, 32, 1, 1, Args>), grid, dim3(kThreads), 0, s, p);
  } else if (p.M <= 16) {
    hipLaunchKernelGGL((cache_attend_kernel<FMT, 16, 1, 4, Args>), dim3(p.workers), dim3(kThreads), 0, s, p);
  } else if (p.M <= 32) {
    hipLaunchKernelGGL((cache_attend_kernel<FMT, 32, 1, 4, Args>), dim3(p.workers), dim3(kThreads), 0, s, p);
  } else {
    hipLaunchKernelGGL((cache_attend_kernel<FMT, 32, 2, 2, Args>), dim3(p.workers), dim3(kThreads), 0, s, p);
  }
  const hipError_t e = hipGetLastError();
  if constexpr (kSeen<Args>) {
    if (p.parts == 1) return e;
  }
  return e == hipSuccess ? launch_join(p, s) : e;
}

}  // namespace

CacheSplit cache_attend_split(int fmt, int B, int Hkv, int capacity, int M) {
  const int waves = attend_waves(fmt, M <= 16 ? 16 : 32);      // workgroups per CU
  const int64_t pairs = (int64_t)B * Hkv;
  CacheSplit r;
  // Waves by themselves, which merge nothing, where there are pairs for every
  // wave: with 256 to 2048 pairs of 0 to 600 tokens in 8 bits 15.5, 16.3, 21.4 and
  // 27.0 us, workgroups 13.9, 17.3, 24.6 and 39.5; of 500 to 4000 tokens in 4 bits
  // with 24 rows 39.7, 52.6, 84.2 and 163, workgroups 34.7, 51.6, 86.3 and 165.
  // More than 32 rows need two waves, so a worker there is always a workgroup.
  r.alone = M <= 32 && pairs >= 256 * kWaves;
  r.piece_units = r.alone ? kPieceAlone : kPieceGroup;
  const int64_t most = 256 * waves * (r.alone ? kWaves : 1);
  const int64_t units = pairs * ((capacity + kCacheTile - 1) / kCacheTile + r.piece_units);
  const int64_t need = (units + kMinShare - 1) / kMinShare;
  r.workers = (int)(need < most ? need : most);
  return r;
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

template <typename Args>
static hipError_t attend_of(const Args &p, int fmt, hipStream_t s) {
  if (fmt == kCacheBf16) return attend<kCacheBf16>(p, s);
  if (fmt == kCacheMx8) return attend<kCacheMx8>(p, s);
  return attend<kCacheMx4>(p, s);
}
hipError_t launch_cache_attend(const CacheAttendArgs &p, int fmt, hipStream_t s) { return attend_of(p, fmt, s); }
hipError_t launch_cache_attend_seen(const CacheSeenArgs &p, int fmt, hipStream_t s) { return attend_of(p, fmt, s); }

}  // namespace ss
