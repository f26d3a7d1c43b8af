// Internal interface between the paged cache's host code (ss_cache_host.cpp) and
// its gfx950 kernels (ss_cache.hip).  Not part of the public ABI.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace ss {

constexpr int kCacheDim = 128;          // channels of a row
constexpr int kCacheTile = 32;          // tokens a wave attends per step
constexpr int kCacheMaxRequests = 4096; // requests of one call: 64 chunks of 64, and their starts and ends fit a workgroup's LDS
constexpr int kCacheMaxTree = 64;       // rows of a tree: bits of a row's word
constexpr int kCacheBf16 = 0, kCacheMx8 = 1, kCacheMx4 = 2;

// Bytes of one K or V row and of its scales, by format.
constexpr int cache_row_bytes(int fmt) { return fmt == kCacheBf16 ? 256 : fmt == kCacheMx8 ? 128 : 64; }
constexpr int cache_scale_bytes(int fmt) { return fmt == kCacheBf16 ? 0 : 4; }
// A page holds, per KV head, a block of K rows, V rows, K scales, V scales.
constexpr uint32_t cache_head_bytes(int fmt, int page_tokens) {
  return (uint32_t)page_tokens * 2u * (uint32_t)(cache_row_bytes(fmt) + cache_scale_bytes(fmt));
}

// The cache and the rows of a call, as every kernel reads them.
struct CacheArgs {
  uint8_t *pages;
  const int32_t *table;      // [B][table_stride]: page of each page_tokens tokens
  const int32_t *row_start;  // [B + 1], or null: max_rows rows each
  const int32_t *end;        // [B]: tokens of the request once its rows are in
  uint64_t page_stride;      // bytes between pages
  uint32_t head_bytes;       // bytes between the heads' blocks of a page
  int32_t B, Hkv;
  int32_t page_shift;        // log2 of the tokens per page
  int32_t num_pages, table_stride;
  int32_t capacity;          // table_stride << page_shift: tokens a request's table reaches
  int32_t num_rows, max_rows;
};

struct CacheRowsArgs : CacheArgs {
  uint16_t *k, *v;           // bf16 rows: read by the write, written by the read
  int64_t row_stride;        // elements between a row and the next
  int64_t head_stride;       // elements between a KV head and the next
};

struct CacheAppendArgs : CacheArgs {
  const uint16_t *k, *v, *q;       // bf16 rows; q may be null
  uint16_t *q_out;                 // may be q
  int64_t row_stride, q_row_stride, q_out_row_stride;
  const int32_t *positions;        // [num_rows], or null: the tokens' own
  const float *inv_freq;           // [rotary_dim / 2]
  float scale;                     // of sine and cosine
  int32_t Hq;
  int32_t rotary_dim;              // channels that turn, a multiple of 16
  int32_t interleaved;             // pairs are neighbours, not half of rotary_dim apart
};

struct CacheKeepArgs : CacheArgs {
  const int32_t *kept;             // [num_rows]: request b's from its first row's place on
  const int32_t *num_kept;         // [B]
};

struct CacheAttendArgs : CacheArgs {
  const uint16_t *q;
  int64_t q_row_stride;
  float *out, *lse;                     // lse may be null
  const float *prev_out, *prev_lse;     // both or neither
  float *part_a, *part_ml;              // states of the pieces: [2 workers][rows][128], [2 workers][rows][2]; rows: M, of a block in groups
  int32_t Hq, G;
  uint32_t g_inv;                       // ceil(65536 / G): r / G = r * g_inv >> 16 where r * G < 65536 (r < 512, G <= 64)
  int32_t M;                            // rows per KV head: max_rows * G
  int32_t workers;                      // shares that the call's units are cut into
  int32_t alone;                        // a worker is a wave, not a workgroup
  int32_t piece_units;                  // what a piece costs beside its tiles, in tiles
  int32_t causal;
  float scale_log2;                     // softmax_scale * log2(e)
};

// Rows of one KV head that a piece of the attention of many rows holds at most (more are attended in blocks of as many), and
// the tokens of its tiles.
constexpr int kCacheGroupBlock = 128, kCacheGroupTile = 32;
constexpr int kCacheMaxRows = 64;      // rows per KV head of the other attentions

// Rows that see a tree, or a window and the first tokens, instead of a chain.
struct CacheSeenArgs : CacheAttendArgs {
  const uint64_t *tree;   // [num_rows]: bit j: the row sees the request's j-th row's token; null: a chain
  int32_t window;         // tokens up to its own that a row sees of those before the request's rows; 0: all
  int32_t sinks;          // first tokens that it sees as well
  int32_t parts;          // a worker has one of as many parts of a (request, KV head, block of rows); 0: shares of all the units
};

struct CacheGroupArgs : CacheSeenArgs {};

// How the attention over a cache of this kind is split; M query rows per KV head.
struct CacheSplit {
  int workers;
  bool alone;
  int piece_units;
};
CacheSplit cache_attend_split(int fmt, int B, int Hkv, int capacity, int M);
// From how many rows per KV head on the rows of a tree are attended in groups, and how that is split.
// 16 x 32768 tokens with 40 and 64 rows in bf16 465 and 481 us, with waves for themselves 516 and 528; in 8
// bits 587 and 595, 368 and 385; in 4 bits 566 and 568, 311 and 324; 96 rows in 8 bits 617 and, as two blocks of waves, 707.
constexpr int cache_group_rows(int fmt) { return fmt == kCacheBf16 ? 33 : 65; }
CacheSplit cache_group_split(int fmt, int B, int Hkv, int capacity, int M);
// Into how many parts of as many tiles (of 32 tokens) each of `wholes` (request, KV head, block of rows) is cut, a workgroup to a
// part, with at most `most` workgroups; 1: nothing to join; 0: cut by the lengths, into equal shares of all the units.
// Few tiles are not cut.  One request, 8 KV heads, 64 rows on 32 heads in bf16: 4 tiles 14.1 us, cut 16.5; 8 tiles 19.2 and 17.9;
// 16 tiles 29.4 and 18.6.  16 requests of one row over 10 tiles 11.4 and 15.8.
// Where a window makes the lengths alike, equal parts save the 2 to 5 us in which a worker finds its share.  The lengths themselves lie on
// the device, though, and where one request fills its window and the others hold 40 tokens the call waits for its parts' workgroups
// alone.  So parts are short.  Parts and shares, us, all windows full and one alone:
//   16 requests of 8 rows, 64 per KV head, 4 bits, window 1024 (18 tiles a part) 28.5, 32.9 and 26.2, 23.3; 4096 (66) 61.8, 58.0 and 59.7, 30.3
//   64 requests of one row, bf16, window 512 (18) 27.7, 30.1 and 18.5, 19.4; 1024 (34) 45.7, 48.0 and 29.4, 19.1; 4096 (132) 168, 171 and 90.6, 26.1
//   16 trees of 32 rows, 128 per KV head, 8 bits, window 1024 (9) 43.8, 45.7 and 39.4, 31.3; 2048 (17) 62.0, 65.2 and 55.6, 35.7; 4096 (33) 95.8,
//   98.6 and 89.6, 42.8
constexpr int kCachePartTiles = 20, kCacheGroupPartTiles = 10;     // of the longest part
inline int cache_attend_parts(int64_t tiles, int64_t wholes, int64_t most, bool alike, bool group) {
  if (tiles <= (wholes < 64 ? 4 : 16)) return 1;
  if (!alike) return 0;
  int64_t parts = most / wholes;
  parts = parts > tiles / 4 ? tiles / 4 : parts;
  parts = parts < 1 ? 1 : parts;
  return (tiles + parts - 1) / parts <= (group ? kCacheGroupPartTiles : kCachePartTiles) ? (int)parts : 0;
}

// Launch wrappers; return hipGetLastError() of the launch.
hipError_t launch_cache_write(const CacheRowsArgs &p, int fmt, hipStream_t s);
hipError_t launch_cache_read(const CacheRowsArgs &p, int fmt, hipStream_t s);
hipError_t launch_cache_attend(const CacheAttendArgs &p, int fmt, hipStream_t s);
hipError_t launch_cache_append(const CacheAppendArgs &p, int fmt, hipStream_t s);
hipError_t launch_cache_keep(const CacheKeepArgs &p, int fmt, hipStream_t s);
hipError_t launch_cache_attend_seen(const CacheSeenArgs &p, int fmt, hipStream_t s);
hipError_t launch_cache_attend_group(const CacheGroupArgs &p, int fmt, hipStream_t s);

}  // namespace ss
