// Internal interface between the paged cache's host code (ss_cache_host.cpp) and
// its gfx950 kernels (ss_cache.hip).  Not part of the public ABI.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace ss {

constexpr int kCacheDim = 128;          // channels of a row
constexpr int kCacheTile = 32;          // tokens a wave attends per step
constexpr int kCacheMaxRequests = 4096; // requests of one call: 64 chunks of 64, and their starts and ends fit a workgroup's LDS
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

struct CacheAttendArgs : CacheArgs {
  const uint16_t *q;
  int64_t q_row_stride;
  float *out, *lse;                     // lse may be null
  const float *prev_out, *prev_lse;     // both or neither
  float *part_a, *part_ml;              // states of the pieces: [2 workers][M][128], [2 workers][M][2]
  int32_t Hq, G;
  uint32_t g_inv;                       // ceil(65536 / G): r / G = r * g_inv >> 16 for r < 64, G <= 64
  int32_t M;                            // rows per KV head: max_rows * G
  int32_t workers;                      // shares that the call's units are cut into
  int32_t alone;                        // a worker is a wave, not a workgroup
  int32_t piece_units;                  // what a piece costs beside its tiles, in tiles
  int32_t causal;
  float scale_log2;                     // softmax_scale * log2(e)
};

// How the attention over a cache of this kind is split; M query rows per KV head.
struct CacheSplit {
  int workers;
  bool alone;
  int piece_units;
};
CacheSplit cache_attend_split(int fmt, int B, int Hkv, int capacity, int M);

// Launch wrappers; return hipGetLastError() of the launch.
hipError_t launch_cache_write(const CacheRowsArgs &p, int fmt, hipStream_t s);
hipError_t launch_cache_read(const CacheRowsArgs &p, int fmt, hipStream_t s);
hipError_t launch_cache_attend(const CacheAttendArgs &p, int fmt, hipStream_t s);

}  // namespace ss
