// Host side of the paged cache: argument checks and launches.  A call keeps
// nothing: its tables and lengths are the caller's device arrays, so that a
// captured call follows them from replay to replay.
#include "specstream.h"

#include <cmath>

#include "ss_cache.h"
#include "ss_error.h"

namespace {

// the attention counts the requests in chunks of 64, one lane for each of 64 chunks at most
static_assert(SS_CACHE_MAX_REQUESTS <= ss::kCacheMaxRequests && ss::kCacheMaxRequests <= 64 * 64, "requests beyond a wave's chunks would be dropped");
// a workgroup of 256 threads takes 16 rows
static_assert(((int64_t)SS_CACHE_MAX_ROWS + 15) / 16 * 256 < (int64_t(1) << 32), "a launch's threads are counted in 32 bits");

using ss::fail;
using ss::hip_fail;

constexpr float kLog2e = 1.4426950408889634f;

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

ss_status check_desc(const ss_cache_desc *d) {
  if (d == nullptr) return fail(SS_ERR_INVALID_ARGUMENT, "cache descriptor is null");
  if (d->num_requests < 1) return fail(SS_ERR_INVALID_ARGUMENT, "num_requests must be >= 1 (got %d)", d->num_requests);
  if (d->num_requests > SS_CACHE_MAX_REQUESTS)
    return fail(SS_ERR_UNSUPPORTED, "num_requests %d > %d", d->num_requests, SS_CACHE_MAX_REQUESTS);
  if (d->num_kv_heads < 1) return fail(SS_ERR_INVALID_ARGUMENT, "num_kv_heads must be >= 1 (got %d)", d->num_kv_heads);
  if (d->num_kv_heads > SS_CACHE_MAX_KV_HEADS)
    return fail(SS_ERR_UNSUPPORTED, "num_kv_heads %d > %d", d->num_kv_heads, SS_CACHE_MAX_KV_HEADS);
  if (d->head_dim != ss::kCacheDim) return fail(SS_ERR_UNSUPPORTED, "head_dim %d is not built (only 128)", d->head_dim);
  if (d->format < SS_CACHE_BF16 || d->format > SS_CACHE_MXFP4)
    return fail(SS_ERR_INVALID_ARGUMENT, "format %d is none of the cache formats", d->format);
  if (d->page_tokens < 16 || d->page_tokens > 256 || (d->page_tokens & (d->page_tokens - 1)) != 0)
    return fail(SS_ERR_INVALID_ARGUMENT, "page_tokens must be 16, 32, 64, 128 or 256 (got %d)", d->page_tokens);
  if (d->num_pages < 1) return fail(SS_ERR_INVALID_ARGUMENT, "num_pages must be >= 1 (got %d)", d->num_pages);
  if (d->table_stride < 1) return fail(SS_ERR_INVALID_ARGUMENT, "table_stride must be >= 1 (got %d)", d->table_stride);
  const int64_t tokens = (int64_t)d->table_stride * d->page_tokens;
  if (tokens > (int64_t(1) << 30)) return fail(SS_ERR_UNSUPPORTED, "table_stride %d reaches more than 2^30 tokens", d->table_stride);
  // tiles of all requests and heads are counted in 32 bits
  const int64_t tiles = (tokens + ss::kCacheTile - 1) / ss::kCacheTile;
  if (tiles * d->num_requests > (int64_t(1) << 30) / d->num_kv_heads)
    return fail(SS_ERR_UNSUPPORTED, "num_requests x table_stride x num_kv_heads reaches more than 2^35 tokens");
  const int64_t page = (int64_t)d->num_kv_heads * ss::cache_head_bytes(d->format, d->page_tokens);
  if (d->page_stride != 0 && (d->page_stride < page || d->page_stride % 16 != 0))
    return fail(SS_ERR_INVALID_ARGUMENT, "page_stride must be 0 or a multiple of 16 of at least %lld bytes (got %lld)",
                (long long)page, (long long)d->page_stride);
  if (d->max_rows < 1) return fail(SS_ERR_INVALID_ARGUMENT, "max_rows must be >= 1 (got %d)", d->max_rows);
  return SS_OK;
}

ss_status check_attend_desc(const ss_cache_desc *d) {
  const ss_status s = check_desc(d);
  if (s != SS_OK) return s;
  if (d->num_q_heads < 1 || d->num_q_heads % d->num_kv_heads != 0)
    return fail(SS_ERR_INVALID_ARGUMENT, "num_q_heads must be a positive multiple of num_kv_heads (got %d, %d)",
                d->num_q_heads, d->num_kv_heads);
  if (d->max_rows > SS_MAX_CANDIDATES)
    return fail(SS_ERR_INVALID_ARGUMENT, "max_rows must be at most %d for an attention (got %d)", SS_MAX_CANDIDATES, d->max_rows);
  if ((int64_t)d->max_rows * (d->num_q_heads / d->num_kv_heads) > SS_MAX_ROWS_PER_KV_HEAD)
    return fail(SS_ERR_UNSUPPORTED, "rows per KV head %d x %d > %d", d->max_rows, d->num_q_heads / d->num_kv_heads,
                SS_MAX_ROWS_PER_KV_HEAD);
  if (!(d->softmax_scale > 0.f) || !std::isfinite(d->softmax_scale * kLog2e))
    return fail(SS_ERR_INVALID_ARGUMENT, "softmax_scale must be positive and finite, times log2(e) too (got %g)", (double)d->softmax_scale);
  if (d->causal != 0 && d->causal != 1) return fail(SS_ERR_INVALID_ARGUMENT, "causal must be 0 or 1 (got %d)", d->causal);
  return SS_OK;
}

// What a write and a read share beside check_call's: a launch has fewer than 2^32 threads.
ss_status check_rows(int32_t num_rows) {
  if (num_rows > SS_CACHE_MAX_ROWS) return fail(SS_ERR_UNSUPPORTED, "num_rows %d > %d", num_rows, SS_CACHE_MAX_ROWS);
  return SS_OK;
}

// The arguments that all calls share.
ss_status check_call(const ss_cache_desc *d, const void *pages, const int32_t *page_table, int32_t num_rows,
                     const int32_t *row_start, const int32_t *end, hipStream_t stream) {
  if (pages == nullptr || !aligned(pages, 16)) return fail(SS_ERR_INVALID_ARGUMENT, "pages must be non-null and 16-byte aligned");
  if (page_table == nullptr || end == nullptr || !aligned(page_table, 4) || !aligned(end, 4) || !aligned(row_start, 4))
    return fail(SS_ERR_INVALID_ARGUMENT, "page_table and end must be non-null, they and row_start 4-byte aligned");
  if (num_rows < 1) return fail(SS_ERR_INVALID_ARGUMENT, "num_rows must be >= 1 (got %d)", num_rows);
  if (row_start == nullptr && (int64_t)d->num_requests * d->max_rows != num_rows)
    return fail(SS_ERR_INVALID_ARGUMENT, "without row_start num_rows must be num_requests x max_rows (got %d, %d x %d)", num_rows,
                d->num_requests, d->max_rows);
  // a launch goes to the current device; on another device's stream it would
  // run where the caller's arrays are not
  int current = -1;
  hipDevice_t of_stream = -1;
  hipError_t e = hipGetDevice(&current);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  if (stream != nullptr) {
    e = hipStreamGetDevice(stream, &of_stream);
    if (e != hipSuccess) return hip_fail(e, "hipStreamGetDevice");
    if (of_stream != current)
      return fail(SS_ERR_INVALID_ARGUMENT, "the stream belongs to device %d, the current device is %d", (int)of_stream, current);
  }
  return SS_OK;
}

void fill(ss::CacheArgs *p, const ss_cache_desc *d, const void *pages, const int32_t *page_table, int32_t num_rows,
          const int32_t *row_start, const int32_t *end) {
  p->pages = static_cast<uint8_t *>(const_cast<void *>(pages));
  p->table = page_table;
  p->row_start = row_start;
  p->end = end;
  p->head_bytes = ss::cache_head_bytes(d->format, d->page_tokens);
  p->page_stride = d->page_stride != 0 ? (uint64_t)d->page_stride : (uint64_t)d->num_kv_heads * p->head_bytes;
  p->B = d->num_requests;
  p->Hkv = d->num_kv_heads;
  p->page_shift = __builtin_ctz((unsigned)d->page_tokens);
  p->num_pages = d->num_pages;
  p->table_stride = d->table_stride;
  p->capacity = d->table_stride << p->page_shift;
  p->num_rows = num_rows;
  p->max_rows = d->max_rows;
}

struct AttendLayout {
  int M;
  ss::CacheSplit split;
  size_t ml, bytes;   // offset of the maxima and sums; all of it
  explicit AttendLayout(const ss_cache_desc *d) {
    M = d->max_rows * (d->num_q_heads / d->num_kv_heads);
    split = ss::cache_attend_split(d->format, d->num_requests, d->num_kv_heads, d->table_stride * d->page_tokens, M);
    const size_t rows = 2 * (size_t)split.workers * (size_t)M;
    ml = rows * ss::kCacheDim * sizeof(float);
    bytes = (ml + rows * 2 * sizeof(float) + 255) / 256 * 256;
  }
};

}  // namespace

extern "C" {

size_t ss_cache_page_bytes(const ss_cache_desc *desc) {
  if (check_desc(desc) != SS_OK) return 0;
  return (size_t)desc->num_kv_heads * ss::cache_head_bytes(desc->format, desc->page_tokens);
}

size_t ss_cache_attend_workspace_bytes(const ss_cache_desc *desc) {
  if (check_attend_desc(desc) != SS_OK) return 0;
  return AttendLayout(desc).bytes;
}

ss_status ss_cache_write(const ss_cache_desc *desc, void *pages, const int32_t *page_table, const void *k, const void *v,
                         int64_t row_stride, int32_t num_rows, const int32_t *row_start, const int32_t *end,
                         hipStream_t stream) {
  ss_status s = check_desc(desc);
  if (s != SS_OK) return s;
  const int64_t packed = (int64_t)desc->num_kv_heads * ss::kCacheDim;
  if (k == nullptr || v == nullptr || !aligned(k, 16) || !aligned(v, 16))
    return fail(SS_ERR_INVALID_ARGUMENT, "k and v must be non-null and 16-byte aligned");
  if (row_stride != 0 && (row_stride < packed || row_stride % 8 != 0))
    return fail(SS_ERR_INVALID_ARGUMENT, "row_stride must be 0 or a multiple of 8 of at least %lld elements (got %lld)",
                (long long)packed, (long long)row_stride);
  s = check_rows(num_rows);
  if (s != SS_OK) return s;
  s = check_call(desc, pages, page_table, num_rows, row_start, end, stream);
  if (s != SS_OK) return s;
  ss::CacheRowsArgs p;
  fill(&p, desc, pages, page_table, num_rows, row_start, end);
  p.k = static_cast<uint16_t *>(const_cast<void *>(k));
  p.v = static_cast<uint16_t *>(const_cast<void *>(v));
  p.row_stride = row_stride != 0 ? row_stride : packed;
  p.head_stride = ss::kCacheDim;
  const hipError_t e = ss::launch_cache_write(p, desc->format, stream);
  return e == hipSuccess ? SS_OK : hip_fail(e, "cache write launch");
}

ss_status ss_cache_read(const ss_cache_desc *desc, const void *pages, const int32_t *page_table, void *k, void *v,
                        int32_t kv_layout, int32_t num_rows, const int32_t *row_start, const int32_t *end,
                        hipStream_t stream) {
  ss_status s = check_desc(desc);
  if (s != SS_OK) return s;
  if (k == nullptr || v == nullptr || !aligned(k, 16) || !aligned(v, 16))
    return fail(SS_ERR_INVALID_ARGUMENT, "k and v must be non-null and 16-byte aligned");
  if (kv_layout < SS_KV_TOKEN_MAJOR || kv_layout > SS_KV_HEAD_MAJOR_KV)
    return fail(SS_ERR_INVALID_ARGUMENT, "kv_layout %d is none of the chunk layouts", kv_layout);
  if (kv_layout == SS_KV_HEAD_MAJOR_KV && static_cast<uint16_t *>(v) != static_cast<uint16_t *>(k) + ss::kCacheDim)
    return fail(SS_ERR_INVALID_ARGUMENT, "SS_KV_HEAD_MAJOR_KV takes v = k + head_dim elements");
  s = check_rows(num_rows);
  if (s != SS_OK) return s;
  s = check_call(desc, pages, page_table, num_rows, row_start, end, stream);
  if (s != SS_OK) return s;
  ss::CacheRowsArgs p;
  fill(&p, desc, pages, page_table, num_rows, row_start, end);
  p.k = static_cast<uint16_t *>(k);
  p.v = static_cast<uint16_t *>(v);
  const int64_t d = ss::kCacheDim;
  p.row_stride = kv_layout == SS_KV_TOKEN_MAJOR ? d * desc->num_kv_heads : kv_layout == SS_KV_HEAD_MAJOR ? d : 2 * d;
  p.head_stride = kv_layout == SS_KV_TOKEN_MAJOR ? d : p.row_stride * num_rows;
  const hipError_t e = ss::launch_cache_read(p, desc->format, stream);
  return e == hipSuccess ? SS_OK : hip_fail(e, "cache read launch");
}

ss_status ss_cache_attend(const ss_cache_desc *desc, const void *pages, const int32_t *page_table, const void *q,
                          int64_t q_row_stride, int32_t num_rows, const int32_t *row_start, const int32_t *end,
                          float *out, float *lse, const float *prev_out, const float *prev_lse, void *workspace,
                          size_t workspace_bytes, hipStream_t stream) {
  ss_status s = check_attend_desc(desc);
  if (s != SS_OK) return s;
  const int64_t packed = (int64_t)desc->num_q_heads * ss::kCacheDim;
  if (q == nullptr || out == nullptr || !aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4))
    return fail(SS_ERR_INVALID_ARGUMENT, "q and out must be non-null and 16-byte aligned, lse null or 4-byte aligned");
  if (q_row_stride != 0 && (q_row_stride < packed || q_row_stride % 8 != 0))
    return fail(SS_ERR_INVALID_ARGUMENT, "q_row_stride must be 0 or a multiple of 8 of at least %lld elements (got %lld)",
                (long long)packed, (long long)q_row_stride);
  if ((prev_out == nullptr) != (prev_lse == nullptr))
    return fail(SS_ERR_INVALID_ARGUMENT, "prev_out and prev_lse come together");
  if (!aligned(prev_out, 16) || !aligned(prev_lse, 4))
    return fail(SS_ERR_INVALID_ARGUMENT, "prev_out must be 16-byte and prev_lse 4-byte aligned");
  const AttendLayout layout(desc);
  if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < layout.bytes)
    return fail(SS_ERR_WORKSPACE, "workspace must be 256-byte aligned and hold %zu bytes (got %p, %zu)", layout.bytes, workspace,
                workspace_bytes);
  s = check_call(desc, pages, page_table, num_rows, row_start, end, stream);
  if (s != SS_OK) return s;
  ss::CacheAttendArgs p;
  fill(&p, desc, pages, page_table, num_rows, row_start, end);
  p.q = static_cast<const uint16_t *>(q);
  p.q_row_stride = q_row_stride != 0 ? q_row_stride : packed;
  p.out = out;
  p.lse = lse;
  p.prev_out = prev_out;
  p.prev_lse = prev_lse;
  p.part_a = static_cast<float *>(workspace);
  p.part_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) + layout.ml);
  p.Hq = desc->num_q_heads;
  p.G = desc->num_q_heads / desc->num_kv_heads;
  p.g_inv = (65536u + (uint32_t)p.G - 1) / (uint32_t)p.G;
  p.M = layout.M;
  p.workers = layout.split.workers;
  p.alone = layout.split.alone;
  p.piece_units = layout.split.piece_units;
  p.causal = desc->causal;
  p.scale_log2 = desc->softmax_scale * kLog2e;
  const hipError_t e = ss::launch_cache_attend(p, desc->format, stream);
  return e == hipSuccess ? SS_OK : hip_fail(e, "cache attention launch");
}

}  // extern "C"
