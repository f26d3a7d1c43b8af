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
// a row's word has a bit for every node; keeping a path holds a tree's rows in registers
static_assert(SS_CACHE_MAX_TREE == ss::kCacheMaxTree && SS_CACHE_MAX_TREE == 64, "nodes of a tree are bits of 64");
// rows of a KV head are divided by G with a multiplication, exact where row x G < 2^16
static_assert(SS_CACHE_MAX_TREE_ROWS_PER_KV_HEAD * SS_MAX_ROWS_PER_KV_HEAD < 65536, "a row's query and head come from a multiplication");
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

// most, most_per_head: rows of a request, and of them and the query heads on one KV head
ss_status check_attend_desc(const ss_cache_desc *d, int most = SS_MAX_CANDIDATES, int most_per_head = SS_MAX_ROWS_PER_KV_HEAD) {
  const ss_status s = check_desc(d);
  if (s != SS_OK) return s;
  if (d->num_q_heads < 1 || d->num_q_heads % d->num_kv_heads != 0)
    return fail(SS_ERR_INVALID_ARGUMENT, "num_q_heads must be a positive multiple of num_kv_heads (got %d, %d)",
                d->num_q_heads, d->num_kv_heads);
  if (d->max_rows > most)
    return fail(SS_ERR_INVALID_ARGUMENT, "max_rows must be at most %d for an attention (got %d)", most, d->max_rows);
  if ((int64_t)d->max_rows * (d->num_q_heads / d->num_kv_heads) > most_per_head)
    return fail(SS_ERR_UNSUPPORTED, "rows per KV head %d x %d > %d", d->max_rows, d->num_q_heads / d->num_kv_heads, most_per_head);
  if (!(d->softmax_scale > 0.f) || !std::isfinite(d->softmax_scale * kLog2e))
    return fail(SS_ERR_INVALID_ARGUMENT, "softmax_scale must be positive and finite, times log2(e) too (got %g)", (double)d->softmax_scale);
  if (d->causal != 0 && d->causal != 1) return fail(SS_ERR_INVALID_ARGUMENT, "causal must be 0 or 1 (got %d)", d->causal);
  return SS_OK;
}

ss_status check_tree_desc(const ss_cache_desc *d) {
  const ss_status s = check_attend_desc(d, SS_CACHE_MAX_TREE, SS_CACHE_MAX_TREE_ROWS_PER_KV_HEAD);
  if (s != SS_OK) return s;
  if (d->num_q_heads / d->num_kv_heads > SS_MAX_ROWS_PER_KV_HEAD)
    return fail(SS_ERR_UNSUPPORTED, "query heads per KV head %d > %d", d->num_q_heads / d->num_kv_heads, SS_MAX_ROWS_PER_KV_HEAD);
  // a launch's grid has a workgroup for every row and head of a request, at most
  if ((int64_t)d->max_rows * d->num_q_heads > 32768)
    return fail(SS_ERR_UNSUPPORTED, "max_rows x num_q_heads %d x %d > 32768", d->max_rows, d->num_q_heads);
  // tiles of all requests, heads and blocks of rows are counted in 32 bits
  const int64_t tiles = ((int64_t)d->table_stride * d->page_tokens + ss::kCacheTile - 1) / ss::kCacheTile * d->num_requests;
  const int blocks = (d->max_rows * (d->num_q_heads / d->num_kv_heads) + ss::kCacheGroupBlock - 1) / ss::kCacheGroupBlock;
  if (tiles > (int64_t(1) << 30) / d->num_kv_heads / blocks)
    return fail(SS_ERR_UNSUPPORTED, "num_requests x table_stride x num_kv_heads x %d blocks of rows reaches more than 2^35 tokens", blocks);
  return SS_OK;
}

ss_status check_window(int32_t window, int32_t sinks, int32_t least) {
  if (window < least || sinks < 0)
    return fail(SS_ERR_INVALID_ARGUMENT, "window must be >= %d and sinks >= 0 (got %d, %d)", least, window, sinks);
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

static_assert(ss::kCacheMaxRows == SS_MAX_ROWS_PER_KV_HEAD, "more rows are attended in groups");

struct AttendLayout {
  int M, blocks;      // rows per KV head, and the blocks that they are attended in
  bool group;         // attended by the kernel of many rows
  ss::CacheSplit split;
  size_t ml, bytes;   // offset of the maxima and sums; all of it
  explicit AttendLayout(const ss_cache_desc *d, bool grouped = false) {      // grouped: many rows may be
    M = d->max_rows * (d->num_q_heads / d->num_kv_heads);
    group = grouped && M >= ss::cache_group_rows(d->format);
    const int reach = d->table_stride * d->page_tokens;
    blocks = group ? (M + ss::kCacheGroupBlock - 1) / ss::kCacheGroupBlock : 1;
    split = group ? ss::cache_group_split(d->format, d->num_requests, d->num_kv_heads, reach, M)
                  : ss::cache_attend_split(d->format, d->num_requests, d->num_kv_heads, reach, M);
    const size_t rows = 2 * (size_t)split.workers * (size_t)(blocks > 1 ? ss::kCacheGroupBlock : M);
    ml = rows * ss::kCacheDim * sizeof(float);
    bytes = (ml + rows * 2 * sizeof(float) + 255) / 256 * 256;
  }
};

// What the rows of a tree or in a window see, and whether the call is cut into parts.
void fill_seen(ss::CacheSeenArgs *p, const ss_cache_desc *d, const AttendLayout &layout, const uint64_t *tree, int32_t window, int32_t sinks) {
  p->tree = tree;
  p->window = window;
  p->sinks = sinks;
  int64_t reach = p->capacity;
  // a window's tokens begin and end within a tile, and so do the first ones
  if (window > 0 && (int64_t)window + sinks + d->max_rows < reach) reach = (int64_t)window + sinks + d->max_rows + 3 * ss::kCacheTile;
  const int wholes = p->B * p->Hkv * layout.blocks;
  // workgroups a CU: two for groups (16 trees of 32 rows in a window of 1024 43.3 us, with one, whose parts are too long, 45.7), else one
  // (16 requests of 8 rows, 64 per KV head, in a window of 1024 28.0, two 29.3)
  const int fill = layout.group ? 512 : 256, most = p->workers < fill ? p->workers : fill;
  p->parts = layout.split.alone ? 0 : ss::cache_attend_parts((reach + ss::kCacheTile - 1) / ss::kCacheTile, wholes, most, reach < p->capacity, layout.group);
  if (p->parts > 0) p->workers = wholes * p->parts;
}

// The checks and arguments that the attentions share, once the descriptor is checked.
ss_status prepare_attend(ss::CacheAttendArgs *p, const AttendLayout &layout, const ss_cache_desc *desc, const void *pages, const int32_t *page_table, const void *q,
                         int64_t q_row_stride, int32_t num_rows, const int32_t *row_start, const int32_t *end, float *out, float *lse,
                         const float *prev_out, const float *prev_lse, void *workspace, size_t workspace_bytes, hipStream_t stream) {
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
  if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < layout.bytes)
    return fail(SS_ERR_WORKSPACE, "workspace must be 256-byte aligned and hold %zu bytes (got %p, %zu)", layout.bytes, workspace,
                workspace_bytes);
  const ss_status s = check_call(desc, pages, page_table, num_rows, row_start, end, stream);
  if (s != SS_OK) return s;
  fill(p, desc, pages, page_table, num_rows, row_start, end);
  p->q = static_cast<const uint16_t *>(q);
  p->q_row_stride = q_row_stride != 0 ? q_row_stride : packed;
  p->out = out;
  p->lse = lse;
  p->prev_out = prev_out;
  p->prev_lse = prev_lse;
  p->part_a = static_cast<float *>(workspace);
  p->part_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) + layout.ml);
  p->Hq = desc->num_q_heads;
  p->G = desc->num_q_heads / desc->num_kv_heads;
  p->g_inv = (65536u + (uint32_t)p->G - 1) / (uint32_t)p->G;
  p->M = layout.M;
  p->workers = layout.split.workers;
  p->alone = layout.split.alone;
  p->piece_units = layout.split.piece_units;
  p->causal = desc->causal;
  p->scale_log2 = desc->softmax_scale * kLog2e;
  return SS_OK;
}

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
  ss::CacheAttendArgs p;
  s = prepare_attend(&p, AttendLayout(desc), desc, pages, page_table, q, q_row_stride, num_rows, row_start, end, out, lse, prev_out, prev_lse, workspace,
                     workspace_bytes, stream);
  if (s != SS_OK) return s;
  const hipError_t e = ss::launch_cache_attend(p, desc->format, stream);
  return e == hipSuccess ? SS_OK : hip_fail(e, "cache attention launch");
}

size_t ss_cache_attend_tree_workspace_bytes(const ss_cache_desc *desc) {
  if (check_tree_desc(desc) != SS_OK) return 0;
  return AttendLayout(desc, true).bytes;
}

ss_status ss_cache_attend_tree(const ss_cache_desc *desc, const void *pages, const int32_t *page_table, const uint64_t *tree,
                               int32_t window, int32_t sinks, const void *q, int64_t q_row_stride, int32_t num_rows,
                               const int32_t *row_start, const int32_t *end, float *out, float *lse, const float *prev_out,
                               const float *prev_lse, void *workspace, size_t workspace_bytes, hipStream_t stream) {
  ss_status s = check_tree_desc(desc);
  if (s != SS_OK) return s;
  if (tree == nullptr || !aligned(tree, 8)) return fail(SS_ERR_INVALID_ARGUMENT, "tree must be non-null and 8-byte aligned");
  s = check_window(window, sinks, 0);
  if (s != SS_OK) return s;
  const AttendLayout layout(desc, true);
  ss::CacheGroupArgs p;
  s = prepare_attend(&p, layout, desc, pages, page_table, q, q_row_stride, num_rows, row_start, end, out, lse, prev_out, prev_lse, workspace,
                     workspace_bytes, stream);
  if (s != SS_OK) return s;
  fill_seen(&p, desc, layout, tree, window, sinks);
  const hipError_t e = layout.group ? ss::launch_cache_attend_group(p, desc->format, stream)
                                    : ss::launch_cache_attend_seen(p, desc->format, stream);
  return e == hipSuccess ? SS_OK : hip_fail(e, "cache tree attention launch");
}

ss_status ss_cache_attend_window(const ss_cache_desc *desc, const void *pages, const int32_t *page_table, int32_t window,
                                 int32_t sinks, const void *q, int64_t q_row_stride, int32_t num_rows, const int32_t *row_start,
                                 const int32_t *end, float *out, float *lse, const float *prev_out, const float *prev_lse,
                                 void *workspace, size_t workspace_bytes, hipStream_t stream) {
  ss_status s = check_attend_desc(desc);
  if (s != SS_OK) return s;
  if (desc->causal != 1) return fail(SS_ERR_INVALID_ARGUMENT, "a window takes causal = 1");
  s = check_window(window, sinks, 1);
  if (s != SS_OK) return s;
  const AttendLayout layout(desc);
  ss::CacheSeenArgs p;
  s = prepare_attend(&p, layout, desc, pages, page_table, q, q_row_stride, num_rows, row_start, end, out, lse, prev_out, prev_lse, workspace,
                     workspace_bytes, stream);
  if (s != SS_OK) return s;
  fill_seen(&p, desc, layout, nullptr, window, sinks);
  const hipError_t e = ss::launch_cache_attend_seen(p, desc->format, stream);
  return e == hipSuccess ? SS_OK : hip_fail(e, "cache window attention launch");
}

ss_status ss_cache_append(const ss_cache_desc *desc, void *pages, const int32_t *page_table, const ss_rope_desc *rope,
                          const int32_t *positions, const void *k, const void *v, int64_t row_stride, const void *q,
                          int64_t q_row_stride, void *q_out, int64_t q_out_row_stride, int32_t num_rows,
                          const int32_t *row_start, const int32_t *end, hipStream_t stream) {
  ss_status s = check_desc(desc);
  if (s != SS_OK) return s;
  if (rope == nullptr) return fail(SS_ERR_INVALID_ARGUMENT, "rope descriptor is null");
  if (rope->rotary_dim < 1 || rope->rotary_dim > ss::kCacheDim)
    return fail(SS_ERR_INVALID_ARGUMENT, "rotary_dim must be 1..%d (got %d)", ss::kCacheDim, rope->rotary_dim);
  if (rope->rotary_dim % 16 != 0) return fail(SS_ERR_UNSUPPORTED, "rotary_dim %d is not built (only multiples of 16)", rope->rotary_dim);
  if (rope->interleaved != 0 && rope->interleaved != 1)
    return fail(SS_ERR_INVALID_ARGUMENT, "interleaved must be 0 or 1 (got %d)", rope->interleaved);
  if (!(rope->scale > 0.f) || !std::isfinite(rope->scale))
    return fail(SS_ERR_INVALID_ARGUMENT, "rope scale must be positive and finite (got %g)", (double)rope->scale);
  if (rope->inv_freq == nullptr || !aligned(rope->inv_freq, 4) || !aligned(positions, 4))
    return fail(SS_ERR_INVALID_ARGUMENT, "inv_freq must be non-null, it and positions 4-byte aligned");
  const int64_t packed = (int64_t)desc->num_kv_heads * ss::kCacheDim;
  if (k == nullptr || v == nullptr || !aligned(k, 16) || !aligned(v, 16))
    return fail(SS_ERR_INVALID_ARGUMENT, "k and v must be non-null and 16-byte aligned");
  if (row_stride != 0 && (row_stride < packed || row_stride % 8 != 0))
    return fail(SS_ERR_INVALID_ARGUMENT, "row_stride must be 0 or a multiple of 8 of at least %lld elements (got %lld)",
                (long long)packed, (long long)row_stride);
  if ((q == nullptr) != (q_out == nullptr)) return fail(SS_ERR_INVALID_ARGUMENT, "q and q_out come together");
  int64_t q_packed = 0;
  if (q != nullptr) {
    if (!aligned(q, 16) || !aligned(q_out, 16)) return fail(SS_ERR_INVALID_ARGUMENT, "q and q_out must be 16-byte aligned");
    if (desc->num_q_heads < 1 || desc->num_q_heads % desc->num_kv_heads != 0)
      return fail(SS_ERR_INVALID_ARGUMENT, "num_q_heads must be a positive multiple of num_kv_heads (got %d, %d)", desc->num_q_heads,
                  desc->num_kv_heads);
    // a launch's grid has a workgroup for every two query heads, at most
    if (desc->num_q_heads > 65536) return fail(SS_ERR_UNSUPPORTED, "num_q_heads %d > 65536", desc->num_q_heads);
    q_packed = (int64_t)desc->num_q_heads * ss::kCacheDim;
    for (const int64_t stride : {q_row_stride, q_out_row_stride})
      if (stride != 0 && (stride < q_packed || stride % 8 != 0))
        return fail(SS_ERR_INVALID_ARGUMENT, "q_row_stride and q_out_row_stride must be 0 or a multiple of 8 of at least %lld elements (got %lld)",
                    (long long)q_packed, (long long)stride);
    if (q == q_out && (q_row_stride != 0 ? q_row_stride : q_packed) != (q_out_row_stride != 0 ? q_out_row_stride : q_packed))
      return fail(SS_ERR_INVALID_ARGUMENT, "q_out may be q with the same row stride only");
  }
  s = check_rows(num_rows);
  if (s != SS_OK) return s;
  s = check_call(desc, pages, page_table, num_rows, row_start, end, stream);
  if (s != SS_OK) return s;
  ss::CacheAppendArgs p;
  fill(&p, desc, pages, page_table, num_rows, row_start, end);
  p.k = static_cast<const uint16_t *>(k);
  p.v = static_cast<const uint16_t *>(v);
  p.q = static_cast<const uint16_t *>(q);
  p.q_out = static_cast<uint16_t *>(q_out);
  p.row_stride = row_stride != 0 ? row_stride : packed;
  p.q_row_stride = q_row_stride != 0 ? q_row_stride : q_packed;
  p.q_out_row_stride = q_out_row_stride != 0 ? q_out_row_stride : q_packed;
  p.positions = positions;
  p.inv_freq = rope->inv_freq;
  p.scale = rope->scale;
  p.Hq = desc->num_q_heads;
  p.rotary_dim = rope->rotary_dim;
  p.interleaved = rope->interleaved;
  const hipError_t e = ss::launch_cache_append(p, desc->format, stream);
  return e == hipSuccess ? SS_OK : hip_fail(e, "cache append launch");
}

ss_status ss_cache_keep(const ss_cache_desc *desc, void *pages, const int32_t *page_table, const int32_t *kept,
                        const int32_t *num_kept, int32_t num_rows, const int32_t *row_start, const int32_t *end,
                        hipStream_t stream) {
  ss_status s = check_desc(desc);
  if (s != SS_OK) return s;
  if (desc->max_rows > SS_CACHE_MAX_TREE)
    return fail(SS_ERR_INVALID_ARGUMENT, "max_rows must be at most %d to keep a path (got %d)", SS_CACHE_MAX_TREE, desc->max_rows);
  if (kept == nullptr || num_kept == nullptr || !aligned(kept, 4) || !aligned(num_kept, 4))
    return fail(SS_ERR_INVALID_ARGUMENT, "kept and num_kept must be non-null and 4-byte aligned");
  s = check_call(desc, pages, page_table, num_rows, row_start, end, stream);
  if (s != SS_OK) return s;
  ss::CacheKeepArgs p;
  fill(&p, desc, pages, page_table, num_rows, row_start, end);
  p.kept = kept;
  p.num_kept = num_kept;
  const hipError_t e = ss::launch_cache_keep(p, desc->format, stream);
  return e == hipSuccess ? SS_OK : hip_fail(e, "cache keep launch");
}

}  // extern "C"
