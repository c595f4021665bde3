// Host side of the latent cache, of attention over it and over dense rows: argument validation and launches.
// Every argument is checked before the first launch; nothing allocates, synchronises or keeps state.
#include <cmath>

#include "scd_latent.h"
#include "scd_serve_host.h"

namespace {

using namespace scd;

constexpr int64_t kMostWorkgroups = (int64_t{1} << 23) - 1;  // of 512 threads: below 2^32 in a launch
constexpr double kLog2e = 1.4426950408889634;

scd_status_t check_latent_shape(const scd_latent_cache_t* c) {
  if (c == nullptr) return fail(SCD_ERR_NULL, "cache is NULL");
  if (c->n_pages < 1 || c->max_pages < 1)
    return fail(SCD_ERR_SHAPE, "cache needs n_pages and max_pages >= 1 (got %d, %d)", c->n_pages, c->max_pages);
  if (c->latent_dim < 32 || c->latent_dim > 512 || c->latent_dim % 32 != 0)
    return fail(SCD_ERR_UNSUPPORTED, "latent_dim %d unsupported (multiples of 32 up to 512)", c->latent_dim);
  if (c->turned_dim != 32 && c->turned_dim != 64)
    return fail(SCD_ERR_UNSUPPORTED, "turned_dim %d unsupported (32 or 64)", c->turned_dim);
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128)
    return fail(SCD_ERR_UNSUPPORTED, "page_tokens %d unsupported (16, 32, 64 or 128)", c->page_tokens);
  return SCD_OK;
}

scd_status_t check_latent(const scd_latent_cache_t* c) {
  SCD_TRY(check_latent_shape(c));
  if (c->pages == nullptr) return fail(SCD_ERR_NULL, "pages is NULL");
  if (!aligned16(c->pages)) return fail(SCD_ERR_ALIGN, "pages is not 16-byte aligned");
  if (c->page_table == nullptr) return fail(SCD_ERR_NULL, "page_table is NULL");
  if (reinterpret_cast<uintptr_t>(c->page_table) % 4 != 0)
    return fail(SCD_ERR_ALIGN, "page_table is not aligned to its entries");
  return SCD_OK;
}

LatentPages pages_of(const scd_latent_cache_t* c) {
  int lg = 4;
  while ((1 << lg) < c->page_tokens) ++lg;
  return {static_cast<char*>(c->pages), c->page_table, c->n_pages, c->max_pages, c->page_tokens, lg,
          c->latent_dim, c->turned_dim};
}

// The heads' matrices [heads][plain or value][latent_dim].
scd_status_t check_heads(const void* w_k, const void* w_v, int32_t plain, int32_t value) {
  if (plain < 32 || plain > 256 || plain % 32 != 0)
    return fail(SCD_ERR_UNSUPPORTED, "plain_dim %d unsupported (multiples of 32 up to 256)", plain);
  if (value < 32 || value > 256 || value % 32 != 0)
    return fail(SCD_ERR_UNSUPPORTED, "value_dim %d unsupported (multiples of 32 up to 256)", value);
  if (w_k == nullptr) return fail(SCD_ERR_NULL, "w_k is NULL");
  if (w_v == nullptr) return fail(SCD_ERR_NULL, "w_v is NULL");
  if (!aligned16(w_k)) return fail(SCD_ERR_ALIGN, "w_k is not 16-byte aligned");
  if (!aligned16(w_v)) return fail(SCD_ERR_ALIGN, "w_v is not 16-byte aligned");
  return SCD_OK;
}

scd_status_t check_scale(double scale) {
  if (!std::isfinite(scale) || !std::isfinite(static_cast<float>(scale * kLog2e)))
    return fail(SCD_ERR_SHAPE, "softmax_scale must be finite");
  return SCD_OK;
}

scd_status_t check_workspace(const void* ws, size_t bytes, size_t need) {
  if (need > 0 && ws == nullptr) return fail(SCD_ERR_NULL, "workspace is NULL");
  if (need > 0 && !aligned16(ws)) return fail(SCD_ERR_ALIGN, "workspace is not 16-byte aligned");
  if (bytes < need) return fail(SCD_ERR_SHAPE, "workspace_bytes %zu < %zu needed", bytes, need);
  return SCD_OK;
}

// Rows of all heads are counted in 31 bits, and so are workgroups.
scd_status_t check_counts(int64_t n_tokens, int64_t n_heads) {
  if (n_heads > 65535) return fail(SCD_ERR_UNSUPPORTED, "more than 65535 heads");
  if (n_tokens * n_heads >= int64_t{1} << 27) return fail(SCD_ERR_UNSUPPORTED, "n_tokens * n_heads reaches 2^27");
  if (n_tokens > 65535) return fail(SCD_ERR_UNSUPPORTED, "more than 65535 tokens");
  return SCD_OK;
}

}  // namespace

extern "C" {

scd_status_t scd_latent_append(const scd_latent_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                               const scd_rows_t* latent, const scd_rows_t* turned, const scd_rotary_t* rotary,
                               const void* table, int64_t max_position, hipStream_t stream) {
  SCD_TRY(check_latent(cache));
  SCD_TRY(check_batch(batch));
  SCD_TRY(check_dtype(dtype));
  SCD_TRY(check_rows(latent, "latent", 1, cache->latent_dim, dtype, batch->n_tokens, false));
  SCD_TRY(check_rows(turned, "turned", 1, cache->turned_dim, dtype, batch->n_tokens, false));
  LatentAppendParams p{};
  if (rotary != nullptr) {
    SCD_TRY(check_rotary(rotary));
    if (rotary->head_dim != cache->turned_dim)
      return fail(SCD_ERR_SHAPE, "rotary has head_dim %d, the cache's turned_dim is %d", rotary->head_dim,
                  cache->turned_dim);
    SCD_TRY(check_table(table, max_position));
    p.turn = turn_of(rotary, table, max_position);
  }
  if (batch->n_tokens == 0) return ok();
  p.cache = pages_of(cache);
  p.batch = batch_of(batch);
  p.c = rows_of(latent, dtype);
  p.k = rows_of(turned, dtype);
  return launched(launch_latent_append(dtype == SCD_BF16, p, stream), "latent append");
}

scd_status_t scd_latent_expand(const scd_latent_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                               int32_t n_heads, int32_t plain_dim, int32_t value_dim, const void* w_k, const void* w_v,
                               const scd_rows_t* k_out, const scd_rows_t* v_out, hipStream_t stream) {
  SCD_TRY(check_latent(cache));
  SCD_TRY(check_batch(batch));
  SCD_TRY(check_dtype(dtype));
  SCD_TRY(check_heads(w_k, w_v, plain_dim, value_dim));
  if (n_heads < 1) return fail(SCD_ERR_SHAPE, "n_heads must be >= 1 (got %d)", n_heads);
  if (n_heads > 65535) return fail(SCD_ERR_UNSUPPORTED, "more than 65535 heads");
  SCD_TRY(check_rows(k_out, "k_out", n_heads, plain_dim + cache->turned_dim, dtype, batch->n_tokens, true));
  SCD_TRY(check_rows(v_out, "v_out", n_heads, value_dim, dtype, batch->n_tokens, true));
  if (batch->n_tokens == 0) return ok();
  LatentExpandParams p{};
  p.cache = pages_of(cache);
  p.batch = batch_of(batch);
  p.k = rows_of(k_out, dtype);
  p.v = rows_of(v_out, dtype);
  p.w_k = static_cast<const char*>(w_k);
  p.w_v = static_cast<const char*>(w_v);
  p.heads = n_heads;
  p.plain = plain_dim;
  p.value = value_dim;
  return launched(launch_latent_expand(dtype == SCD_BF16, p, stream), "latent expand");
}

size_t scd_latent_attend_workspace_bytes(const scd_latent_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                                         int32_t n_heads) {
  if (check_latent_shape(cache) != SCD_OK || check_batch(batch) != SCD_OK || check_dtype(dtype) != SCD_OK ||
      n_heads < 1 || batch->n_tokens == 0 || check_counts(batch->n_tokens, n_heads) != SCD_OK)
    return 0;
  return latent_sizes(dtype == SCD_BF16, pages_of(cache), batch_of(batch), n_heads).total();
}

scd_status_t scd_latent_attend(const scd_latent_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                               double softmax_scale, int32_t plain_dim, int32_t value_dim, const void* w_k,
                               const void* w_v, const scd_rows_t* q, const scd_rows_t* out, void* workspace,
                               size_t workspace_bytes, hipStream_t stream) {
  SCD_TRY(check_latent(cache));
  SCD_TRY(check_batch(batch));
  SCD_TRY(check_dtype(dtype));
  SCD_TRY(check_scale(softmax_scale));
  SCD_TRY(check_heads(w_k, w_v, plain_dim, value_dim));
  SCD_TRY(check_rows(q, "q", 0, plain_dim + cache->turned_dim, dtype, batch->n_tokens, false));
  SCD_TRY(check_counts(batch->n_tokens, q->n_heads));
  SCD_TRY(check_rows(out, "out", q->n_heads, value_dim, dtype, batch->n_tokens, true));
  if (batch->n_tokens == 0) return ok();
  const LatentSizes z = latent_sizes(dtype == SCD_BF16, pages_of(cache), batch_of(batch), q->n_heads);
  if (z.plan.grid > kMostWorkgroups) return fail(SCD_ERR_UNSUPPORTED, "the call needs more than 2^23 workgroups");
  SCD_TRY(check_workspace(workspace, workspace_bytes, z.total()));
  LatentAttendParams p{};
  p.cache = pages_of(cache);
  p.batch = batch_of(batch);
  p.plan = z.plan;
  p.q = rows_of(q, dtype);
  p.out = rows_of(out, dtype);
  p.w_k = static_cast<const char*>(w_k);
  p.w_v = static_cast<const char*>(w_v);
  p.heads = q->n_heads;
  p.plain = plain_dim;
  p.value = value_dim;
  p.scale = static_cast<float>(softmax_scale * kLog2e);
  char* ws = static_cast<char*>(workspace);
  p.zeros = ws;
  p.absorbed = p.zeros + z.zeros;
  p.shares = reinterpret_cast<LatentShare*>(p.absorbed + z.absorbed);
  p.parts = reinterpret_cast<RowParts*>(p.absorbed + z.absorbed + z.shares);
  p.slots = reinterpret_cast<float*>(p.absorbed + z.absorbed + z.shares + z.parts);
  return launched(launch_latent_attend(dtype == SCD_BF16, p, stream), "latent attend");
}

static scd_status_t check_held(const scd_batch_t* batch, const scd_batch_t* held) {
  SCD_TRY(check_batch(batch));
  if (held == nullptr) return fail(SCD_ERR_NULL, "held is NULL");
  SCD_TRY(check_batch(held));
  if (held->n_seqs != batch->n_seqs)
    return fail(SCD_ERR_SHAPE, "held has %d requests, the batch %d", held->n_seqs, batch->n_seqs);
  if (held->n_tokens > (int64_t{1} << 31) - 128) return fail(SCD_ERR_UNSUPPORTED, "held has more than 2^31 - 128 rows");
  return SCD_OK;
}

size_t scd_rows_attend_workspace_bytes(const scd_batch_t* batch, const scd_batch_t* held, int32_t dtype, int32_t n_heads,
                                       int32_t n_kv_heads, int32_t key_dim, int32_t value_dim) {
  if (check_held(batch, held) != SCD_OK || check_dtype(dtype) != SCD_OK || n_heads < 1 || n_kv_heads < 1 ||
      n_heads % n_kv_heads != 0 || batch->n_tokens == 0 || key_dim < 32 || value_dim < 32 || key_dim > 192 ||
      value_dim > 128)
    return 0;
  // rows that start on 16 bytes or not: enough for both
  const auto size = [&](bool wide) {
    return rows_sizes(dtype == SCD_BF16, wide, batch_of(batch), held->n_tokens, n_heads, n_kv_heads, value_dim).total();
  };
  return size(true) > size(false) ? size(true) : size(false);
}

scd_status_t scd_rows_attend(const scd_batch_t* batch, const scd_batch_t* held, int32_t dtype, double softmax_scale,
                             int32_t key_dim, int32_t value_dim, const scd_rows_t* q, const scd_rows_t* k,
                             const scd_rows_t* v, const scd_rows_t* out, void* workspace, size_t workspace_bytes,
                             hipStream_t stream) {
  SCD_TRY(check_held(batch, held));
  SCD_TRY(check_dtype(dtype));
  SCD_TRY(check_scale(softmax_scale));
  if (key_dim < 32 || key_dim > 192 || key_dim % 32 != 0)
    return fail(SCD_ERR_UNSUPPORTED, "key_dim %d unsupported (multiples of 32 up to 192)", key_dim);
  if (value_dim < 32 || value_dim > 128 || value_dim % 32 != 0)
    return fail(SCD_ERR_UNSUPPORTED, "value_dim %d unsupported (multiples of 32 up to 128)", value_dim);
  SCD_TRY(check_rows(q, "q", 0, key_dim, dtype, batch->n_tokens, false));
  SCD_TRY(check_rows(k, "k", 0, key_dim, dtype, held->n_tokens, false));
  SCD_TRY(check_rows(v, "v", k->n_heads, value_dim, dtype, held->n_tokens, false));
  if (q->n_heads % k->n_heads != 0)
    return fail(SCD_ERR_SHAPE, "q has %d heads, not a multiple of k's %d", q->n_heads, k->n_heads);
  if (q->n_heads > 65535) return fail(SCD_ERR_UNSUPPORTED, "more than 65535 heads");
  if (batch->n_tokens * q->n_heads >= int64_t{1} << 31)
    return fail(SCD_ERR_UNSUPPORTED, "n_tokens * n_heads reaches 2^31");
  SCD_TRY(check_rows(out, "out", q->n_heads, value_dim, dtype, batch->n_tokens, true));
  if (batch->n_tokens == 0) return ok();
  RowsAttendParams p{};
  p.k = rows_of(k, dtype);
  p.v = rows_of(v, dtype);
  const RowsSizes z = rows_sizes(dtype == SCD_BF16, rows_wide(p.k, p.v), batch_of(batch), held->n_tokens, q->n_heads,
                                 k->n_heads, value_dim);
  if (z.plan.grid > kMostWorkgroups) return fail(SCD_ERR_UNSUPPORTED, "the call needs more than 2^23 workgroups");
  SCD_TRY(check_workspace(workspace, workspace_bytes, scd_rows_attend_workspace_bytes(batch, held, dtype, q->n_heads,
                                                                                      k->n_heads, key_dim, value_dim)));
  p.batch = batch_of(batch);
  p.held = batch_of(held);
  p.plan = z.plan;
  p.q = rows_of(q, dtype);
  p.out = rows_of(out, dtype);
  p.key = key_dim;
  p.value = value_dim;
  p.scale = static_cast<float>(softmax_scale * kLog2e);
  char* ws = static_cast<char*>(workspace);
  p.parts = z.plan.cut ? reinterpret_cast<RowParts*>(ws) : nullptr;
  p.slots = z.plan.cut ? reinterpret_cast<float*>(ws + z.parts) : nullptr;
  return launched(launch_rows_attend(dtype == SCD_BF16, p, stream), "rows attend");
}

}  // extern "C"
