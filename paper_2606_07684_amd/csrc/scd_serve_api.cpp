// Host side of the serving operators: argument validation and launches.  Every argument is checked
// before the first launch; nothing allocates, synchronises or keeps state.
#include <cmath>

#include "scd_serve_host.h"

namespace scd {

scd_status_t check_dtype(int32_t dtype) {
  if (dtype != SCD_F32 && dtype != SCD_BF16) return fail(SCD_ERR_SHAPE, "dtype %d unknown", dtype);
  return SCD_OK;
}

scd_status_t check_rotary(const scd_rotary_t* r) {
  if (r == nullptr) return fail(SCD_ERR_NULL, "rotary is NULL");
  if (r->head_dim < 2 || r->head_dim % 2 != 0)
    return fail(SCD_ERR_SHAPE, "head_dim must be positive and even (got %d)", r->head_dim);
  if (r->head_dim > 2 * scd::kMaxTurnPairs)
    return fail(SCD_ERR_UNSUPPORTED, "head_dim %d above %d", r->head_dim, 2 * scd::kMaxTurnPairs);
  if (r->rotary_dim < 2 || r->rotary_dim % 2 != 0 || r->rotary_dim > r->head_dim)
    return fail(SCD_ERR_SHAPE, "rotary_dim %d must be even, at least 2 and at most head_dim %d",
                r->rotary_dim, r->head_dim);
  if (r->layout != SCD_ROTARY_HALF && r->layout != SCD_ROTARY_INTERLEAVED)
    return fail(SCD_ERR_SHAPE, "rotary layout %d unknown", r->layout);
  if (r->scaling < SCD_ROTARY_NONE || r->scaling > SCD_ROTARY_GIVEN)
    return fail(SCD_ERR_SHAPE, "rotary scaling %d unknown", r->scaling);
  if (r->scaling != SCD_ROTARY_GIVEN && (!(r->theta > 1.0) || !std::isfinite(r->theta)))
    return fail(SCD_ERR_SHAPE, "rotary theta must be > 1 and finite");
  if (!(r->attention_factor > 0.0) || !std::isfinite(r->attention_factor))
    return fail(SCD_ERR_SHAPE, "attention_factor must be > 0 and finite");
  if ((r->scaling == SCD_ROTARY_LINEAR || r->scaling == SCD_ROTARY_NTK ||
       r->scaling == SCD_ROTARY_BY_PARTS) &&
      (!(r->factor > 0.0) || !std::isfinite(r->factor)))
    return fail(SCD_ERR_SHAPE, "rotary factor must be > 0 and finite");
  if (r->scaling == SCD_ROTARY_NTK && r->rotary_dim < 4)
    return fail(SCD_ERR_SHAPE, "rotary_dim must be at least 4 for NTK scaling");
  if (r->scaling == SCD_ROTARY_BY_PARTS &&
      (!(r->low < r->high) || !std::isfinite(r->low) || !std::isfinite(r->high) ||
       r->trained_positions < 1))
    return fail(SCD_ERR_SHAPE, "by-parts scaling needs low < high and trained_positions >= 1");
  return SCD_OK;
}

scd_status_t check_table(const void* table, int64_t max_position) {
  if (table == nullptr) return fail(SCD_ERR_WORKSPACE, "rotary table is NULL");
  if (!aligned16(table)) return fail(SCD_ERR_ALIGN, "rotary table is not 16-byte aligned");
  if (max_position < 1) return fail(SCD_ERR_WORKSPACE, "max_position must be >= 1");
  return SCD_OK;
}

scd_status_t check_rows(const scd_rows_t* r, const char* name, int32_t heads, int32_t head_dim,
                        int32_t dtype, int64_t n_tokens, bool written) {
  if (r == nullptr) return fail(SCD_ERR_NULL, "%s is NULL", name);
  if (r->n_heads < 1 || (heads != 0 && r->n_heads != heads))
    return fail(SCD_ERR_SHAPE, "%s has %d heads, expected %d", name, r->n_heads, heads);
  if (r->data == nullptr && n_tokens > 0) return fail(SCD_ERR_NULL, "%s data is NULL", name);
  const uintptr_t element = dtype == SCD_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(r->data) % element != 0)
    return fail(SCD_ERR_ALIGN, "%s data is not aligned to its element", name);
  if (r->token_stride < 0 || r->head_stride < 0)
    return fail(SCD_ERR_SHAPE, "%s has a negative stride", name);
  // heads inside a token, or tokens inside a head, one after another
  const int64_t nh = r->n_heads, hs = r->head_stride, ts = r->token_stride;
  if (written && n_tokens > 0 &&
      !((nh == 1 || hs >= head_dim) && (n_tokens == 1 || ts >= head_dim) &&
        (nh == 1 || n_tokens == 1 || ts >= (nh - 1) * hs + head_dim ||
         hs >= (n_tokens - 1) * ts + head_dim)))
    return fail(SCD_ERR_SHAPE, "%s: rows overlap", name);
  return SCD_OK;
}

scd::Rows rows_of(const scd_rows_t* r, int32_t dtype) {
  const int64_t wide = dtype == SCD_BF16 ? 8 : 4;
  return {static_cast<char*>(r->data), r->token_stride, r->head_stride, r->n_heads,
          aligned16(r->data) && r->token_stride % wide == 0 && r->head_stride % wide == 0};
}

scd::SeqBatch batch_of(const scd_batch_t* b) {
  return {b->cu_seqlens, b->pos0, b->n_tokens, b->n_seqs};
}

scd::Turn turn_of(const scd_rotary_t* r, const void* table, int64_t max_position) {
  return {static_cast<const float2*>(table), max_position, r->rotary_dim,
          r->layout == SCD_ROTARY_INTERLEAVED};
}

scd_status_t launched(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(SCD_ERR_HIP, "%s launch failed: %s", what, hipGetErrorString(e));
  return ok();
}

}  // namespace scd

namespace {

using scd::aligned16;
using scd::batch_of;
using scd::check_batch;
using scd::check_dtype;
using scd::check_rotary;
using scd::check_rows;
using scd::check_table;
using scd::fail;
using scd::launched;
using scd::ok;
using scd::rows_of;
using scd::turn_of;

scd_status_t check_cache_shape(const scd_cache_t* c) {
  if (c == nullptr) return fail(SCD_ERR_NULL, "cache is NULL");
  if (c->n_pages < 1 || c->n_kv_heads < 1 || c->max_pages < 1)
    return fail(SCD_ERR_SHAPE, "cache needs n_pages, n_kv_heads and max_pages >= 1 (got %d, %d, %d)",
                c->n_pages, c->n_kv_heads, c->max_pages);
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128)
    return fail(SCD_ERR_UNSUPPORTED, "head_dim %d unsupported (32, 64 or 128)", c->head_dim);
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128)
    return fail(SCD_ERR_UNSUPPORTED, "page_tokens %d unsupported (16, 32, 64 or 128)", c->page_tokens);
  if (c->n_kv_heads > 65536) return fail(SCD_ERR_UNSUPPORTED, "n_kv_heads above 65536");
  return SCD_OK;
}

scd_status_t check_cache(const scd_cache_t* c) {
  SCD_TRY(check_cache_shape(c));
  const struct {
    const void* p;
    const char* name;
  } need[] = {{c->k_pages, "k_pages"}, {c->v_pages, "v_pages"}, {c->k_scales, "k_scales"},
              {c->v_scales, "v_scales"}};
  for (const auto& n : need) {
    if (n.p == nullptr) return fail(SCD_ERR_NULL, "%s is NULL", n.name);
    if (!aligned16(n.p)) return fail(SCD_ERR_ALIGN, "%s is not 16-byte aligned", n.name);
  }
  if (c->page_table == nullptr) return fail(SCD_ERR_NULL, "page_table is NULL");
  if (reinterpret_cast<uintptr_t>(c->page_table) % 4 != 0)
    return fail(SCD_ERR_ALIGN, "page_table is not aligned to its entries");
  return SCD_OK;
}

scd::PagedCache cache_of(const scd_cache_t* c) {
  int lg = 4;
  while ((1 << lg) < c->page_tokens) ++lg;
  return {c->k_pages, c->v_pages, c->k_scales, c->v_scales, c->page_table,
          c->n_pages, c->n_kv_heads, c->max_pages, c->page_tokens, lg};
}

}  // namespace

extern "C" {

size_t scd_rotary_table_bytes(const scd_rotary_t* rotary, int64_t max_position) {
  if (check_rotary(rotary) != SCD_OK || max_position < 1 || max_position > (int64_t{1} << 31)) return 0;
  return static_cast<size_t>(max_position) * static_cast<size_t>(rotary->rotary_dim / 2) * sizeof(float2);
}

scd_status_t scd_rotary_table(const scd_rotary_t* rotary, int64_t max_position, void* table,
                              size_t table_bytes, hipStream_t stream) {
  SCD_TRY(check_rotary(rotary));
  SCD_TRY(check_table(table, max_position));
  if (max_position > (int64_t{1} << 31))
    return fail(SCD_ERR_UNSUPPORTED, "max_position above 2^31");
  const size_t need = scd_rotary_table_bytes(rotary, max_position);
  if (table_bytes < need)
    return fail(SCD_ERR_WORKSPACE, "table_bytes %zu < %zu needed", table_bytes, need);
  if (rotary->scaling == SCD_ROTARY_GIVEN && rotary->frequencies == nullptr)
    return fail(SCD_ERR_NULL, "frequencies is NULL");
  scd::TurnTableParams p{};
  p.pairs = rotary->rotary_dim / 2;
  p.gain = rotary->attention_factor;
  p.table = static_cast<float2*>(table);
  p.n = max_position * p.pairs;
  const double rd = rotary->rotary_dim;
  double theta = rotary->theta;
  if (rotary->scaling == SCD_ROTARY_NTK) theta *= std::pow(rotary->factor, rd / (rd - 2.0));
  for (int i = 0; i < p.pairs; ++i) {
    if (rotary->scaling == SCD_ROTARY_GIVEN) {
      p.w[i] = rotary->frequencies[i];
      continue;
    }
    double w = std::pow(theta, -2.0 * i / rd);
    if (rotary->scaling == SCD_ROTARY_LINEAR) w /= rotary->factor;
    if (rotary->scaling == SCD_ROTARY_BY_PARTS) {
      const double turns = static_cast<double>(rotary->trained_positions) * w / 6.283185307179586;
      const double g = std::fmin(1.0, std::fmax(0.0, (turns - rotary->low) / (rotary->high - rotary->low)));
      w = (1.0 - g) * w / rotary->factor + g * w;
    }
    p.w[i] = w;
  }
  return launched(scd::launch_turn_table(p, stream), "rotary table");
}

scd_status_t scd_rotary(const scd_rotary_t* rotary, const scd_batch_t* batch, const void* table,
                        int64_t max_position, int32_t dtype, int32_t transpose,
                        const scd_rows_t* q, const scd_rows_t* k, const scd_rows_t* q_out,
                        const scd_rows_t* k_out, hipStream_t stream) {
  SCD_TRY(check_rotary(rotary));
  SCD_TRY(check_batch(batch));
  SCD_TRY(check_dtype(dtype));
  SCD_TRY(check_table(table, max_position));
  if ((k == nullptr) != (k_out == nullptr))
    return fail(SCD_ERR_NULL, "k and k_out go together");
  scd::RotaryParams p{};
  const scd_rows_t* in[2] = {q, k};
  const scd_rows_t* out[2] = {q_out, k_out};
  const char* names[2][2] = {{"q", "q_out"}, {"k", "k_out"}};
  const int64_t n = batch->n_tokens;
  for (int i = 0; i < 2; ++i) {
    if (i == 1 && k == nullptr) break;
    SCD_TRY(check_rows(in[i], names[i][0], 0, rotary->head_dim, dtype, n, false));
    SCD_TRY(check_rows(out[i], names[i][1], in[i]->n_heads, rotary->head_dim, dtype, n, true));
    if (n > 0 && in[i]->data == out[i]->data &&
        (in[i]->token_stride != out[i]->token_stride || in[i]->head_stride != out[i]->head_stride))
      return fail(SCD_ERR_SHAPE, "%s in place needs the strides of %s", names[i][1], names[i][0]);
    p.in[i] = rows_of(in[i], dtype);
    p.out[i] = rows_of(out[i], dtype);
  }
  if (int64_t{p.in[0].n_heads} + p.in[1].n_heads > 65536)
    return fail(SCD_ERR_UNSUPPORTED, "more than 65536 heads");
  if (n == 0) return ok();
  p.batch = batch_of(batch);
  p.turn = turn_of(rotary, table, max_position);
  p.head_dim = rotary->head_dim;
  p.transpose = transpose != 0;
  return launched(scd::launch_rotary(dtype == SCD_BF16, p, stream), "rotary");
}

scd_status_t scd_cache_append(const scd_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                              const scd_rows_t* k, const scd_rows_t* v,
                              const scd_rotary_t* rotary, const void* table,
                              int64_t max_position, hipStream_t stream) {
  SCD_TRY(check_cache(cache));
  SCD_TRY(check_batch(batch));
  SCD_TRY(check_dtype(dtype));
  SCD_TRY(check_rows(k, "k", cache->n_kv_heads, cache->head_dim, dtype, batch->n_tokens, false));
  SCD_TRY(check_rows(v, "v", cache->n_kv_heads, cache->head_dim, dtype, batch->n_tokens, false));
  scd::CacheAppendParams p{};
  if (rotary != nullptr) {
    SCD_TRY(check_rotary(rotary));
    if (rotary->head_dim != cache->head_dim)
      return fail(SCD_ERR_SHAPE, "rotary has head_dim %d, the cache %d", rotary->head_dim, cache->head_dim);
    SCD_TRY(check_table(table, max_position));
    p.turn = turn_of(rotary, table, max_position);
  }
  if (batch->n_tokens == 0) return ok();
  p.cache = cache_of(cache);
  p.batch = batch_of(batch);
  p.rows[0] = rows_of(k, dtype);
  p.rows[1] = rows_of(v, dtype);
  return launched(scd::launch_cache_append(dtype == SCD_BF16, cache->head_dim, p, stream), "cache append");
}

scd_status_t scd_cache_read(const scd_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                            const scd_rows_t* k_out, const scd_rows_t* v_out, hipStream_t stream) {
  SCD_TRY(check_cache(cache));
  SCD_TRY(check_batch(batch));
  SCD_TRY(check_dtype(dtype));
  SCD_TRY(check_rows(k_out, "k_out", cache->n_kv_heads, cache->head_dim, dtype, batch->n_tokens, true));
  SCD_TRY(check_rows(v_out, "v_out", cache->n_kv_heads, cache->head_dim, dtype, batch->n_tokens, true));
  if (batch->n_tokens == 0) return ok();
  scd::CacheReadParams p{};
  p.cache = cache_of(cache);
  p.batch = batch_of(batch);
  p.rows[0] = rows_of(k_out, dtype);
  p.rows[1] = rows_of(v_out, dtype);
  return launched(scd::launch_cache_read(dtype == SCD_BF16, cache->head_dim, p, stream), "cache read");
}

size_t scd_cache_attend_workspace_bytes(const scd_cache_t* cache, const scd_batch_t* batch,
                                        int32_t n_q_heads) {
  if (check_cache_shape(cache) != SCD_OK || check_batch(batch) != SCD_OK || n_q_heads < 1 ||
      n_q_heads % cache->n_kv_heads != 0 || batch->n_tokens == 0)
    return 0;
  return scd::attend_workspace(cache_of(cache), batch_of(batch), n_q_heads / cache->n_kv_heads,
                               cache->head_dim);
}

scd_status_t scd_cache_attend(const scd_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                              double softmax_scale, const scd_rows_t* q, const scd_rows_t* out,
                              void* workspace, size_t workspace_bytes, hipStream_t stream) {
  SCD_TRY(check_cache(cache));
  SCD_TRY(check_batch(batch));
  SCD_TRY(check_dtype(dtype));
  if (!std::isfinite(softmax_scale) || !std::isfinite(static_cast<float>(softmax_scale)))
    return fail(SCD_ERR_SHAPE, "softmax_scale must be finite");
  SCD_TRY(check_rows(q, "q", 0, cache->head_dim, dtype, batch->n_tokens, false));
  if (q->n_heads % cache->n_kv_heads != 0)
    return fail(SCD_ERR_SHAPE, "q has %d heads, not a multiple of n_kv_heads %d", q->n_heads,
                cache->n_kv_heads);
  if (q->n_heads > 65536) return fail(SCD_ERR_UNSUPPORTED, "more than 65536 query heads");
  if (batch->n_tokens * q->n_heads >= int64_t{1} << 31)
    return fail(SCD_ERR_UNSUPPORTED, "n_tokens * n_heads reaches 2^31");
  SCD_TRY(check_rows(out, "out", q->n_heads, cache->head_dim, dtype, batch->n_tokens, true));
  if (batch->n_tokens == 0) return ok();
  const size_t need = scd_cache_attend_workspace_bytes(cache, batch, q->n_heads);
  if (need > 0 && workspace == nullptr) return fail(SCD_ERR_NULL, "workspace is NULL");
  if (need > 0 && !aligned16(workspace)) return fail(SCD_ERR_ALIGN, "workspace is not 16-byte aligned");
  if (workspace_bytes < need)
    return fail(SCD_ERR_SHAPE, "workspace_bytes %zu < %zu needed", workspace_bytes, need);
  scd::CacheAttendParams p{};
  p.cache = cache_of(cache);
  p.batch = batch_of(batch);
  p.q = rows_of(q, dtype);
  p.out = rows_of(out, dtype);
  p.group = q->n_heads / cache->n_kv_heads;
  p.scale = static_cast<float>(softmax_scale);
  p.by_group = scd::FastDiv(p.group);
  p.by_heads = scd::FastDiv(cache->n_kv_heads);
  return launched(scd::launch_cache_attend(dtype == SCD_BF16, cache->head_dim, p, workspace, stream),
                  "cache attend");
}

}  // extern "C"
