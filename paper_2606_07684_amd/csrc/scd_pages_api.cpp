// Host side of the operations on pages: argument validation and launches.
#include "scd_pages.h"
#include "scd_serve_host.h"

namespace {

using namespace scd;

scd_status_t check_pool(const scd_pages_t* p, const char* name) {
  if (p == nullptr) return fail(SCD_ERR_NULL, "%s is NULL", name);
  if (p->n_pages < 1 || p->n_seqs < 1 || p->max_pages < 1)
    return fail(SCD_ERR_SHAPE, "%s needs n_pages, n_seqs and max_pages >= 1 (got %d, %d, %d)", name, p->n_pages,
                p->n_seqs, p->max_pages);
  // the kernels step 32-bit indexes by up to 4096
  if (p->n_pages > 1 << 30 || p->n_seqs > 1 << 30 || p->max_pages > 1 << 30)
    return fail(SCD_ERR_UNSUPPORTED, "%s: n_pages, n_seqs and max_pages up to 2^30 (got %d, %d, %d)", name, p->n_pages,
                p->n_seqs, p->max_pages);
  if (p->page_tokens < 1) return fail(SCD_ERR_SHAPE, "page_tokens must be >= 1 (got %d)", p->page_tokens);
  const struct {
    const void* p;
    const char* name;
  } need[] = {{p->refs, "refs"}, {p->page_table, "page_table"}, {p->held, "held"}};
  for (const auto& n : need) {
    if (n.p == nullptr) return fail(SCD_ERR_NULL, "%s of %s is NULL", n.name, name);
    if (reinterpret_cast<uintptr_t>(n.p) % 4 != 0)
      return fail(SCD_ERR_ALIGN, "%s of %s is not aligned to its entries", n.name, name);
  }
  return SCD_OK;
}

scd_status_t check_moves(const scd_moves_t* m, int64_t need) {
  if (m == nullptr) return fail(SCD_ERR_NULL, "moves is NULL");
  if (m->status == nullptr) return fail(SCD_ERR_NULL, "moves has no status");
  if (m->pairs == nullptr && need > 0) return fail(SCD_ERR_NULL, "moves has no pairs");
  if (reinterpret_cast<uintptr_t>(m->status) % 4 != 0 || reinterpret_cast<uintptr_t>(m->pairs) % 4 != 0)
    return fail(SCD_ERR_ALIGN, "moves is not aligned to its entries");
  if (m->capacity < 0 || m->capacity < need)
    return fail(SCD_ERR_SHAPE, "moves holds %d pairs, %lld may be needed", m->capacity, static_cast<long long>(need));
  return SCD_OK;
}

scd_status_t check_list(const int32_t* list, int32_t n, const char* name) {
  if (n < 0) return fail(SCD_ERR_SHAPE, "%s has %d entries", name, n);
  if (n > 1 << 20) return fail(SCD_ERR_UNSUPPORTED, "%s has more than 2^20 entries", name);
  if (n > 0 && list == nullptr) return fail(SCD_ERR_NULL, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(list) % 4 != 0) return fail(SCD_ERR_ALIGN, "%s is not aligned to its entries", name);
  return SCD_OK;
}

scd_status_t check_workspace(const scd_pages_t* p, const void* ws, size_t bytes) {
  const size_t need = pages_workspace(p->n_pages);
  if (ws == nullptr) return fail(SCD_ERR_NULL, "workspace is NULL");
  if (!aligned16(ws)) return fail(SCD_ERR_ALIGN, "workspace is not 16-byte aligned");
  if (bytes < need) return fail(SCD_ERR_SHAPE, "workspace_bytes %zu < %zu needed", bytes, need);
  return SCD_OK;
}

PagePool pool_of(const scd_pages_t* p) {
  return {p->refs, p->page_table, p->held, p->n_pages, p->n_seqs, p->max_pages, p->page_tokens};
}
PageMoves moves_of(const scd_moves_t* m) { return {m->pairs, m->status, m->capacity}; }

}  // namespace

extern "C" {

size_t scd_pages_workspace_bytes(const scd_pages_t* pages) {
  if (check_pool(pages, "pages") != SCD_OK) return 0;
  return pages_workspace(pages->n_pages);
}

scd_status_t scd_pages_free(const scd_pages_t* pages, int32_t n, const int32_t* seqs, hipStream_t stream) {
  SCD_TRY(check_pool(pages, "pages"));
  SCD_TRY(check_list(seqs, n, "seqs"));
  if (n == 0) return ok();
  return launched(launch_pages_free(pool_of(pages), n, seqs, stream), "pages free");
}

scd_status_t scd_pages_fork(const scd_pages_t* pages, int32_t n, const int32_t* src, const int32_t* dst,
                            hipStream_t stream) {
  SCD_TRY(check_pool(pages, "pages"));
  SCD_TRY(check_list(src, n, "src"));
  SCD_TRY(check_list(dst, n, "dst"));
  if (n == 0) return ok();
  return launched(launch_pages_fork(pool_of(pages), n, src, dst, stream), "pages fork");
}

scd_status_t scd_pages_reserve(const scd_pages_t* pages, const scd_batch_t* batch, const scd_moves_t* moves,
                               void* workspace, size_t workspace_bytes, hipStream_t stream) {
  SCD_TRY(check_pool(pages, "pages"));
  SCD_TRY(check_batch(batch));
  if (batch->n_seqs != pages->n_seqs)
    return fail(SCD_ERR_SHAPE, "the batch has %d requests, pages %d", batch->n_seqs, pages->n_seqs);
  SCD_TRY(check_moves(moves, pages->n_seqs));
  SCD_TRY(check_workspace(pages, workspace, workspace_bytes));
  return launched(launch_pages_reserve(pool_of(pages), batch_of(batch), moves_of(moves), static_cast<int32_t*>(workspace),
                                       stream), "pages reserve");
}

scd_status_t scd_pages_compact(const scd_pages_t* pages, const scd_pages_t* out, const scd_moves_t* moves,
                               void* workspace, size_t workspace_bytes, hipStream_t stream) {
  SCD_TRY(check_pool(pages, "pages"));
  if (out == nullptr) out = pages;
  SCD_TRY(check_pool(out, "out"));
  if (out->n_pages != pages->n_pages || out->n_seqs != pages->n_seqs || out->max_pages != pages->max_pages ||
      out->page_tokens != pages->page_tokens)
    return fail(SCD_ERR_SHAPE, "out and pages differ in their sizes");
  SCD_TRY(check_moves(moves, pages->n_pages / 2));
  SCD_TRY(check_workspace(pages, workspace, workspace_bytes));
  return launched(launch_pages_compact(pool_of(pages), pool_of(out), moves_of(moves), static_cast<int32_t*>(workspace),
                                       stream), "pages compact");
}

scd_status_t scd_pages_copy(int32_t n_planes, const scd_plane_t* planes, int32_t n_pages, const scd_moves_t* moves,
                            hipStream_t stream) {
  if (n_planes < 0) return fail(SCD_ERR_SHAPE, "n_planes must be >= 0 (got %d)", n_planes);
  if (n_planes > 0 && planes == nullptr) return fail(SCD_ERR_NULL, "planes is NULL");
  if (n_pages < 1) return fail(SCD_ERR_SHAPE, "n_pages must be >= 1 (got %d)", n_pages);
  SCD_TRY(check_moves(moves, 0));
  for (int32_t i = 0; i < n_planes; ++i) {
    if (planes[i].data == nullptr) return fail(SCD_ERR_NULL, "plane %d is NULL", i);
    if (!aligned16(planes[i].data)) return fail(SCD_ERR_ALIGN, "plane %d is not 16-byte aligned", i);
    if (planes[i].page_bytes < 4 || planes[i].page_bytes % 4 != 0 || planes[i].page_bytes > int64_t{1} << 30)
      return fail(SCD_ERR_SHAPE, "plane %d has pages of %lld bytes: a multiple of 4 up to 2^30 is needed", i,
                  static_cast<long long>(planes[i].page_bytes));
  }
  if (moves->capacity == 0) return ok();
  for (int32_t i = 0; i < n_planes; i += kMostPlanes) {
    PagesCopyParams p{};
    p.n_planes = n_planes - i < kMostPlanes ? n_planes - i : kMostPlanes;
    for (int32_t j = 0; j < p.n_planes; ++j)
      p.planes[j] = {static_cast<char*>(planes[i + j].data), planes[i + j].page_bytes};
    p.n_pages = n_pages;
    p.moves = moves_of(moves);
    SCD_TRY(launched(launch_pages_copy(p, stream), "pages copy"));
  }
  return ok();
}

}  // extern "C"
