// Internal declarations of the operations on pages of caches.
#pragma once

#include "scd_serve.h"

namespace scd {

struct PagePool {
  int32_t* refs;        // [n_pages] table entries that name a page
  int32_t* table;       // [n_seqs][cols]
  int32_t* held;        // [n_seqs]
  int32_t n_pages, n_seqs, cols, page;
};

struct PageMoves {
  int32_t* pairs;       // [capacity][2] from, to
  int32_t* status;      // [4]
  int32_t capacity;
};

struct PagePlane {
  char* data;
  int64_t page_bytes;
};
constexpr int kMostPlanes = 128;  // of a launch
struct PagesCopyParams {
  PagePlane planes[kMostPlanes];
  int32_t n_planes, n_pages;
  PageMoves moves;
};
static_assert(sizeof(PagesCopyParams) <= 4096, "kernel argument block");

size_t pages_workspace(int64_t n_pages);
hipError_t launch_pages_free(const PagePool& p, int n, const int32_t* seqs, hipStream_t stream);
hipError_t launch_pages_fork(const PagePool& p, int n, const int32_t* src, const int32_t* dst, hipStream_t stream);
hipError_t launch_pages_reserve(const PagePool& p, const SeqBatch& b, const PageMoves& m, int32_t* ws, hipStream_t stream);
hipError_t launch_pages_compact(const PagePool& p, const PagePool& out, const PageMoves& m, int32_t* ws,
                                hipStream_t stream);
hipError_t launch_pages_copy(const PagesCopyParams& p, hipStream_t stream);

}  // namespace scd
