// Pages of caches given back, shared, reserved and moved to the front (gfx950).
//
// A page is in use while table entries name it; refs counts them.  What a call hands out is decided by
// numbers alone: the lowest free pages, to requests in their order and a request's positions in theirs.  All
// of it is integers, a few hundred to some ten thousand, so the calls are chains of dependent memory accesses
// of one workgroup (a workgroup a request where requests are on their own); the contents are moved by
// pages_copy_kernel, which HBM bounds.  48 forks of 16 requests: free and fork 4.8 us each, reserve 11 to 12, and the copy of
// their 48 pages of 32 layers, 126 MB read and written, 20; 124 pages of 16 layers, 520 MB, 112 us, 4.7 TB/s.
#include <algorithm>

#include "scd_pages.h"
#include "scd_serve_device.h"

namespace scd {
using namespace dev;

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;

// Whether value v is among list[0 .. n).  Every workgroup reads the list, so that calls of many requests take the square
// of their number: 1000 freed 9 us and forked 13, 10000 29 and 61, 100000 1.2 and 3.4 ms.
template <int kThreads>
__device__ inline bool listed(const int32_t* list, int n, int v, int tid) {
  int found = 0;
  for (int i = tid; i < n; i += kThreads) found |= list[i] == v;
  return __syncthreads_or(found) != 0;
}

// Workgroup i takes request seqs[i] out of its pages; one named before it in the list is left to that one.
__global__ __launch_bounds__(256) void pages_free_kernel(PagePool p, const int32_t* seqs) {
  const int tid = threadIdx.x, i = blockIdx.x, b = seqs[i];
  if (b < 0 || b >= p.n_seqs || listed<256>(seqs, i, b, tid)) return;
  int32_t* row = p.table + static_cast<int64_t>(b) * p.cols;
  for (int j = tid; j < p.cols; j += 256) {
    const int id = row[j];
    // a count that is zero already stays zero
    if (id >= 0 && id < p.n_pages && atomicSub(p.refs + id, 1) <= 0) atomicAdd(p.refs + id, 1);
    row[j] = -1;
  }
  if (tid == 0) p.held[b] = 0;
}

// Workgroup i gives request dst[i] the pages of what src[i] holds.
__global__ __launch_bounds__(256) void pages_fork_kernel(PagePool p, int n, const int32_t* src, const int32_t* dst) {
  const int tid = threadIdx.x, i = blockIdx.x, from = src[i], to = dst[i];
  if (from < 0 || from >= p.n_seqs || to < 0 || to >= p.n_seqs) return;
  // A row that is written is written by one workgroup and read by no other: the first pair that names it,
  // and no pair that takes it for a source.
  if (listed<256>(dst, i, to, tid) || listed<256>(dst, n, from, tid)) return;
  int32_t* row = p.table + static_cast<int64_t>(to) * p.cols;
  const int32_t* old = p.table + static_cast<int64_t>(from) * p.cols;
  int any = p.held[to] != 0;
  for (int j = tid; j < p.cols; j += 256) any |= row[j] >= 0 && row[j] < p.n_pages;
  if (__syncthreads_or(any)) return;
  const int64_t held = p.held[from];
  for (int j = tid; j < p.cols; j += 256) {
    int id = static_cast<int64_t>(j) * p.page < held ? old[j] : -1;
    id = id >= 0 && id < p.n_pages ? id : -1;
    row[j] = id;
    if (id >= 0) atomicAdd(p.refs + id, 1);
  }
  if (tid == 0) p.held[to] = static_cast<int32_t>(held);
}

// Sum over the workgroup of x, and of the threads before this one.
struct PlanLds {
  int64_t wave[kPlanWaves];
};
template <typename I>
__device__ inline I plan_scan(I x, PlanLds& lds, int tid, I& total) {
  const int lane = tid & 63, wave = tid >> 6;
  I sum = x;
  for (int o = 1; o < 64; o <<= 1) {
    const I other = __shfl_up(sum, o);
    if (lane >= o) sum += other;
  }
  __syncthreads();  // the last scan's readers are done
  if (lane == 63) lds.wave[wave] = sum;
  __syncthreads();
  I before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const I v = static_cast<I>(lds.wave[w]);
    if (w < wave) before += v;
    total += v;
  }
  return before + sum - x;
}

// The same call where no request writes to more than two pages, as in a step of one token or few each: a thread a
// request, all it knows in registers, four dependent memory accesses in all (lengths, entries, counts, results).
// False, and nothing done, where some request writes to more.
struct FewLds {
  PlanLds scan;
  int shared, pages[2 * kPlanThreads], writer[2 * kPlanThreads];  // entries of pages that others name too
  int free[2 * kPlanThreads];
};
__device__ inline bool reserve_few(const PagePool& p, const SeqBatch& batch, const PageMoves& m, FewLds& lds, int tid) {
  // the lowest pages' counts come meanwhile
  int first[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) first[e] = 4 * tid + e < p.n_pages ? p.refs[4 * tid + e] : 1;
  if (tid == 0) lds.shared = 0;
  int lo = 0, n_columns = 0, held = 0;
  bool wrong = false;
  if (tid < p.n_seqs) {
    const Span s = span_of(batch, tid);
    held = p.held[tid];
    const int64_t n = s.end - s.begin;
    if (n > 0) {
      const int64_t hi = div_up_to(held < 0 ? 0 : held + n + p.page - 1, p.page);
      lo = held < 0 ? 0 : held / p.page;
      wrong = held < 0 || hi > p.cols;
      const int64_t columns = wrong ? 0 : hi - lo;
      n_columns = columns > 2 ? 3 : static_cast<int>(columns);
    }
  }
  if (__syncthreads_or(n_columns > 2)) return false;
  const int refused = __syncthreads_count(wrong);
  if (refused > 0) {
    if (tid < 4) m.status[tid] = tid == 3 ? refused : 0;
    return true;
  }
  const int64_t row = static_cast<int64_t>(tid) * p.cols + lo;
  int id[2], refs[2];
  bool missing[2], left[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) id[e] = e < n_columns ? p.table[row + e] : 0;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    missing[e] = e < n_columns && (id[e] < 0 || id[e] >= p.n_pages);
    refs[e] = e < n_columns && !missing[e] ? p.refs[id[e]] : 0;
    if (refs[e] > 1) {
      const int at = atomicAdd(&lds.shared, 1);
      lds.pages[at] = id[e];
      lds.writer[at] = tid;
    }
  }
  __syncthreads();
  const int shared = lds.shared;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    left[e] = false;
    if (refs[e] > 1) {
      int writers = 0, last = -1;
      for (int i = 0; i < shared; ++i)
        if (lds.pages[i] == id[e]) {
          ++writers;
          last = lds.writer[i] > last ? lds.writer[i] : last;
        }
      left[e] = tid != last || refs[e] > writers;
    }
  }
  // begun pages that are left are the only ones whose contents move: a request has one at most, its first
  const bool moved = left[0] && static_cast<int64_t>(lo) * p.page < held;
  const int taken = (missing[0] || left[0]) + (missing[1] || left[1]);
  int total;
  const int before = plan_scan(taken | (moved ? 1 : 0) << 16, lds.scan, tid, total);
  const int wanted = total & 0xffff, moves = total >> 16;
  int found = 0;
  for (int id0 = 0; id0 < p.n_pages && found < wanted; id0 += 4 * kPlanThreads) {
    const int at0 = id0 + 4 * tid;
    bool open[4];
    int n = 0, all;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      open[e] = at0 + e < p.n_pages && (id0 == 0 ? first[e] : p.refs[at0 + e]) <= 0;
      n += open[e];
    }
    int at = found + plan_scan(n, lds.scan, tid, all);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (open[e]) {
        if (at < 2 * kPlanThreads) lds.free[at] = at0 + e;
        ++at;
      }
    found += all;
  }
  if (found < wanted || moves > m.capacity) {
    if (tid < 4) m.status[tid] = tid == 2 ? std::max(wanted - found, 1) : 0;
    return true;
  }
  __syncthreads();
  int take = before & 0xffff;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    if (!missing[e] && !left[e]) continue;
    const int to = lds.free[take++];
    p.table[row + e] = to;
    p.refs[to] = 1;
    if (left[e]) atomicSub(p.refs + id[e], 1);
    if (e == 0 && moved) {
      m.pairs[2 * static_cast<int64_t>(before >> 16)] = id[0];
      m.pairs[2 * static_cast<int64_t>(before >> 16) + 1] = to;
    }
  }
  if (tid < 4) m.status[tid] = tid == 0 ? moves : 0;
  return true;
}

// Pages that the new tokens of every request go to, one workgroup for all.  A missing page is taken, and so
// is one in place of a page that others name too; where that holds earlier positions its contents are to be
// moved (a move is listed).  If all that name a page are to write to it, the last of them keeps it.
// The columns that requests write to are taken one after another, a thread each, requests in order: what a column takes is
// then the count of those before it.  10448 pages of 1000 requests 87 us (322
// with a wave a request), 1280 of 130 requests 45 (61), 11348 of 130 requests 87 (80).
struct ColumnsLds {
  int64_t first[kPlanThreads];  // of a request's columns among those of 1024 requests
  int lo[kPlanThreads], held[kPlanThreads];
};
__global__ __launch_bounds__(kPlanThreads) void pages_reserve_kernel(PagePool p, SeqBatch batch, PageMoves m, int32_t* ws) {
  __shared__ PlanLds lds;
  __shared__ FewLds few;
  __shared__ ColumnsLds columns;
  const int tid = threadIdx.x;
  if (p.n_seqs <= kPlanThreads && reserve_few(p, batch, m, few, tid)) return;
  int32_t* writers = ws;                        // [n_pages] requests that write to a shared page
  int32_t* keeper = writers + p.n_pages;        // [n_pages] the last of them
  int32_t* free = keeper + p.n_pages;           // [n_pages] free pages, lowest first

  const auto load = [](const int32_t* at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
  const auto store = [](int32_t* at, int v) { __hip_atomic_store(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
  // visit(there, b, at, id, begun): every thread at once, columns in order; `there` false past the last.  `begun`: the page
  // holds earlier positions.  Requests that do not fit the table are counted and have no columns.
  int refused = 0;
  const auto each = [&](auto&& visit) {
    for (int b0 = 0; b0 < p.n_seqs; b0 += kPlanThreads) {
      const int b = b0 + tid;
      int64_t lo = 0, hi = 0, held = 0;
      bool wrong = false;
      if (b < p.n_seqs) {
        const Span s = span_of(batch, b);
        const int64_t n = s.end - s.begin;
        held = p.held[b];
        if (n > 0) {
          wrong = held < 0 || div_ceil(held + n, p.page) > p.cols;
          lo = wrong ? 0 : div_up_to(held, p.page);
          hi = wrong ? 0 : div_ceil(held + n, p.page);
        }
      }
      refused += __syncthreads_count(wrong);  // and the last thousand's readers are done
      int64_t total;
      columns.first[tid] = plan_scan<int64_t>(hi - lo, lds, tid, total);
      columns.lo[tid] = static_cast<int>(lo);
      columns.held[tid] = static_cast<int>(held);
      __syncthreads();
      for (int64_t u0 = 0; u0 < total; u0 += kPlanThreads) {
        const int64_t u = u0 + tid;
        const bool there = u < total;
        int at = 0;  // the last request whose columns begin at or before u
        for (int step = kPlanThreads / 2; step > 0; step >>= 1)
          if (columns.first[at + step] <= u) at += step;
        const int64_t j = columns.lo[at] + (u - columns.first[at]);
        const int64_t entry = there ? static_cast<int64_t>(b0 + at) * p.cols + j : 0;
        const int id = there ? p.table[entry] : -1;
        visit(there, b0 + at, entry, id >= 0 && id < p.n_pages ? id : -1, j * p.page < columns.held[at]);
      }
    }
    __threadfence();
    __syncthreads();
  };
  // A page's keeper writes to it, the others take pages of their own: its only owner; of several the last,
  // and none if requests that do not write name it too.
  each([&](bool, int b, int64_t, int id, bool) {
    if (id < 0) return;
    store(writers + id, 0);
    store(keeper + id, p.refs[id] > 1 ? -1 : b);
  });
  if (refused > 0) {
    if (tid < 4) m.status[tid] = tid == 3 ? refused : 0;
    return;
  }
  each([&](bool, int b, int64_t, int id, bool) {
    if (id < 0 || p.refs[id] <= 1) return;
    atomicAdd(writers + id, 1);
    atomicMax(keeper + id, b);
  });
  each([&](bool, int b, int64_t, int id, bool) {
    if (id < 0) return;
    const int refs = p.refs[id];
    if (refs > 1 && load(keeper + id) == b && refs > load(writers + id)) store(keeper + id, -1);
  });
  int64_t taken = 0, moved = 0, wanted, moves;
  each([&](bool there, int b, int64_t, int id, bool begun) {
    const bool left = id >= 0 && load(keeper + id) != b;
    taken += there && (id < 0 || left);
    moved += left && begun;
  });
  plan_scan<int64_t>(taken, lds, tid, wanted);
  plan_scan<int64_t>(moved, lds, tid, moves);
  int found = 0;
  for (int id0 = 0; id0 < p.n_pages && found < wanted; id0 += 4 * kPlanThreads) {
    const int id = id0 + 4 * tid;
    bool open[4];
    int n = 0, total;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      open[e] = id + e < p.n_pages && p.refs[id + e] <= 0;
      n += open[e];
    }
    int at = found + plan_scan(n, lds, tid, total);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (open[e]) free[at++] = id + e;
    found += total;
  }
  if (found < wanted || moves > m.capacity) {
    const int64_t missing = wanted - found < 1 ? 1 : (wanted - found < 0x7fffffff ? wanted - found : 0x7fffffff);
    if (tid < 4) m.status[tid] = tid == 2 ? static_cast<int>(missing) : 0;
    return;
  }
  __threadfence();
  __syncthreads();
  // All is decided, by keepers alone: from here on tables and counts are written.
  int64_t take = 0, move = 0;
  each([&](bool there, int b, int64_t entry, int id, bool begun) {
    const bool left = id >= 0 && load(keeper + id) != b, taking = there && (id < 0 || left), moving = left && begun;
    int all;  // columns that take a page, and in the upper half those whose page moves: up to 1024 of each
    const int before = plan_scan((taking ? 1 : 0) | (moving ? 1 << 16 : 0), lds, tid, all);
    if (taking) {
      const int to = free[take + (before & 0xffff)];
      p.table[entry] = to;
      p.refs[to] = 1;
      if (left) atomicSub(p.refs + id, 1);
      if (moving) {
        const int64_t k = 2 * (move + (before >> 16));
        m.pairs[k] = id;
        m.pairs[k + 1] = to;
      }
    }
    take += all & 0xffff;
    move += all >> 16;
  });
  if (tid < 4) m.status[tid] = tid == 0 ? static_cast<int>(moves) : 0;
}

// The pages in use become pages 0 .. n - 1: the k-th of those behind goes to the k-th free one in front.
__global__ __launch_bounds__(kPlanThreads) void pages_compact_kernel(PagePool p, int32_t* refs_out, PageMoves m,
                                                                     int32_t* ws) {
  __shared__ PlanLds lds;
  const int tid = threadIdx.x;
  int32_t* to = ws;                 // [n_pages] where a page goes
  int32_t* high = to + p.n_pages;   // [n_pages] pages that move, counts with them
  int32_t* hole = high + p.n_pages;
  int mine = 0, used;
  for (int id = tid; id < p.n_pages; id += kPlanThreads) mine += p.refs[id] > 0;
  plan_scan(mine, lds, tid, used);
  int highs = 0, holes = 0;
  for (int id0 = 0; id0 < p.n_pages; id0 += 4 * kPlanThreads) {
    const int id = id0 + 4 * tid;
    int refs[4], n = 0, k = 0, total;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      refs[e] = id + e < p.n_pages ? p.refs[id + e] : 0;
      n += refs[e] > 0 && id + e >= used;
      k += id + e < used && refs[e] <= 0;
    }
    int at = highs + plan_scan(n, lds, tid, total);
    highs += total;
    int gap = holes + plan_scan(k, lds, tid, total);
    holes += total;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (id + e >= p.n_pages) continue;
      to[id + e] = id + e;
      if (refs[e] > 0 && id + e >= used) high[at++] = id + e;
      if (id + e < used && refs[e] <= 0) hole[gap++] = id + e;
      refs_out[id + e] = refs[e] > 0 ? refs[e] : 0;
    }
  }
  __threadfence();
  __syncthreads();
  // as many holes in front as pages behind; no more than half of the pool, which the list holds
  for (int k = tid; k < highs; k += kPlanThreads) {
    const int from = high[k], gap = hole[k];
    to[from] = gap;
    refs_out[gap] = refs_out[from];
    refs_out[from] = 0;
    m.pairs[2 * static_cast<int64_t>(k)] = from;
    m.pairs[2 * static_cast<int64_t>(k) + 1] = gap;
  }
  if (tid < 4) m.status[tid] = tid == 0 ? highs : tid == 1 ? used : 0;
}

__global__ __launch_bounds__(256) void pages_rename_kernel(PagePool p, int32_t* table_out, const int32_t* to, int64_t n) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int id = p.table[i];
    table_out[i] = id >= 0 && id < p.n_pages ? to[id] : -1;
  }
}

// Units of kPiece bytes of one move of one plane, dealt to as many workgroups as the chip holds: the count of
// moves is read on the device.  Four 16-byte loads a thread are under way before the first store.
constexpr int kPiece = 16384;
__global__ __launch_bounds__(256) void pages_copy_kernel(PagesCopyParams p, int64_t pieces) {
  const int tid = threadIdx.x;
  int n = p.moves.status[0];
  n = n < 0 ? 0 : (n > p.moves.capacity ? p.moves.capacity : n);
  const int64_t units = pieces * n;  // pieces: of a page in all planes
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    // a move's pieces lie in different planes: neighbours take the same piece of neighbouring moves
    const int64_t piece = unit / n;
    const int k = static_cast<int>(unit - piece * n);
    int64_t left = piece;
    int plane = 0;
    for (;; ++plane) {
      const int64_t of = (p.planes[plane].page_bytes + kPiece - 1) / kPiece;
      if (left < of) break;
      left -= of;
    }
    const int from = p.moves.pairs[2 * static_cast<int64_t>(k)], to = p.moves.pairs[2 * static_cast<int64_t>(k) + 1];
    if (from < 0 || from >= p.n_pages || to < 0 || to >= p.n_pages) continue;
    const int64_t bytes = p.planes[plane].page_bytes, at = left * kPiece;
    const char* src = p.planes[plane].data + from * bytes + at;
    char* dst = p.planes[plane].data + to * bytes + at;
    const int size = static_cast<int>(bytes - at < kPiece ? bytes - at : kPiece);
    if (bytes % 16 == 0) {
      u32x4 x[kPiece / 4096];
#pragma unroll
      for (int j = 0; j < kPiece / 4096; ++j)
        if (16 * tid + 4096 * j < size) x[j] = *reinterpret_cast<const u32x4*>(src + 16 * tid + 4096 * j);
#pragma unroll
      for (int j = 0; j < kPiece / 4096; ++j)
        if (16 * tid + 4096 * j < size) *reinterpret_cast<u32x4*>(dst + 16 * tid + 4096 * j) = x[j];
    } else {
      for (int i = 4 * tid; i < size; i += 1024)
        *reinterpret_cast<uint32_t*>(dst + i) = *reinterpret_cast<const uint32_t*>(src + i);
    }
  }
}

size_t pages_workspace(int64_t n_pages) {
  return static_cast<size_t>(3 * n_pages) * sizeof(int32_t);
}

hipError_t launch_pages_free(const PagePool& p, int n, const int32_t* seqs, hipStream_t stream) {
  hipLaunchKernelGGL(pages_free_kernel, dim3(n), dim3(256), 0, stream, p, seqs);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PagePool& p, int n, const int32_t* src, const int32_t* dst, hipStream_t stream) {
  hipLaunchKernelGGL(pages_fork_kernel, dim3(n), dim3(256), 0, stream, p, n, src, dst);
  return hipGetLastError();
}

hipError_t launch_pages_reserve(const PagePool& p, const SeqBatch& b, const PageMoves& m, int32_t* ws,
                                hipStream_t stream) {
  hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(kPlanThreads), 0, stream, p, b, m, ws);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagePool& p, const PagePool& out, const PageMoves& m, int32_t* ws,
                                hipStream_t stream) {
  hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(kPlanThreads), 0, stream, p, out.refs, m, ws);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t n = static_cast<int64_t>(p.n_seqs) * p.cols;
  hipLaunchKernelGGL(pages_rename_kernel, dim3(static_cast<unsigned>(std::min<int64_t>((n + 255) / 256, 2048))), dim3(256),
                     0, stream, p, out.table, ws, n);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PagesCopyParams& p, hipStream_t stream) {
  int64_t pieces = 0;
  for (int i = 0; i < p.n_planes; ++i) pieces += (p.planes[i].page_bytes + kPiece - 1) / kPiece;
  const int64_t blocks = std::min<int64_t>(2048, pieces * p.moves.capacity);
  hipLaunchKernelGGL(pages_copy_kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, p, pieces);
  return hipGetLastError();
}

}  // namespace scd
