// Attention of absorbed queries over the paged latents (gfx950): every head's query row, already in the
// latents' space, against the rows that all heads share.
//
// A latent row is key and value at once: it is fetched once (16 bytes a lane, straight into LDS, a ring of
// blocks ahead of the arithmetic) and read there twice, as rows for the scores and, transposed on the way
// out of LDS, for the weighted sum.  With 16 to 64 query rows a position the arithmetic is a fifth to a half
// of what the matrix cores do in the time a row takes to arrive, so the call is bound by HBM while there are
// enough positions, and a workgroup a CU with two blocks in flight is what keeps HBM busy.
#pragma once

#include "scd_attend_core.h"

namespace scd {
using namespace dev;

// kWide: the widest latent that this instance takes; NT: 16-row tiles of a wave.
template <typename T, int kWide, int NT>
struct LatentShape {
  static constexpr int kParts = sizeof(T) == 2 ? 2 : 1;         // summands of an absorbed query
  static constexpr int kVec = Elem<T>::kVec;
  static constexpr int kMostTurned = 64;
  static constexpr int kBlock = 2 * Elem<T>::kStep;             // positions of an LDS block
  // 16-byte pieces of an LDS row: an odd number, so that a column's pieces lie in different banks
  static constexpr int kPieces = (kWide + kMostTurned) / kVec + 1;
  typedef dev::Copies<kBlock, kPieces> Copies;
  static constexpr int kRow = kPieces * kVec;                   // elements
  static constexpr int kBlockBytes = Copies::kBytes;
  static constexpr int kRing = kBlockBytes * 4 <= 110 * 1024 ? 4 : kBlockBytes * 3 <= 150 * 1024 ? 3 : 2;
  static constexpr int kIds = 1024;
  static constexpr int kFrags = (kWide + kMostTurned) / (4 * kVec), kTiles = kWide / 16;
  typedef AttendCore<T, kFrags, kTiles, NT, kParts, kRow, kRow> Core;
  static constexpr int kLds = kRing * kBlockBytes + kIds * 4;
};

template <typename T, int kWide, int NT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void latent_attend_kernel(LatentAttendParams p) {
  typedef LatentShape<T, kWide, NT> S;
  typedef typename S::Core Core;
  constexpr int kStep = Elem<T>::kStep, kVec = S::kVec;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ ShareLds lds;
  int* ids = reinterpret_cast<int*>(smem + S::kRing * S::kBlockBytes);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, g = lane >> 4;

  const int64_t cap = p.plan.cap;
  const auto length = [&](const Span& s, int) {
    const int64_t n = s.pos0 + (s.end - s.begin);
    return n < 0 ? int64_t{0} : (n > cap ? cap : n);
  };
  Share sh;
  if (!find_share<256>(p.batch, p.plan, S::kBlock, 2, blockIdx.x, lds, tid, length, sh)) return;
  sh.len = uniform(sh.len);

  const int width = p.cache.latent + p.cache.turned;
  const int n_rows = static_cast<int>(sh.span.end - sh.span.begin) * p.heads;
  const int row0 = sh.tile * p.plan.rows;
  const int tile_rows = n_rows - row0 < p.plan.rows ? n_rows - row0 : p.plan.rows;
  // positions the tile's last row attends to, and this share's blocks of them
  int64_t seen = sh.span.pos0 + (row0 + tile_rows - 1) / p.heads + 1;
  seen = seen < 0 ? 0 : (seen > sh.len ? sh.len : seen);
  const int blocks = static_cast<int>((seen + S::kBlock - 1) / S::kBlock);
  const int first = static_cast<int>(static_cast<int64_t>(blocks) * sh.part / sh.parts);
  const int last = static_cast<int>(static_cast<int64_t>(blocks) * (sh.part + 1) / sh.parts);
  const int64_t unit = sh.first + static_cast<int64_t>(sh.part) * sh.tiles;
  if (sh.part == 0 && tid < tile_rows)
    p.parts[sh.span.begin * p.heads + row0 + tid] =
        RowParts{static_cast<int>(sh.first), sh.tiles, sh.parts, tid};

  // waves side by side over the tile's rows, and, where rows are few, over a block's two steps
  const int wr = wave % p.plan.row_groups, wp = wave / p.plan.row_groups;
  const bool both = p.plan.row_groups == 4;
  const bool works = both || wp < 2;

  Core core;
  core.clear();
  int lowest = 0x7fffffff;  // of the tile's limits
  {
    const int64_t low = sh.span.pos0 + row0 / p.heads;
    lowest = low < -1 ? -1 : (low >= seen ? static_cast<int>(seen) - 1 : static_cast<int>(low));
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    int row = (wr * NT + n) * 16 + lr;
    row = row0 + (row < tile_rows ? row : tile_rows - 1);
    const int64_t at = sh.span.pos0 + row / p.heads;
    core.limit[n] = at < 0 ? -1 : (at >= sh.len ? static_cast<int>(sh.len) - 1 : static_cast<int>(at));
    const T* q = reinterpret_cast<const T*>(p.absorbed) + (sh.span.begin * p.heads + row) * (S::kParts * width);
#pragma unroll
    for (int i = 0; i < S::kParts; ++i)
#pragma unroll
      for (int f = 0; f < S::kFrags; ++f) {
        union { u32x4 u; typename Core::Frag v; } x;
        x.u = u32x4{0, 0, 0, 0};
        if (works && 4 * kVec * f < width) x.u = *reinterpret_cast<const u32x4*>(q + i * width + 4 * kVec * f + kVec * g);
        core.q[n][i][f] = x.v;
      }
  }

  if (first < last) {
    // page of every column from `window` on, -1 for a hole
    const int lg = p.cache.page_log2;
    const auto column = [&](int block) { return static_cast<int>((static_cast<int64_t>(block) * S::kBlock) >> lg); };
    int window = column(first);
    const auto fill = [&] {
      const int64_t cols = p.cache.cols;
      for (int i = tid; i < S::kIds; i += 256) {
        const int64_t col = static_cast<int64_t>(window) + i;
        const int id = col < cols ? p.cache.table[sh.b * cols + col] : -1;
        ids[i] = id >= 0 && id < p.cache.n_pages ? id : -1;
      }
    };
    fill();
    __syncthreads();

    // a lane's pieces: the page of their row among the block's, their place in it, the column among the window's
    const int pieces = width / kVec;
    const uint32_t row_bytes = static_cast<uint32_t>(width * sizeof(T));
    const uint64_t page_bytes = static_cast<uint64_t>(row_bytes) << lg;
    const int mask = (1 << lg) - 1;
    uint32_t place[S::Copies::kMine];
    int page[S::Copies::kMine];
#pragma unroll
    for (int j = 0; j < S::Copies::kMine; ++j) {
      const int row = S::Copies::row(wave, j, lane);
      page[j] = row >> lg;
      place[j] = (row & mask) * row_bytes + 16 * S::Copies::piece(wave, j, lane, pieces);
    }
    const int last_column = static_cast<int>((seen - 1) >> lg);
    const auto fetch = [&](int block, int slot) {
      const int pos0 = block * S::kBlock, col0 = pos0 >> lg;
      const uint32_t in_page = (pos0 & mask) * row_bytes;  // a page of more than a block
      int id[S::Copies::kMine];
#pragma unroll
      for (int j = 0; j < S::Copies::kMine; ++j) {
        // columns behind the last one that is seen are its page again
        const int col = col0 + page[j];
        id[j] = ids[(col < last_column ? col : last_column) - window];
      }
#pragma unroll
      for (int j = 0; j < S::Copies::kMine; ++j) {
        const uint32_t p0 = id[j] < 0 ? 0 : id[j];  // a hole's rows are left out: any page will do
        copy16(p.cache.pages + (p0 * page_bytes + (in_page + place[j])),
               smem + slot * S::kBlockBytes + S::Copies::index(wave, j) * 1024);
      }
    };
    constexpr int kAhead = S::kRing - 1;
    // the window covers the blocks up to this one
    const auto covered = [&](int block) {
      return (((static_cast<int64_t>(block) + 1) * S::kBlock - 1) >> lg) < static_cast<int64_t>(window) + S::kIds;
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fetch(first + i < last ? first + i : last - 1, i);
    int slot = 0;
    for (int block = first; block < last; ++block) {
      wait_copies<(kAhead - 1) * S::Copies::kMine>();
      lds_barrier();
      const int next = block + kAhead < last ? block + kAhead : last - 1;
      if (!covered(next)) {
        lds_barrier();
        window = column(block);
        fill();
        __syncthreads();
      }
      fetch(next, slot == 0 ? S::kRing - 1 : slot - 1);
      if (works) {
        const int pos = block * S::kBlock;
        const T* rows = reinterpret_cast<const T*>(smem + slot * S::kBlockBytes);
        // holes among the block's pages, a bit for every 16 positions
        const int col = static_cast<int>((static_cast<int64_t>(pos) + 16 * (lane & 3)) >> lg) - window;
        const int holes = static_cast<int>(__ballot(lane < S::kBlock / 16 && pos + 16 * lane < seen && ids[col] < 0));
        const bool careful = holes != 0 || pos + S::kBlock - 1 > lowest;
        for (int st = both ? 0 : wp; st < (both ? 2 : wp + 1); ++st) {
          const T* at = rows + st * kStep * S::kRow;
          const int bits = holes >> (st * (kStep / 16));
          if (careful) {
            core.template step<true>(at, at, 1.f, pos + st * kStep, bits, lane);
          } else {
            core.template step<false>(at, at, 1.f, pos + st * kStep, bits, lane);
          }
        }
      }
      slot = slot + 1 == S::kRing ? 0 : slot + 1;
    }
    wait_copies<0>();
  }

  // the two steps' halves become one through LDS, in which no copy is under way any more
  constexpr int kLine = kWide + 4;
  if (!both) {
    float* rest = reinterpret_cast<float*>(smem);
    lds_barrier();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float* row = rest + ((wr * NT + n) * 16 + lr) * kLine;
      if (wp == 1) {
        const float total = core.sum(n);
        if (g == 0) {
          row[kWide] = core.m[n];
          row[kWide + 1] = total;
        }
#pragma unroll
        for (int c = 0; c < S::kTiles; ++c) *reinterpret_cast<f32x4*>(row + 16 * c + 4 * g) = core.o[n][c];
      }
    }
    lds_barrier();
    if (wp != 0) return;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float* row = rest + ((wr * NT + n) * 16 + lr) * kLine;
      const float other = row[kWide], now = fmaxf(core.m[n], other), base = now == -INFINITY ? 0.f : now;
      const float mine = __builtin_amdgcn_exp2f(core.m[n] - base), its = __builtin_amdgcn_exp2f(other - base);
      core.l[n] = core.sum(n) * mine + row[kWide + 1] * its;
      core.m[n] = now;
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(row + 16 * c + 4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) core.o[n][c][i] = core.o[n][c][i] * mine + x[i] * its;
      }
    }
  }
  const int line = p.cache.latent + 2;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = (wr * NT + n) * 16 + lr;
    const float total = both ? core.sum(n) : core.l[n];
    if (row < tile_rows) {
      // lines of latent + 2 values: two-float stores keep to their alignment
      float* out = p.slots + (unit * p.plan.rows + row) * line;
      if (g == 0) *reinterpret_cast<float2*>(out) = make_float2(core.m[n], total);
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c)
        if (16 * c < p.cache.latent) {
          float2* to = reinterpret_cast<float2*>(out + 2 + 16 * c + 4 * g);
          to[0] = make_float2(core.o[n][c][0], core.o[n][c][1]);
          to[1] = make_float2(core.o[n][c][2], core.o[n][c][3]);
        }
    }
  }
}

template <typename T, int kWide, int NT>
hipError_t launch_latent_shape(const LatentAttendParams& p, hipStream_t stream) {
  typedef LatentShape<T, kWide, NT> S;
  constexpr int join = 32 * (kWide + 4) * 4 * NT;
  static_assert(join <= S::kRing * S::kBlockBytes, "the halves' join fits the ring");
  hipLaunchKernelGGL((latent_attend_kernel<T, kWide, NT>), dim3(static_cast<unsigned>(p.plan.grid)), dim3(256), S::kLds,
                     stream, p);
  return hipGetLastError();
}

hipError_t launch_latent_core_bf16(const LatentAttendParams& p, hipStream_t stream);
hipError_t launch_latent_core_f32(const LatentAttendParams& p, hipStream_t stream);

}  // namespace scd
