// Attention of absorbed queries over the paged latents (gfx950): every head's query row, already in the
// latents' space, against the rows that all heads share.
//
// A latent row is key and value at once: it is fetched once (16 bytes a lane, straight into LDS, a ring of
// blocks ahead of the arithmetic) and read there twice, as rows for the scores and, transposed on the way
// out of LDS, for the weighted sum.  With 16 to 64 query rows a position the arithmetic is a fifth to a half
// of what the matrix cores do in the time a row takes to arrive, so the call is bound by HBM while there are
// enough positions, and a workgroup a CU with two blocks in flight is what keeps HBM busy.  A token of 16 requests of 1K to
// 16K positions, 32 heads, r = 256: 31.5 to 32 us, of which 6 to 7 before the first block, then some 4 TB/s of cached rows.
#pragma once

#include "scd_attend_core.h"

namespace scd {
using namespace dev;

// kWide: the widest latent that this instance takes; kWaves waves, of which kHalves share a row's value channels: a
// wave's chain of LDS reads, scores, weights and products is far longer than its instructions take to issue, so a CU
// needs two on every SIMD, and where rows are few they are had by halves of the channels (both form the scores).
template <typename T, int kWide, int kWaves, int kHalves>
struct LatentShape {
  static constexpr int kVec = Elem<T>::kVec;
  static constexpr int kMostTurned = 64;
  static constexpr int kBlock = latent_block(sizeof(T) == 2);   // positions of an LDS block: two steps of a wave
  // 16-byte pieces of an LDS row: an odd number, so that a column's pieces lie in different banks
  static constexpr int kPieces = (kWide + kMostTurned) / kVec + 1;
  typedef dev::Copies<kBlock, kPieces, kWaves> Copies;
  static constexpr int kRow = kPieces * kVec;                   // elements
  static constexpr int kBlockBytes = Copies::kBytes;
  static constexpr int kRing = kBlockBytes * 4 <= 110 * 1024 ? 4 : kBlockBytes * 3 <= 150 * 1024 ? 3 : 2;
  static constexpr int kIds = 1024;
  static constexpr int kFrags = (kWide + kMostTurned) / (4 * kVec), kTiles = kWide / 16 / kHalves;
  static constexpr int kLatentFrags = kWide / (4 * kVec);
  // bf16 queries in the latents' space have a second summand
  static constexpr int kLow = sizeof(T) == 2 ? kLatentFrags : 0;
  typedef AttendCore<T, kFrags, kTiles, 1, kLow, kRow, kRow> Core;
  static constexpr int kLds = kRing * kBlockBytes + kIds * 4;
};

// kPadded: cached rows have a narrower latent or key than kWide and 64 channels.  LDS then holds zeros for the rest, so that
// no product of the queries' zeros there is one with an infinity.
template <typename T, int kWide, int kWaves, int kHalves, bool kPadded>
__global__ __launch_bounds__(64 * kWaves) void latent_attend_kernel(LatentAttendParams p) {
  typedef LatentShape<T, kWide, kWaves, kHalves> S;
  typedef typename S::Core Core;
  constexpr int kStep = Elem<T>::kStep, kVec = S::kVec;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  int* ids = reinterpret_cast<int*>(smem + S::kRing * S::kBlockBytes);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, g = lane >> 4;

  const LatentShare sh = p.shares[blockIdx.x];
  if (sh.b < 0) return;
  const int64_t begin = sh.begin, held = sh.held;
  int64_t len = held + sh.tokens;
  len = len < 0 ? 0 : (len > p.plan.cap ? p.plan.cap : len);

  const int width = p.cache.latent + p.cache.turned;
  const int n_rows = sh.tokens * p.heads;
  const int row0 = sh.tile * p.plan.rows;
  const int tile_rows = n_rows - row0 < p.plan.rows ? n_rows - row0 : p.plan.rows;
  // positions the tile's last row attends to, and this share's blocks of them
  int64_t seen = held + (row0 + tile_rows - 1) / p.heads + 1;
  seen = seen < 0 ? 0 : (seen > len ? len : seen);
  const int blocks = static_cast<int>((seen + S::kBlock - 1) / S::kBlock);
  const int first = static_cast<int>(static_cast<int64_t>(blocks) * sh.part / sh.parts);
  const int last = static_cast<int>(static_cast<int64_t>(blocks) * (sh.part + 1) / sh.parts);
  const int64_t slot = uniform(sh.first + static_cast<int64_t>(sh.part) * sh.tiles);
  if (sh.part == 0 && tid < tile_rows)
    p.parts[begin * p.heads + row0 + tid] =
        RowParts{sh.first, sh.tiles, sh.parts, tid};

  // waves side by side over the tile's rows, over halves of the value channels, and, where rows are few, over a
  // block's two steps
  const int groups = p.plan.row_groups, wr = wave % groups, rest = wave / groups;
  const int wc = rest % kHalves, wp = rest / kHalves;
  const bool both = groups * kHalves == kWaves;
  const bool works = both || wp < 2;

  Core core;
  core.clear();
  int lowest = 0x7fffffff;  // of the tile's limits
  {
    const int64_t low = held + row0 / p.heads;
    lowest = low < -1 ? -1 : (low >= seen ? static_cast<int>(seen) - 1 : static_cast<int>(low));
  }
  int my_row = wr * 16 + lr;
  my_row = row0 + (my_row < tile_rows ? my_row : tile_rows - 1);
  {
    const int64_t at = held + my_row / p.heads;
    core.limit[0] = at < 0 ? -1 : (at >= len ? static_cast<int>(len) - 1 : static_cast<int>(at));
  }

  if (first < last) {
    // page of every column from `window` on, -1 for a hole
    const int lg = p.cache.page_log2;
    const auto column = [&](int block) { return static_cast<int>((static_cast<int64_t>(block) * S::kBlock) >> lg); };
    int window = column(first);
    const auto fill = [&] {
      const int64_t cols = p.cache.cols;
      for (int i = tid; i < S::kIds; i += 64 * kWaves) {
        const int64_t col = static_cast<int64_t>(window) + i;
        const int id = col < cols ? p.cache.table[sh.b * cols + col] : -1;
        ids[i] = id >= 0 && id < p.cache.n_pages ? id : -1;
      }
    };
    fill();
    __syncthreads();

    // A lane's pieces: the page of their row among the block's, their place in it, the column among the window's.  An LDS
    // row is a latent of kWide channels and a key of 64.
    const uint32_t row_bytes = static_cast<uint32_t>(width * sizeof(T));
    const uint64_t page_bytes = static_cast<uint64_t>(row_bytes) << lg;
    const int mask = (1 << lg) - 1;
    uint32_t place[S::Copies::kMine];  // the page (one of four at most) in bits 28 and 29, bit 31: zeros
#pragma unroll
    for (int j = 0; j < S::Copies::kMine; ++j) {
      const int row = S::Copies::row(wave, j, lane), at = (row & mask) * row_bytes;
      if constexpr (kPadded) {
        const int piece = S::Copies::piece(wave, j, lane);
        const bool key = piece >= kWide / kVec;
        const int of = key ? piece - kWide / kVec : piece, have = (key ? p.cache.turned : p.cache.latent) / kVec;
        place[j] = of < have ? (at + 16 * (of + (key ? p.cache.latent / kVec : 0))) | (row >> lg) << 28 : 1u << 31;
      } else {
        place[j] = (at + 16 * S::Copies::piece(wave, j, lane, (kWide + S::kMostTurned) / kVec)) | (row >> lg) << 28;
      }
    }
    const int last_column = static_cast<int>((seen - 1) >> lg);
    const auto fetch = [&](int block, int ring) {
      const int pos0 = block * S::kBlock, col0 = pos0 >> lg;
      const uint32_t in_page = (pos0 & mask) * row_bytes;  // a page of more than a block
      int id[S::Copies::kMine];
#pragma unroll
      for (int j = 0; j < S::Copies::kMine; ++j) {
        // columns behind the last one that is seen are its page again
        const int col = col0 + static_cast<int>(kPadded ? place[j] >> 28 & 3 : place[j] >> 28);
        id[j] = ids[(col < last_column ? col : last_column) - window];
      }
#pragma unroll
      for (int j = 0; j < S::Copies::kMine; ++j) {
        const uint32_t p0 = id[j] < 0 ? 0 : id[j];  // a hole's rows are left out: any page will do
        const char* at = p.cache.pages + (p0 * page_bytes + (in_page + (place[j] & 0xfffffff)));
        copy16(kPadded && static_cast<int>(place[j]) < 0 ? p.zeros : at,
               smem + ring * S::kBlockBytes + S::Copies::index(wave, j) * 1024);
      }
    };
    constexpr int kAhead = S::kRing - 1;
    // the window covers the blocks up to this one
    const auto covered = [&](int block) {
      return (((static_cast<int64_t>(block) + 1) * S::kBlock - 1) >> lg) < static_cast<int64_t>(window) + S::kIds;
    };
    // The tile's queries come by way of the ring's end, 16 bytes a lane of every row once: the waves that share a row
    // and rows' pieces in memory order would fetch it many times.  The blocks that fit in front of them are on their
    // way meanwhile.
    const int line = query_width(sizeof(T) == 2, p.cache.latent, p.cache.turned), query_pieces = line / kVec | 1;
    const int query_bytes = tile_rows * query_pieces * 16;
    char* queries = smem + S::kRing * S::kBlockBytes - ((query_bytes + 1023) & ~1023);
    const int early = static_cast<int>(queries - smem) / S::kBlockBytes < kAhead
                          ? static_cast<int>(queries - smem) / S::kBlockBytes : kAhead;
    const char* from = p.absorbed + (begin * p.heads + row0) * (line * static_cast<int64_t>(sizeof(T)));
    for (int i = wave * 64; i < tile_rows * query_pieces; i += 64 * kWaves) {
      const int row = (i + lane) / query_pieces, piece = i + lane - row * query_pieces;
      if (row < tile_rows && piece < line / kVec) copy16(from + (row * line + kVec * piece) * sizeof(T), queries + 16 * i);
    }
    for (int i = 0; i < early; ++i) fetch(first + i < last ? first + i : last - 1, i);
    if (early == kAhead) {
      wait_copies<kAhead * S::Copies::kMine>();
    } else {
      wait_copies<0>();
    }
    lds_barrier();
    const T* q = reinterpret_cast<const T*>(queries) + (my_row - row0) * query_pieces * kVec;
#pragma unroll
    for (int f = 0; f < S::kFrags; ++f) {
      union { u32x4 u; typename Core::Frag v; } x, y;
      x.u = y.u = u32x4{0, 0, 0, 0};
      const int of = f < S::kLatentFrags ? f : f - S::kLatentFrags;
      if (!kPadded || 4 * kVec * of < (f < S::kLatentFrags ? p.cache.latent : p.cache.turned))
        x.u = *reinterpret_cast<const u32x4*>(q + (f < S::kLatentFrags ? 0 : p.cache.latent) + 4 * kVec * of + kVec * g);
      core.q[0][f] = x.v;
      if (f < S::kLow) {
        if (!kPadded || 4 * kVec * f < p.cache.latent) y.u = *reinterpret_cast<const u32x4*>(q + width + 4 * kVec * f + kVec * g);
        core.low[0][f < S::kLow ? f : 0] = y.v;
      }
    }
    if (early < kAhead) {
      lds_barrier();
      for (int i = early; i < kAhead; ++i) fetch(first + i < last ? first + i : last - 1, i);
    }
    const float scale = fabsf(p.scale);
    int ring = 0;
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
      fetch(next, ring == 0 ? S::kRing - 1 : ring - 1);
      if (works) {
        const int pos = block * S::kBlock;
        const T* rows = reinterpret_cast<const T*>(smem + ring * S::kBlockBytes);
        // holes among the block's pages, a bit for every 16 positions
        const int col = static_cast<int>((static_cast<int64_t>(pos) + 16 * (lane & 3)) >> lg) - window;
        const int holes = static_cast<int>(__ballot(lane < S::kBlock / 16 && pos + 16 * lane < seen && ids[col] < 0));
        const bool careful = holes != 0 || pos + S::kBlock - 1 > lowest;
        for (int st = both ? 0 : wp; st < (both ? 2 : wp + 1); ++st) {
          const T* at = rows + st * kStep * S::kRow;
          const int bits = holes >> (st * (kStep / 16));
          if (careful) {
            core.template step<true>(at, at + wc * (kWide / kHalves), scale, pos + st * kStep, bits, lane);
          } else {
            core.template step<false>(at, at + wc * (kWide / kHalves), scale, pos + st * kStep, bits, lane);
          }
        }
      }
      ring = ring + 1 == S::kRing ? 0 : ring + 1;
    }
    wait_copies<0>();
    settle();
  }

  // what the two steps' waves have becomes one through LDS, in which no copy is under way any more
  constexpr int kLine = kWide + 4, kMine = kWide / kHalves;
  // the lane's place, which the loop above has no registers to keep
  const int at_lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), at_row = at_lane & 15, at_g = at_lane >> 4;
  float total = core.sum(0);
  if (!both) {
    float* row = reinterpret_cast<float*>(smem) + (wr * 16 + at_row) * kLine;
    lds_barrier();
    if (wp == 1) {
      if (at_g == 0) {
        row[kWide] = core.m[0];
        row[kWide + 1] = total;
      }
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c) *reinterpret_cast<f32x4*>(row + wc * kMine + 16 * c + 4 * at_g) = core.o[0][c];
    }
    lds_barrier();
    if (wp != 0) return;
    const float other = row[kWide], now = fmaxf(core.m[0], other), base = now == -INFINITY ? 0.f : now;
    const float mine = __builtin_amdgcn_exp2f(core.m[0] - base), its = __builtin_amdgcn_exp2f(other - base);
    total = total * mine + row[kWide + 1] * its;
    core.m[0] = now;
#pragma unroll
    for (int c = 0; c < S::kTiles; ++c) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(row + wc * kMine + 16 * c + 4 * at_g);
#pragma unroll
      for (int i = 0; i < 4; ++i) core.o[0][c][i] = core.o[0][c][i] * mine + x[i] * its;
    }
  }
  const int line = p.cache.latent + 2, row = wr * 16 + at_row;
  if (row < tile_rows) {
    // lines of latent + 2 values: two-float stores keep to their alignment
    float* out = p.slots + (slot * p.plan.rows + row) * line;
    if (at_g == 0 && wc == 0) *reinterpret_cast<float2*>(out) = make_float2(core.m[0], total);
#pragma unroll
    for (int c = 0; c < S::kTiles; ++c)
      if (wc * kMine + 16 * c < p.cache.latent) {
        float2* to = reinterpret_cast<float2*>(out + 2 + wc * kMine + 16 * c + 4 * at_g);
        to[0] = make_float2(core.o[0][c][0], core.o[0][c][1]);
        to[1] = make_float2(core.o[0][c][2], core.o[0][c][3]);
      }
  }
}

template <typename T, int kWide, int kWaves, int kHalves>
hipError_t launch_latent_shape(const LatentAttendParams& p, hipStream_t stream) {
  typedef LatentShape<T, kWide, kWaves, kHalves> S;
  static_assert((kHalves == 1 ? 64 : 32) * (kWide + 4) * 4 <= S::kRing * S::kBlockBytes, "the steps' join fits the ring");
  static_assert((kWaves * 16 / (kHalves == 2 ? 2 : 1)) * (((S::kLow > 0 ? 2 : 1) * kWide + 64) / S::kVec + 1) * 16 + 1024 <=
                    S::kRing * S::kBlockBytes, "the queries fit the ring");
  static_assert(S::kTiles % 4 == 0, "value tiles are read by fours");
  const dim3 grid(static_cast<unsigned>(p.plan.grid)), block(64 * kWaves);
  if (p.cache.latent == kWide && p.cache.turned == S::kMostTurned) {
    hipLaunchKernelGGL((latent_attend_kernel<T, kWide, kWaves, kHalves, false>), grid, block, S::kLds, stream, p);
  } else {
    hipLaunchKernelGGL((latent_attend_kernel<T, kWide, kWaves, kHalves, true>), grid, block, S::kLds, stream, p);
  }
  return hipGetLastError();
}
// Few rows with halves of the channels, more without: 64 rows are four waves for each of a block's steps, 128 eight
// (above 128 channels registers are too few for that, and up to 64 there is nothing to halve); latents above 256 channels, whose queries
// alone are 144 registers, up to 32 rows in four waves.
template <typename T>
hipError_t launch_latent_as(const LatentAttendParams& p, hipStream_t stream) {
  if (p.cache.latent <= 64) return launch_latent_shape<T, 64, 8, 1>(p, stream);
  if (p.cache.latent <= 128)
    return p.plan.rows >= 64 ? launch_latent_shape<T, 128, 8, 1>(p, stream) : launch_latent_shape<T, 128, 8, 2>(p, stream);
  if (p.cache.latent <= 256) return launch_latent_shape<T, 256, 8, 2>(p, stream);
  return launch_latent_shape<T, 512, 4, 2>(p, stream);
}

}  // namespace scd
