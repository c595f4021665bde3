// Causal attention over dense keys and values (gfx950), key and value rows of different widths, grouped heads.
//
// A workgroup takes a tile of query rows of one KV head (its group's heads side by side) and goes through the
// positions in blocks that four waves fetch into LDS ahead of the arithmetic.  With 128 rows the matrix cores
// and the LDS reads of the right operands take about the same time, and the softmax's exponentials and maxima run
// beside them in the other workgroup of the CU.  2048 rows behind 6144 positions, 32 heads of 192 and 128: 320 to 344 us,
// 875 to 940 TFLOP/s, the matrix cores busy 38% of the time, the vector units 36%, LDS 31%, on two waves a SIMD: within a
// wave the products wait for the keys, the exponentials for the scores, the values' products for both, and for their own
// reads out of LDS.  A token of 64 requests of 8000 positions, 8 key heads: 368 us, 5.7 TB/s.
#pragma once

#include "scd_attend_core.h"

namespace scd {
using namespace dev;

// kWide: all rows of keys and values start on 16 bytes.
template <typename T, int kKey, int kValue, int NT, bool kWide>
struct RowsShape {
  static constexpr int kVec = Elem<T>::kVec, kStep = Elem<T>::kStep;
  // With 128 rows a wave has work enough for a step of positions between two barriers, and blocks of one leave room
  // for a second workgroup on the CU; tiles of fewer rows have two waves take a step each.
  static constexpr int kBlock = NT == 2 ? kStep : 2 * kStep;
  static constexpr int kKeyPieces = kKey / kVec + 1;
  // a column of keys takes 16 rows by 16 bytes; of values, transposed, 8 rows by 32 bytes or 4 by 64: each in its own banks
  static constexpr int kValuePieces = kValue / kVec + (sizeof(T) == 2 ? 2 : 1);
  typedef Copies<kBlock, kKeyPieces> KeyCopies;
  typedef Copies<kBlock, kValuePieces> ValueCopies;
  static constexpr int kBlockBytes = KeyCopies::kBytes + ValueCopies::kBytes;
  static constexpr int kRing = kBlockBytes * 3 <= 80 * 1024 ? 3 : kBlockBytes * 2 <= 80 * 1024 ? 2 :
                               kBlockBytes * 3 <= 156 * 1024 ? 3 : 2;
  static constexpr int kMine = KeyCopies::kMine + ValueCopies::kMine;
  typedef AttendCore<T, kKey / (4 * kVec), kValue / 16, NT, 0, kKeyPieces * kVec, kValuePieces * kVec> Core;
};

// Rows that do not start on 16 bytes, element by element.
template <typename T, int kBlock, int kPieces>
__device__ inline void fetch_odd_rows(const T* from, int64_t stride, int pieces, int pos0, int seen, char* to, int wave,
                                      int lane) {
  constexpr int kVec = Elem<T>::kVec;
  typedef Copies<kBlock, kPieces> C;
#pragma unroll 1
  for (int j = 0; j < C::kMine; ++j) {
    const int row = C::row(wave, j, lane), pos = pos0 + row < seen ? pos0 + row : seen - 1;
    const T* src = from + pos * stride + kVec * C::piece(wave, j, lane, pieces);
    union { T t[kVec]; u32x4 v; } x;
#pragma unroll
    for (int e = 0; e < kVec; ++e) x.t[e] = src[e];
    *reinterpret_cast<u32x4*>(to + C::index(wave, j) * 1024 + 16 * lane) = x.v;
  }
}

template <typename T, int kKey, int kValue, int NT, bool kWide>
__global__ __launch_bounds__(256, 2) void rows_attend_kernel(RowsAttendParams p) {
  typedef RowsShape<T, kKey, kValue, NT, kWide> S;
  typedef typename S::Core Core;
  constexpr int kStep = S::kStep, kVec = S::kVec, kKeyBytes = S::KeyCopies::kBytes;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ ShareLds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, g = lane >> 4;

  // positions that a request's rows can attend to: those its dense rows hold, up to its last query's
  const auto length = [&](const Span& s, int b) {
    const Span held = span_of(p.held, b);
    const int64_t rows = held.end - held.begin, upto = s.pos0 + (s.end - s.begin) - held.pos0;
    return upto < 0 ? int64_t{0} : (upto < rows ? upto : rows);
  };
  Share sh;
  if (!find_share<256>(p.batch, p.plan, S::kBlock, 2, blockIdx.x, lds, tid, length, sh)) return;
  const Span held = uniform(span_of(p.held, sh.b));
  sh.len = uniform(sh.len);
  // the tiles that see most come first
  const int tile = sh.tiles - 1 - sh.tile;

  const int group = p.plan.per_token;
  const int n_rows = static_cast<int>(sh.span.end - sh.span.begin) * group;
  const int row0 = tile * p.plan.rows;
  const int tile_rows = n_rows - row0 < p.plan.rows ? n_rows - row0 : p.plan.rows;
  const int64_t base = sh.span.pos0 - held.pos0;  // the first query's place among the dense rows
  int64_t seen = base + (row0 + tile_rows - 1) / group + 1;
  seen = seen < 0 ? 0 : (seen > sh.len ? sh.len : seen);
  const int blocks = static_cast<int>((seen + S::kBlock - 1) / S::kBlock);
  const int first = static_cast<int>(static_cast<int64_t>(blocks) * sh.part / sh.parts);
  const int last = static_cast<int>(static_cast<int64_t>(blocks) * (sh.part + 1) / sh.parts);
  const int64_t unit = sh.first + static_cast<int64_t>(sh.part) * sh.tiles;
  if (p.parts != nullptr && sh.part == 0 && tid < tile_rows) {
    const int row = row0 + tid;
    p.parts[(sh.span.begin + row / group) * p.q.n_heads + sh.head * group + row % group] =
        RowParts{static_cast<int>(sh.first), sh.tiles, sh.parts, tid};
  }

  const int wr = wave % p.plan.row_groups, wp = wave / p.plan.row_groups;
  const bool both = p.plan.row_groups == 4;
  const bool works = both || wp < 2;

  Core core;
  core.clear();
  int lowest = 0;
  {
    const int64_t low = base + row0 / group;
    lowest = low < -1 ? -1 : (low >= seen ? static_cast<int>(seen) - 1 : static_cast<int>(low));
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    int row = (wr * NT + n) * 16 + lr;
    row = row0 + (row < tile_rows ? row : tile_rows - 1);
    const int64_t at = base + row / group;
    core.limit[n] = at < 0 ? -1 : (at >= sh.len ? static_cast<int>(sh.len) - 1 : static_cast<int>(at));
    const T* q = reinterpret_cast<const T*>(p.q.data) + (sh.span.begin + row / group) * p.q.token +
                 (sh.head * group + row % group) * p.q.head;
#pragma unroll
    for (int f = 0; f < kKey / (4 * kVec); ++f) {
      union { T t[kVec]; u32x4 u; typename Core::Frag v; } x;
      x.u = u32x4{0, 0, 0, 0};
      if (works) {
        const T* from = q + 4 * kVec * f + kVec * g;
        if (p.q.wide) {
          x.u = *reinterpret_cast<const u32x4*>(from);
        } else {
#pragma unroll
          for (int e = 0; e < kVec; ++e) x.t[e] = from[e];
        }
        // a negative scale is its magnitude and queries of the other sign
        if (p.scale < 0.f) x.u ^= sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
      }
      core.q[n][f] = x.v;
    }
  }

  if (first < last) {
    const float scale = fabsf(p.scale);
    const T* keys = reinterpret_cast<const T*>(p.k.data) + held.begin * p.k.token + sh.head * p.k.head;
    const T* vals = reinterpret_cast<const T*>(p.v.data) + held.begin * p.v.token + sh.head * p.v.head;
    // where a lane's pieces lie from the block's first row on
    const int key_pieces = kKey / kVec, value_pieces = p.value / kVec;
    const uint32_t key_stride = static_cast<uint32_t>(p.k.token * sizeof(T)), value_stride = static_cast<uint32_t>(p.v.token * sizeof(T));
    uint32_t key_at[S::KeyCopies::kMine], value_at[S::ValueCopies::kMine];
    if constexpr (kWide) {
#pragma unroll
      for (int j = 0; j < S::KeyCopies::kMine; ++j)
        key_at[j] = S::KeyCopies::row(wave, j, lane) * key_stride + 16 * S::KeyCopies::piece(wave, j, lane, key_pieces);
#pragma unroll
      for (int j = 0; j < S::ValueCopies::kMine; ++j)
        value_at[j] = S::ValueCopies::row(wave, j, lane) * value_stride + 16 * S::ValueCopies::piece(wave, j, lane, value_pieces);
    }
    const int end = static_cast<int>(seen);
    const auto fetch = [&](int block, int slot) {
      char* to = smem + slot * S::kBlockBytes;
      const int pos0 = block * S::kBlock;
      if constexpr (kWide) {
        const char* kb = reinterpret_cast<const char*>(keys + static_cast<int64_t>(pos0) * p.k.token);
        const char* vb = reinterpret_cast<const char*>(vals + static_cast<int64_t>(pos0) * p.v.token);
        // rows from `end` on are behind the region: zeros
        const int64_t rows = end - pos0 - 1;
        const int64_t key_bytes = rows * key_stride + 16 * key_pieces, value_bytes = rows * value_stride + 16 * value_pieces;
#pragma unroll
        for (int j = 0; j < S::KeyCopies::kMine; ++j) copy16(kb, key_bytes, key_at[j], to + S::KeyCopies::index(wave, j) * 1024);
#pragma unroll
        for (int j = 0; j < S::ValueCopies::kMine; ++j)
          copy16(vb, value_bytes, value_at[j], to + kKeyBytes + S::ValueCopies::index(wave, j) * 1024);
      } else {
        fetch_odd_rows<T, S::kBlock, S::kKeyPieces>(keys, p.k.token, key_pieces, pos0, end, to, wave, lane);
        fetch_odd_rows<T, S::kBlock, S::kValuePieces>(vals, p.v.token, value_pieces, pos0, end, to + kKeyBytes, wave, lane);
      }
    };
    constexpr int kAhead = S::kRing - 1;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fetch(first + i < last ? first + i : last - 1, i);
    // blocks that all rows of the tile see whole, then those that some leave a part of out
    int slot = 0;
    const int whole = (lowest + 1) / S::kBlock;
    const auto run = [&](int block, auto careful) {
      wait_copies<(kAhead - 1) * S::kMine>();
      lds_barrier();
      fetch(block + kAhead < last ? block + kAhead : last - 1, slot == 0 ? S::kRing - 1 : slot - 1);
      if (works) {
        const char* at = smem + slot * S::kBlockBytes;
        const T* k = reinterpret_cast<const T*>(at);
        const T* v = reinterpret_cast<const T*>(at + kKeyBytes);
        constexpr int kSteps = S::kBlock / kStep;
        for (int st = both ? 0 : wp; st < (both ? kSteps : wp + 1); ++st)
          core.template step<decltype(careful)::value != 0>(k + st * kStep * (S::kKeyPieces * kVec),
                                                            v + st * kStep * (S::kValuePieces * kVec), scale,
                                                            block * S::kBlock + st * kStep, 0, lane);
      }
      slot = slot + 1 == S::kRing ? 0 : slot + 1;
    };
    int block = first;
    for (; block < last && block < whole; ++block) run(block, IntC<0>{});
    for (; block < last; ++block) run(block, IntC<1>{});
    wait_copies<0>();
    settle();
  }

  constexpr int kLine = kValue + 4;
  if (!both) {
    float* rest = reinterpret_cast<float*>(smem);
    lds_barrier();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float* row = rest + ((wr * NT + n) * 16 + lr) * kLine;
      if (wp == 1) {
        const float total = core.sum(n);
        if (g == 0) {
          row[kValue] = core.m[n];
          row[kValue + 1] = total;
        }
#pragma unroll
        for (int c = 0; c < kValue / 16; ++c) *reinterpret_cast<f32x4*>(row + 16 * c + 4 * g) = core.o[n][c];
      }
    }
    lds_barrier();
    if (wp != 0) return;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float* row = rest + ((wr * NT + n) * 16 + lr) * kLine;
      const float other = row[kValue], now = fmaxf(core.m[n], other), zero = now == -INFINITY ? 0.f : now;
      const float mine = __builtin_amdgcn_exp2f(core.m[n] - zero), its = __builtin_amdgcn_exp2f(other - zero);
      core.l[n] = core.sum(n) * mine + row[kValue + 1] * its;
      core.m[n] = now;
#pragma unroll
      for (int c = 0; c < kValue / 16; ++c) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(row + 16 * c + 4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) core.o[n][c][i] = core.o[n][c][i] * mine + x[i] * its;
      }
    }
  }
  const int line = p.value + 2;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int in_tile = (wr * NT + n) * 16 + lr, row = row0 + in_tile;
    const float total = both ? core.sum(n) : core.l[n];
    if (in_tile >= tile_rows) continue;
    if (sh.parts > 1) {
      float* out = p.slots + (unit * p.plan.rows + in_tile) * line;
      if (g == 0) *reinterpret_cast<float2*>(out) = make_float2(core.m[n], total);
#pragma unroll
      for (int c = 0; c < kValue / 16; ++c)
        if (16 * c < p.value) {
          float2* to = reinterpret_cast<float2*>(out + 2 + 16 * c + 4 * g);
          to[0] = make_float2(core.o[n][c][0], core.o[n][c][1]);
          to[1] = make_float2(core.o[n][c][2], core.o[n][c][3]);
        }
      continue;
    }
    const float by = total == 0.f ? 0.f : 1.f / total;
    T* out = reinterpret_cast<T*>(p.out.data) + (sh.span.begin + row / group) * p.out.token +
             (sh.head * group + row % group) * p.out.head + 4 * g;
#pragma unroll
    for (int c = 0; c < kValue / 16; ++c)
      if (16 * c < p.value) {
        const f32x4 x = core.o[n][c] * by;
        if (p.out.wide) {
          if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint2*>(out + 16 * c) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
          } else {
            *reinterpret_cast<f32x4*>(out + 16 * c) = x;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) store1(out + 16 * c + i, x[i]);
        }
      }
  }
}

template <typename T, int kKey, int kValue, int NT, bool kWide>
hipError_t launch_rows_shape(const RowsAttendParams& p, hipStream_t stream) {
  typedef RowsShape<T, kKey, kValue, NT, kWide> S;
  static_assert(NT == 2 || 32 * (kValue + 4) * 4 <= S::kRing * S::kBlockBytes, "the halves' join fits the ring");
  hipLaunchKernelGGL((rows_attend_kernel<T, kKey, kValue, NT, kWide>), dim3(static_cast<unsigned>(p.plan.grid)), dim3(256),
                     S::kRing * S::kBlockBytes, stream, p);
  return hipGetLastError();
}
// Keys of every width have an instance of their own: a padded one would multiply zeros of the query by whatever lies
// behind a key's row, and by infinities of its last piece.  Values are padded: their columns past the row are not stored.
template <typename T, int kKey, int NT, bool kWide>
hipError_t launch_rows_key(const RowsAttendParams& p, hipStream_t stream) {
  return p.value <= 64 ? launch_rows_shape<T, kKey, 64, NT, kWide>(p, stream)
                       : launch_rows_shape<T, kKey, 128, NT, kWide>(p, stream);
}
template <typename T, int NT, bool kWide>
hipError_t launch_rows_as(const RowsAttendParams& p, hipStream_t stream) {
  switch (p.key) {
    case 32: return launch_rows_key<T, 32, NT, kWide>(p, stream);
    case 64: return launch_rows_key<T, 64, NT, kWide>(p, stream);
    case 96: return launch_rows_key<T, 96, NT, kWide>(p, stream);
    case 128: return launch_rows_key<T, 128, NT, kWide>(p, stream);
    case 160: return launch_rows_key<T, 160, NT, kWide>(p, stream);
    case 192: return launch_rows_key<T, 192, NT, kWide>(p, stream);
  }
  return hipErrorInvalidValue;  // refused before
}

hipError_t launch_rows_bf16(const RowsAttendParams& p, hipStream_t stream);
hipError_t launch_rows_f32(const RowsAttendParams& p, hipStream_t stream);
hipError_t launch_odd_rows(bool bf16, const RowsAttendParams& p, hipStream_t stream);

}  // namespace scd
