// The dense keys and values of cached latents (gfx950), for prompts: k_h = [W_k,h c | key], v_h = W_v,h c.
//
// A wave keeps 32 rows of the heads' matrices in registers for the whole call and takes tiles of cached rows
// from LDS, so the matrices are read once a workgroup and the latents once for every 256 channels; what is
// written, heads x (plain + turned + value) channels a row, is 20 times what is read and bounds the call: 20000 positions of
// 28 heads, r = 96, 98 to 104 us, 3.6 TB/s; of 32 heads, r = 256, 136 to 140 us, 3.1 TB/s and 610 TFLOP/s.
#include <algorithm>

#include "scd_attend_core.h"

namespace scd {
using namespace dev;

__device__ inline f32x16 mma32(const bf16x8& a, const bf16x8& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mma32(const f32x4& a, const f32x4& b, f32x16 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// 16 bytes of a row, element by element where it does not start on 16 bytes.
__device__ inline void put(uint16_t* out, bool wide, const u32x4& x) {
  if (wide) {
    *reinterpret_cast<u32x4*>(out) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = static_cast<uint16_t>(x[e >> 1] >> (16 * (e & 1)));
  }
}
__device__ inline void put(float* out, bool wide, const u32x4& x) {
  if (wide) {
    *reinterpret_cast<u32x4*>(out) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = __uint_as_float(x[e]);
  }
}

template <typename T, int kWide>
struct ExpandShape {
  static constexpr int kWaves = sizeof(T) == 4 && kWide == 512 ? 4 : 8;  // the latter's matrices are 256 registers
  static constexpr int kThreads = 64 * kWaves;
  static constexpr int kVec = Elem<T>::kVec, kRows = 32;
  static constexpr int kBuffers = sizeof(T) == 2 || kWide <= 256 ? 2 : 1;
  static constexpr int kPieces = (kWide + 64) / kVec + 1;  // of an LDS row, odd
  typedef dev::Copies<kRows, kPieces, kWaves> Copies;
  // a wave's results on their way out: 32 channels a row, and 16 bytes that keep rows off each other's banks
  static constexpr int kOutRow = 32 * sizeof(T) + 16, kOutBytes = kRows * kOutRow;
  static constexpr int kTiles = 16;                        // whose rows' places are looked up at once
  static constexpr int kLds = kBuffers * Copies::kBytes + kWaves * kOutBytes;
};

template <typename T, int kWide>
__global__ __launch_bounds__((ExpandShape<T, kWide>::kThreads)) void latent_expand_kernel(LatentExpandParams p, int64_t tiles) {
  typedef ExpandShape<T, kWide> S;
  constexpr int kVec = S::kVec, kRows = S::kRows, kRow = S::kPieces * kVec;
  constexpr int kFrags = kWide / (2 * kVec), kSure = kWide == 64 ? 32 : kWide / 2 + 32;  // channels that any latent has
  typedef typename Elem<T>::Frag Frag;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int64_t places[S::kTiles][kRows];  // byte of a row in the pages, -1: a hole, -2: no such row
  __shared__ int partly[S::kTiles];             // whether some of a tile's rows have no place
  constexpr int kStaged = 256;                  // requests whose bounds are kept in LDS
  __shared__ int bounds[kStaged + 1], starts[kStaged];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int latent = p.cache.latent, width = latent + p.cache.turned;
  char* const mine = smem + S::kBuffers * S::Copies::kBytes + wave * S::kOutBytes;

  // the wave's 32 channels: of a head's keys, or of its values
  const int per_head = (p.plain + p.value) / 32;
  const int group = blockIdx.x * S::kWaves + wave;
  const bool works = group < p.heads * per_head;
  const int head = works ? group / per_head : 0;
  int c0 = works ? (group - head * per_head) * 32 : 0;
  const bool values = c0 >= p.plain;
  if (values) c0 -= p.plain;
  Frag w[kFrags];
  {
    // matrix row m of the tile is channel row_of_lds(m): a lane then holds 16 adjacent channels of a result
    const T* at = reinterpret_cast<const T*>(values ? p.w_v : p.w_k) +
                  (static_cast<int64_t>(head) * (values ? p.value : p.plain) + c0 + row_of_lds(col)) * latent + kVec * half;
#pragma unroll
    for (int f = 0; f < kFrags; ++f) {
      union { u32x4 u; Frag v; } x;
      x.u = u32x4{0, 0, 0, 0};  // the pieces that lie there are the latent's last one again
      if (2 * kVec * f < latent) x.u = *reinterpret_cast<const u32x4*>(at + 2 * kVec * f);
      w[f] = x.v;
    }
  }
  const Rows& rows = values ? p.v : p.k;

  const bool staged = p.batch.n_seqs <= kStaged;
  if (staged) {
    for (int b = tid; b <= p.batch.n_seqs; b += S::kThreads) {
      bounds[b] = p.batch.cu != nullptr ? p.batch.cu[b] : (b == 0 ? 0 : 0x7fffffff);
      if (b < p.batch.n_seqs) starts[b] = p.batch.pos0 != nullptr ? p.batch.pos0[b] : 0;
    }
  }
  const auto resolve = [&](int64_t t) -> int64_t {
    if (t >= p.batch.n_tokens) return -2;
    int b = 0, hi = p.batch.n_seqs - 1;  // the last request that begins at or before t
    int64_t pos;
    if (staged) {
      if (t >= bounds[p.batch.n_seqs]) return -2;
      while (b < hi) {
        const int mid = (b + hi + 1) >> 1;
        if (bounds[mid] <= t) b = mid; else hi = mid - 1;
      }
      pos = t - bounds[b] + starts[b];
    } else {
      if (t >= p.batch.cu[p.batch.n_seqs]) return -2;
      while (b < hi) {
        const int mid = (b + hi + 1) >> 1;
        if (p.batch.cu[mid] <= t) b = mid; else hi = mid - 1;
      }
      pos = t - p.batch.cu[b] + (p.batch.pos0 != nullptr ? p.batch.pos0[b] : 0);
    }
    const int64_t column = pos >> p.cache.page_log2;
    if (pos < 0 || column >= p.cache.cols) return -1;
    const int id = p.cache.table[static_cast<int64_t>(b) * p.cache.cols + column];
    if (id < 0 || id >= p.cache.n_pages) return -1;
    return ((static_cast<int64_t>(id) << p.cache.page_log2) + (pos & (p.cache.page - 1))) *
           (width * static_cast<int64_t>(sizeof(T)));
  };
  // a row's latent, its last piece again up to kWide channels, and the shared key behind them
  const auto source = [&](int piece) {
    constexpr int kLatent = kWide / kVec;
    const int mine = latent / kVec, key = p.cache.turned / kVec;
    return piece < kLatent ? (piece < mine ? piece : mine - 1) : mine + (piece - kLatent < key ? piece - kLatent : key - 1);
  };
  const auto fetch = [&](const int64_t* from, int buffer) {
#pragma unroll
    for (int j = 0; j < S::Copies::kMine; ++j) {
      const int64_t place = from[S::Copies::row(wave, j, lane)];
      copy16(p.cache.pages + (place < 0 ? 0 : place) + 16 * source(S::Copies::piece(wave, j, lane, S::kPieces)),
             smem + buffer * S::Copies::kBytes + S::Copies::index(wave, j) * 1024);
    }
  };

  constexpr int kPer = 32 / kVec, kAt = 64 / kPer;  // pieces of a result's row, rows of a store
  constexpr int kStores = kRows / kAt;
  // heads' shared keys: rows of the tile dealt to the waves of the workgroup that has the first channels of a head
  const int first_group = blockIdx.x * S::kWaves;
  const int key_head = (first_group + per_head - 1) / per_head;  // the only one, if a head has as many groups as there are waves
  const bool keys = per_head >= S::kWaves && key_head * per_head < first_group + S::kWaves && key_head < p.heads;
  const int key_pieces = p.cache.turned / kVec;
  // where a lane's pieces of a tile go, from its first row's channels on
  const bool near = rows.token < (int64_t{1} << 23);  // a tile's rows lie within 32 bits
  uint32_t out_at[kStores];
#pragma unroll
  for (int j = 0; j < kStores; ++j)
    out_at[j] = static_cast<uint32_t>((j * kAt + lane / kPer) * rows.token + kVec * (lane % kPer)) * sizeof(T);
  char* const out_first = rows.data + (static_cast<int64_t>(head) * rows.head + c0) * sizeof(T);

  // row `row` of a tile's shared keys, behind every head's own channels
  const auto put_key = [&](int64_t tile, int h, int row, int piece, const char* from, int64_t place) {
    if (place == -2) return;
    u32x4 x = *reinterpret_cast<const u32x4*>(from + (row * kRow + kWide + kVec * piece) * sizeof(T));
    if (place < 0) x = u32x4{0, 0, 0, 0};
    put(reinterpret_cast<T*>(p.k.data) + (tile * kRows + row) * p.k.token + h * p.k.head + p.plain + kVec * piece, p.k.wide, x);
  };

  const int64_t step = gridDim.y;
  int it = 0;  // of the buffer
  for (int64_t tile0 = blockIdx.y; tile0 < tiles; tile0 += S::kTiles * step) {
    // places of the next kTiles tiles' rows; the last readers are done
    __syncthreads();
    if (tid < S::kTiles) partly[tid] = 0;
    __syncthreads();
    for (int i = tid; i < S::kTiles * kRows; i += S::kThreads) {
      const int64_t tile = tile0 + (i / kRows) * step;
      const int64_t place = resolve(tile * kRows + i % kRows);
      places[i / kRows][i % kRows] = place;
      if (place < 0) partly[i / kRows] = 1;
    }
    __syncthreads();
    fetch(places[0], it);
    // The first copies have landed when all has; from then on at most the stores may be under way that every
    // working wave issues, at least, behind a tile's copies.  (Where rows are missing there are fewer, and then the
    // tiles behind have no rows either.)
    for (int k = 0; k < S::kTiles && tile0 + k * step < tiles; ++k) {
      if (S::kBuffers == 2 && k > 0 && works) wait_copies<kStores>(); else wait_copies<0>();
      lds_barrier();
      const int64_t tile = tile0 + k * step;
      const char* from = smem + it * S::Copies::kBytes;
      const bool more = k + 1 < S::kTiles && tile + step < tiles;
      const bool whole = uniform(partly[k]) == 0;
      if (S::kBuffers == 2) {
        it ^= 1;
        if (more) fetch(places[k + 1], it);
      }
      if (works) {
        const T* at = reinterpret_cast<const T*>(from) + col * kRow + kVec * half;
        f32x16 acc;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.f;
        // pieces that the latent does not have are left out: there the matrix is zeros and the row its last piece again,
        // and an infinity of it would be NaN
#pragma unroll
        for (int c = 0; c < kWide; c += 32)
          if (c < kSure || c < latent) {
#pragma unroll
            for (int f = c / (2 * kVec); f < (c + 32) / (2 * kVec); ++f)
              acc = mma32(w[f], *reinterpret_cast<const Frag*>(at + 2 * kVec * f), acc);
          }
        settle();
        // out through LDS: whole runs of a row's 32 channels at a time
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = acc[i];
        if (!whole && places[k][col] < 0) {
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = 0.f;
        }
        T* to = reinterpret_cast<T*>(mine + col * S::kOutRow) + 16 * half;
        store8(to, true, x);
        store8(to + 8, true, x + 8);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const char* piece = mine + (lane / kPer) * S::kOutRow + 16 * (lane % kPer);
        u32x4 y[kStores];
#pragma unroll
        for (int j = 0; j < kStores; ++j) y[j] = *reinterpret_cast<const u32x4*>(piece + j * kAt * S::kOutRow);
        char* out = out_first + tile * kRows * rows.token * static_cast<int64_t>(sizeof(T));
        if (whole && rows.wide && near) {
#pragma unroll
          for (int j = 0; j < kStores; ++j) *reinterpret_cast<u32x4*>(out + out_at[j]) = y[j];
        } else {
#pragma unroll
          for (int j = 0; j < kStores; ++j) {
            const int row = j * kAt + lane / kPer;
            T* row_at = reinterpret_cast<T*>(out) + row * rows.token + kVec * (lane % kPer);
            if (places[k][row] != -2) put(row_at, rows.wide, y[j]);
          }
        }
      }
      if (keys) {
        for (int i = tid; i < kRows * key_pieces; i += S::kThreads) {
          const int row = i / key_pieces, piece = i - row * key_pieces;
          put_key(tile, key_head, row, piece, from, places[k][row]);
        }
      } else if (works && !values && c0 == 0) {
        for (int i = lane; i < kRows * key_pieces; i += 64) {
          const int row = i / key_pieces, piece = i - row * key_pieces;
          put_key(tile, head, row, piece, from, places[k][row]);
        }
      }
      if (S::kBuffers == 1) {
        lds_barrier();  // the only buffer is read
        if (more) fetch(places[k + 1], 0);
      }
    }
  }
}

template <typename T, int kWide>
static hipError_t expand_as(const LatentExpandParams& p, hipStream_t stream) {
  typedef ExpandShape<T, kWide> S;
  static_assert(S::kLds + S::kTiles * S::kRows * 8 <= 160 * 1024, "LDS of a CU");
  const int64_t tiles = (p.batch.n_tokens + S::kRows - 1) / S::kRows;
  const int x = (p.heads * ((p.plain + p.value) / 32) + S::kWaves - 1) / S::kWaves;
  const int64_t y = std::min<int64_t>(tiles, std::min<int64_t>(65535, std::max(1, 1024 / x)));
  hipLaunchKernelGGL((latent_expand_kernel<T, kWide>), dim3(x, static_cast<unsigned>(y)), dim3(S::kThreads), S::kLds, stream, p,
                     tiles);
  return hipGetLastError();
}

hipError_t launch_latent_expand(bool bf16, const LatentExpandParams& p, hipStream_t stream) {
  if (p.cache.latent <= 64) return bf16 ? expand_as<uint16_t, 64>(p, stream) : expand_as<float, 64>(p, stream);
  if (p.cache.latent <= 128) return bf16 ? expand_as<uint16_t, 128>(p, stream) : expand_as<float, 128>(p, stream);
  if (p.cache.latent <= 256) return bf16 ? expand_as<uint16_t, 256>(p, stream) : expand_as<float, 256>(p, stream);
  return bf16 ? expand_as<uint16_t, 512>(p, stream) : expand_as<float, 512>(p, stream);
}

}  // namespace scd
