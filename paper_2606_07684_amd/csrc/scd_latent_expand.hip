// The dense keys and values of cached latents (gfx950), for prompts: k_h = [W_k,h c | key], v_h = W_v,h c.
//
// A wave keeps 32 rows of the heads' matrices in registers for the whole call and takes tiles of cached rows
// from LDS, so the matrices are read once a workgroup and the latents once for every 128 channels; what is
// written, heads x (plain + turned + value) channels a row, is 20 times what is read and bounds the call.
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

template <typename T, int kWide>
__global__ __launch_bounds__(256) void latent_expand_kernel(LatentExpandParams p, int64_t tiles) {
  constexpr int kVec = Elem<T>::kVec, kRows = sizeof(T) == 2 ? 64 : 32, kSub = kRows / 32;
  constexpr int kPieces = (kWide + 64) / kVec + 1, kRow = kPieces * kVec;
  constexpr int kFrags = kWide / (2 * kVec), kFixed = (kWide == 128 ? 32 : kWide / 2) / (2 * kVec);
  typedef typename Elem<T>::Frag Frag;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int64_t places[3][kRows];  // byte of a row in the pages, -1: a hole, -2: no such row
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int latent = p.cache.latent, width = latent + p.cache.turned, frags = latent / (2 * kVec);

  // the wave's 32 channels: of a head's keys, or of its values
  const int per_head = (p.plain + p.value) / 32;
  const int group = blockIdx.x * 4 + wave;
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
    for (int f = 0; f < kFrags; ++f)
      if (f < kFixed || f < frags) w[f] = *reinterpret_cast<const Frag*>(at + 2 * kVec * f);
  }
  const Rows& rows = values ? p.v : p.k;

  const auto resolve = [&](int64_t tile, int64_t* to) {
    if (tid >= kRows) return;
    const int64_t t = tile * kRows + tid;
    int64_t place = -2;
    if (t < p.batch.n_tokens) {
      int b = 0;
      int64_t begin = 0;
      bool mine = true;
      if (p.batch.cu != nullptr) {
        int hi = p.batch.n_seqs - 1;  // the last request that begins at or before t
        while (b < hi) {
          const int mid = (b + hi + 1) >> 1;
          if (p.batch.cu[mid] <= t) b = mid; else hi = mid - 1;
        }
        begin = p.batch.cu[b];
        mine = t < p.batch.cu[p.batch.n_seqs];
      }
      if (mine) {
        const int64_t pos = t - begin + (p.batch.pos0 != nullptr ? p.batch.pos0[b] : 0);
        const int64_t column = pos >> p.cache.page_log2;
        place = -1;
        if (pos >= 0 && column < p.cache.cols) {
          const int id = p.cache.table[static_cast<int64_t>(b) * p.cache.cols + column];
          if (id >= 0 && id < p.cache.n_pages)
            place = ((static_cast<int64_t>(id) << p.cache.page_log2) + (pos & (p.cache.page - 1))) *
                    (width * static_cast<int64_t>(sizeof(T)));
        }
      }
    }
    to[tid] = place;
  };
  const int pieces = width / kVec;
  const auto fetch = [&](const int64_t* from, int buffer) {
    constexpr int kCopies = (kRows * kPieces + 63) / 64;
    for (int j = wave; j < kCopies; j += 4) {
      const int slot = j * 64 + lane, row = slot / kPieces, piece = slot - row * kPieces;
      if (row < kRows && piece < pieces) {
        const int64_t place = from[row];
        copy16(p.cache.pages + (place < 0 ? 0 : place) + 16 * piece, smem + buffer * (kRows * kPieces * 16) + j * 1024);
      }
    }
  };

  int64_t tile = blockIdx.y;
  resolve(tile, places[0]);
  __syncthreads();
  fetch(places[0], 0);
  for (int it = 0; tile < tiles; ++it, tile += gridDim.y) {
    const int now = it % 3, next = (it + 1) % 3;
    resolve(tile + gridDim.y, places[next]);
    wait_copies<0>();
    lds_barrier();
    if (tile + gridDim.y < tiles) fetch(places[next], (it + 1) & 1);
    if (!works) continue;
    const T* at = reinterpret_cast<const T*>(smem + (it & 1) * (kRows * kPieces * 16));
    f32x16 acc[kSub];
#pragma unroll
    for (int s = 0; s < kSub; ++s)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[s][i] = 0.f;
#pragma unroll
    for (int f = 0; f < kFrags; ++f)
      if (f < kFixed || f < frags) {
#pragma unroll
        for (int s = 0; s < kSub; ++s)
          acc[s] = mma32(w[f], *reinterpret_cast<const Frag*>(at + (32 * s + col) * kRow + 2 * kVec * f + kVec * half), acc[s]);
      }
#pragma unroll
    for (int s = 0; s < kSub; ++s) {
      const int64_t place = places[now][32 * s + col];
      if (place == -2) continue;
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = place < 0 ? 0.f : acc[s][i];
      T* out = reinterpret_cast<T*>(rows.data) + (tile * kRows + 32 * s + col) * rows.token + head * rows.head + c0 + 16 * half;
      store8(out, rows.wide, x);
      store8(out + 8, rows.wide, x + 8);
    }
    if (!values && c0 == 0) {
      // the shared key behind this head's own channels
      const int per_row = p.cache.turned / kVec;
      for (int i = lane; i < kRows * per_row; i += 64) {
        const int row = i / per_row, piece = i - row * per_row;
        const int64_t place = places[now][row];
        if (place == -2) continue;
        uint4 x = *reinterpret_cast<const uint4*>(at + row * kRow + latent + kVec * piece);
        if (place < 0) x = make_uint4(0, 0, 0, 0);
        T* out = reinterpret_cast<T*>(rows.data) + (tile * kRows + row) * rows.token + head * rows.head + p.plain + kVec * piece;
        if (rows.wide) {
          *reinterpret_cast<uint4*>(out) = x;
        } else {
          const uint32_t bits[4] = {x.x, x.y, x.z, x.w};
          for (int e = 0; e < kVec; ++e) {
            if constexpr (sizeof(T) == 2) {
              out[e] = static_cast<uint16_t>(bits[e >> 1] >> (16 * (e & 1)));
            } else {
              out[e] = __uint_as_float(bits[e]);
            }
          }
        }
      }
    }
  }
}

template <typename T, int kWide>
static hipError_t expand_as(const LatentExpandParams& p, hipStream_t stream) {
  constexpr int kRows = sizeof(T) == 2 ? 64 : 32, kPieces = (kWide + 64) / Elem<T>::kVec + 1;
  const int64_t tiles = (p.batch.n_tokens + kRows - 1) / kRows;
  const int x = (p.heads * ((p.plain + p.value) / 32) + 3) / 4;
  const int64_t y = std::min<int64_t>(tiles, std::min<int64_t>(65535, std::max(1, 1024 / x)));
  hipLaunchKernelGGL((latent_expand_kernel<T, kWide>), dim3(x, static_cast<unsigned>(y)), dim3(256),
                     2 * kRows * kPieces * 16, stream, p, tiles);
  return hipGetLastError();
}

hipError_t launch_latent_expand(bool bf16, const LatentExpandParams& p, hipStream_t stream) {
  if (p.cache.latent <= 128) return bf16 ? expand_as<uint16_t, 128>(p, stream) : expand_as<float, 128>(p, stream);
  if (p.cache.latent <= 256) return bf16 ? expand_as<uint16_t, 256>(p, stream) : expand_as<float, 256>(p, stream);
  return bf16 ? expand_as<uint16_t, 512>(p, stream) : expand_as<float, 512>(p, stream);
}

}  // namespace scd
