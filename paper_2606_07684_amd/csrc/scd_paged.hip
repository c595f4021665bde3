// The paged 8-bit cache: rows appended (keys rotated on the way) and read back (gfx950).
#include "scd_serve_device.h"

namespace scd {
using namespace dev;

// Scales below this are 0, so that 1 / scale is finite.
constexpr float kSmallestScale = 1.17549435e-38f;

// Eight channels from 8 * chunk of a row, turned to position `pos`.
template <typename T>
__device__ inline void turned8(const Turn& turn, const T* row, bool wide, int chunk, int64_t pos,
                               float* x) {
  load8(row + 8 * chunk, wide, x);
  if (turn.table == nullptr || 8 * chunk >= turn.dim) return;
  pos = pos < 0 ? 0 : (pos >= turn.max_pos ? turn.max_pos - 1 : pos);
  const int half = turn.dim / 2;
  const float2* cs = turn.table + pos * half;
  float unused;
  if (turn.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (8 * chunk + 2 * i < turn.dim)
        turn_pair(x[2 * i], x[2 * i + 1], cs[4 * chunk + i], x[2 * i], x[2 * i + 1]);
    return;
  }
  if (half % 8 == 0) {  // the other halves of the eight pairs are adjacent too
    float y[8];
    const bool first = 8 * chunk < half;
    const int at = first ? 8 * chunk : 8 * chunk - half;
    load8(row + (first ? 8 * chunk + half : at), wide, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (first) turn_pair(x[i], y[i], cs[at + i], x[i], unused);
      else turn_pair(y[i], x[i], cs[at + i], unused, x[i]);
    }
    return;
  }
  for (int i = 0; i < 8; ++i) {
    const int c = 8 * chunk + i;
    if (c < half) turn_pair(x[i], load1(row + c + half), cs[c], x[i], unused);
    else if (c < turn.dim) turn_pair(load1(row + c - half), x[i], cs[c - half], unused, x[i]);
  }
}

__device__ inline int quantised(float x) {
  return static_cast<int>(fminf(fmaxf(rintf(x), -127.f), 127.f));
}
__device__ inline uint32_t pack4(const float* f) {
  return (quantised(f[0]) & 255) | (quantised(f[1]) & 255) << 8 | (quantised(f[2]) & 255) << 16 |
         static_cast<uint32_t>(quantised(f[3]) & 255) << 24;
}
__device__ inline void unpack4(uint32_t w, float* f) {
  f[0] = static_cast<float>(static_cast<int8_t>(w));
  f[1] = static_cast<float>(static_cast<int8_t>(w >> 8));
  f[2] = static_cast<float>(static_cast<int8_t>(w >> 16));
  f[3] = static_cast<float>(static_cast<int32_t>(w) >> 24);
}

// One workgroup per page that new rows touch, KV head and branch.  The page's new rows (at most
// kSteps x 8 channels a thread) stay in registers between the maximum and the quantisation, so every
// row is read once.
template <typename T, int kDim, int kSteps>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheAppendParams p, int64_t units) {
  constexpr int kChunks = kDim / 8, kRows = 256 / kChunks;
  __shared__ LocateLds lds;
  __shared__ float wave_top[4];
  const int tid = threadIdx.x, chunk = tid % kChunks;
  const int lg = p.cache.page_log2;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int kv = static_cast<int>(unit & 1);
    const int h = static_cast<int>((unit >> 1) % p.cache.heads);
    Located at;
    const bool found = locate<256>(p.batch.n_seqs, (unit >> 1) / p.cache.heads, lds, tid, [&](int b) -> int64_t {
      const Span s = span_of(p.batch, b);
      const int64_t end = s.pos0 + s.end - s.begin;
      return s.end > s.begin && end > 0 ? ((end - 1) >> lg) - ((s.pos0 < 0 ? 0 : s.pos0) >> lg) + 1 : 0;
    }, at);
    if (!found) return;
    const Span s = span_of(p.batch, at.b);
    const int64_t from = s.pos0 < 0 ? 0 : s.pos0;
    const int64_t base = ((from >> lg) + at.local) << lg;  // position of the page's first slot
    const int64_t end = s.pos0 + s.end - s.begin;
    const int lo = static_cast<int>(from > base ? from - base : 0);
    const int hi = static_cast<int>(end - base < p.cache.page ? end - base : p.cache.page);
    const int page = page_of(p.cache, at.b, base);
    if (page < 0) continue;
    const Rows& rows = p.rows[kv];
    const T* src = reinterpret_cast<const T*>(rows.data) + h * rows.head;
    int8_t* dst = (kv ? p.cache.v : p.cache.k) + page_at(p.cache, page, h, kDim);
    float* scale_at = (kv ? p.cache.v_scale : p.cache.k_scale) + static_cast<int64_t>(page) * p.cache.heads + h;
    Turn turn = p.turn;
    if (kv) turn.table = nullptr;
    float x[kSteps][8];
    float top = 0.f;
    bool finite = true;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int slot = i * kRows + tid / kChunks;
      if (slot >= lo && slot < hi) {
        const int64_t pos = base + slot;
        turned8(turn, src + (s.begin + pos - s.pos0) * rows.token, rows.wide, chunk, pos, x[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          top = fmaxf(top, fabsf(x[i][j]));
          finite = finite && fabsf(x[i][j]) <= 3.40282347e38f;
        }
      }
    }
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    finite = __all(finite);
    if ((tid & 63) == 0) wave_top[tid >> 6] = finite ? top : __builtin_nanf("");
    const float old = lo > 0 ? *scale_at : 0.f;
    __syncthreads();
    float scale = old;
    for (int w = 0; w < 4; ++w) {
      const float a = wave_top[w] * (1.f / 127.f);
      scale = a > scale || a != a ? a : scale;
    }
    if (scale < kSmallestScale) scale = 0.f;
    const float inv = scale > 0.f ? 1.f / scale : 0.f;
    if (tid == 0) *scale_at = scale;
    if (scale > old && lo > 0) {  // earlier rows to the new scale
      const float ratio = old * inv;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int slot = i * kRows + tid / kChunks;
        if (slot < lo) {
          uint2* w = reinterpret_cast<uint2*>(dst + slot * kDim + 8 * chunk);
          uint2 v = *w;
          float f[8];
          unpack4(v.x, f);
          unpack4(v.y, f + 4);
          for (int j = 0; j < 8; ++j) f[j] *= ratio;
          *w = make_uint2(pack4(f), pack4(f + 4));
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int slot = i * kRows + tid / kChunks;
      if (slot >= lo && slot < hi) {
        float f[8];
        for (int j = 0; j < 8; ++j) f[j] = x[i][j] * inv;
        *reinterpret_cast<uint2*>(dst + slot * kDim + 8 * chunk) = make_uint2(pack4(f), pack4(f + 4));
      }
    }
    __syncthreads();  // wave_top is written again
  }
}

// One wave per row: both branches of every head, 16 channels a lane at a time.
template <typename T, int kDim>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheReadParams p) {
  constexpr int kChunks = kDim / 16;
  const int lane = threadIdx.x & 63;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); t < p.batch.n_tokens;
       t += static_cast<int64_t>(gridDim.x) * 4) {
    const int b = request_of(p.batch, t, lane);
    const Span s = span_of(p.batch, b);
    const int64_t pos = t - s.begin + s.pos0;
    const int page = page_of(p.cache, b, pos);
    for (int idx = lane; idx < 2 * p.cache.heads * kChunks; idx += 64) {
      const int kv = idx >= p.cache.heads * kChunks;
      const int h = idx / kChunks - (kv ? p.cache.heads : 0), chunk = idx % kChunks;
      float f[16];
      if (page < 0) {
        for (int i = 0; i < 16; ++i) f[i] = 0.f;
      } else {
        const int8_t* src = (kv ? p.cache.v : p.cache.k) + page_at(p.cache, page, h, kDim) +
                            (pos & (p.cache.page - 1)) * kDim + 16 * chunk;
        const float scale = (kv ? p.cache.v_scale : p.cache.k_scale)[static_cast<int64_t>(page) * p.cache.heads + h];
        const uint4 w = *reinterpret_cast<const uint4*>(src);
        unpack4(w.x, f);
        unpack4(w.y, f + 4);
        unpack4(w.z, f + 8);
        unpack4(w.w, f + 12);
        for (int i = 0; i < 16; ++i) f[i] *= scale;
      }
      const Rows& rows = p.rows[kv];
      T* dst = reinterpret_cast<T*>(rows.data) + t * rows.token + h * rows.head + 16 * chunk;
      store8(dst, rows.wide, f);
      store8(dst + 8, rows.wide, f + 8);
    }
  }
}

template <typename T, int kDim>
static hipError_t launch_append_as(const CacheAppendParams& p, hipStream_t stream) {
  // Pages touched: a request's n rows lie in at most (n - 2) / page + 2 of them.
  const int64_t n = p.batch.n_tokens, requests = p.batch.n_seqs < n ? p.batch.n_seqs : n;
  const int64_t pages = n / p.cache.page + 2 * requests;
  const int64_t units = (pages < n ? pages : n) * p.cache.heads * 2;
  const dim3 grid(static_cast<unsigned>(units < kMaxGrid ? units : kMaxGrid)), block(256);
  const int steps = p.cache.page * kDim / 2048;
  switch (steps <= 1 ? 1 : steps) {
    case 1: hipLaunchKernelGGL((cache_append_kernel<T, kDim, 1>), grid, block, 0, stream, p, units); break;
    case 2: hipLaunchKernelGGL((cache_append_kernel<T, kDim, 2>), grid, block, 0, stream, p, units); break;
    case 4: hipLaunchKernelGGL((cache_append_kernel<T, kDim, 4>), grid, block, 0, stream, p, units); break;
    default: hipLaunchKernelGGL((cache_append_kernel<T, kDim, 8>), grid, block, 0, stream, p, units); break;
  }
  return hipGetLastError();
}

hipError_t launch_cache_append(bool bf16, int head_dim, const CacheAppendParams& p,
                               hipStream_t stream) {
  if (bf16)
    return head_dim == 128 ? launch_append_as<uint16_t, 128>(p, stream)
           : head_dim == 64 ? launch_append_as<uint16_t, 64>(p, stream)
                            : launch_append_as<uint16_t, 32>(p, stream);
  return head_dim == 128 ? launch_append_as<float, 128>(p, stream)
         : head_dim == 64 ? launch_append_as<float, 64>(p, stream)
                          : launch_append_as<float, 32>(p, stream);
}

template <typename T, int kDim>
static hipError_t launch_read_as(const CacheReadParams& p, hipStream_t stream) {
  const int64_t blocks = (p.batch.n_tokens + 3) / 4;
  hipLaunchKernelGGL((cache_read_kernel<T, kDim>),
                     dim3(static_cast<unsigned>(blocks < kMaxGrid ? blocks : kMaxGrid)), dim3(256), 0,
                     stream, p);
  return hipGetLastError();
}

hipError_t launch_cache_read(bool bf16, int head_dim, const CacheReadParams& p, hipStream_t stream) {
  if (bf16)
    return head_dim == 128 ? launch_read_as<uint16_t, 128>(p, stream)
           : head_dim == 64 ? launch_read_as<uint16_t, 64>(p, stream)
                            : launch_read_as<uint16_t, 32>(p, stream);
  return head_dim == 128 ? launch_read_as<float, 128>(p, stream)
         : head_dim == 64 ? launch_read_as<float, 64>(p, stream)
                          : launch_read_as<float, 32>(p, stream);
}

}  // namespace scd
