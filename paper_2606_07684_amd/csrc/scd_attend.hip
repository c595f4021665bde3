// Causal attention of new tokens over the paged 8-bit cache (gfx950).
//
// out = sum_j p_j v_j with p the softmax over the cached positions of scale * (q . k_j), in one pass
// with a running maximum and sum: when the maximum grows from m to m', what is summed so far is
// multiplied by e^(m - m').
#include "scd_serve_device.h"

namespace scd {
using namespace dev;

// One wave per query row: 64 positions at a time, one a lane for the scores, then one after another
// for the sum over values.
template <typename T, int kDim>
__global__ __launch_bounds__(64) void cache_attend_kernel(CacheAttendParams p, int64_t units) {
  __shared__ float q[kDim], weight[64];
  __shared__ int64_t row_at[64];
  const int lane = threadIdx.x;
  constexpr int kOwn = (kDim + 63) / 64;
  const bool owner = lane < kDim;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int64_t t = unit / p.q.n_heads;
    const int head = static_cast<int>(unit - t * p.q.n_heads), h = head / p.group;
    const int b = request_of(p.batch, t, lane);
    const Span s = span_of(p.batch, b);
    const int64_t n = t - s.begin + s.pos0 + 1;  // positions it attends to
    const T* src = reinterpret_cast<const T*>(p.q.data) + t * p.q.token + head * p.q.head;
    for (int c = lane; c < kDim; c += 64) q[c] = load1(src + c) * p.scale;
    __syncthreads();
    float m = -INFINITY, l = 0.f, acc[kOwn] = {};
    for (int64_t j0 = 0; j0 < n; j0 += 64) {
      const int64_t j = j0 + lane;
      const int page = j < n ? page_of(p.cache, b, j) : -1;
      float score = -INFINITY;
      if (page >= 0) {
        row_at[lane] = page_at(p.cache, page, h, kDim) + (j & (p.cache.page - 1)) * kDim;
        const uint4* k = reinterpret_cast<const uint4*>(p.cache.k + row_at[lane]);
        float sum = 0.f;
        for (int c = 0; c < kDim / 16; ++c) {
          const uint4 w = k[c];
          const uint32_t word[4] = {w.x, w.y, w.z, w.w};
          for (int i = 0; i < 16; ++i)
            sum += q[16 * c + i] * static_cast<float>(static_cast<int8_t>(word[i >> 2] >> (8 * (i & 3))));
        }
        score = sum * p.cache.k_scale[static_cast<int64_t>(page) * p.cache.heads + h];
        if (score != score) score = INFINITY;  // NaN: the row becomes NaN
      }
      float top = score;
      for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
      top = fmaxf(top, m);
      if (top == -INFINITY) continue;
      const float w = page >= 0 ? expf(score - top) : 0.f;
      const float fade = expf(m - top);
      m = top;
      float sum = w;
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
      l = l * fade + sum;
      __syncthreads();
      weight[lane] = page >= 0 ? w * p.cache.v_scale[static_cast<int64_t>(page) * p.cache.heads + h] : 0.f;
      if (page < 0) row_at[lane] = -1;
      __syncthreads();
      if (owner) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          float a = acc[i] * fade;
          for (int jj = 0; jj < 64; ++jj)
            if (row_at[jj] >= 0) a += weight[jj] * static_cast<float>(p.cache.v[row_at[jj] + lane + 64 * i]);
          acc[i] = a;
        }
      }
      __syncthreads();
    }
    T* dst = reinterpret_cast<T*>(p.out.data) + t * p.out.token + head * p.out.head;
    if (owner)
      for (int i = 0; i < kOwn; ++i) store1(dst + lane + 64 * i, l != 0.f ? acc[i] / l : 0.f);
    __syncthreads();
  }
}

size_t attend_workspace(const PagedCache&, const SeqBatch&, int, int) { return 0; }

template <typename T>
static hipError_t launch_attend_as(int head_dim, const CacheAttendParams& p, hipStream_t stream) {
  const int64_t units = p.batch.n_tokens * p.q.n_heads;
  const dim3 grid(static_cast<unsigned>(units < kMaxGrid ? units : kMaxGrid)), block(64);
  if (head_dim == 128) hipLaunchKernelGGL((cache_attend_kernel<T, 128>), grid, block, 0, stream, p, units);
  else if (head_dim == 64) hipLaunchKernelGGL((cache_attend_kernel<T, 64>), grid, block, 0, stream, p, units);
  else hipLaunchKernelGGL((cache_attend_kernel<T, 32>), grid, block, 0, stream, p, units);
  return hipGetLastError();
}

hipError_t launch_cache_attend(bool bf16, int head_dim, const CacheAttendParams& p, void*,
                               hipStream_t stream) {
  return bf16 ? launch_attend_as<uint16_t>(head_dim, p, stream) : launch_attend_as<float>(head_dim, p, stream);
}

}  // namespace scd
