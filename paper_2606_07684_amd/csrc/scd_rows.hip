// Attention over dense rows: how a call is laid out, and the join of tiles that are cut (gfx950).
#include <algorithm>

#include "scd_rows_attend.h"

namespace scd {
using namespace dev;

// out = (sum_s 2^(m_s - m) o_s) / (sum_s 2^(m_s - m) l_s): a wave a query row, two channels a lane.
template <typename T>
__global__ __launch_bounds__(256) void rows_join_kernel(RowsAttendParams p, int64_t rows) {
  const int lane = threadIdx.x & 63, line = p.value + 2;
  int64_t end = p.batch.n_tokens;
  if (p.batch.cu != nullptr) end = std::min<int64_t>(end, p.batch.cu[p.batch.n_seqs]);
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); i < rows;
       i += static_cast<int64_t>(gridDim.x) * 4) {
    const int64_t t = i / p.q.n_heads;
    if (t >= end) return;
    const RowParts r = p.parts[i];
    const int64_t last = r.first + static_cast<int64_t>(r.count - 1) * r.step;
    if (r.count <= 1 || r.first < 0 || r.step < 0 || r.row < 0 || r.row >= p.plan.rows || last >= p.plan.grid) continue;
    const auto slot = [&](int s) {
      return p.slots + ((r.first + static_cast<int64_t>(s) * r.step) * p.plan.rows + r.row) * line;
    };
    float m = -INFINITY, l = 0.f;
    for (int s = lane; s < r.count; s += 64) m = fmaxf(m, slot(s)[0]);
    for (int x = 32; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
    const float base = m == -INFINITY ? 0.f : m;
    float2 o = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int s = 0; s < r.count; ++s) {
      const float* at = slot(s);
      const float2 ml = *reinterpret_cast<const float2*>(at);
      const float w = __builtin_amdgcn_exp2f(ml.x - base);
      l += w * ml.y;
      if (2 * lane < p.value) {
        const float2 x = *reinterpret_cast<const float2*>(at + 2 + 2 * lane);
        o.x += w * x.x;
        o.y += w * x.y;
      }
    }
    const float by = l == 0.f ? 0.f : 1.f / l;
    if (2 * lane < p.value) {
      T* out = reinterpret_cast<T*>(p.out.data) + t * p.out.token + (i - t * p.q.n_heads) * p.out.head + 2 * lane;
      store1(out, o.x * by);
      store1(out + 1, o.y * by);
    }
  }
}

RowsSizes rows_sizes(bool bf16, bool wide, const SeqBatch& b, int64_t held_rows, int heads, int kv_heads, int value) {
  RowsSizes z{};
  SharePlan& plan = z.plan;
  const int group = heads / kv_heads;
  const int64_t requests = std::min<int64_t>(b.n_seqs, b.n_tokens), rows = b.n_tokens * group;
  const int64_t mean = (rows + requests - 1) / requests;
  plan.rows = mean <= 16 ? 16 : mean <= 32 ? 32 : mean <= 64 || !bf16 || !wide ? 64 : 128;
  plan.row_groups = plan.rows >= 64 ? 4 : plan.rows / 16;
  plan.heads = kv_heads;
  plan.per_token = group;
  plan.cap = held_rows;
  const int64_t least = ((rows + plan.rows - 1) / plan.rows) * kv_heads;
  const int64_t tiles = (rows / plan.rows + requests) * kv_heads;
  plan.cut = least < 2 * kFill;
  plan.grid = tiles;
  if (!plan.cut) return z;
  const int block = plan.rows == 128 || !bf16 ? 32 : 64;
  const int64_t goal = std::max(tiles, share_goal(std::min<int64_t>(tiles, 2 * kFill - 1)));
  const int64_t most = std::max<int64_t>(1, ((held_rows + block - 1) / block + 1) / 2);  // shares of two blocks each
  plan.grid = tiles > goal / most ? goal : tiles * most;
  if (most == 1) {
    plan.cut = 0;
    return z;
  }
  const auto up = [](size_t n) { return (n + 255) & ~size_t{255}; };
  z.parts = up(static_cast<size_t>(b.n_tokens) * heads * sizeof(RowParts));
  z.slots = up(static_cast<size_t>(plan.grid) * plan.rows * (value + 2) * sizeof(float));
  return z;
}

hipError_t launch_rows_attend(bool bf16, const RowsAttendParams& p, hipStream_t stream) {
  const hipError_t e = !rows_wide(p.k, p.v) ? launch_odd_rows(bf16, p, stream)
                       : bf16             ? launch_rows_bf16(p, stream)
                                          : launch_rows_f32(p, stream);
  if (e != hipSuccess || !p.plan.cut) return e;
  const int64_t rows = p.batch.n_tokens * p.q.n_heads;
  const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((rows + 3) / 4, kMaxGrid));
  if (bf16) {
    hipLaunchKernelGGL((rows_join_kernel<uint16_t>), dim3(blocks), dim3(256), 0, stream, p, rows);
  } else {
    hipLaunchKernelGGL((rows_join_kernel<float>), dim3(blocks), dim3(256), 0, stream, p, rows);
  }
  return hipGetLastError();
}

}  // namespace scd
