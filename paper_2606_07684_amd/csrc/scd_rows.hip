// Attention over dense rows: how a call is laid out, and the join of tiles that are cut (gfx950).
#include <algorithm>

#include "scd_rows_attend.h"

namespace scd {
using namespace dev;

// out = (sum_s 2^(m_s - m) o_s) / (sum_s 2^(m_s - m) l_s): kWaves waves a query row, which deal its shares among them
// and meet in LDS, two channels a lane, eight shares' values on the way at once.
template <typename T, int kWaves>
__global__ __launch_bounds__(256) void rows_join_kernel(RowsAttendParams p, int64_t rows) {
  __shared__ float halves[4][128 + 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, line = p.value + 2;
  const int32_t stop = p.batch.cu != nullptr ? p.batch.cu[p.batch.n_seqs] : 0x7fffffff;
  constexpr int kRows = 4 / kWaves;
  for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * kRows; i0 < rows; i0 += static_cast<int64_t>(gridDim.x) * kRows) {
    const int64_t i = i0 + (kWaves == 1 ? wave : 0);
    if (i >= rows) return;
    const int64_t t = i / p.q.n_heads;
    if (t >= stop) return;  // behind the last request, and so is what follows
    const RowParts r = p.parts[i];
    const int64_t last = r.first + static_cast<int64_t>(r.count - 1) * r.step;
    if (r.count <= 1 || r.first < 0 || r.step < 0 || r.row < 0 || r.row >= p.plan.rows || last >= p.plan.grid ||
        r.count > p.plan.grid)
      continue;
    const int count = uniform(r.count);
    const float* row = p.slots + (static_cast<int64_t>(uniform(r.first)) * p.plan.rows + uniform(r.row)) * line + 2 * lane;
    const int64_t step = static_cast<int64_t>(uniform(r.step)) * p.plan.rows * line;
    const bool mine = 2 * lane < p.value;
    float m = -INFINITY, l = 0.f;
    float2 o = make_float2(0.f, 0.f);
    for (int s0 = kWaves == 1 ? 0 : wave; s0 < count; s0 += 8 * kWaves) {
      float2 ml[8], x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int s = s0 + u * kWaves;
        ml[u] = make_float2(-INFINITY, 0.f);
        x[u] = make_float2(0.f, 0.f);
        if (s < count) ml[u] = *reinterpret_cast<const float2*>(row + s * step - 2 * lane);
        if (s < count && mine) x[u] = *reinterpret_cast<const float2*>(row + s * step + 2);
      }
      float now = m;
#pragma unroll
      for (int u = 0; u < 8; ++u) now = fmaxf(now, ml[u].x);
      const float base = now == -INFINITY ? 0.f : now, old = __builtin_amdgcn_exp2f(m - base);
      m = now;
      l *= old;
      o.x *= old;
      o.y *= old;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float w = __builtin_amdgcn_exp2f(ml[u].x - base);
        l += w * ml[u].y;
        o.x += w * x[u].x;
        o.y += w * x[u].y;
      }
    }
    if constexpr (kWaves == 4) {
      __syncthreads();  // the last row's readers are done
      if (lane == 0) *reinterpret_cast<float2*>(&halves[wave][0]) = make_float2(m, l);
      if (mine) *reinterpret_cast<float2*>(&halves[wave][2 + 2 * lane]) = o;
      __syncthreads();
      if (wave != 0) continue;
      const float now = fmaxf(fmaxf(halves[0][0], halves[1][0]), fmaxf(halves[2][0], halves[3][0]));
      const float base = now == -INFINITY ? 0.f : now;
      l = 0.f;
      o = make_float2(0.f, 0.f);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float by = __builtin_amdgcn_exp2f(halves[w][0] - base);
        l += by * halves[w][1];
        if (mine) {
          o.x += by * halves[w][2 + 2 * lane];
          o.y += by * halves[w][3 + 2 * lane];
        }
      }
    }
    const float by = l == 0.f ? 0.f : 1.f / l;
    if (mine) {
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
  // Joins cost a prompt more than idle CUs do: it is cut for one workgroup a CU, and not from 256 tiles on.  Where requests
  // hold many more positions than query rows, bf16 calls are cut for the two workgroups that a CU takes (fp32 ones fill
  // it), to 448 tiles.  In us, this rule's side first.  Prompts of 32 heads of 192 and 128: 512 tokens 34 | 37 cut for two,
  // 1000 tokens (256 tiles) 44 whole | 55 cut, 1500 behind 3000 174 | 193; fp32 of 500 tokens 63 whole | 86, 256 behind
  // 2000 137 | 150 for two.  Long: 512 rows behind 8000 114 for two | 144, 1000 behind 8000 205 cut | 264; a token of 10
  // requests of 4000 175 cut | 191; 256 behind 1000, not long, 35 | 39 for two.
  const bool lengthy = bf16 && held_rows > 3 * b.n_tokens && held_rows >= 2048 * requests;
  plan.fill = lengthy ? 512 : 256;
  plan.whole = lengthy ? 448 : 256;
  plan.cut = least < plan.whole;
  plan.grid = tiles;
  if (!plan.cut) return z;
  const int block = plan.rows == 128 || !bf16 ? 32 : 64;
  const int64_t goal = std::max(tiles, share_goal(std::min<int64_t>(tiles, plan.whole - 1), plan.fill));
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
  // four waves a row while there are few rows, which then have many shares (one request of 8000 positions 41 -> 17 us);
  // with 4096 rows (a prompt of 128 tokens) a wave a row is faster, 17 us to 25
  const int64_t rows = p.batch.n_tokens * p.q.n_heads;
  const bool few = rows <= 1024;
  const unsigned blocks = static_cast<unsigned>(std::min<int64_t>(few ? rows : (rows + 3) / 4, kMaxGrid));
  if (bf16) {
    if (few) {
      hipLaunchKernelGGL((rows_join_kernel<uint16_t, 4>), dim3(blocks), dim3(256), 0, stream, p, rows);
    } else {
      hipLaunchKernelGGL((rows_join_kernel<uint16_t, 1>), dim3(blocks), dim3(256), 0, stream, p, rows);
    }
  } else if (few) {
    hipLaunchKernelGGL((rows_join_kernel<float, 4>), dim3(blocks), dim3(256), 0, stream, p, rows);
  } else {
    hipLaunchKernelGGL((rows_join_kernel<float, 1>), dim3(blocks), dim3(256), 0, stream, p, rows);
  }
  return hipGetLastError();
}

}  // namespace scd
