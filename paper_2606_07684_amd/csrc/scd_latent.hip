// The latent cache (gfx950): rows into pages, queries into the latents' space, the shares of attention
// joined and taken out of it again.
#include <algorithm>

#include "scd_attend_core.h"

namespace scd {
using namespace dev;

// ---- append ------------------------------------------------------------------------------------------
// A wave a token: the latent's bits as they are, the shared key a channel a lane, turned in fp32 and rounded
// once.  Bound by HBM for prompts and by three memory accesses one after the other (owner, page, row) for a
// few tokens.
template <typename T>
__global__ __launch_bounds__(256) void latent_append_kernel(LatentAppendParams p) {
  constexpr int kVec = 16 / sizeof(T);
  const int lane = threadIdx.x & 63;
  const int latent = p.cache.latent, turned = p.cache.turned, width = latent + turned;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); t < p.batch.n_tokens;
       t += static_cast<int64_t>(gridDim.x) * 4) {
    // the row is fetched while its place is looked up
    const T* c = reinterpret_cast<const T*>(p.c.data) + t * p.c.token;
    const T* k = reinterpret_cast<const T*>(p.k.data) + t * p.k.token;
    u32x4 piece[2];
    if (p.c.wide) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if ((lane + 64 * j) * kVec < latent) piece[j] = reinterpret_cast<const u32x4*>(c)[lane + 64 * j];
    }
    int partner = lane;
    bool second = false;
    if (p.turn.table != nullptr && lane < p.turn.dim) {
      const int half = p.turn.dim / 2;
      second = p.turn.interleaved ? lane & 1 : lane >= half;
      partner = p.turn.interleaved ? lane ^ 1 : (second ? lane - half : lane + half);
    }
    const T own = lane < turned ? k[lane] : T{}, other = lane < turned ? k[partner] : T{};

    const Owner owner = owner_of(p.batch, t, lane);
    const int64_t pos = t - owner.begin + owner.pos0;
    const int64_t col = pos >> p.cache.page_log2;
    if (pos < 0 || col >= p.cache.cols) continue;
    if (p.batch.cu != nullptr && t >= p.batch.cu[p.batch.n_seqs]) continue;  // behind the last request
    const int id = p.cache.table[static_cast<int64_t>(owner.b) * p.cache.cols + col];
    if (id < 0 || id >= p.cache.n_pages) continue;
    T* row = reinterpret_cast<T*>(p.cache.pages) +
             ((static_cast<int64_t>(id) << p.cache.page_log2) + (pos & (p.cache.page - 1))) * width;
    if (p.c.wide) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if ((lane + 64 * j) * kVec < latent) reinterpret_cast<u32x4*>(row)[lane + 64 * j] = piece[j];
    } else {
      for (int i = lane; i < latent; i += 64) row[i] = c[i];
    }
    if (lane < turned) {
      T out = own;
      if (partner != lane) {
        const int64_t at = pos < p.turn.max_pos ? pos : p.turn.max_pos - 1;
        const int pair = p.turn.interleaved ? lane >> 1 : (second ? partner : lane);
        const float2 cs = p.turn.table[at * (p.turn.dim / 2) + pair];
        float x, y;
        const float a = load1(second ? &other : &own), b = load1(second ? &own : &other);
        turn_pair(a, b, cs, x, y);
        store1(&out, second ? y : x);
      }
      row[latent + lane] = out;
    }
  }
}

template <typename T>
static hipError_t launch_append_as(const LatentAppendParams& p, hipStream_t stream) {
  const int64_t blocks = (p.batch.n_tokens + 3) / 4;
  hipLaunchKernelGGL((latent_append_kernel<T>), dim3(static_cast<unsigned>(std::min(blocks, kMaxGrid))), dim3(256), 0,
                     stream, p);
  return hipGetLastError();
}
hipError_t launch_latent_append(bool bf16, const LatentAppendParams& p, hipStream_t stream) {
  return bf16 ? launch_append_as<uint16_t>(p, stream) : launch_append_as<float>(p, stream);
}

// ---- queries into the latents' space -------------------------------------------------------------------
__device__ inline void put_query(uint16_t* row, int width, int i, float x) {
  // two bf16 summands hold 16 bits of a query: a score's error then stays below what the rounding of the
  // result to bf16 adds, as in a product of unrounded queries
  const __bf16 high = static_cast<__bf16>(x);
  row[i] = __builtin_bit_cast(uint16_t, high);
  row[width + i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x - static_cast<float>(high)));
}
__device__ inline void put_query(float* row, int, int i, float x) { row[i] = x; }

__device__ inline f32x4 load4(const uint16_t* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  return f32x4{bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)};
}
__device__ inline f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }

// absorbed_h = scale [ q_h[:plain] W_k,h | q_h[plain:] ]: workgroup (h, a few tokens), four latent channels a
// thread, the matrix's rows dealt to groups of threads whose sums meet in LDS.  The matrix is read once for
// kTokens tokens; with few tokens that read is the call.
template <typename T, int kTokens>
__global__ __launch_bounds__(256) void latent_query_kernel(LatentAttendParams p) {
  __shared__ float q[kTokens][256 + 64];
  __shared__ __attribute__((aligned(16))) float sums[kTokens * 1024];
  const int tid = threadIdx.x, h = blockIdx.x;
  const int64_t t0 = static_cast<int64_t>(blockIdx.y) * kTokens;
  const int n = static_cast<int>(p.batch.n_tokens - t0 < kTokens ? p.batch.n_tokens - t0 : kTokens);
  const int latent = p.cache.latent, turned = p.cache.turned, width = latent + turned;
  const int wide = p.plain + turned;
  for (int i = tid; i < kTokens * wide; i += 256) {
    const int t = i / wide, c = i - t * wide;
    float x = 0.f;
    if (t < n) x = load1(reinterpret_cast<const T*>(p.q.data) + (t0 + t) * p.q.token + h * p.q.head + c);
    q[t][c] = x * p.scale;
  }
  __syncthreads();
  const int quads = latent / 4, groups = 256 / quads;
  const int group = tid / quads, quad = tid - group * quads;
  f32x4 acc[kTokens];
#pragma unroll
  for (int t = 0; t < kTokens; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (group < groups) {
    const T* w = reinterpret_cast<const T*>(p.w_k) + static_cast<int64_t>(h) * p.plain * latent + 4 * quad;
#pragma unroll 8
    for (int d = group; d < p.plain; d += groups) {
      const f32x4 x = load4(w + static_cast<int64_t>(d) * latent);
#pragma unroll
      for (int t = 0; t < kTokens; ++t) {
        const float y = q[t][d];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] += x[i] * y;
      }
    }
#pragma unroll
    for (int t = 0; t < kTokens; ++t)
      *reinterpret_cast<f32x4*>(&sums[(group * kTokens + t) * latent + 4 * quad]) = acc[t];
  }
  __syncthreads();
  constexpr int kParts = sizeof(T) == 2 ? 2 : 1;
  for (int i = tid; i < n * width; i += 256) {
    const int t = i / width, c = i - t * width;
    float x = 0.f;
    if (c < latent) {
      for (int g = 0; g < groups; ++g) x += sums[(g * kTokens + t) * latent + c];
    } else {
      x = q[t][p.plain + c - latent];
    }
    put_query(reinterpret_cast<T*>(p.absorbed) + ((t0 + t) * p.heads + h) * (kParts * width), width, c, x);
  }
}

// ---- shares joined, results out of the latents' space ----------------------------------------------------
// out_h = W_v,h (sum_s 2^(m_s - m) o_s) / (sum_s 2^(m_s - m) l_s) over a row's shares s: workgroup (h, tokens
// of it).  One token's shares are dealt to the four waves, several tokens are dealt as they are.  The joined
// rows, as two bf16 summands, are the right operands of the product with W_v,h, whose rows come from memory
// as they lie.
template <typename T>
__global__ __launch_bounds__(256) void latent_out_kernel(LatentAttendParams p, int tokens) {
  constexpr int kParts = sizeof(T) == 2 ? 2 : 1, kMost = 512;
  constexpr int kVec = Elem<T>::kVec, kRow = kMost + kVec;  // 16-byte pieces of a row: odd
  __shared__ __attribute__((aligned(16))) T rows[kParts][16][kRow];
  __shared__ float halves[4][kMost + 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, g = lane >> 4;
  const int h = blockIdx.x, latent = p.cache.latent, line = latent + 2;
  const int64_t t0 = static_cast<int64_t>(blockIdx.y) * tokens;
  int64_t end = p.batch.n_tokens;
  if (p.batch.cu != nullptr) end = std::min<int64_t>(end, p.batch.cu[p.batch.n_seqs]);
  if (t0 >= end) return;

  const auto put = [&](int t, int c, float x) {
    if constexpr (sizeof(T) == 2) {
      const __bf16 high = static_cast<__bf16>(x);
      rows[0][t][c] = __builtin_bit_cast(uint16_t, high);
      rows[1][t][c] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x - static_cast<float>(high)));
    } else {
      rows[0][t][c] = x;
    }
  };
  // shares from, from + by, ... of a token's row: their sum in the lane's channels 2 lane + 128 j
  const auto join = [&](int64_t t, int from, int by, float2 (&o)[4], float& m, float& l) {
    const RowParts r = p.parts[t * p.heads + h];
    const int64_t last = r.first + static_cast<int64_t>(r.count - 1) * r.step;
    const bool fits = r.first >= 0 && r.step >= 0 && r.row >= 0 && r.row < p.plan.rows && last < p.plan.grid;
    const int count = fits ? r.count : 0;
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = make_float2(0.f, 0.f);
    const auto slot = [&](int s) {
      return p.slots + ((r.first + static_cast<int64_t>(s) * r.step) * p.plan.rows + r.row) * line;
    };
    for (int s = lane; s < count; s += 64) m = fmaxf(m, slot(s)[0]);
    for (int x = 32; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll 4
    for (int s = from; s < count; s += by) {
      const float* at = slot(s);
      const float2 ml = *reinterpret_cast<const float2*>(at);
      const float w = __builtin_amdgcn_exp2f(ml.x - base);
      l += w * ml.y;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (2 * lane + 128 * j < latent) {
          const float2 x = *reinterpret_cast<const float2*>(at + 2 + 2 * lane + 128 * j);
          o[j].x += w * x.x;
          o[j].y += w * x.y;
        }
    }
  };
  float2 o[4];
  float m, l;
  if (tokens == 1) {
    join(t0, wave, 4, o, m, l);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (2 * lane + 128 * j < latent) {
        halves[wave][2 * lane + 128 * j] = o[j].x;
        halves[wave][2 * lane + 128 * j + 1] = o[j].y;
      }
    if (lane == 0) halves[wave][latent] = l;
    __syncthreads();
    l = halves[0][latent] + halves[1][latent] + halves[2][latent] + halves[3][latent];
    const float by = l == 0.f ? 0.f : 1.f / l;
    for (int c = tid; c < latent; c += 256)
      put(0, c, (halves[0][c] + halves[1][c] + halves[2][c] + halves[3][c]) * by);
  } else {
    for (int t = wave; t < tokens; t += 4) {
      if (t0 + t >= end) break;
      join(t0 + t, 0, 1, o, m, l);
      const float by = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (2 * lane + 128 * j < latent) {
          put(t, 2 * lane + 128 * j, o[j].x * by);
          put(t, 2 * lane + 128 * j + 1, o[j].y * by);
        }
    }
  }
  __syncthreads();
  // columns past the tokens hold anything: a column's sum is its own
  for (int c0 = 16 * wave; c0 < p.value; c0 += 64) {
    const T* w = reinterpret_cast<const T*>(p.w_v) + (static_cast<int64_t>(h) * p.value + c0 + lr) * latent + kVec * g;
    f32x4 acc{0.f, 0.f, 0.f, 0.f};
    for (int f = 0; f < latent; f += 8 * 4 * kVec) {
      typename Elem<T>::Frag a[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (f + 4 * kVec * j < latent) a[j] = *reinterpret_cast<const typename Elem<T>::Frag*>(w + f + 4 * kVec * j);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (f + 4 * kVec * j < latent) {
#pragma unroll
          for (int i = 0; i < kParts; ++i)
            acc = mma(a[j], *reinterpret_cast<const typename Elem<T>::Frag*>(&rows[i][lr][f + 4 * kVec * j + kVec * g]), acc);
        }
    }
    const int64_t t = t0 + lr;
    if (lr < tokens && t < end) {
      T* out = reinterpret_cast<T*>(p.out.data) + t * p.out.token + h * p.out.head + c0 + 4 * g;
      if (p.out.wide) {
        if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]));
        } else {
          *reinterpret_cast<f32x4*>(out) = acc;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) store1(out + i, acc[i]);
      }
    }
  }
}

// ---- plan and launches -----------------------------------------------------------------------------------
LatentSizes latent_sizes(bool bf16, const LatentPages& c, const SeqBatch& b, int heads) {
  LatentSizes z{};
  SharePlan& plan = z.plan;
  const int64_t requests = std::min<int64_t>(b.n_seqs, b.n_tokens), rows = b.n_tokens * heads;
  const int64_t mean = (rows + requests - 1) / requests;
  const bool two = bf16 && c.latent <= 128;
  plan.rows = mean <= 16 ? 16 : mean <= 32 ? 32 : mean <= 64 || !two ? 64 : 128;
  plan.row_groups = plan.rows >= 64 ? 4 : plan.rows / 16;
  plan.heads = 1;
  plan.per_token = heads;
  plan.cut = 1;
  plan.cap = std::min<int64_t>(static_cast<int64_t>(c.cols) * c.page, (int64_t{1} << 31) - 128);
  const int64_t tiles = rows / plan.rows + requests;
  const int64_t goal = std::max(tiles, share_goal(std::min<int64_t>(tiles, 2 * kFill - 1)));
  const int block = bf16 ? 64 : 32;
  const int64_t most = std::max<int64_t>(1, ((plan.cap + block - 1) / block + 1) / 2);  // shares of two blocks each
  plan.grid = tiles > goal / most ? goal : tiles * most;
  const auto up = [](size_t n) { return (n + 255) & ~size_t{255}; };
  const size_t eb = bf16 ? 2 : 4, parts = bf16 ? 2 : 1;
  z.absorbed = up(static_cast<size_t>(rows) * parts * (c.latent + c.turned) * eb);
  z.parts = up(static_cast<size_t>(rows) * sizeof(RowParts));
  z.slots = up(static_cast<size_t>(plan.grid) * plan.rows * (c.latent + 2) * sizeof(float));
  return z;
}

template <typename T, int kTokens>
static void query_as(const LatentAttendParams& p, hipStream_t stream) {
  const int64_t y = (p.batch.n_tokens + kTokens - 1) / kTokens;
  hipLaunchKernelGGL((latent_query_kernel<T, kTokens>), dim3(p.heads, static_cast<unsigned>(y)), dim3(256), 0, stream, p);
}
template <typename T>
static hipError_t attend_as(const LatentAttendParams& p, hipStream_t stream) {
  const int64_t rows = p.batch.n_tokens * p.heads;
  if (rows <= 512) {
    query_as<T, 1>(p, stream);
  } else if (rows <= 2048) {
    query_as<T, 4>(p, stream);
  } else {
    query_as<T, 8>(p, stream);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  e = launch_latent_core(sizeof(T) == 2, p, stream);
  if (e != hipSuccess) return e;
  const int tokens = rows <= 512 ? 1 : static_cast<int>(std::min<int64_t>(16, (rows + 255) / 256));
  const int64_t y = (p.batch.n_tokens + tokens - 1) / tokens;
  hipLaunchKernelGGL((latent_out_kernel<T>), dim3(p.heads, static_cast<unsigned>(y)), dim3(256), 0, stream, p, tokens);
  return hipGetLastError();
}

hipError_t launch_latent_attend(bool bf16, const LatentAttendParams& p, hipStream_t stream) {
  return bf16 ? attend_as<uint16_t>(p, stream) : attend_as<float>(p, stream);
}

hipError_t launch_latent_core_bf16(const LatentAttendParams& p, hipStream_t stream);
hipError_t launch_latent_core_f32(const LatentAttendParams& p, hipStream_t stream);
hipError_t launch_latent_core(bool bf16, const LatentAttendParams& p, hipStream_t stream) {
  return bf16 ? launch_latent_core_bf16(p, stream) : launch_latent_core_f32(p, stream);
}

}  // namespace scd
