// The latent cache (gfx950): rows into pages, queries into the latents' space, the shares of attention
// joined and taken out of it again.
#include <algorithm>

#include "scd_attend_core.h"

namespace scd {
using namespace dev;

// ---- append ------------------------------------------------------------------------------------------
// A wave a token: the latent's bits as they are, the shared key a channel a lane, turned in fp32 and rounded
// once.  Bound by three memory accesses one after the other (owner, page, row): all of the call for a few tokens (64
// tokens 3.3 us), and of a prompt what its waves spend most of their time on, a token each (30000 tokens of 256 + 64
// channels 14 us, 2.7 TB/s of the 5 that a copy reaches).
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
// Channel i of an absorbed query of `width` channels, the first `latent` of them products.
__device__ inline void put_query(uint16_t* row, int latent, int width, int i, float x) {
  // Two bf16 summands hold 16 bits of a product: a score's error then stays below what the rounding of the
  // result to bf16 adds, as in a product of unrounded queries.  The turned channels are the query's own.
  const __bf16 high = static_cast<__bf16>(x);
  row[i] = __builtin_bit_cast(uint16_t, high);
  if (i < latent) row[width + i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x - static_cast<float>(high)));
}
__device__ inline void put_query(float* row, int, int, int i, float x) { row[i] = x; }

// Sums of the lanes up to each lane.
__device__ inline int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // from 1, 2, 4, 8 lanes before, in rows of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // rows 1 and 3: from the row before
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // rows 2 and 3: from lane 31
  return x;
}

// What every workgroup of the attention takes, by one workgroup beside those of the queries: there it costs
// nothing, and the attention, whose start is a chain of memory accesses, finds it with one.
__device__ inline void plan_shares(const LatentAttendParams& p, int block, int tid) {
  // a request among 256 after another
  struct Entry { int64_t begin, held, first; int tokens, tiles, blocks; };
  __shared__ Entry entries[256];
  __shared__ int64_t sums[2][4];
  const int lane = tid & 63, wave = tid >> 6, shift = 31 - __builtin_clz(block);
  const auto load = [&](int b) {
    Entry e{0, 0, 0, 0, 0, 0};
    if (b < p.batch.n_seqs) {
      const Span s = span_of(p.batch, b);
      e.begin = s.begin;
      e.held = s.pos0;
      e.tokens = static_cast<int>(s.end - s.begin);
      int64_t n = s.pos0 + e.tokens;
      n = n < 0 ? 0 : (n > p.plan.cap ? p.plan.cap : n);
      e.blocks = static_cast<int>((n + block - 1) >> shift);
      e.tiles = static_cast<int>((static_cast<uint32_t>(e.tokens) * static_cast<uint32_t>(p.heads) + p.plan.rows - 1) /
                                 static_cast<uint32_t>(p.plan.rows));
    }
    return e;
  };
  // sum over the workgroup of x and y, both below 2^31 a thread of a wave at least
  const auto total_of = [&](int64_t x, int64_t y, int64_t& tx, int64_t& ty) {
    for (int o = 32; o > 0; o >>= 1) {
      x += __shfl_xor(x, o);
      y += __shfl_xor(y, o);
    }
    __syncthreads();  // the last sums' readers are done
    if (lane == 0) {
      sums[0][wave] = x;
      sums[1][wave] = y;
    }
    __syncthreads();
    tx = sums[0][0] + sums[0][1] + sums[0][2] + sums[0][3];
    ty = sums[1][0] + sums[1][1] + sums[1][2] + sums[1][3];
  };
  // as of find_share, from the tiles, all their blocks and those of the longest
  const auto chunk_of = [&](int64_t tiles, int64_t work, int64_t longest) {
    if (tiles <= 0 || tiles >= p.plan.whole) return 0x7fffffffu;
    const int64_t goal = share_goal(tiles, p.plan.fill);
    const int64_t mixed = div_ceil(work, goal - tiles), even = div_ceil(longest, div_up_to(goal, tiles));
    const int64_t chunk = mixed < even ? mixed : even;
    return chunk < 1 ? 1u : static_cast<uint32_t>(chunk);
  };
  const auto parts_of = [](const Entry& e, uint32_t chunk) {
    const uint32_t n = e.blocks;
    return n <= chunk ? 1u : (n + chunk - 1) / chunk;
  };
  // the workgroups whose shares are [first, next), of the requests b0 .. b0 + count - 1 in `entries`
  const auto deal = [&](int b0, int count, int64_t first, int64_t next, int total, uint32_t chunk) {
    for (int w = tid; w < total; w += 256) {
      const int64_t unit = xcd_remap(w, total);
      if (unit < first || unit >= next) continue;
      int lo = 0, hi = count - 1;
      while (lo < hi) {  // the last request whose shares begin at or before the unit
        const int mid = (lo + hi + 1) >> 1;
        if (entries[mid].first <= unit) lo = mid; else hi = mid - 1;
      }
      const Entry e = entries[lo];
      const uint32_t local = static_cast<uint32_t>(unit - e.first);
      LatentShare out;
      out.b = b0 + lo;
      out.tokens = e.tokens;
      out.tiles = e.tiles;
      out.part = static_cast<int>(local / static_cast<uint32_t>(e.tiles));
      out.tile = static_cast<int>(local) - out.part * e.tiles;
      out.parts = static_cast<int>(parts_of(e, chunk));
      out.first = static_cast<int>(e.first) + out.tile;
      out.pad = 0;
      out.begin = e.begin;
      out.held = e.held;
      p.shares[w] = out;
    }
  };
  const auto none = [&](int64_t from) {
    for (int64_t w = from + tid; w < p.plan.grid; w += 256) p.shares[w].b = -1;
  };
  const int64_t most = (p.batch.n_tokens * p.heads / p.plan.rows + p.batch.n_seqs) * ((p.plan.cap + block - 1) >> shift);
  if (p.batch.n_seqs <= 64 && most < int64_t{1} << 31) {
    // one wave's lanes hold the requests, sums in 32 bits
    if (wave == 0) {
      Entry e = load(lane);
      const int tiles = __builtin_amdgcn_readlane(wave_scan(e.tiles), 63);
      const int work = __builtin_amdgcn_readlane(wave_scan(e.tiles * e.blocks), 63);
      int longest = e.tiles > 0 ? e.blocks : 0;
      for (int o = 32; o > 0; o >>= 1) {
        const int other = __shfl_xor(longest, o);
        longest = other > longest ? other : longest;
      }
      const uint32_t chunk = chunk_of(tiles, work, longest);
      const int shares = e.tiles * static_cast<int>(parts_of(e, chunk)), sum = wave_scan(shares);
      e.first = sum - shares;
      entries[lane] = e;
      if (lane == 63) {
        sums[0][0] = sum;
        sums[0][1] = chunk;
      }
    }
    __syncthreads();
    const int64_t total = sums[0][0] < 0 ? 0 : (sums[0][0] < p.plan.grid ? sums[0][0] : p.plan.grid);
    deal(0, p.batch.n_seqs, 0, total, static_cast<int>(total), static_cast<uint32_t>(sums[0][1]));
    none(total);
    return;
  }
  int64_t tiles = 0, work = 0, longest = 0, total = 0, rest = 0;
  for (int b = tid; b < p.batch.n_seqs; b += 256) {
    const Entry e = load(b);
    tiles += e.tiles;
    work += static_cast<int64_t>(e.tiles) * e.blocks;
    longest = e.tiles > 0 && e.blocks > longest ? e.blocks : longest;
  }
  total_of(tiles, work, tiles, work);
  for (int o = 32; o > 0; o >>= 1) {
    const int64_t other = __shfl_xor(longest, o);
    longest = other > longest ? other : longest;
  }
  __syncthreads();  // the sums' readers are done
  if (lane == 0) sums[0][wave] = longest;
  __syncthreads();
  for (int w = 0; w < 4; ++w) longest = sums[0][w] > longest ? sums[0][w] : longest;
  const uint32_t chunk = chunk_of(tiles, work, longest);
  for (int b = tid; b < p.batch.n_seqs; b += 256) {
    const Entry e = load(b);
    total += static_cast<int64_t>(e.tiles) * parts_of(e, chunk);
  }
  total_of(total, rest, total, rest);
  total = total < p.plan.grid ? total : p.plan.grid;
  int64_t first = 0;
  for (int b0 = 0; b0 < p.batch.n_seqs; b0 += 256) {
    Entry mine = load(b0 + tid);
    const int64_t n = static_cast<int64_t>(mine.tiles) * parts_of(mine, chunk);
    int64_t sum = n;
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t other = __shfl_up(sum, o);
      if (lane >= o) sum += other;
    }
    __syncthreads();  // the last round's readers are done
    if (lane == 63) sums[1][wave] = sum;
    __syncthreads();
    mine.first = first + sum - n;
    for (int w = 0; w < wave; ++w) mine.first += sums[1][w];
    const int64_t next = first + sums[1][0] + sums[1][1] + sums[1][2] + sums[1][3];
    entries[tid] = mine;
    __syncthreads();
    deal(b0, p.batch.n_seqs - b0 < 256 ? p.batch.n_seqs - b0 : 256, first, next, static_cast<int>(total), chunk);
    first = next;
  }
  none(total);
}

// absorbed_h = [ q_h[:plain] W_k,h | q_h[plain:] ], of the other sign for a negative scale:
// workgroup (h, a few tokens), eight latent channels a thread, the matrix's rows dealt to groups of threads whose sums meet
// in LDS.  The matrix is read once for kTokens tokens; with few tokens that read, and the memory accesses in front of it,
// are the call (16 tokens of 32 heads 6.8 us).
template <typename T, int kTokens>
__global__ __launch_bounds__(256) void latent_query_kernel(LatentAttendParams p) {
  constexpr int kAhead = 16;  // rows of the matrix under way for a thread
  __shared__ float q[kTokens][256 + 64];
  __shared__ __attribute__((aligned(16))) float sums[kTokens * 2048];
  const int tid = threadIdx.x, h = static_cast<int>(blockIdx.x) - 1;
  if (h >= p.heads) return;
  if (h < 0) {
    if (blockIdx.y == 0) {
      if (tid < 64) reinterpret_cast<uint32_t*>(p.zeros)[tid] = 0;
      plan_shares(p, latent_block(sizeof(T) == 2), tid);
    }
    return;
  }
  const int64_t t0 = static_cast<int64_t>(blockIdx.y) * kTokens;
  const int n = static_cast<int>(p.batch.n_tokens - t0 < kTokens ? p.batch.n_tokens - t0 : kTokens);
  const int latent = p.cache.latent, turned = p.cache.turned, width = latent + turned;
  const int wide = p.plain + turned;
  const int eights = latent / 8, groups = 256 / eights;
  const int group = tid / eights, eight = tid - group * eights;
  const bool works = group < groups;
  const T* w = reinterpret_cast<const T*>(p.w_k) + static_cast<int64_t>(h) * p.plain * latent + 8 * eight;
  // the first rows are on their way while the queries are
  constexpr int kWords = sizeof(T) / 2;
  u32x4 x[kAhead][kWords];
  const auto rows = [&](int d0) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
#pragma unroll
      for (int i = 0; i < kWords; ++i)
        if (works && d0 + j * groups < p.plain)
          x[j][i] = reinterpret_cast<const u32x4*>(w + static_cast<int64_t>(d0 + j * groups) * latent)[i];
  };
  rows(group);
  for (int i = tid; i < kTokens * wide; i += 256) {
    const int t = i / wide, c = i - t * wide;
    float y = 0.f;
    if (t < n) y = load1(reinterpret_cast<const T*>(p.q.data) + (t0 + t) * p.q.token + h * p.q.head + c);
    q[t][c] = p.scale < 0.f ? -y : y;
  }
  __syncthreads();
  float acc[kTokens][8];
#pragma unroll
  for (int t = 0; t < kTokens; ++t)
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[t][i] = 0.f;
  for (int d0 = group; d0 < p.plain; d0 += kAhead * groups) {
    if (d0 != group) rows(d0);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int d = d0 + j * groups;
      if (works && d < p.plain) {
        float f[8];
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            f[2 * i] = bf16_lo(x[j][0][i]);
            f[2 * i + 1] = bf16_hi(x[j][0][i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(x[j][i >> 2][i & 3]);
        }
#pragma unroll
        for (int t = 0; t < kTokens; ++t) {
          const float y = q[t][d];
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[t][i] += f[i] * y;
        }
      }
    }
  }
  if (works) {
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
      float* to = &sums[(group * kTokens + t) * latent + 8 * eight];
      *reinterpret_cast<f32x4*>(to) = f32x4{acc[t][0], acc[t][1], acc[t][2], acc[t][3]};
      *reinterpret_cast<f32x4*>(to + 4) = f32x4{acc[t][4], acc[t][5], acc[t][6], acc[t][7]};
    }
  }
  __syncthreads();
  const int line = query_width(sizeof(T) == 2, latent, turned);
  for (int i = tid; i < n * width; i += 256) {
    const int t = i / width, c = i - t * width;
    float y = 0.f;
    if (c < latent) {
      for (int g = 0; g < groups; ++g) y += sums[(g * kTokens + t) * latent + c];
    } else {
      y = q[t][p.plain + c - latent];
    }
    put_query(reinterpret_cast<T*>(p.absorbed) + ((t0 + t) * p.heads + h) * line, latent, width, c, y);
  }
}

// ---- shares joined, results out of the latents' space ----------------------------------------------------
// out_h = W_v,h (sum_s 2^(m_s - m) o_s) / (sum_s 2^(m_s - m) l_s) over a row's shares s: workgroup (h, tokens
// of it).  One or two tokens' shares are dealt to the four waves, more tokens are dealt as they are.  The joined
// rows, as two bf16 summands, are the right operands of the product with W_v,h, whose rows come from memory
// as they lie.  Bound by latency: shares' places, shares, product (16 tokens of 32 heads 9.9 us).
template <typename T, int kMost>
__global__ __launch_bounds__(256) void latent_out_kernel(LatentAttendParams p, int tokens) {
  constexpr int kParts = sizeof(T) == 2 ? 2 : 1, kPairs = kMost / 128;
  constexpr int kVec = Elem<T>::kVec, kRow = kMost + kVec;  // 16-byte pieces of a row: odd
  __shared__ __attribute__((aligned(16))) T rows[kParts][16][kRow];
  __shared__ float halves[4][kMost + 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, g = lane >> 4;
  const int h = blockIdx.x, latent = p.cache.latent, line = latent + 2;
  if (h >= p.heads) return;
  const int64_t t0 = static_cast<int64_t>(blockIdx.y) * tokens;
  // rows behind the last request are left alone: joined like the others (their entries are checked), not stored
  const int32_t stop = p.batch.cu != nullptr ? p.batch.cu[p.batch.n_seqs] : 0x7fffffff;

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
  const auto join = [&](int64_t t, int from, int by, float2 (&o)[kPairs], float& m, float& l) {
    const RowParts r = p.parts[t * p.heads + h];
    const int64_t last = r.first + static_cast<int64_t>(r.count - 1) * r.step;
    const bool fits = r.first >= 0 && r.step >= 0 && r.row >= 0 && r.row < p.plan.rows && last < p.plan.grid &&
                      r.count <= p.plan.grid;
    const int count = uniform(fits ? r.count : 0);
    const float* row = p.slots + (static_cast<int64_t>(uniform(r.first)) * p.plan.rows + uniform(r.row)) * line;
    const int64_t step = static_cast<int64_t>(uniform(r.step)) * p.plan.rows * line;
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) o[j] = make_float2(0.f, 0.f);
    // eight shares at a time, all of their values on the way before the first is used
    for (int s0 = from; s0 < count; s0 += 8 * by) {
      float2 ml[8], x[8][kPairs];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int s = s0 + u * by;
        ml[u] = make_float2(-INFINITY, 0.f);
        if (s < count) ml[u] = *reinterpret_cast<const float2*>(row + s * step);
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
          x[u][j] = make_float2(0.f, 0.f);
          if (s < count && 2 * lane + 128 * j < latent)
            x[u][j] = *reinterpret_cast<const float2*>(row + s * step + 2 + 2 * lane + 128 * j);
        }
      }
      float now = m;
#pragma unroll
      for (int u = 0; u < 8; ++u) now = fmaxf(now, ml[u].x);
      const float base = now == -INFINITY ? 0.f : now, old = __builtin_amdgcn_exp2f(m - base);
      m = now;
      l *= old;
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        o[j].x *= old;
        o[j].y *= old;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float w = __builtin_amdgcn_exp2f(ml[u].x - base);
        l += w * ml[u].y;
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
          o[j].x += w * x[u][j].x;
          o[j].y += w * x[u][j].y;
        }
      }
    }
  };
  typedef typename Elem<T>::Frag Frag;
  // the first 8 pieces of the wave's first two tiles of value rows come while the shares are joined
  const T* wv = reinterpret_cast<const T*>(p.w_v) + (static_cast<int64_t>(h) * p.value + lr) * latent + kVec * g;
  const auto pieces = [&](int c0, int f, Frag (&a)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c0 < p.value && f + 4 * kVec * j < latent)
        a[j] = *reinterpret_cast<const Frag*>(wv + static_cast<int64_t>(c0) * latent + f + 4 * kVec * j);
  };
  Frag ahead[2][8];
  pieces(16 * wave, 0, ahead[0]);
  pieces(16 * wave + 64, 0, ahead[1]);
  float2 o[kPairs];
  float m, l;
  if (tokens <= 2) {
    // the waves of a token (4, or 2 of two tokens) leave their shares' sums in LDS
    const int per = 4 / tokens, t = wave / per;
    join(t0 + t < p.batch.n_tokens ? t0 + t : t0, wave - t * per, per, o, m, l);
#pragma unroll
    for (int j = 0; j < kPairs; ++j)
      if (2 * lane + 128 * j < latent) *reinterpret_cast<float2*>(&halves[wave][2 + 2 * lane + 128 * j]) = o[j];
    if (lane == 0) *reinterpret_cast<float2*>(&halves[wave][0]) = make_float2(m, l);
    __syncthreads();
    for (int i = tid; i < tokens * latent; i += 256) {
      const int row = tokens == 1 || i < latent ? 0 : 1, c = i - row * latent, w0 = row * per;
      float top = -INFINITY, sum = 0.f, x = 0.f;
      for (int w = w0; w < w0 + per; ++w) top = fmaxf(top, halves[w][0]);
      const float base = top == -INFINITY ? 0.f : top;
      for (int w = w0; w < w0 + per; ++w) {
        const float by = __builtin_amdgcn_exp2f(halves[w][0] - base);
        sum += by * halves[w][1];
        x += by * halves[w][2 + c];
      }
      put(row, c, sum == 0.f ? 0.f : x / sum);
    }
  } else {
    for (int t = wave; t < tokens; t += 4) {
      if (t0 + t >= p.batch.n_tokens) break;
      join(t0 + t, 0, 1, o, m, l);
      const float by = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int j = 0; j < kPairs; ++j)
        if (2 * lane + 128 * j < latent) {
          put(t, 2 * lane + 128 * j, o[j].x * by);
          put(t, 2 * lane + 128 * j + 1, o[j].y * by);
        }
    }
  }
  __syncthreads();
  // columns past the tokens hold anything: a column's sum is its own
  for (int c0 = 16 * wave; c0 < p.value; c0 += 64) {
    f32x4 acc{0.f, 0.f, 0.f, 0.f};
    for (int f = 0; f < latent; f += 8 * 4 * kVec) {
      Frag a[8];
      if (c0 < 128 && f == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] = c0 < 64 ? ahead[0][j] : ahead[1][j];
      } else {
        pieces(c0, f, a);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (f + 4 * kVec * j < latent) {
#pragma unroll
          for (int i = 0; i < kParts; ++i)
            acc = mma(a[j], *reinterpret_cast<const Frag*>(&rows[i][lr][f + 4 * kVec * j + kVec * g]), acc);
        }
    }
    settle();
    const int64_t t = t0 + lr;
    if (lr < tokens && t < p.batch.n_tokens && t < stop) {
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
  plan.rows = mean <= 16 ? 16 : mean <= 32 || c.latent > 256 ? 32 : mean <= 64 || c.latent > 128 ? 64 : 128;
  // Few tiles are more tiles of half the height, but not below what a token of 32 heads has, whose rows a second tile would
  // fetch again (us, halved | whole): two tokens of 16 requests of 1000 32 | 37, of 4000 41 | 45; 64 tokens behind 2000 47 |
  // 51; 5 tokens of 4 requests, 64 heads, r = 128, 29 | 32; a token of 16 of 4000 at r = 512 60 | 61.  The other sides: 128
  // tokens behind 2000 70 | 71, 200 118 | 105; a token of 16 requests of 1K to 16K, 32 heads, 51 | 45.
  if (plan.rows > (c.latent > 256 ? 16 : 32) && rows <= 32 * plan.rows) plan.rows /= 2;
  plan.row_groups = plan.rows / 16;
  plan.heads = 1;
  plan.per_token = heads;
  plan.cut = 1;
  plan.fill = 256;  // eight waves and most of a CU's LDS each
  plan.cap = std::min<int64_t>(static_cast<int64_t>(c.cols) * c.page, (int64_t{1} << 31) - 128);
  const int64_t tiles = rows / plan.rows + requests;
  plan.whole = 512;
  const int64_t goal = std::max(tiles, share_goal(std::min<int64_t>(tiles, plan.whole - 1), plan.fill));
  const int block = latent_block(bf16);
  const int64_t most = std::max<int64_t>(1, (plan.cap + block - 1) / block);  // shares of a block each
  plan.grid = tiles > goal / most ? goal : tiles * most;
  const auto up = [](size_t n) { return (n + 255) & ~size_t{255}; };
  z.zeros = 256;
  z.absorbed = up(static_cast<size_t>(rows) * query_width(bf16, c.latent, c.turned) * (bf16 ? 2 : 4));
  z.shares = up(static_cast<size_t>(plan.grid) * sizeof(LatentShare));
  z.parts = up(static_cast<size_t>(rows) * sizeof(RowParts));
  z.slots = up(static_cast<size_t>(plan.grid) * plan.rows * (c.latent + 2) * sizeof(float));
  return z;
}

// From half a megabyte of matrices on, a multiple of the XCDs that workgroups are dealt to: a head's workgroups, one behind
// another in y, then share one, and its matrix is read into one L2.  Queries of 16 tokens of 32 heads, 2 MB: 8.0 us spread
// over all XCDs, 6.8 so; of 37 fp32 tokens of 8 heads, 128 KB: 4.8 spread, 6.7 so.
static unsigned heads_grid(int heads, int64_t matrix_bytes) {
  return matrix_bytes < int64_t{1} << 19 ? heads : (heads + kNumXcd - 1) / kNumXcd * kNumXcd;
}

template <typename T, int kTokens>
static void query_as(const LatentAttendParams& p, hipStream_t stream) {
  const int64_t y = (p.batch.n_tokens + kTokens - 1) / kTokens;
  hipLaunchKernelGGL((latent_query_kernel<T, kTokens>), dim3(heads_grid(p.heads + 1, int64_t{p.heads} * p.plain * p.cache.latent * sizeof(T)),
                                                               static_cast<unsigned>(y)), dim3(256), 0, stream, p);
}
template <typename T>
static hipError_t attend_as(const LatentAttendParams& p, hipStream_t stream) {
  const int64_t rows = p.batch.n_tokens * p.heads;
  // one token a workgroup or four, whole calls in us: 16 tokens of 16 heads 28.5 | 31.2, a token of 64 requests of 32
  // heads 47.9 | 45.8, 200 tokens 115 | 105
  if (rows <= 1024) {
    query_as<T, 1>(p, stream);
  } else {
    query_as<T, 4>(p, stream);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  e = launch_latent_core(sizeof(T) == 2, p, stream);
  if (e != hipSuccess) return e;
  // a workgroup a CU while there are so few tokens: a token of 16 requests of 32 heads 34.0 us (16 tokens a workgroup 41.6,
  // one 36.2), of 64 requests 45.7 (48.2, 63.7)
  const int tokens = static_cast<int>(std::min<int64_t>(std::max<int64_t>(1, rows / 256), 16));
  const int64_t y = (p.batch.n_tokens + tokens - 1) / tokens;
  const dim3 grid(heads_grid(p.heads, int64_t{p.heads} * p.value * p.cache.latent * sizeof(T)), static_cast<unsigned>(y));
  if (p.cache.latent <= 128) {
    hipLaunchKernelGGL((latent_out_kernel<T, 128>), grid, dim3(256), 0, stream, p, tokens);
  } else if (p.cache.latent <= 256) {
    hipLaunchKernelGGL((latent_out_kernel<T, 256>), grid, dim3(256), 0, stream, p, tokens);
  } else {
    hipLaunchKernelGGL((latent_out_kernel<T, 512>), grid, dim3(256), 0, stream, p, tokens);
  }
  return hipGetLastError();
}

hipError_t launch_latent_attend(bool bf16, const LatentAttendParams& p, hipStream_t stream) {
  return bf16 ? attend_as<uint16_t>(p, stream) : attend_as<float>(p, stream);
}

hipError_t launch_latent_core(bool bf16, const LatentAttendParams& p, hipStream_t stream) {
  return bf16 ? launch_latent_core_bf16(p, stream) : launch_latent_core_f32(p, stream);
}

}  // namespace scd
