// Causal attention of new tokens over the paged 8-bit cache (gfx950).
//
// out = sum_j p_j v_j with p the softmax over the cached positions of scale * (q . k_j), in one pass
// with a running maximum and sum: when the maximum grows from m to m', what is summed so far is
// multiplied by e^(m - m').  Both products run on the matrix cores with fp32 accumulation:
//  - cached values are whole numbers of at most 127, exact in fp16 and bf16; a page's key scale
//    multiplies the scores, its value scale the weights, so no value is scaled one by one.
//  - scores in fp16: a query row is multiplied by the power of two that brings its largest element to
//    2^14 (its scores by the inverse).  bf16 rows are then exact down to 2^-28 of that element; fp32
//    rows are split into two parts (22 bits and their sign).
//  - sums over values in bf16, the weights split into two parts for bf16 output (16 bits; its own
//    rounding has 8) and three for fp32: the parts keep the whole exponent range, so a channel in
//    which the heaviest positions are zero still has its bits.
//  - a value scale is f 2^e with f in [1, 2).  The running maximum is that of log2 of the weight plus
//    e, what a position can add to the sum; the softmax's own sum takes the weights times 2^-e.
#include <algorithm>

#include "scd_serve_device.h"

namespace scd {
using namespace dev;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef const __attribute__((address_space(4))) int32_t* uniform_ints_t;
typedef const __attribute__((address_space(4))) float* uniform_floats_t;

constexpr float kLog2e = 1.44269504f;
constexpr int kLift = 14;  // the largest element of a query row is brought to 2^kLift
constexpr int kLeastExponent = -90;  // of a value scale: 2^90 times 2^31 positions fits the sum

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline f32x4 mfma16(const f16x8& a, const f16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

__device__ inline f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Two bytes (sign bit flipped: value + 128) with 0x64 above each are the halves 1152 + value; less
// 1152 they are the values.
__device__ inline uint32_t halves(uint32_t biased) {
  const f16x2 offset = {static_cast<_Float16>(-1152.f), static_cast<_Float16>(-1152.f)};
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, biased) + offset);
}
// Eight adjacent bytes as fp16.
__device__ inline f16x8 bytes_as_f16(uint32_t a, uint32_t b) {
  a ^= 0x80808080u;
  b ^= 0x80808080u;
  u32x4 w;
  w[0] = halves(__builtin_amdgcn_perm(0x64646464u, a, 0x04010400u));
  w[1] = halves(__builtin_amdgcn_perm(0x64646464u, a, 0x04030402u));
  w[2] = halves(__builtin_amdgcn_perm(0x64646464u, b, 0x04010400u));
  w[3] = halves(__builtin_amdgcn_perm(0x64646464u, b, 0x04030402u));
  return __builtin_bit_cast(f16x8, w);
}
// Byte kByte of eight words as bf16: fp32 of a byte is exact in its upper half.
template <int kByte> __device__ inline float byte_as_f32(uint32_t w) {
  return static_cast<float>(static_cast<int8_t>(w >> (8 * kByte)));
}
template <int kByte> __device__ inline bf16x8 byte_column_as_bf16(const uint32_t (&w)[8]) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = __builtin_amdgcn_perm(__float_as_uint(byte_as_f32<kByte>(w[2 * i + 1])),
                                 __float_as_uint(byte_as_f32<kByte>(w[2 * i])), 0x07060302u);
  return __builtin_bit_cast(bf16x8, r);
}

// Positions the page table can name (cut off where positions would pass 31 bits).
__device__ inline int64_t positions_held(const PagedCache& c) {
  const int64_t n = static_cast<int64_t>(c.cols) << c.page_log2, most = (int64_t{1} << 31) - 64;
  return n < most ? n : most;
}

// Rows of one tile: query rows (token, head of the group) of one request and KV head.
struct Tile {
  int b;
  int64_t row0;      // first row, in the request
  int rows;          // rows of the tile that exist
  int64_t first;     // packed row of the request's first token
  int64_t pos0;
};

// Tiles of kRows rows of all requests, one after another.
template <int kRows, int kThreads = 256>
__device__ inline bool tile_of(const CacheAttendParams& p, int64_t index, LocateLds& lds, int tid, Tile& t) {
  Located at;
  if (!locate<kThreads>(p.batch, index, lds, tid,
                        [&](const Span& s) { return ((s.end - s.begin) * p.group + kRows - 1) / kRows; }, at))
    return false;
  t.b = at.b;
  t.row0 = at.local * kRows;
  const int64_t left = (at.span.end - at.span.begin) * p.group - t.row0;
  t.rows = static_cast<int>(left < kRows ? left : kRows);
  t.first = at.span.begin;
  t.pos0 = at.span.pos0;
  return true;
}
__host__ __device__ inline int64_t tiles_bound(int64_t n_tokens, int32_t n_seqs, int group, int rows) {
  const int64_t requests = n_seqs < n_tokens ? n_seqs : n_tokens;
  return n_tokens * group / rows + requests;
}

// Splits of a tile that has `blocks` blocks of 32 positions, when a launch has up to `most`: at least
// two blocks for each of a workgroup's four waves.
__device__ inline int splits_of(int64_t blocks, int most) {
  const int64_t n = (blocks + 7) / 8;
  return static_cast<int>(n < 1 ? 1 : (n < most ? n : most));
}

// One workgroup per tile of 16 kBlocks query rows, KV head and share of the positions.  Its four waves
// take blocks of 32 positions in turn, straight from the pages into registers in the layout of the
// matrix operands, so no value passes through LDS:
//   scores^T [32 x 16] = K Q^T: a lane holds positions (4g + i, 16 + 4g + i) of one query row, which
//   is the operand layout of   out^T [d x 16] += V^T P^T   with the positions in that order.
// The contraction over channels, and the order of the output channels over the matrix rows, are
// permuted so that every lane reads adjacent bytes.
template <typename T, int kDim, int kBlocks>
__global__ __launch_bounds__(256) void cache_attend_rows_kernel(CacheAttendParams p, int most_splits,
                                                               int64_t units, float* partial,
                                                               float* partial_ml) {
  constexpr int kParts = sizeof(T) == 2 ? 1 : 2;    // of a query element
  constexpr int kWeights = sizeof(T) == 2 ? 2 : 3;  // of a weight
  constexpr int kRows = 16 * kBlocks;
  constexpr int kSteps = kDim / 32;   // matrix steps over channels
  constexpr int kOut = kDim / 16;     // output channels a lane holds of each of its four matrix rows
  constexpr int kPitch = kDim + 4;
  __shared__ LocateLds locate_lds;
  __shared__ float joined[4][16][kPitch];
  __shared__ float joined_m[4][kRows], joined_l[4][kRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const uniform_ints_t table = (uniform_ints_t)(p.cache.table);
  const uniform_floats_t k_scale = (uniform_floats_t)(p.cache.k_scale);
  const uniform_floats_t v_scale = (uniform_floats_t)(p.cache.v_scale);

  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int h = static_cast<int>(unit % p.cache.heads);
    const int64_t rest = unit / p.cache.heads;
    const int split = static_cast<int>(rest % most_splits);
    Tile t;
    if (!tile_of<kRows>(p, rest / most_splits, locate_lds, tid, t)) return;
    const int64_t last_row = t.row0 + t.rows - 1;
    int64_t seen = t.pos0 + last_row / p.group + 1;  // positions the tile's last row attends to
    const int64_t held = positions_held(p.cache);
    seen = seen < 0 ? 0 : (seen < held ? seen : held);
    const int64_t blocks = (seen + 31) >> 5;
    const int splits = splits_of(blocks, most_splits);
    if (split >= splits) continue;
    const int begin = static_cast<int>(blocks * split / splits), end = static_cast<int>(blocks * (split + 1) / splits);
    const int64_t free_until = t.pos0 + t.row0 / p.group + 1;  // positions every row attends to

    // queries
    f16x8 q[kBlocks][kParts][kSteps];
    float factor[kBlocks];
    int limit[kBlocks];  // last position of the lane's row
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) {
      int64_t row = t.row0 + 16 * n + r;
      row = row > last_row ? last_row : row;
      const int64_t token = row / p.group;
      const int head = h * p.group + static_cast<int>(row - token * p.group);
      const T* src = reinterpret_cast<const T*>(p.q.data) + (t.first + token) * p.q.token + head * p.q.head + g * (kDim / 4);
      float x[kSteps][8];
      float top = 0.f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        load8(src + 8 * s, p.q.wide, x[s]);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[s][j]));
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      int e = (__float_as_uint(top) >> 23) & 255;
      e = e < kLift + 1 ? kLift + 1 : (e > 254 ? 254 : e);
      const float lift = __uint_as_float(static_cast<uint32_t>(254 + kLift - e) << 23);
      factor[n] = __uint_as_float(static_cast<uint32_t>(e - kLift) << 23) * (p.scale * kLog2e);
      const int64_t reach = t.pos0 + token;
      limit[n] = static_cast<int>(reach < held ? reach : held);
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float v = x[s][j] * lift;
          const _Float16 hi = static_cast<_Float16>(v);
          q[n][0][s][j] = hi;
          if constexpr (kParts == 2) q[n][1][s][j] = static_cast<_Float16>(v - static_cast<float>(hi));
        }
    }

    f32x4 acc[kBlocks][kOut];
    float m[kBlocks], l[kBlocks];
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) {
      m[n] = -INFINITY;
      l[n] = 0.f;
#pragma unroll
      for (int c = 0; c < kOut; ++c) acc[n][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // Blocks are fetched one ahead of the arithmetic, their pages' numbers another one ahead.
    const auto pages_of = [&](int block) {
      int2 id;
      int* const out[2] = {&id.x, &id.y};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int col = ((block << 5) + 16 * i) >> p.cache.page_log2;
        *out[i] = col < p.cache.cols ? table[static_cast<int64_t>(t.b) * p.cache.cols + col] : -1;
      }
      return id;
    };
    struct Fetched {
      uint32_t kw[2][kDim / 16];
      uint32_t vw[kDim / 64 > 0 ? kDim / 64 : 1][8];
      float ks[2], vs[2];
      bool hole[2];
    };
    const auto fetch = [&](Fetched& f, int block, int2 ids) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int id = i == 0 ? ids.x : ids.y;
        f.hole[i] = id < 0 || id >= p.cache.n_pages;
        id = f.hole[i] ? 0 : id;
        const int64_t at = static_cast<int64_t>(id) * p.cache.heads + h;
        f.ks[i] = f.hole[i] ? 0.f : k_scale[at];
        f.vs[i] = f.hole[i] ? 0.f : v_scale[at];
        const int64_t byte = page_at(p.cache, id, h, kDim) + ((((block << 5) + 16 * i) & (p.cache.page - 1)) * kDim);
        // keys: position r of the half, channels g * kDim / 4 on
        const int8_t* src = p.cache.k + byte + (r * kDim + g * (kDim / 4));
        if constexpr (kDim >= 64) {
#pragma unroll
          for (int c = 0; c < kDim / 64; ++c) {
            const uint4 w = *reinterpret_cast<const uint4*>(src + 16 * c);
            f.kw[i][4 * c] = w.x; f.kw[i][4 * c + 1] = w.y; f.kw[i][4 * c + 2] = w.z; f.kw[i][4 * c + 3] = w.w;
          }
        } else {
          const uint2 w = *reinterpret_cast<const uint2*>(src);
          f.kw[i][0] = w.x; f.kw[i][1] = w.y;
        }
        // values: channels kOut * r on, of positions 4g + j of the half
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          src = p.cache.v + byte + ((4 * g + j) * kDim + kOut * r);
          if constexpr (kDim == 128) {
            const uint2 w = *reinterpret_cast<const uint2*>(src);
            f.vw[0][4 * i + j] = w.x;
            f.vw[1][4 * i + j] = w.y;
          } else if constexpr (kDim == 64) {
            f.vw[0][4 * i + j] = *reinterpret_cast<const uint32_t*>(src);
          } else {
            f.vw[0][4 * i + j] = *reinterpret_cast<const uint16_t*>(src);
          }
        }
      }
    };
    const auto attend = [&](const Fetched& fetched, int block) {
      const int at = block << 5;
      const auto& kw = fetched.kw;
      const auto& vw = fetched.vw;
      const float (&ks)[2] = fetched.ks;
      const float (&vs)[2] = fetched.vs;
      // scores
      f32x4 score[kBlocks][2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int n = 0; n < kBlocks; ++n) score[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const f16x8 k = bytes_as_f16(kw[i][2 * s], kw[i][2 * s + 1]);
#pragma unroll
          for (int n = 0; n < kBlocks; ++n)
#pragma unroll
            for (int part = 0; part < kParts; ++part) score[n][i] = mfma16(k, q[n][part][s], score[n][i]);
        }
      }
      // value scales as f 2^e (e at least kLeastExponent, where f may be below 1 or 0)
      float part_scale[2], exponent[2], back[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int e = (__float_as_uint(vs[i]) >> 23) & 255;
        e = e < 127 + kLeastExponent ? 127 + kLeastExponent : (e > 253 ? 253 : e);
        back[i] = __uint_as_float(static_cast<uint32_t>(254 - e) << 23);
        part_scale[i] = vs[i] * back[i];
        exponent[i] = static_cast<float>(e - 127);
      }
      const bool masked = at + 32 > free_until || fetched.hole[0] || fetched.hole[1];
      bf16x8 w[kBlocks][kWeights];
#pragma unroll
      for (int n = 0; n < kBlocks; ++n) {
        float x[8];
        bool hidden[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float f = ks[i] * factor[n];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[4 * i + j] = fmaf(score[n][i][j], f, exponent[i]);
            hidden[4 * i + j] = masked && (fetched.hole[i] || at + 16 * i + 4 * g + j > limit[n]);
            if (hidden[4 * i + j]) x[4 * i + j] = -INFINITY;
          }
        }
        float top = m[n];
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, x[j]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -INFINITY ? 0.f : top;
        const float fade = exp2_fast(m[n] - base);
        m[n] = top;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float e = exp2_fast(x[j] - base);
          sum[j >> 2] += e;
          float v = hidden[j] ? 0.f : e * part_scale[j >> 2];
#pragma unroll
          for (int k = 0; k < kWeights; ++k) {
            w[n][k][j] = static_cast<__bf16>(v);
            v -= static_cast<float>(w[n][k][j]);
          }
        }
        l[n] = l[n] * fade + sum[0] * back[0] + sum[1] * back[1];
#pragma unroll
        for (int c = 0; c < kOut; ++c) acc[n][c] *= fade;
      }
      // values
      const auto out = [&](auto byte, int word) {
        constexpr int kByte = decltype(byte)::value;
        const bf16x8 v = byte_column_as_bf16<kByte>(vw[word]);
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
          for (int part = 0; part < kWeights; ++part)
            acc[n][4 * word + kByte] = mfma16(v, w[n][part], acc[n][4 * word + kByte]);
      };
      out(IntC<0>{}, 0);
      out(IntC<1>{}, 0);
      if constexpr (kOut >= 4) {
        out(IntC<2>{}, 0);
        out(IntC<3>{}, 0);
      }
      if constexpr (kOut == 8) {
        out(IntC<0>{}, 1);
        out(IntC<1>{}, 1);
        out(IntC<2>{}, 1);
        out(IntC<3>{}, 1);
      }
    };
    int block = begin + wave;
    if (block < end) {
      Fetched now, next;
      fetch(now, block, pages_of(block));
      int2 ids = pages_of(block + 4);
      while (true) {
        if (block + 4 < end) {
          fetch(next, block + 4, ids);
          ids = pages_of(block + 8);
        }
        attend(now, block);
        block += 4;
        if (block >= end) break;
        if (block + 4 < end) {
          fetch(now, block + 4, ids);
          ids = pages_of(block + 8);
        }
        attend(next, block);
        block += 4;
        if (block >= end) break;
      }
    }

    // join the waves, 16 rows at a time
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) {
      l[n] += __shfl_xor(l[n], 16);
      l[n] += __shfl_xor(l[n], 32);
      if (g == 0) {
        joined_m[wave][16 * n + r] = m[n];
        joined_l[wave][16 * n + r] = l[n];
      }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) {
      float top = joined_m[0][16 * n + r];
      for (int v = 1; v < 4; ++v) top = fmaxf(top, joined_m[v][16 * n + r]);
      const float mine = exp2_fast(m[n] - (top == -INFINITY ? 0.f : top));
      float* dst = joined[wave][r];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < kOut; ++c) dst[kOut * (4 * g + i) + c] = acc[n][c][i] * mine;
      __syncthreads();
      for (int item = tid; item < 16 * (kDim / 8); item += 256) {
        const int row = item / (kDim / 8), chunk = item % (kDim / 8);
        if (16 * n + row < t.rows) {
          float f[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            f[j] = 0.f;
            for (int v = 0; v < 4; ++v) f[j] += joined[v][row][8 * chunk + j];
          }
          float rm = joined_m[0][16 * n + row];
          for (int v = 1; v < 4; ++v) rm = fmaxf(rm, joined_m[v][16 * n + row]);
          const float base = rm == -INFINITY ? 0.f : rm;
          float rl = 0.f;
          for (int v = 0; v < 4; ++v) rl += joined_l[v][16 * n + row] * exp2_fast(joined_m[v][16 * n + row] - base);
          if (splits == 1) {
            const int64_t token = (t.row0 + 16 * n + row) / p.group;
            const int head = h * p.group + static_cast<int>(t.row0 + 16 * n + row - token * p.group);
            const float inv_l = rl != 0.f ? 1.f / rl : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] *= inv_l;
            store8(reinterpret_cast<T*>(p.out.data) + (t.first + token) * p.out.token + head * p.out.head + 8 * chunk,
                   p.out.wide, f);
          } else {
            const int64_t at = unit * kRows + 16 * n + row;
            store8(partial + at * kDim + 8 * chunk, true, f);
            if (chunk == 0) *reinterpret_cast<float2*>(partial_ml + 2 * at) = make_float2(rm, rl);
          }
        }
      }
      __syncthreads();
    }
  }
}

// ---- whole prompts ---------------------------------------------------------------------------------
// One workgroup per tile of 32 kWaves query rows, KV head and share of the positions.  64 positions at
// a time are converted to fp16 once, into LDS (keys as rows, values transposed), and every wave takes
// them for its 32 rows: scores^T [64 x 32] = K Q^T, then out^T [d x 32] += V^T P^T on 32 x 32 x 16
// matrix steps, the weights going from the one to the other in registers.  Weights are one fp16 part
// of 11 bits (2^kPromptLift is the largest; below 2^-24 of that they lose bits), and the softmax's sum
// takes them as rounded, so their rounding has no bias.
constexpr int kPromptLift = 11;   // the running maximum may lag by kPromptSlack: 2^15 fits fp16
constexpr float kPromptSlack = 4.f;
constexpr int kPromptTokens = 64;
constexpr int kListed = 1024;     // groups of 16 positions whose pages and scales are held in LDS

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

__device__ inline f32x16 mfma32(const f16x8& a, const f16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
// Byte kByte of four words as fp16.
template <int kByte> __device__ inline uint2 byte_column_as_f16(const uint32_t (&w)[4]) {
  constexpr uint32_t sel = 0x0c000c04u + 0x00010001u * kByte;  // bytes: kByte of the first, 0, of the second, 0
  return make_uint2(halves(__builtin_amdgcn_perm(w[0], w[1], sel) ^ 0x64806480u),
                    halves(__builtin_amdgcn_perm(w[2], w[3], sel) ^ 0x64806480u));
}
// The larger of x and the other half-wave's x.
__device__ inline float max_of_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int kDim, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void cache_attend_prompt_kernel(CacheAttendParams p, int most_splits,
                                                                            int64_t units, float* partial,
                                                                            float* partial_ml) {
  typedef uint16_t T;
  constexpr int kRows = 32 * kWaves, kThreads = 64 * kWaves;
  constexpr int kSteps = kDim / 16, kOut = kDim / 32;
  constexpr int kPitchK = kDim + 8, kPitchV = kPromptTokens + 8;   // halves
  constexpr int kPieces = kPromptTokens * kDim / 16;                // 16-byte pieces of either branch
  constexpr int kLoads = (kPieces + kThreads - 1) / kThreads;
  struct Group {
    int page;
    float key_scale, exponent, back;
  };
  __shared__ LocateLds locate_lds;
  __shared__ _Float16 keys[2][kPromptTokens][kPitchK];
  __shared__ _Float16 values[2][kDim][kPitchV];
  __shared__ Group groups[kListed];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int r = lane & 31, half = lane >> 5;

  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int h = static_cast<int>(unit % p.cache.heads);
    const int64_t rest = unit / p.cache.heads;
    const int split = static_cast<int>(rest % most_splits);
    Tile t;
    if (!tile_of<kRows, kThreads>(p, rest / most_splits, locate_lds, tid, t)) return;
    const int64_t last_row = t.row0 + t.rows - 1;
    const int64_t held = positions_held(p.cache);
    int64_t seen = t.pos0 + last_row / p.group + 1;
    seen = seen < 0 ? 0 : (seen < held ? seen : held);
    const int64_t blocks = (seen + 31) >> 5;
    const int splits = splits_of(blocks, most_splits);
    if (split >= splits) continue;
    const int begin = static_cast<int>(blocks * split / splits) << 5;
    const int end = static_cast<int>(blocks * (split + 1) / splits) << 5;

    // queries, lifted as in the kernel above; a negative scale turns their sign
    f16x8 q[kSteps];
    float factor;
    int limit, free_until, wave_end;
    {
      const int64_t wave_row = t.row0 + 32 * wave;
      const int64_t wave_last = wave_row + 31 < last_row ? wave_row + 31 : last_row;
      int64_t row = wave_row + r;
      row = row > last_row ? last_row : row;
      const int64_t token = row / p.group;
      const int head = h * p.group + static_cast<int>(row - token * p.group);
      const T* src = reinterpret_cast<const T*>(p.q.data) + (t.first + token) * p.q.token + head * p.q.head + 8 * half;
      float x[kSteps][8];
      float top = 0.f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        load8(src + 16 * s, p.q.wide, x[s]);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[s][j]));
      }
      top = max_of_halves(top);
      int e = (__float_as_uint(top) >> 23) & 255;
      e = e < kLift + 1 ? kLift + 1 : (e > 254 ? 254 : e);
      float lift = __uint_as_float(static_cast<uint32_t>(254 + kLift - e) << 23);
      if (p.scale < 0.f) lift = -lift;
      factor = __uint_as_float(static_cast<uint32_t>(e - kLift) << 23) * (fabsf(p.scale) * kLog2e);
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) q[s][j] = static_cast<_Float16>(x[s][j] * lift);
      const auto position = [&](int64_t row) {
        const int64_t pos = t.pos0 + row / p.group;
        return static_cast<int>(pos < -1 ? -1 : (pos < held ? pos : held));
      };
      limit = position(row);
      free_until = uniform(position(wave_row)) + 1;
      wave_end = wave_row > last_row ? 0 : uniform(position(wave_last)) + 1;
    }

    f32x16 acc[kOut];
#pragma unroll
    for (int c = 0; c < kOut; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
    float m = -INFINITY, l = 0.f;

    for (int chunk = begin; chunk < end; chunk += 16 * kListed) {
      const int chunk_end = chunk + 16 * kListed < end ? chunk + 16 * kListed : end;
      const int tiles = (chunk_end - chunk + kPromptTokens - 1) / kPromptTokens;
      // pages and scales of the chunk's groups; a hole, and what lies past the end, weighs nothing
      for (int i = tid; i < 4 * tiles; i += kThreads) {
        const int pos = chunk + 16 * i;
        Group group{0, 0.f, -INFINITY, 0.f};
        const int page = pos < chunk_end ? page_of(p.cache, t.b, pos) : -1;
        if (page >= 0) {
          const int64_t at = static_cast<int64_t>(page) * p.cache.heads + h;
          float vs = p.cache.v_scale[at];
          vs = vs < 7.8886091e-31f ? 7.8886091e-31f : vs;  // 2^-100: 2^27 positions fit the sum
          group = Group{page, p.cache.k_scale[at], __builtin_amdgcn_logf(vs), 1.f / vs};
        }
        groups[i] = group;
      }
      __syncthreads();

      uint4 kraw[kLoads];
      uint32_t vraw[kLoads][4];
      const auto load = [&](int tile) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int piece = i * kThreads + tid;
          if (kPieces % kThreads != 0 && piece >= kPieces) break;
          const int key = piece / (kDim / 16);
          int page = uniform(groups[4 * tile + uniform(key >> 4)].page);
          const int64_t in_page = (chunk + kPromptTokens * tile + 16 * uniform(key >> 4)) & (p.cache.page - 1);
          const int8_t* src = p.cache.k + page_at(p.cache, page, h, kDim) + in_page * kDim;
          kraw[i] = *reinterpret_cast<const uint4*>(src + (key & 15) * kDim + 16 * (piece % (kDim / 16)));
          const int four = piece / (kDim / 4);  // four positions, four channels
          page = uniform(groups[4 * tile + uniform(four >> 2)].page);
          const int64_t in_page_v = (chunk + kPromptTokens * tile + 16 * uniform(four >> 2)) & (p.cache.page - 1);
          src = p.cache.v + page_at(p.cache, page, h, kDim) + in_page_v * kDim + 4 * (piece % (kDim / 4));
#pragma unroll
          for (int j = 0; j < 4; ++j)
            vraw[i][j] = *reinterpret_cast<const uint32_t*>(src + (4 * (four & 3) + j) * kDim);
        }
      };
      const auto store = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int piece = i * kThreads + tid;
          if (kPieces % kThreads != 0 && piece >= kPieces) break;
          _Float16* dst = &keys[buffer][piece / (kDim / 16)][16 * (piece % (kDim / 16))];
          *reinterpret_cast<f16x8*>(dst) = bytes_as_f16(kraw[i].x, kraw[i].y);
          *reinterpret_cast<f16x8*>(dst + 8) = bytes_as_f16(kraw[i].z, kraw[i].w);
          // positions 16t + 8a + 4b + (0..3) stand at 16t + 8b + 4a: the order of the score registers
          const int four = piece / (kDim / 4), c = 4 * (piece % (kDim / 4));
          const int at = 16 * (four >> 2) + 8 * (four & 1) + 4 * ((four >> 1) & 1);
          *reinterpret_cast<uint2*>(&values[buffer][c][at]) = byte_column_as_f16<0>(vraw[i]);
          *reinterpret_cast<uint2*>(&values[buffer][c + 1][at]) = byte_column_as_f16<1>(vraw[i]);
          *reinterpret_cast<uint2*>(&values[buffer][c + 2][at]) = byte_column_as_f16<2>(vraw[i]);
          *reinterpret_cast<uint2*>(&values[buffer][c + 3][at]) = byte_column_as_f16<3>(vraw[i]);
        }
      };

      load(0);
      store(0);
      if (tiles > 1) load(1);
      __syncthreads();
      for (int tile = 0; tile < tiles; ++tile) {
        const int buffer = tile & 1, at = chunk + kPromptTokens * tile;
        if (tile + 1 < tiles) store(buffer ^ 1);
        if (tile + 2 < tiles) load(tile + 2);
        if (at < wave_end) {
          f32x16 score[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int j = 0; j < 16; ++j) score[i][j] = 0.f;
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
              score[i] = mfma32(*reinterpret_cast<const f16x8*>(&keys[buffer][32 * i + r][16 * s + 8 * half]), q[s], score[i]);
          }
          float f[4], exponent[4], back[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const Group group = groups[4 * tile + i];
            f[i] = group.key_scale * factor;
            exponent[i] = group.exponent;
            back[i] = group.back;
          }
          const bool masked = at + kPromptTokens > free_until;
          if (masked) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (at + 32 * i + 8 * (j >> 2) + 4 * half + (j & 3) > limit) score[i][j] = -INFINITY;
          }
          float top = -INFINITY;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float best = score[i >> 1][8 * (i & 1)];
#pragma unroll
            for (int j = 1; j < 8; ++j) best = fmaxf(best, score[i >> 1][8 * (i & 1) + j]);
            if (best > -INFINITY) top = fmaxf(top, fmaf(best, f[i], exponent[i]));
          }
          top = max_of_halves(top);
          if (__any(top > m + kPromptSlack)) {
            const float now = fmaxf(m, top);
            const float fade = exp2_fast(m - (now == -INFINITY ? 0.f : now));
            m = now;
            l *= fade;
#pragma unroll
            for (int c = 0; c < kOut; ++c)
#pragma unroll
              for (int i = 0; i < 16; ++i) acc[c][i] *= fade;
          }
          const float base = (m == -INFINITY ? 0.f : m) - kPromptLift;
          f16x8 w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float offset = exponent[i] - base;
            float sum = 0.f;
            u32x4 packed;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float e[2];
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const float s = score[i >> 1][8 * (i & 1) + 2 * j + k];
                e[k] = exp2_fast(fmaf(s, f[i], offset));
                if (masked && s == -INFINITY) e[k] = 0.f;
              }
              const auto pair = __builtin_amdgcn_cvt_pkrtz(e[0], e[1]);
              packed[j] = __builtin_bit_cast(uint32_t, pair);
              sum = __builtin_amdgcn_fdot2(pair, decltype(pair){1, 1}, sum, false);
            }
            w[i] = __builtin_bit_cast(f16x8, packed);
            if (sum != 0.f) l = fmaf(sum, back[i], l);
          }
#pragma unroll
          for (int c = 0; c < kOut; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              acc[c] = mfma32(*reinterpret_cast<const f16x8*>(&values[buffer][32 * c + r][16 * i + 8 * half]), w[i], acc[c]);
        }
        __syncthreads();
      }
    }

    l += __shfl_xor(l, 32);
    const int64_t row = t.row0 + 32 * wave + r;
    if (row <= last_row) {
      if (splits == 1) {
        const int64_t token = row / p.group;
        const int head = h * p.group + static_cast<int>(row - token * p.group);
        T* dst = reinterpret_cast<T*>(p.out.data) + (t.first + token) * p.out.token + head * p.out.head;
        const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
        for (int c = 0; c < kOut; ++c)
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const int at = 32 * c + 8 * a + 4 * half;
            const uint2 v = make_uint2(pack_bf16x2(acc[c][4 * a] * inv, acc[c][4 * a + 1] * inv),
                                       pack_bf16x2(acc[c][4 * a + 2] * inv, acc[c][4 * a + 3] * inv));
            if (p.out.wide) {
              *reinterpret_cast<uint2*>(dst + at) = v;
            } else {
              dst[at] = static_cast<uint16_t>(v.x);
              dst[at + 1] = static_cast<uint16_t>(v.x >> 16);
              dst[at + 2] = static_cast<uint16_t>(v.y);
              dst[at + 3] = static_cast<uint16_t>(v.y >> 16);
            }
          }
      } else {
        const int64_t at = unit * kRows + 32 * wave + r;
#pragma unroll
        for (int c = 0; c < kOut; ++c)
#pragma unroll
          for (int a = 0; a < 4; ++a)
            *reinterpret_cast<float4*>(partial + at * kDim + 32 * c + 8 * a + 4 * half) =
                make_float4(acc[c][4 * a], acc[c][4 * a + 1], acc[c][4 * a + 2], acc[c][4 * a + 3]);
        if (half == 0) *reinterpret_cast<float2*>(partial_ml + 2 * at) = make_float2(m, l);
      }
    }
  }
}

// Joins the shares of every row that was split: one workgroup per row, its threads over channels
// (four each) and shares.
template <typename T, int kDim, int kRows>
__global__ __launch_bounds__(256) void cache_attend_join_kernel(CacheAttendParams p, int most_splits,
                                                               int64_t units, const float* partial,
                                                               const float* partial_ml) {
  constexpr int kLanes = kDim / 4, kShares = 256 / kLanes;
  __shared__ LocateLds locate_lds;
  __shared__ float4 sums[kShares][kLanes];
  __shared__ float tops[kShares], totals[kShares];
  const int tid = threadIdx.x, c = tid % kLanes, share = tid / kLanes;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int row = static_cast<int>(unit % kRows);
    const int h = static_cast<int>(unit / kRows % p.cache.heads);
    const int64_t index = unit / kRows / p.cache.heads;
    Tile t;
    if (!tile_of<kRows>(p, index, locate_lds, tid, t)) return;
    if (row >= t.rows) continue;
    int64_t seen = t.pos0 + (t.row0 + t.rows - 1) / p.group + 1;
    const int64_t held = positions_held(p.cache);
    seen = seen < 0 ? 0 : (seen < held ? seen : held);
    const int splits = splits_of((seen + 31) >> 5, most_splits);
    if (splits == 1) continue;
    const int64_t first = (index * most_splits * p.cache.heads + h) * kRows + row;
    const int64_t step = static_cast<int64_t>(p.cache.heads) * kRows;
    float top = -INFINITY, total = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = share; s < splits; s += kShares) {
      const int64_t at = first + s * step;
      const float2 ml = *reinterpret_cast<const float2*>(partial_ml + 2 * at);
      const float4 x = *reinterpret_cast<const float4*>(partial + at * kDim + 4 * c);
      const float now = fmaxf(top, ml.x), base = now == -INFINITY ? 0.f : now;
      const float fade = exp2_fast(top - base), w = exp2_fast(ml.x - base);
      top = now;
      total = total * fade + ml.y * w;
      sum.x = sum.x * fade + x.x * w;
      sum.y = sum.y * fade + x.y * w;
      sum.z = sum.z * fade + x.z * w;
      sum.w = sum.w * fade + x.w * w;
    }
    sums[share][c] = sum;
    if (c == 0) {
      tops[share] = top;
      totals[share] = total;
    }
    __syncthreads();
    if (share == 0) {
      float all = tops[0];
      for (int s = 1; s < kShares; ++s) all = fmaxf(all, tops[s]);
      const float base = all == -INFINITY ? 0.f : all;
      float f[4] = {0.f, 0.f, 0.f, 0.f}, l = 0.f;
      for (int s = 0; s < kShares; ++s) {
        const float w = exp2_fast(tops[s] - base);
        l += totals[s] * w;
        f[0] += sums[s][c].x * w;
        f[1] += sums[s][c].y * w;
        f[2] += sums[s][c].z * w;
        f[3] += sums[s][c].w * w;
      }
      const int64_t token = (t.row0 + row) / p.group;
      const int head = h * p.group + static_cast<int>(t.row0 + row - token * p.group);
      T* dst = reinterpret_cast<T*>(p.out.data) + (t.first + token) * p.out.token + head * p.out.head + 4 * c;
      const float inv = l != 0.f ? 1.f / l : 0.f;
      for (int j = 0; j < 4; ++j) store1(dst + j, f[j] * inv);
    }
    __syncthreads();
  }
}

// How a call is laid out over workgroups, from its arguments alone.
struct AttendPlan {
  int rows;          // query rows of a tile
  int splits;        // most shares of a tile
  int64_t tiles;     // bound
};
constexpr int kPromptWaves = 8, kPromptRows = 32 * kPromptWaves;
static AttendPlan attend_plan(const PagedCache& c, const SeqBatch& b, int group, int head_dim, bool bf16) {
  AttendPlan plan;
  const int64_t requests = b.n_seqs < b.n_tokens ? b.n_seqs : b.n_tokens;
  const int64_t mean = b.n_tokens * group / requests;  // rows of a request and KV head
  const bool prompt = bf16 && head_dim >= 64 && mean >= kPromptRows;
  plan.rows = prompt ? kPromptRows : mean <= 16 ? 16 : (mean <= 32 || !bf16) ? 32 : 64;
  plan.tiles = tiles_bound(b.n_tokens, b.n_seqs, group, plan.rows);
  const int64_t most = (static_cast<int64_t>(c.cols) * c.page + 255) / 256;
  const int64_t target = prompt ? 256 : 2048;
  const int64_t want = (target + plan.tiles * c.heads - 1) / (plan.tiles * c.heads);
  plan.splits = static_cast<int>(want < most ? want : most);
  return plan;
}

size_t attend_workspace(const PagedCache& c, const SeqBatch& b, int group, int head_dim) {
  size_t most = 0;
  for (int bf16 = 0; bf16 < 2; ++bf16) {
    const AttendPlan plan = attend_plan(c, b, group, head_dim, bf16 != 0);
    if (plan.splits == 1) continue;
    const size_t rows = static_cast<size_t>(plan.tiles * c.heads * plan.splits) * plan.rows;
    most = std::max(most, rows * (head_dim + 2) * sizeof(float));
  }
  return most;
}

template <typename T, int kDim, int kRows>
static hipError_t launch_tiles_as(const AttendPlan& plan, const CacheAttendParams& p, float* workspace,
                                  hipStream_t stream) {
  const int64_t units = plan.tiles * p.cache.heads * plan.splits;
  float* ml = workspace + units * kRows * kDim;
  const auto grid = [](int64_t n) { return dim3(static_cast<unsigned>(n < kMaxGrid / 2 ? n : kMaxGrid / 2)); };
  if constexpr (kRows == kPromptRows)
    hipLaunchKernelGGL((cache_attend_prompt_kernel<kDim, kPromptWaves>), grid(units), dim3(64 * kPromptWaves), 0,
                       stream, p, plan.splits, units, workspace, ml);
  else
    hipLaunchKernelGGL((cache_attend_rows_kernel<T, kDim, kRows / 16>), grid(units), dim3(256), 0, stream, p,
                       plan.splits, units, workspace, ml);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.splits == 1) return e;
  const int64_t rows = plan.tiles * p.cache.heads * kRows;
  hipLaunchKernelGGL((cache_attend_join_kernel<T, kDim, kRows>), grid(rows), dim3(256), 0, stream, p, plan.splits,
                     rows, workspace, ml);
  return hipGetLastError();
}

template <typename T, int kDim>
static hipError_t launch_attend_as(const CacheAttendParams& p, float* workspace, hipStream_t stream) {
  const AttendPlan plan = attend_plan(p.cache, p.batch, p.group, kDim, sizeof(T) == 2);
  if constexpr (sizeof(T) == 2 && kDim >= 64)
    if (plan.rows == kPromptRows) return launch_tiles_as<T, kDim, kPromptRows>(plan, p, workspace, stream);
  if constexpr (sizeof(T) == 2)
    if (plan.rows == 64) return launch_tiles_as<T, kDim, 64>(plan, p, workspace, stream);
  if (plan.rows == 32) return launch_tiles_as<T, kDim, 32>(plan, p, workspace, stream);
  return launch_tiles_as<T, kDim, 16>(plan, p, workspace, stream);
}

hipError_t launch_cache_attend(bool bf16, int head_dim, const CacheAttendParams& p, void* workspace,
                               hipStream_t stream) {
  float* ws = static_cast<float*>(workspace);
  if (bf16)
    return head_dim == 128 ? launch_attend_as<uint16_t, 128>(p, ws, stream)
           : head_dim == 64 ? launch_attend_as<uint16_t, 64>(p, ws, stream)
                            : launch_attend_as<uint16_t, 32>(p, ws, stream);
  return head_dim == 128 ? launch_attend_as<float, 128>(p, ws, stream)
         : head_dim == 64 ? launch_attend_as<float, 64>(p, ws, stream)
                          : launch_attend_as<float, 32>(p, ws, stream);
}

}  // namespace scd
