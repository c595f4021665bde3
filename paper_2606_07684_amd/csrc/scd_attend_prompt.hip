// Attention of whole prompts over the paged 8-bit cache (gfx950).
#include "scd_attend.h"

namespace scd {
using namespace dev;

// Rows of one tile: query rows (token, head of the group) of one request and KV head.
struct Tile {
  int b;
  int64_t row0;      // first row, in the request
  int rows;          // rows of the tile that exist
  int64_t first;     // packed row of the request's first token
  int64_t pos0;
};

template <int kRows>
__device__ inline void set_tile(const CacheAttendParams& p, const Span& span, int b, int64_t index, Tile& t) {
  t.b = b;
  t.row0 = index * kRows;
  const int64_t left = (span.end - span.begin) * p.group - t.row0;
  t.rows = static_cast<int>(left < kRows ? left : kRows);
  t.first = span.begin;
  t.pos0 = span.pos0;
}
// Tiles of kRows rows of all requests, one after another.
template <int kRows>
__device__ inline int64_t tiles_in(const CacheAttendParams& p, const Span& s) {
  return ((s.end - s.begin) * p.group + kRows - 1) / kRows;
}
template <int kRows, int kThreads>
__device__ inline bool tile_of(const CacheAttendParams& p, int64_t index, LocateLds& lds, int tid, Tile& t) {
  Located at;
  if (!locate<kThreads>(p.batch, index, lds, tid, [&](const Span& s) { return tiles_in<kRows>(p, s); }, at))
    return false;
  set_tile<kRows>(p, at.span, at.b, at.local, t);
  return true;
}
// Shares of a tile that has `blocks` blocks of 32 positions, when a launch has up to `most`: one for every eight blocks
// begun, equal to a block (nine make two shares, of four and five).
__device__ inline int splits_of(int64_t blocks, int most) {
  const int64_t n = (blocks + 7) / 8;
  return static_cast<int>(n < 1 ? 1 : (n < most ? n : most));
}

// One workgroup per tile of 32 kWaves query rows, KV head and share of the positions.  64 positions at
// a time are converted to fp16 once, into LDS (keys as rows, values transposed), and every wave takes
// them for its 32 rows: scores^T [64 x 32] = K Q^T, then out^T [d x 32] += V^T P^T on 32 x 32 x 16
// matrix steps, the weights going from the one to the other in registers.  The softmax's sum is
// fp32.  The values take their weights as one fp16 part: 11 bits, rounded to the nearest, which is finer than the
// output's own 8 and needs one matrix step; 2^kPromptLift is the largest, and below 2^-25 of that a weight
// (times its value scale, so what it can add to the output) loses bits.
//
// Bound by the vector units beside the matrix cores: per 64 positions a SIMD's two waves take 2048 cycles of matrix
// steps, about 3000 of exponentials, conversions and maxima, and the CU's LDS 2600 of reads and stores; taking turns
// they need 5100.  2048 rows of an 8192-token prompt, 32 heads over 8 of 128, take 277 to 294 us: 817 to 868
// TFLOP/s, where a library product of 8192^3 reaches 1175.
constexpr int kPromptLift = 11;   // the running maximum may lag by kPromptSlack: 2^15 fits fp16
constexpr float kPromptSlack = 4.f;
// The softmax's sum of a chunk is taken of the weights that the values take, divided by the value scales, where these are
// less than 2^kAlike apart (and from the loudest page of earlier chunks): a position that fp32's range leaves out is then
// below 2^-57 of the heaviest.  Otherwise, and where a scale is 0, the sum is of exponentials of its own.
constexpr float kAlike = 40.f;
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
template <int kDim, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void cache_attend_prompt_kernel(CacheAttendParams p, int most_splits,
                                                                            int64_t tiles, float* partial,
                                                                            float* partial_sum) {
  typedef uint16_t T;
  constexpr int kRows = 32 * kWaves, kThreads = 64 * kWaves;
  constexpr int kSteps = kDim / 16, kOut = kDim / 32;
  constexpr int kPitchK = kDim + 8, kPitchV = kPromptTokens + 8;   // halves
  constexpr int kPieces = kPromptTokens * kDim / 16;                // 16-byte pieces of either branch
  constexpr int kLoads = (kPieces + kThreads - 1) / kThreads;
  __shared__ LocateLds locate_lds;
  __shared__ _Float16 keys[2][kPromptTokens][kPitchK];
  __shared__ _Float16 values[2][kDim][kPitchV];
  __shared__ float4 scales[kListed];   // of keys; log2 of that of values, the loudest over it; 0, or -inf for a hole
  __shared__ float2 range[kWaves];
  __shared__ int64_t places[kListed];  // byte of a group's first position, in either branch's pages
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int r = lane & 31, half = lane >> 5;

  const int64_t units = tiles * p.cache.heads * most_splits;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int h = static_cast<int>(unit % p.cache.heads);
    const int64_t rest = unit / p.cache.heads;
    const int split = static_cast<int>(rest % most_splits);
    Tile t;
    // the last tiles, which see the most positions, first
    if (!tile_of<kRows, kThreads>(p, tiles - 1 - rest / most_splits, locate_lds, tid, t)) continue;
    const int64_t last_row = t.row0 + t.rows - 1;
    const int64_t held = positions_held(p.cache);
    int64_t seen = t.pos0 + last_row / p.group + 1;
    seen = seen < 0 ? 0 : (seen < held ? seen : held);
    const int64_t blocks = (seen + 31) >> 5;
    const int splits = splits_of(blocks, most_splits);
    if (split >= splits) continue;
    const int begin = static_cast<int>(blocks * split / splits) << 5;
    const int end = static_cast<int>(blocks * (split + 1) / splits) << 5;

    // queries, lifted so that the largest element is 2^kLift; a negative scale turns their sign
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
    float m = -INFINITY;           // base of the weights: log2 of a weight times its value scale
    float n = -INFINITY, l = 0.f;  // the softmax's sum, l 2^n, but for the present chunk's
    float l_even = 0.f;            // that of the present chunk, l_even 2^(m - loudest), if its pages are alike

    for (int chunk = begin, chunk_end; chunk < end; chunk = chunk_end) {
      chunk_end = end - chunk < 16 * kListed ? end : chunk + 16 * kListed;  // no further: end may be close to 2^31
      const int tiles = (chunk_end - chunk + kPromptTokens - 1) / kPromptTokens;
      // Pages and scales of the chunk's groups; a hole, and what lies past the end, weighs nothing.  Nor do values of a
      // scale of 0 (the least other one is 2^-126), which still have their part in the sum.
      float least = INFINITY, most = -INFINITY;
      for (int i = tid; i < 4 * tiles; i += kThreads) {
        const int pos = chunk + 16 * i;
        float4 scale = make_float4(0.f, -INFINITY, 0.f, -INFINITY);
        int page = pos < chunk_end && pos < seen ? page_of(p.cache, t.b, pos) : -1;
        if (page >= 0) {
          const int64_t at = static_cast<int64_t>(page) * p.cache.heads + h;
          const float vs = p.cache.v_scale[at];
          scale = make_float4(p.cache.k_scale[at], vs < 1.17549435e-38f ? -INFINITY : __builtin_amdgcn_logf(vs), 0.f, 0.f);
          least = scale.y > -INFINITY ? fminf(least, scale.y) : -INFINITY;  // also where it is not a number
          most = fmaxf(most, scale.y);
        } else {
          page = 0;
        }
        scales[i] = scale;
        places[i] = page_at(p.cache, page, h, kDim) + (pos & (p.cache.page - 1)) * kDim;
      }
      least = -max_of_wave(-least);
      most = max_of_wave(most);
      if (lane == 0) range[wave] = make_float2(least, most);
      __syncthreads();
      for (int i = 0; i < kWaves; ++i) {
        least = fminf(least, range[i].x);
        most = fmaxf(most, range[i].y);
      }
      const float loudest = uniform(most);
      const bool alike = loudest - uniform(least) < kAlike;
      for (int i = tid; i < 4 * tiles; i += kThreads)
        if (alike && scales[i].w == 0.f) scales[i].z = exp2_fast(loudest - scales[i].y);
      __syncthreads();
      // and rows whose weights have the base of an earlier chunk's far louder pages
      const bool even = alike && !__any(m - n - loudest > kAlike);

      // Raw bytes on their way to LDS: keys of one tile, values of the one before it.
      uint4 kraw[kLoads];
      uint32_t vraw[kLoads][4];
      // A thread's pieces of either branch lie in the same groups of 16 positions.
      int64_t place[kLoads], place_after[kLoads];  // of the tiles that values and keys are fetched of next
      const auto find = [&](int tile) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          place[i] = place_after[i];
          const int group = 4 * tile + (i * kThreads + tid) / kDim;
          place_after[i] = places[group < 4 * tiles ? group : 0];
        }
      };
      const auto load_keys = [&] {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int piece = i * kThreads + tid;
          if (kPieces % kThreads != 0 && piece >= kPieces) break;
          const int8_t* src = p.cache.k + place_after[i] + (piece / (kDim / 16) & 15) * kDim + 16 * (piece % (kDim / 16));
          kraw[i] = *reinterpret_cast<const uint4*>(src);
        }
      };
      const auto load_values = [&] {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int piece = i * kThreads + tid;
          if (kPieces % kThreads != 0 && piece >= kPieces) break;
          const int four = piece / (kDim / 4);  // four positions, four channels
          const int8_t* src = p.cache.v + place[i] + 4 * (four & 3) * kDim + 4 * (piece % (kDim / 4));
#pragma unroll
          for (int j = 0; j < 4; ++j) vraw[i][j] = *reinterpret_cast<const uint32_t*>(src + j * kDim);
        }
      };
      const auto store_keys = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int piece = i * kThreads + tid;
          if (kPieces % kThreads != 0 && piece >= kPieces) break;
          _Float16* dst = &keys[buffer][piece / (kDim / 16)][16 * (piece % (kDim / 16))];
          *reinterpret_cast<f16x8*>(dst) = bytes_as_f16(kraw[i].x, kraw[i].y);
          *reinterpret_cast<f16x8*>(dst + 8) = bytes_as_f16(kraw[i].z, kraw[i].w);
        }
      };
      const auto store_values = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int piece = i * kThreads + tid;
          if (kPieces % kThreads != 0 && piece >= kPieces) break;
          // Positions 16t + 8a + 4b + (0..3) stand at 16t + 8b + 4a, the order of the score registers, and
          // channel c's pieces of 8 are exchanged by bits of c, so that the 32 lanes of a store, four channels
          // apart, reach all banks.
          const int four = piece / (kDim / 4), c = 4 * (piece % (kDim / 4));
          const int eight = (2 * (four >> 2) + (four & 1)) ^ (c >> 4 & 7), at = 8 * eight + 4 * ((four >> 1) & 1);
          *reinterpret_cast<uint2*>(&values[buffer][c][at]) = byte_column_as_f16<0>(vraw[i]);
          *reinterpret_cast<uint2*>(&values[buffer][c + 1][at]) = byte_column_as_f16<1>(vraw[i]);
          *reinterpret_cast<uint2*>(&values[buffer][c + 2][at]) = byte_column_as_f16<2>(vraw[i]);
          *reinterpret_cast<uint2*>(&values[buffer][c + 3][at]) = byte_column_as_f16<3>(vraw[i]);
        }
      };
      const auto stage = [&](int tile) {
        if (tile + 1 < tiles) store_keys((tile + 1) & 1);
        if (tile < tiles) store_values(tile & 1);
        if (tile + 2 < tiles) load_keys();
        if (tile + 1 < tiles) load_values();
        find(tile + 3);
      };

      f32x16 score[2];
      f16x8 w[4];
      const auto live = [&](int tile) { return chunk + kPromptTokens * tile < wave_end; };
      // Operands are read kReads matrix steps before the one that takes them, in this order: left to itself
      // the compiler keeps one or two and waits for LDS at every step.
      constexpr int kReads = 4;
      const auto steps = [&](auto count, auto operand, auto step) {
        constexpr int kCount = decltype(count)::value;
        f16x8 a[kReads];
#pragma unroll
        for (int i = 0; i < kReads; ++i) a[i] = operand(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
          step(i, a[i % kReads]);
          if (i + kReads < kCount) a[i % kReads] = operand(i + kReads);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      const auto products = [&](int tile) {
        if (tile > 0 && live(tile - 1)) {
          const _Float16* rows = values[(tile - 1) & 1][r];
          const auto operand = [&](int i) {  // of channel 32c + r, its piece 2t + half
            const int c = i % kOut, eight = (2 * (i / kOut) + half) ^ ((2 * c + (r >> 4)) & 7);
            return *reinterpret_cast<const f16x8*>(rows + 32 * c * kPitchV + 8 * eight);
          };
          steps(IntC<4 * kOut>{}, operand,
                [&](int i, const f16x8& a) { acc[i % kOut] = mfma32(a, w[i / kOut], acc[i % kOut]); });
        }
        if (tile < tiles && live(tile)) {
          const _Float16* rows = &keys[tile & 1][r][8 * half];
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) score[i][j] = 0.f;
          steps(IntC<2 * kSteps>{}, [&](int i) { return *reinterpret_cast<const f16x8*>(rows + 32 * (i % 2) * kPitchK + 16 * (i / 2)); },
                [&](int i, const f16x8& a) { score[i % 2] = mfma32(a, q[i / 2], score[i % 2]); });
        }
      };
      const auto weights = [&](int tile) {
        const int at = chunk + kPromptTokens * tile;
        if (at >= wave_end) return;
        float f[4], exponent[4], back[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 scale = scales[4 * tile + i];
          f[i] = scale.x * factor;
          exponent[i] = scale.y;
          back[i] = scale.z;
        }
        const bool masked = at + kPromptTokens > free_until;
        const auto hide = [&](float with) {
          int shown = limit - at - 4 * half;  // compared with constants, not with a register each
          asm volatile("" : "+v"(shown));     // and only where something is hidden
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (32 * i + 8 * (j >> 2) + (j & 3) > shown) score[i][j] = with;
        };
        if (masked) hide(-INFINITY);
        if (__builtin_expect(!even, 0)) {  // the softmax's sum by exponentials of its own
          float top = n;
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 8 * (i & 1); j < 8 * (i & 1) + 8; ++j)
              if (score[i >> 1][j] > -INFINITY)
                top = fmaxf(top, fmaf(score[i >> 1][j], f[i], scales[4 * tile + i].w));
          if (top > -INFINITY) {
            l *= exp2_fast(n - top);
            n = top;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int j = 8 * (i & 1); j < 8 * (i & 1) + 8; ++j)
                if (score[i >> 1][j] > -INFINITY)
                  l += exp2_fast(fmaf(score[i >> 1][j], f[i], scales[4 * tile + i].w) - n);
          }
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
          l_even *= fade;
#pragma unroll
          for (int c = 0; c < kOut; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[c][i] *= fade;
        }
        const float base = (m == -INFINITY ? 0.f : m) - kPromptLift;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float offset = exponent[i] - base;
#pragma unroll
          for (int j = 8 * (i & 1); j < 8 * (i & 1) + 8; ++j) score[i >> 1][j] = exp2_fast(fmaf(score[i >> 1][j], f[i], offset));
        }
        if (masked) hide(0.f);  // whatever the scale: one that is not a number stays with the rows that see it
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float sum = 0.f;
          u32x4 packed;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float a = score[i >> 1][8 * (i & 1) + 2 * j], b = score[i >> 1][8 * (i & 1) + 2 * j + 1];
            packed[j] = __builtin_bit_cast(uint32_t, f16x2{static_cast<_Float16>(a), static_cast<_Float16>(b)});
            sum += a + b;
          }
          w[i] = __builtin_bit_cast(f16x8, packed);
          if (sum != 0.f) l_even = fmaf(sum, back[i], l_even);
        }
      };

      // The waves of a SIMD, one of either half of the workgroup, take turns: while one keeps the matrix cores
      // busy the other works on its weights and stages bytes.  Between two barriers, in slots 2j and 2j + 1,
      // the first and the second half read the keys of tile j and the values of tile j - 1, and the keys of
      // tile j + 1 and the values of tile j are stored to the other buffers.
      const auto slot_end = [] {
        __builtin_amdgcn_sched_barrier(0);
        lds_barrier();
        __builtin_amdgcn_sched_barrier(0);
      };
      find(0);
      find(0);
      load_keys();
      store_keys(0);
      find(1);
      if (tiles > 1) load_keys();
      load_values();
      find(2);
      lds_barrier();
      const bool second = wave >= kWaves / 2;
      if (second) {
        stage(0);
        slot_end();
      }
      for (int tile = 0; tile <= tiles; ++tile) {
        __builtin_amdgcn_s_setprio(1);
        products(tile);
        __builtin_amdgcn_s_setprio(0);
        slot_end();
        if (tile < tiles) weights(tile);
        stage(second ? tile + 1 : tile);
        slot_end();
      }
      if (!second) slot_end();
      if (even && l_even != 0.f) {
        const float alone = m - loudest, now = fmaxf(n, alone);
        l = l * exp2_fast(n - now) + l_even * (1.f / (1 << kPromptLift)) * exp2_fast(alone - now);
        n = now;
      }
      l_even = 0.f;
      __syncthreads();
    }

    // out = acc 2^(m - n - kPromptLift) / l, in two steps as the power may be out of range
    const float both = max_of_halves(n);
    if (both > -INFINITY) l *= exp2_fast(n - both);
    l += __shfl_xor(l, 32);
    const float power = both > -INFINITY ? exp2_fast(0.5f * (m - both - kPromptLift)) : 0.f;
    const float inv = l != 0.f ? power / l : 0.f;
#pragma unroll
    for (int c = 0; c < kOut; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[c][i] = acc[c][i] * inv * power;
    const int64_t row = t.row0 + 32 * wave + r;
    if (row <= last_row) {
      if (splits == 1) {
        const int64_t token = row / p.group;
        const int head = h * p.group + static_cast<int>(row - token * p.group);
        T* dst = reinterpret_cast<T*>(p.out.data) + (t.first + token) * p.out.token + head * p.out.head;
#pragma unroll
        for (int c = 0; c < kOut; ++c)
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const int at = 32 * c + 8 * a + 4 * half;
            const uint2 v = make_uint2(pack_bf16x2(acc[c][4 * a], acc[c][4 * a + 1]),
                                       pack_bf16x2(acc[c][4 * a + 2], acc[c][4 * a + 3]));
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
        if (half == 0) *reinterpret_cast<float2*>(partial_sum + 2 * at) = part_sum(both, l);
      }
    }
  }
}

// Joins the shares of the tiles that were split: one workgroup per 16 rows, four channels a thread, eight shares
// on their way at once.
template <int kDim>
__global__ __launch_bounds__(256) void cache_attend_join_kernel(CacheAttendParams p, int most_splits, int64_t tiles,
                                                               const float* partial, const float* partial_sum) {
  constexpr int kFours = kDim / 4, kParts = kPromptRows / 16, kBatch = 8;
  __shared__ LocateLds locate_lds;
  __shared__ float2 sums[kMostSplits][16];
  const int tid = threadIdx.x;
  const int64_t units = tiles * p.cache.heads * kParts;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int row0 = static_cast<int>(unit % kParts) * 16;
    const int h = static_cast<int>(unit / kParts % p.cache.heads);
    const int64_t index = unit / kParts / p.cache.heads;
    Tile t;
    if (!tile_of<kPromptRows, 256>(p, index, locate_lds, tid, t)) return;
    if (row0 >= t.rows) continue;
    const int splits = splits_of(blocks_to(positions_held(p.cache), static_cast<int>(t.pos0),
                                           p.by_group.of(static_cast<int>(t.row0) + t.rows - 1)), most_splits);
    if (splits == 1) continue;
    const int64_t first = ((tiles - 1 - index) * most_splits * p.cache.heads + h) * kPromptRows + row0;
    const int64_t step = static_cast<int64_t>(p.cache.heads) * kPromptRows;
    const int rows = t.rows - row0 < 16 ? t.rows - row0 : 16;
    for (int i = tid; i < splits * 16; i += 256)
      if (i % 16 < rows)
        sums[i / 16][i % 16] = *reinterpret_cast<const float2*>(partial_sum + 2 * (first + i / 16 * step + i % 16));
    __syncthreads();
    for (int item = tid; item < rows * kFours; item += 256) {
      const int row = item / kFours, c = 4 * (item % kFours);
      float top = -INFINITY;
      for (int s = 0; s < splits; ++s) top = fmaxf(top, sums[s][row].x);
      const float base = join_base(top, kMostSplits);
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};
      float l = 0.f;
      for (int s0 = 0; s0 < splits; s0 += kBatch) {
        f32x4 v[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
          v[k] = *reinterpret_cast<const f32x4*>(partial + (first + (s0 + k < splits ? s0 + k : s0) * step + row) * kDim + c);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          const float2 x = sums[s0 + k < splits ? s0 + k : s0][row];
          const float w = s0 + k < splits ? x.y * exp2_fast(x.x - base) : 0.f;
          l += w;
          sum += v[k] * w;
        }
      }
      const int at = static_cast<int>(t.row0) + row0 + row, token = p.by_group.of(at);
      uint16_t* dst = reinterpret_cast<uint16_t*>(p.out.data) + (t.first + token) * p.out.token +
                      (h * p.group + at - token * p.group) * p.out.head + c;
      const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) store1(dst + j, sum[j] * inv);
    }
    __syncthreads();
  }
}

template <int kDim>
static hipError_t launch_prompt_as(const CacheAttendParams& p, int64_t tiles, int splits, float* workspace,
                                   hipStream_t stream) {
  const int64_t units = tiles * p.cache.heads * splits;
  workspace += kCounterBytes / sizeof(float);  // the counts of the other kernel stay zero
  float* sums = workspace + units * kPromptRows * kDim;
  const auto grid = [](int64_t n) { return dim3(static_cast<unsigned>(n < kMaxGrid / 2 ? n : kMaxGrid / 2)); };
  hipLaunchKernelGGL((cache_attend_prompt_kernel<kDim, kPromptWaves>), grid(units), dim3(64 * kPromptWaves), 0,
                     stream, p, splits, tiles, workspace, sums);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  hipLaunchKernelGGL((cache_attend_join_kernel<kDim>), grid(tiles * p.cache.heads * (kPromptRows / 16)), dim3(256), 0,
                     stream, p, splits, tiles, workspace, sums);
  return hipGetLastError();
}

hipError_t launch_attend_prompt(int head_dim, const CacheAttendParams& p, int64_t tiles, int splits, float* workspace,
                                hipStream_t stream) {
  return head_dim == 128 ? launch_prompt_as<128>(p, tiles, splits, workspace, stream)
                         : launch_prompt_as<64>(p, tiles, splits, workspace, stream);
}

}  // namespace scd
