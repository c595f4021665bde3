// The step that attention over latents and over dense rows share (gfx950): the scores of 16 query rows a
// wave (or two times 16) against a step of positions that lie in LDS, the softmax's running maximum and
// sum, and the weighted sum of the values.
//
//   s_j = q . k_j,  m = max_j s_j,  l = sum_j 2^(s_j - m),  o = sum_j 2^(s_j - m) v_j
//
// in powers of two: q or the scores carry log2(e).  Scores are formed transposed, positions as matrix rows
// and query rows as columns, so that a lane's scores belong to one query row and are, as they stand, the
// right operand of the second product: weights never leave the registers.  That product's contraction runs
// over the positions in the order the lanes hold them, which the transposing LDS reads of the values follow.
#pragma once

#include "scd_serve_device.h"
#include "scd_latent.h"

namespace scd {
namespace dev {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4_t;

// kStep positions a wave takes at once, kVec channels of a 16-byte piece.
template <typename T> struct Elem;
template <> struct Elem<uint16_t> {
  static constexpr int kStep = 32, kVec = 8;
  typedef bf16x8 Frag;
};
template <> struct Elem<float> {
  static constexpr int kStep = 16, kVec = 4;
  typedef f32x4 Frag;
};

__device__ inline f32x4 mma(const bf16x8& a, const bf16x8& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// 16 channels: contraction step j takes channel 4 g + j of lane group g.
__device__ inline f32x4 mma(const f32x4& a, const f32x4& b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// kCount tiles of 16 value channels, transposed on the way out of LDS: half 0 of tile c holds, of the lane's channel,
// the positions 4 g .. 4 g + 3 and half 1 the same 16 positions on, kHalf bytes behind.  The reads and the wait for
// them are one piece of assembly: the compiler takes a transposing read for one that waits for every copy under way
// into LDS, which would empty the ring of blocks at every step.
template <int kFirst, int kHalf>
__device__ inline void read_values4(uint32_t at, s16x4 (&h)[8]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8 offset:%9\n\t"
      "ds_read_b64_tr_b16 %1, %8 offset:%10\n\t"
      "ds_read_b64_tr_b16 %2, %8 offset:%11\n\t"
      "ds_read_b64_tr_b16 %3, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %4, %8 offset:%13\n\t"
      "ds_read_b64_tr_b16 %5, %8 offset:%14\n\t"
      "ds_read_b64_tr_b16 %6, %8 offset:%15\n\t"
      "ds_read_b64_tr_b16 %7, %8 offset:%16\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(h[0]), "=&v"(h[1]), "=&v"(h[2]), "=&v"(h[3]), "=&v"(h[4]), "=&v"(h[5]), "=&v"(h[6]), "=&v"(h[7])
      : "v"(at), "n"(kFirst), "n"(kFirst + kHalf), "n"(kFirst + 32), "n"(kFirst + 32 + kHalf), "n"(kFirst + 64),
        "n"(kFirst + 64 + kHalf), "n"(kFirst + 96), "n"(kFirst + 96 + kHalf)
      : "memory");
}

// Between matrix instructions and, behind a branch, the first use of their results: the compiler inserts the wait
// states that such a use needs within a block, but was seen to leave them out across one (the last of 16 results
// was then read a few cycles before it was written).
__device__ inline void settle() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 3" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Two values rounded to bf16 by one instruction.
__device__ inline uint32_t both_bf16(float x, float y) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
}

// Whether one of the 16-byte piece's values is not finite.
__device__ inline bool odd_piece(const uint16_t* p) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad |= (w[i] & 0x7f800000u) == 0x7f800000u || (w[i] & 0x7f80u) == 0x7f80u;
  return bad;
}
__device__ inline bool odd_piece(const float* p) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  return (v.x & 0x7f800000u) == 0x7f800000u || (v.y & 0x7f800000u) == 0x7f800000u ||
         (v.z & 0x7f800000u) == 0x7f800000u || (v.w & 0x7f800000u) == 0x7f800000u;
}

// The largest value of the four lanes that hold a query row's positions (16 lanes apart).
__device__ inline float row_top(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// kFrags pieces of 4 kVec channels that a score contracts, kTiles tiles of 16 value channels, NT tiles of 16
// query rows, the queries' first kLow pieces with a second summand; kKeyRow, kValueRow elements between LDS rows.
template <typename T, int kFrags, int kTiles, int NT, int kLow, int kKeyRow, int kValueRow>
struct AttendCore {
  typedef typename Elem<T>::Frag Frag;
  static constexpr int kStep = Elem<T>::kStep, kVec = Elem<T>::kVec, kSub = kStep / 16;
  // A row's base m follows its largest score once that is ahead by more than this: weights stay below 2^8, and
  // most steps neither compare scores across lanes nor scale what they have.
  static constexpr float kSlack = 8.f;
  // Whether a bf16 call's weight is two bf16 summands, 16 bits.  With one, 8 bits, results are off by what one more
  // rounding to bf16 would add (relative error against 64 bits 2.3e-3 over dense rows, 1.8e-3 to 1.9e-3 over latents;
  // 1.66e-3 with two, which is the result's own rounding).  The second summand is a product more.  In tiles of one 16-row
  // tile a wave its time is hidden behind the memory or small (a token of 64 requests of 8000 positions 368 us either way,
  // 64 rows behind 8000 54 | 55; over latents a token of 16 requests of 1K to 16K 45 | 46, 200 tokens behind 2000 102 |
  // 108).  In prompts' tiles of two it adds all of it (2048 rows behind 6144 320 | 400 us, 512 behind 8000 120 | 139):
  // those round weights once.
  static constexpr bool kRest = NT == 1;

  Frag q[NT][kFrags], low[NT][kLow > 0 ? kLow : 1];
  f32x4 o[NT][kTiles];
  float m[NT], l[NT];  // l: this lane's positions only
  int limit[NT];       // last position the lane's row attends to

  __device__ void clear() {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n] = -INFINITY;
      l[n] = 0.f;
#pragma unroll
      for (int c = 0; c < kTiles; ++c) o[n][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Positions pos .. pos + kStep - 1 at LDS rows k, v; scale >= 0.  kCareful: some row leaves some of them out
  // (behind its limit, or in a hole: bit t of `holes` for positions 16 t on); weights there are zero and values
  // that are not finite do not count.  A value that is not finite makes its channel NaN for the rows that attend
  // to it.  The sum that divides is of the weights themselves, not of their bf16 summands.
  template <bool kCareful>
  __device__ void step(const T* k, const T* v, float scale, int pos, int holes, int lane) {
    const int lr = lane & 15, g = lane >> 4;
    f32x4 s[kSub][NT];
#pragma unroll
    for (int t = 0; t < kSub; ++t)
#pragma unroll
      for (int n = 0; n < NT; ++n) s[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    const T* row = k + lr * kKeyRow + kVec * g;
#pragma unroll
    for (int f = 0; f < kFrags; ++f)
#pragma unroll
      for (int t = 0; t < kSub; ++t) {
        const Frag a = *reinterpret_cast<const Frag*>(row + 16 * t * kKeyRow + 4 * kVec * f);
#pragma unroll
        for (int n = 0; n < NT; ++n) s[t][n] = mma(a, q[n][f], s[t][n]);
        if (f < kLow) {
#pragma unroll
          for (int n = 0; n < NT; ++n) s[t][n] = mma(a, low[n][f < kLow ? f : 0], s[t][n]);
        }
      }
    bool odd = false;
    if constexpr (kCareful) {
      constexpr int kRowPieces = 16 / kVec * kTiles;
      for (int i = lane; i < kStep * kRowPieces; i += 64) {
        const int r = i / kRowPieces, c = i - r * kRowPieces;
        odd |= odd_piece(v + r * kValueRow + kVec * c);
      }
      odd = __any(odd);
    }
    float top[NT];
    bool ahead = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      top[n] = -INFINITY;
#pragma unroll
      for (int t = 0; t < kSub; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!kCareful || seen(n, t, i, pos, holes, g)) top[n] = fmaxf(top[n], s[t][n][i]);
      // where nothing is seen, a scale of 0 must not make it something
      if (!kCareful || top[n] != -INFINITY) top[n] *= scale;
      ahead |= top[n] > m[n] + kSlack;
    }
    if (__any(ahead)) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        // by the row's own scores alone, so that a row's result does not depend on the rows beside it
        const float most = row_top(top[n]), now = most > m[n] + kSlack ? most : m[n];
        const float by = __builtin_amdgcn_exp2f(m[n] - (now == -INFINITY ? 0.f : now));
        m[n] = now;
        l[n] *= by;
#pragma unroll
        for (int c = 0; c < kTiles; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n][c][i] *= by;
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float base = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
      for (int t = 0; t < kSub; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][n][i], scale, -base));
          if constexpr (kCareful) w = seen(n, t, i, pos, holes, g) ? w : 0.f;
          s[t][n][i] = w;
          l[n] += w;
        }
    }
    weigh<kCareful>(v, s, odd, pos, holes, lr, g);
  }

  // The row's sum over the lanes that hold its positions.
  __device__ float sum(int n) const {
    float x = l[n];
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
  }

 private:
  __device__ bool seen(int n, int t, int i, int pos, int holes, int g) const {
    return pos + 16 * t + 4 * g + i <= limit[n] && !(holes >> t & 1);
  }

  // Tiles kTile .. kTile + 3 and those behind them.  odd (of all lanes alike): some value is not finite; such values are
  // taken out and counted beside the product.
  template <int kTile, bool kCareful>
  __device__ void weigh_tiles(uint32_t at, const bf16x8 (&w)[NT], const bf16x8 (&rest)[NT], bool odd, int pos, int holes,
                              int g) {
    if constexpr (kTile < kTiles) {
      union { s16x4 h[8]; bf16x8 v[4]; uint32_t u[16]; } a;
      read_values4<32 * kTile, 32 * kValueRow>(at, a.h);
      if (kCareful && odd) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          union { bf16x8 v; uint32_t u[4]; } flag;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // two values' exponents at once: all ones carry into the bit above them
            const uint32_t top = ((a.u[4 * c + e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
            const uint32_t bad = top | (top - (top >> 15));
            flag.u[e] = bad & 0x3f803f80u;
            a.u[4 * c + e] &= ~bad;
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            asm volatile("" : "+v"(pos));  // formed again for every tile: registers are short
            bf16x8 ones;
#pragma unroll
            for (int e = 0; e < 8; ++e) ones[e] = static_cast<__bf16>(seen(n, e >> 2, e & 3, pos, holes, g) ? 1.f : 0.f);
            const f32x4 x = mma(flag.v, ones, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (x[i] > 0.f) o[n][kTile + c][i] = __builtin_nanf("");
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int n = 0; n < NT; ++n) o[n][kTile + c] = mma(a.v[c], w[n], o[n][kTile + c]);
      if constexpr (kRest) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int n = 0; n < NT; ++n) o[n][kTile + c] = mma(a.v[c], rest[n], o[n][kTile + c]);
      }
      weigh_tiles<kTile + 4, kCareful>(at, w, rest, odd, pos, holes, g);
    }
  }

  template <bool kCareful>
  __device__ void weigh(const T* v, const f32x4 (&s)[kSub][NT], bool odd, int pos, int holes, int lr, int g) {
    if constexpr (sizeof(T) == 2) {
      bf16x8 w[NT], rest[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        union { uint32_t u[4]; bf16x8 v; } high, low;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = s[e >> 1][n][2 * (e & 1)], y = s[e >> 1][n][2 * (e & 1) + 1];
          high.u[e] = both_bf16(x, y);
          if constexpr (kRest) low.u[e] = both_bf16(x - bf16_lo(high.u[e]), y - bf16_hi(high.u[e]));
        }
        w[n] = high.v;
        if constexpr (kRest) rest[n] = low.v;
      }
      const uint32_t at = static_cast<uint32_t>(
          reinterpret_cast<uintptr_t>((lds_s16x4_t)(v + (4 * g + (lr >> 2)) * kValueRow + 4 * (lr & 3))));
      weigh_tiles<0, kCareful>(at, w, rest, odd, pos, holes, g);
    } else if (kCareful && odd) {
      weigh_f32<true>(v, s, pos, holes, lr, g);
    } else {
      weigh_f32<false>(v, s, pos, holes, lr, g);
    }
  }

  template <bool kOdd>
  __device__ void weigh_f32(const T* v, const f32x4 (&s)[kSub][NT], int pos, int holes, int lr, int g) {
    if constexpr (sizeof(T) == 4) {
      const T* at = v + 4 * g * kValueRow + lr;
#pragma unroll
      for (int c = 0; c < kTiles; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float a = at[i * kValueRow + 16 * c];
          if constexpr (kOdd) {
            const bool bad = (__float_as_uint(a) & 0x7f800000u) == 0x7f800000u;
            if (bad) a = 0.f;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const f32x4 x = __builtin_amdgcn_mfma_f32_16x16x4f32(
                  bad ? 1.f : 0.f, seen(n, 0, i, pos, holes, g) ? 1.f : 0.f, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (x[e] > 0.f) o[n][c][e] = __builtin_nanf("");
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n)
            o[n][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, s[0][n][i], o[n][c], 0, 0, 0);
        }
    }
  }
};

// A value that all lanes hold, in a scalar register.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<int>(x));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<int>(x >> 32));
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ inline Span uniform(const Span& s) { return Span{uniform(s.begin), uniform(s.end), uniform(s.pos0)}; }

// 16 bytes a lane from memory into LDS, `to` the wave's first byte.
__device__ inline void copy16(const void* from, char* to) {
  __builtin_amdgcn_global_load_lds(from, (lds_void_t)to, 16, 0, 0);
}

// A lane's 16 bytes at `at` of a region (the same for all lanes) of `bytes` bytes; zeros behind its end.
constexpr int kRegionFlags = 0x00020000;
__device__ inline void copy16(const void* region, int64_t bytes, uint32_t at, char* to) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
      reinterpret_cast<void*>(uniform(reinterpret_cast<int64_t>(region))), 0,
      uniform(static_cast<int>(bytes < 0x7fffffff ? bytes : 0x7fffffff)), kRegionFlags);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t)to, 16, at, 0, 0, 0);
}

// The 64-lane copies that bring a block of kRows rows of `pieces` 16-byte pieces into LDS rows of kPieces, dealt to
// kWaves waves: copy j of a wave fills kilobyte index(wave, j) of the block's region of kBytes bytes.  Every wave
// issues kMine of them, the last ones twice where they do not come out even, so that one count of copies under way
// holds for all; LDS pieces that a row does not have get its last one again.
template <int kRows, int kPieces, int kWaves = 4>
struct Copies {
  static constexpr int kAll = (kRows * kPieces + 63) / 64, kMine = (kAll + kWaves - 1) / kWaves, kBytes = kAll * 1024;
  static __device__ int index(int wave, int j) { return wave + kWaves * j < kAll ? wave + kWaves * j : kAll - 1; }
  static __device__ int row(int wave, int j, int lane) {
    const int r = (index(wave, j) * 64 + lane) / kPieces;
    return r < kRows ? r : kRows - 1;
  }
  static __device__ int piece(int wave, int j, int lane) { return (index(wave, j) * 64 + lane) % kPieces; }
  static __device__ int piece(int wave, int j, int lane, int pieces) {
    const int c = piece(wave, j, lane);
    return c < pieces ? c : pieces - 1;
  }
};

// s_waitcnt vmcnt(n), the other counters left alone.
template <int n>
__device__ inline void wait_copies() {
  static_assert(n >= 0 && n < 64, "counter range");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (n & 15) | (n >> 4) << 14);
}

// ---- shares ------------------------------------------------------------------------------------------
// A request's query rows make tiles, its positions blocks of kBlock.  While there are fewer than plan.whole tiles,
// every tile's positions are cut into shares of at most `chunk` blocks, so that the shares of all
// tiles are no more than the goal, by either of  sum ceil(blocks / chunk) <= sum blocks / chunk + tiles  and
// sum ceil(blocks / chunk) <= tiles ceil(most blocks / chunk):  the first where lengths differ, the second, which cuts
// equal tiles evenly, where they do not (512 rows behind 8000 positions, 32 heads, 256 us by the first alone, 143 so).
struct Share {
  Span span;
  int64_t len;     // positions of the request
  int b, head, tile, tiles, part, parts;
  int64_t first;   // unit of the tile's first share; share s is unit first + s * tiles
};
struct ShareLds {
  int64_t wave[3][16];
  LocateLds found;
};

template <typename Length>
struct Tiles {
  const SharePlan& p;
  Length length;   // positions of request b with this span
  int block;       // a power of two
  __device__ int64_t tiles(const Span& s) const {
    return div_ceil((s.end - s.begin) * p.per_token, p.rows);
  }
  __device__ int64_t blocks(const Span& s, int b) const { return (length(s, b) + block - 1) >> (31 - __builtin_clz(block)); }
};

// The share that workgroup `block` takes; false past the last.  Every thread calls it and gets the answer.
// Shares are dealt to the XCDs in contiguous ranges, of the shares there are (a launch may have more workgroups), so
// that those that read the same rows share an L2 and every XCD gets as many.
template <int kThreads, typename Length>
__device__ inline bool find_share(const SeqBatch& s, const SharePlan& p, int block, int least, int workgroup,
                                  ShareLds& lds, int tid, Length length, Share& out) {
  const Tiles<Length> of{p, length, block};
  // two sums and a maximum over the requests
  const auto all = [&](auto count, int64_t (&total)[3]) {
    total[0] = total[1] = total[2] = 0;
    if (s.n_seqs == 1) {
      count(span_of(s, 0), 0, total);
      return;
    }
    for (int b = tid; b < s.n_seqs; b += kThreads) count(span_of(s, b), b, total);
    for (int o = 32; o > 0; o >>= 1) {
      total[0] += __shfl_xor(total[0], o);
      total[1] += __shfl_xor(total[1], o);
      const int64_t other = __shfl_xor(total[2], o);
      total[2] = other > total[2] ? other : total[2];
    }
    __syncthreads();  // the last sum's readers are done
    if ((tid & 63) == 0)
      for (int i = 0; i < 3; ++i) lds.wave[i][tid >> 6] = total[i];
    __syncthreads();
    total[0] = total[1] = total[2] = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
      total[0] += lds.wave[0][w];
      total[1] += lds.wave[1][w];
      total[2] = lds.wave[2][w] > total[2] ? lds.wave[2][w] : total[2];
    }
  };
  int64_t chunk = int64_t{1} << 40, total[3];
  if (p.cut) {
    // all tiles, all blocks of all tiles, and those of the longest
    all([&](const Span& span, int b, int64_t (&t)[3]) {
      const int64_t n = of.tiles(span), blocks = of.blocks(span, b);
      t[0] += n;
      t[1] += n * blocks;
      t[2] = n > 0 && blocks > t[2] ? blocks : t[2];
    }, total);
    const int64_t tiles = total[0] * p.heads, work = total[1] * p.heads;
    if (tiles > 0 && tiles < p.whole) {
      const int64_t goal = share_goal(tiles, p.fill);
      const int64_t mixed = div_ceil(work, goal - tiles), even = div_ceil(total[2], div_up_to(goal, tiles));
      chunk = mixed < even ? mixed : even;
      chunk = chunk < least ? least : chunk;
    }
  }
  const auto parts_of = [&](const Span& span, int b) {
    const int64_t n = of.blocks(span, b);
    return n <= chunk ? int64_t{1} : div_ceil(n, chunk);
  };
  // heads one after another, each with all requests' shares; every head has as many
  all([&](const Span& span, int b, int64_t (&t)[3]) { t[0] += of.tiles(span) * parts_of(span, b); }, total);
  const int64_t per_head = total[0];
  if (per_head == 0 || workgroup >= per_head * p.heads) return false;
  const int64_t unit = xcd_remap(workgroup, static_cast<int>(per_head * p.heads));
  if (unit >= p.grid) return false;  // more rows than the batch has, by boundaries that fall: the workspace ends here
  out.head = static_cast<int>(div_up_to(unit, per_head));
  const int64_t left = unit - out.head * per_head;
  Located at;
  if (s.n_seqs == 1) {
    at.b = 0;
    at.span = span_of(s, 0);
    at.local = left;
  } else {
    // locate() calls the count once for every request of this thread, in order
    int next = tid;
    const auto count = [&](const Span& span) {
      const int b = next;
      next += kThreads;
      return b < s.n_seqs ? of.tiles(span) * parts_of(span, b) : int64_t{0};
    };
    if (!locate<kThreads>(s, left, lds.found, tid, count, at)) return false;
  }
  out.first = unit - at.local;
  out.b = uniform(at.b);
  out.span = uniform(at.span);
  out.head = uniform(out.head);
  out.first = uniform(out.first);
  const int64_t local = uniform(at.local);
  out.len = length(out.span, out.b);
  out.tiles = static_cast<int>(of.tiles(out.span));
  out.parts = uniform(static_cast<int>(parts_of(out.span, out.b)));
  out.part = static_cast<int>(div_up_to(local, out.tiles));
  out.tile = static_cast<int>(local - static_cast<int64_t>(out.part) * out.tiles);
  out.first += out.tile;
  return true;
}

}  // namespace dev
}  // namespace scd
