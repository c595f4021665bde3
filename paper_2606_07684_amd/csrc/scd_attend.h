// Causal attention of new tokens over the paged 8-bit cache (gfx950): what its two kernels share.
//
// out = sum_j p_j v_j with p the softmax over the cached positions of scale * (q . k_j), in one pass
// with a running maximum and sum: when the maximum grows from m to m', what is summed so far is
// multiplied by e^(m - m').  Both products run on the matrix cores with fp32 accumulation:
//  - cached values are whole numbers of at most 127, exact in fp16 and bf16; a page's key scale
//    multiplies the scores, its value scale the weights, so no value is scaled one by one.
//  - scores in fp16: a query row is multiplied by the power of two that brings its largest element to
//    2^14 (its scores by the inverse).  bf16 rows are then exact down to 2^-28 of that element; fp32
//    rows are split into two parts of 11 bits: what a third would add, 2^-22 of an element and less, is about what the fp32
//    sums of up to 128 products leave open, at half as many matrix steps again for the scores.
//  - a page's value scale goes into the exponent: the running maximum is that of log2 of a position's weight
//    times its value scale, what it can add to the output, so the weights that add most to it have all their bits on the
//    matrix cores whatever the scales; the softmax's own sum takes them divided by the scale again.
#pragma once

#include "scd_serve_device.h"

namespace scd {
namespace dev {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef const __attribute__((address_space(4))) int32_t* uniform_ints_t;
typedef const __attribute__((address_space(4))) float* uniform_floats_t;

constexpr float kLog2e = 1.44269504f;
constexpr int kLift = 14;  // the largest element of a query row is brought to 2^kLift
constexpr int kLeastExponent = -90;  // of a value scale: 2^90 times 2^31 positions fits the sum

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline float uniform(float x) { return __int_as_float(uniform(__float_as_int(x))); }
// The larger of x and the other half-wave's x.
__device__ inline float max_of_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// The largest of x over the lanes of the same place in every 16.
__device__ inline float max_of_quarters(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_of_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
// The largest of x over the wave.
__device__ inline float max_of_wave(float x) {
  const auto moved = [&](auto how) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), decltype(how)::value, 15, 15, false));
  };
  x = fmaxf(x, moved(IntC<0xb1>{}));   // lanes exchanged in pairs,
  x = fmaxf(x, moved(IntC<0x4e>{}));   // pairs in fours,
  x = fmaxf(x, moved(IntC<0x141>{}));  // eights mirrored,
  x = fmaxf(x, moved(IntC<0x140>{}));  // sixteens mirrored
  return max_of_quarters(x);
}
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

// What a share of a row's positions leaves for the join beside its own output: its sum l 2^n, as an exponent and a
// fraction in [1/2, 1) (or 0), so that weights of shares are at most 1 whatever their sizes.
__device__ inline float2 part_sum(float n, float l) {
  return make_float2(n + static_cast<float>(__builtin_amdgcn_frexp_expf(l)), __builtin_amdgcn_frexp_mantf(l));
}
// Base of the exponents of up to `most` shares, `top` the largest: their weights' sum is at most 1, so what is joined is in
// the range of what is joined from.
__device__ inline float join_base(float top, int most) {
  return (top == -INFINITY ? 0.f : top) + static_cast<float>(32 - __builtin_clz(most - 1));
}

// Positions the page table can name (cut off where positions would pass 31 bits).
__device__ inline int64_t positions_held(const PagedCache& c) {
  const int64_t n = static_cast<int64_t>(c.cols) << c.page_log2, most = (int64_t{1} << 31) - 64;
  return n < most ? n : most;
}

// Query rows of a request and KV head: row i is head h * group + i % group of its token i / group.  A call
// has less than 2^31 of them in all.
struct Request {
  int begin, end;  // packed rows of its tokens
  int pos0;
};
__device__ inline Request request_at(const SeqBatch& s, int b) {
  const Span span = span_of(s, b);
  return Request{static_cast<int>(span.begin), static_cast<int>(span.end), static_cast<int>(span.pos0)};
}
// Blocks of 32 positions up to the one of the request's token `token`.
__device__ inline int blocks_to(int64_t held, int pos0, int token) {
  const int64_t seen = static_cast<int64_t>(pos0) + token + 1;
  return static_cast<int>(((seen < 0 ? 0 : (seen < held ? seen : held)) + 31) >> 5);
}
// Last position a token attends to, as far as it can be held.
__device__ inline int reach_of(int64_t held, int pos0, int token) {
  const int64_t pos = static_cast<int64_t>(pos0) + token;
  return static_cast<int>(pos < -1 ? -1 : (pos < held ? pos : held));
}

}  // namespace dev

// Workspace: a count for each workgroup of a launch (0 between calls), then partial sums.
constexpr int kRowsWorkers = 512;
constexpr size_t kCounterBytes = kRowsWorkers * sizeof(int);

// A few rows of a request: rows of a tile, waves of a workgroup, steps of the longest segment up to which all stay
// whole, and workgroups whose parts cost a step to leave and join.  (Tiles of 32 and 64 rows halve the conversions but
// leave one wave a SIMD its registers: 64 requests of 5 rows over 8 KV heads of 128 and up to 4K positions take 136 us
// in tiles of 32 and 122 us in tiles of 16.  Eight waves a workgroup join more on the spot, but four, two workgroups a
// CU, hide one's ends behind the other: 64 requests over 16 KV heads of 64 take 111 and 86 us.)
constexpr int kRowTile = 16, kRowWaves = 4, kUncutSteps = 4, kWorkersAStep = 40;
// Mean parts of a segment, at most: one workgroup joins them.  (16, 64 and 128 are no faster than the 24 us of one
// request of 32K positions over 4 heads.)
constexpr int kMostParts = 32;

constexpr int kPromptWaves = 8, kPromptRows = 32 * kPromptWaves;
constexpr int kMostSplits = 64;   // shares of a prompt's tile

}  // namespace scd
