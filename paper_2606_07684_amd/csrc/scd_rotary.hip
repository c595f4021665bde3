// Rotary positions of packed queries and keys (gfx950).
//
// y = R(p) x per head: pair i of rotary_dim / 2 pairs turns by p * w_i, (a, b) -> (a cos - b sin,
// b cos + a sin); the transposed form has -sin.  Every element is read and written once, so the
// kernel is bound by HBM; cosines and sines are fp32 table entries (evaluated in fp64), shared by all
// heads of a token.  8192 tokens of 32 + 8 heads of 128 in bf16 take 34.4 us (168 MB, 4.9 TB/s; a large copy
// moves 5.2); 16 tokens 3.5 us, the launch and two memory accesses one after the other.
#include "scd_serve_device.h"

namespace scd {
using namespace dev;

__global__ void turn_table_kernel(TurnTableParams p) {
  const int64_t stride = static_cast<int64_t>(gridDim.x) * blockDim.x;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < p.n; i += stride) {
    const int64_t pos = i / p.pairs;
    double s, c;
    sincos(static_cast<double>(pos) * p.w[i - pos * p.pairs], &s, &c);
    p.table[i] = make_float2(static_cast<float>(c * p.gain), static_cast<float>(s * p.gain));
  }
}

// A wave takes 64 items of one token: an item is two groups of kVec channels of one head, the two
// halves of kVec pairs (HALF) or 2 kVec adjacent channels (INTERLEAVED, and past rotary_dim).
template <typename T, int kVec>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p, int items_per_head, int parts,
                                                     int64_t units) {
  const int lane = threadIdx.x & 63;
  const int turning = p.turn.dim / (2 * kVec);
  const int heads = p.in[0].n_heads + p.in[1].n_heads;
  for (int64_t unit = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); unit < units;
       unit += static_cast<int64_t>(gridDim.x) * 4) {
    const int64_t t = unit / parts;
    const int idx = static_cast<int>(unit - t * parts) * 64 + lane;
    const Owner owner = owner_of(p.batch, t, lane);
    int64_t pos = t - owner.begin + owner.pos0;
    pos = pos < 0 ? 0 : (pos >= p.turn.max_pos ? p.turn.max_pos - 1 : pos);
    if (idx >= heads * items_per_head) continue;
    int h = idx / items_per_head;
    const int item = idx - h * items_per_head;
    const bool key = h >= p.in[0].n_heads;
    if (key) h -= p.in[0].n_heads;
    const Rows& in = p.in[key];
    const Rows& out = p.out[key];
    const T* src = reinterpret_cast<const T*>(in.data) + t * in.token + h * in.head;
    T* dst = reinterpret_cast<T*>(out.data) + t * out.token + h * out.head;
    if (item >= turning) {  // past rotary_dim
      if (in.data == out.data) continue;
      const int c = p.turn.dim + (item - turning) * 2 * kVec;
      for (int g = c; g < c + 2 * kVec && g < p.head_dim; g += kVec) {
        if constexpr (kVec == 8) {
          float f[8];
          load8(src + g, true, f);
          store8(dst + g, true, f);
        } else {
          dst[g] = src[g];
        }
      }
      continue;
    }
    const float2* cs = p.turn.table + pos * (p.turn.dim / 2) + item * kVec;
    const int c0 = p.turn.interleaved ? item * 2 * kVec : item * kVec;
    const int c1 = p.turn.interleaved ? c0 + kVec : c0 + p.turn.dim / 2;
    float x[2 * kVec];
    if constexpr (kVec == 8) {
      load8(src + c0, true, x);
      load8(src + c1, true, x + 8);
    } else {
      x[0] = load1(src + c0);
      x[1] = load1(src + c1);
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      float2 w = cs[i];
      if (p.transpose) w.y = -w.y;
      if (p.turn.interleaved) {
        turn_pair(x[2 * i], x[2 * i + 1], w, x[2 * i], x[2 * i + 1]);
      } else {
        turn_pair(x[i], x[kVec + i], w, x[i], x[kVec + i]);
      }
    }
    if constexpr (kVec == 8) {
      store8(dst + c0, true, x);
      store8(dst + c1, true, x + 8);
    } else {
      store1(dst + c0, x[0]);
      store1(dst + c1, x[1]);
    }
  }
}

hipError_t launch_turn_table(const TurnTableParams& p, hipStream_t stream) {
  if (p.n <= 0) return hipSuccess;
  const int64_t blocks = (p.n + 255) / 256;
  hipLaunchKernelGGL(turn_table_kernel, dim3(static_cast<unsigned>(blocks < kMaxGrid ? blocks : kMaxGrid)),
                     dim3(256), 0, stream, p);
  return hipGetLastError();
}

template <typename T, int kVec>
static hipError_t launch_rotary_as(const RotaryParams& p, hipStream_t stream) {
  const int turning = p.turn.dim / (2 * kVec);
  const int per_head = turning + (p.head_dim - p.turn.dim + 2 * kVec - 1) / (2 * kVec);
  const int parts = ((p.in[0].n_heads + p.in[1].n_heads) * per_head + 63) / 64;
  const int64_t units = p.batch.n_tokens * parts;
  const int64_t blocks = (units + 3) / 4;
  hipLaunchKernelGGL((rotary_kernel<T, kVec>),
                     dim3(static_cast<unsigned>(blocks < kMaxGrid ? blocks : kMaxGrid)), dim3(256), 0,
                     stream, p, per_head, parts, units);
  return hipGetLastError();
}

hipError_t launch_rotary(bool bf16, const RotaryParams& p, hipStream_t stream) {
  bool wide = p.turn.dim % 16 == 0 && p.head_dim % 8 == 0;
  for (int i = 0; i < 2; ++i)
    if (p.in[i].n_heads > 0) wide = wide && p.in[i].wide && p.out[i].wide;
  if (bf16) return wide ? launch_rotary_as<uint16_t, 8>(p, stream) : launch_rotary_as<uint16_t, 1>(p, stream);
  return wide ? launch_rotary_as<float, 8>(p, stream) : launch_rotary_as<float, 1>(p, stream);
}

}  // namespace scd
