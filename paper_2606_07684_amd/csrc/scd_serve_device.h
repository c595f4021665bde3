// Device helpers of the serving operators (gfx950).
#pragma once

#include "scd_device.h"
#include "scd_serve.h"

namespace scd {
namespace dev {

// Workgroups of 256 threads one launch holds: kernels step over what is beyond it, so a launch stays
// below 2^32 work-items.
constexpr int64_t kMaxGrid = int64_t{1} << 23;

// a / b for a >= 0, b > 0; in 32 bits where both fit, which takes a tenth of the time.
__device__ inline int64_t div_up_to(int64_t a, int64_t b) {
  if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
  return a / b;
}
__device__ inline int64_t div_ceil(int64_t a, int64_t b) { return div_up_to(a + b - 1, b); }

// Rows of request b, kept inside the batch whatever cu holds.
struct Span {
  int64_t begin, end;
  int64_t pos0;
};
__device__ inline Span span_of(const SeqBatch& s, int b) {
  Span r{0, s.n_tokens, s.pos0 != nullptr ? s.pos0[b] : 0};
  if (s.cu != nullptr) {
    r.begin = s.cu[b];
    r.end = s.cu[b + 1];
    r.begin = r.begin < 0 ? 0 : (r.begin > s.n_tokens ? s.n_tokens : r.begin);
    r.end = r.end < r.begin ? r.begin : (r.end > s.n_tokens ? s.n_tokens : r.end);
  }
  return r;
}

// Request, first row and held tokens of row t (the same for the whole wave): the last b with cu[b] <= t.
// Each step reads 64 boundaries at once, and the last one the held tokens with them, so 64 requests
// take one memory access and 4096 two.
struct Owner {
  int b;
  int64_t begin, pos0;
};
__device__ inline Owner owner_of(const SeqBatch& s, int64_t t, int lane) {
  if (s.cu == nullptr) return Owner{0, 0, s.pos0 != nullptr ? s.pos0[0] : 0};
  int lo = 0, n = s.n_seqs;
  while (n > 64) {
    const int step = (n + 63) >> 6;
    const int i = lane * step;
    const bool under = i < n && (i == 0 || s.cu[lo + i] <= t);
    const int at = (__popcll(__ballot(under)) - 1) * step;
    lo += at;
    n = n - at < step ? n - at : step;
  }
  const int start = lane < n ? s.cu[lo + lane] : 0;
  const int held = lane < n && s.pos0 != nullptr ? s.pos0[lo + lane] : 0;
  const int at = __builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < n && (lane == 0 || start <= t))) - 1);
  return Owner{lo + at, __builtin_amdgcn_readlane(start, at), __builtin_amdgcn_readlane(held, at)};
}

// Page of position p of request b, or -1: out of the table, or a hole.
__device__ inline int page_of(const PagedCache& c, int b, int64_t p) {
  const int64_t col = p >> c.page_log2;
  if (p < 0 || col >= c.cols) return -1;
  const int id = c.table[static_cast<int64_t>(b) * c.cols + col];
  return id >= 0 && id < c.n_pages ? id : -1;
}

// First byte of a page's rows of one head.
__device__ inline int64_t page_at(const PagedCache& c, int page, int head, int d) {
  return (static_cast<int64_t>(page) * c.heads + head) * (c.page * static_cast<int64_t>(d));
}

// Work units of requests one after another, count(span) of each: the request and its rows, and the
// place among its units, of `unit`; false past the last.  Every thread of the workgroup calls it and
// gets the answer.
struct Located {
  Span span;
  int64_t local;
  int b;
};
struct LocateLds {
  int64_t wave_sum[16];
  Located found;
};
template <int kThreads, typename Count>
__device__ inline bool locate(const SeqBatch& s, int64_t unit, LocateLds& lds, int tid, Count count,
                              Located& out) {
  if (s.n_seqs == 1) {
    out.b = 0;
    out.local = unit;
    out.span = span_of(s, 0);
    return unit < count(out.span);
  }
  const int lane = tid & 63, wave = tid >> 6;
  for (int base = 0; base < s.n_seqs; base += kThreads) {
    Span span{0, 0, 0};
    if (base + tid < s.n_seqs) span = span_of(s, base + tid);
    const int64_t mine = count(span);
    int64_t sum = mine;
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t other = __shfl_up(sum, o);
      if (lane >= o) sum += other;
    }
    __syncthreads();  // the last round's readers are done
    if (tid == 0) lds.found.b = -1;
    if (lane == 63) lds.wave_sum[wave] = sum;
    __syncthreads();
    int64_t before = 0, total = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w < wave) before += lds.wave_sum[w];
      total += lds.wave_sum[w];
    }
    const int64_t first = before + sum - mine;
    if (unit >= first && unit < first + mine) lds.found = Located{span, unit - first, base + tid};
    __syncthreads();
    if (lds.found.b >= 0) {
      out = lds.found;
      return true;
    }
    unit -= total;
  }
  return false;
}

// Eight channels of a row in fp32.  Rows that start on 16 bytes take 16-byte accesses.
template <typename T> __device__ inline void load8(const T* p, bool wide, float* f);
template <> __device__ inline void load8<uint16_t>(const uint16_t* p, bool wide, float* f) {
  if (wide) {
    unpack8(*reinterpret_cast<const uint4*>(p), f);
  } else {
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(static_cast<uint32_t>(p[i]) << 16);
  }
}
template <> __device__ inline void load8<float>(const float* p, bool wide, float* f) {
  if (wide) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
    for (int i = 0; i < 8; ++i) f[i] = p[i];
  }
}
template <typename T> __device__ inline void store8(T* p, bool wide, const float* f);
template <> __device__ inline void store8<uint16_t>(uint16_t* p, bool wide, const float* f) {
  const uint4 v = pack8(f);
  if (wide) {
    *reinterpret_cast<uint4*>(p) = v;
  } else {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    for (int i = 0; i < 8; ++i) p[i] = static_cast<uint16_t>(w[i >> 1] >> (16 * (i & 1)));
  }
}
template <> __device__ inline void store8<float>(float* p, bool wide, const float* f) {
  if (wide) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
  } else {
    for (int i = 0; i < 8; ++i) p[i] = f[i];
  }
}
__device__ inline float load1(const uint16_t* p) { return __uint_as_float(static_cast<uint32_t>(*p) << 16); }
__device__ inline float load1(const float* p) { return *p; }
__device__ inline void store1(uint16_t* p, float f) { *p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }
__device__ inline void store1(float* p, float f) { *p = f; }

// The two channels of a pair turned by (c, s): products and sums rounded one by one, so that a row
// turned here and quantised has the bits of one turned, kept in fp32 and quantised.
__device__ inline void turn_pair(float a, float b, float2 cs, float& x, float& y) {
#pragma clang fp contract(off)
  x = a * cs.x - b * cs.y;
  y = b * cs.x + a * cs.y;
}

}  // namespace dev
}  // namespace scd
