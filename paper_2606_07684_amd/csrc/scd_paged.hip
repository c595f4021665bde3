// The paged 8-bit cache: rows appended (keys rotated on the way) and read back (gfx950).
#include "scd_serve_device.h"

namespace scd {
using namespace dev;

// Scales below this are 0, so that 1 / scale is finite.
constexpr float kSmallestScale = 1.17549435e-38f;

// How a row's 16-channel items turn.
enum class TurnKind : int {
  kNone,         // as they are
  kHalf,         // item i < dim / 16: channels 8i.. and dim / 2 + 8i.., the two halves of 8 pairs
  kInterleaved,  // item i: channels 16i.., 8 adjacent pairs
  kOdd           // rotary_dim not a multiple of 16: channels 16i.., each with its partner wherever it is
};

// First channels of the two 8-channel groups of an item.
template <TurnKind kKind>
__device__ inline int2 item_channels(const Turn& turn, int item) {
  if (kKind == TurnKind::kHalf && 16 * item < turn.dim) return make_int2(8 * item, turn.dim / 2 + 8 * item);
  return make_int2(16 * item, 16 * item + 8);
}
// An item's 16 channels turned by the table's row `cs` (its 8 pairs in registers but for kOdd).
template <TurnKind kKind, typename T>
__device__ inline void turn_item(const Turn& turn, const T* row, int item, const float2 (&cs)[8],
                                 const float2* table_row, float (&x)[16]) {
  if constexpr (kKind == TurnKind::kHalf) {
    if (16 * item < turn.dim) {
#pragma unroll
      for (int i = 0; i < 8; ++i) turn_pair(x[i], x[8 + i], cs[i], x[i], x[8 + i]);
    }
  } else if constexpr (kKind == TurnKind::kInterleaved) {
    if (16 * item < turn.dim) {
#pragma unroll
      for (int i = 0; i < 8; ++i) turn_pair(x[2 * i], x[2 * i + 1], cs[i], x[2 * i], x[2 * i + 1]);
    }
  } else if constexpr (kKind == TurnKind::kOdd) {
    float unused;
    const int half = turn.dim / 2;
    for (int i = 0; i < 16; ++i) {
      const int c = 16 * item + i;
      if (c >= turn.dim) break;
      if (turn.interleaved) {
        if (c % 2 == 0) turn_pair(x[i], x[i + 1], table_row[c / 2], x[i], x[i + 1]);
      } else if (c < half) {
        turn_pair(x[i], load1(row + c + half), table_row[c], x[i], unused);
      } else {
        turn_pair(load1(row + c - half), x[i], table_row[c - half], unused, x[i]);
      }
    }
  }
}

// Four values of at most 127 in magnitude (and a rounding) rounded to whole numbers, ties to even, as bytes:
// 1.5 * 2^23 more, a float's last bits are the number's.  The sum must not take the caller's product in.
__device__ inline uint32_t pack4(const float* f) {
#pragma clang fp contract(off)
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(f[i] + 12582912.f);
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400u),
                               __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), 0x05040100u);
}
__device__ inline void unpack4(uint32_t w, float* f) {
  f[0] = static_cast<float>(static_cast<int8_t>(w));
  f[1] = static_cast<float>(static_cast<int8_t>(w >> 8));
  f[2] = static_cast<float>(static_cast<int8_t>(w >> 16));
  f[3] = static_cast<float>(static_cast<int32_t>(w) >> 24);
}

// Sixteen channels of a row as they lie in memory, to be turned and quantised later.
template <typename T> struct RawItem;
template <> struct RawItem<uint16_t> {
  uint4 a, b;
  __device__ void load(const uint16_t* row, int2 c, bool wide) {
    if (wide) {
      a = *reinterpret_cast<const uint4*>(row + c.x);
      b = *reinterpret_cast<const uint4*>(row + c.y);
    } else {
      uint32_t w[8];
      for (int i = 0; i < 8; ++i) {
        const uint16_t* p = row + (i < 4 ? c.x + 2 * i : c.y + 2 * (i - 4));
        w[i] = p[0] | static_cast<uint32_t>(p[1]) << 16;
      }
      a = make_uint4(w[0], w[1], w[2], w[3]);
      b = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
  __device__ void get(float (&x)[16]) const {
    unpack8(a, x);
    unpack8(b, x + 8);
  }
};
template <> struct RawItem<float> {
  float x[16];
  __device__ void load(const float* row, int2 c, bool wide) {
    load8(row + c.x, wide, x);
    load8(row + c.y, wide, x + 8);
  }
  __device__ void get(float (&y)[16]) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x[i];
  }
};

// The new rows of one page that a workgroup appends, [lo, hi) of its slots.
struct PageRows {
  Located at;
  int64_t base;  // position of the page's first slot
  int lo, hi;
  int page;      // -1: a hole
};
template <int kThreads>
__device__ inline bool page_rows(const CacheAppendParams& p, int64_t index, LocateLds& lds, int tid, PageRows& r) {
  const int lg = p.cache.page_log2;
  if (!locate<kThreads>(p.batch, index, lds, tid, [&](const Span& s) -> int64_t {
        const int64_t end = s.pos0 + s.end - s.begin;
        return s.end > s.begin && end > 0 ? ((end - 1) >> lg) - ((s.pos0 < 0 ? 0 : s.pos0) >> lg) + 1 : 0;
      }, r.at))
    return false;
  const Span& s = r.at.span;
  const int64_t from = s.pos0 < 0 ? 0 : s.pos0, end = s.pos0 + s.end - s.begin;
  r.base = ((from >> lg) + r.at.local) << lg;
  r.lo = static_cast<int>(from > r.base ? from - r.base : 0);
  r.hi = static_cast<int>(end - r.base < p.cache.page ? end - r.base : p.cache.page);
  r.page = page_of(p.cache, r.at.b, r.base);
  return true;
}
// Table row of a position (at or past the table's end: its last).
__device__ inline const float2* table_row(const Turn& turn, int64_t pos) {
  return turn.table + (pos >= turn.max_pos ? turn.max_pos - 1 : pos) * (turn.dim / 2);
}
template <TurnKind kKind>
__device__ inline void load_pairs(const Turn& turn, int64_t pos, int item, float2 (&cs)[8]) {
  if constexpr (kKind == TurnKind::kHalf || kKind == TurnKind::kInterleaved) {
    if (16 * item >= turn.dim) return;
    const float4* src = reinterpret_cast<const float4*>(table_row(turn, pos) + 8 * item);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 w = src[j];
      cs[2 * j] = make_float2(w.x, w.y);
      cs[2 * j + 1] = make_float2(w.z, w.w);
    }
  }
}
// Magnitudes are compared as the bits of fp32 less the sign: what is not finite is above all that is.
__device__ inline uint32_t top_of(const float (&x)[16], uint32_t top) {
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const uint32_t bits = __float_as_uint(x[j]) & 0x7fffffffu;
    top = bits > top ? bits : top;
  }
  return top;
}
__device__ inline uint32_t wave_top_of(uint32_t top) {
  for (int o = 32; o > 0; o >>= 1) {
    const uint32_t other = __shfl_xor(top, o);
    top = other > top ? other : top;
  }
  return top;
}
// Scale of a page and head that had `held` (0: none) and takes magnitudes up to that of the bits `top`.
__device__ inline float scale_with(float held, uint32_t top) {
  const float a = top < 0x7f800000u ? __uint_as_float(top) * (1.f / 127.f) : __builtin_nanf("");
  const float scale = a > held || a != a ? a : held;
  return scale < kSmallestScale ? 0.f : scale;
}
__device__ inline void requantise(int8_t* at, float ratio) {
#pragma clang fp contract(off)
  uint4* w = reinterpret_cast<uint4*>(at);
  const uint4 v = *w;
  float f[16];
  unpack4(v.x, f);
  unpack4(v.y, f + 4);
  unpack4(v.z, f + 8);
  unpack4(v.w, f + 12);
#pragma unroll
  for (int j = 0; j < 16; ++j) f[j] *= ratio;
  *w = make_uint4(pack4(f), pack4(f + 4), pack4(f + 8), pack4(f + 12));
}
template <TurnKind kKind>
__device__ inline void store_item(int8_t* row, int2 at, float (&x)[16], float inv) {
#pragma clang fp contract(off)
#pragma unroll
  for (int j = 0; j < 16; ++j) x[j] *= inv;
  const uint4 v = make_uint4(pack4(x), pack4(x + 4), pack4(x + 8), pack4(x + 12));
  if (kKind == TurnKind::kHalf) {
    *reinterpret_cast<uint2*>(row + at.x) = make_uint2(v.x, v.y);
    *reinterpret_cast<uint2*>(row + at.y) = make_uint2(v.z, v.w);
  } else {
    *reinterpret_cast<uint4*>(row + at.x) = v;
  }
}

// Many rows: a workgroup takes one page, one item of 16 channels a thread, and pairs_per of its (branch, head)
// pairs one after another.  A head's rows stay in registers between the maximum and the
// quantisation, the next two heads' are on their way meanwhile, and a thread's cosines and sines serve all heads.
// Bound by HBM: rows are read once, in the model's type, and written once, in 8 bits.  8192 rows of 8 heads of 128 in
// bf16, keys rotated, take 15 us (50 MB, 3.3 TB/s: one round of workgroups, so its start and end weigh); 111,169
// rows 160 to 180 us (683 MB, 3.8 to 4.2 TB/s).
template <typename T, int kDim, int kThreads, TurnKind kKind>
__device__ inline void append_page(const CacheAppendParams& p, int kv, int first_head, int last_head,
                                   const PageRows& r, uint32_t (*wave_top)[kThreads / 64], int tid) {
  constexpr int kItems = kDim / 16;
  const int item = tid % kItems, slot = tid / kItems;
  const Rows& rows = p.rows[kv];
  const T* row = reinterpret_cast<const T*>(rows.data) + (r.at.span.begin + r.base + slot - r.at.span.pos0) * rows.token;
  int8_t* pages = kv ? p.cache.v : p.cache.k;
  float* scales = (kv ? p.cache.v_scale : p.cache.k_scale) + static_cast<int64_t>(r.page) * p.cache.heads;
  const int2 at = item_channels<kKind>(p.turn, item);
  const bool mine = slot >= r.lo && slot < r.hi;
  RawItem<T> raw[2];
  float old[2];
  float2 cs[8];
  float scale_before = 0.f;
  const auto fetch = [&](int h) {
    if (h >= last_head) return;
    const int k = (h - first_head) & 1;
    if (mine) {
      if (k == 0) raw[0].load(row + h * rows.head, at, rows.wide);
      else raw[1].load(row + h * rows.head, at, rows.wide);
    }
    const float scale = r.lo > 0 ? scales[h] : 0.f;
    if (k == 0) old[0] = scale;
    else old[1] = scale;
  };
  fetch(first_head);
  fetch(first_head + 1);
  if (mine) load_pairs<kKind>(p.turn, r.base + slot, item, cs);
  const auto append_head = [&](auto which, int h) {
    constexpr int k = decltype(which)::value;
    float x[16];
    uint32_t top = 0;
    if (mine) {
      raw[k].get(x);
      turn_item<kKind>(p.turn, row, item, cs, nullptr, x);
      top = top_of(x, top);
    }
    const float held = old[k];
    fetch(h + 2);
    top = wave_top_of(top);
    uint32_t* tops = wave_top[k];
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    lds_barrier();  // the loads on their way stay so
    uint32_t all = tops[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) all = tops[w] > all ? tops[w] : all;
    const float scale = scale_with(held, all);
    const float inv = scale > 0.f ? 1.f / scale : 0.f;
    // A head's scale is stored a barrier late: a wave that has no new rows of the page comes to this one with its load
    // of the old scale on its way still, but not to the next, before which it needs it.
    if (tid == 0 && h > first_head) scales[h - 1] = scale_before;
    scale_before = scale;
    int8_t* dst = pages + page_at(p.cache, r.page, h, kDim) + slot * kDim;
    if (mine) store_item<kKind>(dst, at, x, inv);
    else if (slot < r.lo && scale > held) requantise(dst + 16 * item, held * inv);
  };
  for (int h = first_head; h < last_head; h += 2) {
    append_head(IntC<0>{}, h);
    if (h + 1 < last_head) append_head(IntC<1>{}, h + 1);
  }
  lds_barrier();  // and wave_top is written again
  if (tid == 0) scales[last_head - 1] = scale_before;
}

template <typename T, int kDim, int kThreads, TurnKind kKind>
__global__ __launch_bounds__(kThreads) void cache_append_pages_kernel(CacheAppendParams p, int pairs_per, int shares,
                                                                     int64_t units) {
  __shared__ LocateLds lds;
  __shared__ uint32_t wave_top[2][kThreads / 64];
  const int tid = threadIdx.x;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    // of the 2 n_kv_heads (branch, head) pairs, keys first
    const int heads = p.cache.heads, first = static_cast<int>(unit % shares) * pairs_per;
    const int last = first + pairs_per < 2 * heads ? first + pairs_per : 2 * heads;
    PageRows r;
    if (!page_rows<kThreads>(p, unit / shares, lds, tid, r)) return;
    if (r.page < 0) continue;
    if (first < heads)
      append_page<T, kDim, kThreads, kKind>(p, 0, first, last < heads ? last : heads, r, wave_top, tid);
    if (last > heads)
      append_page<T, kDim, kThreads, TurnKind::kNone>(p, 1, first > heads ? first - heads : 0, last - heads, r, wave_top, tid);
  }
}

// A few rows of a page (and any number where rotary_dim is odd in 16s): a wave takes one branch of one page and
// head, 64 items at a time, first for the maximum and then for the quantisation, the first 64 read once.  Latency:
// one row of each of 64 requests, 8 heads of 128, takes 5 us.
template <typename T, int kDim, TurnKind kKind>
__device__ inline void append_few(const CacheAppendParams& p, int kv, int h, const PageRows& r, int lane) {
  constexpr int kItems = kDim / 16;
  const Rows& rows = p.rows[kv];
  const T* src = reinterpret_cast<const T*>(rows.data) + (r.at.span.begin + r.base - r.at.span.pos0) * rows.token + h * rows.head;
  float* scale_at = (kv ? p.cache.v_scale : p.cache.k_scale) + static_cast<int64_t>(r.page) * p.cache.heads + h;
  int8_t* dst = (kv ? p.cache.v : p.cache.k) + page_at(p.cache, r.page, h, kDim);
  const int first = r.lo * kItems, last = r.hi * kItems;
  const int item = lane % kItems;  // 64 is a multiple of kItems
  const int2 at = item_channels<kKind>(p.turn, item);
  const auto fetch = [&](int i, float (&x)[16]) {
    const int slot = i / kItems;
    const T* row = src + slot * rows.token;
    RawItem<T> raw;
    float2 cs[8];
    raw.load(row, at, rows.wide);
    load_pairs<kKind>(p.turn, r.base + slot, item, cs);
    raw.get(x);
    turn_item<kKind>(p.turn, row, item, cs, kKind == TurnKind::kOdd ? table_row(p.turn, r.base + slot) : nullptr, x);
  };
  const float held = r.lo > 0 ? *scale_at : 0.f;
  float x[16];
  uint32_t top = 0;
  if (first + lane < last) {
    fetch(first + lane, x);
    top = top_of(x, top);
  }
  for (int i = first + 64 + lane; i < last; i += 64) {
    float y[16];
    fetch(i, y);
    top = top_of(y, top);
  }
  top = wave_top_of(top);
  const float scale = scale_with(held, top);
  const float inv = scale > 0.f ? 1.f / scale : 0.f;
  if (lane == 0) *scale_at = scale;
  if (first + lane < last) store_item<kKind>(dst + (first + lane) / kItems * kDim, at, x, inv);
  for (int i = first + 64 + lane; i < last; i += 64) {
    fetch(i, x);
    store_item<kKind>(dst + i / kItems * kDim, at, x, inv);
  }
  if (scale > held)
    for (int i = lane; i < first; i += 64) requantise(dst + i * 16, held * inv);
}

template <typename T, int kDim, TurnKind kKind>
__global__ __launch_bounds__(256) void cache_append_few_kernel(CacheAppendParams p, int shares, int64_t units) {
  __shared__ LocateLds lds;
  const int tid = threadIdx.x;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    // four of the 2 n_kv_heads (branch, head) pairs a workgroup, keys first
    const int pair = static_cast<int>(unit % shares) * 4 + __builtin_amdgcn_readfirstlane(tid >> 6);
    PageRows r;
    if (!page_rows<256>(p, unit / shares, lds, tid, r)) return;
    if (r.page < 0 || pair >= 2 * p.cache.heads) continue;
    const int kv = pair >= p.cache.heads;
    if (kv) append_few<T, kDim, TurnKind::kNone>(p, kv, pair - p.cache.heads, r, tid & 63);
    else append_few<T, kDim, kKind>(p, kv, pair, r, tid & 63);
  }
}

// One wave per row: both branches of every head, 16 channels a lane at a time.  Bound by HBM: 111,169 rows of 8 heads
// of 128 into bf16 take 145 us (683 MB, 4.7 TB/s).
template <typename T, int kDim>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheReadParams p) {
  constexpr int kChunks = kDim / 16;
  const int lane = threadIdx.x & 63;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); t < p.batch.n_tokens;
       t += static_cast<int64_t>(gridDim.x) * 4) {
    const Owner owner = owner_of(p.batch, t, lane);
    const int64_t pos = t - owner.begin + owner.pos0;
    const int page = page_of(p.cache, owner.b, pos);
    for (int idx = lane; idx < 2 * p.cache.heads * kChunks; idx += 64) {
      const int kv = idx >= p.cache.heads * kChunks;
      const int h = idx / kChunks - (kv ? p.cache.heads : 0), chunk = idx % kChunks;
      float f[16];
      if (page < 0) {
        for (int i = 0; i < 16; ++i) f[i] = 0.f;
      } else {
        const int8_t* src = (kv ? p.cache.v : p.cache.k) + page_at(p.cache, page, h, kDim) +
                            (pos & (p.cache.page - 1)) * kDim + 16 * chunk;
        const float scale = (kv ? p.cache.v_scale : p.cache.k_scale)[static_cast<int64_t>(page) * p.cache.heads + h];
        const uint4 w = *reinterpret_cast<const uint4*>(src);
        unpack4(w.x, f);
        unpack4(w.y, f + 4);
        unpack4(w.z, f + 8);
        unpack4(w.w, f + 12);
        for (int i = 0; i < 16; ++i) f[i] *= scale;
      }
      const Rows& rows = p.rows[kv];
      T* dst = reinterpret_cast<T*>(rows.data) + t * rows.token + h * rows.head + 16 * chunk;
      store8(dst, rows.wide, f);
      store8(dst + 8, rows.wide, f + 8);
    }
  }
}

// Pages that a batch touches, at most: a request's n rows lie in at most (n - 2) / page + 2 of them.
static int64_t pages_bound(const SeqBatch& b, int page) {
  const int64_t requests = b.n_seqs < b.n_tokens ? b.n_seqs : b.n_tokens;
  const int64_t bound = b.n_tokens / page + 2 * requests;
  return bound < b.n_tokens ? bound : b.n_tokens;
}
static dim3 grid_of(int64_t units) { return dim3(static_cast<unsigned>(units < kMaxGrid / 4 ? units : kMaxGrid / 4)); }

template <typename T, int kDim, TurnKind kKind>
static hipError_t launch_append_few(const CacheAppendParams& p, hipStream_t stream) {
  const int shares = (2 * p.cache.heads + 3) / 4;
  const int64_t units = pages_bound(p.batch, p.cache.page) * shares;
  hipLaunchKernelGGL((cache_append_few_kernel<T, kDim, kKind>), grid_of(units), dim3(256), 0, stream, p, shares, units);
  return hipGetLastError();
}

template <typename T, int kDim, int kPage, TurnKind kKind>
static hipError_t launch_append_pages(const CacheAppendParams& p, hipStream_t stream) {
  constexpr int kThreads = kPage * kDim / 16 < 64 ? 64 : kPage * kDim / 16;
  const int64_t pages = pages_bound(p.batch, kPage);
  // As many pairs to a workgroup as leave 512 workgroups: what a workgroup pays once (finding its page, its rows'
  // cosines and sines) is about what two pairs cost.
  const int64_t pairs = 2 * p.cache.heads, most = pages * pairs / 512;
  const int pairs_per = static_cast<int>(most < 1 ? 1 : (most < pairs ? most : pairs));
  const int shares = static_cast<int>((pairs + pairs_per - 1) / pairs_per);
  const int64_t units = pages * shares;
  hipLaunchKernelGGL((cache_append_pages_kernel<T, kDim, kThreads, kKind>), grid_of(units), dim3(kThreads), 0, stream, p,
                     pairs_per, shares, units);
  return hipGetLastError();
}

template <typename T, int kDim, TurnKind kKind>
static hipError_t launch_append_kind(const CacheAppendParams& p, hipStream_t stream) {
  // Few rows leave most of a page's workgroup idle, many keep a head's one wave at its page for long.  Rotated bf16
  // rows of 8 heads of 128 in pages of 64, behind 1000, us as a wave a head / a workgroup a page:
  //   1 request    16 rows 5.0 / 5.0    32 rows 5.9 / 5.1    64 rows  7.5 / 5.2     128 rows 10.1 / 5.3
  //   16 requests  16 rows 5.8 / 6.6    32 rows 6.8 / 7.8    64 rows  8.5 / 8.1     128 rows 11.4 / 9.0
  //   64 requests  16 rows 6.1 / 8.7    32 rows 8.4 / 12.2   64 rows 12.1 / 14.6    128 rows 18.0 / 18.0
  // The rule is that of one request: of 16 and 64 a wave a head is the faster side up to 32 and 128 rows.
  const int64_t requests = p.batch.n_seqs < p.batch.n_tokens ? p.batch.n_seqs : p.batch.n_tokens;
  if (kKind == TurnKind::kOdd || p.batch.n_tokens < 32 * requests) return launch_append_few<T, kDim, kKind>(p, stream);
  if constexpr (kKind != TurnKind::kOdd) {
    if (p.cache.page == 16) return launch_append_pages<T, kDim, 16, kKind>(p, stream);
    if (p.cache.page == 32) return launch_append_pages<T, kDim, 32, kKind>(p, stream);
    if (p.cache.page == 64) return launch_append_pages<T, kDim, 64, kKind>(p, stream);
    // fp32 rows of 128 channels would leave 1024 threads no registers
    if constexpr (sizeof(T) == 4 && kDim == 128) return launch_append_few<T, kDim, kKind>(p, stream);
    else return launch_append_pages<T, kDim, 128, kKind>(p, stream);
  }
  return hipSuccess;
}

template <typename T, int kDim>
static hipError_t launch_append_as(const CacheAppendParams& p, hipStream_t stream) {
  if (p.turn.table == nullptr) return launch_append_kind<T, kDim, TurnKind::kNone>(p, stream);
  if (p.turn.dim % 16 != 0) return launch_append_kind<T, kDim, TurnKind::kOdd>(p, stream);
  return p.turn.interleaved ? launch_append_kind<T, kDim, TurnKind::kInterleaved>(p, stream)
                            : launch_append_kind<T, kDim, TurnKind::kHalf>(p, stream);
}

hipError_t launch_cache_append(bool bf16, int head_dim, const CacheAppendParams& p,
                               hipStream_t stream) {
  if (bf16)
    return head_dim == 128 ? launch_append_as<uint16_t, 128>(p, stream)
           : head_dim == 64 ? launch_append_as<uint16_t, 64>(p, stream)
                            : launch_append_as<uint16_t, 32>(p, stream);
  return head_dim == 128 ? launch_append_as<float, 128>(p, stream)
         : head_dim == 64 ? launch_append_as<float, 64>(p, stream)
                          : launch_append_as<float, 32>(p, stream);
}

template <typename T, int kDim>
static hipError_t launch_read_as(const CacheReadParams& p, hipStream_t stream) {
  const int64_t blocks = (p.batch.n_tokens + 3) / 4;
  hipLaunchKernelGGL((cache_read_kernel<T, kDim>),
                     dim3(static_cast<unsigned>(blocks < kMaxGrid ? blocks : kMaxGrid)), dim3(256), 0,
                     stream, p);
  return hipGetLastError();
}

hipError_t launch_cache_read(bool bf16, int head_dim, const CacheReadParams& p, hipStream_t stream) {
  if (bf16)
    return head_dim == 128 ? launch_read_as<uint16_t, 128>(p, stream)
           : head_dim == 64 ? launch_read_as<uint16_t, 64>(p, stream)
                            : launch_read_as<uint16_t, 32>(p, stream);
  return head_dim == 128 ? launch_read_as<float, 128>(p, stream)
         : head_dim == 64 ? launch_read_as<float, 64>(p, stream)
                          : launch_read_as<float, 32>(p, stream);
}

}  // namespace scd
