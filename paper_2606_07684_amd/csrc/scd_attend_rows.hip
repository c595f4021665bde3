// Attention of a few rows of every request over the paged 8-bit cache (gfx950).
//
// Work is counted in steps (a block of 32 positions for each of a workgroup's waves) of a segment, the pair of a
// tile of query rows and a KV head.  All steps, one segment after another, are cut into equal shares, one a
// workgroup, so requests of any lengths load the chip evenly.  A workgroup that does not hold all of a segment
// leaves its sums in the workspace, and the last to do so joins them, in the order of the positions, so
// results do not depend on which is last.  Where that would cost more than it evens out, segments stay whole.
//
// Weights are split into two bf16 parts for bf16 output (16 bits; its own rounding has 8) and three for fp32: the
// parts keep fp32's exponent range, so a channel in which the heaviest positions are zero still has its bits, down to
// 2^-110 of them.
//
// Bound by the pages' bytes where segments are long: one token of 16 requests of 1K to 16K positions, 32 heads over
// 8 of 128, takes 67 to 69 us (295 MB, 4.3 TB/s; a large copy moves 5.2).  Of a wave's 430 instructions a block of 32
// positions some 180 turn bytes into operands, so with two waves a SIMD arithmetic alone would take about a third of
// that.  Short contexts are latency: 333 positions of one request take 8.7 us, 2.3 to find the work and fetch
// its first block, 2.7 for the blocks, 2 to join the waves, the rest the launch.  One request of 32K positions
// over 4 heads takes 24 us, 7 of them the join of its 128 parts by 4 workgroups.
#include "scd_attend.h"

namespace scd {
using namespace dev;

struct RowsLayout {
  int most_workers;
  int step_log2;  // blocks of a step
};

constexpr int kThreads = 64 * kRowWaves;

__device__ inline int tiles_of(const CacheAttendParams& p, const Request& r) {
  return static_cast<int>((static_cast<uint32_t>((r.end - r.begin) * p.group) + kRowTile - 1) / kRowTile);
}
__device__ inline int steps_of(const CacheAttendParams& p, const RowsLayout& layout, int64_t held, const Request& r) {
  const int n = (blocks_to(held, r.pos0, r.end - r.begin - 1) + (1 << layout.step_log2) - 1) >> layout.step_log2;
  return n < 1 ? 1 : n;
}

// A workgroup's share [unit, share_end) of all `total` units (steps, or segments where they stay whole), and the
// request, segment and step it begins in.  Worker w's share begins at floor(total w / workers).
struct Share {
  int worker, workers, total, each, over;  // each = total / workers, over the rest
  int unit, end;
  int b, segment, step;
  Request request;
  bool cut;
  __device__ int begin_of(int w) const { return each * w + over * w / workers; }
  // Worker whose share holds unit u.
  __device__ int worker_of(int u) const {
    int w = static_cast<int>(static_cast<float>(u) * workers / total);
    w = w < 0 ? 0 : (w < workers ? w : workers - 1);
    while (begin_of(w) > u) --w;
    while (w + 1 < workers && begin_of(w + 1) <= u) ++w;
    return w;
  }
};
struct ShareLds {
  int2 wave_sum[kThreads / 64];
  int wave_longest[kThreads / 64];
  Request request;
  int b, local;
};
__device__ inline bool share_of(const CacheAttendParams& p, const RowsLayout& layout, int64_t held, ShareLds& lds,
                                int tid, Share& s) {
  const int n = p.batch.n_seqs, lane = tid & 63, wave = tid >> 6;
  struct Scan {
    Request request;
    int2 mine, first, all;  // segments and steps: of this thread's request, before it, of all threads'
    int longest;            // steps of a segment of any of them, at most
  };
  const auto scan = [&](int base) {
    Scan c;
    c.request = base + tid < n ? request_at(p.batch, base + tid) : Request{0, 0, 0};
    c.mine.x = tiles_of(p, c.request) * p.cache.heads;
    const int steps = steps_of(p, layout, held, c.request);
    c.mine.y = c.mine.x * steps;
    int2 sum = c.mine;
    int longest = c.mine.x > 0 ? steps : 0;
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(sum.x, o), y = __shfl_up(sum.y, o), z = __shfl_up(longest, o);
      if (lane >= o) {
        longest = max(longest, z);
        sum.x += x;
        sum.y += y;
      }
    }
    __syncthreads();  // the last round's readers are done
    if (lane == 63) {
      lds.wave_sum[wave] = sum;
      lds.wave_longest[wave] = longest;
    }
    __syncthreads();
    c.first = make_int2(sum.x - c.mine.x, sum.y - c.mine.y);
    c.all = make_int2(0, 0);
    c.longest = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
      const int2 v = lds.wave_sum[w];
      if (w < wave) {
        c.first.x += v.x;
        c.first.y += v.y;
      }
      c.all.x += v.x;
      c.all.y += v.y;
      c.longest = max(c.longest, lds.wave_longest[w]);
    }
    return c;
  };
  Scan c;
  int2 all;
  int longest;
  if (n == 1) {
    c.request = request_at(p.batch, 0);
    all.x = tiles_of(p, c.request) * p.cache.heads;
    longest = steps_of(p, layout, held, c.request);
    all.y = all.x * longest;
  } else {
    c = scan(0);
    all = c.all;
    longest = c.longest;
    for (int base = kThreads; base < n; base += kThreads) {
      c = scan(base);
      all.x += c.all.x;
      all.y += c.all.y;
      longest = max(longest, c.longest);
    }
  }
  all.x = uniform(all.x);
  all.y = uniform(all.y);
  longest = uniform(longest);
  const int64_t parts = kMostParts * static_cast<int64_t>(all.x);
  const int able = static_cast<int>(parts < layout.most_workers ? parts : layout.most_workers);
  if (able < 1) return false;
  // Whole segments take the longest of them (several, if a workgroup has as many); shares the mean, and what leaving
  // and joining them costs, about two steps and one more for every 40 workgroups that do.  New tokens of each of so many
  // requests behind as many positions, 32 heads over 8 of 128, us whole / cut:
  //   1 of 1   behind 600 11.2 / 10.1   1000 14.7 / 10.9      4 of 4   behind 600 13.3 / 15.3   1000 16.8 / 16.5
  //   1 of 16  behind 600 12.5 / 27.0   1000 16.9 / 24.5   2000 26.7 / 28.5   4000 45.0 / 36.6
  //   8 of 16  behind 600 14.0 / 30.9   1000 18.6 / 32.2   2000 28.0 / 38.1   4000 46.5 / 54.5
  const int64_t whole = static_cast<int64_t>((all.x + layout.most_workers - 1) / layout.most_workers) * longest;
  const int sharers = able < all.y ? able : all.y;
  s.cut = longest > kUncutSteps && whole > all.y / sharers + 2 + sharers / kWorkersAStep;
  s.total = s.cut ? all.y : all.x;
  s.workers = able < s.total ? able : s.total;
  s.worker = blockIdx.x;
  if (s.worker >= s.workers) return false;
  s.each = s.total / s.workers;
  s.over = s.total - s.each * s.workers;
  s.unit = s.begin_of(s.worker);
  s.end = s.begin_of(s.worker + 1);
  int local = s.unit;
  s.b = 0;
  s.request = c.request;
  if (n > 1) {
    int before = 0;
    for (int base = 0; base < n; base += kThreads) {
      if (n > kThreads) c = scan(base);
      const int mine = s.cut ? c.mine.y : c.mine.x, first = before + (s.cut ? c.first.y : c.first.x);
      const int here = s.cut ? c.all.y : c.all.x;
      if (s.unit < before + here) {
        if (s.unit >= first && s.unit < first + mine) {
          lds.request = c.request;
          lds.b = base + tid;
          lds.local = s.unit - first;
        }
        __syncthreads();
        break;
      }
      before += here;
    }
    s.request = Request{uniform(lds.request.begin), uniform(lds.request.end), uniform(lds.request.pos0)};
    s.b = uniform(lds.b);
    local = uniform(lds.local);
  }
  const int steps = s.cut ? steps_of(p, layout, held, s.request) : 1;
  s.segment = local / steps;
  s.step = local - s.segment * steps;
  return true;
}

// What a workgroup leaves for another, perhaps on another XCD whose L2 does not see this one's: stores of agent
// scope go through to memory, and have arrived once they are waited for; the one that reads them invalidates its
// caches first.  (A release fence would do for the stores, but writes back a whole L2 each time, at three times
// the run time of 512 workgroups.)
__device__ inline void leave2(float* p, float a, float b) {
  const uint64_t v = static_cast<uint64_t>(__float_as_uint(a)) | static_cast<uint64_t>(__float_as_uint(b)) << 32;
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline float2 take2(const float* p) { return *reinterpret_cast<const float2*>(p); }

// What a workgroup leaves of a row that it does not finish: rows of two slots a worker (0: of a segment that
// began before its share, 1: of one that goes on after it), outputs of their own positions, then their softmax's sums
// (part_sum), then a count a worker of the parts left of the segment that begins in its share.  Counts are 0 between
// calls.
struct Partials {
  float* rows;
  float* sums;
  int* count;
};

// Powers of two that the value scales of a part's pages may lie from the first one's for the softmax's sum to be taken of the
// weights that the values take, divided by the scales: a position that fp32's range leaves out is then below 2^-77 of the
// heaviest.  Otherwise the sum is of exponentials of its own.
constexpr int kNear = 24;

// The waves take a step's blocks straight from the pages into registers in the layout of the
// matrix operands, so no value passes through LDS:
//   scores^T [32 x 16] = K Q^T: a lane holds positions (4g + i, 16 + 4g + i) of one query row, which
//   is the operand layout of   out^T [d x 16] += V^T P^T   with the positions in that order.
// The contraction over channels, and the order of the output channels over the matrix rows, are
// permuted so that every lane reads adjacent bytes.
template <typename T, int kDim>
__global__ __launch_bounds__(kThreads, 2) void cache_attend_rows_kernel(CacheAttendParams p, RowsLayout layout,
                                                                       Partials partial) {
  constexpr int kParts = sizeof(T) == 2 ? 1 : 2;    // of a query element
  constexpr int kWeights = sizeof(T) == 2 ? 2 : 3;  // of a weight
  constexpr int kSteps = kDim / 32;   // matrix steps over channels
  constexpr int kOut = kDim / 16;     // output channels a lane holds of each of its four matrix rows
  constexpr int kPitch = kDim + 4;
  constexpr int kPairs = kDim / 2;
  constexpr int kAhead = 1;          // blocks on their way
  __shared__ ShareLds share_lds;
  __shared__ float joined[kRowWaves][16][kPitch];
  __shared__ float joined_m[kRowWaves][kRowTile];
  __shared__ float2 joined_sum[kRowWaves][kRowTile];
  __shared__ __attribute__((aligned(16))) float team_sums[kThreads][8];
  __shared__ int arrived;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const uniform_ints_t table = (uniform_ints_t)(p.cache.table);
  const uniform_floats_t k_scale = (uniform_floats_t)(p.cache.k_scale);
  const uniform_floats_t v_scale = (uniform_floats_t)(p.cache.v_scale);
  const int64_t held = positions_held(p.cache);

  Share share;
  if (!share_of(p, layout, held, share_lds, tid, share)) return;
  int seg_steps = share.cut ? steps_of(p, layout, held, share.request) : 1;

  while (true) {
    const int b = uniform(share.b), pos0 = share.request.pos0, step = share.step;
    const int step_end = seg_steps - step < share.end - share.unit ? seg_steps : step + share.end - share.unit;
    const int tile = uniform(p.by_heads.of(share.segment)), h = uniform(share.segment - tile * p.cache.heads);
    const int row0 = tile * kRowTile;
    const int all_rows = (share.request.end - share.request.begin) * p.group;
    const int rows = all_rows - row0 < kRowTile ? all_rows - row0 : kRowTile;
    const int last_row = row0 + rows - 1;
    const int blocks = blocks_to(held, pos0, p.by_group.of(last_row));
    const int begin = share.cut ? (step << layout.step_log2 < blocks ? step << layout.step_log2 : blocks) : 0;
    const int end = uniform(share.cut && step_end << layout.step_log2 < blocks ? step_end << layout.step_log2 : blocks);
    const int free_until = uniform(reach_of(held, pos0, p.by_group.of(row0)) + 1);  // positions every row attends to

    // queries, as they lie in memory
    float qx[kSteps][8];
    int limit;  // last position of the lane's row
    {
      const int row = row0 + r < last_row ? row0 + r : last_row;
      const int token = p.by_group.of(row), head = h * p.group + row - token * p.group;
      const T* src = reinterpret_cast<const T*>(p.q.data) + (share.request.begin + token) * p.q.token + head * p.q.head + g * (kDim / 4);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) load8(src + 8 * s, p.q.wide, qx[s]);
      limit = reach_of(held, pos0, token);
    }

    // Blocks are fetched kAhead ahead of the arithmetic, their pages' numbers another one ahead.
    const auto pages_of = [&](int block) {
      int2 id;
      int* const out[2] = {&id.x, &id.y};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // in groups of 16 positions: a block looked up ahead may begin past 31 bits
        const int col = (2 * block + i) >> (p.cache.page_log2 - 4);
        *out[i] = col < p.cache.cols ? table[static_cast<int64_t>(b) * p.cache.cols + col] : -1;
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
    int block = uniform(begin) + wave;
    Fetched ring[kAhead + 1];
    int2 ids;
    if (block < end) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (block + i * kRowWaves < end) fetch(ring[i], block + i * kRowWaves, pages_of(block + i * kRowWaves));
      ids = pages_of(block + kAhead * kRowWaves);
    }

    // queries, lifted and split
    f16x8 q[kParts][kSteps];
    float factor;
    {
      float top = 0.f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(qx[s][j]));
      top = max_of_quarters(top);
      int e = (__float_as_uint(top) >> 23) & 255;
      e = e < kLift + 1 ? kLift + 1 : (e > 254 ? 254 : e);
      const float lift = __uint_as_float(static_cast<uint32_t>(254 + kLift - e) << 23);
      factor = __uint_as_float(static_cast<uint32_t>(e - kLift) << 23) * (p.scale * kLog2e);
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float v = qx[s][j] * lift;
          const _Float16 hi = static_cast<_Float16>(v);
          q[0][s][j] = hi;
          if constexpr (kParts == 2) q[1][s][j] = static_cast<_Float16>(v - static_cast<float>(hi));
        }
    }

    f32x4 acc[kOut];
    float m = -INFINITY;      // running maximum of log2 of a weight times its value scale
    float n = -INFINITY;      // the softmax's sum is l 2^(m - own), or l 2^n once the pages' value scales are far apart
    float l = 0.f;
    int own = 0;              // a value scale's (biased) exponent that the others are near
    bool apart = false;
#pragma unroll
    for (int c = 0; c < kOut; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};

    const auto attend = [&](const Fetched& fetched, int block) {
      const int at = block << 5;
      const auto& kw = fetched.kw;
      const auto& vw = fetched.vw;
      const float (&ks)[2] = fetched.ks;
      const float (&vs)[2] = fetched.vs;
      // scores
      f32x4 score[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        score[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const f16x8 k = bytes_as_f16(kw[i][2 * s], kw[i][2 * s + 1]);
#pragma unroll
          for (int part = 0; part < kParts; ++part) score[i] = mfma16(k, q[part][s], score[i]);
        }
      }
      // value scales as f 2^e (e at least kLeastExponent, where f may be below 1 or 0)
      float part_scale[2], exponent[2], back[2];
      bool far = false;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int e = (uniform(__float_as_int(vs[i])) >> 23) & 255;
        e = e < 127 + kLeastExponent ? 127 + kLeastExponent : (e > 253 ? 253 : e);
        part_scale[i] = vs[i] * __uint_as_float(static_cast<uint32_t>(254 - e) << 23);
        exponent[i] = static_cast<float>(e - 127);
        const bool hole = uniform(fetched.hole[i]);
        own = own == 0 && !hole ? e : own;
        const int off = hole ? 0 : e - own;
        far = far || static_cast<unsigned>(off + kNear) > 2 * kNear;
        back[i] = __uint_as_float(static_cast<uint32_t>(127 - off) << 23);
      }
      if (__builtin_expect(far && !apart, 0)) {
        apart = true;
        n = m - static_cast<float>(own - 127);
      }
      const bool masked = at + 32 > free_until || fetched.hole[0] || fetched.hole[1];
      const auto hidden = [&](int j) { return fetched.hole[j >> 2] || at + 16 * (j >> 2) + 4 * g + (j & 3) > limit; };
      float x[8];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float f = ks[i] * factor;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * i + j] = fmaf(score[i][j], f, exponent[i]);
      }
      if (masked) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (hidden(j)) x[j] = -INFINITY;
      }
      if (__builtin_expect(apart, 0)) {  // the softmax's sum by exponentials of its own
        float top = n;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (x[j] > -INFINITY) top = fmaxf(top, score[j >> 2][j & 3] * (ks[j >> 2] * factor));
        if (top > -INFINITY) {
          l *= exp2_fast(n - top);
          n = top;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (x[j] > -INFINITY) l += exp2_fast(score[j >> 2][j & 3] * (ks[j >> 2] * factor) - n);
        }
      }
      float top = m;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, x[j]);
      top = max_of_quarters(top);
      const float base = top == -INFINITY ? 0.f : top;
      if (__any(top > m)) {
        const float fade = exp2_fast(m - base);
        m = top;
        l = apart ? l : l * fade;
#pragma unroll
        for (int c = 0; c < kOut; ++c) acc[c] *= fade;
      }
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = exp2_fast(x[j] - base);
        sum[j >> 2] += e;
        x[j] = e * part_scale[j >> 2];
      }
      if (!apart) l += sum[0] * back[0] + sum[1] * back[1];
      if (masked) {  // nor does a scale that is not a number reach rows that do not see it
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (hidden(j)) x[j] = 0.f;
      }
      bf16x8 w[kWeights];
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int k = 0; k < kWeights; ++k) {
          w[k][j] = static_cast<__bf16>(x[j]);
          x[j] -= static_cast<float>(w[k][j]);
        }
      // values
      const auto out = [&](auto byte, int word) {
        constexpr int kByte = decltype(byte)::value;
        const bf16x8 v = byte_column_as_bf16<kByte>(vw[word]);
#pragma unroll
        for (int part = 0; part < kWeights; ++part) acc[4 * word + kByte] = mfma16(v, w[part], acc[4 * word + kByte]);
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
    while (block < end) {
#pragma unroll
      for (int i = 0; i <= kAhead; ++i) {
        if (block + kAhead * kRowWaves < end) {
          fetch(ring[(i + kAhead) % (kAhead + 1)], block + kAhead * kRowWaves, ids);
          ids = pages_of(block + (kAhead + 1) * kRowWaves);
        }
        attend(ring[i], block);
        block += kRowWaves;
        if (block >= end) break;
      }
    }

    // join the waves
    const bool whole = step == 0 && step_end == seg_steps;
    const int slot = 2 * share.worker + (step == 0);
    const auto store2 = [&](int row, int c, float x, float y) {
      const int token = p.by_group.of(row0 + row), head = h * p.group + row0 + row - token * p.group;
      T* dst = reinterpret_cast<T*>(p.out.data) + (share.request.begin + token) * p.out.token + head * p.out.head + c;
      if (!p.out.wide) {
        store1(dst, x);
        store1(dst + 1, y);
      } else if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint32_t*>(dst) = pack_bf16x2(x, y);
      } else {
        *reinterpret_cast<float2*>(dst) = make_float2(x, y);
      }
    };
    if (apart) {
      const float all = max_of_quarters(n);
      l *= exp2_fast(n - (all == -INFINITY ? 0.f : all));
      n = all;
    } else if (m > -INFINITY) {
      n = m - static_cast<float>(own - 127);
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
      joined_m[wave][r] = m;
      joined_sum[wave][r] = make_float2(n, l);
    }
    lds_barrier();
    if (r < rows) {
      float top = joined_m[0][r];
      for (int v = 1; v < kRowWaves; ++v) top = fmaxf(top, joined_m[v][r]);
      const float mine = exp2_fast(m - (top == -INFINITY ? 0.f : top));
      float* dst = joined[wave][r];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < kOut; ++c) dst[kOut * (4 * g + i) + c] = acc[c][i] * mine;
    }
    lds_barrier();
    for (int item = tid; item < rows * kPairs; item += kThreads) {
      const int row = item / kPairs, c = 2 * (item % kPairs);
      float x = 0.f, y = 0.f, top = -INFINITY, sum_top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int v = 0; v < kRowWaves; ++v) {
        const float2 f = *reinterpret_cast<const float2*>(&joined[v][row][c]);
        x += f.x;
        y += f.y;
        top = fmaxf(top, joined_m[v][row]);
        sum_top = fmaxf(sum_top, joined_sum[v][row].x);
      }
      const float base = sum_top == -INFINITY ? 0.f : sum_top;
#pragma unroll
      for (int v = 0; v < kRowWaves; ++v) sum += joined_sum[v][row].y * exp2_fast(joined_sum[v][row].x - base);
      // x 2^(top - base) / sum, in two steps as the power may be out of range
      const float power = exp2_fast(0.5f * (top - base));
      const float inv = sum != 0.f ? power / sum : 0.f;
      x = x * inv * power;
      y = y * inv * power;
      if (whole) {
        store2(row, c, x, y);
      } else {
        const int64_t to = static_cast<int64_t>(slot) * kRowTile + row;
        leave2(partial.rows + to * kDim + c, x, y);
        if (c == 0) {
          const float2 part = part_sum(sum_top, sum);
          leave2(partial.sums + 2 * to, part.x, part.y);
        }
      }
    }
    lds_barrier();

    if (!whole) {
      const int seg_begin = share.unit - step;
      const int first = share.worker_of(seg_begin), last = share.worker_of(seg_begin + seg_steps - 1);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      lds_barrier();
      if (tid == 0)
        arrived = __hip_atomic_fetch_add(partial.count + first, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      lds_barrier();
      if (arrived == last - first) {
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        if (tid == 0) __hip_atomic_store(partial.count + first, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        // Four channels of every row, and where they leave threads over, several threads a four's parts.
        // The parts' sums go through LDS where it holds them.
        const int parts = last - first + 1;
        const auto row_from = [&](int i, int row) { return static_cast<int64_t>(2 * (first + i) + (i == 0)) * kRowTile + row; };
        float2* const staged = reinterpret_cast<float2*>(&joined[0][0][0]);
        const bool fits = parts * rows <= kRowWaves * 16 * kPitch / 2;
        if (fits)
          for (int i = tid; i < parts * rows; i += kThreads) {
            const int part = i / rows;
            staged[i] = take2(partial.sums + 2 * row_from(part, i - part * rows));
          }
        lds_barrier();
        constexpr int kFours = kDim / 4;
        const int items = rows * kFours;
        const int teams = items >= kThreads ? 1 : kThreads / items;
        for (int item0 = 0; item0 < items; item0 += kThreads) {
          const int item = item0 + (teams == 1 ? tid : tid % items), team = teams == 1 ? 0 : tid / items;
          const bool busy = item < items && team < teams;
          const int row = busy ? item / kFours : 0, c = 4 * (item % kFours);
          const auto sum_of = [&](int i) { return fits ? staged[i * rows + row] : take2(partial.sums + 2 * row_from(i, row)); };
          f32x4 x = {0.f, 0.f, 0.f, 0.f};
          float sum = 0.f;
          if (busy) {
            float top = -INFINITY;
            for (int i = 0; i < parts; ++i) top = fmaxf(top, sum_of(i).x);
            const float base = join_base(top, kRowsWorkers);
            constexpr int kBatch = 8;  // parts on their way at once
            for (int i0 = team; i0 < parts; i0 += kBatch * teams) {
              f32x4 v[kBatch];
#pragma unroll
              for (int k = 0; k < kBatch; ++k) {
                const int i = i0 + k * teams;
                v[k] = *reinterpret_cast<const f32x4*>(partial.rows + row_from(i < parts ? i : i0, row) * kDim + c);
              }
#pragma unroll
              for (int k = 0; k < kBatch; ++k) {
                const int i = i0 + k * teams;
                const float2 s = sum_of(i < parts ? i : i0);
                const float w = i < parts ? s.y * exp2_fast(s.x - base) : 0.f;
                sum += w;
                x += v[k] * w;
              }
            }
          }
          if (teams > 1) {
            *reinterpret_cast<f32x4*>(team_sums[tid]) = x;
            team_sums[tid][4] = sum;
            lds_barrier();
            if (team == 0)
              for (int k = 1; k < teams; ++k) {
                x += *reinterpret_cast<const f32x4*>(team_sums[k * items + item]);
                sum += team_sums[k * items + item][4];
              }
          }
          if (busy && team == 0) {
            const float inv = sum != 0.f ? 1.f / sum : 0.f;
            store2(row, c, x[0] * inv, x[1] * inv);
            store2(row, c + 2, x[2] * inv, x[3] * inv);
          }
        }
        lds_barrier();
      }
    }

    share.unit += step_end - step;
    if (share.unit >= share.end) break;
    share.step = 0;
    if (++share.segment == tiles_of(p, share.request) * p.cache.heads) {
      share.segment = 0;
      do {
        if (++share.b >= p.batch.n_seqs) return;
        share.request = request_at(p.batch, share.b);
      } while (share.request.end == share.request.begin);
      share.request = Request{uniform(share.request.begin), uniform(share.request.end), uniform(share.request.pos0)};
      seg_steps = share.cut ? steps_of(p, layout, held, share.request) : 1;
    }
  }
}

template <typename T, int kDim>
static hipError_t launch_rows_as(const CacheAttendParams& p, const RowsLayout& layout, float* workspace, hipStream_t stream) {
  Partials partial;
  partial.count = reinterpret_cast<int*>(workspace);
  partial.rows = workspace + kCounterBytes / sizeof(float);
  partial.sums = partial.rows + static_cast<int64_t>(2) * layout.most_workers * kRowTile * kDim;
  hipLaunchKernelGGL((cache_attend_rows_kernel<T, kDim>), dim3(layout.most_workers), dim3(kThreads), 0, stream, p, layout,
                     partial);
  return hipGetLastError();
}

hipError_t launch_attend_rows(bool bf16, int head_dim, const CacheAttendParams& p, int workers, int step_log2,
                              float* workspace, hipStream_t stream) {
  const RowsLayout layout{workers, step_log2};
  if (bf16)
    return head_dim == 128 ? launch_rows_as<uint16_t, 128>(p, layout, workspace, stream)
           : head_dim == 64 ? launch_rows_as<uint16_t, 64>(p, layout, workspace, stream)
                            : launch_rows_as<uint16_t, 32>(p, layout, workspace, stream);
  return head_dim == 128 ? launch_rows_as<float, 128>(p, layout, workspace, stream)
         : head_dim == 64 ? launch_rows_as<float, 64>(p, layout, workspace, stream)
                          : launch_rows_as<float, 32>(p, layout, workspace, stream);
}

}  // namespace scd
