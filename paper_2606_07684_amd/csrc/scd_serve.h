// Internal declarations of the serving operators: rotary positions, the paged 8-bit cache and
// attention over it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace scd {

// A packed batch of new tokens: request b owns rows [cu[b], cu[b + 1]) and holds pos0[b] tokens.
struct SeqBatch {
  const int32_t* cu;    // [n_seqs + 1] or null (one request)
  const int32_t* pos0;  // [n_seqs] or null
  int64_t n_tokens;
  int32_t n_seqs;
};

// Strided rows: channel c of head h of token t is data[t * token + h * head + c].
struct Rows {
  char* data;
  int64_t token, head;  // elements
  int32_t n_heads;
  int32_t wide;         // every row starts on 16 bytes
};

struct PagedCache {
  int8_t* k;            // [n_pages][heads][page][d]
  int8_t* v;
  float* k_scale;       // [n_pages][heads]
  float* v_scale;
  const int32_t* table; // [n_seqs][cols]
  int32_t n_pages, heads, cols;
  int32_t page, page_log2;
};

struct Turn {           // rotary positions
  const float2* table;  // [max_pos][dim / 2] (cos, sin); null: rows are taken as they are
  int64_t max_pos;
  int32_t dim;
  int32_t interleaved;
};

struct RotaryParams {
  Rows in[2], out[2];   // queries, keys (n_heads 0: none)
  SeqBatch batch;
  Turn turn;
  int32_t head_dim;
  int32_t transpose;
};

struct CacheAppendParams {
  PagedCache cache;
  SeqBatch batch;
  Rows rows[2];         // keys, values
  Turn turn;            // of the keys
};

struct CacheReadParams {
  PagedCache cache;
  SeqBatch batch;
  Rows rows[2];
};

// Division of 0 <= n < 2^31 by a number known on the host: a product, a sum and a shift.
struct FastDiv {
  uint32_t mul = 1, shift = 0;
  FastDiv() = default;
  explicit FastDiv(uint32_t d) {
    while ((uint64_t{1} << shift) < d) ++shift;
    mul = static_cast<uint32_t>((((uint64_t{1} << shift) - d) << 32) / d + 1);
  }
  __device__ int of(int n) const {
    return static_cast<int>((__umulhi(static_cast<uint32_t>(n), mul) + static_cast<uint32_t>(n)) >> shift);
  }
};

struct CacheAttendParams {
  PagedCache cache;
  SeqBatch batch;
  Rows q, out;
  int32_t group;        // query heads per KV head
  float scale;
  FastDiv by_group, by_heads;  // by group, by cache.heads
};

constexpr int kMaxTurnPairs = 256;
struct TurnTableParams {
  double w[kMaxTurnPairs];  // radians per position
  double gain;
  float2* table;
  int64_t n;                // entries
  int32_t pairs;
};
static_assert(sizeof(TurnTableParams) <= 4096, "kernel argument block");

hipError_t launch_turn_table(const TurnTableParams& p, hipStream_t stream);
hipError_t launch_rotary(bool bf16, const RotaryParams& p, hipStream_t stream);
hipError_t launch_cache_append(bool bf16, int head_dim, const CacheAppendParams& p,
                               hipStream_t stream);
hipError_t launch_cache_read(bool bf16, int head_dim, const CacheReadParams& p, hipStream_t stream);

// A few rows of every request in `workers` workgroups, steps of 2^step_log2 blocks, or whole prompts (bf16,
// head_dim 64 or 128) in up to `splits` shares of each of `tiles` tiles and KV head.
hipError_t launch_attend_rows(bool bf16, int head_dim, const CacheAttendParams& p, int workers, int step_log2,
                              float* workspace, hipStream_t stream);
hipError_t launch_attend_prompt(int head_dim, const CacheAttendParams& p, int64_t tiles, int splits, float* workspace,
                                hipStream_t stream);
size_t attend_workspace(const PagedCache& c, const SeqBatch& b, int group, int head_dim);
hipError_t launch_cache_attend(bool bf16, int head_dim, const CacheAttendParams& p,
                               void* workspace, hipStream_t stream);

}  // namespace scd
