// Internal declarations of the latent cache, of attention over it and over dense rows.
#pragma once

#include "scd_serve.h"

namespace scd {

// Rows of one latent and one rotated key that all heads share.
struct LatentPages {
  char* pages;          // [n_pages][page][width], channels [0, latent) and [latent, width)
  const int32_t* table; // [n_seqs][cols]
  int32_t n_pages, cols;
  int32_t page, page_log2;
  int32_t latent, turned;
};

struct LatentAppendParams {
  LatentPages cache;
  SeqBatch batch;
  Rows c, k;            // one head each
  Turn turn;            // table null: keys as they are
};

struct LatentExpandParams {
  LatentPages cache;
  SeqBatch batch;
  Rows k, v;
  const char* w_k;      // [heads][plain][latent]
  const char* w_v;      // [heads][value][latent]
  int32_t heads, plain, value;
};

// How the positions that a call's tiles of query rows attend to are cut into shares, one a workgroup.
struct SharePlan {
  int32_t rows;         // query rows of a tile
  int32_t row_groups;   // waves side by side over a tile's rows
  int32_t heads;        // KV heads, each with tiles of its own
  int32_t per_token;    // query rows a token has in a tile's head
  int32_t cut;          // whether tiles are cut at all
  int32_t fill;         // workgroups that fill the chip: its 256 CUs, times those that one holds at once
  int32_t whole;        // tiles from which on none is cut
  int64_t cap;          // positions a request can hold
  int64_t grid;         // workgroups launched: a bound on the shares
};

// Shares that fewer than `whole` tiles may be cut into: a multiple of the workgroups that fill the chip, two a tile at
// least.
__host__ __device__ inline int64_t share_goal(int64_t tiles, int fill) {
  return static_cast<int64_t>((2 * static_cast<uint32_t>(tiles) + fill - 1) / fill) * fill;
}

// A query row's shares in the workspace, left by the first of them: share s is slot first + s * step.
struct RowParts {
  int32_t first, step, count, row;
};

// What a workgroup of attention over latents takes: a tile of a request's query rows and a share of its positions.
struct LatentShare {
  int32_t b, tokens;    // request (-1: nothing), its new tokens
  int32_t tile, tiles, part, parts;
  int32_t first;        // slot of the tile's first share
  int32_t pad;
  int64_t begin, held;  // first packed row, tokens held before
};

// Elements of an absorbed query: latent and turned channels, in bf16 the latent ones' second summands behind them.
__host__ __device__ inline int query_width(bool bf16, int latent, int turned) {
  return bf16 ? 2 * latent + turned : latent + turned;
}

struct LatentAttendParams {
  LatentPages cache;
  SeqBatch batch;
  SharePlan plan;
  Rows q, out;
  const char* w_k;
  const char* w_v;
  int32_t heads, plain, value;
  float scale;          // of the scores, times log2(e)
  char* zeros;          // 256 bytes of them
  char* absorbed;       // [n_tokens * heads][query_width]
  LatentShare* shares;  // [grid]
  RowParts* parts;      // [n_tokens * heads]
  float* slots;         // [grid][rows][latent + 2]
};

struct RowsAttendParams {
  SeqBatch batch, held; // of query rows, of key and value rows
  SharePlan plan;
  Rows q, k, v, out;
  int32_t key, value;   // channels
  float scale;
  RowParts* parts;      // [n_tokens * n_heads]; null: nothing is cut
  float* slots;
};

hipError_t launch_latent_append(bool bf16, const LatentAppendParams& p, hipStream_t stream);
hipError_t launch_latent_expand(bool bf16, const LatentExpandParams& p, hipStream_t stream);

// Positions of a block of attention over latents.
__host__ __device__ constexpr int latent_block(bool bf16) { return bf16 ? 64 : 32; }

// Absorbed queries, attention over the latents, the shares' join with the value matrices applied.
struct LatentSizes {
  SharePlan plan;
  size_t zeros, absorbed, shares, parts, slots;  // bytes of the workspace
  size_t total() const { return zeros + absorbed + shares + parts + slots; }
};
LatentSizes latent_sizes(bool bf16, const LatentPages& c, const SeqBatch& b, int heads);
hipError_t launch_latent_attend(bool bf16, const LatentAttendParams& p, hipStream_t stream);
hipError_t launch_latent_core(bool bf16, const LatentAttendParams& p, hipStream_t stream);
hipError_t launch_latent_core_bf16(const LatentAttendParams& p, hipStream_t stream);
hipError_t launch_latent_core_f32(const LatentAttendParams& p, hipStream_t stream);

struct RowsSizes {
  SharePlan plan;
  size_t parts, slots;
  size_t total() const { return parts + slots; }
};
// Rows that are fetched 16 bytes at a time, a block's from its first one on in 32 bits.
inline bool rows_wide(const Rows& k, const Rows& v) {
  return k.wide && v.wide && k.token < (int64_t{1} << 22) && v.token < (int64_t{1} << 22);
}
RowsSizes rows_sizes(bool bf16, bool wide, const SeqBatch& b, int64_t held_rows, int heads, int kv_heads, int value);
hipError_t launch_rows_attend(bool bf16, const RowsAttendParams& p, hipStream_t stream);

}  // namespace scd
