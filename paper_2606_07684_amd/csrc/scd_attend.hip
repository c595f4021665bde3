// Attention over the paged 8-bit cache: which kernel a call takes, and how it is laid out.
#include <algorithm>

#include "../../include/scd.h"
#include "scd_attend.h"

namespace scd {

static_assert(kCounterBytes == SCD_ATTEND_COUNTER_BYTES, "part of the workspace that is zero between calls");

// From a call's arguments alone.
struct AttendPlan {
  int rows;          // query rows of a tile
  int64_t tiles;     // bound
  int splits;        // prompts: most shares of a tile
  int workers;       // a few rows: workgroups
  int step_log2;     // a few rows: blocks of a step
  size_t bytes;      // workspace
};
static AttendPlan attend_plan(const PagedCache& c, const SeqBatch& b, int group, int head_dim, bool bf16) {
  AttendPlan plan{};
  const int64_t requests = b.n_seqs < b.n_tokens ? b.n_seqs : b.n_tokens;
  // Rows of a request and KV head, on average.  From half a tile of the prompts' kernel on it takes the call, where it
  // has the type and head_dim.  New tokens of each request, 32 heads over 8 of 128, us as a few rows / as a prompt:
  //   1 request behind  1000   8 14.7 / 19.4   16 16.0 / 20.4   32  17.2 / 22.7   64  17.4 / 28.3
  //   1 request behind  8000                                    32  40.1 / 36.4   64  54.1 / 41.1
  //   1 request behind 30000                                    32  74.8 / 49.7   64 122.1 / 83.6
  //   16 requests, 1000        8 18.4 / 37.7   16 25.2 / 39.3   32  44.0 / 44.9   64  85.5 / 50.7
  //   64 requests, 1000        8 51.3 / 69.3   16 94.8 / 71.4   32 179.4 / 82.6   64 344.1 / 111.0
  // The two sides meet at 32 tokens (128 rows) of each of 16 requests, or of one that holds some thousands of positions;
  // what a request holds is known on the device only, so it is not part of the rule.  It is on the slower side for 32 and 64
  // tokens of one request behind 1000, and for 16 of each of 64 requests.  One kernel takes all of a call: 1500 tokens of one
  // request and one of each of 63 behind 2000 take 177 us so, and 66 and 49 as two calls.
  const int64_t mean = b.n_tokens * group / requests;
  const bool prompt = bf16 && head_dim >= 64 && mean >= kPromptRows / 2;
  plan.rows = prompt ? kPromptRows : kRowTile;
  plan.tiles = b.n_tokens * group / plan.rows + requests;
  const int64_t positions = static_cast<int64_t>(c.cols) * c.page, segments = plan.tiles * c.heads;
  const size_t row = static_cast<size_t>(head_dim + 2) * sizeof(float);
  if (prompt) {
    // As many shares as give the chip's 256 CUs a workgroup each, but no more than one for every 256 positions.
    const int64_t most = (positions + 255) / 256, want = (256 + segments - 1) / segments;
    plan.splits = static_cast<int>(std::min<int64_t>(std::min(want, most), kMostSplits));
    if (plan.splits > 1) plan.bytes = kCounterBytes + segments * plan.splits * plan.rows * row;
    return plan;
  }
  const auto steps = [&] { return (positions + (int64_t{32} << plan.step_log2) - 1) >> (5 + plan.step_log2); };
  while (1 << plan.step_log2 < kRowWaves) ++plan.step_log2;
  while (segments * steps() >= int64_t{1} << 31 && steps() > 1) ++plan.step_log2;  // the kernel counts in 31 bits
  const int64_t able = steps() <= kUncutSteps ? segments : segments * std::min<int64_t>(steps(), kMostParts);
  plan.workers = static_cast<int>(std::min<int64_t>(able, kRowsWorkers));
  if (steps() > kUncutSteps) plan.bytes = kCounterBytes + 2 * plan.workers * plan.rows * row;
  return plan;
}

size_t attend_workspace(const PagedCache& c, const SeqBatch& b, int group, int head_dim) {
  return std::max(attend_plan(c, b, group, head_dim, false).bytes, attend_plan(c, b, group, head_dim, true).bytes);
}

hipError_t launch_cache_attend(bool bf16, int head_dim, const CacheAttendParams& p, void* workspace,
                               hipStream_t stream) {
  const AttendPlan plan = attend_plan(p.cache, p.batch, p.group, head_dim, bf16);
  float* ws = static_cast<float*>(workspace);
  if (plan.rows == kPromptRows) return launch_attend_prompt(head_dim, p, plan.tiles, plan.splits, ws, stream);
  return launch_attend_rows(bf16, head_dim, p, plan.workers, plan.step_log2, ws, stream);
}

}  // namespace scd
