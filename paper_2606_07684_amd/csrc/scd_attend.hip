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
  //   1 request behind  1000   8 14.0 / 18.4   16 15.8 / 19.4   32  17.0 / 21.8   64  17.3 / 27.2
  //   1 request behind  8000                                    32  42.3 / 36.0   64  56.4 / 41.8
  //   1 request behind 30000                                    32  81.3 / 52.8   64 127.9 / 86.8
  //   16 requests, 1000        8 19.3 / 37.1   16 26.4 / 39.5   32  47.6 / 45.2   64  89.1 / 52.0
  //   64 requests, 1000        8 52.7 / 68.7   16 97.1 / 70.6   32 182.1 / 86.2   64 350.5 / 118.2
  // What a request holds already is known on the device only, so it is not part of the rule.
  const int64_t mean = b.n_tokens * group / requests;
  const bool prompt = bf16 && head_dim >= 64 && mean >= kPromptRows / 2;
  plan.rows = prompt ? kPromptRows : kRowTile;
  plan.tiles = b.n_tokens * group / plan.rows + requests;
  const int64_t positions = static_cast<int64_t>(c.cols) * c.page, segments = plan.tiles * c.heads;
  const size_t row = static_cast<size_t>(head_dim + 2) * sizeof(float);
  if (prompt) {
    // Shares of at least 256 positions, as many as give the chip's 256 CUs a workgroup each.
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
