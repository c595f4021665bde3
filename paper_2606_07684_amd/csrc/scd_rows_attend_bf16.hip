// Causal attention over dense bf16 rows.
#include "scd_rows_attend.h"

namespace scd {

hipError_t launch_rows_bf16(const RowsAttendParams& p, hipStream_t stream) {
  return p.plan.rows == 128 ? launch_rows_as<uint16_t, 2, true>(p, stream) : launch_rows_as<uint16_t, 1, true>(p, stream);
}

}  // namespace scd
