// Causal attention over dense fp32 rows.
#include "scd_rows_attend.h"

namespace scd {

hipError_t launch_rows_f32(const RowsAttendParams& p, hipStream_t stream) {
  return launch_rows_as<float, 1, true>(p, stream);
}

}  // namespace scd
