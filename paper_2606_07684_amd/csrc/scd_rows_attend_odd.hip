// Causal attention over dense rows that do not start on 16 bytes.
#include "scd_rows_attend.h"

namespace scd {

hipError_t launch_odd_rows(bool bf16, const RowsAttendParams& p, hipStream_t stream) {
  return bf16 ? launch_rows_as<uint16_t, 1, false>(p, stream) : launch_rows_as<float, 1, false>(p, stream);
}

}  // namespace scd
