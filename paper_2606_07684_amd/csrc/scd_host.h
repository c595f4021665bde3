// Host-side helpers shared by the C ABI's translation units.
#pragma once

#include "../../include/scd.h"

namespace scd {

// Records the detail of a non-OK status for scd_last_error and returns the status.
scd_status_t fail(scd_status_t s, const char* fmt, ...);
// Clears the detail and returns SCD_OK.
scd_status_t ok();
bool aligned16(const void* p);
scd_status_t check_batch(const scd_batch_t* b);

}  // namespace scd

#define SCD_TRY(expr)                  \
  do {                                 \
    const scd_status_t s_ = (expr);    \
    if (s_ != SCD_OK) return s_;       \
  } while (0)
