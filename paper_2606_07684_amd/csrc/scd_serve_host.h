// Argument checks that the serving operators' entry points share.
#pragma once

#include "scd_host.h"
#include "scd_serve.h"

namespace scd {

scd_status_t check_dtype(int32_t dtype);
scd_status_t check_rotary(const scd_rotary_t* r);
scd_status_t check_table(const void* table, int64_t max_position);
// Strided rows of `heads` heads (0: any positive number).  `written`: no two elements may share an
// address.
scd_status_t check_rows(const scd_rows_t* r, const char* name, int32_t heads, int32_t head_dim,
                        int32_t dtype, int64_t n_tokens, bool written);
Rows rows_of(const scd_rows_t* r, int32_t dtype);
SeqBatch batch_of(const scd_batch_t* b);
Turn turn_of(const scd_rotary_t* r, const void* table, int64_t max_position);
scd_status_t launched(hipError_t e, const char* what);

}  // namespace scd
