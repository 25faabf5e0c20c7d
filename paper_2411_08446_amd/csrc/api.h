// What the files with entry points share: the calling thread's error text and checks of arguments (internal to the library).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/lshmoe.h"

namespace lshmoe {

// Records the description that lshmoe_last_error returns, and returns the status.
lshmoe_status fail(lshmoe_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
lshmoe_status ok();   // clears it
lshmoe_status hip_fail(const char* what, hipError_t e);

inline bool dtype_ok(int dt) { return dt == LSHMOE_F32 || dt == LSHMOE_BF16; }
inline size_t item_size(int dt) { return dt == LSHMOE_BF16 ? 2 : 4; }

constexpr int64_t kMaxAssignments = (int64_t)1 << 30;

// dtype known, rows of whole 16-byte pieces
lshmoe_status check_row(int d, int dt);

}  // namespace lshmoe
