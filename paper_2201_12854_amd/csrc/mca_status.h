// What the sources of the C ABI share: status with a reason, alignment (internal to libmca).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "mca.h"

namespace mca {

// Keeps the reason for mca_last_error of this thread and returns st.
mca_status fail(mca_status st, const char* fmt, ...);
// Clears it and returns MCA_OK.
mca_status ok();

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t align256(size_t v) { return (v + 255) & ~size_t(255); }

}  // namespace mca
