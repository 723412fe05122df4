// Host helpers shared by the library's translation units: the per-thread error
// message behind la_last_error_message() and the launch check.
#pragma once
#include <stdint.h>

#include "linattn.h"

namespace la {
namespace host {

// Records the message and returns s.
__attribute__((visibility("hidden"), format(printf, 2, 3))) la_status fail(la_status s, const char *fmt, ...);

// Turns a pending HIP error (a failed launch) into LA_ERR_HIP.
__attribute__((visibility("hidden"))) la_status hip_check(const char *what);

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace host
}  // namespace la
