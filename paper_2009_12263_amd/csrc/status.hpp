// What the host files of the library share: the message of a failing call and checks of pointers.
#pragma once
#include <stdint.h>

#include "../../include/flexgemm.h"

namespace fg {

// Notes the message that fg_last_error() returns and gives the status back.
fg_status fail(fg_status st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

inline bool aligned_to(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace fg
