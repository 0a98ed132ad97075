// The error report shared by the library's translation units.
#pragma once
#include "m2r2.h"

namespace m2r2 {

// Keeps the message for m2r2_last_error() on this thread and returns `st`.
m2r2_status set_error(m2r2_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

}  // namespace m2r2
