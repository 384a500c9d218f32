// The reason of a failing call, kept for bacon_last_error().
#pragma once

#include "../../include/bacon.h"

namespace bacon {

// Keeps the reason for the calling thread and returns s.
bacon_status fail(bacon_status s, const char *fmt, ...);

}  // namespace bacon
