// Errors of the operators that need no encoder handle: a status, and the message that
// epd_op_last_error() returns on the calling thread.
#pragma once

#include "../../include/epd_encode.h"
#include "epd_internal.h"

namespace epd {
epd_status op_fail(epd_status status, const char* format, ...) __attribute__((format(printf, 2, 3)));
}  // namespace epd
