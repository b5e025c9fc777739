// Errors of the operators that need no encoder handle: a status, and the message that
// epd_op_last_error() returns on the calling thread.
#pragma once

#include "../../include/epd_encode.h"
#include "epd_internal.h"

namespace epd {
epd_status op_fail(epd_status status, const char* format, ...) __attribute__((format(printf, 2, 3)));
// EPD_ERR_HIP for the launch that returned e.  The runtime keeps e as its last error as well: taken from there, so that the program's next
// look at it finds no failure that was reported already.
epd_status op_launch_failed(const char* who, hipError_t e);
}  // namespace epd
