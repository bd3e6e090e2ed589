// The error message of calls that have no context.
#pragma once

#include "dsm.h"

namespace dsm {

// Records the message that dsm_last_error(NULL) returns on this thread, and
// returns the status (dsm_runtime.cpp).
dsm_status set_thread_error(dsm_status st, const char* message);

}  // namespace dsm
