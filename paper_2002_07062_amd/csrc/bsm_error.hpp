// The thread-local message behind bsm_last_error(), for the other C-ABI sources (internal).
#pragma once

#include "bsm.h"

namespace bsm {

// Keeps `message` for bsm_last_error() and returns `st`.
bsm_status report(bsm_status st, const char* message);

}  // namespace bsm
