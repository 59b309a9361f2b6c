// The calling thread's last error (sdnn_last_error), shared by the sources of the C ABI.
#pragma once

#include "sdnn.h"

namespace sdnn {

sdnn_status set_error(sdnn_status s, const char *msg) noexcept;  // records the text and returns s

}  // namespace sdnn
