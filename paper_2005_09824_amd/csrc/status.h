// What an entry point returns when it refuses: the status, with lfmmi_last_error()'s text set.
#pragma once
#include <hip/hip_runtime.h>

#include <string>

#include "../../include/lfmmi.h"

namespace lfmmi {

lfmmi_status fail(lfmmi_status st, const std::string& msg);
lfmmi_status fail_hip(hipError_t e, const char* what);
lfmmi_status fail_memory() noexcept;  // host memory, where an exception must not leave

}  // namespace lfmmi
