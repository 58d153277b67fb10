// Shared by the host-side files of the C ABI: error reports and the checks of what every call brings.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/sparsed.h"

namespace sparsed {

// Sets the thread's error message and returns the status.
sparsed_status fail(sparsed_status st, const char* fmt, ...);
sparsed_status hip_fail(hipError_t e, const char* what);
// The caller's workspace, checked: present, large enough, 256-byte aligned.
sparsed_status caller_workspace(const sparsed_exec* ex, size_t need, const char* what, char** out);

}  // namespace sparsed
