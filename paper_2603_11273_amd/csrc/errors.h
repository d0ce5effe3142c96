// The calling thread's error message, shared by the files that hold entry points.
#pragma once

#include <string>

#include "../../include/asr.h"

namespace asr {
// Records msg for asr_last_error and returns s.
asr_status fail(asr_status s, const std::string& msg);
}  // namespace asr
