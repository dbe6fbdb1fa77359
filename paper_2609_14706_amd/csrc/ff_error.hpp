// The message that ff_last_error gives, for entry points outside ff_engine.hip.
#pragma once

#include "ff.h"

namespace ff {
// Records msg as this thread's last error and returns s.
ff_status report(ff_status s, const char* msg) noexcept;
}  // namespace ff
