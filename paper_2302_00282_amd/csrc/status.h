// The message that xenos_last_error() gives, shared by the host sources behind the C ABI.
#pragma once
#include "../../include/xenos.h"

namespace xenos {

// Records the message for this thread and returns `st`.
__attribute__((format(printf, 2, 3))) xenos_status fail(xenos_status st, const char* fmt, ...);

}  // namespace xenos
