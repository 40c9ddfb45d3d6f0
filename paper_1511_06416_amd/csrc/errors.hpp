// The calling thread's last error message (same_last_error), shared by the
// translation units of the C ABI.
#pragma once

#include <string>

namespace same {

// Records msg and returns code.
int record_error(int code, const std::string &msg);

}  // namespace same
