// The calling thread's error message (outlets_last_error), for the C entries.
#pragma once

#include <string>

namespace outlets {

// Records `msg` and returns rc.
int fail(int rc, const std::string& msg);

}  // namespace outlets
