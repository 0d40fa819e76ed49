// The library's last-error text, shared by the files that hold entry points
// of the C ABI (defined in engine.hip).
#pragma once

#include <string>

#include "archer.h"

// Record msg as the calling thread's last error and return s.
archer_status archer_fail(archer_status s, const std::string& msg);
