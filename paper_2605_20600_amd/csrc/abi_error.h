// The error message of the C ABI, shared by the files that hold entry points.
#pragma once

#include <string>

#include "../../include/headkv.h"

namespace headkv {

// Keeps `msg` for headkv_last_error() on this thread and returns `code`.
headkv_status set_error(headkv_status code, const std::string& msg);

}  // namespace headkv
