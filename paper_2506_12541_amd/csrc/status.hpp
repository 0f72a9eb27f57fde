// The calling thread's last error (read by bsa_last_error), shared by the files that hold C
// entry points.
#pragma once
#include <string>

#include "../../include/bsa.h"

namespace bsa {

void clear_error();
bsa_status_t set_error(bsa_status_t s, const std::string& msg);   // returns s

}  // namespace bsa
