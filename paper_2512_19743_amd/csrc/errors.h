// The calling thread's error text (apml_last_error), for the entry points
// outside api.hip.
#pragma once

#include "../../include/apml.h"

namespace apml {

apml_status fail_with(apml_status st, const char *msg);
void clear_error();

} // namespace apml
