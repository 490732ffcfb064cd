// What the library's host files share.
#pragma once

#include "../../include/dbt.h"

namespace dbt {

// Record the message that dbt_last_error(NULL) returns in this thread, and hand the status back.
dbt_status op_error(dbt_status st, const char *fmt, ...);

}  // namespace dbt
