// Status codes with their thread-local text (uf_last_error), shared by the C ABI's
// translation units.
#pragma once

#include "uf.h"

namespace uf {

__attribute__((format(printf, 2, 3))) int fail(int status, const char* fmt, ...);
int ok();

}  // namespace uf
