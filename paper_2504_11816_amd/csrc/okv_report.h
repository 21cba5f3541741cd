// Where entry points outside okv_api.hip leave the message that okv_last_error(NULL) returns.
#pragma once

namespace okv {

// Records the message and returns `code`.
int report(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

}  // namespace okv
