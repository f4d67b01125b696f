// The status that an entry point returns and the text of iabn_last_error.
#pragma once

#include "iabn.h"

namespace iabn_impl {

// Keeps the text for iabn_last_error on this thread; returns `code`.
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// Clears the text; returns IABN_OK.
int ok();

// The status of the launches just made, `what` for the text.
int launched(const char* what);

}  // namespace iabn_impl
