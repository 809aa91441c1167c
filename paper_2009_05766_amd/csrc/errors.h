// What the files of the C ABI share: the text of the last error that has no context.
#pragma once
#include "../../include/netmax.h"

// Records `msg` for netmax_last_error(NULL) on this thread and returns `code`.
int netmax_fail(int code, const char *msg) noexcept;
