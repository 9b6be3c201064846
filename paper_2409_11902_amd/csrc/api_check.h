// What the entry points of every file check and report with (api.hip).
#pragma once
#include <hip/hip_runtime.h>

namespace cac {

// sets the message of cac_last_error() and returns `code`
int fail(int code, const char *fmt, ...);
int check_ptr(const void *p, const char *name);
int check_ws(size_t need, const void *ws, size_t ws_bytes);
bool share_memory(const void *a, size_t a_bytes, const void *b, size_t b_bytes);
int launched(hipError_t e, const char *what);

} // namespace cac
