// What the entry points of every file check and report with (api.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "cac.h"

namespace cac {

// sets the message of cac_last_error() and returns `code`
int fail(int code, const char *fmt, ...);
int check_ptr(const void *p, const char *name);
int check_ws(size_t need, const void *ws, size_t ws_bytes);
bool share_memory(const void *a, size_t a_bytes, const void *b, size_t b_bytes);
int launched(hipError_t e, const char *what);

// A call's buffers: the first `outputs` are written, the others are read or are workspace.  No output may share memory with another
// buffer (null and empty ones are left out).
struct Buffer {
    const void *p;
    size_t bytes;
    const char *name;
};
inline int check_apart(const Buffer *b, int outputs, int all)
{
    for (int i = 0; i < outputs; ++i)
        for (int k = i + 1; k < all; ++k)
            if (b[i].p && b[k].p && b[k].bytes && share_memory(b[i].p, b[i].bytes, b[k].p, b[k].bytes))
                return fail(CAC_ERR_INVALID_ARG, "%s shares memory with %s", b[i].name, b[k].name);
    return CAC_OK;
}

inline size_t bytes_of(int dtype) { return dtype == CAC_F32 ? 4 : 2; }
// of a matrix of rows, from its first number to behind its last
inline size_t rows_bytes(long rows, long columns, long ld, size_t e) { return ((size_t)(rows - 1) * ld + columns) * e; }

} // namespace cac
