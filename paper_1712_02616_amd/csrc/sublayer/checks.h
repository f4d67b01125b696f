// Checks of arguments that the sublayer's entry points share.
#pragma once

#include <stdint.h>

#include "errors.h"

namespace iabn_impl {

inline bool valid_dtype(int dtype) { return dtype == IABN_F32 || dtype == IABN_F16 || dtype == IABN_BF16; }

inline int elem_bytes(int dtype) { return dtype == IABN_F32 ? 4 : 2; }

inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int check_workspace(const void* workspace, size_t bytes, size_t need) {
    if (need == 0) return IABN_OK;
    if (!workspace) return fail(IABN_ERR_NULL, "workspace is NULL");
    if (bytes < need)
        return fail(IABN_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", bytes, need);
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
        return fail(IABN_ERR_WORKSPACE, "workspace is not 16-byte aligned");
    return IABN_OK;
}

}  // namespace iabn_impl
