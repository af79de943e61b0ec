// Checks that the entry points of tperm_experts.h and tperm_decode.h share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tperm_experts.h"

namespace tperm {

constexpr int64_t kRowsMax = ((int64_t)1 << 31) - 1;
// A product's operand that is reached with 32-bit offsets.
constexpr int64_t kOperandBytes = ((int64_t)1 << 32) - 256;

inline bool known_type(int type) { return type == TPERM_TYPE_F32 || type == TPERM_TYPE_F16 || type == TPERM_TYPE_BF16; }
inline bool known_width(int64_t w) { return w >= 1 && w <= TPERM_WIDTH_MAX; }
inline bool known_stride(int64_t stride, int64_t width) { return stride >= width && stride <= (int64_t)1 << 28; }

// tokens * slots, or a status.
inline tperm_status_t count_rows(int64_t tokens, int64_t slots, int64_t experts, int64_t* rows) {
    if (tokens < 0 || slots < 1 || slots > TPERM_SLOTS_MAX || experts < 1 || experts > TPERM_EXPERTS_MAX) return TPERM_ERR_DIMS;
    if (tokens > kRowsMax || tokens * slots > kRowsMax) return TPERM_ERR_TOO_LARGE;
    *rows = tokens * slots;
    return TPERM_OK;
}

// An array of a call.
struct Array {
    const void* p;
    int64_t bytes;      // from the first to behind the last byte that is looked at
    size_t align;
    bool written;
    bool absent() const { return bytes == 0; }
};
inline int64_t matrix_bytes(int64_t rows, int64_t stride, int64_t width, size_t elem) { return rows == 0 ? 0 : ((rows - 1) * stride + width) * (int64_t)elem; }

// NULL, ALIGN, ALIAS over all arrays of a call; those of no bytes are not looked at.
template <size_t N> inline tperm_status_t check(const Array (&a)[N]) {
    for (const Array& x : a)
        if (!x.absent() && x.p == nullptr) return TPERM_ERR_NULL;
    for (const Array& x : a)
        if (!x.absent() && (uintptr_t)x.p % x.align != 0) return TPERM_ERR_ALIGN;
    for (size_t i = 0; i < N; ++i)
        for (size_t j = 0; j < N; ++j) {
            if (i == j || !a[i].written || a[i].absent() || a[j].absent()) continue;
            const uintptr_t p = (uintptr_t)a[i].p, q = (uintptr_t)a[j].p;
            if (p < q + (uintptr_t)a[j].bytes && q < p + (uintptr_t)a[i].bytes) return TPERM_ERR_ALIAS;
        }
    return TPERM_OK;
}

inline tperm_status_t launched(hipError_t e) {
    if (e == hipSuccess) return TPERM_OK;
    (void)hipGetLastError();
    return TPERM_ERR_HIP;
}

}  // namespace tperm
