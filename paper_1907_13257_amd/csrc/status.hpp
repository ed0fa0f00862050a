// status.hpp -- status codes and the calling thread's error detail, shared by
// the translation units that define entry points of the C ABI (api.cpp,
// operators.cpp).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/lstm355.h"

namespace lstm355 {

// Each sets the detail that lstm_last_error_detail returns.
lstm_status_t hip_status(const char *what, hipError_t e);   // LSTM_OK for hipSuccess
lstm_status_t invalid(const char *what);
lstm_status_t short_buffer(const char *what, size_t given, size_t need);

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned8(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace lstm355

#define TRY_HIP(what, expr)                                  \
    do {                                                     \
        hipError_t e_ = (expr);                              \
        if (e_ != hipSuccess) return hip_status(what, e_);   \
    } while (0)
