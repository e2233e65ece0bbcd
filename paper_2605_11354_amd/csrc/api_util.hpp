// What the files of the C ABI share: the description of the last failure, pointer checks, workspace slices.
#pragma once
#include "../../include/sla.h"
#include "sla_common.hpp"

#include <stddef.h>

namespace sla {

// records the description that sla_last_error() returns on this thread and passes the status on
__attribute__((visibility("hidden"))) sla_status_t fail(sla_status_t st, const char *fmt, ...);

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }
template <class T> T *at(void *ws, size_t off) { return (T *)((char *)ws + off); }

}  // namespace sla

#define SLA_REQ_PTR(ptr)                                                                              \
    do {                                                                                              \
        if (!(ptr)) return fail(SLA_ERR_INVALID_ARG, #ptr " is NULL");                                \
        if (!aligned((ptr), 16)) return fail(SLA_ERR_INVALID_ARG, #ptr " must be 16-byte aligned");   \
    } while (0)
#define SLA_OPT_PTR(ptr)                                                                              \
    do {                                                                                              \
        if ((ptr) && !aligned((ptr), 16)) return fail(SLA_ERR_INVALID_ARG, #ptr " must be 16-byte aligned"); \
    } while (0)
#define SLA_HIP(call)                                                                                 \
    do {                                                                                              \
        hipError_t e_ = (call);                                                                       \
        if (e_ != hipSuccess) return fail(SLA_ERR_HIP, "%s failed: %s", #call, hipGetErrorString(e_)); \
    } while (0)
