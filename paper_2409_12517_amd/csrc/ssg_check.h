// What the entry points share: the error text, the checks of arguments.  Host code.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/ssg.h"

namespace ssg {
constexpr size_t kErrorText = 512;
char *error_text();                  // this thread's, kErrorText bytes
}

namespace {

[[maybe_unused]] ssg_status fail(ssg_status code, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(ssg::error_text(), ssg::kErrorText, fmt, ap);
    va_end(ap);
    return code;
}

[[maybe_unused]] bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
[[maybe_unused]] bool extent_ok(int64_t v) { return v > 0 && (v % 16) == 0; }

[[maybe_unused]] ssg_status check_launch(const char *what) {
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(SSG_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    return SSG_OK;
}

// An error some earlier HIP call of the process left behind would otherwise be reported as this entry
// point's own launch failure: it is read (which clears it) and reported before anything is enqueued.
[[maybe_unused]] ssg_status check_entry(const char *what) {
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return fail(SSG_ERR_HIP, "%s: a HIP error was already pending on entry (%s); nothing was launched", what,
                    hipGetErrorString(e));
    return SSG_OK;
}

#define SSG_REQUIRE_PTR(p)                                                                     \
    do {                                                                                       \
        if ((p) == nullptr) return fail(SSG_ERR_ARG, "%s: %s is NULL", __func__, #p);          \
        if (!aligned16(p)) return fail(SSG_ERR_ARG, "%s: %s is not 16-byte aligned", __func__, #p); \
    } while (0)
#define SSG_OPTIONAL_PTR(p)                                                                    \
    do {                                                                                       \
        if ((p) != nullptr && !aligned16(p))                                                   \
            return fail(SSG_ERR_ARG, "%s: %s is not 16-byte aligned", __func__, #p);           \
    } while (0)
#define SSG_REQUIRE_SCALAR_PTR(p)                                                              \
    do {                                                                                       \
        if ((p) == nullptr) return fail(SSG_ERR_ARG, "%s: %s is NULL", __func__, #p);          \
        if (reinterpret_cast<uintptr_t>(p) & 3u)                                               \
            return fail(SSG_ERR_ARG, "%s: %s is not 4-byte aligned", __func__, #p);            \
    } while (0)

[[maybe_unused]] bool dtype_ok(int dt) { return dt == SSG_BF16 || dt == SSG_F32; }
[[maybe_unused]] size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

}  // namespace
