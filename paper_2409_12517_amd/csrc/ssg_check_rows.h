// Checks of rows and of buffers of quantized rows, shared by the entry points that take them.  Host code.
#pragma once
#include <algorithm>

#include "ssg_check.h"
#include "ssg_internal.h"

namespace {

// (an empty tensor may have no address)
[[maybe_unused]] ssg_status check_ptr(const char *who, const char *name, const void *p, size_t align, bool needed) {
    if (!p) return needed ? fail(SSG_ERR_ARG, "%s: %s is NULL", who, name) : SSG_OK;
    if (reinterpret_cast<uintptr_t>(p) & (align - 1)) return fail(SSG_ERR_ARG, "%s: %s is not %zu-byte aligned", who, name, align);
    return SSG_OK;
}
#define SSG_CHECK(call)                          \
    do {                                         \
        const ssg_status rc_ = (call);           \
        if (rc_ != SSG_OK) return rc_;           \
    } while (0)

constexpr int64_t kMaxI8K = 131056;          // 128 * 128 * K stays below 2^31
constexpr int64_t kMaxI8Rows = (int64_t)1 << 26;

[[maybe_unused]] ssg_status check_i8_shape(const char *who, int64_t rows, int64_t K) {
    if (rows < 0 || rows > kMaxI8Rows) return fail(SSG_ERR_SHAPE, "%s: %lld rows (0 to %lld)", who, (long long)rows, (long long)kMaxI8Rows);
    if (!extent_ok(K) || K > kMaxI8K) return fail(SSG_ERR_SHAPE, "%s: K = %lld must be a positive multiple of 16 up to %lld", who, (long long)K, (long long)kMaxI8K);
    return SSG_OK;
}
[[maybe_unused]] size_t i8_scale_offset(int64_t rows, int64_t K) { return align256((size_t)ssg::i8_code_bytes(rows, K)); }
[[maybe_unused]] size_t i8_bytes(int64_t rows, int64_t K) { return std::max<size_t>(i8_scale_offset(rows, K) + align256((size_t)ssg::i8_up(rows, 16) * 4), 256); }
[[maybe_unused]] const float *i8_scales(const void *q, int64_t rows, int64_t K) {
    return reinterpret_cast<const float *>(static_cast<const uint8_t *>(q) + i8_scale_offset(rows, K));
}
[[maybe_unused]] ssg_status check_i8_buffer(const char *who, const char *name, const void *q, size_t bytes, int64_t rows, int64_t K) {
    SSG_CHECK(check_ptr(who, name, q, 256, true));
    const size_t need = i8_bytes(rows, K);
    if (bytes < need) return fail(SSG_ERR_WORKSPACE, "%s: %s holds %zu bytes, %zu needed", who, name, bytes, need);
    return SSG_OK;
}
[[maybe_unused]] ssg_status check_rows_of(const char *who, const char *name, const void *p, ssg_dtype dt, int64_t rows, int64_t cols, int64_t ld) {
    if (!dtype_ok(dt)) return fail(SSG_ERR_ARG, "%s: data type %d of %s", who, (int)dt, name);
    const int64_t unit = dt == SSG_BF16 ? 8 : 4;
    if (ld < cols || ld % unit != 0 || ld > ((int64_t)1 << 31))
        return fail(SSG_ERR_SHAPE, "%s: %lld elements between rows of %s (at least %lld, rows start on 16 bytes)", who, (long long)ld, name, (long long)cols);
    return check_ptr(who, name, p, 16, rows > 0);
}

}  // namespace
