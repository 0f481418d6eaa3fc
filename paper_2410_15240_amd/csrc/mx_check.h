// Argument checks that the C entries of the microscaled operators share. Internal to the library.
#pragma once
#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdarg>
#include <cstdio>

#include "fastrack.h"
#include "mx.h"

#define FT_EXPORT extern "C" __attribute__((visibility("default")))

namespace fastrack {
namespace check {

inline int fail(int code, const char *fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return set_error(code, buf);
}

inline int done(hipError_t e, const char *what)
{
    return e == hipSuccess ? FASTRACK_OK : fail(FASTRACK_EHIP, "%s: %s", what, hipGetErrorString(e));
}

inline hipStream_t as_stream(void *s) { return reinterpret_cast<hipStream_t>(s); }

constexpr uint64_t kMaxDim = 0x7FFFFFFFull;

// Compute units of the current device. A plan does not depend on having one: without a
// device the workspace of this GPU's 256 is told.
inline int num_cu()
{
    static std::atomic<int> cache[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64)
        return 256;
    n = cache[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0)
            return 256;
        cache[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

// The bytes of an operand: [b, e), and where they are rows with gaps, the rows' stride and width.
struct Span {
    const char *name;
    uintptr_t b, e;
    uint64_t ld = 0, width = 0;
};

inline Span rows_span(const char *name, const void *p, uint64_t ld, uint64_t rows, uint64_t cols, uint32_t type)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    const uint64_t size = mx_type_size(type), n = rows && cols ? ((rows - 1) * ld + cols) * size : 0;
    return {name, b, b + n, ld * size, cols * size};
}

inline Span codes_span(const char *name, const void *p, uint32_t fmt, uint64_t rows, uint64_t cols)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return {name, b, b + rows * mx_blocks(cols) * mx_block_bytes(fmt), 0, 0};
}

inline Span scales_span(const char *name, const void *p, uint64_t rows, uint64_t cols)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return {name, b, b + rows * mx_blocks(cols), 0, 0};
}

inline bool overlap(const Span &a, const Span &b)
{
    if (!(a.b < b.e && b.b < a.e && a.b < a.e && b.b < b.e))
        return false;
    if (a.ld == b.ld && a.width <= a.ld && b.width <= b.ld && a.ld) {   // side by side in the rows of one wider tensor
        const uint64_t d = b.b >= a.b ? (b.b - a.b) % a.ld : (a.ld - (a.b - b.b) % a.ld) % a.ld;
        return !(d >= a.width && d + b.width <= a.ld);
    }
    return true;
}

// No output may overlap an input or another output.
template <int NO, int NI>
int check_apart(const Span (&outs)[NO], const Span (&ins)[NI])
{
    for (int i = 0; i < NO; ++i) {
        for (int j = 0; j < NI; ++j)
            if (overlap(outs[i], ins[j]))
                return fail(FASTRACK_EINVAL, "%s overlaps %s", outs[i].name, ins[j].name);
        for (int j = 0; j < i; ++j)
            if (overlap(outs[i], outs[j]))
                return fail(FASTRACK_EINVAL, "%s overlaps %s", outs[i].name, outs[j].name);
    }
    return FASTRACK_OK;
}

inline int check_dims(uint64_t a, uint64_t b, uint64_t c = 0)
{
    if (a > kMaxDim || b > kMaxDim || c > kMaxDim)
        return fail(FASTRACK_EINVAL, "a size is above 2^31 - 1");
    return FASTRACK_OK;
}

inline int check_type(uint32_t type)
{
    if (type > kFp32)
        return fail(FASTRACK_EINVAL, "unknown element type %u", type);
    return FASTRACK_OK;
}

// A float matrix: where the elements lie.
inline int check_rows(const char *name, const void *p, uint64_t ld, uint64_t rows, uint64_t cols, uint32_t type, bool out)
{
    if (rows == 0 || cols == 0)
        return FASTRACK_OK;
    if (!p)
        return fail(FASTRACK_EINVAL, "%s must be non-NULL", name);
    if (reinterpret_cast<uintptr_t>(p) % mx_type_size(type))
        return fail(FASTRACK_EINVAL, "%s must be aligned to its element type", name);
    if (ld > 1ull << 40)
        return fail(FASTRACK_EINVAL, "%s: row stride out of range", name);
    if (out && rows > 1 && ld < cols)
        return fail(FASTRACK_EINVAL, "%s: rows of %llu elements overlap at a stride of %llu", name,
                    (unsigned long long)cols, (unsigned long long)ld);
    return FASTRACK_OK;
}

inline int check_mx(const char *name, const uint8_t *codes, const uint8_t *scales, uint64_t rows, uint64_t cols)
{
    if (rows == 0 || cols == 0)
        return FASTRACK_OK;
    if (!codes || !scales)
        return fail(FASTRACK_EINVAL, "the codes and scales of %s must be non-NULL", name);
    if (reinterpret_cast<uintptr_t>(codes) % 16)
        return fail(FASTRACK_EINVAL, "the codes of %s must be 16-byte aligned", name);
    return FASTRACK_OK;
}

inline int check_work(const void *work, uint64_t have, uint64_t need)
{
    if (need == 0)
        return FASTRACK_OK;
    if (have < need || !work)
        return fail(FASTRACK_EINVAL, "workspace of %llu bytes, the call needs %llu", (unsigned long long)(work ? have : 0),
                    (unsigned long long)need);
    if (reinterpret_cast<uintptr_t>(work) % 16)
        return fail(FASTRACK_EINVAL, "the workspace must be 16-byte aligned");
    return FASTRACK_OK;
}

#define FT_TRY(...)                \
    do {                           \
        const int rc_ = (__VA_ARGS__); \
        if (rc_ != FASTRACK_OK)    \
            return rc_;            \
    } while (0)

inline void *mut(const void *p) { return const_cast<void *>(p); }
inline uint8_t *mut8(const uint8_t *p) { return const_cast<uint8_t *>(p); }

inline int check_format(uint32_t fmt)
{
    if (fmt != kMx4 && fmt != kMx8)
        return fail(FASTRACK_EINVAL, "unknown MX format %u", fmt);
    return FASTRACK_OK;
}

}  // namespace check
}  // namespace fastrack
