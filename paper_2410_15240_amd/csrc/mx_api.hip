// C entries of the microscaled (MX) operators: argument checks, then the launch.
#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdarg>
#include <cstdio>

#include "fastrack.h"
#include "mx.h"

using namespace fastrack;

#define FT_EXPORT extern "C" __attribute__((visibility("default")))

namespace {

int fail(int code, const char *fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return set_error(code, buf);
}

int done(hipError_t e, const char *what)
{
    return e == hipSuccess ? FASTRACK_OK : fail(FASTRACK_EHIP, "%s: %s", what, hipGetErrorString(e));
}

hipStream_t as_stream(void *s) { return reinterpret_cast<hipStream_t>(s); }

constexpr uint64_t kMaxDim = 0x7FFFFFFFull;

// Compute units of the current device. A plan does not depend on having one: without a
// device the workspace of this GPU's 256 is told.
int num_cu()
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

Span rows_span(const char *name, const void *p, uint64_t ld, uint64_t rows, uint64_t cols, uint32_t type)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    const uint64_t size = mx_type_size(type), n = rows && cols ? ((rows - 1) * ld + cols) * size : 0;
    return {name, b, b + n, ld * size, cols * size};
}

Span codes_span(const char *name, const void *p, uint32_t fmt, uint64_t rows, uint64_t cols)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return {name, b, b + rows * mx_blocks(cols) * mx_block_bytes(fmt), 0, 0};
}

Span scales_span(const char *name, const void *p, uint64_t rows, uint64_t cols)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return {name, b, b + rows * mx_blocks(cols), 0, 0};
}

bool overlap(const Span &a, const Span &b)
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

int check_dims(uint64_t a, uint64_t b, uint64_t c = 0)
{
    if (a > kMaxDim || b > kMaxDim || c > kMaxDim)
        return fail(FASTRACK_EINVAL, "a size is above 2^31 - 1");
    return FASTRACK_OK;
}

int check_type(uint32_t type)
{
    if (type > kFp32)
        return fail(FASTRACK_EINVAL, "unknown element type %u", type);
    return FASTRACK_OK;
}

// A float matrix: where the elements lie.
int check_rows(const char *name, const void *p, uint64_t ld, uint64_t rows, uint64_t cols, uint32_t type, bool out)
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

int check_mx(const char *name, const uint8_t *codes, const uint8_t *scales, uint64_t rows, uint64_t cols)
{
    if (rows == 0 || cols == 0)
        return FASTRACK_OK;
    if (!codes || !scales)
        return fail(FASTRACK_EINVAL, "the codes and scales of %s must be non-NULL", name);
    if (reinterpret_cast<uintptr_t>(codes) % 16)
        return fail(FASTRACK_EINVAL, "the codes of %s must be 16-byte aligned", name);
    return FASTRACK_OK;
}

int check_work(const void *work, uint64_t have, uint64_t need)
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

void *mut(const void *p) { return const_cast<void *>(p); }
uint8_t *mut8(const uint8_t *p) { return const_cast<uint8_t *>(p); }

int check_format(uint32_t fmt)
{
    if (fmt != kMx4 && fmt != kMx8)
        return fail(FASTRACK_EINVAL, "unknown MX format %u", fmt);
    return FASTRACK_OK;
}

}  // namespace

FT_EXPORT uint64_t fastrack_mx_code_bytes(uint32_t format, uint64_t rows, uint64_t cols)
{
    if ((format != kMx4 && format != kMx8) || rows > kMaxDim || cols > kMaxDim)
        return 0;
    return rows * mx_blocks(cols) * mx_block_bytes(format);
}

FT_EXPORT uint64_t fastrack_mx_scale_bytes(uint64_t rows, uint64_t cols)
{
    return rows > kMaxDim || cols > kMaxDim ? 0 : rows * mx_blocks(cols);
}

FT_EXPORT int fastrack_mx_quantize(uint32_t format, uint32_t type, const void *d_x, uint64_t ldx, uint64_t rows,
                                   uint64_t cols, uint8_t *d_codes, uint8_t *d_scales, void *stream)
{
    clear_error();
    FT_TRY(check_format(format));
    FT_TRY(check_type(type));
    FT_TRY(check_dims(rows, cols));
    FT_TRY(check_rows("d_x", d_x, ldx, rows, cols, type, false));
    FT_TRY(check_mx("the output", d_codes, d_scales, rows, cols));
    FT_TRY(check_apart<2, 1>({codes_span("d_codes", d_codes, format, rows, cols), scales_span("d_scales", d_scales, rows, cols)},
                             {rows_span("d_x", d_x, ldx, rows, cols, type)}));
    return done(launch_mx_quantize(format, type, {mut(d_x), ldx}, rows, cols, {d_codes, d_scales}, as_stream(stream)),
                "quantize launch");
}

FT_EXPORT int fastrack_mx_dequantize(uint32_t format, const uint8_t *d_codes, const uint8_t *d_scales, uint64_t rows,
                                     uint64_t cols, uint32_t type, void *d_out, uint64_t ld_out, void *stream)
{
    clear_error();
    FT_TRY(check_format(format));
    FT_TRY(check_type(type));
    FT_TRY(check_dims(rows, cols));
    FT_TRY(check_mx("the input", d_codes, d_scales, rows, cols));
    FT_TRY(check_rows("d_out", d_out, ld_out, rows, cols, type, true));
    FT_TRY(check_apart<1, 2>({rows_span("d_out", d_out, ld_out, rows, cols, type)},
                             {codes_span("d_codes", d_codes, format, rows, cols),
                              scales_span("d_scales", d_scales, rows, cols)}));
    return done(launch_mx_dequantize(format, type, {mut8(d_codes), mut8(d_scales)}, rows, cols, {d_out, ld_out},
                                     as_stream(stream)),
                "dequantize launch");
}

FT_EXPORT int fastrack_mx_act(uint32_t act, uint32_t type, const void *d_x, uint64_t ldx, const void *d_gate,
                              uint64_t ld_gate, uint64_t rows, uint64_t cols, void *d_y, uint64_t ldy, uint8_t *d_xcodes,
                              uint8_t *d_xscales, uint8_t *d_gcodes, uint8_t *d_gscales, void *stream)
{
    clear_error();
    if (act > kGelu)
        return fail(FASTRACK_EINVAL, "unknown activation %u", act);
    FT_TRY(check_type(type));
    FT_TRY(check_dims(rows, cols));
    const bool gate = d_gate != nullptr;
    const uint64_t gr = gate ? rows : 0;
    FT_TRY(check_rows("d_x", d_x, ldx, rows, cols, type, false));
    FT_TRY(check_rows("d_gate", d_gate, ld_gate, gr, cols, type, false));
    FT_TRY(check_rows("d_y", d_y, ldy, rows, cols, type, true));
    FT_TRY(check_mx("the kept x", d_xcodes, d_xscales, rows, cols));
    FT_TRY(check_mx("the kept gate", d_gcodes, d_gscales, gr, cols));
    FT_TRY(check_apart<5, 2>({rows_span("d_y", d_y, ldy, rows, cols, type),
                              codes_span("d_xcodes", d_xcodes, kMx8, rows, cols),
                              scales_span("d_xscales", d_xscales, rows, cols),
                              codes_span("d_gcodes", d_gcodes, kMx8, gr, cols),
                              scales_span("d_gscales", d_gscales, gr, cols)},
                             {rows_span("d_x", d_x, ldx, rows, cols, type),
                              rows_span("d_gate", d_gate, ld_gate, gr, cols, type)}));
    return done(launch_mx_act(act, type, {mut(d_x), ldx}, {mut(d_gate), ld_gate}, rows, cols, {d_y, ldy},
                              {d_xcodes, d_xscales}, {d_gcodes, d_gscales}, as_stream(stream)),
                "activation launch");
}

FT_EXPORT int fastrack_mx_act_grad(uint32_t act, uint32_t type, const void *d_dy, uint64_t ld_dy, const uint8_t *d_xcodes,
                                   const uint8_t *d_xscales, const uint8_t *d_gcodes, const uint8_t *d_gscales,
                                   uint64_t rows, uint64_t cols, void *d_dx, uint64_t ld_dx, void *d_dgate,
                                   uint64_t ld_dgate, void *stream)
{
    clear_error();
    if (act > kGelu)
        return fail(FASTRACK_EINVAL, "unknown activation %u", act);
    FT_TRY(check_type(type));
    FT_TRY(check_dims(rows, cols));
    const bool gate = d_gcodes != nullptr;
    const uint64_t gr = gate ? rows : 0;
    FT_TRY(check_rows("d_dy", d_dy, ld_dy, rows, cols, type, false));
    FT_TRY(check_mx("the kept x", d_xcodes, d_xscales, rows, cols));
    FT_TRY(check_mx("the kept gate", d_gcodes, d_gscales, gr, cols));
    FT_TRY(check_rows("d_dx", d_dx, ld_dx, rows, cols, type, true));
    FT_TRY(check_rows("d_dgate", d_dgate, ld_dgate, gr, cols, type, true));
    FT_TRY(check_apart<2, 5>({rows_span("d_dx", d_dx, ld_dx, rows, cols, type),
                              rows_span("d_dgate", d_dgate, ld_dgate, gr, cols, type)},
                             {rows_span("d_dy", d_dy, ld_dy, rows, cols, type),
                              codes_span("d_xcodes", d_xcodes, kMx8, rows, cols),
                              scales_span("d_xscales", d_xscales, rows, cols),
                              codes_span("d_gcodes", d_gcodes, kMx8, gr, cols),
                              scales_span("d_gscales", d_gscales, gr, cols)}));
    return done(launch_mx_act_grad(act, type, {mut(d_dy), ld_dy}, {mut8(d_xcodes), mut8(d_xscales)},
                                   {mut8(d_gcodes), mut8(d_gscales)}, rows, cols, {d_dx, ld_dx}, {d_dgate, ld_dgate},
                                   as_stream(stream)),
                "activation gradient launch");
}

namespace {

MxProduct product(uint32_t op, uint32_t type, const void *a, uint64_t lda, const uint8_t *codes, const uint8_t *scales,
                  uint64_t m, uint64_t n, uint64_t k, uint32_t ctype, void *c, uint64_t ldc, bool accumulate, void *work,
                  uint64_t work_bytes)
{
    return {op, type, {mut(a), lda}, {mut8(codes), mut8(scales)}, m, n, k, ctype, {c, ldc}, accumulate, work, work_bytes};
}

int run_product(const char *aname, const char *cname, const MxProduct &p, void *stream)
{
    FT_TRY(check_type(p.type));
    FT_TRY(check_type(p.ctype));
    FT_TRY(check_dims(p.m, p.n, p.k));
    const uint32_t fmt = p.op == kWeightGrad ? kMx8 : kMx4;
    const uint64_t a_cols = p.op == kLinear ? p.k : p.n;
    const uint64_t q_rows = p.op == kWeightGrad ? p.m : p.n;
    const uint64_t c_rows = p.op == kWeightGrad ? p.n : p.m, c_cols = p.op == kLinear ? p.n : p.k;
    if ((c_rows + 127) / 128 * ((c_cols + 127) / 128) > 1ull << 24)
        return fail(FASTRACK_EINVAL, "more than 2^24 output tiles of 128 x 128");
    FT_TRY(check_rows(aname, p.a.p, p.a.ld, p.m, a_cols, p.type, false));
    FT_TRY(check_mx("the MX operand", p.q.codes, p.q.scales, q_rows, p.k));
    FT_TRY(check_rows(cname, p.c.p, p.c.ld, c_rows, c_cols, p.ctype, true));
    if (c_rows == 0 || c_cols == 0)
        return FASTRACK_OK;
    const int cus = num_cu();
    const uint64_t need = mx_product_work(p, cus);
    FT_TRY(check_work(p.work, p.work_bytes, need));
    const uintptr_t w = reinterpret_cast<uintptr_t>(p.work);
    FT_TRY(check_apart<2, 3>({rows_span(cname, p.c.p, p.c.ld, c_rows, c_cols, p.ctype), {"the workspace", w, w + need, 0, 0}},
                             {rows_span(aname, p.a.p, p.a.ld, p.m, a_cols, p.type),
                              codes_span("d_codes", p.q.codes, fmt, q_rows, p.k),
                              scales_span("d_scales", p.q.scales, q_rows, p.k)}));
    return done(launch_mx_product(p, cus, as_stream(stream)), "product launch");
}

}  // namespace

FT_EXPORT uint64_t fastrack_mx_work_bytes(uint32_t op, uint32_t type, const void *d_a, uint64_t lda, uint64_t m, uint64_t n,
                                          uint64_t k)
{
    if (m > kMaxDim || n > kMaxDim || k > kMaxDim || op > FASTRACK_MX_LINEAR_MX || type > kFp32)
        return 0;
    if (op == FASTRACK_MX_LINEAR_MX)
        return mx4_product_work({{}, {}, m, n, k, 0, {}, nullptr, 0}, num_cu());
    return mx_product_work(product(op, type, d_a, lda, nullptr, nullptr, m, n, k, 0, nullptr, 0, false, nullptr, 0), num_cu());
}

FT_EXPORT int fastrack_mx_linear(uint32_t type, const void *d_x, uint64_t ldx, const uint8_t *d_codes,
                                 const uint8_t *d_scales, uint64_t m, uint64_t n, uint64_t k, uint32_t out_type, void *d_y,
                                 uint64_t ldy, void *d_work, uint64_t work_bytes, void *stream)
{
    clear_error();
    return run_product("d_x", "d_y", product(kLinear, type, d_x, ldx, d_codes, d_scales, m, n, k, out_type, d_y, ldy, false,
                                             d_work, work_bytes), stream);
}

FT_EXPORT int fastrack_mx_linear_grad_input(uint32_t type, const void *d_dy, uint64_t ld_dy, const uint8_t *d_codes,
                                            const uint8_t *d_scales, uint64_t m, uint64_t n, uint64_t k,
                                            uint32_t out_type, void *d_dx, uint64_t ld_dx, void *d_work,
                                            uint64_t work_bytes, void *stream)
{
    clear_error();
    return run_product("d_dy", "d_dx", product(kGradInput, type, d_dy, ld_dy, d_codes, d_scales, m, n, k, out_type, d_dx,
                                               ld_dx, false, d_work, work_bytes), stream);
}

FT_EXPORT int fastrack_mx_weight_grad(uint32_t type, const void *d_dy, uint64_t ld_dy, const uint8_t *d_codes,
                                      const uint8_t *d_scales, uint64_t m, uint64_t n, uint64_t k, uint32_t out_type,
                                      void *d_dw, uint64_t ld_dw, uint32_t accumulate, void *d_work, uint64_t work_bytes,
                                      void *stream)
{
    clear_error();
    if (accumulate > 1 || (accumulate && out_type != kFp32))
        return fail(FASTRACK_EINVAL, "accumulate is 0, or 1 with a 32-bit gradient");
    return run_product("d_dy", "d_dw", product(kWeightGrad, type, d_dy, ld_dy, d_codes, d_scales, m, n, k, out_type, d_dw,
                                               ld_dw, accumulate != 0, d_work, work_bytes), stream);
}

FT_EXPORT int fastrack_mx_linear_mx(const uint8_t *d_xcodes, const uint8_t *d_xscales, const uint8_t *d_codes,
                                    const uint8_t *d_scales, uint64_t m, uint64_t n, uint64_t k, uint32_t out_type,
                                    void *d_y, uint64_t ldy, void *d_work, uint64_t work_bytes, void *stream)
{
    clear_error();
    FT_TRY(check_type(out_type));
    FT_TRY(check_dims(m, n, k));
    if ((m + 127) / 128 * ((n + 127) / 128) > 1ull << 24)
        return fail(FASTRACK_EINVAL, "more than 2^24 output tiles of 128 x 128");
    FT_TRY(check_mx("x", d_xcodes, d_xscales, m, k));
    FT_TRY(check_mx("w", d_codes, d_scales, n, k));
    FT_TRY(check_rows("d_y", d_y, ldy, m, n, out_type, true));
    if (m == 0 || n == 0)
        return FASTRACK_OK;
    const Mx4Product p = {{mut8(d_xcodes), mut8(d_xscales)}, {mut8(d_codes), mut8(d_scales)}, m, n, k, out_type,
                          {d_y, ldy}, d_work, work_bytes};
    const int cus = num_cu();
    const uint64_t need = mx4_product_work(p, cus);
    FT_TRY(check_work(d_work, work_bytes, need));
    const uintptr_t w = reinterpret_cast<uintptr_t>(d_work);
    FT_TRY(check_apart<2, 4>({rows_span("d_y", d_y, ldy, m, n, out_type), {"the workspace", w, w + need, 0, 0}},
                             {codes_span("d_xcodes", d_xcodes, kMx4, m, k), scales_span("d_xscales", d_xscales, m, k),
                              codes_span("d_codes", d_codes, kMx4, n, k), scales_span("d_scales", d_scales, n, k)}));
    return done(launch_mx4_product(p, cus, as_stream(stream)), "product launch");
}
