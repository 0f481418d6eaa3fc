// C entries of the microscaled operators around a model's layers: argument checks, then the launch.
#include <cmath>

#include "mx_check.h"
#include "mx_model.h"

using namespace fastrack;
using namespace fastrack::check;

namespace {

int check_index(uint32_t type)
{
    if (type > FASTRACK_I64)
        return fail(FASTRACK_EINVAL, "unknown index type %u", type);
    return FASTRACK_OK;
}

int check_ids(const void *ids, uint32_t type, uint64_t m)
{
    if (m == 0)
        return FASTRACK_OK;
    if (!ids)
        return fail(FASTRACK_EINVAL, "d_ids must be non-NULL");
    if (reinterpret_cast<uintptr_t>(ids) % (type == FASTRACK_I64 ? 8 : 4))
        return fail(FASTRACK_EINVAL, "d_ids must be aligned to its element type");
    return FASTRACK_OK;
}

Span ids_span(const void *ids, uint32_t type, uint64_t m)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(ids);
    return {"d_ids", b, b + m * (type == FASTRACK_I64 ? 8 : 4)};
}

// `step` elements between neighbours.
Span floats_span(const char *name, const void *p, uint64_t n, uint64_t step = 1)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return {name, b, p && n ? b + ((n - 1) * step + 1) * 4 : b};
}

Span work_span(const void *work, uint64_t need)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(work);
    return {"the workspace", b, b + need};
}

int check_floats(const char *name, const void *p, uint64_t n)
{
    if (n == 0)
        return FASTRACK_OK;
    if (!p)
        return fail(FASTRACK_EINVAL, "%s must be non-NULL", name);
    if (reinterpret_cast<uintptr_t>(p) % 4)
        return fail(FASTRACK_EINVAL, "%s must be aligned to its element type", name);
    return FASTRACK_OK;
}

int check_weight(const char *name, const void *p, uint32_t wtype, uint64_t cols)
{
    return check_rows(name, p, cols, 1, cols, wtype, false);
}

int check_norm_types(uint32_t type, uint32_t wtype)
{
    FT_TRY(check_type(type));
    FT_TRY(check_type(wtype));
    if (wtype != type && wtype != kFp32)
        return fail(FASTRACK_EINVAL, "weights are of the rows' type or 32-bit floats");
    return FASTRACK_OK;
}

constexpr uint64_t kMostTokens = (1ull << 22) - 1;   // workgroups of 1024 threads: fewer than 2^32 of these

}  // namespace

FT_EXPORT int fastrack_mx_norm(uint32_t type, const void *d_x, uint64_t ldx, const void *d_residual, uint64_t ld_residual,
                               const void *d_gate, uint64_t ld_gate, uint64_t rows, uint64_t cols, uint32_t weight_type,
                               const void *d_weight, const void *d_post_weight, float scale, float eps, void *d_y, uint64_t ldy,
                               void *d_hidden, uint64_t ld_hidden, uint8_t *d_ucodes, uint8_t *d_uscales, float *d_inverse,
                               uint8_t *d_vcodes, uint8_t *d_vscales, float *d_post_inverse, uint8_t *d_gcodes, uint8_t *d_gscales,
                               void *stream)
{
    clear_error();
    FT_TRY(check_norm_types(type, weight_type));
    FT_TRY(check_dims(rows, cols));
    if (!(eps >= 0.0f) || std::isinf(eps) || std::isnan(scale))
        return fail(FASTRACK_EINVAL, "eps must be finite and not negative, scale a number");
    if (rows == 0 || cols == 0)
        return FASTRACK_OK;
    const bool post = d_post_weight != nullptr, gate = d_gate != nullptr;
    const uint64_t rr = d_residual ? rows : 0, gr = gate ? rows : 0, hr = d_hidden ? rows : 0, vr = post || gate ? rows : 0;
    FT_TRY(check_rows("d_x", d_x, ldx, rows, cols, type, false));
    FT_TRY(check_rows("d_residual", d_residual, ld_residual, rr, cols, type, false));
    FT_TRY(check_rows("d_gate", d_gate, ld_gate, gr, cols, type, false));
    FT_TRY(check_weight("d_weight", d_weight, weight_type, cols));
    if (post)
        FT_TRY(check_weight("d_post_weight", d_post_weight, weight_type, cols));
    FT_TRY(check_rows("d_y", d_y, ldy, rows, cols, type, true));
    FT_TRY(check_rows("d_hidden", d_hidden, ld_hidden, hr, cols, type, true));
    FT_TRY(check_mx("the kept norm", d_ucodes, d_uscales, rows, cols));
    FT_TRY(check_mx("the kept block", d_vcodes, d_vscales, vr, cols));
    FT_TRY(check_mx("the kept gate", d_gcodes, d_gscales, gr, cols));
    FT_TRY(check_floats("d_inverse", d_inverse, rows));
    FT_TRY(check_floats("d_post_inverse", d_post_inverse, post ? rows : 0));
    FT_TRY(check_apart<10, 5>({rows_span("d_y", d_y, ldy, rows, cols, type), rows_span("d_hidden", d_hidden, ld_hidden, hr, cols, type),
                               codes_span("d_ucodes", d_ucodes, kMx8, rows, cols), scales_span("d_uscales", d_uscales, rows, cols),
                               codes_span("d_vcodes", d_vcodes, kMx8, vr, cols), scales_span("d_vscales", d_vscales, vr, cols),
                               codes_span("d_gcodes", d_gcodes, kMx8, gr, cols), scales_span("d_gscales", d_gscales, gr, cols),
                               floats_span("d_inverse", d_inverse, rows), floats_span("d_post_inverse", d_post_inverse, post ? rows : 0)},
                              {rows_span("d_x", d_x, ldx, rows, cols, type),
                               rows_span("d_residual", d_residual, ld_residual, rr, cols, type),
                               rows_span("d_gate", d_gate, ld_gate, gr, cols, type),
                               rows_span("d_weight", d_weight, cols, 1, cols, weight_type),
                               rows_span("d_post_weight", d_post_weight, cols, post ? 1 : 0, cols, weight_type)}));
    Norm n = {};
    n.type = type, n.wtype = weight_type;
    n.rows = rows, n.cols = cols;
    n.x = {mut(d_x), ldx}, n.r = {mut(d_residual), ld_residual}, n.g = {mut(d_gate), ld_gate};
    n.y = {d_y, ldy}, n.h = {d_hidden, ld_hidden};
    n.w2 = d_weight, n.w1 = d_post_weight;
    n.scale = scale, n.eps = eps;
    n.u = {d_ucodes, d_uscales};
    if (vr)
        n.v = {d_vcodes, d_vscales};
    if (gate)
        n.gq = {d_gcodes, d_gscales};
    n.inv2 = d_inverse, n.inv1 = d_post_inverse;
    return done(launch_mx_norm(n, num_cu(), as_stream(stream)), "norm launch");
}

FT_EXPORT uint64_t fastrack_mx_norm_grad_work_bytes(uint64_t rows, uint64_t cols, uint32_t post)
{
    return rows > kMaxDim || cols > kMaxDim ? 0 : mx_norm_grad_work(rows, cols, post != 0, num_cu()) * 4;
}

FT_EXPORT int fastrack_mx_norm_grad(uint32_t type, const void *d_dy, uint64_t ld_dy, const void *d_dhidden, uint64_t ld_dhidden,
                                    uint64_t rows, uint64_t cols, uint32_t weight_type, const void *d_weight, const void *d_post_weight,
                                    float scale, const uint8_t *d_ucodes, const uint8_t *d_uscales, const float *d_inverse,
                                    const uint8_t *d_vcodes, const uint8_t *d_vscales, const float *d_post_inverse, const uint8_t *d_gcodes,
                                    const uint8_t *d_gscales, void *d_dx, uint64_t ld_dx, void *d_dresidual, uint64_t ld_dresidual,
                                    void *d_dgate, uint64_t ld_dgate, float *d_dweight, float *d_dpost_weight, void *d_work,
                                    uint64_t work_bytes, void *stream)
{
    clear_error();
    FT_TRY(check_norm_types(type, weight_type));
    FT_TRY(check_dims(rows, cols));
    if (std::isnan(scale))
        return fail(FASTRACK_EINVAL, "scale must be a number");
    if (cols == 0)
        return FASTRACK_OK;
    const bool post = d_post_weight != nullptr, gate = d_gcodes != nullptr;
    const uint64_t hr = d_dhidden ? rows : 0, gr = gate ? rows : 0, vr = post || gate ? rows : 0, rr = d_dresidual ? rows : 0;
    FT_TRY(check_rows("d_dy", d_dy, ld_dy, rows, cols, type, false));
    FT_TRY(check_rows("d_dhidden", d_dhidden, ld_dhidden, hr, cols, type, false));
    FT_TRY(check_weight("d_weight", d_weight, weight_type, cols));
    if (post)
        FT_TRY(check_weight("d_post_weight", d_post_weight, weight_type, cols));
    FT_TRY(check_mx("the kept norm", d_ucodes, d_uscales, rows, cols));
    FT_TRY(check_mx("the kept block", d_vcodes, d_vscales, vr, cols));
    FT_TRY(check_mx("the kept gate", d_gcodes, d_gscales, gr, cols));
    FT_TRY(check_floats("d_inverse", d_inverse, rows));
    FT_TRY(check_floats("d_post_inverse", d_post_inverse, post ? rows : 0));
    FT_TRY(check_rows("d_dx", d_dx, ld_dx, rows, cols, type, true));
    FT_TRY(check_rows("d_dresidual", d_dresidual, ld_dresidual, rr, cols, type, true));
    FT_TRY(check_rows("d_dgate", d_dgate, ld_dgate, gr, cols, type, true));
    FT_TRY(check_floats("d_dweight", d_dweight, cols));
    FT_TRY(check_floats("d_dpost_weight", d_dpost_weight, post ? cols : 0));
    const int cus = num_cu();
    const uint64_t need = mx_norm_grad_work(rows, cols, post, cus) * 4;
    FT_TRY(check_work(d_work, work_bytes, need));
    FT_TRY(check_apart<6, 12>({rows_span("d_dx", d_dx, ld_dx, rows, cols, type),
                               rows_span("d_dresidual", d_dresidual, ld_dresidual, rr, cols, type),
                               rows_span("d_dgate", d_dgate, ld_dgate, gr, cols, type), floats_span("d_dweight", d_dweight, cols),
                               floats_span("d_dpost_weight", d_dpost_weight, post ? cols : 0), work_span(d_work, need)},
                              {rows_span("d_dy", d_dy, ld_dy, rows, cols, type),
                               rows_span("d_dhidden", d_dhidden, ld_dhidden, hr, cols, type),
                               rows_span("d_weight", d_weight, cols, 1, cols, weight_type),
                               rows_span("d_post_weight", d_post_weight, cols, post ? 1 : 0, cols, weight_type),
                               codes_span("d_ucodes", d_ucodes, kMx8, rows, cols), scales_span("d_uscales", d_uscales, rows, cols),
                               codes_span("d_vcodes", d_vcodes, kMx8, vr, cols), scales_span("d_vscales", d_vscales, vr, cols),
                               codes_span("d_gcodes", d_gcodes, kMx8, gr, cols), scales_span("d_gscales", d_gscales, gr, cols),
                               floats_span("d_inverse", d_inverse, rows),
                               floats_span("d_post_inverse", d_post_inverse, post ? rows : 0)}));
    NormGrad n = {};
    n.type = type, n.wtype = weight_type;
    n.rows = rows, n.cols = cols;
    n.dy = {mut(d_dy), ld_dy}, n.dh = {mut(d_dhidden), ld_dhidden};
    n.dx = {d_dx, ld_dx}, n.dr = {d_dresidual, ld_dresidual}, n.dg = {d_dgate, ld_dgate};
    n.w2 = d_weight, n.w1 = d_post_weight;
    n.scale = scale;
    n.u = {mut8(d_ucodes), mut8(d_uscales)};
    if (vr)
        n.v = {mut8(d_vcodes), mut8(d_vscales)};
    n.gq = {mut8(d_gcodes), mut8(d_gscales)};
    n.inv2 = d_inverse, n.inv1 = d_post_inverse;
    n.dw2 = d_dweight, n.dw1 = d_dpost_weight;
    n.work = reinterpret_cast<float *>(d_work);
    return done(launch_mx_norm_grad(n, cus, as_stream(stream)), "norm gradient launch");
}

FT_EXPORT int fastrack_mx_embedding(uint32_t index_type, const void *d_ids, uint64_t m, const uint8_t *d_codes,
                                    const uint8_t *d_scales, uint64_t rows, uint64_t cols, float scale, uint32_t type, void *d_y,
                                    uint64_t ldy, void *stream)
{
    clear_error();
    FT_TRY(check_index(index_type));
    FT_TRY(check_type(type));
    FT_TRY(check_dims(m, rows, cols));
    FT_TRY(check_ids(d_ids, index_type, m));
    FT_TRY(check_mx("the table", d_codes, d_scales, rows, cols));
    FT_TRY(check_rows("d_y", d_y, ldy, m, cols, type, true));
    FT_TRY(check_apart<1, 3>({rows_span("d_y", d_y, ldy, m, cols, type)},
                             {ids_span(d_ids, index_type, m), codes_span("d_codes", d_codes, kMx4, rows, cols),
                              scales_span("d_scales", d_scales, rows, cols)}));
    const Embedding e = {{d_ids, index_type}, m, rows, cols, {mut8(d_codes), mut8(d_scales)}, scale, type, {d_y, ldy}};
    return done(launch_mx_embedding(e, as_stream(stream)), "embedding launch");
}

FT_EXPORT uint64_t fastrack_mx_embedding_grad_work_bytes(uint64_t m, uint64_t rows, uint64_t cols)
{
    return m > kMaxDim || rows > kMaxDim || cols > kMaxDim ? 0 : mx_embedding_grad_work(m, rows, cols);
}

FT_EXPORT int fastrack_mx_embedding_grad(uint32_t index_type, const void *d_ids, uint32_t type, const void *d_dy, uint64_t ld_dy,
                                         uint64_t m, uint64_t rows, uint64_t cols, float scale, uint32_t out_type, void *d_dw,
                                         uint64_t ld_dw, uint32_t accumulate, void *d_work, uint64_t work_bytes, void *stream)
{
    clear_error();
    FT_TRY(check_index(index_type));
    FT_TRY(check_type(type));
    FT_TRY(check_type(out_type));
    FT_TRY(check_dims(m, rows, cols));
    if (accumulate > 1 || (accumulate && out_type != kFp32))
        return fail(FASTRACK_EINVAL, "accumulate is 0, or 1 with a 32-bit gradient");
    FT_TRY(check_ids(d_ids, index_type, m));
    FT_TRY(check_rows("d_dy", d_dy, ld_dy, m, cols, type, false));
    FT_TRY(check_rows("d_dw", d_dw, ld_dw, rows, cols, out_type, true));
    if ((m + 15) / 16 * ((cols + 511) / 512) >= 1ull << 26)   // waves: fewer than 2^32 threads
        return fail(FASTRACK_EINVAL, "2^26 pieces of 16 tokens and 512 columns, or more");
    const uint64_t need = mx_embedding_grad_work(m, rows, cols);
    FT_TRY(check_work(d_work, work_bytes, need));
    FT_TRY(check_apart<2, 2>({rows_span("d_dw", d_dw, ld_dw, rows, cols, out_type), work_span(d_work, need)},
                             {ids_span(d_ids, index_type, m), rows_span("d_dy", d_dy, ld_dy, m, cols, type)}));
    const EmbeddingGrad e = {{d_ids, index_type}, type, {mut(d_dy), ld_dy}, m, rows, cols, scale, out_type, {d_dw, ld_dw},
                             accumulate != 0, d_work};
    return done(launch_mx_embedding_grad(e, as_stream(stream)), "embedding gradient launch");
}

namespace {

Loss loss_of(uint32_t type, const void *x, uint64_t ldx, const uint8_t *codes, const uint8_t *scales, uint32_t index_type,
             const void *ids, uint64_t m, uint64_t n, uint64_t k, float scale)
{
    Loss l = {};
    l.type = type;
    l.x = {mut(x), ldx};
    l.w = {mut8(codes), mut8(scales)};
    l.ids = {ids, index_type};
    l.m = m, l.n = n, l.k = k;
    l.scale = scale;
    return l;
}

int check_loss(const Loss &l)
{
    FT_TRY(check_index(l.ids.wide));
    FT_TRY(check_type(l.type));
    FT_TRY(check_dims(l.m, l.n, l.k));
    if (l.m > kMostTokens)
        return fail(FASTRACK_EINVAL, "more than 2^22 - 1 tokens");
    if (l.m && l.n == 0)
        return fail(FASTRACK_EINVAL, "a vocabulary of no classes");
    if ((l.n + 127) / 128 * ((l.k + 127) / 128) > 1ull << 24 || (l.m + 127) / 128 * ((l.k + 127) / 128) > 1ull << 24)
        return fail(FASTRACK_EINVAL, "more than 2^24 output tiles of 128 x 128");
    FT_TRY(check_rows("d_x", l.x.p, l.x.ld, l.m, l.k, l.type, false));
    FT_TRY(check_mx("w", l.w.codes, l.w.scales, l.n, l.k));
    return check_ids(l.ids.p, l.ids.wide, l.m);
}

}  // namespace

FT_EXPORT uint64_t fastrack_mx_loss_work_bytes(uint32_t type, const void *d_x, uint64_t ldx, uint64_t m, uint64_t n, uint64_t k)
{
    if (type > kFp32 || m > kMostTokens || n > kMaxDim || k > kMaxDim)
        return 0;
    return mx_loss_work(loss_of(type, d_x, ldx, nullptr, nullptr, 0, nullptr, m, n, k, 1.0f), num_cu());
}

FT_EXPORT int fastrack_mx_loss(uint32_t type, const void *d_x, uint64_t ldx, const uint8_t *d_codes, const uint8_t *d_scales,
                               uint32_t index_type, const void *d_ids, uint64_t m, uint64_t n, uint64_t k, float scale,
                               float *d_loss, float *d_lse, void *d_work, uint64_t work_bytes, void *stream)
{
    clear_error();
    Loss l = loss_of(type, d_x, ldx, d_codes, d_scales, index_type, d_ids, m, n, k, scale);
    FT_TRY(check_loss(l));
    FT_TRY(check_floats("d_loss", d_loss, m));
    FT_TRY(check_floats("d_lse", d_lse, m));
    if (m == 0)
        return FASTRACK_OK;
    const int cus = num_cu();
    const uint64_t need = mx_loss_work(l, cus);
    FT_TRY(check_work(d_work, work_bytes, need));
    FT_TRY(check_apart<3, 4>({floats_span("d_loss", d_loss, m), floats_span("d_lse", d_lse, m), work_span(d_work, need)},
                             {rows_span("d_x", d_x, ldx, m, k, type), codes_span("d_codes", d_codes, kMx4, n, k),
                              scales_span("d_scales", d_scales, n, k), ids_span(d_ids, index_type, m)}));
    l.loss = d_loss, l.lse = d_lse;
    l.work = d_work;
    return done(launch_mx_loss(l, cus, as_stream(stream)), "loss launch");
}

FT_EXPORT uint64_t fastrack_mx_loss_grad_work_bytes(uint32_t type, const void *d_x, uint64_t ldx, uint64_t m, uint64_t n, uint64_t k,
                                                    uint32_t dx, uint32_t dx_type, uint32_t dw, uint32_t dw_type)
{
    if (type > kFp32 || dx_type > kFp32 || dw_type > kFp32 || m > kMostTokens || n > kMaxDim || k > kMaxDim)
        return 0;
    Loss l = loss_of(type, d_x, ldx, nullptr, nullptr, 0, nullptr, m, n, k, 1.0f);
    uint8_t some;   // (the plan asks which gradients there are, not where)
    l.dx = {dx ? &some : nullptr, k}, l.dx_type = dx_type;
    l.x8.codes = dw ? &some : nullptr, l.dw_type = dw_type;
    return mx_loss_grad_work(l, num_cu());
}

FT_EXPORT int fastrack_mx_loss_grad(uint32_t type, const void *d_x, uint64_t ldx, const uint8_t *d_codes, const uint8_t *d_scales,
                                    const uint8_t *d_xcodes, const uint8_t *d_xscales, uint32_t index_type, const void *d_ids,
                                    const float *d_dloss, uint64_t dloss_step, const float *d_lse, uint64_t m, uint64_t n, uint64_t k,
                                    float scale, uint32_t dx_type, void *d_dx, uint64_t ld_dx, uint32_t dw_type, void *d_dw,
                                    uint64_t ld_dw, uint32_t accumulate, void *d_work, uint64_t work_bytes, void *stream)
{
    clear_error();
    Loss l = loss_of(type, d_x, ldx, d_codes, d_scales, index_type, d_ids, m, n, k, scale);
    FT_TRY(check_loss(l));
    FT_TRY(check_type(dx_type));
    FT_TRY(check_type(dw_type));
    if (accumulate > 1 || (accumulate && dw_type != kFp32))
        return fail(FASTRACK_EINVAL, "accumulate is 0, or 1 with a 32-bit gradient");
    if (dloss_step > 1ull << 40)
        return fail(FASTRACK_EINVAL, "d_dloss: stride out of range");
    const bool weight = d_dw != nullptr;
    const uint64_t xr = weight ? m : 0, wr = weight ? n : 0, dr = d_dx ? m : 0;
    FT_TRY(check_floats("d_dloss", d_dloss, m));
    FT_TRY(check_floats("d_lse", d_lse, m));
    FT_TRY(check_mx("the kept x", d_xcodes, d_xscales, xr, k));
    FT_TRY(check_rows("d_dx", d_dx, ld_dx, dr, k, dx_type, true));
    FT_TRY(check_rows("d_dw", d_dw, ld_dw, wr, k, dw_type, true));
    if (k == 0)
        return FASTRACK_OK;
    l.lse = const_cast<float *>(d_lse);
    l.dloss = d_dloss, l.dloss_step = dloss_step;
    if (weight) {
        static uint8_t none;   // a kept x of no tokens may have no address
        l.x8 = {d_xcodes ? mut8(d_xcodes) : &none, mut8(d_xscales)};
    }
    l.dx = {d_dx, ld_dx}, l.dx_type = dx_type;
    l.dw = {d_dw, ld_dw}, l.dw_type = dw_type;
    l.accumulate = accumulate != 0;
    l.work = d_work;
    const int cus = num_cu();
    const uint64_t need = mx_loss_grad_work(l, cus);
    FT_TRY(check_work(d_work, work_bytes, need));
    FT_TRY(check_apart<3, 8>({rows_span("d_dx", d_dx, ld_dx, dr, k, dx_type), rows_span("d_dw", d_dw, ld_dw, wr, k, dw_type),
                              work_span(d_work, need)},
                             {rows_span("d_x", d_x, ldx, m, k, type), codes_span("d_codes", d_codes, kMx4, n, k),
                              scales_span("d_scales", d_scales, n, k), codes_span("d_xcodes", d_xcodes, kMx8, xr, k),
                              scales_span("d_xscales", d_xscales, xr, k), ids_span(d_ids, index_type, m),
                              floats_span("d_dloss", d_dloss, m, dloss_step), floats_span("d_lse", d_lse, m)}));
    return done(launch_mx_loss_grad(l, cus, as_stream(stream)), "loss gradient launch");
}
