// C ABI of the layers in 8 bits (include/aif_q8.h): context, checks of arguments, launches.  Nothing is held between calls.
#include "../../include/aif_q8.h"
#include "aif_q8_dev.h"

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>

using namespace aif;

struct aif_q8_ctx {
    int device = 0, n_cu = 256;
    char err[512] = "";
};

namespace {
constexpr int Q8_MAX_NORM = 16384;                  // columns of a row that aif_q8_rows keeps in registers
constexpr int Q8_MAX_WIDTH = 1 << 20;
constexpr int Q8_MAX_ROWS = 1 << 30;                 // of a product: what its tiles count lies within 32 bits
constexpr int64_t Q8_MAX_RESULT = (int64_t)1 << 44;
constexpr int64_t Q8_MAX_CODE_STRIDE = 1 << 23;     // 256 rows of a tile lie within 32 bits
thread_local char g_q8_init_error[512] = "";

aif_status qfail(aif_q8_ctx *c, aif_status st, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(c ? c->err : g_q8_init_error, 512, fmt, ap);
    va_end(ap);
    return st;
}

#define Q8_RUN(ctxp, expr)                                                                             \
    do {                                                                                               \
        hipError_t e_ = (expr);                                                                        \
        if (e_ != hipSuccess) return qfail(ctxp, AIF_EDEVICE, "%s: %s", #expr, hipGetErrorString(e_)); \
    } while (0)

#define Q8_TRY(expr)                        \
    do {                                    \
        const aif_status st_ = (expr);      \
        if (st_ != AIF_OK) return st_;      \
    } while (0)

aif_status check_device(aif_q8_ctx *c)
{
    int cur = -1;
    Q8_RUN(c, hipGetDevice(&cur));
    if (cur != c->device) return qfail(c, AIF_EDEVICE, "context belongs to device %d, current device is %d", c->device, cur);
    return AIF_OK;
}

aif_status check_dtype(aif_q8_ctx *c, int dtype, int32_t n_rows)
{
    if (dtype != AIF_F32 && dtype != AIF_BF16) return qfail(c, AIF_EINVAL, "unknown dtype %d", dtype);
    if (n_rows < 0) return qfail(c, AIF_EINVAL, "negative n_rows %d", n_rows);
    return AIF_OK;
}

aif_status check_width(aif_q8_ctx *c, const char *what, int32_t width, int32_t of, int32_t most)
{
    if (width <= 0) return qfail(c, AIF_EINVAL, "%s %d is not positive", what, width);
    if (width % of) return qfail(c, AIF_ESHAPE, "%s %d is not a multiple of %d", what, width, of);
    if (width > most) return qfail(c, AIF_ERANGE, "%s %d is above %d", what, width, most);
    return AIF_OK;
}

// Rows of dtype: their stride in elements to `stride`.
aif_status check_rows(aif_q8_ctx *c, const char *what, const void *p, int64_t given, int32_t width, bool f32, int64_t &stride)
{
    if ((uintptr_t)p % 16 || given % (f32 ? 4 : 8)) return qfail(c, AIF_EINVAL, "%s: tensors and strides must be multiples of 16 bytes", what);
    if (given != 0 && (given < width || given >= (int64_t)1 << 33))
        return qfail(c, AIF_EINVAL, "%s: stride %lld below the row's %d, or 2^33 and above", what, (long long)given, width);
    stride = given ? given : width;
    return AIF_OK;
}

aif_status check_matrix(aif_q8_ctx *c, const char *what, const aif_q8_matrix &m, int32_t width, Q8Mat &to)
{
    const int64_t across = (width + Q8_BLOCK - 1) / Q8_BLOCK;
    if (!m.codes || !m.scales) return qfail(c, AIF_EINVAL, "%s: NULL codes or scales", what);
    if ((uintptr_t)m.codes % 16 || m.stride % 16) return qfail(c, AIF_EINVAL, "%s: codes and their stride must be multiples of 16 bytes", what);
    if ((uintptr_t)m.scales % 4 || m.scale_stride % 4) return qfail(c, AIF_EINVAL, "%s: scales and their stride must be multiples of 4 bytes", what);
    if (m.stride != 0 && (m.stride < width || m.stride >= Q8_MAX_CODE_STRIDE))
        return qfail(c, AIF_EINVAL, "%s: stride %lld below the row's %d, or 2^23 and above", what, (long long)m.stride, width);
    if (m.scale_stride != 0 && (m.scale_stride < across || m.scale_stride >= Q8_MAX_CODE_STRIDE))
        return qfail(c, AIF_EINVAL, "%s: scale_stride %lld below the row's %lld, or 2^23 and above", what, (long long)m.scale_stride, (long long)across);
    to = Q8Mat{(uint8_t *)m.codes, (uint8_t *)m.scales, m.stride ? m.stride : (int64_t)(width + 15) / 16 * 16, m.scale_stride ? m.scale_stride : (across + 3) / 4 * 4};
    return AIF_OK;
}

// What is written lies beside what is read; `in_place`: or where that lies, row for row.
aif_status check_apart(aif_q8_ctx *c, const char *what, const void *out, int64_t stride, const char *other, const void *p, int64_t p_stride, bool in_place)
{
    if (!out || out != p || (in_place && stride == p_stride)) return AIF_OK;
    return qfail(c, AIF_EINVAL, in_place ? "%s is %s with another stride" : "%s is %s", what, other);
}

aif_status check_convert(aif_q8_ctx *c, const aif_q8_convert_args *a, Q8ConvertCall &to)
{
    if (!c || !a) return qfail(c, AIF_EINVAL, "NULL argument");
    Q8_TRY(check_dtype(c, a->dtype, a->n_rows));
    Q8_TRY(check_width(c, "width", a->width, 8, Q8_MAX_WIDTH));
    if (a->block_rows != 1 && a->block_rows != Q8_BLOCK) return qfail(c, AIF_EINVAL, "block_rows %d is neither 1 nor %d", a->block_rows, Q8_BLOCK);
    to.f32 = a->dtype == AIF_F32;
    to.n_rows = a->n_rows, to.width = a->width, to.block_rows = a->block_rows;
    if (a->n_rows == 0) return AIF_OK;
    if (!a->rows) return qfail(c, AIF_EINVAL, "rows: NULL tensor pointer");
    Q8_TRY(check_rows(c, "rows", a->rows, a->stride, a->width, to.f32, to.stride));
    Q8_TRY(check_matrix(c, "q", a->q, a->width, to.q));
    Q8_TRY(check_apart(c, "q", a->q.codes, 0, "rows", a->rows, 0, false));
    to.rows = a->rows;
    return AIF_OK;
}

}  // namespace

extern "C" {

aif_status aif_q8_init(aif_q8_ctx **out)
{
    if (!out) return qfail(nullptr, AIF_EINVAL, "NULL argument");
    int device = -1, n_cu = 0;
    Q8_RUN(nullptr, hipGetDevice(&device));
    Q8_RUN(nullptr, hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, device));
    aif_q8_ctx *c = new (std::nothrow) aif_q8_ctx();
    if (!c) return qfail(nullptr, AIF_ENOMEM, "out of host memory");
    c->device = device;
    if (n_cu > 0) c->n_cu = n_cu;
    *out = c;
    return AIF_OK;
}

void aif_q8_destroy(aif_q8_ctx *ctx) { delete ctx; }

const char *aif_q8_last_error(const aif_q8_ctx *ctx) { return ctx ? ctx->err : g_q8_init_error; }

aif_status aif_q8_rows(aif_q8_ctx *c, const aif_q8_rows_args *a, void *stream)
{
    if (!c || !a) return qfail(c, AIF_EINVAL, "NULL argument");
    Q8_TRY(check_dtype(c, a->dtype, a->n_rows));
    if (a->reserved) return qfail(c, AIF_EINVAL, "reserved field is not zero");
    Q8RowsCall r{};
    r.f32 = a->dtype == AIF_F32;
    Q8_TRY(check_width(c, "width", a->width, r.f32 && !a->q_out.codes ? 4 : 8, Q8_MAX_NORM));
    if (a->norm != 0 && a->norm != 1) return qfail(c, AIF_EINVAL, "norm %d is neither 0 nor 1", a->norm);
    if (a->norm && !(a->eps > 0.f && std::isfinite(a->eps))) return qfail(c, AIF_EINVAL, "eps is not a positive number");
    if (!a->sum_out && !a->out && !a->q_out.codes) return qfail(c, AIF_EINVAL, "no output");
    r.n_rows = a->n_rows, r.width = a->width, r.norm = a->norm != 0, r.eps = a->eps;
    if (a->n_rows == 0) return AIF_OK;
    if (!a->x) return qfail(c, AIF_EINVAL, "x: NULL tensor pointer");
    Q8_TRY(check_rows(c, "x", a->x, a->x_stride, a->width, r.f32, r.x_stride));
    if (a->residual) Q8_TRY(check_rows(c, "residual", a->residual, a->residual_stride, a->width, r.f32, r.residual_stride));
    if (a->sum_out) Q8_TRY(check_rows(c, "sum_out", a->sum_out, a->sum_stride, a->width, r.f32, r.sum_stride));
    if (a->out) Q8_TRY(check_rows(c, "out", a->out, a->out_stride, a->width, r.f32, r.out_stride));
    if (a->norm && a->weight && (uintptr_t)a->weight % 16) return qfail(c, AIF_EINVAL, "weight is not 16-byte aligned");
    if (a->q_out.codes) Q8_TRY(check_matrix(c, "q_out", a->q_out, a->width, r.q));
    Q8_TRY(check_apart(c, "sum_out", a->sum_out, r.sum_stride, "x", a->x, r.x_stride, true));
    Q8_TRY(check_apart(c, "sum_out", a->sum_out, r.sum_stride, "residual", a->residual, r.residual_stride, true));
    Q8_TRY(check_apart(c, "out", a->out, r.out_stride, "x", a->x, r.x_stride, true));
    Q8_TRY(check_apart(c, "out", a->out, r.out_stride, "residual", a->residual, r.residual_stride, true));
    Q8_TRY(check_apart(c, "out", a->out, 0, "sum_out", a->sum_out, 0, false));
    for (const void *p : {a->x, a->residual, a->weight, (const void *)a->sum_out, (const void *)a->out}) Q8_TRY(check_apart(c, "q_out", a->q_out.codes, 0, "another tensor", p, 0, false));
    if (a->norm) for (const void *p : {(const void *)a->sum_out, (const void *)a->out}) Q8_TRY(check_apart(c, "weight", a->weight, 0, "an output", p, 0, false));
    Q8_TRY(check_device(c));
    r.x = a->x, r.residual = a->residual, r.weight = a->norm ? a->weight : nullptr, r.sum_out = a->sum_out, r.out = a->out;
    Q8_RUN(c, launch_q8_rows(r, (hipStream_t)stream));
    return AIF_OK;
}

aif_status aif_q8_linear(aif_q8_ctx *c, const aif_q8_linear_args *a, void *stream)
{
    if (!c || !a) return qfail(c, AIF_EINVAL, "NULL argument");
    Q8_TRY(check_dtype(c, a->dtype, a->n_rows));
    if (a->reserved) return qfail(c, AIF_EINVAL, "reserved field is not zero");
    Q8LinearCall r{};
    r.f32 = a->dtype == AIF_F32;
    Q8_TRY(check_width(c, "k", a->k, 8, Q8_MAX_WIDTH));
    Q8_TRY(check_width(c, "n", a->n, r.f32 && !a->q_out.codes ? 4 : 8, Q8_MAX_WIDTH));
    if (a->n_rows > Q8_MAX_ROWS || (int64_t)a->n_rows * a->n > Q8_MAX_RESULT) return qfail(c, AIF_ERANGE, "%d rows of %d columns are above 2^30 or 2^44 in all", a->n_rows, a->n);
    if (a->activation < AIF_Q8_NONE || a->activation > AIF_Q8_GATE) return qfail(c, AIF_EINVAL, "unknown activation %d", a->activation);
    if ((a->activation == AIF_Q8_GATE) != (a->up.codes != nullptr)) return qfail(c, AIF_EINVAL, "up goes with the gate, and with nothing else");
    if (a->activation == AIF_Q8_GATE && a->bias) return qfail(c, AIF_EINVAL, "a gated layer has no bias");
    if ((a->out != nullptr) == (a->q_out.codes != nullptr)) return qfail(c, AIF_EINVAL, "one of out and q_out is wanted");
    r.m = a->n_rows, r.n = a->n, r.k = a->k, r.act = a->activation;
    if (a->n_rows == 0) return AIF_OK;
    Q8_TRY(check_matrix(c, "a", a->a, a->k, r.a));
    Q8_TRY(check_matrix(c, "w", a->w, a->k, r.w));
    if (a->up.codes) Q8_TRY(check_matrix(c, "up", a->up, a->k, r.up));
    if (a->bias && (uintptr_t)a->bias % 16) return qfail(c, AIF_EINVAL, "bias is not 16-byte aligned");
    if (a->residual) Q8_TRY(check_rows(c, "residual", a->residual, a->residual_stride, a->n, r.f32, r.residual_stride));
    if (a->out) Q8_TRY(check_rows(c, "out", a->out, a->out_stride, a->n, r.f32, r.out_stride));
    else Q8_TRY(check_matrix(c, "q_out", a->q_out, a->n, r.q));
    Q8_TRY(check_apart(c, "out", a->out, r.out_stride, "residual", a->residual, r.residual_stride, true));
    for (const void *p : {(const void *)a->a.codes, (const void *)a->w.codes, (const void *)a->up.codes, a->bias}) Q8_TRY(check_apart(c, "the result", a->out ? a->out : a->q_out.codes, 0, "an operand", p, 0, false));
    Q8_TRY(check_apart(c, "q_out", a->q_out.codes, 0, "residual", a->residual, 0, false));
    Q8_TRY(check_device(c));
    r.bias = a->bias, r.residual = a->residual, r.out = a->out;
    Q8_RUN(c, launch_q8_linear(r, c->n_cu, (hipStream_t)stream));
    return AIF_OK;
}

aif_status aif_q8_weights(aif_q8_ctx *c, const aif_q8_convert_args *a, void *stream)
{
    Q8ConvertCall r{};
    Q8_TRY(check_convert(c, a, r));
    if (r.n_rows == 0) return AIF_OK;
    Q8_TRY(check_device(c));
    Q8_RUN(c, launch_q8_weights(r, (hipStream_t)stream));
    return AIF_OK;
}

aif_status aif_q8_values(aif_q8_ctx *c, const aif_q8_convert_args *a, void *stream)
{
    Q8ConvertCall r{};
    Q8_TRY(check_convert(c, a, r));
    if (r.n_rows == 0) return AIF_OK;
    Q8_TRY(check_device(c));
    Q8_RUN(c, launch_q8_values(r, (hipStream_t)stream));
    return AIF_OK;
}

}  // extern "C"
