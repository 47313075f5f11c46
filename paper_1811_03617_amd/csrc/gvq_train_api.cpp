// C ABI of the operators around an aggregated gradient: 4-bit microscaled matrices, their products and layers, and Muon's step.
// Argument checking only; the arithmetic is in gvq_mx.hip, gvq_mx_product.hip and gvq_muon.hip.
#include <math.h>

#include "gvq_muon.h"
#include "gvq_mx.h"

static bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
static bool is_dtype(gvq_dtype_t t) { return t == GVQ_F32 || t == GVQ_BF16; }
static int64_t size_of(gvq_dtype_t t) { return t == GVQ_BF16 ? 2 : 4; }
static bool in_range(int64_t n) { return n >= 0 && n <= GVQ_MX_MAX; }
static int64_t scales_of(int64_t rows, int64_t cols) { return rows * (gvq_mx_row_bytes(cols) / 16); }
static int64_t codes_of(int64_t rows, int64_t cols) { return rows * gvq_mx_row_bytes(cols); }
static int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

extern "C" {

int64_t gvq_mx_code_bytes(int64_t rows, int64_t cols)
{
    return in_range(rows) && in_range(cols) ? codes_of(rows, cols) : GVQ_EINVAL;
}

int64_t gvq_mx_scale_bytes(int64_t rows, int64_t cols)
{
    return in_range(rows) && in_range(cols) ? scales_of(rows, cols) : GVQ_EINVAL;
}

int gvq_mx_quantize(const void* x, gvq_dtype_t dtype, int64_t rows, int64_t cols, int64_t ld, const void* noise, int64_t noise_ld,
                    void* codes, void* scales, void* codes_t, void* scales_t, void* stream)
{
    if (!is_dtype(dtype) || !in_range(rows) || !in_range(cols) || ld < cols || (noise && noise_ld < cols)) return GVQ_EINVAL;
    if (rows == 0 || cols == 0) return GVQ_OK;
    if (!codes != !scales || !codes_t != !scales_t || (!codes && !codes_t)) return GVQ_EINVAL;
    if (!x) return GVQ_EINVAL;
    if (!aligned(x, size_of(dtype)) || !aligned(codes, 16) || !aligned(scales, 16) || !aligned(codes_t, 16) || !aligned(scales_t, 16))
        return GVQ_EALIGN;
    MxQuantArgs a{};
    a.x = x; a.rows = rows; a.cols = cols; a.ld = ld;
    a.noise = (const unsigned char*)noise; a.noise_ld = noise_ld;
    a.codes = (unsigned char*)codes; a.scales = (unsigned char*)scales;
    a.codes_t = (unsigned char*)codes_t; a.scales_t = (unsigned char*)scales_t;
    return gvq_launch_mx_quantize(a, dtype, (hipStream_t)stream);
}

int gvq_mx_dequantize(const void* codes, const void* scales, int64_t rows, int64_t cols, void* out, gvq_dtype_t out_dtype, int64_t ld,
                      void* stream)
{
    if (!is_dtype(out_dtype) || !in_range(rows) || !in_range(cols) || ld < cols) return GVQ_EINVAL;
    if (rows == 0 || cols == 0) return GVQ_OK;
    if (!codes || !scales || !out) return GVQ_EINVAL;
    if (!aligned(codes, 16) || !aligned(scales, 16) || !aligned(out, size_of(out_dtype))) return GVQ_EALIGN;
    return gvq_launch_mx_dequantize(codes, scales, rows, cols, out, out_dtype, ld, (hipStream_t)stream);
}

int gvq_mx_matmul(const void* a_codes, const void* a_scales, const void* b_codes, const void* b_scales, int64_t m, int64_t n, int64_t k,
                  void* out, gvq_dtype_t out_dtype, int64_t ld, int accumulate, void* stream)
{
    if (!is_dtype(out_dtype) || !in_range(m) || !in_range(n) || !in_range(k) || ld < n) return GVQ_EINVAL;
    if (m == 0 || n == 0) return GVQ_OK;
    if (!out || (k > 0 && (!a_codes || !a_scales || !b_codes || !b_scales))) return GVQ_EINVAL;
    if (!aligned(a_codes, 16) || !aligned(a_scales, 16) || !aligned(b_codes, 16) || !aligned(b_scales, 16) ||
        !aligned(out, size_of(out_dtype)))
        return GVQ_EALIGN;
    return gvq_launch_mx_matmul(a_codes, a_scales, b_codes, b_scales, m, n, k, out, out_dtype, ld, accumulate != 0, (hipStream_t)stream);
}

int64_t gvq_mx_linear_workspace(int64_t rows, int64_t n_in)
{
    return in_range(rows) && in_range(n_in) ? up256(codes_of(rows, n_in)) + up256(scales_of(rows, n_in)) : GVQ_EINVAL;
}

int gvq_mx_linear(const void* x, gvq_dtype_t dtype, int64_t rows, int64_t n_in, int64_t ld_x, const void* w_codes, const void* w_scales,
                  int64_t n_out, void* y, gvq_dtype_t y_dtype, int64_t ld_y, void* workspace, void* stream)
{
    if (!is_dtype(dtype) || !is_dtype(y_dtype) || !in_range(rows) || !in_range(n_in) || !in_range(n_out) || ld_x < n_in || ld_y < n_out)
        return GVQ_EINVAL;
    if (rows == 0 || n_out == 0) return GVQ_OK;
    if (!y || (n_in > 0 && (!x || !w_codes || !w_scales || !workspace))) return GVQ_EINVAL;
    if (!aligned(x, size_of(dtype)) || !aligned(y, size_of(y_dtype)) || !aligned(w_codes, 16) || !aligned(w_scales, 16) ||
        !aligned(workspace, 16))
        return GVQ_EALIGN;
    if (n_in > 0 && gvq_mx_few_numbers_takes(x, dtype, rows, ld_x, n_out, n_in))
        return gvq_launch_mx_few_numbers(x, dtype, ld_x, w_codes, w_scales, rows, n_out, n_in, y, y_dtype, ld_y, (hipStream_t)stream);
    char* w = (char*)workspace;
    char* ws = w + up256(codes_of(rows, n_in));
    if (n_in > 0) {
        const int rc = gvq_mx_quantize(x, dtype, rows, n_in, ld_x, nullptr, 0, w, ws, nullptr, nullptr, stream);
        if (rc != GVQ_OK) return rc;
    }
    return gvq_launch_mx_matmul(w, ws, w_codes, w_scales, rows, n_out, n_in, y, y_dtype, ld_y, false, (hipStream_t)stream);
}

int64_t gvq_mx_linear_backward_workspace(int64_t rows, int64_t n_in, int64_t n_out)
{
    if (!in_range(rows) || !in_range(n_in) || !in_range(n_out)) return GVQ_EINVAL;
    return up256(codes_of(rows, n_out)) + up256(scales_of(rows, n_out)) + up256(codes_of(n_out, rows)) + up256(scales_of(n_out, rows)) +
           up256(codes_of(n_in, rows)) + up256(scales_of(n_in, rows));
}

int gvq_mx_linear_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, gvq_dtype_t dtype, int64_t rows, int64_t n_in,
                           int64_t n_out, const void* noise, int64_t noise_ld, const void* wt_codes, const void* wt_scales, void* dx,
                           gvq_dtype_t dx_dtype, int64_t ld_dx, void* dw, gvq_dtype_t dw_dtype, int64_t ld_dw, int accumulate,
                           void* workspace, void* stream)
{
    if (!is_dtype(dtype) || (dx && !is_dtype(dx_dtype)) || (dw && !is_dtype(dw_dtype)) || !in_range(rows) || !in_range(n_in) || !in_range(n_out))
        return GVQ_EINVAL;
    if (ld_dy < n_out || (noise && noise_ld < n_out) || (dx && ld_dx < n_in) || (dw && (ld_x < n_in || ld_dw < n_in))) return GVQ_EINVAL;
    if (n_in == 0 || (rows == 0 && n_out == 0)) return GVQ_OK;
    if (!dx && !dw) return GVQ_EINVAL;
    const bool some = rows > 0 && n_out > 0;
    if (some && (!dy || !workspace || (dx && (!wt_codes || !wt_scales)) || (dw && !x))) return GVQ_EINVAL;
    if (!aligned(dy, size_of(dtype)) || !aligned(workspace, 16) ||
        (dx && (!aligned(dx, size_of(dx_dtype)) || !aligned(wt_codes, 16) || !aligned(wt_scales, 16))) ||
        (dw && (!aligned(dw, size_of(dw_dtype)) || !aligned(x, size_of(dtype)))))
        return GVQ_EALIGN;
    char* at = (char*)workspace;
    auto take = [&](int64_t bytes) { char* was = at; at += up256(bytes); return was; };
    char *q = take(codes_of(rows, n_out)), *qs = take(scales_of(rows, n_out)), *qt = take(codes_of(n_out, rows)),
         *qts = take(scales_of(n_out, rows)), *xt = take(codes_of(n_in, rows)), *xts = take(scales_of(n_in, rows));
    int rc = GVQ_OK;
    if (some) {
        rc = gvq_mx_quantize(dy, dtype, rows, n_out, ld_dy, noise, noise_ld, dx ? q : nullptr, dx ? qs : nullptr, dw ? qt : nullptr,
                             dw ? qts : nullptr, stream);
        if (rc == GVQ_OK && dw) rc = gvq_mx_quantize(x, dtype, rows, n_in, ld_x, nullptr, 0, nullptr, nullptr, xt, xts, stream);
    }
    if (rc == GVQ_OK && dx && rows > 0)
        rc = gvq_launch_mx_matmul(q, qs, wt_codes, wt_scales, rows, n_in, n_out, dx, dx_dtype, ld_dx, false, (hipStream_t)stream);
    if (rc == GVQ_OK && dw && n_out > 0)
        rc = gvq_launch_mx_matmul(qt, qts, xt, xts, n_out, n_in, rows, dw, dw_dtype, ld_dw, accumulate != 0, (hipStream_t)stream);
    return rc;
}

int64_t gvq_orthogonalize_workspace(int64_t batch, int64_t rows, int64_t cols)
{
    MuonPlan p;
    return gvq_muon_plan(MuonMatrix{batch, rows, cols}, &p) ? p.bytes : GVQ_EINVAL;
}

static bool good_steps(const double* coef, int steps, double eps)
{
    if (steps < 1 || steps > GVQ_MAX_STEPS || !(eps >= 0.0) || isinf(eps)) return false;
    for (int i = 0; coef && i < 3 * steps; ++i)
        if (!isfinite(coef[i])) return false;
    return true;
}

int gvq_orthogonalize(const void* g, gvq_dtype_t dtype, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride,
                      const double* coef, int steps, double eps, void* out, gvq_dtype_t out_dtype, int64_t ld_out, int64_t stride_out,
                      void* workspace, void* stream)
{
    MuonPlan p;
    if (!is_dtype(dtype) || !is_dtype(out_dtype) || !gvq_muon_plan(MuonMatrix{batch, rows, cols}, &p) || !good_steps(coef, steps, eps))
        return GVQ_EINVAL;
    if (ld < cols || ld_out < cols || stride < 0 || stride_out < 0) return GVQ_EINVAL;
    if (batch == 0 || rows == 0 || cols == 0) return GVQ_OK;
    // matrices of the result do not overlap
    if (!g || !out || !workspace || (batch > 1 && stride_out < (rows - 1) * ld_out + cols)) return GVQ_EINVAL;
    if (!aligned(g, size_of(dtype)) || !aligned(out, size_of(out_dtype)) || !aligned(workspace, 16)) return GVQ_EALIGN;
    MuonArgs a{};
    a.x = MuonMatrix{batch, rows, cols};
    a.grad = g; a.grad_dtype = dtype; a.ld_grad = ld; a.stride_grad = stride;
    a.coef = coef; a.steps = steps; a.eps = eps;
    a.out = out; a.out_dtype = out_dtype; a.ld_out = ld_out; a.stride_out = stride_out;
    a.workspace = (char*)workspace;
    return gvq_launch_muon(a, (hipStream_t)stream);
}

int gvq_muon_step(void* weight, gvq_dtype_t weight_dtype, int64_t ld_weight, const void* grad, gvq_dtype_t grad_dtype, int64_t ld_grad,
                  float* momentum, int64_t ld_momentum, int64_t rows, int64_t cols, double lr, double beta, double weight_decay,
                  int nesterov, double scale, const double* coef, int steps, double eps, void* workspace, void* stream)
{
    MuonPlan p;
    if (!is_dtype(weight_dtype) || !is_dtype(grad_dtype) || !gvq_muon_plan(MuonMatrix{1, rows, cols}, &p) || !good_steps(coef, steps, eps))
        return GVQ_EINVAL;
    if (!isfinite(lr) || !isfinite(beta) || !isfinite(weight_decay) || !isfinite(scale)) return GVQ_EINVAL;
    if (ld_weight < cols || ld_grad < cols || ld_momentum < cols) return GVQ_EINVAL;
    if (rows == 0 || cols == 0) return GVQ_OK;
    if (!weight || !grad || !momentum || !workspace) return GVQ_EINVAL;
    if (!aligned(weight, size_of(weight_dtype)) || !aligned(grad, size_of(grad_dtype)) || !aligned(momentum, 4) || !aligned(workspace, 16))
        return GVQ_EALIGN;
    MuonArgs a{};
    a.x = MuonMatrix{1, rows, cols};
    a.grad = grad; a.grad_dtype = grad_dtype; a.ld_grad = ld_grad;
    a.momentum = momentum; a.ld_momentum = ld_momentum;
    a.beta = (float)beta; a.nesterov = nesterov != 0;
    a.coef = coef; a.steps = steps; a.eps = eps;
    a.out = weight; a.out_dtype = weight_dtype; a.ld_out = ld_weight;
    a.update = 1; a.keep = (float)(1.0 - lr * weight_decay); a.rate = (float)(lr * scale);
    a.workspace = (char*)workspace;
    return gvq_launch_muon(a, (hipStream_t)stream);
}

}  // extern "C"
