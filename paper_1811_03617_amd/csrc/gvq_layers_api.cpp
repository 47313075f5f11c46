// C ABI of the 8-bit layers, the gated block made of them, and the loss on a teacher's top logits.
// Argument checking only; the arithmetic is in gvq_i8.hip, gvq_i8_product.hip and gvq_distill.hip.
#include <math.h>

#include "gvq_distill.h"
#include "gvq_i8.h"

static bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
static bool is_dtype(gvq_dtype_t t) { return t == GVQ_F32 || t == GVQ_BF16; }
static bool is_activation(gvq_activation_t t) { return t == GVQ_SILU || t == GVQ_GELU; }
static int64_t size_of(gvq_dtype_t t) { return t == GVQ_BF16 ? 2 : 4; }
static bool in_range(int64_t n) { return n >= 0 && n <= GVQ_MX_MAX; }
static bool is_sum(int64_t n) { return n >= 0 && n <= GVQ_I8_MAX_SUM; }
static int64_t codes_of(int64_t rows, int64_t cols) { return rows * gvq_i8_row_bytes(cols); }
static int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }
static int64_t matrix_of(int64_t rows, int64_t cols) { return up256(codes_of(rows, cols)) + up256(4 * rows); }
static int64_t chunks_of(int64_t rows) { return (rows + gvq_i8_chunk_rows(rows) - 1) / gvq_i8_chunk_rows(rows); }
static int64_t peaks_of(int64_t rows, int64_t cols) { return up256(4 * chunks_of(rows) * cols); }

namespace {
// Pieces of a workspace one behind the other.
struct Pieces {
    char* at;
    char* take(int64_t bytes)
    {
        char* was = at;
        at += up256(bytes);
        return was;
    }
};
struct Codes {
    signed char* codes;
    float* scales;
};
Codes take_matrix(Pieces& p, int64_t rows, int64_t cols)
{
    signed char* c = (signed char*)p.take(codes_of(rows, cols));
    return Codes{c, (float*)p.take(4 * rows)};
}

I8QuantArgs matrix(const void* x, int64_t rows, int64_t cols, int64_t ld, Codes q, Codes qt, void* peaks)
{
    I8QuantArgs a{};
    a.x = x; a.rows = rows; a.cols = cols; a.ld = ld;
    a.codes = q.codes; a.scales = q.scales;
    a.codes_t = qt.codes; a.scales_t = qt.scales;
    a.peaks = (unsigned int*)peaks;
    return a;
}
int quantize(const void* x, gvq_dtype_t dtype, int64_t rows, int64_t cols, int64_t ld, Codes q, Codes qt, void* peaks, void* stream)
{
    const I8QuantArgs a = matrix(x, rows, cols, ld, q, qt, peaks);
    return gvq_launch_i8_quantize(&a, 1, dtype, (hipStream_t)stream);
}

// A sum over nothing has no scales.
I8ProductArgs product(const void* a_codes, const void* a_scales, const void* b_codes, const void* b_scales, int64_t m, int64_t n, int64_t k,
                      void* out, int64_t ld, bool accumulate)
{
    I8ProductArgs a{};
    a.a = (const signed char*)a_codes; a.b = (const signed char*)b_codes;
    a.a_scales = k > 0 ? (const float*)a_scales : nullptr;
    a.b_scales = k > 0 ? (const float*)b_scales : nullptr;
    a.ldk = gvq_i8_row_bytes(k);
    a.m = (int)m; a.n = (int)n;
    a.out = out; a.ld = ld; a.accumulate = accumulate;
    return a;
}
}  // namespace

extern "C" {

int64_t gvq_i8_code_bytes(int64_t rows, int64_t cols)
{
    return in_range(rows) && in_range(cols) ? codes_of(rows, cols) : GVQ_EINVAL;
}

int64_t gvq_i8_quantize_workspace(int64_t rows, int64_t cols)
{
    return in_range(rows) && in_range(cols) ? peaks_of(rows, cols) : GVQ_EINVAL;
}

int gvq_i8_quantize(const void* x, gvq_dtype_t dtype, int64_t rows, int64_t cols, int64_t ld, void* codes, float* scales, void* codes_t,
                    float* scales_t, void* workspace, void* stream)
{
    if (!is_dtype(dtype) || !in_range(rows) || !in_range(cols) || ld < cols) return GVQ_EINVAL;
    if (rows == 0 || cols == 0) return GVQ_OK;
    if (!codes != !scales || !codes_t != !scales_t || (!codes && !codes_t) || !x || (codes_t && !workspace)) return GVQ_EINVAL;
    if (!aligned(x, size_of(dtype)) || !aligned(codes, 16) || !aligned(scales, 16) || !aligned(codes_t, 16) || !aligned(scales_t, 16) ||
        (codes_t && !aligned(workspace, 16)))
        return GVQ_EALIGN;
    return quantize(x, dtype, rows, cols, ld, Codes{(signed char*)codes, scales}, Codes{(signed char*)codes_t, scales_t}, workspace, stream);
}

int gvq_i8_dequantize(const void* codes, const float* scales, int64_t rows, int64_t cols, void* out, gvq_dtype_t out_dtype, int64_t ld,
                      void* stream)
{
    if (!is_dtype(out_dtype) || !in_range(rows) || !in_range(cols) || ld < cols) return GVQ_EINVAL;
    if (rows == 0 || cols == 0) return GVQ_OK;
    if (!codes || !scales || !out) return GVQ_EINVAL;
    if (!aligned(codes, 16) || !aligned(scales, 16) || !aligned(out, size_of(out_dtype))) return GVQ_EALIGN;
    return gvq_launch_i8_dequantize(codes, scales, rows, cols, out, out_dtype, ld, (hipStream_t)stream);
}

int gvq_i8_matmul(const void* a_codes, const float* a_scales, const void* b_codes, const float* b_scales, int64_t m, int64_t n, int64_t k,
                  void* out, gvq_dtype_t out_dtype, int64_t ld, int accumulate, void* stream)
{
    if (!is_dtype(out_dtype) || !in_range(m) || !in_range(n) || !is_sum(k) || ld < n) return GVQ_EINVAL;
    if (m == 0 || n == 0) return GVQ_OK;
    if (!out || (k > 0 && (!a_codes || !a_scales || !b_codes || !b_scales))) return GVQ_EINVAL;
    if (!aligned(a_codes, 16) || !aligned(a_scales, 16) || !aligned(b_codes, 16) || !aligned(b_scales, 16) || !aligned(out, size_of(out_dtype)))
        return GVQ_EALIGN;
    return gvq_launch_i8_product(product(a_codes, a_scales, b_codes, b_scales, m, n, k, out, ld, accumulate != 0), I8_PLAIN, out_dtype,
                                 (hipStream_t)stream);
}

int64_t gvq_i8_linear_workspace(int64_t rows, int64_t n_in)
{
    return in_range(rows) && is_sum(n_in) ? matrix_of(rows, n_in) : GVQ_EINVAL;
}

// linear (both = 1) and gated (2: w has twice n_out rows).
static int forward(const void* x, gvq_dtype_t dtype, int64_t rows, int64_t n_in, int64_t ld_x, const void* w_codes, const float* w_scales,
                   int64_t n_out, int both, int activation, void* y, gvq_dtype_t y_dtype, int64_t ld_y, void* workspace, void* stream)
{
    if (!is_dtype(dtype) || !is_dtype(y_dtype) || !in_range(rows) || !is_sum(n_in) || !in_range(n_out) || !in_range(both * n_out) || ld_x < n_in ||
        ld_y < n_out)
        return GVQ_EINVAL;
    if (rows == 0 || n_out == 0) return GVQ_OK;
    if (!y || (n_in > 0 && (!x || !w_codes || !w_scales || !workspace))) return GVQ_EINVAL;
    if (!aligned(y, size_of(y_dtype)) ||
        (n_in > 0 && (!aligned(x, size_of(dtype)) || !aligned(w_codes, 16) || !aligned(w_scales, 16) || !aligned(workspace, 16))))
        return GVQ_EALIGN;
    const I8Mode mode = both == 1 ? I8_PLAIN : I8_GATED;
    Codes q{nullptr, nullptr};
    if (n_in > 0) {
        Pieces p{(char*)workspace};
        q = take_matrix(p, rows, n_in);
    }
    I8ProductArgs a = product(q.codes, q.scales, w_codes, w_scales, rows, n_out, n_in, y, ld_y, false);
    a.activation = activation;
    if (n_in > 0) {
        if (gvq_i8_few_numbers_takes(x, dtype, rows, ld_x, n_in, mode))
            return gvq_launch_i8_few_numbers(a, x, dtype, ld_x, n_in, mode, y_dtype, (hipStream_t)stream);
        const int rc = quantize(x, dtype, rows, n_in, ld_x, q, Codes{nullptr, nullptr}, nullptr, stream);
        if (rc != GVQ_OK) return rc;
    }
    return gvq_launch_i8_product(a, mode, y_dtype, (hipStream_t)stream);
}

int gvq_i8_linear(const void* x, gvq_dtype_t dtype, int64_t rows, int64_t n_in, int64_t ld_x, const void* w_codes, const float* w_scales,
                  int64_t n_out, void* y, gvq_dtype_t y_dtype, int64_t ld_y, void* workspace, void* stream)
{
    return forward(x, dtype, rows, n_in, ld_x, w_codes, w_scales, n_out, 1, 0, y, y_dtype, ld_y, workspace, stream);
}

int64_t gvq_i8_linear_backward_workspace(int64_t rows, int64_t n_in, int64_t n_out)
{
    if (!is_sum(rows) || !in_range(n_in) || !is_sum(n_out)) return GVQ_EINVAL;
    return matrix_of(rows, n_out) + matrix_of(n_out, rows) + peaks_of(rows, n_out) + matrix_of(n_in, rows) + peaks_of(rows, n_in);
}

// Whether there is nothing to do, or the arguments are refused: what a backward pass looks at before it begins.  dy: of the layer's outputs, or
// null where it is about to be made.  Only dx sums the outputs, only dw the rows.
static int look_at_backward(const void* dy, bool dy_is_given, int64_t ld_dy, const void* x, int64_t ld_x, gvq_dtype_t dtype, int64_t rows, int64_t n_in,
                            int64_t n_out, const void* wt_codes, const float* wt_scales, const void* dx, gvq_dtype_t dx_dtype, int64_t ld_dx,
                            const void* dw, gvq_dtype_t dw_dtype, int64_t ld_dw, const void* workspace, bool* nothing)
{
    *nothing = false;
    if (!is_dtype(dtype) || (dx && !is_dtype(dx_dtype)) || (dw && !is_dtype(dw_dtype)) || !in_range(rows) || !in_range(n_in) || !in_range(n_out) ||
        (dw && !is_sum(rows)) || (dx && !is_sum(n_out)))
        return GVQ_EINVAL;
    if (ld_dy < n_out || (dx && ld_dx < n_in) || (dw && (ld_x < n_in || ld_dw < n_in))) return GVQ_EINVAL;
    *nothing = n_in == 0 || (rows == 0 && n_out == 0);
    if (*nothing) return GVQ_OK;
    if (!dx && !dw) return GVQ_EINVAL;
    const bool some = rows > 0 && n_out > 0;
    if (some && ((dy_is_given && !dy) || !workspace || (dx && (!wt_codes || !wt_scales)) || (dw && !x))) return GVQ_EINVAL;
    if ((some && (!aligned(dy, size_of(dtype)) || !aligned(workspace, 16))) ||
        (dx && (!aligned(dx, size_of(dx_dtype)) || !aligned(wt_codes, 16) || !aligned(wt_scales, 16))) ||
        (dw && (!aligned(dw, size_of(dw_dtype)) || !aligned(x, size_of(dtype)))))
        return GVQ_EALIGN;
    return GVQ_OK;
}

int gvq_i8_linear_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, gvq_dtype_t dtype, int64_t rows, int64_t n_in,
                           int64_t n_out, const void* wt_codes, const float* wt_scales, void* dx, gvq_dtype_t dx_dtype, int64_t ld_dx, void* dw,
                           gvq_dtype_t dw_dtype, int64_t ld_dw, int accumulate, void* workspace, void* stream)
{
    bool nothing;
    int rc = look_at_backward(dy, true, ld_dy, x, ld_x, dtype, rows, n_in, n_out, wt_codes, wt_scales, dx, dx_dtype, ld_dx, dw, dw_dtype, ld_dw,
                              workspace, &nothing);
    if (rc != GVQ_OK || nothing) return rc;
    const bool some = rows > 0 && n_out > 0;
    Pieces p{(char*)workspace};
    const Codes none{nullptr, nullptr};
    Codes q = none, qt = none, xt = none;
    if (some) {
        void *y_peaks = nullptr, *x_peaks = nullptr;
        if (dx) q = take_matrix(p, rows, n_out);
        if (dw) {
            qt = take_matrix(p, n_out, rows);
            y_peaks = p.take(peaks_of(rows, n_out));
            xt = take_matrix(p, n_in, rows);
            x_peaks = p.take(peaks_of(rows, n_in));
        }
        const I8QuantArgs both[2] = {matrix(dy, rows, n_out, ld_dy, q, qt, y_peaks), matrix(x, rows, n_in, ld_x, none, xt, x_peaks)};
        rc = gvq_launch_i8_quantize(both, dw ? 2 : 1, dtype, (hipStream_t)stream);
        if (rc != GVQ_OK) return rc;
    }
    const I8ProductArgs to_x = product(q.codes, q.scales, wt_codes, wt_scales, rows, n_in, n_out, dx, ld_dx, false),
                        to_w = product(qt.codes, qt.scales, xt.codes, xt.scales, n_out, n_in, rows, dw, ld_dw, accumulate != 0);
    const bool want_x = dx && rows > 0, want_w = dw && n_out > 0;
    if (want_x && want_w) return gvq_launch_i8_products(to_x, dx_dtype, to_w, dw_dtype, (hipStream_t)stream);
    if (want_x) return gvq_launch_i8_product(to_x, I8_PLAIN, dx_dtype, (hipStream_t)stream);
    return want_w ? gvq_launch_i8_product(to_w, I8_PLAIN, dw_dtype, (hipStream_t)stream) : GVQ_OK;
}

int gvq_i8_gated(const void* x, gvq_dtype_t dtype, int64_t rows, int64_t n_in, int64_t ld_x, const void* w_codes, const float* w_scales, int64_t n,
                 gvq_activation_t activation, void* h, gvq_dtype_t h_dtype, int64_t ld_h, void* workspace, void* stream)
{
    if (!is_activation(activation)) return GVQ_EINVAL;
    return forward(x, dtype, rows, n_in, ld_x, w_codes, w_scales, n, 2, activation, h, h_dtype, ld_h, workspace, stream);
}

static int look_at_gradient(const void* dh, int64_t ld_dh, const void* x, int64_t ld_x, gvq_dtype_t dtype, int64_t rows, int64_t n_in, int64_t n,
                            const void* w_codes, const float* w_scales, gvq_activation_t activation, const void* dg, bool dg_is_given,
                            int64_t ld_dg, const void* workspace)
{
    if (!is_activation(activation) || !is_dtype(dtype) || !in_range(rows) || !is_sum(n_in) || !in_range(n) || !in_range(2 * n) || ld_x < n_in ||
        ld_dh < n || ld_dg < 2 * n)
        return GVQ_EINVAL;
    if (rows == 0 || n == 0) return GVQ_OK;
    if (!dh || (dg_is_given && !dg) || (n_in > 0 && (!x || !w_codes || !w_scales || !workspace))) return GVQ_EINVAL;
    if (!aligned(dh, size_of(dtype)) || !aligned(dg, size_of(dtype)) ||
        (n_in > 0 && (!aligned(x, size_of(dtype)) || !aligned(w_codes, 16) || !aligned(w_scales, 16) || !aligned(workspace, 16))))
        return GVQ_EALIGN;
    return GVQ_OK;
}

int gvq_i8_gated_gradient(const void* dh, int64_t ld_dh, const void* x, int64_t ld_x, gvq_dtype_t dtype, int64_t rows, int64_t n_in, int64_t n,
                          const void* w_codes, const float* w_scales, gvq_activation_t activation, void* dg, int64_t ld_dg, void* workspace,
                          void* stream)
{
    int rc = look_at_gradient(dh, ld_dh, x, ld_x, dtype, rows, n_in, n, w_codes, w_scales, activation, dg, true, ld_dg, workspace);
    if (rc != GVQ_OK || rows == 0 || n == 0) return rc;
    Codes q{nullptr, nullptr};
    if (n_in > 0) {
        Pieces p{(char*)workspace};
        q = take_matrix(p, rows, n_in);
        rc = quantize(x, dtype, rows, n_in, ld_x, q, Codes{nullptr, nullptr}, nullptr, stream);
        if (rc != GVQ_OK) return rc;
    }
    I8ProductArgs a = product(q.codes, q.scales, w_codes, w_scales, rows, n, n_in, dg, ld_dg, false);
    a.activation = activation;
    a.dh = dh; a.ld_dh = ld_dh;
    return gvq_launch_i8_product(a, I8_INNER, dtype, (hipStream_t)stream);
}

// [gradient of the inner sums, in the widest type][what the two calls need, one after the other]
int64_t gvq_i8_gated_backward_workspace(int64_t rows, int64_t n_in, int64_t n)
{
    const int64_t inner = gvq_i8_linear_workspace(rows, n_in), outer = n >= 0 && n <= GVQ_I8_MAX_SUM / 2 ? gvq_i8_linear_backward_workspace(rows, n_in, 2 * n) : GVQ_EINVAL;
    if (inner < 0 || outer < 0) return GVQ_EINVAL;
    return up256(8 * rows * n) + (inner > outer ? inner : outer);
}

int gvq_i8_gated_backward(const void* dh, int64_t ld_dh, const void* x, int64_t ld_x, gvq_dtype_t dtype, int64_t rows, int64_t n_in, int64_t n,
                          const void* w_codes, const float* w_scales, const void* wt_codes, const float* wt_scales, gvq_activation_t activation,
                          void* dx, gvq_dtype_t dx_dtype, int64_t ld_dx, void* dw, gvq_dtype_t dw_dtype, int64_t ld_dw, int accumulate,
                          void* workspace, void* stream)
{
    if (!in_range(n)) return GVQ_EINVAL;
    bool nothing;
    int rc = look_at_gradient(dh, ld_dh, x, ld_x, dtype, rows, n_in, n, w_codes, w_scales, activation, nullptr, false, 2 * n, workspace);
    if (rc == GVQ_OK)
        rc = look_at_backward(nullptr, false, 2 * n, x, ld_x, dtype, rows, n_in, 2 * n, wt_codes, wt_scales, dx, dx_dtype, ld_dx, dw, dw_dtype, ld_dw,
                              workspace, &nothing);
    if (rc != GVQ_OK || nothing) return rc;
    Pieces p{(char*)workspace};
    void* dg = rows > 0 && n > 0 ? p.take(8 * rows * n) : nullptr;
    rc = gvq_i8_gated_gradient(dh, ld_dh, x, ld_x, dtype, rows, n_in, n, w_codes, w_scales, activation, dg, 2 * n, p.at, stream);
    if (rc != GVQ_OK) return rc;
    return gvq_i8_linear_backward(dg, 2 * n, x, ld_x, dtype, rows, n_in, 2 * n, wt_codes, wt_scales, dx, dx_dtype, ld_dx, dw, dw_dtype, ld_dw,
                                  accumulate, p.at, stream);
}

int64_t gvq_distill_workspace(int64_t rows, int64_t vocab, int64_t n_top)
{
    if (!in_range(rows) || !in_range(vocab) || n_top < 0 || n_top > GVQ_MAX_TOP) return GVQ_EINVAL;
    const int parts = gvq_distill_parts(rows, vocab);
    return parts > 1 ? up256(8 * rows * parts) : 0;
}

int gvq_distill(const void* logits, gvq_dtype_t dtype, int64_t rows, int64_t vocab, int64_t ld, const void* top, gvq_dtype_t top_dtype,
                const int64_t* index, int64_t n_top, int64_t ld_top, int64_t ld_index, const float* weight, double temperature, float* loss,
                void* grad, int64_t ld_grad, void* workspace, void* stream)
{
    if (!is_dtype(dtype) || !is_dtype(top_dtype) || !in_range(rows) || !in_range(vocab) || n_top < 0 || n_top > GVQ_MAX_TOP) return GVQ_EINVAL;
    if (ld < vocab || ld_top < n_top || ld_index < n_top || (grad && ld_grad < vocab)) return GVQ_EINVAL;
    if (grad && grad == logits && ld_grad != ld && rows > 1) return GVQ_EINVAL;   // in place, but other rows' places
    if (!(temperature >= 1e-3 && temperature <= 1e3)) return GVQ_EINVAL;
    if (rows == 0) return GVQ_OK;
    if (!loss || (vocab > 0 && !logits) || (n_top > 0 && (!top || !index)) || (gvq_distill_parts(rows, vocab) > 1 && !workspace)) return GVQ_EINVAL;
    if (!aligned(logits, size_of(dtype)) || !aligned(top, size_of(top_dtype)) || !aligned(index, 8) || !aligned(weight, 4) || !aligned(loss, 4) ||
        !aligned(grad, size_of(dtype)) || !aligned(workspace, 16))
        return GVQ_EALIGN;
    DistillArgs a{};
    a.logits = logits; a.rows = rows; a.ld = ld; a.vocab = (int)vocab;
    a.top = top; a.top_bf16 = top_dtype == GVQ_BF16; a.ld_top = ld_top;
    a.index = index; a.ld_index = ld_index; a.n_top = (int)n_top;
    a.weight = weight;
    a.t64 = temperature; a.t = (float)temperature; a.per_t = (float)(1.0 / temperature); a.log2_t = (float)(1.4426950408889634 / temperature);
    a.loss = loss; a.grad = grad; a.ld_grad = ld_grad;
    return gvq_launch_distill(a, dtype, workspace, (hipStream_t)stream);
}

}  // extern "C"
