// C ABI of the dense operators: argument checks and kernel sequencing.  Contracts are in include/sidco.h.
#include <math.h>

#include "sidco_dense.h"
#include "sidco_ortho_plan.h"

using namespace sidco;

namespace {

constexpr int64_t kMaxRows = INT32_MAX;
constexpr int64_t kMaxInner = 1 << 24;  // k of a product: a tile's rows are addressed with 32 bits

bool element_type(int dtype) { return dtype == SIDCO_GRAD_F32 || dtype == SIDCO_GRAD_F16 || dtype == SIDCO_GRAD_BF16; }
int type_of(int dtype) { return dtype == SIDCO_GRAD_F16 ? kGradF16 : (dtype == SIDCO_GRAD_BF16 ? kGradBf16 : kGradF32); }
bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool aligned_type(const void* p, int dtype) { return aligned(p, dtype == SIDCO_GRAD_F32 ? 4 : 2); }
bool extent(int64_t n) { return n >= 1 && n <= kMaxRows; }

int64_t code_bytes(int64_t rows, int64_t cols) { return rows * (mx4_padded(cols) / 2); }
int64_t scale_bytes(int64_t rows, int64_t cols) { return rows * (mx4_padded(cols) / kMxBlock); }

int check_packed(const uint8_t* codes, const uint8_t* scales)
{
    if (!codes || !scales) return SIDCO_ERR_NULL;
    return aligned(codes, 16) && aligned(scales, 8) ? SIDCO_OK : SIDCO_ERR_ALIGN;
}

int check_result(const void* c, int c_dtype, int64_t n, int64_t ldc, float alpha, int accumulate)
{
    if (!c) return SIDCO_ERR_NULL;
    if (!element_type(c_dtype) || !isfinite(alpha) || (accumulate != 0 && accumulate != 1)) return SIDCO_ERR_ARG;
    if (ldc < n || ldc > kMaxRows) return SIDCO_ERR_SIZE;
    return aligned_type(c, c_dtype) ? SIDCO_OK : SIDCO_ERR_ALIGN;
}

constexpr int64_t kMaxSide = 1 << 21;  // of a matrix that is orthogonalised
constexpr sidco_newton_schulz kNewtonSchulz = {5, 3.4445f, -4.7750f, 2.0315f, 1e-7f, SIDCO_NS_BY_TYPE};

int check_newton_schulz(const sidco_newton_schulz& o)
{
    if (o.steps < 1 || o.steps > 100) return SIDCO_ERR_STAGES;
    if (!isfinite(o.a) || !isfinite(o.b) || !isfinite(o.c) || !(o.eps >= 0.0f) || !isfinite(o.eps)) return SIDCO_ERR_ARG;
    if (o.precision != SIDCO_NS_BY_TYPE && o.precision != SIDCO_NS_HALF && o.precision != SIDCO_NS_FULL) return SIDCO_ERR_ARG;
    return SIDCO_OK;
}

int check_batch(int batch, int64_t rows, int64_t cols)
{
    if (batch < 1 || batch > 65535 || rows < 1 || rows > kMaxSide || cols < 1 || cols > kMaxSide) return SIDCO_ERR_SIZE;
    // a tile's place in the batch has 31 bits
    const int64_t tiles = ((rows + 63) / 64) * ((cols + 63) / 64);
    return tiles <= (int64_t)INT32_MAX / batch ? SIDCO_OK : SIDCO_ERR_SIZE;
}

int paired_steps(const sidco_newton_schulz& o, int out_dtype)
{
    if (o.precision == SIDCO_NS_FULL) return o.steps;
    if (o.precision == SIDCO_NS_HALF) return 0;
    return ortho_paired(o.steps, o.a, o.b, o.c, type_of(out_dtype) == kGradBf16);
}

void take_options(OrthoCall& q, const sidco_newton_schulz& o, int out_dtype)
{
    q.steps = o.steps;
    q.a = o.a;
    q.b = o.b;
    q.c = o.c;
    q.eps = o.eps;
    q.paired = paired_steps(o, out_dtype);
}

int orthogonalize(void* stream, OrthoCall& q, const sidco_newton_schulz& o, int out_dtype)
{
    take_options(q, o, out_dtype);
    if (ortho_one_block(q.rows, q.cols, q.ldx, q.paired > 0)) {
        launch_orthogonalize(q, nullptr, (hipStream_t)stream);
        return launched();
    }
    StreamScratch ws(stream, ortho_scratch(q));
    if (ws.rc != SIDCO_OK) return ws.rc;
    launch_orthogonalize(q, ws.data, (hipStream_t)stream);
    return launched();
}

}  // namespace

extern "C" {

int64_t sidco_mx4_code_bytes(int64_t rows, int64_t cols)
{
    return extent(rows) && extent(cols) ? code_bytes(rows, cols) : SIDCO_ERR_SIZE;
}

int64_t sidco_mx4_scale_bytes(int64_t rows, int64_t cols)
{
    return extent(rows) && extent(cols) ? scale_bytes(rows, cols) : SIDCO_ERR_SIZE;
}

int sidco_mx4_compress(void* stream, const void* grad, int grad_dtype, float* residual, int64_t d, uint8_t* codes, uint8_t* scales)
{
    if (!grad || !codes || !scales) return SIDCO_ERR_NULL;
    if (!element_type(grad_dtype)) return SIDCO_ERR_ARG;
    if (!extent(d)) return SIDCO_ERR_SIZE;
    if (!aligned_type(grad, grad_dtype) || !aligned(residual, 4)) return SIDCO_ERR_ALIGN;
    if (int rc = check_packed(codes, scales)) return rc;
    if (residual && (const void*)residual == grad) return SIDCO_ERR_ARG;
    launch_mx4_compress(grad, type_of(grad_dtype), residual, d, codes, scales, (hipStream_t)stream);
    return launched();
}

int sidco_mx4_aggregate(void* stream, const uint8_t* codes, int64_t code_stride, const uint8_t* scales, int64_t scale_stride,
                        int workers, int64_t d, float scale, int accumulate, float* dense)
{
    if (!codes || !scales || !dense) return SIDCO_ERR_NULL;
    if (!extent(d) || workers < 1) return SIDCO_ERR_SIZE;
    if (!isfinite(scale) || (accumulate != 0 && accumulate != 1)) return SIDCO_ERR_ARG;
    if (int rc = check_packed(codes, scales)) return rc;
    if (!aligned(dense, 4)) return SIDCO_ERR_ALIGN;
    if (workers > 1) {
        if (code_stride < code_bytes(1, d) || scale_stride < scale_bytes(1, d)) return SIDCO_ERR_SIZE;
        if (code_stride % 16 != 0 || scale_stride % 8 != 0) return SIDCO_ERR_ALIGN;
    }
    launch_mx4_aggregate(codes, code_stride, scales, scale_stride, workers, d, scale, accumulate != 0, dense, (hipStream_t)stream);
    return launched();
}

int sidco_mx4_quantize(void* stream, const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes,
                       uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t)
{
    if (!x || (!codes && !codes_t)) return SIDCO_ERR_NULL;
    if (!element_type(dtype)) return SIDCO_ERR_ARG;
    if (!extent(rows) || !extent(cols) || ldx < cols || ldx > kMaxRows) return SIDCO_ERR_SIZE;
    if ((mx4_padded(rows) / 128) * (mx4_padded(cols) / 128) > (int64_t)INT32_MAX) return SIDCO_ERR_SIZE;
    if (!aligned_type(x, dtype)) return SIDCO_ERR_ALIGN;
    if (codes || scales)
        if (int rc = check_packed(codes, scales)) return rc;
    if (codes_t || scales_t)
        if (int rc = check_packed(codes_t, scales_t)) return rc;
    launch_mx4_quantize(x, type_of(dtype), rows, cols, ldx, codes, scales, codes_t, scales_t, (hipStream_t)stream);
    return launched();
}

int sidco_mx4_dequantize(void* stream, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* out, int dtype,
                         int64_t ldo)
{
    if (!out) return SIDCO_ERR_NULL;
    if (int rc = check_packed(codes, scales)) return rc;
    if (!element_type(dtype)) return SIDCO_ERR_ARG;
    if (!extent(rows) || !extent(cols) || ldo < cols || ldo > kMaxRows) return SIDCO_ERR_SIZE;
    if (!aligned_type(out, dtype)) return SIDCO_ERR_ALIGN;
    launch_mx4_dequantize(codes, scales, rows, cols, out, type_of(dtype), ldo, (hipStream_t)stream);
    return launched();
}

int sidco_mx4_matmul(void* stream, const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales,
                     int64_t m, int64_t n, int64_t k, float alpha, int accumulate, void* c, int c_dtype, int64_t ldc)
{
    if (int rc = check_packed(a_codes, a_scales)) return rc;
    if (int rc = check_packed(b_codes, b_scales)) return rc;
    if (!extent(m) || !extent(n) || k < 1 || k > kMaxInner) return SIDCO_ERR_SIZE;
    if (int rc = check_result(c, c_dtype, n, ldc, alpha, accumulate)) return rc;
    if (((m + 63) / 64) * ((n + 63) / 64) > (int64_t)INT32_MAX) return SIDCO_ERR_SIZE;
    const Mx4Product p = {a_codes, a_scales, b_codes, b_scales, m, n, k, alpha, accumulate != 0, c, type_of(c_dtype), ldc};
    launch_mx4_product(p, (hipStream_t)stream);
    return launched();
}

size_t sidco_workspace_bytes_mx4_linear(int64_t rows, int64_t k)
{
    if (!extent(rows) || k < 1 || k > kMaxInner) return 0;
    return workspace_with_scratch((size_t)(code_bytes(rows, k) + scale_bytes(rows, k)));
}

int sidco_mx4_linear(void* stream, const void* x, int x_dtype, int64_t rows, int64_t k, int64_t ldx, const uint8_t* w_codes,
                     const uint8_t* w_scales, int64_t n, float alpha, int accumulate, void* c, int c_dtype, int64_t ldc)
{
    if (!x) return SIDCO_ERR_NULL;
    if (int rc = check_packed(w_codes, w_scales)) return rc;
    if (!element_type(x_dtype)) return SIDCO_ERR_ARG;
    if (!extent(rows) || !extent(n) || k < 1 || k > kMaxInner || ldx < k || ldx > kMaxRows) return SIDCO_ERR_SIZE;
    if ((mx4_padded(rows) / 128) * (mx4_padded(k) / 128) > (int64_t)INT32_MAX) return SIDCO_ERR_SIZE;
    if (((rows + 63) / 64) * ((n + 63) / 64) > (int64_t)INT32_MAX) return SIDCO_ERR_SIZE;
    if (!aligned_type(x, x_dtype)) return SIDCO_ERR_ALIGN;
    if (int rc = check_result(c, c_dtype, n, ldc, alpha, accumulate)) return rc;
    if (mx4_takes_x(rows, n, k)) {
        const Mx4Product p = {nullptr, nullptr, w_codes, w_scales, rows, n, k, alpha, accumulate != 0, c, type_of(c_dtype), ldc};
        launch_mx4_product_x(p, x, type_of(x_dtype), ldx, (hipStream_t)stream);
        return launched();
    }
    StreamScratch ws(stream, (size_t)(code_bytes(rows, k) + scale_bytes(rows, k)));
    if (ws.rc != SIDCO_OK) return ws.rc;
    uint8_t* codes = (uint8_t*)ws.data;
    uint8_t* scales = codes + code_bytes(rows, k);
    launch_mx4_quantize(x, type_of(x_dtype), rows, k, ldx, codes, scales, nullptr, nullptr, (hipStream_t)stream);
    const Mx4Product p = {codes, scales, w_codes, w_scales, rows, n, k, alpha, accumulate != 0, c, type_of(c_dtype), ldc};
    launch_mx4_product(p, (hipStream_t)stream);
    return launched();
}

void sidco_newton_schulz_default(sidco_newton_schulz* opt)
{
    if (opt) *opt = kNewtonSchulz;
}

size_t sidco_workspace_bytes_orthogonalize(int batch, int64_t rows, int64_t cols, int out_dtype, const sidco_newton_schulz* opt)
{
    const sidco_newton_schulz o = opt ? *opt : kNewtonSchulz;
    if (check_batch(batch, rows, cols) != SIDCO_OK || !element_type(out_dtype) || check_newton_schulz(o) != SIDCO_OK) return 0;
    OrthoCall q = {};
    q.batch = batch;
    q.rows = rows;
    q.cols = cols;
    take_options(q, o, out_dtype);
    return workspace_with_scratch(ortho_scratch(q));
}

int sidco_orthogonalize(void* stream, const void* x, int x_dtype, int64_t ldx, int64_t x_stride, int batch, int64_t rows, int64_t cols,
                        const sidco_newton_schulz* opt, void* out, int out_dtype, int64_t ldo, int64_t out_stride)
{
    if (!x || !out) return SIDCO_ERR_NULL;
    if (!element_type(x_dtype) || !element_type(out_dtype)) return SIDCO_ERR_ARG;
    if (int rc = check_batch(batch, rows, cols)) return rc;
    if (ldx < cols || ldo < cols || ldx > kMaxRows || ldo > kMaxRows) return SIDCO_ERR_SIZE;
    if (batch > 1 && (x_stride < rows * ldx || out_stride < rows * ldo)) return SIDCO_ERR_SIZE;
    if (!aligned_type(x, x_dtype) || !aligned_type(out, out_dtype)) return SIDCO_ERR_ALIGN;
    const sidco_newton_schulz o = opt ? *opt : kNewtonSchulz;
    if (int rc = check_newton_schulz(o)) return rc;
    OrthoCall q = {};
    q.x = x;
    q.x_type = type_of(x_dtype);
    q.ldx = ldx;
    q.x_stride = x_stride;
    q.batch = batch;
    q.rows = rows;
    q.cols = cols;
    q.out = out;
    q.out_type = type_of(out_dtype);
    q.ldo = ldo;
    q.out_stride = out_stride;
    return orthogonalize(stream, q, o, out_dtype);
}

int sidco_muon_step(void* stream, const void* grad, int grad_dtype, float* momentum, void* weight, int weight_dtype, int batch,
                    int64_t rows, int64_t cols, float lr, float mu, int nesterov, float weight_decay, float scale,
                    const sidco_newton_schulz* opt)
{
    if (!grad || !momentum || !weight) return SIDCO_ERR_NULL;
    if (!element_type(grad_dtype) || !element_type(weight_dtype)) return SIDCO_ERR_ARG;
    if (int rc = check_batch(batch, rows, cols)) return rc;
    if (!isfinite(lr) || !isfinite(mu) || !isfinite(weight_decay) || !isfinite(scale) || (nesterov != 0 && nesterov != 1))
        return SIDCO_ERR_ARG;
    if (!aligned_type(grad, grad_dtype) || !aligned(momentum, 4) || !aligned_type(weight, weight_dtype)) return SIDCO_ERR_ALIGN;
    if (grad == (const void*)momentum || grad == weight || (void*)momentum == weight) return SIDCO_ERR_ARG;
    const sidco_newton_schulz o = opt ? *opt : kNewtonSchulz;
    if (int rc = check_newton_schulz(o)) return rc;
    OrthoCall q = {};
    q.x = grad;
    q.x_type = type_of(grad_dtype);
    q.ldx = cols;
    q.x_stride = rows * cols;
    q.momentum = momentum;
    q.mu = mu;
    q.nesterov = nesterov != 0;
    q.batch = batch;
    q.rows = rows;
    q.cols = cols;
    q.out = weight;
    q.out_type = type_of(weight_dtype);
    q.ldo = cols;
    q.out_stride = rows * cols;
    q.update = true;
    q.keep = 1.0f - lr * weight_decay;
    q.gain = -lr * scale;
    return orthogonalize(stream, q, o, weight_dtype);
}

}  // extern "C"
