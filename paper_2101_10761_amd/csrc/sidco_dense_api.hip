// C ABI of the dense operators: argument checks and kernel sequencing.  Contracts are in include/sidco.h.
#include <math.h>

#include "sidco_dense.h"

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
    if (m <= kFewRows)
        launch_mx4_few(p, (hipStream_t)stream);
    else
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
    StreamScratch ws(stream, (size_t)(code_bytes(rows, k) + scale_bytes(rows, k)));
    if (ws.rc != SIDCO_OK) return ws.rc;
    uint8_t* codes = (uint8_t*)ws.data;
    uint8_t* scales = codes + code_bytes(rows, k);
    launch_mx4_quantize(x, type_of(x_dtype), rows, k, ldx, codes, scales, nullptr, nullptr, (hipStream_t)stream);
    const Mx4Product p = {codes, scales, w_codes, w_scales, rows, n, k, alpha, accumulate != 0, c, type_of(c_dtype), ldc};
    if (rows <= kFewRows)
        launch_mx4_few(p, (hipStream_t)stream);
    else
        launch_mx4_product(p, (hipStream_t)stream);
    return launched();
}

}  // extern "C"
