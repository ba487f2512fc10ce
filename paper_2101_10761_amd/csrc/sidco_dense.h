// Internal declarations of the dense operators: 4-bit microscaled gradients, matrices and products, and the orthogonalised
// update.  Element types are the gradient's (kGradF32, kGradF16, kGradBf16).
#ifndef SIDCO_DENSE_H
#define SIDCO_DENSE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sidco_internal.h"

namespace sidco {

constexpr int kMxBlock = 32;   // elements that share an exponent
constexpr int kMxPad = 256;    // a row's elements are padded to this: a 128-byte line of codes, 8 exponents

constexpr int64_t mx4_padded(int64_t n) { return (n + kMxPad - 1) / kMxPad * kMxPad; }

void launch_mx4_compress(const void* grad, int type, float* residual, int64_t d, uint8_t* codes, uint8_t* scales, hipStream_t s);
void launch_mx4_aggregate(const uint8_t* codes, int64_t code_stride, const uint8_t* scales, int64_t scale_stride, int workers,
                          int64_t d, float scale, bool accumulate, float* dense, hipStream_t s);
void launch_mx4_quantize(const void* x, int type, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes, uint8_t* scales,
                         uint8_t* codes_t, uint8_t* scales_t, hipStream_t s);
void launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* out, int type, int64_t ldo,
                           hipStream_t s);

// C = alpha A B^T (+ C): A has m rows, B n rows, both of k columns
struct Mx4Product {
    const uint8_t *a, *a_scales, *b, *b_scales;
    int64_t m, n, k;
    float alpha;
    bool accumulate;
    void* c;
    int type;
    int64_t ldc;
};
void launch_mx4_product(const Mx4Product& p, hipStream_t s);
// The same with rows of A as they are, quantised on the way: where mx4_takes_x(m, n, k).
bool mx4_takes_x(int64_t m, int64_t n, int64_t k);
void launch_mx4_product_x(const Mx4Product& p, const void* x, int type, int64_t ldx, hipStream_t s);

// A batch of matrices orthogonalised, out of x or of the momentum that x moves, into out or into the weights there
struct OrthoCall {
    const void* x;
    int x_type;
    int64_t ldx, x_stride;
    float* momentum;  // NULL: x itself
    float mu;
    bool nesterov;
    int batch;
    int64_t rows, cols;
    int steps;
    float a, b, c, eps;
    int paired;       // steps from the first on whose operands have 22 bits; the others' have 11
    void* out;
    int out_type;
    int64_t ldo, out_stride;
    bool update;      // out = keep * out + gain * result
    float keep, gain;
};
size_t ortho_scratch(const OrthoCall& q);  // of x, ldx and out it needs nothing
void launch_orthogonalize(const OrthoCall& q, char* scratch, hipStream_t s);  // scratch may be NULL for ortho_one_block

}  // namespace sidco
#endif
