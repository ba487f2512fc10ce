// Internal declarations of a language model's operators: the embedding and its gradient, dropout, and softmax cross entropy
// over a vocabulary.  Element types are the gradient's (kGradF32, kGradF16, kGradBf16).
#ifndef SIDCO_LANGUAGE_H
#define SIDCO_LANGUAGE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sidco_internal.h"

namespace sidco {

// Words: what stands at place i is a row of the table, or with a value outside [0, vocab) padding.
struct Words {
    const void* at;
    bool wide;  // 64 bits
    int64_t n;
    int64_t vocab;
};

// Rows of `cols` elements, `ld` apart.
struct Matrix {
    void* at;
    int type;
    int64_t ld;
};

struct Lookup {
    Words words;
    Matrix table;  // read for the lookup, written for its gradient
    Matrix rows;   // a row for each word: written, or read
    int64_t cols;
    float scale;
    bool accumulate;
};
void launch_embedding(const Lookup& q, hipStream_t s);
size_t embedding_grad_scratch(int64_t n, int64_t cols);
void launch_embedding_grad(const Lookup& q, char* scratch, hipStream_t s);

struct Dropout {
    int64_t rows, cols;
    Matrix x, residual, y;  // residual.at may be NULL; it has y's type
    uint32_t threshold;     // of a 16-bit number that is kept
    uint64_t seed, offset;
    const uint64_t* more;   // added to the offset; may be NULL
};
void launch_dropout(const Dropout& q, hipStream_t s);

}  // namespace sidco
#endif
