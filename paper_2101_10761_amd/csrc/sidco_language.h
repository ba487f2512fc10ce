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
bool embedding_grad_fits(int64_t n, int64_t cols);  // one launch's blocks
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

// Logits are x w^T: words.n rows of x, words.vocab rows of w, both of one type and of `dim` columns.
struct Entropy {
    Words words;
    int64_t dim;
    Matrix x, w;
    float *loss, *lse;         // written by the forward pass, either may be NULL; read by the gradient, loss may be NULL
    const float* loss_grad;    // NULL: ones
    Matrix x_grad, w_grad;     // one of the two may be NULL
    bool accumulate;           // onto w_grad
};
constexpr int64_t kEntropyMaxRows = 1 << 22, kEntropyMaxDim = 1 << 21;
size_t entropy_scratch(const Entropy& q);       // of x, w only how their rows lie
size_t entropy_grad_scratch(const Entropy& q);  // and of the gradients which there are and w_grad's type
void launch_entropy(const Entropy& q, char* scratch, hipStream_t s);
void launch_entropy_grad(const Entropy& q, char* scratch, hipStream_t s);

}  // namespace sidco
#endif
