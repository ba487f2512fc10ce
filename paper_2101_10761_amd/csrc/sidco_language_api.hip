// C ABI of a language model's operators: argument checks and kernel sequencing.  Contracts are in include/sidco.h.
#include <math.h>

#include "sidco_language.h"

using namespace sidco;

namespace {

bool extent(int64_t n) { return n >= 1 && n <= INT32_MAX; }
bool element_type(int dtype) { return dtype == SIDCO_GRAD_F32 || dtype == SIDCO_GRAD_F16 || dtype == SIDCO_GRAD_BF16; }
int type_of(int dtype) { return dtype == SIDCO_GRAD_F16 ? kGradF16 : (dtype == SIDCO_GRAD_BF16 ? kGradBf16 : kGradF32); }
bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool flag(int f) { return f == 0 || f == 1; }

// Of a matrix of `cols` columns; rows are the caller's.
int check_matrix(const void* p, int dtype, int64_t cols, int64_t ld)
{
    if (!p) return SIDCO_ERR_NULL;
    if (!element_type(dtype)) return SIDCO_ERR_ARG;
    if (!extent(cols) || ld < cols || ld > INT32_MAX) return SIDCO_ERR_SIZE;
    return aligned(p, dtype == SIDCO_GRAD_F32 ? 4 : 2) ? SIDCO_OK : SIDCO_ERR_ALIGN;
}

int check_words(const void* words, int type, int64_t n, int64_t vocab)
{
    if (!words) return SIDCO_ERR_NULL;
    if (type != SIDCO_WORD_I32 && type != SIDCO_WORD_I64) return SIDCO_ERR_ARG;
    if (!extent(n) || !extent(vocab)) return SIDCO_ERR_SIZE;
    return aligned(words, type == SIDCO_WORD_I64 ? 8 : 4) ? SIDCO_OK : SIDCO_ERR_ALIGN;
}

Matrix matrix(const void* p, int dtype, int64_t ld) { return {(void*)p, type_of(dtype), ld}; }

bool entropy_sizes(int64_t n, int64_t dim, int64_t vocab)
{
    if (n < 1 || n > kEntropyMaxRows || dim < 1 || dim > kEntropyMaxDim || !extent(vocab)) return false;
    // a tile's number has 31 bits
    return ((n + 63) / 64) * ((vocab + 63) / 64) <= (int64_t)INT32_MAX && ((vocab + 63) / 64) * ((dim + 63) / 64) <= (int64_t)INT32_MAX;
}

int check_entropy(const void* x, const void* w, int dtype, int64_t n, int64_t dim, int64_t vocab, int64_t ldx, int64_t ldw, const void* words,
                  int word_type)
{
    if (int rc = check_words(words, word_type, n, vocab)) return rc;
    if (int rc = check_matrix(x, dtype, dim, ldx)) return rc;
    if (int rc = check_matrix(w, dtype, dim, ldw)) return rc;
    return entropy_sizes(n, dim, vocab) ? SIDCO_OK : SIDCO_ERR_SIZE;
}

// Of calls with these sizes: x and w as if they had to be laid out, their rows starting at whole 32-bit words or between them,
// which the rule for few rows tells apart.
Entropy any_entropy(int64_t n, int64_t dim, int64_t vocab, int dtype, bool between = true)
{
    Entropy q = {};
    q.words = {nullptr, true, n, vocab};
    q.dim = dim;
    q.x = q.w = {between ? (void*)2 : (void*)4, type_of(dtype), between ? dim : dim + dim % 2};
    return q;
}

}  // namespace

extern "C" {

int sidco_embedding(void* stream, const void* table, int table_dtype, int64_t vocab, int64_t dim, int64_t ldt, const void* words,
                    int word_type, int64_t n, float scale, void* out, int out_dtype, int64_t ldo)
{
    if (int rc = check_words(words, word_type, n, vocab)) return rc;
    if (int rc = check_matrix(table, table_dtype, dim, ldt)) return rc;
    if (int rc = check_matrix(out, out_dtype, dim, ldo)) return rc;
    if (!isfinite(scale) || table == out) return SIDCO_ERR_ARG;
    const Lookup q = {{words, word_type == SIDCO_WORD_I64, n, vocab}, matrix(table, table_dtype, ldt), matrix(out, out_dtype, ldo), dim, scale, false};
    launch_embedding(q, (hipStream_t)stream);
    return launched();
}

size_t sidco_workspace_bytes_embedding_grad(int64_t n, int64_t dim)
{
    return extent(n) && extent(dim) && embedding_grad_fits(n, dim) ? workspace_with_scratch(embedding_grad_scratch(n, dim)) : 0;
}

int sidco_embedding_grad(void* stream, const void* grad, int grad_dtype, int64_t n, int64_t dim, int64_t ldg, const void* words,
                         int word_type, int64_t vocab, float scale, int accumulate, void* table_grad, int table_dtype, int64_t ldt)
{
    if (int rc = check_words(words, word_type, n, vocab)) return rc;
    if (int rc = check_matrix(grad, grad_dtype, dim, ldg)) return rc;
    if (int rc = check_matrix(table_grad, table_dtype, dim, ldt)) return rc;
    if (!embedding_grad_fits(n, dim)) return SIDCO_ERR_SIZE;
    if (!isfinite(scale) || !flag(accumulate) || grad == table_grad) return SIDCO_ERR_ARG;
    const Lookup q = {{words, word_type == SIDCO_WORD_I64, n, vocab}, matrix(table_grad, table_dtype, ldt), matrix(grad, grad_dtype, ldg), dim,
                      scale, accumulate != 0};
    const size_t bytes = embedding_grad_scratch(n, dim);
    if (bytes == 0) {
        launch_embedding_grad(q, nullptr, (hipStream_t)stream);
        return launched();
    }
    StreamScratch ws(stream, bytes);
    if (ws.rc != SIDCO_OK) return ws.rc;
    launch_embedding_grad(q, ws.data, (hipStream_t)stream);
    return launched();
}

int64_t sidco_dropout_blocks(int64_t rows, int64_t cols)
{
    return extent(rows) && extent(cols) ? rows * ((cols + 7) / 8) : SIDCO_ERR_SIZE;
}

int sidco_dropout(void* stream, const void* x, int x_dtype, int64_t rows, int64_t cols, int64_t ldx, double p, uint64_t seed,
                  uint64_t offset, const uint64_t* device_offset, const void* residual, int64_t ldr, void* y, int y_dtype, int64_t ldy)
{
    if (!extent(rows)) return SIDCO_ERR_SIZE;
    if (int rc = check_matrix(x, x_dtype, cols, ldx)) return rc;
    if (int rc = check_matrix(y, y_dtype, cols, ldy)) return rc;
    if (residual)
        if (int rc = check_matrix(residual, y_dtype, cols, ldr)) return rc;
    if (!aligned(device_offset, 8)) return SIDCO_ERR_ALIGN;
    if (!(p >= 0.0 && p <= 1.0)) return SIDCO_ERR_ARG;
    if (x == y && rows > 1 && (x_dtype != y_dtype || ldx != ldy)) return SIDCO_ERR_ARG;
    if (x == y && x_dtype != y_dtype) return SIDCO_ERR_ARG;
    if (residual && residual == y && rows > 1 && ldr != ldy) return SIDCO_ERR_ARG;
    const Dropout q = {rows, cols, matrix(x, x_dtype, ldx), matrix(residual, y_dtype, ldr), matrix(y, y_dtype, ldy),
                       (uint32_t)floor(65536.0 * p + 0.5), seed, offset, device_offset};
    launch_dropout(q, (hipStream_t)stream);
    return launched();
}

size_t sidco_workspace_bytes_cross_entropy(int64_t n, int64_t dim, int64_t vocab, int dtype)
{
    if (!entropy_sizes(n, dim, vocab) || !element_type(dtype)) return 0;
    const size_t most = entropy_scratch(any_entropy(n, dim, vocab, dtype)), other = entropy_scratch(any_entropy(n, dim, vocab, dtype, false));
    return workspace_with_scratch(other > most ? other : most);
}

int sidco_cross_entropy(void* stream, const void* x, const void* w, int dtype, int64_t n, int64_t dim, int64_t vocab, int64_t ldx, int64_t ldw,
                        const void* targets, int word_type, float* loss, float* lse)
{
    if (!loss && !lse) return SIDCO_ERR_NULL;
    if (int rc = check_entropy(x, w, dtype, n, dim, vocab, ldx, ldw, targets, word_type)) return rc;
    if (!aligned(loss, 4) || !aligned(lse, 4)) return SIDCO_ERR_ALIGN;
    if (loss == lse) return SIDCO_ERR_ARG;
    Entropy q = {};
    q.words = {targets, word_type == SIDCO_WORD_I64, n, vocab};
    q.dim = dim;
    q.x = matrix(x, dtype, ldx);
    q.w = matrix(w, dtype, ldw);
    q.loss = loss;
    q.lse = lse;
    StreamScratch ws(stream, entropy_scratch(q));
    if (ws.rc != SIDCO_OK) return ws.rc;
    launch_entropy(q, ws.data, (hipStream_t)stream);
    return launched();
}

size_t sidco_workspace_bytes_cross_entropy_grad(int64_t n, int64_t dim, int64_t vocab, int dtype, int w_grad_dtype)
{
    if (!entropy_sizes(n, dim, vocab) || !element_type(dtype) || (w_grad_dtype != dtype && w_grad_dtype != SIDCO_GRAD_F32)) return 0;
    size_t most = 0;
    for (int which = 1; which <= 3; ++which) {  // a call for one gradient alone takes larger pieces
        Entropy q = any_entropy(n, dim, vocab, dtype);
        if (which & 1) q.x_grad = q.x;
        if (which & 2) q.w_grad = {(void*)1, type_of(w_grad_dtype), dim};
        const size_t bytes = entropy_grad_scratch(q);
        most = bytes > most ? bytes : most;
    }
    return workspace_with_scratch(most);
}

int sidco_cross_entropy_grad(void* stream, const void* x, const void* w, int dtype, int64_t n, int64_t dim, int64_t vocab, int64_t ldx,
                             int64_t ldw, const void* targets, int word_type, const float* lse, const float* loss_grad, void* x_grad,
                             int64_t ldgx, void* w_grad, int w_grad_dtype, int64_t ldgw, int accumulate)
{
    return sidco_cross_entropy_grad_of_loss(stream, x, w, dtype, n, dim, vocab, ldx, ldw, targets, word_type, nullptr, lse, loss_grad, x_grad, ldgx,
                                            w_grad, w_grad_dtype, ldgw, accumulate);
}

int sidco_cross_entropy_grad_of_loss(void* stream, const void* x, const void* w, int dtype, int64_t n, int64_t dim, int64_t vocab, int64_t ldx,
                                     int64_t ldw, const void* targets, int word_type, const float* loss, const float* lse,
                                     const float* loss_grad, void* x_grad, int64_t ldgx, void* w_grad, int w_grad_dtype, int64_t ldgw,
                                     int accumulate)
{
    if (!lse || (!x_grad && !w_grad)) return SIDCO_ERR_NULL;
    if (int rc = check_entropy(x, w, dtype, n, dim, vocab, ldx, ldw, targets, word_type)) return rc;
    if (!aligned(loss, 4) || !aligned(lse, 4) || !aligned(loss_grad, 4)) return SIDCO_ERR_ALIGN;
    if (x_grad)
        if (int rc = check_matrix(x_grad, dtype, dim, ldgx)) return rc;
    if (w_grad) {
        if (int rc = check_matrix(w_grad, w_grad_dtype, dim, ldgw)) return rc;
        if (w_grad_dtype != dtype && w_grad_dtype != SIDCO_GRAD_F32) return SIDCO_ERR_ARG;
    }
    if (!flag(accumulate) || (x_grad && (x_grad == x || x_grad == w || x_grad == w_grad)) || (w_grad && (w_grad == x || w_grad == w)))
        return SIDCO_ERR_ARG;
    Entropy q = {};
    q.words = {targets, word_type == SIDCO_WORD_I64, n, vocab};
    q.dim = dim;
    q.x = matrix(x, dtype, ldx);
    q.w = matrix(w, dtype, ldw);
    q.loss = (float*)loss;
    q.lse = (float*)lse;
    q.loss_grad = loss_grad;
    if (x_grad) q.x_grad = matrix(x_grad, dtype, ldgx);
    if (w_grad) q.w_grad = matrix(w_grad, w_grad_dtype, ldgw);
    q.accumulate = accumulate != 0;
    StreamScratch ws(stream, entropy_grad_scratch(q));
    if (ws.rc != SIDCO_OK) return ws.rc;
    launch_entropy_grad(q, ws.data, (hipStream_t)stream);
    return launched();
}

}  // extern "C"
