// Host-only paths of a language model's operators - sizes, plans and argument checks that return before any HIP call - in a
// build whose host code is instrumented with -fsanitize=address,undefined.  No GPU is needed.  What the operators use of the
// library's other sources is stood in for.
#include <cmath>
#include <cstdint>
#include <cstdio>

#include "sidco.h"
#include "sidco_internal.h"

namespace sidco {
StreamScratch::StreamScratch(void*, size_t) : rc(SIDCO_ERR_WORKSPACE), data(nullptr) {}
StreamScratch::~StreamScratch() {}
size_t workspace_with_scratch(size_t bytes) { return 4096 + bytes; }
int launched() { return SIDCO_ERR_HIP; }
}  // namespace sidco

static int failures = 0;
#define EXPECT(cond)                                      \
    do {                                                  \
        if (!(cond)) {                                    \
            ++failures;                                   \
            std::printf("line %d: %s\n", __LINE__, #cond); \
        }                                                 \
    } while (0)

int main()
{
    alignas(16) static float x[64], y[64], z[64];
    alignas(16) static int64_t words[8];
    const int64_t most = INT32_MAX, big = (int64_t)1 << 31;

    EXPECT(sidco_embedding(nullptr, x, 0, most, most, most, words, 1, most, NAN, y, 0, most) == SIDCO_ERR_ARG);
    EXPECT(sidco_embedding(nullptr, x, 0, INT64_MAX, 4, 4, words, 1, 4, 1.0f, y, 0, 4) == SIDCO_ERR_SIZE);
    EXPECT(sidco_embedding(nullptr, x, 0, 4, 4, INT64_MIN, words, 1, 4, 1.0f, y, 0, 4) == SIDCO_ERR_SIZE);
    EXPECT(sidco_embedding_grad(nullptr, x, 0, most, most, most, words, 1, most, 1.0f, 0, y, 0, most) == SIDCO_ERR_SIZE);
    EXPECT(sidco_embedding_grad(nullptr, x, 0, most, 4, 4, words, 1, 4, 1.0f, 0, y, 0, 4) == SIDCO_ERR_SIZE);
    EXPECT(sidco_embedding_grad(nullptr, x, 0, (int64_t)1 << 27, 4, 4, words, 1, 4, 1.0f, 0, y, 0, 4) == SIDCO_ERR_WORKSPACE);
    EXPECT(sidco_embedding_grad(nullptr, x, 0, 9, most, most, words, 1, 4, 1.0f, 0, y, 0, most) == SIDCO_ERR_SIZE);
    EXPECT(sidco_embedding_grad(nullptr, x, 0, 4, 4, 4, words, 1, 4, 1.0f, 0, x, 0, 4) == SIDCO_ERR_ARG);
    EXPECT(sidco_workspace_bytes_embedding_grad((int64_t)1 << 27, 512) > 0 && sidco_workspace_bytes_embedding_grad(8, most) > 0);
    EXPECT(sidco_workspace_bytes_embedding_grad(((int64_t)1 << 27) + 1, 1) == 0 && sidco_workspace_bytes_embedding_grad(most, most) == 0);
    EXPECT(sidco_workspace_bytes_embedding_grad(big, 1) == 0 && sidco_workspace_bytes_embedding_grad(1, INT64_MIN) == 0);

    EXPECT(sidco_dropout_blocks(most, most) == most * ((int64_t)1 << 28));
    EXPECT(sidco_dropout(nullptr, x, 0, 4, 4, 4, INFINITY, 0, 0, nullptr, nullptr, 0, y, 0, 4) == SIDCO_ERR_ARG);
    EXPECT(sidco_dropout(nullptr, x, 0, INT64_MAX, 4, 4, 0.5, 0, 0, nullptr, nullptr, 0, y, 0, 4) == SIDCO_ERR_SIZE);
    EXPECT(sidco_dropout(nullptr, x, 0, 4, 4, 4, 0.5, UINT64_MAX, UINT64_MAX, nullptr, z, 3, y, 0, 4) == SIDCO_ERR_SIZE);

    const int64_t rows = (int64_t)1 << 22, dim = (int64_t)1 << 21;
    for (int t = 0; t < 3; ++t) {
        for (int64_t n : {(int64_t)1, (int64_t)32, (int64_t)33, (int64_t)700, (int64_t)2049, (int64_t)8192, (int64_t)16385, rows})
            for (int64_t d : {(int64_t)1, (int64_t)64, (int64_t)1500, (int64_t)4096, dim})
                for (int64_t v : {(int64_t)1, (int64_t)300, (int64_t)10000, (int64_t)131072, (int64_t)4000000, most}) {
                    const bool fits = ((n + 63) / 64) * ((v + 63) / 64) <= most && ((v + 63) / 64) * ((d + 63) / 64) <= most;
                    EXPECT((sidco_workspace_bytes_cross_entropy(n, d, v, t) > 0) == fits);
                    EXPECT((sidco_workspace_bytes_cross_entropy_grad(n, d, v, t, t) > 0) == fits);
                    if (fits) EXPECT(sidco_workspace_bytes_cross_entropy_grad(n, d, v, t, 0) >= sidco_workspace_bytes_cross_entropy_grad(n, d, v, t, t));
                    const int want = fits ? SIDCO_ERR_WORKSPACE : SIDCO_ERR_SIZE;
                    EXPECT(sidco_cross_entropy(nullptr, x, y, t, n, d, v, d, d, words, 1, z, nullptr) == want);
                    EXPECT(sidco_cross_entropy_grad(nullptr, x, y, t, n, d, v, d, d, words, 1, z, nullptr, z + 16, d, z + 32, 0, d, 1) == want);
                    EXPECT(sidco_cross_entropy_grad(nullptr, x, y, t, n, d, v, d, d, words, 1, z, nullptr, z + 16, d, nullptr, 0, 0, 0) == want);
                    EXPECT(sidco_cross_entropy_grad(nullptr, x, y, t, n, d, v, d, d, words, 1, z, nullptr, nullptr, 0, z + 32, t, d, 0) == want);
                }
    }
    EXPECT(sidco_cross_entropy(nullptr, x, y, 0, INT64_MAX, 4, 4, 4, 4, words, 1, z, nullptr) == SIDCO_ERR_SIZE);
    EXPECT(sidco_cross_entropy(nullptr, x, y, 0, 4, INT64_MIN, 4, 4, 4, words, 1, z, nullptr) == SIDCO_ERR_SIZE);
    EXPECT(sidco_cross_entropy_grad(nullptr, x, y, 0, 4, 4, INT64_MAX, 4, 4, words, 1, z, nullptr, z + 16, 4, nullptr, 0, 0, 0) == SIDCO_ERR_SIZE);
    EXPECT(sidco_workspace_bytes_cross_entropy(INT64_MAX, INT64_MAX, INT64_MAX, 0) == 0);

    std::printf("%d failures\n", failures);
    return failures != 0;
}
