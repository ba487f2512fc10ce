// The dense operators' host-only paths - sizes, defaults and argument checks that return before any HIP call - in a build
// whose host code is instrumented with -fsanitize=address,undefined.  No GPU is needed.
#include <cmath>
#include <cstdint>
#include <cstdio>

#include "sidco.h"

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
    alignas(16) static uint8_t c[256], s[16];
    const int64_t big = (int64_t)1 << 31, most = INT32_MAX;

    EXPECT(sidco_mx4_code_bytes(most, most) == most * ((most + 255) / 256) * 128);
    EXPECT(sidco_mx4_scale_bytes(most, most) == most * ((most + 255) / 256) * 8);
    EXPECT(sidco_mx4_code_bytes(0, 1) == SIDCO_ERR_SIZE && sidco_mx4_scale_bytes(1, big) == SIDCO_ERR_SIZE);
    EXPECT(sidco_workspace_bytes_mx4_linear(most, (int64_t)1 << 24) > 0 && sidco_workspace_bytes_mx4_linear(1, INT64_MAX) == 0);

    EXPECT(sidco_mx4_compress(nullptr, nullptr, 0, y, 8, c, s) == SIDCO_ERR_NULL);
    EXPECT(sidco_mx4_compress(nullptr, x, 0, y, INT64_MAX, c, s) == SIDCO_ERR_SIZE);
    EXPECT(sidco_mx4_compress(nullptr, x, 0, y, INT64_MIN, c, s) == SIDCO_ERR_SIZE);
    EXPECT(sidco_mx4_compress(nullptr, x, 0, x, 8, c, s) == SIDCO_ERR_ARG);
    EXPECT(sidco_mx4_aggregate(nullptr, c, 128, s, 8, 0, 8, 1.0f, 0, x) == SIDCO_ERR_SIZE);
    EXPECT(sidco_mx4_aggregate(nullptr, c, INT64_MIN, s, 8, 2, 8, 1.0f, 0, x) == SIDCO_ERR_SIZE);
    EXPECT(sidco_mx4_aggregate(nullptr, c, 128, s, 8, 2, 8, NAN, 0, x) == SIDCO_ERR_ARG);
    EXPECT(sidco_mx4_quantize(nullptr, x, 0, most, most, most, c, s, c, s) == SIDCO_ERR_SIZE);
    EXPECT(sidco_mx4_quantize(nullptr, x, 0, 1, 1, INT64_MAX, c, s, c, s) == SIDCO_ERR_SIZE);
    EXPECT(sidco_mx4_quantize(nullptr, x, 9, 1, 1, 1, c, s, c, s) == SIDCO_ERR_ARG);
    EXPECT(sidco_mx4_dequantize(nullptr, c, s, 1, big, x, 0, big) == SIDCO_ERR_SIZE);
    EXPECT(sidco_mx4_matmul(nullptr, c, s, c, s, most, most, 1, 1.0f, 0, x, 0, most) == SIDCO_ERR_SIZE);
    EXPECT(sidco_mx4_matmul(nullptr, c, s, c, s, 1, 1, INT64_MAX, 1.0f, 0, x, 0, 1) == SIDCO_ERR_SIZE);
    EXPECT(sidco_mx4_linear(nullptr, x, 0, most, (int64_t)1 << 24, most, c, s, most, 1.0f, 0, y, 0, most) == SIDCO_ERR_SIZE);

    sidco_newton_schulz o;
    sidco_newton_schulz_default(nullptr);
    sidco_newton_schulz_default(&o);
    EXPECT(o.steps == 5);
    EXPECT(sidco_workspace_bytes_orthogonalize(1, (int64_t)1 << 21, (int64_t)1 << 21, SIDCO_GRAD_F32, &o) > 0);
    EXPECT(sidco_workspace_bytes_orthogonalize(65535, (int64_t)1 << 21, (int64_t)1 << 21, SIDCO_GRAD_F32, &o) == 0);
    EXPECT(sidco_workspace_bytes_orthogonalize(1, INT64_MAX, 1, SIDCO_GRAD_F32, nullptr) == 0);
    EXPECT(sidco_orthogonalize(nullptr, x, 0, INT64_MAX, 0, 1, 2, 2, nullptr, y, 0, 2, 0) == SIDCO_ERR_SIZE);
    EXPECT(sidco_orthogonalize(nullptr, x, 0, 2, INT64_MIN, 2, 2, 2, nullptr, y, 0, 2, 4) == SIDCO_ERR_SIZE);
    o.steps = 0;
    EXPECT(sidco_orthogonalize(nullptr, x, 0, 2, 4, 1, 2, 2, &o, y, 0, 2, 4) == SIDCO_ERR_STAGES);
    EXPECT(sidco_muon_step(nullptr, x, 0, y, z, 0, 1, 2, 2, NAN, 0.9f, 1, 0.0f, 1.0f, nullptr) == SIDCO_ERR_ARG);
    EXPECT(sidco_muon_step(nullptr, x, 0, y, y, 0, 1, 2, 2, 0.1f, 0.9f, 1, 0.0f, 1.0f, nullptr) == SIDCO_ERR_ARG);

    std::printf("%d failures\n", failures);
    return failures != 0;
}
