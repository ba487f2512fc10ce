// What calls of a language model's operators ask the workspace for, against what the library says that they need at most.  Every
// call ends at its request: no GPU is needed.
#include <cstdint>
#include <cstdio>

#include "sidco.h"
#include "sidco_internal.h"

static size_t asked = 0;
constexpr size_t kHead = 4096;

namespace sidco {
StreamScratch::StreamScratch(void*, size_t bytes) : rc(SIDCO_ERR_WORKSPACE), data(nullptr) { asked = bytes; }
StreamScratch::~StreamScratch() {}
size_t workspace_with_scratch(size_t bytes) { return kHead + bytes; }
int launched() { return SIDCO_ERR_HIP; }
}  // namespace sidco

static int calls = 0, failures = 0;

static void check(int rc, size_t most, const char* what, int t, int64_t n, int64_t d, int64_t v, int64_t ldx, int64_t ldw, uintptr_t off)
{
    ++calls;
    if (rc == SIDCO_ERR_WORKSPACE && asked + kHead <= most) return;
    if (++failures <= 20)
        std::printf("%s: type %d, %lld x %lld x %lld, strides %lld and %lld, %llu bytes off: error %d, asks for %zu of %zu\n", what, t, (long long)n,
                    (long long)d, (long long)v, (long long)ldx, (long long)ldw, (unsigned long long)off, rc, asked + kHead, most);
}

int main()
{
    const int64_t rows[] = {1, 2, 15, 16, 17, 31, 32, 33, 40, 48, 63, 64, 65, 66, 80, 95, 96, 97, 100, 127, 128, 129, 200, 256, 257, 700, 2049, 8192, 16384,
                            16385, 20000, 40000};
    const int64_t dims[] = {1, 7, 8, 9, 10, 31, 64, 66, 72, 100, 128, 500, 512, 700, 1024, 1500, 1501, 2048, 2050, 4096, 4097, 8192};
    const int64_t vocabs[] = {1, 5, 10, 50, 100, 300, 700, 1000, 3000, 10000, 50257, 131072, 1000003};
    const uintptr_t x = 1 << 20, w = 1 << 21, words = 1 << 22, loss = 1 << 23, lse = 1 << 24, dx = 1 << 25, dw = 1 << 26;  // never dereferenced
    for (int t = 0; t < 3; ++t)
        for (int64_t n : rows)
            for (int64_t d : dims)
                for (int64_t v : vocabs) {
                    const size_t most = sidco_workspace_bytes_cross_entropy(n, d, v, t);
                    const size_t same = sidco_workspace_bytes_cross_entropy_grad(n, d, v, t, t);
                    const size_t full = sidco_workspace_bytes_cross_entropy_grad(n, d, v, t, 0);
                    for (int64_t gap : {0, 1, 2, 64 - (int)(d % 64)})
                        for (uintptr_t off : {0, 2, 4, 16}) {
                            if (t == 0 && off == 2) continue;
                            const int64_t ldx = d + gap, ldw = d + gap;
                            void *px = (void*)(x + off), *pw = (void*)(w + off);
                            check(sidco_cross_entropy(nullptr, px, pw, t, n, d, v, ldx, ldw, (void*)words, 1, (float*)loss, (float*)lse), most, "losses", t, n,
                                  d, v, ldx, ldw, off);
                            for (int which = 1; which <= 3; ++which)
                                for (int o : {t, 0}) {
                                    check(sidco_cross_entropy_grad(nullptr, px, pw, t, n, d, v, ldx, ldw, (void*)words, 1, (float*)lse, nullptr,
                                                                   which & 1 ? (void*)dx : nullptr, d, which & 2 ? (void*)dw : nullptr, o, d, 0),
                                          o == t ? same : full, "gradients", t, n, d, v, ldx, ldw, off);
                                }
                        }
                }
    std::printf("%d calls, %d failures\n", calls, failures);
    return failures != 0;
}
