// Dropout from a counter-based generator: the mask is a function of seed and place and is formed wherever it is needed, in
// the forward and again in the backward pass.
//
// Block b of a seed's sequence is Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// 2011) of the counter (b mod 2^32, b / 2^32, 0, 0) with the seed as its key: four words, read as eight 16-bit numbers, low
// halves first.  Sixteen bits an element: the generator's two multiplications a round are what could take longer than
// memory, and a probability that is off by at most 2^-17, with a scale that belongs to the probability used, biases nothing.
#include "sidco_elements.h"

namespace sidco {
namespace {

struct Words4 {
    uint32_t w[4];
};

__device__ __forceinline__ Words4 philox(uint64_t block, uint64_t seed)
{
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = 0, c3 = 0;
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

template <class X, class Y>
struct Drop {
    const X* x;
    const Y* residual;
    Y* y;
    int64_t ldx, ldr, ldy, rows, cols, per_row;  // per_row: blocks of the sequence
    uint32_t threshold;
    float scale;
    uint64_t seed, offset;
    const uint64_t* more;
    int lanes;
};

// Bound by memory: 65536 x 4096 in bf16 with a residual, 1.61 GB, 274 us, 5.9 TB/s; 700 x 1500 in fp32 4.4 us, a launch and one trip
// to memory.
template <class X, class Y>
__global__ __launch_bounds__(kRowBlock) void k_dropout(Drop<X, Y> p)
{
    const uint64_t first = p.offset + (p.more ? *p.more : 0);
    const int lane = threadIdx.x & (p.lanes - 1);
    const int64_t per = kRowBlock / p.lanes, row0 = threadIdx.x / p.lanes;
    for (int64_t r = (int64_t)blockIdx.x * per + row0; r < p.rows; r += (int64_t)gridDim.x * per)
        for (int64_t u = (int64_t)blockIdx.y * p.lanes + lane; u < p.per_row; u += (int64_t)gridDim.y * p.lanes) {
            const int64_t c = u * 8, left = p.cols - c;
            Eight<X> x;
            Eight<Y> y;
            x.load(p.x + r * p.ldx + c, left);
            if (p.residual) y.load(p.residual + r * p.ldr + c, left);
            const Words4 w = philox(first + (uint64_t)(r * p.per_row + u), p.seed);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t number = i % 2 ? w.w[i / 2] >> 16 : w.w[i / 2] & 0xffff;
                const float kept = number >= p.threshold ? x.get(i) * p.scale : 0.0f;
                y.set(i, p.residual ? kept + y.get(i) : kept);
            }
            y.store(p.y + r * p.ldy + c, left);
        }
}

}  // namespace

void launch_dropout(const Dropout& q, hipStream_t s)
{
    const RowGrid g(q.cols);
    const int64_t per_row = (q.cols + 7) / 8, blocks = (q.rows + g.per - 1) / g.per, across = (per_row + g.lanes - 1) / g.lanes;
    const dim3 grid((uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20), (uint32_t)(across < 65535 ? across : 65535));
    by_element(q.x.type, [&](auto x) {
        by_element(q.y.type, [&](auto y) {
            typedef typename decltype(x)::T X;
            typedef typename decltype(y)::T Y;
            const float scale = q.threshold < 65536 ? (float)(65536.0 / (65536 - q.threshold)) : 0.0f;
            const Drop<X, Y> p = {(const X*)q.x.at, (const Y*)q.residual.at, (Y*)q.y.at, q.x.ld, q.residual.ld, q.y.ld, q.rows, q.cols,
                                  per_row, q.threshold, scale, q.seed, q.offset, q.more, g.lanes};
            k_dropout<X, Y><<<grid, kRowBlock, 0, s>>>(p);
        });
    });
}

}  // namespace sidco
