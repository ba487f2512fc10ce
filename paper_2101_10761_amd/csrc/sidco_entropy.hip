// Softmax cross entropy of rows x against a vocabulary's weight w, in pieces, without keeping the logits.
//
//   l = x w^T,  lse_i = log sum_v exp l_iv,  loss_i = lse_i - l_i,t,
//   P_iv = g_i (exp(l_iv - lse_i) - [v = t_i]),  dx = P w,  dw = P^T x.
//
// The forward pass is one product whose tiles go out as the largest logit of each row and the sum of exponentials below it, in
// powers of two and without the row's word, whose logit goes out by itself; a second kernel joins the tiles' pairs to z = sum over
// v != t of exp(l_v - l_t), loss = log(1 + z), lse = l_t + loss: a small loss is not the difference of two large numbers.  The
// gradient forms the logits again, a piece of the vocabulary at a
// time, and P leaves the product's registers both by rows of x and by words, for the two products that contract over words
// and over rows: four products for the three that an arithmetic minimum takes, and no N x V array.
//
// Products are those of sidco_product.h and want both operands by rows along the contraction, in whole lines of 128 bytes.
// 16-bit operands that lie like that are read where they are; others, and the transposes that the gradient needs, are laid out
// in the workspace first.  fp32 operands become pairs of halves, 22 bits, under a power of two for each matrix, and a product is
// three: low high + high low + high high.
//
// P is in halves, times a power of two, for its smallest elements would reach theirs: 11 bits, or as a pair 22.  Its rounding adds
// up like a rounding of the gradient itself, so that it takes more bits than the gradient has: one half for bf16 gradients (an
// error of 1.7e-3 in the 2-norm, the gradient's own rounding; with P in bf16 it was up to 2.4e-3), a pair for those of halves and
// of fp32 (2.1e-4 for halves; with one half up to 3.1e-4).  bf16 operands of the products with P are halves too, exactly but for
// those under 2^-24 of the largest, under a power of two as for fp32; they multiply at nearly the rate of bf16 (a training pass
// of 8192 x 4096 x 131072 takes 3 % longer).  A row whose gradient is far below the largest has a power of two of its own in P by
// rows, and leaves it in P by words.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "sidco_elements.h"
#include "sidco_product.h"

namespace sidco {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr double kLn2 = 0.69314718055994530942;
constexpr float kFar = 3.0e38f;  // stands for an infinite largest logit

// How element types are multiplied: what the operands of the logits are held in, whether operands are pairs, whether those of the
// gradient's products, always halves, are scaled, and whether P is a pair in all of them.
struct ModeF32 {
    typedef float T;
    typedef _Float16 H;
    typedef HalfCore Core;
    static constexpr bool kPairs = true, kScaled = true, kPairP = true;
};
struct ModeF16 {
    typedef _Float16 T, H;
    typedef HalfCore Core;
    static constexpr bool kPairs = false, kScaled = false, kPairP = true;
};
struct ModeBf16 {
    typedef __bf16 T, H;
    typedef Bf16Core Core;
    static constexpr bool kPairs = false, kScaled = true, kPairP = false;
};
typedef _Float16 G;  // of the gradient's products

template <class F>
void by_mode(int type, const F& f)
{
    if (type == kGradF32)
        f(ModeF32());
    else if (type == kGradF16)
        f(ModeF16());
    else
        f(ModeBf16());
}

// ---- scales ----

// Powers of two: of x and w as the gradient's products (fp32: all) take them, and of P; and whether rows have others besides.
struct Scales {
    float x, w, p;
    int by_row;
};
constexpr int kParts = 2048;             // blocks of k_layout, and partial results of each kind
enum { kTopX, kTopW, kTopG, kLeastG, kPartKinds };  // largest magnitudes, and how far below 2^128 the least of the rows' gradients is

// What x and w are laid out with at first.  Weights whose largest magnitude is 2^-7 to 2^1.5 and rows of 2^-3 to 2^5.5 stay so; k_settle
// lays out others once more.
constexpr float kGuessX = 1024.0f, kGuessW = 16384.0f;

// What brings a largest magnitude to 2^14 to 2^15; 1 for zeros.
__device__ __forceinline__ float scale_of(float top)
{
    if (!(top > 0.0f)) return 1.0f;
    int e = 0;
    (void)frexpf(top, &e);
    e = 15 - e;
    return ldexpf(1.0f, e > 120 ? 120 : e);
}

// Of a power of two.  Two of them may have a product that no float holds.
__device__ __forceinline__ int exponent_of(float scale) { return (int)(__builtin_bit_cast(uint32_t, scale) >> 23) - 127; }

// P's power of two is that of the largest gradient of a row.  Rows far below it, whose P would end in it, have a power of two of
// their own besides in the product for x's gradient, where each row is a sum for itself: what brings `gain`, the row's gradient under
// the common one, to 2^14 to 2^15.  From 2^8 on: so close P has all its bits down to 2^-21 of the row's own gradient, and no tile
// of a batch with gradients like each other takes the way there and back.
constexpr int kRowPower = 8;
__device__ __forceinline__ int row_power(float gain)
{
    const float m = fabsf(gain);
    const int e = m > 0.0f && m < INFINITY ? 14 - exponent_of(m) : 0;
    return e < kRowPower ? 0 : (e < 120 ? e : 120);
}

// What scale_of says, or the guess where it does: the largest is a half with room for rounding, and what halves cannot tell from zero is 2^-32 of it.
__device__ __forceinline__ float settled(float top, float guess)
{
    const float t = top * guess;
    return top == 0.0f || (t >= 128.0f && t < 46340.0f) ? guess : scale_of(top);
}

template <class T>
struct Source {
    const T* at;
    int64_t ld, rows, cols;
    WordList words;  // rows of padding are left out; without an address none is
};

__device__ __forceinline__ float more(float top, float v)
{
    const float m = fabsf(v);
    return m < INFINITY && m > top ? m : top;
}

// The largest of the block's 256 threads, of each kind, in all of them.
template <int Kinds>
__device__ __forceinline__ void block_tops(float (&top)[Kinds], float (*lds)[4])
{
#pragma unroll
    for (int k = 0; k < Kinds; ++k) {
#pragma unroll
        for (int s = 32; s > 0; s >>= 1) top[k] = fmaxf(top[k], __shfl_xor(top[k], s));
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < Kinds; ++k)
        if ((threadIdx.x & 63) == 0) lds[k][threadIdx.x >> 6] = top[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < Kinds; ++k) top[k] = fmaxf(fmaxf(lds[k][0], lds[k][1]), fmaxf(lds[k][2], lds[k][3]));
}

// The largest of two kinds that lie one behind the other, over the blocks of k_layout, for the whole block of 256.  Without branches
// all loads are under way at once: k_settle takes 4.8 us, and 8.4 with them.
__device__ __forceinline__ void joined_tops(const float* part, uint32_t blocks, float (*lds)[4], float (&top)[2])
{
    float v[2][kParts / 256];
#pragma unroll
    for (int kind = 0; kind < 2; ++kind)
#pragma unroll
        for (uint32_t k = 0; k < kParts / 256; ++k) v[kind][k] = part[kind * kParts + min(k * 256 + threadIdx.x, blocks - 1)];
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        top[kind] = 0.0f;
#pragma unroll
        for (int k = 0; k < kParts / 256; ++k) top[kind] = fmaxf(top[kind], v[kind][k]);
    }
    block_tops(top, lds);
}

// ---- operands ----

// Rows of `pitch` elements; what a pair's second numbers are kept in is `low` elements on, 0: there is none.
template <class H>
struct Plane {
    H* at;
    int64_t pitch, low;
};

template <class H>
__device__ __forceinline__ Rows rows_of(const Plane<H>& p, int64_t row, int64_t rows, int64_t col, bool low)
{
    return {p.at + (low ? p.low : 0) + row * p.pitch + col, nullptr, (uint32_t)rows, (uint32_t)(p.pitch * sizeof(H))};
}

// A matrix to be laid out: by its rows, and transposed.  Either plane may have no address.
template <class T, class H>
struct Layout {
    Source<T> from;
    Plane<H> rows;
    Plane<G> turned;
    uint32_t tiles_r, tiles_c;  // of 64 x 64, padding included
};

template <class H, bool Pairs>
__device__ __forceinline__ void put8(const Plane<H>& o, int64_t r, int64_t c, const float (&v)[8])
{
    typedef H h8 __attribute__((ext_vector_type(8)));
    h8 h, l;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        h[i] = (H)v[i];
        l[i] = (H)(v[i] - (float)h[i]);
    }
    H* p = o.at + r * o.pitch + c;
    *(h8*)p = h;
    if (Pairs) *(h8*)(p + o.low) = l;
}

// 64 x 64 elements.  Transposed, rows of padding are zeros whatever they hold: they are multiplied with the zeros that P has for them.
// Returns the largest finite magnitude, or top if that is larger.
template <class M>
__device__ __forceinline__ float lay(const Layout<typename M::T, typename M::H>& p, uint32_t t, float scale, float (*tile)[65], float top)
{
    typedef typename M::H H;
    const int64_t r0 = (int64_t)(t / p.tiles_c) * 64, c0 = (int64_t)(t % p.tiles_c) * 64;
    const int row = threadIdx.x >> 3, col = (threadIdx.x & 7) * 8;
    Eight<typename M::T> e[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int64_t r = r0 + k * 32 + row, c = c0 + col;
        if (r < p.from.rows && c < p.from.cols) {
            e[k].load(p.from.at + r * p.from.ld + c, p.from.cols - c);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) e[k].set(i, 0.0f);
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int64_t r = r0 + k * 32 + row, c = c0 + col;
        const bool none = p.from.words.at && r < p.from.rows && p.from.words.none(r);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = e[k].get(i);
            if (M::kScaled && !none) top = more(top, v[i]);
            if (M::kPairs) v[i] *= scale;
        }
        if (p.rows.at && r < p.from.rows && c < p.rows.pitch) put8<H, M::kPairs>(p.rows, r, c, v);
        if (p.turned.at) {
#pragma unroll
            for (int i = 0; i < 8; ++i) tile[k * 32 + row][col + i] = none ? 0.0f : (M::kPairs ? v[i] : v[i] * scale);
        }
    }
    if (!p.turned.at) return top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = k * 32 + row;
        if (c0 + c >= p.from.cols || r0 + col >= p.turned.pitch) continue;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = tile[col + i][c];
        put8<G, M::kPairs>(p.turned, c0 + c, r0 + col, v);
    }
    __syncthreads();
    return top;
}

// x and w laid out with the guessed scales, and the largest finite magnitudes of x, w and the rows' gradient, and that one's least, a partial
// result from each block (not in the forward pass of 16-bit operands, which nothing is scaled in).  The magnitudes are only known behind a pass over
// everything: to find them first and lay out then is one read more.  Bound by memory: 700 and 10000 rows of 1500 fp32, 64 MB read and
// 128 MB written (two halves of each by rows and transposed), 28 to 34 us; with the pass before it the training step took 391, not 378.
template <class M, bool Scaled>
__global__ __launch_bounds__(256) void k_layout(Layout<typename M::T, typename M::H> x, Layout<typename M::T, typename M::H> w, Source<float> g, float* part)
{
    __shared__ float tile[64][65];
    __shared__ float lds[kPartKinds][4];
    const uint32_t first = x.tiles_r * x.tiles_c, all = first + w.tiles_r * w.tiles_c;
    float top[kPartKinds] = {0.0f, 0.0f, g.at ? 0.0f : 1.0f, 0.0f};  // a gradient without an address is ones
    for (uint32_t t = blockIdx.x; t < all; t += gridDim.x) {
        if (t < first)
            top[0] = lay<M>(x, t, M::kScaled ? kGuessX : 1.0f, tile, top[0]);
        else
            top[1] = lay<M>(w, t - first, M::kScaled ? kGuessW : 1.0f, tile, top[1]);
    }
    if (!Scaled) return;
    if (g.at) {
        for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < g.rows; r += (int64_t)gridDim.x * 256)
            if (!g.words.none(r)) {
                top[kTopG] = more(top[kTopG], g.at[r]);
                if (const float m = fabsf(g.at[r]); m > 0.0f && m < INFINITY) top[kLeastG] = fmaxf(top[kLeastG], (float)(128 - exponent_of(m)));
            }
    }
    block_tops(top, lds);
    if (threadIdx.x == 0) {
#pragma unroll
        for (int k = 0; k < kPartKinds; ++k) part[k * kParts + blockIdx.x] = top[k];
    }
}

// The scales that the largest magnitudes ask for, and what was laid out with another one once more.  A piece of w after the first
// leaves those of x and P as they are.  4.8 us where the guess does, two lists of 2048 partial results for each block and two more
// for the first; about 32 where all of that size is laid out again.
constexpr uint32_t kSettleBlocks = 512;
template <class M>
__global__ __launch_bounds__(256) void k_settle(Layout<typename M::T, typename M::H> x, Layout<typename M::T, typename M::H> w, uint32_t blocks, bool later,
                                                const float* part, Scales* scales)
{
    __shared__ float tile[64][65];
    __shared__ float lds[2][4];
    const uint32_t first = x.tiles_r * x.tiles_c, all = first + w.tiles_r * w.tiles_c;
    float sx = 1.0f, sw = 1.0f;
    if (M::kScaled) {
        float top[2];
        joined_tops(part + kTopX * kParts, blocks, lds, top);
        if (!later) sx = settled(top[0], kGuessX);
        sw = settled(top[1], kGuessW);
    }
    if (blockIdx.x == 0 && later && threadIdx.x == 0) scales->w = sw;
    if (blockIdx.x == 0 && !later) {
        float top[2];
        joined_tops(part + kTopG * kParts, blocks, lds, top);
        const float sp = scale_of(top[0]);
        // by_row as row_power has it of the least one
        if (threadIdx.x == 0) *scales = {sx, sw, sp, top[1] > 0.0f && 14 - (128 - (int)top[1] + exponent_of(sp)) >= kRowPower};
    }
    if (!M::kScaled) return;
    const uint32_t from = sx == kGuessX ? first : 0, to = sw == kGuessW ? first : all;
    for (uint32_t t = from + blockIdx.x; t < to; t += gridDim.x) {
        if (t < first)
            (void)lay<M>(x, t, sx, tile, 0.0f);
        else
            (void)lay<M>(w, t - first, sw, tile, 0.0f);
    }
}

// ---- the products ----

// The largest of three; a NaN among them is left out.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

// Terms of a product of pairs and single numbers, the small ones first.
template <int Terms, class Tl, class H>
__device__ __forceinline__ void take(Tl& t, int term, const Plane<H>& a, int64_t rows_a, const Plane<H>& b, int64_t rows_b, int64_t col, uint32_t m0,
                                     uint32_t n0)
{
    t.take(rows_of(a, 0, rows_a, col, Terms > 1 && term == 0), rows_of(b, 0, rows_b, col, Terms == 3 && term == 1), m0, n0);
}

template <class Tl, class H>
constexpr int lds_of()
{
    return Tl::kLds + Tl::kWaves * Tl::template out_bytes<H>();
}

struct Places {
    uint32_t tm, tn, total;  // total: of all splits
    __device__ __forceinline__ void at(uint32_t tile, uint32_t& i, uint32_t& j, uint32_t& split) const
    {
        const uint32_t w = xcd_run(tile, total);
        split = w / (tm * tn);
        tile_of(w - split * (tm * tn), tm, tn, i, j);
    }
};

// Logits of a tile as its rows' largest, in powers of two, and sums of 2^(logit - largest): pairs `width` a row, one for each
// wave's columns.  The logit of a row's word is written down by the wave that has it.  Bound by the matrix cores: 8192 x 4096 x 131072
// in bf16 5.9 to 6.1 ms, 1.45 to 1.49 PFLOP/s (a large library product reaches 1.52); 2049 x 1024 x 49999 in fp16 233 us, 0.9
// (1.30), with 16 lines to a tile and its end beside; 700 x 1500 x 10000 in pairs 67 us, 63 GFLOP, 0.94.
template <class H>
struct Forward {
    Plane<H> x, w;
    uint32_t n;      // rows; w has the vocabulary's
    WordList words;  // of these rows
    float2* part;
    uint32_t width;
    float* mine;
    const Scales* scales;
};

template <class M, class Tl>
__global__ __launch_bounds__(Tl::kThreads) void k_logits(Forward<typename M::H> p, Span span, Places places)
{
    __shared__ __align__(1024) char lds[Tl::kLds];
    Tl t;
    t.template run<M::kPairs ? 3 : 1, true>(
        places.total, span, lds,
        [&](uint32_t tile, int term) {
            uint32_t i, j, split;
            places.at(tile, i, j, split);
            take<M::kPairs ? 3 : 1>(t, term, p.x, p.n, p.w, p.words.vocab, 0, i * Tl::kM, j * Tl::kN);
        },
        [&](uint32_t tile) {
            uint32_t ti, tj, split;
            places.at(tile, ti, tj, split);
            const uint32_t m0 = ti * Tl::kM, n0 = tj * Tl::kN;
            const float k = M::kPairs ? kLog2e / (p.scales->x * p.scales->w) : kLog2e;
            const bool edge = n0 + Tl::kN > p.words.vocab;
            const uint32_t place = tj * (Tl::kN / (Tl::kNt * 16)) + t.wave % (Tl::kN / (Tl::kNt * 16));
            t.strips([&](int, uint32_t row, uint32_t col, v4f(&acc)[Tl::kNt]) {
                const uint32_t r = m0 + row, left = p.words.vocab - n0 - col;  // a word's columns, wrapped around if there are none
                const uint32_t here = (r < p.n ? p.words[r] : p.words.vocab) - n0 - col;
                if (edge) {
#pragma unroll
                    for (int j = 0; j < Tl::kNt; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[j][e] = (int)left > j * 16 + e ? acc[j][e] : -INFINITY;
                }
                // of 128 columns one lane has the row's word, or none
                if (here < Tl::kNt * 16 && here % 16 < 4 && here < left) {
                    float mine = 0.0f;
#pragma unroll
                    for (int j = 0; j < Tl::kNt; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool it = here == (uint32_t)(j * 16 + e);
                            mine = it ? acc[j][e] : mine;
                            acc[j][e] = it ? -INFINITY : acc[j][e];
                        }
                    p.mine[r] = mine * k;
                }
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < Tl::kNt; ++j) top = max3(max3(top, acc[j][0], acc[j][1]), acc[j][2], acc[j][3]);
                top *= k;  // k > 0
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                top = fminf(fmaxf(top, -kFar), kFar);
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < Tl::kNt; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(fmaf(acc[j][e], k, -top));
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
                if (t.lane < 16 && r < p.n) p.part[(int64_t)r * p.width + place] = make_float2(top, sum);
            });
        });
}

// ---- few rows ----
//
// Up to 32 rows read each word's weight once and do little with it: bound by memory.  Blocks of eight waves take 16 words after
// 16 words; the waves share the contraction, each keeps its part of x in registers, and the next words' loads go out as soon
// as the ones before are multiplied.  Operands are multiplied as they are, fp32 ones by fp32 instructions.  One row against 131072 x
// 4096 in bf16 169 to 171 us, 6.3 TB/s; 20 against 10000 x 1500 in fp32 20.5 us, 2.9 TB/s: 625 groups of words on 256 blocks, and the
// fp32 instructions of 32 rows, by their cycles 2.7 us a group and CU.
constexpr int kFewWaves = 8, kFewRows = 32;

template <class T>
struct FewCore;
template <>
struct FewCore<float> {
    typedef float piece __attribute__((ext_vector_type(4), aligned(4)));
    static constexpr int kStep = 16;  // elements of a step of a wave: four lanes' pieces
    static __device__ __forceinline__ v4f mul(const piece& a, const piece& b, v4f c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};
template <>
struct FewCore<_Float16> {
    typedef _Float16 piece __attribute__((ext_vector_type(8), aligned(2)));
    static constexpr int kStep = 32;
    static __device__ __forceinline__ v4f mul(const piece& a, const piece& b, const v4f& c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16((v8h)a, (v8h)b, c, 0, 0, 0);
    }
};
template <>
struct FewCore<__bf16> {
    typedef __bf16 piece __attribute__((ext_vector_type(8), aligned(2)));
    typedef __bf16 v8b __attribute__((ext_vector_type(8)));
    static constexpr int kStep = 32;
    static __device__ __forceinline__ v4f mul(const piece& a, const piece& b, const v4f& c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16((v8b)a, (v8b)b, c, 0, 0, 0);
    }
};

template <class T>
struct Few {
    const T *x, *w;
    int64_t ldx, ldw;
    uint32_t n, dim, groups;
    WordList words;
    float2* part;  // a pair for each row and block
    float* mine;
};

// Steps: of the contraction, 8 kStep elements each, as many as there are or one more; Tiles: of 16 rows.
template <class T, int Steps, int Tiles>
__global__ __launch_bounds__(64 * kFewWaves) void k_few(Few<T> p)
{
    typedef FewCore<T> Core;
    typedef typename Core::piece piece;
    constexpr uint32_t kPiece = Core::kStep / 4, kAll = kFewWaves * Core::kStep;
    __shared__ v4f sums[2][kFewWaves][Tiles][64];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const uint32_t at = wave * Core::kStep + q * kPiece;
    // A piece that would reach past the row's end is the row's last one instead, of which `keep` leaves what no other piece holds;
    // of one behind the end nothing.  Only the last two steps have such.  (A branch between them and whole steps would have the
    // compiler wait for all loads at each step.)
    const uint32_t last = p.dim - kPiece;
    v4i keep[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int skip = (int)((Steps - 2 + i) * kAll + at - last);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            if constexpr (sizeof(T) == 4)
                keep[i][d] = d >= skip ? -1 : 0;
            else
                keep[i][d] = (2 * d >= skip ? 0xffff : 0) | (2 * d + 1 >= skip ? (int)0xffff0000 : 0);
        }
    }
    auto load = [&](const T* row, int s) -> piece {
        const uint32_t k = s * kAll + at;
        return *(const piece*)(row + (s + 2 < Steps || k < last ? k : last));
    };
    auto kept = [&](const piece& v, int s) -> piece {
        return s + 2 < Steps ? v : __builtin_bit_cast(piece, __builtin_bit_cast(v4i, v) & keep[s + 2 - Steps]);
    };
    auto row_of = [&](uint32_t group) -> const T* {
        const uint32_t v = group * 16 + r;
        return p.w + (int64_t)(v < p.words.vocab ? v : p.words.vocab - 1) * p.ldw;
    };
    piece x[Tiles][Steps], w[Steps];
    const T* row = row_of(blockIdx.x);
#pragma unroll
    for (int s = 0; s < Steps; ++s) w[s] = load(row, s);
#pragma unroll
    for (int t = 0; t < Tiles; ++t) {
        const T* from = p.x + (int64_t)(t * 16 + r < p.n ? t * 16 + r : 0) * p.ldx;
#pragma unroll
        for (int s = 0; s < Steps; ++s) x[t][s] = kept(load(from, s), s);
    }
    const uint32_t mine = wave * 16 + r;  // the row whose sums this lane joins, if its wave is one of the first
    const uint32_t word = wave < Tiles && mine < p.n ? p.words[mine] : p.words.vocab;
    float top = -kFar, sum = 0.0f;
    uint32_t turn = 0;
    for (uint32_t group = blockIdx.x; group < p.groups; group += gridDim.x, turn ^= 1) {
        row = row_of(group + gridDim.x < p.groups ? group + gridDim.x : group);
        v4f acc[Tiles];
#pragma unroll
        for (int t = 0; t < Tiles; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < Steps; ++s) {
            const piece a = kept(w[s], s);
#pragma unroll
            for (int t = 0; t < Tiles; ++t) acc[t] = Core::mul(a, x[t][s], acc[t]);
            w[s] = load(row, s);  // where the operand was
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int t = 0; t < Tiles; ++t) sums[turn][wave][t][lane] = acc[t];
        __syncthreads();
        if (wave < Tiles) {
            v4f l = sums[turn][0][wave][lane];
#pragma unroll
            for (int k = 1; k < kFewWaves; ++k) l += sums[turn][k][wave][lane];
            l *= kLog2e;
            const uint32_t v = group * 16 + 4 * q;
            float most = top;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool it = word == v + e && word < p.words.vocab;
                if (it) p.mine[mine] = l[e];
                l[e] = v + e < p.words.vocab && !it ? l[e] : -INFINITY;
                most = fmaxf(most, l[e]);
            }
            most = fminf(most, kFar);
            sum *= __builtin_amdgcn_exp2f(top - most);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(l[e] - most);
            top = most;
        }
    }
    if (wave >= Tiles) return;
#pragma unroll
    for (int s = 16; s <= 32; s *= 2) {
        const float other = __shfl_xor(top, s), more = __shfl_xor(sum, s), next = fmaxf(top, other);
        sum = sum * __builtin_amdgcn_exp2f(top - next) + more * __builtin_amdgcn_exp2f(other - next);
        top = next;
    }
    if (q == 0 && mine < p.n) p.part[(int64_t)mine * gridDim.x + blockIdx.x] = make_float2(top, sum);
}

// A row's pairs joined by Lanes threads.  An infinite largest logit has made the sum infinite, a NaN among them a NaN.
template <int Lanes>
__global__ __launch_bounds__(256) void k_join_rows(const float2* part, uint32_t width, int64_t n, WordList words, const float* mine, float* loss,
                                                   float* lse)
{
    const int64_t r = (int64_t)blockIdx.x * (256 / Lanes) + threadIdx.x / Lanes;
    const uint32_t lane = threadIdx.x % Lanes;
    float top = -kFar, sum = 0.0f;
    if (r < n) {
#pragma unroll 4
        for (uint32_t i = lane; i < width; i += Lanes) {
            const float2 v = part[r * width + i];
            const float next = fmaxf(top, v.x);
            sum = sum * __builtin_amdgcn_exp2f(top - next) + v.y * __builtin_amdgcn_exp2f(v.x - next);
            top = next;
        }
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
        const float other = __shfl_xor(top, s), more = __shfl_xor(sum, s), next = fmaxf(top, other);
        sum = sum * __builtin_amdgcn_exp2f(top - next) + more * __builtin_amdgcn_exp2f(other - next);
        top = next;
    }
    if constexpr (Lanes == 256) {
        __shared__ float2 lds[4];
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = make_float2(top, sum);
        __syncthreads();
        top = -kFar, sum = 0.0f;
        for (int i = 0; i < 4; ++i) {
            const float2 v = lds[i];
            const float next = fmaxf(top, v.x);
            sum = sum * __builtin_amdgcn_exp2f(top - next) + v.y * __builtin_amdgcn_exp2f(v.x - next);
            top = next;
        }
    }
    if (lane == 0 && r < n) {
        const bool none = words.none(r);
        const double own = none ? -INFINITY : (double)mine[r], over = (double)top - own;
        double all, more;  // lse, and the loss
        if (over < 64.0) {
            more = log1p((double)sum * exp2(over));
            all = own * kLn2 + more;
            if (own == INFINITY) more = NAN;  // the difference of two infinities
        } else {  // or there is no word, or its logit is a NaN
            all = none || own == -INFINITY ? ((double)top + log2((double)sum)) * kLn2 : ((double)top + log2((double)sum + exp2(-over))) * kLn2;
            more = all - own * kLn2;
        }
        if (lse) lse[r] = (float)all;
        if (loss) loss[r] = none ? 0.0f : (float)more;
    }
}

// P of a piece of the vocabulary, words from `first` on.  Bound by the matrix cores, and a round's end by memory: with all CUs' tiles
// done at once, 256 KB of each (512 KB with low halves) leave at what HBM takes, 11 us (20).  8192 x 4096 x 32768 in bf16 1.65 to 1.69 ms,
// 1.30 to 1.33 PFLOP/s; 2049 x 1024 x 49999 in fp16, P in pairs, 384 us, 0.55; 700 x 1500 x 10000 in pairs 76 us, 0.83.
//
// A row's word has exp(l - lse) - 1, which for a row that knows its word is the difference of two numbers near one, off by what lse
// was rounded by and by l, if lse came from sums in another order as those of few rows do: 2e-6 of a gradient in the 2-norm, and all
// of one such row's.  So it is exp(-loss) - 1 if the loss is given, and else, where all words are in one piece, left out here and
// written by k_own_words from the sum of the row's others: 3e-7.  That takes 4 to 7 us of a launch and 1 % in here.
template <class H>
struct Probs {
    Plane<H> x, w;  // w: the piece's rows
    uint32_t n, count, first;
    WordList words;
    const float *lse, *loss, *loss_grad;  // loss, loss_grad: may be NULL
    Plane<G> out, turned;  // n rows of words, words of n rows; either may have no address
    uint32_t turned_cols;  // with the zeros behind the last row
    const Scales* scales;
    float* row_sums;       // `width` lists of n, one for each wave's columns; NULL: no row's word is left out
    uint32_t width;
    float* left_out;       // exp(l - lse) of the rows' words
};

typedef G h2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ Four16 packed(const v4f& v)
{
    return {__builtin_bit_cast(uint32_t, h2{(G)v[0], (G)v[1]}), __builtin_bit_cast(uint32_t, h2{(G)v[2], (G)v[3]})};
}
// What halves leave of the values.
__device__ __forceinline__ v4f left_over(const v4f& v)
{
    v4f l;
#pragma unroll
    for (int e = 0; e < 4; ++e) l[e] = v[e] - (float)(G)v[e];
    return l;
}
__device__ __forceinline__ v4f ldexp4(v4f v, int by)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = ldexpf(v[e], by);
    return v;
}
// Times 2^-by, in two steps: halves go down to 2^-24.  What is left below 2^-14 is off by 2^-25.
__device__ __forceinline__ void shift_down(Four16& v, int by)
{
    const int first = by < 48 ? by / 2 : 24, second = by < 48 ? by - first : 24;
    const G a = (G)ldexpf(1.0f, -first), b = (G)ldexpf(1.0f, -second);
    v.a = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, v.a) * h2{a, a} * h2{b, b});
    v.b = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, v.b) * h2{a, a} * h2{b, b});
}

template <class M, bool Low, class Tl>
__global__ __launch_bounds__(Tl::kThreads) void k_probs(Probs<typename M::H> p, Span span, Places places)
{
    constexpr bool kLow = Low || M::kPairP;
    __shared__ __align__(1024) char lds[lds_of<Tl, G>()];
    Tl t;
    t.template run<M::kPairs ? 3 : 1, true>(
        places.total, span, lds,
        [&](uint32_t tile, int term) {
            uint32_t i, j, split;
            places.at(tile, i, j, split);
            take<M::kPairs ? 3 : 1>(t, term, p.x, p.n, p.w, p.count, 0, i * Tl::kM, j * Tl::kN);
        },
        [&](uint32_t tile) {
            uint32_t ti, tj, split;
            places.at(tile, ti, tj, split);
            const uint32_t m0 = ti * Tl::kM, n0 = tj * Tl::kN;
            const float k = M::kPairs ? kLog2e / (p.scales->x * p.scales->w) : kLog2e, sp = p.scales->p;
            const bool edge = n0 + Tl::kN > p.count, by_row = p.scales->by_row;
            Four16 high[Tl::kMt][Tl::kNt], low[kLow ? Tl::kMt : 1][Tl::kNt];  // in 16 bits P takes half the room of the sums
            t.strips([&](int i, uint32_t row, uint32_t col, v4f(&acc)[Tl::kNt]) {
                const uint32_t r = m0 + row;
                uint32_t word = p.words.vocab;
                float lse = 0.0f, gain = 0.0f;
                if (r < p.n) {
                    word = p.words[r];
                    lse = p.lse[r] * -kLog2e;
                    gain = (p.loss_grad ? p.loss_grad[r] : 1.0f) * sp;
                }
                if (by_row) gain = ldexpf(gain, row_power(gain));
                const uint32_t here = word - p.first - n0 - col;
                const bool none = word == p.words.vocab;
#pragma unroll
                for (int j = 0; j < Tl::kNt; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[j][e] = __builtin_amdgcn_exp2f(fmaf(acc[j][e], k, lse));
                if (__builtin_expect_with_probability(here < Tl::kNt * 16 && here % 16 < 4, 0, 0.999)) {  // one lane in 128 columns, if any
                    const float own = p.loss && r < p.n ? expm1f(-p.loss[r]) : 0.0f;
                    float is = 0.0f;
#pragma unroll
                    for (int j = 0; j < Tl::kNt; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) is = here == (uint32_t)(j * 16 + e) ? acc[j][e] : is;
                    if (p.row_sums && r < p.n) p.left_out[r] = is;
                    is = p.loss || p.row_sums ? own : is - 1.0f;
#pragma unroll
                    for (int j = 0; j < Tl::kNt; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[j][e] = here == (uint32_t)(j * 16 + e) ? is : acc[j][e];
                }
#pragma unroll
                for (int j = 0; j < Tl::kNt; ++j) acc[j] *= gain;
                if (none) {  // zeros whatever the row holds
#pragma unroll
                    for (int j = 0; j < Tl::kNt; ++j) acc[j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                }
                if (edge) {  // zeros behind the piece's last word
                    const int left = (int)(p.count - n0 - col);
#pragma unroll
                    for (int j = 0; j < Tl::kNt; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[j][e] = left > j * 16 + e ? acc[j][e] : 0.0f;
                }
                v4f part = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < Tl::kNt; ++j) {
                    const v4f v = rounded(acc[j]);
                    part += v;
                    high[i][j] = packed(v);
                    if constexpr (kLow) low[i][j] = packed(left_over(v));
                    if constexpr (kLow && !M::kPairP)  // packed here, not where they are used, which takes what they come from there too
                        asm volatile("" : "+v"(high[i][j].a), "+v"(high[i][j].b), "+v"(low[i][j].a), "+v"(low[i][j].b));
                }
                if (p.row_sums) {
                    float sum = (part[0] + part[1]) + (part[2] + part[3]);
                    sum += __shfl_xor(sum, 16);
                    sum += __shfl_xor(sum, 32);
                    const uint32_t place = tj * (Tl::kN / (Tl::kNt * 16)) + t.wave % (Tl::kN / (Tl::kNt * 16));
                    if (t.lane < 16 && r < p.n) p.row_sums[(int64_t)place * p.n + r] = sum;
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            // Eight neighbours of row r from column c on, of the tile at (m, n); columns behind the last are zeros up to the pitch.  A
            // tile's places are within 32 bits of its first.
            auto put = [](const Plane<G>& o, uint32_t rows, uint32_t cols, uint32_t m, uint32_t n, bool low) {
                char* at = (char*)(o.at + (low ? o.low : 0) + (int64_t)m * o.pitch + n);
                return [at, pitch = (uint32_t)o.pitch * 2, rows = rows - m, cols = cols - n](uint32_t r, uint32_t c, const v4i& v) {
                    if ((int)r < (int)rows && (int)c < (int)cols) *(v4i*)(at + (r * pitch + c * 2)) = v;
                };
            };
            char* by = lds + Tl::kLds;
            if (p.out.at) {
                t.template out16<false>(by, high, put(p.out, p.n, (uint32_t)p.out.pitch, m0, n0, false));
                if constexpr (M::kPairP) t.template out16<false>(by, low, put(p.out, p.n, (uint32_t)p.out.pitch, m0, n0, true));
            }
            if (p.turned.at) {
                if (__builtin_expect(by_row, 0)) {  // words have sums over rows, which share a power of two
                    __builtin_amdgcn_sched_barrier(0);
                    uint32_t r = m0 + t.first_row();
#pragma unroll
                    for (int i = 0; i < Tl::kMt; ++i, r += 16) {
                        asm volatile("" : "+v"(r));
                        const int power = p.loss_grad && r < p.n ? row_power(p.loss_grad[r] * sp) : 0;
#pragma unroll
                        for (int j = 0; j < Tl::kNt; ++j) {
                            shift_down(high[i][j], power);
                            if constexpr (kLow) shift_down(low[i][j], power);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
                t.template out16<true>(by, high, put(p.turned, p.count, p.turned_cols, n0, m0, false));
                if constexpr (kLow) t.template out16<true>(by, low, put(p.turned, p.count, p.turned_cols, n0, m0, true));
            }
        });
}

// The rows' words, which without the loss are left out of P.  One that a row knows well is minus the sum of its others: as near as
// they are, and a row of P adds up to zero.  Another is nearer by itself than by that sum's roundings.  A block has 16 rows, 16 lanes to
// each of them.
constexpr float kKnown = 0.25f;
template <class M, bool Low>
__global__ __launch_bounds__(256) void k_own_words(Probs<typename M::H> p)
{
    __shared__ float lds[16][17];
    const uint32_t at = threadIdx.x & 15, part = threadIdx.x >> 4, r = blockIdx.x * 16 + at;
    float sum = 0.0f;
    if (r < p.n) {
#pragma unroll 8
        for (uint32_t i = part; i < p.width; i += 16) sum += p.row_sums[(int64_t)i * p.n + r];
    }
    lds[part][at] = sum;
    __syncthreads();
    if (part != 0 || r >= p.n) return;
    const uint32_t word = p.words[r];
    if (word == p.words.vocab) return;
    sum = 0.0f;
    for (int i = 0; i < 16; ++i) sum += lds[i][at];
    auto put = [](const Plane<G>& o, int64_t at, float v, bool low) {
        asm volatile("" : "+v"(v));  // see rounded()
        const G high = (G)v;
        o.at[at] = high;
        if (low) o.at[at + o.low] = (G)(v - (float)high);
    };
    const float gain = (p.loss_grad ? p.loss_grad[r] : 1.0f) * p.scales->p, is = p.left_out[r];
    const int power = p.scales->by_row ? row_power(gain) : 0;
    const float v = is > kKnown && is < INFINITY ? -sum : (is - 1.0f) * ldexpf(gain, power);
    if (p.out.at) put(p.out, (int64_t)r * p.out.pitch + word, v, M::kPairP);
    if (p.turned.at) put(p.turned, (int64_t)word * p.turned.pitch + r, ldexpf(v, -power), Low || M::kPairP);
}

// C = 2^e A B^T over the columns that span.lines cover, of split number s from column s * lines on: rounded to T, on top of
// `before` (fp32) and of C itself with `accumulate`.  Each split has a C of its own.  Bound by the matrix cores, at the rate of the
// library's halves, 1.30 PFLOP/s: 8192 x 4096 over 32768 words 1.62 to 1.70 ms, 1.29 to 1.36; 32768 x 4096 over 8192 rows 1.63 to 1.73 ms; 49152
// x 1024 over 2049 rows in two terms 449 us, 0.92 (33 lines a term); 700 x 1500 over 10000 words in pairs, 8 splits, 69 us, 0.91.
struct Product {
    Plane<G> a, b;
    int64_t m, n;
    const Scales* scales;  // 2^e is one over its p and over that of w, or with of_x of x
    bool of_x;
    const float* loss_grad;  // rows of A that may have powers of two of their own; NULL: none has
    void* c;
    int64_t ldc, split_stride;
    bool accumulate;
    const float* before;   // m x n; NULL: nothing
};

template <class T>
__device__ __forceinline__ void finish4(T* c, const float* before, bool accumulate, int64_t left, v4f v)
{
    typedef T t4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
    if (left >= 4) {
        if (before) v += *(const f4*)before;
        if (accumulate) {
            const t4 old = *(const t4*)c;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += (float)old[i];
        }
        t4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (T)v[i];
        *(t4*)c = w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) c[i] = (T)(v[i] + (before ? before[i] : 0.0f) + (accumulate ? (float)c[i] : 0.0f));
    }
}

template <class T, int Terms, class Tl>
__global__ __launch_bounds__(Tl::kThreads) void k_product(Product p, Span span, Places places)
{
    __shared__ __align__(1024) char lds[Tl::kLds];
    Tl t;
    t.template run<Terms>(
        places.total, span, lds,
        [&](uint32_t tile, int term) {
            uint32_t i, j, split;
            places.at(tile, i, j, split);
            take<Terms>(t, term, p.a, p.m, p.b, p.n, (int64_t)split * span.lines * (kLine / (int)sizeof(G)), i * Tl::kM, j * Tl::kN);
        },
        [&](uint32_t tile) {
            uint32_t ti, tj, split;
            places.at(tile, ti, tj, split);
            const int shift = -exponent_of(p.scales->p) - exponent_of(p.of_x ? p.scales->x : p.scales->w);
            auto write = [&](auto by_row) {
                t.each([&](uint32_t row, uint32_t col, v4f v) {
                    const int64_t r = (int64_t)ti * Tl::kM + row, c = (int64_t)tj * Tl::kN + col;
                    if (r >= p.m || c >= p.n) return;
                    v = ldexp4(v, decltype(by_row)::value ? shift - row_power(p.loss_grad[r] * p.scales->p) : shift);
                    finish4<T>((T*)p.c + split * p.split_stride + r * p.ldc + c, p.before ? p.before + r * p.n + c : nullptr, p.accumulate, p.n - c,
                               v);
                });
            };
            if (__builtin_expect(p.loss_grad && p.scales->by_row, 0))
                write(std::true_type());
            else
                write(std::false_type());
        });
}

// The splits' sums joined, in their order.
template <class T>
__global__ __launch_bounds__(256) void k_join_sums(const float* sums, int splits, int64_t m, int64_t n, T* c, int64_t ldc)
{
    const int64_t per = (n + 3) / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= m * per) return;
    const int64_t r = i / per, k = i % per * 4, left = n - k;
    v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < splits; ++s) {
        const float* from = sums + (s * m + r) * n + k;
        typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
        if (left >= 4) {
            v += *(const f4*)from;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += j < left ? from[j] : 0.0f;
        }
    }
    finish4<T>(c + r * ldc + k, nullptr, false, left, v);
}

// ---- the calls ----

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int64_t parts(int64_t n, int64_t of) { return (n + of - 1) / of; }

constexpr int kPer = kLine / 2;  // elements of a line

// Whether a matrix can be read where it is.
template <class M>
bool lies_in_lines(const Matrix& x, int64_t dim)
{
    if (sizeof(typename M::T) != sizeof(typename M::H)) return false;
    return dim % kPer == 0 && x.ld % kPer == 0 && x.ld * (int64_t)sizeof(typename M::H) < (1 << 24) && (uintptr_t)x.at % 16 == 0;
}

// The workspace, handed out in order.
struct Space {
    char* at;
    size_t used;
    template <class T>
    T* get(int64_t count)
    {
        T* p = at ? (T*)(at + used) : nullptr;
        used += (size_t)up(count * (int64_t)sizeof(T), 256);
        return p;
    }
    template <class H>
    Plane<H> plane(int64_t rows, int64_t pitch, bool pairs)
    {
        return {get<H>(rows * pitch * (pairs ? 2 : 1)), pitch, pairs ? rows * pitch : 0};
    }
};

template <class Tl>
struct Shape {
    typedef Tl Is;
};

// f(a tile's type) for the tile of kTileCosts[pick]
template <class Core, class F>
void by_tile(int pick, const F& f)
{
    if (pick == 0)
        f(Shape<Tile<Core, 256, 256, 2, 2, 2>>());
    else if (pick == 1)
        f(Shape<Tile<Core, 192, 192, 2, 2, 3>>());
    else if (pick == 2)
        f(Shape<Tile<Core, 128, 128, 2, 2, 2>>());
    else
        f(Shape<Tile<Core, 64, 64, 2, 2, 4>>());
}

template <class T>
Source<T> source(const Matrix& m, int64_t rows, int64_t cols, const WordList& words = {}, int64_t first = 0)
{
    return {m.at ? (const T*)m.at + first * m.ld : nullptr, m.ld, rows, cols, words};
}

// Which tile: as for the products of codes, the time of a product is that of its rounds, with what these products' ends cost.  A
// round ends with all tiles' stores at once; two blocks to a CU have one's end beside the other's products.  Measured, us a
// kernel, tiles of 256, 192, 128, 64 (n x dim x vocab, pairs of P but for bf16):
//   logits   700 x 1500 x 10000 fp32 98 71 68 103; 2049 x 1024 x 49999 fp16 235 256 265 421; 4000 x 512 x 20000 102 115 102 171;
//            300 x 700 x 5000 bf16 23.6 17.4 12.4 8.2; 512 x 1024 x 32768 bf16 42 59 42 64
//   P        116 84 76 110; 367 387 431 590; 218 210 189 259; 30 20 13.4 8.8; 51 72 46 64
//   w_grad   72 69 73 103; 460 494 498 796; 204 250 257 331; 22.9 15 9.4 8.8; 64 76 51 73
enum Kind { kLogits, kProbs, kProbPairs, kProduct };
struct HalfCost {
    float alone, line, thrice;  // us a line of 128 bytes, one tile to a CU or kTileCosts' per_cu; of pairs, whose lines come three times
    float launch, end[4];
};
constexpr HalfCost kHalfCosts[] = {{1.27f, 1.27f, 1.20f, 8.0f, {9.0f, 23.0f, 34.0f, 16.0f}},
                                   {1.06f, 1.06f, 0.95f, 7.0f, {4.0f, 10.0f, 15.0f, 6.0f}},
                                   {0.80f, 1.27f, 0.95f, 5.5f, {1.0f, 2.0f, 10.0f, 2.5f}},
                                   {0.25f, 0.48f, 0.35f, 4.5f, {0.5f, 1.0f, 1.5f, 1.0f}}};

double half_time(Kind kind, int terms, int pick, int64_t tiles, int64_t lines)
{
    const HalfCost& c = kHalfCosts[pick];
    const int64_t slots = (int64_t)kCus * kTileCosts[pick].per_cu, left = tiles % slots;
    const float line = terms == 3 ? c.thrice : c.line, alone = line < c.alone ? line : c.alone;
    double t = c.launch + (double)(tiles / slots) * (lines * terms * line + c.end[kind]);
    if (left) t += lines * terms * (left <= kCus ? alone : line) + c.end[kind];
    return t;
}

// count(side): tiles of the whole launch.
template <class Count>
int best_half(Kind kind, int terms, const Count& count, int64_t lines, double* time)
{
    int best = 0;
    for (int i = 0; i < 4; ++i) {
        const double t = half_time(kind, terms, i, count(kTileCosts[i].side), lines);
        if (i == 0 || t < *time) *time = t, best = i;
    }
    return best;
}

// Rows in one launch or two: as many large tiles as fill whole rounds or whole tiles, and the rest in tiles of its own.
struct RowPlan {
    int pick, rest_pick;
    int64_t rows;  // of the first launch
};
RowPlan plan_rows(Kind kind, int terms, int64_t m, int64_t n, int64_t lines)
{
    auto tiles = [&](int64_t rows, int64_t side) { return parts(rows, side) * parts(n, side); };
    double least = 0.0, best = 0.0;
    RowPlan plan = {best_half(kind, terms, [&](int64_t side) { return tiles(m, side); }, lines, &least), 0, m};
    best = least;
    for (int i = 0; i < 3; ++i) {
        const int64_t side = kTileCosts[i].side, strip = parts(n, side), slots = (int64_t)kCus * kTileCosts[i].per_cu;
        for (const int64_t rows : {m / side * side, tiles(m, side) / slots * slots / strip * side}) {
            if (rows <= 0 || rows >= m) continue;
            double rest = 0.0;
            const int rest_pick = best_half(kind, terms, [&](int64_t s) { return tiles(m - rows, s); }, lines, &rest);
            const double t = half_time(kind, terms, i, tiles(rows, side), lines) + rest + 5.0 + 0.05 * least;  // two are worth it if clearly better
            if (t < best) best = t, plan = {i, rest_pick, rows};
        }
    }
    return plan;
}

constexpr int64_t kRowsAtOnce = 16384;  // of the forward pass

// The products of that many rows with the vocabulary.
template <class M>
RowPlan forward_plan(int64_t rows, int64_t vocab, int64_t lines)
{
    return plan_rows(kLogits, M::kPairs ? 3 : 1, rows, vocab, lines);
}
int64_t forward_width(int pick, int64_t vocab) { return 2 * parts(vocab, kTileCosts[pick].side); }

// The blocks of k_few, the steps that it takes, and whether it is what a call takes.  It reads the weight once for every 32 rows; the
// way by tiles reads it once, and where it has to be laid out first a second time, for fp32 a third, beside writing it.  us, here /
// there: against 10000 x 1500 fp32 64 rows 44 / 63, 96 rows 64 / 74; 100000 x 2048 fp32 292 / 740, 436 / 791; 10000 x 1502 bf16 33 rows
// 24 / 28; 100000 x 3002 bf16 20 rows 113 / 403.  From 97 rows on the way by tiles is taken whatever the weight: of 128 rows against
// 100000 x 2048 fp32 it takes 666, and four passes here would be 580 by the figures above, against 10000 x 1500 64 and 85.
// Rows of 16 bits that start between two words are read at half the rate: 10000 x 1501 bf16 20 rows 31 / 28, 33 rows 54 / 28; 100000 x
// 3001 207 / 404, 420 / 404.
constexpr int64_t kFewBlocks = 512;
template <class M>
int64_t few_steps(int64_t dim)
{
    return parts(dim, kFewWaves * FewCore<typename M::T>::kStep);
}
template <class M>
bool takes_few(int64_t rows, int64_t dim, const Matrix& w, bool lay_w)
{
    const bool between = sizeof(typename M::T) == 2 && (w.ld % 2 != 0 || (uintptr_t)w.at % 4 != 0);
    return parts(rows, kFewRows) <= (lay_w && !between ? 3 : 1) && dim >= 8 && few_steps<M>(dim) <= 16;
}

// A CU's registers hold two blocks where a wave's operands take few of them.
template <class M>
int64_t few_blocks(int64_t rows, int64_t dim, int64_t vocab)
{
    return std::min(parts(vocab, 16), few_steps<M>(dim) <= (rows <= 16 ? 10 : 6) ? kFewBlocks : kFewBlocks / 2);
}

void join_rows(const float2* pairs, uint32_t width, int64_t rows, const WordList& words, const float* mine, float* loss, float* lse, hipStream_t s)
{
    if (width >= 512 && rows <= 4096)
        k_join_rows<256><<<(uint32_t)rows, 256, 0, s>>>(pairs, width, rows, words, mine, loss, lse);
    else
        k_join_rows<64><<<(uint32_t)parts(rows, 4), 256, 0, s>>>(pairs, width, rows, words, mine, loss, lse);
}

template <class M>
struct ForwardPlan {
    typedef typename M::H H;
    int64_t pitch;
    bool few, lay_x, lay_w;
    float* part;
    Scales* scales;
    Plane<H> x, w;
    float2* pairs;
    float* mine;
    size_t bytes;
    ForwardPlan(const Entropy& q, char* scratch)
    {
        Space s = {scratch, 0};
        const int64_t n = q.words.n, v = q.words.vocab, at_once = std::min(n, kRowsAtOnce);
        pitch = up(q.dim, kPer);
        lay_x = !lies_in_lines<M>(q.x, q.dim);
        lay_w = !lies_in_lines<M>(q.w, q.dim);
        few = takes_few<M>(n, q.dim, q.w, lay_w);
        if (few) lay_x = lay_w = false;
        scales = s.get<Scales>(1);
        part = s.get<float>(M::kPairs ? kPartKinds * kParts : 0);
        x = lay_x ? s.plane<H>(n, pitch, M::kPairs) : Plane<H>{(H*)q.x.at, q.x.ld, 0};
        w = lay_w ? s.plane<H>(v, pitch, M::kPairs) : Plane<H>{(H*)q.w.at, q.w.ld, 0};
        auto pairs_of = [&](int64_t rows) {
            const RowPlan plan = forward_plan<M>(rows, v, pitch / kPer);
            return std::max(plan.rows * forward_width(plan.pick, v), (rows - plan.rows) * forward_width(plan.rest_pick, v));
        };
        pairs = s.get<float2>(few ? n * few_blocks<M>(n, q.dim, v) : std::max(pairs_of(at_once), pairs_of((n - 1) % kRowsAtOnce + 1)));
        mine = s.get<float>(at_once);
        bytes = s.used;
    }
};

WordList list(const Words& w) { return {w.at, w.wide, (uint32_t)w.vocab}; }

// x and w laid out and their scales settled; g is the rows' gradient, or without an address ones.
template <class M, bool Scaled>
void lay_out(const Layout<typename M::T, typename M::H>& x, const Layout<typename M::T, typename M::H>& w, const Source<float>& g, bool later,
             float* part, Scales* scales, hipStream_t s)
{
    const int64_t tiles = (int64_t)x.tiles_r * x.tiles_c + (int64_t)w.tiles_r * w.tiles_c;
    if (tiles == 0) return;  // a later piece of a w that is read where it is
    const uint32_t blocks = (uint32_t)std::min(tiles, (int64_t)kParts);
    k_layout<M, Scaled><<<blocks, 256, 0, s>>>(x, w, g, part);
    if (Scaled) k_settle<M><<<M::kScaled ? std::min(blocks, kSettleBlocks) : 1, 256, 0, s>>>(x, w, blocks, later, part, scales);
}

template <class M>
void forward(const Entropy& q, char* scratch, hipStream_t s)
{
    typedef typename M::T T;
    typedef typename M::H H;
    const ForwardPlan<M> f(q, scratch);
    const int64_t n = q.words.n, v = q.words.vocab;
    if (f.few) {
        const int64_t groups = parts(v, 16), steps = few_steps<M>(q.dim), blocks = few_blocks<M>(n, q.dim, v);
        int64_t r = 0, rows = 0;
        auto go = [&](auto kernel) {
            const Few<T> p = {(const T*)q.x.at + r * q.x.ld, (const T*)q.w.at, q.x.ld, q.w.ld, (uint32_t)rows, (uint32_t)q.dim, (uint32_t)groups,
                              list(q.words).from(r), f.pairs + r * blocks, f.mine + r};
            kernel<<<(uint32_t)blocks, 64 * kFewWaves, 0, s>>>(p);
        };
        auto by_steps = [&](auto tiles) {
            constexpr int kTiles = decltype(tiles)::value;
            // the kernel's steps are the call's or one more
            if (steps <= 1)
                go(k_few<T, 1, kTiles>);
            else if (steps <= 2)
                go(k_few<T, 2, kTiles>);
            else if (steps <= 4)
                go(k_few<T, 4, kTiles>);
            else if (steps <= 6)
                go(k_few<T, 6, kTiles>);
            else if (steps <= 8)
                go(k_few<T, 8, kTiles>);
            else if (steps <= 10)
                go(k_few<T, 10, kTiles>);
            else if (steps <= 12)
                go(k_few<T, 12, kTiles>);
            else if (steps <= 14)
                go(k_few<T, 14, kTiles>);
            else
                go(k_few<T, 16, kTiles>);
        };
        for (; r < n; r += rows) {
            rows = std::min(n - r, (int64_t)kFewRows);
            if (rows <= 16)
                by_steps(std::integral_constant<int, 1>());
            else
                by_steps(std::integral_constant<int, 2>());
        }
        join_rows(f.pairs, (uint32_t)blocks, n, list(q.words), f.mine, q.loss, q.lse, s);
        return;
    }
    if (f.lay_x || f.lay_w) {
        const uint32_t across = (uint32_t)parts(f.pitch, 64);
        const Layout<T, H> lx = {source<T>(q.x, n, q.dim, list(q.words)), f.lay_x ? f.x : Plane<H>{}, {}, f.lay_x ? (uint32_t)parts(n, 64) : 0, across};
        const Layout<T, H> lw = {source<T>(q.w, v, q.dim), f.lay_w ? f.w : Plane<H>{}, {}, f.lay_w ? (uint32_t)parts(v, 64) : 0, across};
        lay_out<M, M::kPairs>(lx, lw, {}, false, f.part, f.scales, s);
    }
    for (int64_t r = 0; r < n; r += kRowsAtOnce) {
        const int64_t rows = std::min(n - r, kRowsAtOnce);
        const Span span = {(uint32_t)(f.x.pitch * sizeof(H)), (uint32_t)(f.w.pitch * sizeof(H)), (uint32_t)(f.pitch / kPer)};
        auto logits = [&](int pick, int64_t row, int64_t rows) {
            const uint32_t width = (uint32_t)forward_width(pick, v);
            const WordList words = list(q.words).from(r + row);
            by_tile<typename M::Core>(pick, [&](auto shape) {
                typedef typename decltype(shape)::Is Tl;
                const Places places = {(uint32_t)parts(rows, Tl::kM), (uint32_t)parts(v, Tl::kN), (uint32_t)(parts(rows, Tl::kM) * parts(v, Tl::kN))};
                const Plane<H> x = {f.x.at + (r + row) * f.x.pitch, f.x.pitch, f.x.low};
                const Forward<H> p = {x, f.w, (uint32_t)rows, words, f.pairs, width, f.mine, f.scales};
                k_logits<M, Tl><<<tile_blocks(pick, places.total), Tl::kThreads, 0, s>>>(p, span, places);
            });
            join_rows(f.pairs, width, rows, words, f.mine, q.loss ? q.loss + r + row : nullptr, q.lse ? q.lse + r + row : nullptr, s);
        };
        const RowPlan plan = forward_plan<M>(rows, v, span.lines);
        logits(plan.pick, 0, plan.rows);
        if (plan.rows < rows) logits(plan.rest_pick, plan.rows, rows - plan.rows);
    }
}

// A piece of the vocabulary: as many words as keep P, both ways, at this size.
constexpr int64_t kPieceBytes = (int64_t)1 << 30;

template <class M>
struct GradPlan {
    // Rows that are a large power of two apart would meet in a few of the memory's channels: a line more between them.
    static int64_t spread(int64_t cols) { return cols * (int64_t)sizeof(G) % 4096 == 0 ? cols + kPer : cols; }

    typedef typename M::H H;
    int64_t pitch, cols_n, cols_v, piece, pieces;  // columns of rows over n and over a piece's words
    int splits, pick_x;   // of the product for x's gradient
    bool lay_x, lay_w, wide;  // wide: w's gradient has more bits than the operands
    float* part;
    Scales* scales;
    Plane<H> x, w;
    Plane<G> xt, wt, p, pt;
    float* sums;
    float *row_sums, *left_out;  // of P, for the rows' words; NULL with several pieces, whose first are multiplied before the last are known
    size_t bytes;
    static constexpr int kTerms = M::kPairs ? 3 : (M::kPairP ? 2 : 1);  // of the product for x's gradient
    GradPlan(const Entropy& q, char* scratch)
    {
        Space s = {scratch, 0};
        const int64_t n = q.words.n, v = q.words.vocab;
        pitch = up(q.dim, kPer);
        cols_n = up(n, kPer);
        lay_x = !lies_in_lines<M>(q.x, q.dim);
        lay_w = !lies_in_lines<M>(q.w, q.dim);
        wide = !M::kPairs && q.w_grad.at && q.w_grad.type == kGradF32;
        const int64_t word = cols_n * (int64_t)sizeof(G) * ((q.x_grad.at ? 1 : 0) + (q.w_grad.at ? 1 : 0));
        const int64_t most = std::min(std::max(kPieceBytes / (word * (M::kPairP ? 2 : 1)), (int64_t)1024), (int64_t)1 << 22);
        pieces = parts(v, most);
        piece = std::min(up(parts(v, pieces), 256), v);
        pieces = parts(v, piece);
        // The contraction over words is long and its tiles may be few.
        splits = 1;
        pick_x = 0;
        int64_t lines = parts(piece, kPer);
        if (q.x_grad.at) {
            double least = 0.0;
            for (int k = 1; k <= 64 && k * 8 <= std::max(lines, (int64_t)8); ++k) {
                double t = 0.0;
                const int64_t each = parts(lines, k);
                const int pick = best_half(kProduct, kTerms, [&](int64_t side) { return parts(n, side) * parts(q.dim, side) * k; }, each, &t);
                if (k > 1) t += 4.0 + 2e-6 * (double)n * (double)q.dim * k;  // sums through memory, and their launch
                if (k == 1 || t < least) least = t, splits = k, pick_x = pick;
            }
        }
        lines = parts(lines, splits) * splits;
        cols_v = lines * kPer;
        const int64_t pitch_n = spread(cols_n), pitch_v = spread(cols_v);
        scales = s.get<Scales>(1);
        part = s.get<float>(kPartKinds * kParts);
        x = lay_x ? s.plane<H>(n, pitch, M::kPairs) : Plane<H>{(H*)q.x.at, q.x.ld, 0};
        w = lay_w ? s.plane<H>(piece, pitch, M::kPairs) : Plane<H>{};
        xt = wt = p = pt = Plane<G>{};
        if (q.w_grad.at) {
            xt = s.plane<G>(q.dim, pitch_n, M::kPairs);
            pt = s.plane<G>(piece, pitch_n, M::kPairP || wide);
        }
        if (q.x_grad.at) {
            wt = s.plane<G>(q.dim, pitch_v, M::kPairs);
            p = s.plane<G>(n, pitch_v, M::kPairP);
        }
        sums = q.x_grad.at && (splits > 1 || pieces > 1) ? s.get<float>(splits * n * q.dim) : nullptr;
        row_sums = left_out = nullptr;
        if (pieces == 1) {
            const int64_t cols = q.x_grad.at ? cols_v : v;
            const RowPlan plan = probs_plan(n, cols);
            row_sums = s.get<float>(std::max(plan.rows * probs_width(plan.pick, cols), (n - plan.rows) * probs_width(plan.rest_pick, cols)));
            left_out = s.get<float>(n);
        }
        bytes = s.used;
    }
    // The launches for P of `cols` words.
    RowPlan probs_plan(int64_t n, int64_t cols) const
    {
        return plan_rows(M::kPairP || wide ? kProbPairs : kProbs, M::kPairs ? 3 : 1, n, cols, pitch / kPer);
    }
    static int64_t probs_width(int pick, int64_t cols) { return 2 * parts(cols, kTileCosts[pick].side); }
};

template <class T, int Terms>
void product_part(int pick, const Product& p, int64_t lines, int splits, hipStream_t s)
{
    by_tile<HalfCore>(pick, [&](auto shape) {
        typedef typename decltype(shape)::Is Tl;
        const uint32_t tm = (uint32_t)parts(p.m, Tl::kM), tn = (uint32_t)parts(p.n, Tl::kN);
        const Places places = {tm, tn, tm * tn * splits};
        const Span span = {(uint32_t)(p.a.pitch * sizeof(G)), (uint32_t)(p.b.pitch * sizeof(G)), (uint32_t)lines};
        k_product<T, Terms, Tl><<<tile_blocks(pick, places.total), Tl::kThreads, 0, s>>>(p, span, places);
    });
}

// The same without splits, in the launches of a plan.
template <class T, int Terms>
void product(const Product& p, int64_t lines, hipStream_t s)
{
    const RowPlan plan = plan_rows(kProduct, Terms, p.m, p.n, lines);
    auto part = [&](int pick, int64_t first, int64_t rows) {
        Product r = p;
        r.a.at += first * p.a.pitch;
        r.m = rows;
        r.c = (T*)p.c + first * p.ldc;
        if (p.before) r.before = p.before + first * p.n;
        product_part<T, Terms>(pick, r, lines, 1, s);
    };
    part(plan.pick, 0, plan.rows);
    if (plan.rows < p.m) part(plan.rest_pick, plan.rows, p.m - plan.rows);
}

template <class M>
void gradient(const Entropy& q, char* scratch, hipStream_t s)
{
    typedef typename M::T T;
    typedef typename M::H H;
    constexpr int kTerms = GradPlan<M>::kTerms;
    const GradPlan<M> g(q, scratch);
    const int64_t n = q.words.n, v = q.words.vocab;
    const WordList words = list(q.words);
    const Source<float> gains = {q.loss_grad, 1, n, 1, words};
    for (int64_t k = 0; k < g.pieces; ++k) {
        const int64_t first = k * g.piece, count = std::min(g.piece, v - first);
        const Plane<H> w = g.lay_w ? g.w : Plane<H>{(H*)q.w.at + first * q.w.ld, q.w.ld, 0};
        // x once, and this piece of w
        Layout<T, H> lx = {source<T>(q.x, n, q.dim, words), g.lay_x ? g.x : Plane<H>{}, g.xt, 0, (uint32_t)parts(g.pitch, 64)};
        Layout<T, H> lw = {source<T>(q.w, count, q.dim, {}, first), g.lay_w ? g.w : Plane<H>{}, g.wt, 0, lx.tiles_c};
        if (k == 0 && (g.lay_x || g.xt.at)) lx.tiles_r = (uint32_t)parts(g.cols_n, 64);
        if (g.lay_w || g.wt.at) lw.tiles_r = (uint32_t)parts(g.wt.at ? g.cols_v : count, 64);
        lay_out<M, true>(lx, lw, k == 0 ? gains : Source<float>{}, k > 0, g.part, g.scales, s);

        const Span span = {(uint32_t)(g.x.pitch * sizeof(H)), (uint32_t)(w.pitch * sizeof(H)), (uint32_t)(g.pitch / kPer)};
        const int64_t wide = g.p.at ? g.cols_v : count;  // padding of P's rows is written with the last tiles
        auto probs = [&](int pick, int64_t row, int64_t rows) {
            by_tile<typename M::Core>(pick, [&](auto shape) {
                typedef typename decltype(shape)::Is Tl;
                const uint32_t tm = (uint32_t)parts(rows, Tl::kM), tn = (uint32_t)parts(wide, Tl::kN);
                const Places places = {tm, tn, tm * tn};
                const Plane<H> x = {g.x.at + row * g.x.pitch, g.x.pitch, g.x.low};
                const Plane<G> out = {g.p.at ? g.p.at + row * g.p.pitch : nullptr, g.p.pitch, g.p.low};
                // columns of the transpose up to the pitch are this launch's if the last rows are
                const Plane<G> turned = {g.pt.at ? g.pt.at + row : nullptr, g.pt.pitch, g.pt.low};
                const Probs<H> p = {x, w, (uint32_t)rows, (uint32_t)count, (uint32_t)first, words.from(row), q.lse + row,
                                    q.loss ? q.loss + row : nullptr, q.loss_grad ? q.loss_grad + row : nullptr, out, turned,
                                    (uint32_t)(row + rows < n ? rows : g.cols_n - row), g.scales, q.loss ? nullptr : g.row_sums,
                                    (uint32_t)g.probs_width(pick, wide), g.left_out};
                auto go = [&](auto kernel, auto own_words) {
                    kernel<<<tile_blocks(pick, places.total), Tl::kThreads, 0, s>>>(p, span, places);
                    if (p.row_sums) own_words<<<(uint32_t)parts(rows, 16), 256, 0, s>>>(p);
                };
                if constexpr (M::kPairP)
                    go(k_probs<M, true, Tl>, k_own_words<M, true>);
                else if (g.wide)
                    go(k_probs<M, true, Tl>, k_own_words<M, true>);
                else
                    go(k_probs<M, false, Tl>, k_own_words<M, false>);
            });
        };
        const RowPlan plan = g.probs_plan(n, wide);
        probs(plan.pick, 0, plan.rows);
        if (plan.rows < n) probs(plan.rest_pick, plan.rows, n - plan.rows);
        if (q.x_grad.at) {
            const int64_t lines = g.cols_v / kPer / g.splits;
            if (g.splits > 1 || k + 1 < g.pieces) {
                const Product p = {g.p, g.wt, n, q.dim, g.scales, false, q.loss_grad, g.sums, q.dim, n * q.dim, k > 0, nullptr};
                product_part<float, kTerms>(g.pick_x, p, lines, g.splits, s);
            } else {
                const Product p = {g.p, g.wt, n, q.dim, g.scales, false, q.loss_grad, q.x_grad.at, q.x_grad.ld, 0, false, g.pieces > 1 ? g.sums : nullptr};
                product_part<T, kTerms>(g.pick_x, p, lines, 1, s);
            }
        }
        if (q.w_grad.at) {
            char* c = (char*)q.w_grad.at + first * q.w_grad.ld * (q.w_grad.type == kGradF32 ? 4 : 2);
            const Product p = {g.pt, g.xt, count, q.dim, g.scales, true, nullptr, c, q.w_grad.ld, 0, q.accumulate, nullptr};
            const int64_t lines = g.cols_n / kPer;
            if constexpr (M::kPairs) {
                product<float, 3>(p, lines, s);
            } else {
                if (g.wide)
                    product<float, 2>(p, lines, s);
                else
                    product<T, kTerms>(p, lines, s);
            }
        }
    }
    if (q.x_grad.at && g.splits > 1)
        k_join_sums<T><<<(uint32_t)parts(n * parts(q.dim, 4), 256), 256, 0, s>>>(g.sums, g.splits, n, q.dim, (T*)q.x_grad.at, q.x_grad.ld);
}

}  // namespace

size_t entropy_scratch(const Entropy& q)
{
    size_t bytes = 0;
    by_mode(q.x.type, [&](auto m) { bytes = ForwardPlan<decltype(m)>(q, nullptr).bytes; });
    return bytes;
}

size_t entropy_grad_scratch(const Entropy& q)
{
    size_t bytes = 0;
    by_mode(q.x.type, [&](auto m) { bytes = GradPlan<decltype(m)>(q, nullptr).bytes; });
    return bytes;
}

void launch_entropy(const Entropy& q, char* scratch, hipStream_t s)
{
    by_mode(q.x.type, [&](auto m) { forward<decltype(m)>(q, scratch, s); });
}

void launch_entropy_grad(const Entropy& q, char* scratch, hipStream_t s)
{
    by_mode(q.x.type, [&](auto m) { gradient<decltype(m)>(q, scratch, s); });
}

}  // namespace sidco
