// The orthogonalised update: momentum, Newton-Schulz products, weights.
//
// X_0 = u / (|u| + eps), transposed if u is tall, so that X is m x n with m <= n; then `steps` times
//   G = X X^T,  P = aI + bG + cG^2,  X <- P X,
// which moves every singular value s to as + bs^3 + cs^5.  All three products are of the form A B^T over the rows of what is
// stored (G and P are symmetric, and X is stored both as it is and transposed), G and P are computed for tiles on and below
// the diagonal and mirrored.  With a in P's diagonal the last product needs no second operand in its epilogue, and the largest
// term of the sum is not rounded twice.
//
// Steps go in groups (sidco_ortho_plan.h): within one the next G is P G P, and X moves once, by the product of the P.
//
// Operands are halves; sums, the norm and the update are fp32 or more.  Singular values stay below 1.5, so X and G are kept
// times 2^14 and P and its products times powers of two that follow from a, b, c: entries far below the largest one keep their
// 11 bits.  Or each operand is a pair of halves, the second one what the first leaves, 22 bits together, and a product is three:
// low high + high low + high high.  Which of the two is decided step by step: what a rounding leaves in directions in which u has
// little or nothing is multiplied by up to a in every step after it, so that halves from the first step on cost a result 1e-3
// where the singular values are alike, but 1.6e-2 to 2.4e-2 where they fall off like 1/k^2 or exp(-k/10) or 32 of them are all there
// are, and 0.15 at rank one (a = 3.4445, five steps).  With pairs in all steps but the last it is 4e-4 to 8e-4, 1.4e-3 at rank
// one, less than a result in bf16 loses by its own rounding (1.7e-3; together 1.7e-3 to 1.8e-3 and 2.4e-3): that is what such a
// result takes.  Results in fp32 and fp16 take pairs throughout (5e-7 to 1.3e-5; 6.5e-5).
#include <math.h>

#include <type_traits>

#include "sidco_dense.h"
#include "sidco_ortho_plan.h"
#include "sidco_product.h"

namespace sidco {
namespace {

constexpr float kScaleX = 16384.0f;
constexpr int kNormBlock = 256;

template <int Type>
struct Elem;
template <>
struct Elem<kGradF32> {
    typedef float T;
};
template <>
struct Elem<kGradF16> {
    typedef _Float16 T;
};
template <>
struct Elem<kGradBf16> {
    typedef __bf16 T;
};

// f(Elem) for an element type
template <class F>
void by_element(int type, const F& f)
{
    if (type == kGradF32)
        f(Elem<kGradF32>());
    else if (type == kGradF16)
        f(Elem<kGradF16>());
    else
        f(Elem<kGradBf16>());
}

// ---- the start: momentum, norm, X and its transpose ----

// Sum over the block; the result is thread 0's.
__device__ __forceinline__ double block_sum(double v, double* lds)
{
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) v += __shfl_down(v, s);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) lds[wave] = v;
    __syncthreads();
    double t = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < (int)(blockDim.x >> 6); ++w) t += lds[w];
    return t;
}

// Eight neighbours, in words of the element's own alignment: a row may start anywhere.
template <class T>
__device__ __forceinline__ void load8(const T* p, float v[8])
{
    if constexpr (sizeof(T) == 4) {
        typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
        const f4 a = *(const f4*)p, b = *(const f4*)(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    } else {
        typedef T t8 __attribute__((ext_vector_type(8), aligned(2)));
        const t8 a = *(const t8*)p;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
    }
}

__device__ __forceinline__ void store8(float* p, const float v[8])
{
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
    *(f4*)p = f4{v[0], v[1], v[2], v[3]};
    *(f4*)(p + 4) = f4{v[4], v[5], v[6], v[7]};
}

template <class T>
struct Start {
    const T* x;        // the matrix, or the gradient
    int64_t ld, stride;
    float* momentum;   // NULL: x alone; else rows of `cols`, matrices of rows * cols
    float mu;
    bool nesterov;
    int64_t rows, cols;
    double* part;      // partial sums of squares, `parts` a matrix
    int parts;
};

// u from the gradient and the momentum that k_norm has moved: n of 8 neighbours, zeros after them
template <class T>
__device__ __forceinline__ void update8(const Start<T>& p, int64_t z, int64_t r, int64_t c, int64_t n, float u[8])
{
    const T* x = p.x + z * p.stride + r * p.ld + c;
    const float* m = p.momentum ? p.momentum + (z * p.rows + r) * p.cols + c : nullptr;
    if (n >= 8) {
        load8(x, u);
        if (m) {
            float old[8];
            load8(m, old);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = p.nesterov ? fmaf(p.mu, old[i], u[i]) : old[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            u[i] = i < n ? (float)x[i] : 0.0f;
            if (m && i < n) u[i] = p.nesterov ? fmaf(p.mu, m[i], u[i]) : m[i];
        }
    }
}

// Moves the momentum and adds up u^2, in 64 bits.  A block takes rows, of a matrix without gaps pieces of kNormRow elements, in
// turn; its sum has a place of its own, so that the total does not depend on which block ends first.  Bound by memory:
// 4096 x 25088, gradient in bf16, 167 us for 1.03 GB, 6.2 TB/s; four of 1500 x 6000 in fp32 75 us for 432 MB, 5.8 TB/s.
constexpr int kNormRow = 16 * kNormBlock;
template <class T>
__global__ __launch_bounds__(kNormBlock) void k_norm(Start<T> p)
{
    __shared__ double lds[kNormBlock / 64];
    const int64_t z = blockIdx.y, all = p.rows * p.cols;
    const bool whole = p.ld == p.cols;
    const int64_t rows = whole ? (all + kNormRow - 1) / kNormRow : p.rows;
    double sum = 0.0;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const int64_t len = whole ? (all - r * kNormRow < kNormRow ? all - r * kNormRow : kNormRow) : p.cols;
        const T* x = p.x + z * p.stride + r * (whole ? kNormRow : p.ld);
        float* m = p.momentum ? p.momentum + z * all + r * (whole ? kNormRow : p.cols) : nullptr;
#pragma unroll 2
        for (int64_t c = threadIdx.x * 8; c < len; c += 8 * kNormBlock) {
            float u[8];
            if (c + 8 <= len) {
                load8(x + c, u);
                if (m) {
                    float moved[8];
                    load8(m + c, moved);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        moved[i] = fmaf(p.mu, moved[i], u[i]);
                        u[i] = p.nesterov ? fmaf(p.mu, moved[i], u[i]) : moved[i];
                    }
                    store8(m + c, moved);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool in = c + i < len;
                    u[i] = in ? (float)x[c + i] : 0.0f;
                    if (m && in) {
                        const float moved = fmaf(p.mu, m[c + i], u[i]);
                        m[c + i] = moved;
                        u[i] = p.nesterov ? fmaf(p.mu, moved, u[i]) : moved;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += (double)u[i] * (double)u[i];
        }
    }
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) p.part[z * p.parts + blockIdx.x] = sum;
}

// Where X and X^T of one matrix after the other lie: rows of `pitch` halves, the low halves `low` after the high ones.
struct Plane {
    _Float16* at;
    int64_t pitch, low, stride;  // low 0: there are none
};

template <bool Full>
__device__ __forceinline__ void put8(const Plane& o, int64_t z, int64_t r, int64_t c, const float v[8])
{
    _Float16* p = o.at + z * o.stride + r * o.pitch + c;
    v8h h, l;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        h[i] = (_Float16)v[i];
        l[i] = (_Float16)(v[i] - (float)h[i]);
    }
    *(v8h*)p = h;
    if (Full) *(v8h*)(p + o.low) = l;
}

// 64 x 64 elements a block: rows go to `natural`, and through LDS to `turned`, the padding of both as zeros.  X is kept both
// ways so that every product reads whole lines along its contraction.  Bound by memory: 4096 x 25088 with momentum, pairs of
// halves, 297 us for 1.44 GB, 4.8 TB/s; four of 1500 x 6000 112 us for 576 MB, 5.1 TB/s.
template <class T, bool Full>
__global__ __launch_bounds__(256) void k_start(Start<T> p, float eps, Plane natural, Plane turned)
{
    __shared__ float tile[64][65];
    __shared__ double lds[4];
    __shared__ double inverse;
    const int64_t z = blockIdx.z;
    double sum = 0.0;
    for (int i = threadIdx.x; i < p.parts; i += 256) sum += p.part[z * p.parts + i];
    const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
    const int row = threadIdx.x >> 3, col = (threadIdx.x & 7) * 8;
    float u[2][8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int64_t r = r0 + k * 32 + row, c = c0 + col;
        update8(p, z, r, c, r < p.rows ? p.cols - c : 0, u[k]);
    }
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) inverse = (double)kScaleX / (sqrt(sum) + (double)eps);
    __syncthreads();
    const double inv = inverse > 1e300 ? 1e300 : inverse;  // zeros stay zeros without eps too; a NaN stays one
    const bool plain = inv > 1e-30 && inv < 1e30;  // else the factor or the elements are not of fp32's range
    const float f = (float)inv;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (plain) {
#pragma unroll
            for (int i = 0; i < 8; ++i) u[k][i] *= f;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) u[k][i] = (float)((double)u[k][i] * inv);
        }
        const int64_t r = r0 + k * 32 + row;
        if (r < p.rows) put8<Full>(natural, z, r, c0 + col, u[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) tile[k * 32 + row][col + i] = u[k][i];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = k * 32 + row;
        if (c0 + c >= p.cols) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) u[k][i] = tile[col + i][c];
        put8<Full>(turned, z, c0 + c, r0 + col, u[k]);
    }
}

// ---- the products ----

// Eight neighbours of row r from column c on, a multiple of 8; columns from `cols` on are padding, to 64, and zero.
__device__ __forceinline__ void put8(const Plane& o, int64_t z, uint32_t rows, uint32_t cols, uint32_t r, uint32_t c, v8h v, bool low)
{
    if (r >= rows || c >= (uint32_t)o.pitch) return;
    if (c + 8 > cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? v[i] : (_Float16)0.0f;
    }
    *(v8h*)(o.at + z * o.stride + (low ? o.low : 0) + (int64_t)r * o.pitch + c) = v;
}

// What a half leaves of v.
__device__ __forceinline__ v4f rest_of(const v4f& v)
{
    v4f r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = v[i] - (float)(_Float16)v[i];
    return r;
}

// The tile at (m0, n0) of a rows x cols matrix to `o`, or with Turn its transpose; value() as in Tile::out.
template <bool Turn, bool Full, class Tl, class Value>
__device__ __forceinline__ void put_tile(Tl& t, char* lds, const Plane& o, int64_t z, uint32_t rows, uint32_t cols, uint32_t m0,
                                         uint32_t n0, const Value& value)
{
    auto at = [&](uint32_t r, uint32_t c, const v4f& v) -> v4f { return value(m0 + r, n0 + c, v); };
    auto store = [&](bool low) {
        return [&, low](uint32_t r, uint32_t c, const v8h& v) {
            put8(o, z, Turn ? cols : rows, Turn ? rows : cols, (Turn ? n0 : m0) + r, (Turn ? m0 : n0) + c, v, low);
        };
    };
    t.template out<_Float16, Turn>(lds, at, store(false));
    if (Full && o.low) t.template out<_Float16, Turn>(lds, [&](uint32_t r, uint32_t c, const v4f& v) { return rest_of(rounded(at(r, c, v))); }, store(true));
}

__device__ __forceinline__ Rows rows_of(const Plane& o, int64_t z, uint32_t rows, bool low = false)
{
    return {o.at + z * o.stride + (low ? o.low : 0), nullptr, rows, (uint32_t)o.pitch * 2};
}

// Operands of the terms of a product: with pairs of halves the small ones first.
template <bool Full, class Tl>
__device__ __forceinline__ void take(Tl& t, int term, const Plane& a, const Plane& b, int64_t z, uint32_t ra, uint32_t rb, uint32_t m0, uint32_t n0)
{
    t.take(rows_of(a, z, ra, Full && term == 0), rows_of(b, z, rb, Full && term == 1), m0, n0);
}

template <class Tl>
constexpr int lds_of()
{
    return Tl::kLds + Tl::kWaves * Tl::template out_bytes<_Float16>();
}

// A product of two symmetric matrices that commute, A B^T = A B: symmetric too.  out = p2 A B + p1 B + p0 I, all with the
// scales of their planes in the factors; p1 = p0 = 0 for a plain product.
struct Symmetric {
    Plane a, b, out;
    float p2, p1, p0;
};

// One or two of them of the same size.  Tiles on and below the diagonal are computed and mirrored: half the operations, and a
// second way out through LDS.  Bound by the matrix cores and by how the tiles meet 256 CUs.  m = 4096 in 253 tiles: pairs of
// halves, three products each, 204 us (2.1e11 operations, 1.0 PFLOP/s), 214 with the polynomial, 401 for two; G over n = 25088
// 1132 us (1.1), in halves 368 us.  Four of m = 1500 in 144 tiles, pairs, 83 and 93 to 97 us (4.1e10, 0.5), two 143; G over n =
// 6000 260 us (0.6).  Six of m = 256, pairs, 8 and 9.7 us, G over n = 2304 30 us.
template <class Tl, bool Full, bool Poly>
__global__ __launch_bounds__(Tl::kThreads) void k_symmetric(Symmetric first, Symmetric second, uint32_t m, uint32_t tiles, uint32_t each,
                                                            uint32_t total)
{
    constexpr int B = Tl::kM;
    __shared__ __align__(1024) char lds[lds_of<Tl>()];
    struct Place {
        bool second;
        int64_t z;
        uint32_t m0, n0;
    };
    auto place = [&](uint32_t tile) -> Place {
        uint32_t w = xcd_run(tile, total), i, j;
        const bool other = w >= each;
        if (other) w -= each;
        tile_of_triangle(w % tiles, i, j);
        return {other, w / tiles, i * B, j * B};
    };
    Tl t;
    t.template run<Full ? 3 : 1>(
        total, (uint32_t)first.a.pitch * 2, lds,
        [&](uint32_t tile, int term) {
            const Place at = place(tile);
            const Symmetric& p = at.second ? second : first;
            take<Full>(t, term, p.a, p.b, at.z, m, m, at.m0, at.n0);
        },
        [&](uint32_t tile) {
            const Place at = place(tile);
            const Symmetric& p = at.second ? second : first;
            const Plane g = p.b;
            const float p2 = p.p2, p1 = p.p1, p0 = p.p0;
            if (Poly) {  // in place: G is read once, and a tile off the diagonal goes out twice
                t.become([&](uint32_t r, uint32_t c, const v4f& v) -> v4f {
                    r += at.m0;
                    c += at.n0;
                    v4f w = {0.0f, 0.0f, 0.0f, 0.0f};
                    if (r < m && c < (uint32_t)g.pitch) {
                        const _Float16* q = g.at + at.z * g.stride + (int64_t)r * g.pitch + c;
                        const v4h h = *(const v4h*)q;
                        v4h l = {0, 0, 0, 0};
                        if (Full) l = *(const v4h*)(q + g.low);
#pragma unroll
                        for (int k = 0; k < 4; ++k) w[k] = fmaf(p2, v[k], fmaf(p1, (float)h[k] + (float)l[k], r == c + k ? p0 : 0.0f));
                    }
                    return w;
                });
            }
            auto value = [&](uint32_t, uint32_t, const v4f& v) -> v4f { return Poly ? v : v * p2; };
            put_tile<false, Full>(t, lds + Tl::kLds, p.out, at.z, m, m, at.m0, at.n0, value);
            if (at.m0 != at.n0) put_tile<true, Full>(t, lds + Tl::kLds, p.out, at.z, m, m, at.m0, at.n0, value);
        });
}

// What the last product goes to: the result, or weights that move by it.
struct Result {
    void* out;
    bool tall;          // it is X transposed
    bool update;
    float keep, gain;   // out = keep * out + gain * X
    int64_t ld, stride, rows, cols;
};

template <class T>
__device__ __forceinline__ void finish4(const Result& o, int64_t z, int64_t r, int64_t c, const v4f& v)
{
    if (r >= o.rows || c >= o.cols) return;
    T* p = (T*)o.out + z * o.stride + r * o.ld + c;
    typedef T t4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if (c + 4 <= o.cols) {
        t4 w;
        if (o.update) {
            const t4 old = *(const t4*)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (T)fmaf(o.gain, v[i], o.keep * (float)old[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (T)v[i];
        }
        *(t4*)p = w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < o.cols) p[i] = (T)(o.update ? fmaf(o.gain, v[i], o.keep * (float)p[i]) : v[i]);
    }
}

template <class T>
__device__ __forceinline__ void finish1(const Result& o, int64_t z, int64_t r, int64_t c, float v)
{
    if (r >= o.rows || c >= o.cols) return;
    T* p = (T*)o.out + z * o.stride + r * o.ld + c;
    *p = (T)(o.update ? fmaf(o.gain, v, o.keep * (float)*p) : v);
}

// X' = Q X: X' and its transpose, or with Last the result, of element type T.  Bound by the matrix cores: m = 4096, n = 25088 in
// halves 736 + 36 us in two launches, 1.09 PFLOP/s (a large library product of the type reaches 1.35), in pairs of halves 1873 +
// 89 us, 1.29; four of 1500 x 6000 in pairs 375 + 72 us (X) and 336 + 73 us (weights), 0.72 and 0.79.
template <class Tl, bool Full, bool Last, class T>
__global__ __launch_bounds__(Tl::kThreads) void k_apply(Plane pm, Plane xt, Plane x2, Plane xt2, uint32_t m, uint32_t n, uint32_t tm, uint32_t tn,
                                                        uint32_t total, uint32_t from, float back, Result o)
{
    constexpr int B = Tl::kM;
    __shared__ __align__(1024) char lds[lds_of<Tl>()];
    struct Place {
        int64_t z;
        uint32_t m0, n0;
    };
    auto place = [&](uint32_t tile) -> Place {
        const uint32_t w = xcd_run(tile, total);
        uint32_t i, j;
        tile_of(w % (tm * tn), tm, tn, i, j);
        return {w / (tm * tn), i * B, from + j * B};
    };
    Tl t;
    t.template run<Full ? 3 : 1>(
        total, (uint32_t)pm.pitch * 2, lds,
        [&](uint32_t tile, int term) {
            const Place at = place(tile);
            take<Full>(t, term, pm, xt, at.z, m, n, at.m0, at.n0);
        },
        [&](uint32_t tile) {
            const Place at = place(tile);
            auto value = [&](uint32_t, uint32_t, const v4f& v) -> v4f { return v * back; };
            if (!Last) {
                put_tile<false, Full>(t, lds + Tl::kLds, x2, at.z, m, n, at.m0, at.n0, value);
                put_tile<true, Full>(t, lds + Tl::kLds, xt2, at.z, m, n, at.m0, at.n0, value);
            } else if (o.tall) {
                t.each([&](uint32_t r, uint32_t c, const v4f& v) {
                    finish4<T>(o, at.z, at.n0 + c + (threadIdx.x & 3), (at.m0 + r) & ~3u, turned(v * back));
                });
            } else {
                t.each([&](uint32_t r, uint32_t c, const v4f& v) { finish4<T>(o, at.z, at.m0 + r, at.n0 + c, v * back); });
            }
        });
}

// ---- a matrix in one block ----
//
// With m <= 64 and X^T in LDS one block does everything, all steps in one launch; the launches of the kernels above, 2 and 17
// for 5 steps, take longer than their work at this size, 5 us and more each.  Bound by the chain of reads, products and
// barriers of a step, and a matrix has one CU: 64 x 576 in 32 bits, momentum and weights with it, 61 us, of which 7 to 9 a step
// and the rest the start and the end.  X^T is kept by rows of 64 (m padded with zeros), so that
//   G = X X^T  reads its operands down the columns, with the transposing read of LDS,
//   X <- P X   reads rows and writes them in place: a row of X^T depends on that row alone, and each wave has its own.
// G and P, being small, are pairs of halves whatever X is.  16-byte piece c of row r is kept at place c ^ (r % 8).
constexpr int kOneWaves = 8;

struct One {
    const void* x;
    int64_t ldx, x_stride;
    float* momentum;
    float mu;
    bool nesterov;
    int rows, cols, m, n;
    int steps;
    float a, b, c, eps, sp;
    int out_type;
    Result o;
};

__device__ __forceinline__ v4h highs(const v4f& v) { return v4h{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]}; }

__device__ __forceinline__ v4f mul16(const v8h& a, const v8h& b, const v4f& c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

template <bool Full>
__device__ __forceinline__ v4f mul16(const v8h (&a)[2], const v8h (&b)[2], v4f c)
{
    if (Full) {
        c = mul16(a[1], b[0], c);
        c = mul16(a[0], b[1], c);
    }
    return mul16(a[0], b[0], c);
}

// a pair of halves times a pair, or with Full false times the high half alone
template <bool Full>
__device__ __forceinline__ v4f mul16_pair(const v8h (&a)[2], const v8h (&b)[2], v4f c)
{
    c = mul16(a[1], b[0], c);
    if (Full) c = mul16(a[0], b[1], c);
    return mul16(a[0], b[0], c);
}

// Cap: rows of X^T that LDS has room for
template <class T, int Cap, bool Full>
__global__ __launch_bounds__(64 * kOneWaves) void k_one(One p)
{
    constexpr int kPlanes = Full ? 2 : 1, kRow = kOneSide * 2, kPlane = Cap * kRow;
    __shared__ __align__(16) char xt[kPlanes * kPlane];
    __shared__ __align__(16) char gp[2 * kOneSide * kRow];  // G, then P, as pairs of halves
    typedef short v4s __attribute__((ext_vector_type(4)));
    auto down = [](char* at) {  // four rows of a column
        return __builtin_bit_cast(v4h, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)at));
    };
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int64_t z = blockIdx.x;
    const int np = (p.n + 31) & ~31;
    auto piece = [](int row, int c) { return row * kRow + ((c ^ (row & 7)) << 4); };  // where 16 bytes of a row are

    // Momentum, norm and X^T: four neighbours of a row of X^T at a time, lanes along the rows in memory, all in registers until
    // the norm is known.  Loads go out in batches: one after the other each would take a memory's latency.
    constexpr int kGroups = Cap / 32, kBatch = 6;  // of 4 elements a lane
    double* sums = (double*)gp;
    float top = 0.0f;
    const bool tall = p.o.tall;
    const T* x = (const T*)p.x + z * p.x_stride;
    float* momentum = p.momentum ? p.momentum + z * p.rows * p.cols : nullptr;
    // Group g has row row0 + 32 g of X^T (tall: of the matrix; else its column), elements m0 to m0 + 3.
    const int row0 = tall ? wave * 4 + q : wave / 4 * 16 + r, m0 = tall ? r * 4 : wave % 4 * 16 + q * 4;
    int xs[4], ms[4];  // element offsets; an element that there is not is read at another's place
    bool in[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        in[i] = m0 + i < p.m;
        const int m = in[i] ? m0 + i : p.m - 1;
        xs[i] = tall ? m : m * (int)p.ldx;
        ms[i] = tall ? m : m * p.cols;
    }
    v4f u[kGroups];
#pragma unroll
    for (int b = 0; b < kGroups; b += kBatch) {
        T new_x[kBatch][4];
        v4f old[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch && b + k < kGroups; ++k) {
            int row = row0 + 32 * (b + k);
            row = row < p.n ? row : p.n - 1;
            const int xr = tall ? row * (int)p.ldx : row, mr = tall ? row * p.cols : row;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                new_x[k][i] = x[xr + xs[i]];
                if (momentum) old[k][i] = momentum[mr + ms[i]];
            }
        }
#pragma unroll
        for (int k = 0; k < kBatch && b + k < kGroups; ++k) {
            const int row = row0 + 32 * (b + k);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool there = in[i] && row < p.n;
                float v = (float)new_x[k][i];
                if (momentum) {
                    const float moved = fmaf(p.mu, old[k][i], v);
                    if (there) momentum[(tall ? row * p.cols : row) + ms[i]] = moved;
                    v = p.nesterov ? fmaf(p.mu, moved, v) : moved;
                }
                v = there ? v : 0.0f;
                u[b + k][i] = v;
                top = fmaxf(top, fabsf(v));
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    // The norm from elements over a power of two near the largest, which keeps their squares in fp32's range.
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
    if (lane == 0) ((float*)sums)[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kOneWaves; ++w) top = fmaxf(top, ((float*)sums)[w]);
    __syncthreads();
    int e = 0;
    (void)frexpf(top, &e);
    const float down_to = top > 0.0f && top < INFINITY ? ldexpf(1.0f, e > 126 ? -126 : (e < -126 ? 126 : -e)) : 1.0f;
    v4f squares = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        u[g] *= down_to;
#pragma unroll
        for (int i = 0; i < 4; ++i) squares[i] = fmaf(u[g][i], u[g][i], squares[i]);
    }
    double sum = (double)squares[0] + (double)squares[1] + (double)squares[2] + (double)squares[3];
    sum = block_sum(sum, sums);
    if (threadIdx.x == 0) sums[kOneWaves] = (double)kScaleX / (sqrt(sum) + (double)p.eps * (double)down_to);
    __syncthreads();
    // zeros alone may ask for more than the largest number; a NaN stays one
    const float inverse = sums[kOneWaves] > 3e38 ? 3e38f : (float)sums[kOneWaves];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const int row = row0 + 32 * g;
        if (row >= np) continue;
        v4f v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = u[g][i] * inverse;
        v = rounded(v);
        char* at = xt + piece(row, m0 >> 3) + (m0 & 4) * 2;
        *(v4h*)at = highs(v);
        if (Full) *(v4h*)(at + kPlane) = highs(rest_of(v));
    }
    __syncthreads();

    for (int step = 0; step < p.steps; ++step) {
        // G: a wave has one of the six tiles below the diagonal, or two of the four on it, over all of X's length
        v4f v2[2] = {};
        const bool on = wave >= 6;
        const int ti = on ? 2 * (wave - 6) : (wave < 1 ? 1 : wave < 3 ? 2 : 3), tj = on ? ti + 1 : (wave < 1 ? 0 : wave < 3 ? wave - 1 : wave - 3);
        auto operands = [&](int k, v8h (&f)[2][2]) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int h = 0; h < kPlanes; ++h) {
                    const int row = k + 8 * q + (r >> 2), e = 16 * (i ? tj : ti) + 4 * (r & 3);
                    char* at = xt + h * kPlane + (e & 4) * 2;
                    const v4h lo = down(at + piece(row, e >> 3)), hi = down(at + piece(row + 4, e >> 3));
                    f[i][h] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                }
        };
        auto products = [&](const v8h (&f)[2][2]) {
            if (on) {
                v2[0] = mul16<Full>(f[0], f[0], v2[0]);
                v2[1] = mul16<Full>(f[1], f[1], v2[1]);
            } else {
                v2[0] = mul16<Full>(f[0], f[1], v2[0]);
            }
        };
        v8h fa[2][2], fb[2][2];  // the next operands are read while these are multiplied
        operands(0, fa);
        for (int k = 0; k < np; k += 64) {
            if (k + 32 < np) operands(k + 32, fb);
            products(fa);
            if (k + 64 < np) operands(k + 64, fa);
            if (k + 32 < np) products(fb);
        }
        // four neighbours of a row of G or P, from element (row, col) on
        auto store4 = [&](int row, int col, v4f v) {
            v = rounded(v);
            char* at = gp + piece(row, col >> 3) + (col & 4) * 2;
            *(v4h*)at = highs(v);
            *(v4h*)(at + kOneSide * kRow) = highs(rest_of(v));
        };
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if (t && !on) break;
            const int i = t ? tj : ti, j = on ? i : tj;  // v[e] is element (16 i + 4 q + e, 16 j + r): by symmetry a row's neighbours
            const v4f v = v2[t] * (1.0f / kScaleX);
            store4(16 * j + r, 16 * i + 4 * q, v);
            if (i != j) store4(16 * i + 4 * q + (r & 3), 16 * j + (r & ~3), turned(v));
        }
        __syncthreads();
        // P: a wave has two neighbouring tiles of a row of them
        v4f pv[2] = {};
        const int pi = wave >> 1, pj = 2 * (wave & 1);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            v8h f[3][2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < 3; ++t)
                    f[t][h] = *(const v8h*)(gp + h * kOneSide * kRow + piece(16 * (t == 0 ? pi : pj + t - 1) + r, 4 * k + q));
#pragma unroll
            for (int t = 0; t < 2; ++t) pv[t] = mul16<true>(f[0], f[1 + t], pv[t]);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int row = 16 * (pj + t) + r, col = 16 * pi + 4 * q;
            const char* at = gp + piece(row, col >> 3) + (col & 4) * 2;
            const v4h gh = *(const v4h*)at, gl = *(const v4h*)(at + kOneSide * kRow);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                pv[t][e] = p.sp * fmaf(p.c / (kScaleX * kScaleX), pv[t][e], fmaf(p.b / kScaleX, (float)gh[e] + (float)gl[e], col + e == row ? p.a : 0.0f));
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < 2; ++t) store4(16 * (pj + t) + r, 16 * pi + 4 * q, pv[t]);
        __syncthreads();
        // X <- P X
        v8h pf[4][2][2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) pf[i][k][h] = *(const v8h*)(gp + h * kOneSide * kRow + piece(16 * i + r, 4 * k + q));
        const bool last = step + 1 == p.steps;
        auto rows_at = [&](int n0, v8h (&f)[2][2]) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int h = 0; h < kPlanes; ++h) f[k][h] = *(const v8h*)(xt + h * kPlane + piece(n0 + r, 4 * k + q));
        };
        v8h ahead[2][2];
        if (wave * 16 < np) rows_at(wave * 16, ahead);
        for (int n0 = wave * 16; n0 < np; n0 += kOneWaves * 16) {
            v8h f[2][2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int h = 0; h < kPlanes; ++h) f[k][h] = ahead[k][h];
            if (n0 + kOneWaves * 16 < np) rows_at(n0 + kOneWaves * 16, ahead);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
                v = mul16_pair<Full>(pf[i][0], f[0], v);
                v = mul16_pair<Full>(pf[i][1], f[1], v);
                if (!last) {
                    v = rounded(v * (1.0f / p.sp));
                    char* at = xt + piece(n0 + r, 2 * i + (q >> 1)) + (q & 1) * 8;
                    *(v4h*)at = highs(v);
                    if (Full) *(v4h*)(at + kPlane) = highs(rest_of(v));
                    continue;
                }
                v *= 1.0f / (kScaleX * p.sp);
                const int row = n0 + r, col = 16 * i + 4 * q;  // of X^T
                if (tall) {
                    if (p.out_type == kGradF32)
                        finish4<float>(p.o, z, row, col, v);
                    else if (p.out_type == kGradF16)
                        finish4<_Float16>(p.o, z, row, col, v);
                    else
                        finish4<__bf16>(p.o, z, row, col, v);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (p.out_type == kGradF32)
                            finish1<float>(p.o, z, col + e, row, v[e]);
                        else if (p.out_type == kGradF16)
                            finish1<_Float16>(p.o, z, col + e, row, v[e]);
                        else
                            finish1<__bf16>(p.o, z, col + e, row, v[e]);
                    }
                }
            }
        }
        __syncthreads();
    }
}

// The launch of k_one.  Where it has room it is faster at every batch; us, 64 x 576 here / 65 x 576 there, batches
// of 3, 64 and 1024: 52 53 233 / 129 199 985, in halves 43 44 174 / 84 118 555; and 64 x 128 20 21 80 / 65 x 128 107 112 591.
template <bool Full>
void one_block(const OrthoCall& q, float sp, hipStream_t s)
{
    const int64_t m = q.rows < q.cols ? q.rows : q.cols, n = q.rows < q.cols ? q.cols : q.rows;
    constexpr int kMost = Full ? kOnePairs : kOneHalves, kFew = 128;  // less LDS for little ones
    const Result o = {q.out, q.rows > q.cols, q.update, q.keep, q.gain, q.ldo, q.out_stride, q.rows, q.cols};
    const One p = {q.x, q.ldx, q.x_stride, q.momentum, q.mu, q.nesterov, (int)q.rows, (int)q.cols, (int)m, (int)n,
                   q.steps, q.a, q.b, q.c, q.eps, sp, q.out_type, o};
    by_element(q.x_type, [&](auto type) {
        typedef typename decltype(type)::T T;
        if (n <= kFew)
            k_one<T, kFew, Full><<<(uint32_t)q.batch, 64 * kOneWaves, 0, s>>>(p);
        else
            k_one<T, kMost, Full><<<(uint32_t)q.batch, 64 * kOneWaves, 0, s>>>(p);
    });
}

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// The workspace of a batch: partial sums, then X, X^T and both once more, and the symmetric matrices, of every matrix.
constexpr int kSmall = 7;  // G, G', P, P', T, Q, Q'
struct Layout {
    int64_t m, n, mp, np;
    OrthoGroups groups;
    int planes, planes2;  // of X and the symmetric matrices; of the second X, which takes turns with the first
    int parts;
    size_t part_bytes, total;
    explicit Layout(const OrthoCall& q)
    {
        m = q.rows < q.cols ? q.rows : q.cols;
        n = q.rows < q.cols ? q.cols : q.rows;
        mp = up(m, 64);
        np = up(n, 64);
        groups = ortho_groups(q.batch, m, n, q.steps, q.paired);
        planes = q.paired > 0 ? 2 : 1;
        planes2 = q.paired > groups.paired ? 2 : 1;  // one group of steps in pairs leaves an X for halves, or the result
        const int64_t want = (q.rows * q.cols + kNormRow - 1) / kNormRow;
        parts = (int)(want < 1024 ? want : 1024);
        part_bytes = (size_t)up((int64_t)q.batch * parts * (int64_t)sizeof(double), 256);
        const int64_t halves = plane(m, np, planes) + plane(n, mp, planes) + plane(m, np, planes2) + plane(n, mp, planes2) + kSmall * plane(m, mp, planes);
        total = part_bytes + (size_t)q.batch * halves * sizeof(_Float16);
    }
    static int64_t plane(int64_t height, int64_t pitch, int count) { return up(height * pitch * count, 128); }
};

template <class Tl>
struct Shape {
    typedef Tl Is;
};

// f(a tile's type) for the tile of kTileCosts[pick]
template <class F>
void by_tile(int pick, const F& f)
{
    if (pick == 0)
        f(Shape<Tile<HalfCore, 256, 256, 2, 2, 2>>());
    else if (pick == 1)
        f(Shape<Tile<HalfCore, 192, 192, 2, 2, 3>>());
    else if (pick == 2)
        f(Shape<Tile<HalfCore, 128, 128, 2, 2, 2>>());
    else
        f(Shape<Tile<HalfCore, 64, 64, 2, 2, 4>>());
}

void orthogonalize(const OrthoCall& q, char* ws, hipStream_t s)
{
    // Scales: the largest powers of two that leave room for the largest element of P, of Q's products of it and of T = P G.
    const float top = ortho_growth(q.a, q.b, q.c);
    auto scale = [](float bound) {
        int e = 0;
        (void)frexpf(32768.0f / fmaxf(bound, 1.0f), &e);
        return ldexpf(1.0f, e - 1 > -10 ? e - 1 : -10);
    };
    const float sx = kScaleX, sp = scale(top), st = scale(2.25f * top);

    if (ortho_one_block(q.rows, q.cols, q.ldx, q.paired > 0)) return q.paired > 0 ? one_block<true>(q, sp, s) : one_block<false>(q, sp, s);

    const Layout l(q);
    const uint32_t batch = (uint32_t)q.batch;
    const int64_t m = l.m, n = l.n;
    const bool tall = q.rows > q.cols;
    _Float16* at = (_Float16*)(ws + l.part_bytes);
    auto plane = [&](int64_t height, int64_t pitch, int count) {
        const int64_t each = l.plane(height, pitch, count);
        Plane p = {at, pitch, count == 2 ? height * pitch : 0, each};
        at += each * q.batch;
        return p;
    };
    Plane x[2], xt[2], g[2], pm[2], qm[2];
    for (int i = 0; i < 2; ++i) {
        x[i] = plane(m, l.np, i ? l.planes2 : l.planes);
        xt[i] = plane(n, l.mp, i ? l.planes2 : l.planes);
        g[i] = plane(m, l.mp, l.planes);
        pm[i] = plane(m, l.mp, l.planes);
        qm[i] = plane(m, l.mp, l.planes);
    }
    const Plane tm = plane(m, l.mp, l.planes);

    by_element(q.x_type, [&](auto type) {
        typedef typename decltype(type)::T T;
        const Start<T> p = {(const T*)q.x, q.ldx, q.x_stride, q.momentum, q.mu, q.nesterov, q.rows, q.cols, (double*)ws, l.parts};
        k_norm<T><<<dim3((uint32_t)l.parts, batch), kNormBlock, 0, s>>>(p);
        const dim3 grid((uint32_t)((q.cols + 63) / 64), (uint32_t)((q.rows + 63) / 64), batch);
        if (q.paired > 0)
            k_start<T, true><<<grid, 256, 0, s>>>(p, q.eps, tall ? xt[0] : x[0], tall ? x[0] : xt[0]);
        else
            k_start<T, false><<<grid, 256, 0, s>>>(p, q.eps, tall ? xt[0] : x[0], tall ? x[0] : xt[0]);
    });

    auto product = [](const Plane& a, float sa, const Plane& b, float sb, const Plane& o, float so) -> Symmetric {
        return {a, b, o, so / (sa * sb), 0.0f, 0.0f};
    };
    auto poly = [&](const Plane& gm, const Plane& o) -> Symmetric { return {gm, gm, o, q.c * sp / (sx * sx), q.b * sp / sx, q.a * sp}; };
    const std::true_type with_poly;
    const std::false_type plain;
    // `steps` steps from x[from], in pairs of halves or halves; what comes out is the result, or an X with or without low halves
    auto pass = [&](auto pairs, int steps, int from, bool last, bool low) {
        constexpr bool Full = decltype(pairs)::value;
        const int64_t segments = Full ? 3 : 1;
        auto symmetric = [&](auto poly, int jobs, const Symmetric& a, const Symmetric& b) {
            const int pick = best_triangle(m, (int64_t)q.batch * jobs, a.a.pitch * 2 / kLine * segments);
            by_tile(pick, [&](auto shape) {
                typedef typename decltype(shape)::Is Tl;
                const uint32_t tri = (uint32_t)triangle_tiles(m, Tl::kM), each = tri * batch;
                k_symmetric<Tl, Full, decltype(poly)::value>
                    <<<tile_blocks(pick, each * jobs), Tl::kThreads, 0, s>>>(a, b, (uint32_t)m, tri, each, each * jobs);
            });
        };
        auto apply_part = [&](int pick, int64_t first, int64_t columns, const Plane& by, float sb) {
            Plane to = x[1 - from], to_t = xt[1 - from];
            if (!low) to.low = to_t.low = 0;
            by_tile(pick, [&](auto shape) {
                typedef typename decltype(shape)::Is Tl;
                const uint32_t ti = (uint32_t)((m + Tl::kM - 1) / Tl::kM), tj = (uint32_t)((columns + Tl::kN - 1) / Tl::kN);
                const Result o = {q.out, tall, q.update, q.keep, q.gain, q.ldo, q.out_stride, q.rows, q.cols};
                auto go = [&](auto kernel, float back) {
                    const uint32_t total = ti * tj * batch;
                    kernel<<<tile_blocks(pick, total), Tl::kThreads, 0, s>>>(by, xt[from], to, to_t, (uint32_t)m, (uint32_t)n, ti, tj, total,
                                                                            (uint32_t)first, back, o);
                };
                if (!last)
                    go(k_apply<Tl, Full, false, float>, 1.0f / sb);
                else if (q.out_type == kGradF32)
                    go(k_apply<Tl, Full, true, float>, 1.0f / (sx * sb));
                else if (q.out_type == kGradF16)
                    go(k_apply<Tl, Full, true, _Float16>, 1.0f / (sx * sb));
                else
                    go(k_apply<Tl, Full, true, __bf16>, 1.0f / (sx * sb));
            });
        };
        const Symmetric gram = product(x[from], sx, x[from], sx, g[0], sx);
        symmetric(plain, 1, gram, gram);
        symmetric(with_poly, 1, poly(g[0], pm[0]), gram);
        Plane by = pm[0];
        float sb = sp, grown = top;
        for (int k = 1; k < steps; ++k) {
            const int now = k & 1, was = 1 - now;
            // T = P G (with it the Q of the step before, which waits for the same P), G = T P, P of it
            const Symmetric t = product(pm[was], sp, g[was], sx, tm, st);
            if (k > 1) {
                const Symmetric grow = product(pm[was], sp, by, sb, qm[was], scale(grown * top));
                symmetric(plain, 2, t, grow);
                by = qm[was], sb = scale(grown *= top);
            } else {
                symmetric(plain, 1, t, t);
            }
            const Symmetric next = product(tm, st, pm[was], sp, g[now], sx);
            symmetric(plain, 1, next, next);
            symmetric(with_poly, 1, poly(g[now], pm[now]), next);
            if (k + 1 == steps) {
                const Symmetric grow = product(pm[now], sp, by, sb, qm[now], scale(grown * top));
                symmetric(plain, 1, grow, grow);
                by = qm[now], sb = scale(grown *= top);
            }
        }
        const TilePlan plan = plan_tiles(m, n, q.batch, l.mp * 2 / kLine * segments);
        apply_part(plan.pick, 0, plan.columns, by, sb);
        if (plan.columns < n) apply_part(plan.rest_pick, plan.columns, n - plan.columns, by, sb);
    };
    for (int done = 0, from = 0; done < q.steps; from = 1 - from) {
        const bool pairs = done < q.paired;
        const int left = (pairs ? q.paired : q.steps) - done, most = pairs ? l.groups.paired : l.groups.halves;
        const int steps = left < most ? left : most;
        done += steps;
        if (pairs)
            pass(std::true_type(), steps, from, done == q.steps, done < q.paired);
        else
            pass(std::false_type(), steps, from, done == q.steps, false);
    }
}

}  // namespace

size_t ortho_scratch(const OrthoCall& q) { return Layout(q).total; }

void launch_orthogonalize(const OrthoCall& q, char* scratch, hipStream_t s) { orthogonalize(q, scratch, s); }

}  // namespace sidco
