// The orthogonalised update: momentum, Newton-Schulz products, weights.
//
// X_0 = u / (|u| + eps), transposed if u is tall, so that X is m x n with m <= n; then `steps` times
//   G = X X^T,  P = aI + bG + cG^2,  X <- P X,
// which moves every singular value s to as + bs^3 + cs^5.  All three products are of the form A B^T over the rows of what is
// stored (G and P are symmetric, and X is stored both as it is and transposed), G and P are computed for tiles on and below
// the diagonal and mirrored.  With a in P's diagonal the last product needs no second operand in its epilogue, and the largest
// term of the sum is not rounded twice.
//
// Operands are halves; sums, the norm and the update are fp32 or more.  Singular values stay below 4, so X and G are kept
// times 2^14 and P times a power of two that follows from a, b, c: entries far below the largest one keep their 11 bits.  Of
// X's relative error of 2^-12 an element, about 1.5e-3 (2-norm) reaches the result, less than a result in bf16 loses; halves
// are used where it has 16 bits.  For a result in 32 bits each operand is a pair of halves, the second one what the first
// leaves, 22 bits together, and a product is three: high high + low high + high low.
#include "sidco_dense.h"
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

// u from the gradient and the momentum that k_norm has moved
template <class T>
__device__ __forceinline__ float update_of(const Start<T>& p, int64_t z, int64_t r, int64_t c)
{
    const float g = (float)p.x[z * p.stride + r * p.ld + c];
    if (!p.momentum) return g;
    const float m = p.momentum[(z * p.rows + r) * p.cols + c];
    return p.nesterov ? fmaf(p.mu, m, g) : m;
}

template <class T>
__global__ __launch_bounds__(kNormBlock) void k_norm(Start<T> p)
{
    __shared__ double lds[kNormBlock / 64];
    const int64_t z = blockIdx.y;
    double sum = 0.0;
    const int64_t n = p.rows * p.cols;
    for (int64_t i = (int64_t)blockIdx.x * kNormBlock + threadIdx.x; i < n; i += (int64_t)gridDim.x * kNormBlock) {
        const int64_t r = i / p.cols, c = i - r * p.cols;
        float u;
        if (p.momentum) {
            float* m = p.momentum + z * n + i;
            const float g = (float)p.x[z * p.stride + r * p.ld + c], moved = fmaf(p.mu, *m, g);
            *m = moved;
            u = p.nesterov ? fmaf(p.mu, moved, g) : moved;
        } else {
            u = (float)p.x[z * p.stride + r * p.ld + c];
        }
        sum += (double)u * (double)u;
    }
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) p.part[z * p.parts + blockIdx.x] = sum;
}

// Where X and X^T of one matrix after the other lie: rows of `pitch` halves, the low halves `low` after the high ones.
struct Plane {
    _Float16* at;
    int64_t pitch, low, stride;
};

template <bool Full>
__device__ __forceinline__ void put(const Plane& o, int64_t z, int64_t r, int64_t c, float v)
{
    _Float16* p = o.at + z * o.stride + r * o.pitch + c;
    const _Float16 h = (_Float16)v;
    *p = h;
    if (Full) p[o.low] = (_Float16)(v - (float)h);
}

// 64 x 64 elements a block: rows go to `natural`, and through LDS to `turned`, the padding of both as zeros.
template <class T, bool Full>
__global__ __launch_bounds__(256) void k_start(Start<T> p, float eps, Plane natural, Plane turned)
{
    __shared__ float tile[64][65];
    __shared__ double lds[4];
    __shared__ double inverse;
    const int64_t z = blockIdx.z;
    double sum = 0.0;
    for (int i = threadIdx.x; i < p.parts; i += 256) sum += p.part[z * p.parts + i];
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) inverse = (double)kScaleX / (sqrt(sum) + (double)eps);
    __syncthreads();
    const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const double inv = inverse;
#pragma unroll 4
    for (int k = 0; k < 16; ++k) {
        const int64_t r = r0 + k * 4 + wave, c = c0 + lane;
        float v = 0.0f;
        if (r < p.rows && c < p.cols) v = (float)((double)update_of(p, z, r, c) * inv);
        tile[k * 4 + wave][lane] = v;
        if (r < p.rows) put<Full>(natural, z, r, c, v);
    }
    __syncthreads();
#pragma unroll 4
    for (int k = 0; k < 16; ++k) {
        const int64_t r = c0 + k * 4 + wave, c = r0 + lane;
        if (r < p.cols) put<Full>(turned, z, r, c, tile[lane][k * 4 + wave]);
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
    if (Full) t.template out<_Float16, Turn>(lds, [&](uint32_t r, uint32_t c, const v4f& v) { return rest_of(at(r, c, v)); }, store(true));
}

__device__ __forceinline__ Rows rows_of(const Plane& o, int64_t z, uint32_t rows, bool low = false)
{
    return {o.at + z * o.stride + (low ? o.low : 0), nullptr, rows, (uint32_t)o.pitch * 2};
}

template <class Tl, bool Full>
__device__ __forceinline__ void products(Tl& t, const Plane& a, const Plane& b, int64_t z, uint32_t ra, uint32_t rb, uint32_t m0, uint32_t n0,
                                         char* lds)
{
    t.clear();
    if (Full) {  // the small ones first
        t.run(rows_of(a, z, ra, true), rows_of(b, z, rb), m0, n0, lds);
        t.run(rows_of(a, z, ra), rows_of(b, z, rb, true), m0, n0, lds);
    }
    t.run(rows_of(a, z, ra), rows_of(b, z, rb), m0, n0, lds);
}

struct Poly {
    float a, b, c, scale;  // of P; scale: what P is kept times
};

// G = X X^T, or with Second P = aI + bG + cG^2; `x` is X or G, `out` G or P, both m x m.
template <class Tl, int B, bool Full, bool Second>
__global__ __launch_bounds__(Tl::kThreads) void k_symmetric(Plane x, Plane out, uint32_t m, uint32_t tiles, Poly p)
{
    __shared__ __align__(1024) char lds[Tl::kLds];
    const uint32_t w = xcd_run(blockIdx.x, gridDim.x);
    const int64_t z = w / tiles;
    uint32_t i, j;
    tile_of_triangle(w % tiles, i, j);
    Tl t;
    products<Tl, Full>(t, x, x, z, m, m, i * B, j * B, lds);
    __syncthreads();
    auto value = [&](uint32_t r, uint32_t c, const v4f& v) -> v4f {
        if (!Second) return v * (1.0f / kScaleX);
        v4f w = {0.0f, 0.0f, 0.0f, 0.0f};
        if (r < m && c < (uint32_t)x.pitch) {
            const _Float16* g = x.at + z * x.stride + (int64_t)r * x.pitch + c;
            const v4h h = *(const v4h*)g;
            v4h l = {0, 0, 0, 0};
            if (Full) l = *(const v4h*)(g + x.low);
            const float c2 = p.c * p.scale / (kScaleX * kScaleX), c1 = p.b * p.scale / kScaleX;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                w[k] = fmaf(c2, v[k], fmaf(c1, (float)h[k] + (float)l[k], r == c + k ? p.a * p.scale : 0.0f));
        }
        return w;
    };
    put_tile<false, Full>(t, lds, out, z, m, m, i * B, j * B, value);
    if (i != j) put_tile<true, Full>(t, lds, out, z, m, m, i * B, j * B, value);
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

// X' = P X: X' and its transpose, or with Last the result, of element type T.
template <class Tl, int B, bool Full, bool Last, class T>
__global__ __launch_bounds__(Tl::kThreads) void k_apply(Plane pm, Plane xt, Plane x2, Plane xt2, uint32_t m, uint32_t n, uint32_t tm, uint32_t tn,
                                                        float back, Result o)
{
    __shared__ __align__(1024) char lds[Tl::kLds];
    const uint32_t w = xcd_run(blockIdx.x, gridDim.x);
    const int64_t z = w / (tm * tn);
    uint32_t i, j;
    tile_of(w % (tm * tn), tm, tn, i, j);
    Tl t;
    products<Tl, Full>(t, pm, xt, z, m, n, i * B, j * B, lds);
    __syncthreads();
    auto value = [&](uint32_t, uint32_t, const v4f& v) -> v4f { return v * back; };
    if (!Last) {
        put_tile<false, Full>(t, lds, x2, z, m, n, i * B, j * B, value);
        put_tile<true, Full>(t, lds, xt2, z, m, n, i * B, j * B, value);
    } else if (o.tall) {
        t.each([&](uint32_t r, uint32_t c, const v4f& v) {
            finish4<T>(o, z, j * B + c + (threadIdx.x & 3), (i * B + r) & ~3u, Tl::turned(v * back));
        });
    } else {
        t.each([&](uint32_t r, uint32_t c, const v4f& v) { finish4<T>(o, z, i * B + r, j * B + c, v * back); });
    }
}

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// The workspace of a batch: partial sums, then X, X^T, both once more, G and P of every matrix.
struct Layout {
    int64_t m, n, mp, np;
    int planes, parts;
    size_t part_bytes, x, g, total;  // halves of one X (or X^T) and one G of a matrix, all planes of them
    Layout(int batch, int64_t rows, int64_t cols, bool full)
    {
        m = rows < cols ? rows : cols;
        n = rows < cols ? cols : rows;
        mp = up(m, 64);
        np = up(n, 64);
        planes = full ? 2 : 1;
        const int64_t want = (rows * cols + 16 * kNormBlock - 1) / (16 * kNormBlock);
        parts = (int)(want < 512 ? want : 512);
        part_bytes = (size_t)up((int64_t)batch * parts * (int64_t)sizeof(double), 256);
        x = (size_t)(m * np) * planes;
        g = (size_t)(m * mp) * planes;
        const size_t xt = (size_t)(n * mp) * planes;
        total = part_bytes + (size_t)batch * 2 * (2 * up((int64_t)x, 128) + 2 * up((int64_t)xt, 128) + 2 * up((int64_t)g, 128));
    }
};

template <class Tl, int B>
struct Square {
    typedef Tl Is;
    static constexpr int kSide = B;
};

template <bool Full>
void orthogonalize(const OrthoCall& q, char* ws, hipStream_t s)
{
    const Layout l(q.batch, q.rows, q.cols, Full);
    const uint32_t batch = (uint32_t)q.batch;
    const int64_t m = l.m, n = l.n;
    const bool tall = q.rows > q.cols;
    _Float16* at = (_Float16*)(ws + l.part_bytes);
    auto plane = [&](int64_t rows, int64_t pitch) {
        const int64_t each = up(rows * pitch * l.planes, 128);
        Plane p = {at, pitch, rows * pitch, each};
        at += each * q.batch;
        return p;
    };
    Plane x[2], xt[2];
    for (int i = 0; i < 2; ++i) x[i] = plane(m, l.np), xt[i] = plane(n, l.mp);
    const Plane g = plane(m, l.mp), pm = plane(m, l.mp);

    auto start = [&](auto type) {
        typedef typename decltype(type)::T T;
        const Start<T> p = {(const T*)q.x, q.ldx, q.x_stride, q.momentum, q.mu, q.nesterov, q.rows, q.cols, (double*)ws, l.parts};
        k_norm<T><<<dim3((uint32_t)l.parts, batch), kNormBlock, 0, s>>>(p);
        const dim3 grid((uint32_t)((q.cols + 63) / 64), (uint32_t)((q.rows + 63) / 64), batch);
        k_start<T, Full><<<grid, 256, 0, s>>>(p, q.eps, tall ? xt[0] : x[0], tall ? x[0] : xt[0]);
    };
    if (q.x_type == kGradF32)
        start(Elem<kGradF32>());
    else if (q.x_type == kGradF16)
        start(Elem<kGradF16>());
    else
        start(Elem<kGradBf16>());

    // P's entries are at most |a| + 1.5 |b| + 2.25 |c| while singular values stay below 1.22
    int e = 0;
    (void)frexpf(32768.0f / (fabsf(q.a) + 1.5f * fabsf(q.b) + 2.25f * fabsf(q.c) + 1e-30f), &e);
    e = e - 1 < 14 ? e - 1 : 14;
    const Poly poly = {q.a, q.b, q.c, ldexpf(1.0f, e)};
    const Result none = {};
    auto tiles = [&](int64_t rows, int64_t cols, int64_t side) { return ((rows + side - 1) / side) * ((cols + side - 1) / side); };
    auto run = [&](auto sym, auto app, const Plane& x0, const Plane& xt0, const Plane& x1, const Plane& xt1, bool last) {
        typedef typename decltype(sym)::Is Sym;
        typedef typename decltype(app)::Is App;
        constexpr int kS = decltype(sym)::kSide, kA = decltype(app)::kSide;
        const uint32_t side = (uint32_t)((m + kS - 1) / kS), tri = side * (side + 1) / 2;
        k_symmetric<Sym, kS, Full, false><<<tri * batch, Sym::kThreads, 0, s>>>(x0, g, (uint32_t)m, tri, poly);
        k_symmetric<Sym, kS, Full, true><<<tri * batch, Sym::kThreads, 0, s>>>(g, pm, (uint32_t)m, tri, poly);
        const uint32_t tm = (uint32_t)((m + kA - 1) / kA), tn = (uint32_t)((n + kA - 1) / kA);
        if (last) {
            const Result o = {q.out, tall, q.update, q.keep, q.gain, q.ldo, q.out_stride, q.rows, q.cols};
            auto finish = [&](auto type) {
                k_apply<App, kA, Full, true, typename decltype(type)::T>
                    <<<tm * tn * batch, App::kThreads, 0, s>>>(pm, xt0, x1, xt1, (uint32_t)m, (uint32_t)n, tm, tn, 1.0f / (kScaleX * poly.scale), o);
            };
            if (q.out_type == kGradF32)
                finish(Elem<kGradF32>());
            else if (q.out_type == kGradF16)
                finish(Elem<kGradF16>());
            else
                finish(Elem<kGradBf16>());
        } else {
            k_apply<App, kA, Full, false, float>
                <<<tm * tn * batch, App::kThreads, 0, s>>>(pm, xt0, x1, xt1, (uint32_t)m, (uint32_t)n, tm, tn, 1.0f / poly.scale, none);
        }
    };
    const int64_t t256 = tiles(m, n, 256) * q.batch, t128 = tiles(m, n, 128) * q.batch;
    const int64_t s256 = tiles(m, m, 256) * q.batch / 2, s128 = tiles(m, m, 128) * q.batch / 2;
    const Square<Tile<HalfCore, 256, 256, 2, 2, 2, 2>, 256> q256;
    const Square<Tile<HalfCore, 128, 128, 2, 2, 2, 2>, 128> q128;
    const Square<Tile<HalfCore, 64, 64, 2, 2, 2, 6>, 64> q64;
    for (int k = 0; k < q.steps; ++k) {
        const bool last = k + 1 == q.steps;
        const Plane &x0 = x[k & 1], &xt0 = xt[k & 1], &x1 = x[~k & 1], &xt1 = xt[~k & 1];
        if (s256 >= 200)
            run(q256, q256, x0, xt0, x1, xt1, last);
        else if (s128 >= 100 && t256 >= 200)
            run(q128, q256, x0, xt0, x1, xt1, last);
        else if (s128 >= 100)
            run(q128, q128, x0, xt0, x1, xt1, last);
        else if (t128 >= 200)
            run(q64, q128, x0, xt0, x1, xt1, last);
        else
            run(q64, q64, x0, xt0, x1, xt1, last);
    }
}

}  // namespace

size_t ortho_scratch(int batch, int64_t rows, int64_t cols, bool full) { return Layout(batch, rows, cols, full).total; }

void launch_orthogonalize(const OrthoCall& q, char* scratch, hipStream_t s)
{
    if (q.full)
        orthogonalize<true>(q, scratch, s);
    else
        orthogonalize<false>(q, scratch, s);
}

}  // namespace sidco
