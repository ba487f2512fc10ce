// 4-bit microscaled numbers: a gradient's exchange with error feedback, matrices along both axes, and their products.
//
// A block is 32 neighbours x_i of a row.  With e = floor(log2 max|x_i|) its exponent byte is max(e - 2, -127) + 127, and its
// codes are x_i / 2^(byte - 127) rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even code, 6 beyond it).
// In the bits of an fp32 magnitude the byte is the exponent field less two, at least 0; a field of 255 (an infinity or a NaN
// in the block) is kept as the byte 255, and the block then stands for NaN.  The division is by a power of two and therefore
// exact; the rounding is the conversion instruction's.
#include "sidco_dense.h"
#include "sidco_product.h"

namespace sidco {
namespace {

typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4h __attribute__((ext_vector_type(4), aligned(2)));

struct F32 {
    typedef float T;
    static __device__ __forceinline__ float widen(T x) { return x; }
    static __device__ __forceinline__ T narrow(float x) { return x; }
};
typedef unsigned short us2 __attribute__((ext_vector_type(2)));

struct F16 {
    typedef _Float16 T;
    // fp32 bits of the magnitude that a 16-bit one has, and two neighbours' codes over `scale` into byte Sel
    static __device__ __forceinline__ uint32_t widen_bits(uint32_t m) { return __float_as_uint((float)__builtin_bit_cast(_Float16, (unsigned short)m)); }
    template <int Sel>
    static __device__ __forceinline__ uint32_t encode2(uint32_t c, uint32_t two, float scale)
    {
        typedef _Float16 v2h __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(v2h, two), scale, Sel);
    }
    static __device__ __forceinline__ float widen(T x) { return (float)x; }
    static __device__ __forceinline__ T narrow(float x) { return (T)x; }
};
struct Bf16 {
    typedef __bf16 T;
    static __device__ __forceinline__ uint32_t widen_bits(uint32_t m) { return m << 16; }
    template <int Sel>
    static __device__ __forceinline__ uint32_t encode2(uint32_t c, uint32_t two, float scale)
    {
        typedef __bf16 v2b __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2b, two), scale, Sel);
    }
    static __device__ __forceinline__ float widen(T x) { return (float)x; }
    static __device__ __forceinline__ T narrow(float x) { return (T)x; }
};

template <class E>
__device__ __forceinline__ void load8(const typename E::T* p, float x[8])
{
    if constexpr (sizeof(typename E::T) == 4) {
        const f4 a = *(const f4*)p, b = *(const f4*)(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
    } else {
        const u4 a = *(const u4h*)p;
        typedef typename E::T t8 __attribute__((ext_vector_type(8)));
        const t8 v = __builtin_bit_cast(t8, a);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = E::widen(v[i]);
    }
}

template <class E>
__device__ __forceinline__ void store8(typename E::T* p, const float x[8])
{
    if constexpr (sizeof(typename E::T) == 4) {
        *(f4*)p = f4{x[0], x[1], x[2], x[3]};
        *(f4*)(p + 4) = f4{x[4], x[5], x[6], x[7]};
    } else {
        typedef typename E::T t8 __attribute__((ext_vector_type(8)));
        t8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = E::narrow(x[i]);
        *(u4h*)p = __builtin_bit_cast(u4, v);
    }
}

// n < 8 elements, zeros after them
template <class E>
__device__ __forceinline__ void load_few(const typename E::T* p, int64_t n, float x[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? E::widen(p[i]) : 0.0f;
}

template <class E>
__device__ __forceinline__ void store_few(typename E::T* p, int64_t n, const float x[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = E::narrow(x[i]);
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

__device__ __forceinline__ uint32_t largest8(const float x[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = larger(m, magnitude(x[i]));
    return m;
}

// the largest over the four lanes of a quad
__device__ __forceinline__ uint32_t largest_of_quad(uint32_t m)
{
    m = larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, true));  // lanes 1 0 3 2
    return larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, true));  // lanes 2 3 0 1
}

// exponent byte of a block whose largest magnitude has these bits
__device__ __forceinline__ uint32_t exponent_byte(uint32_t top)
{
    const uint32_t e = top >> 23;
    return e == 255 ? 255 : (e > 2 ? e - 2 : 0);
}

// 1 / 2^(byte - 127); byte <= 252
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254 - byte) << 23); }
// 2^(byte - 127); NaN for 255
__device__ __forceinline__ float scale_of(uint32_t byte)
{
    return __uint_as_float(byte == 0 ? 0x00400000u : (byte == 255 ? 0x7fc00000u : byte << 23));
}

// the codes of 8 neighbours, the first in the lowest bits
__device__ __forceinline__ uint32_t encode8(const float x[8], uint32_t byte)
{
    const float inv = inverse_scale(byte);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0] * inv, x[1] * inv, 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2] * inv, x[3] * inv, 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4] * inv, x[5] * inv, 1.0f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6] * inv, x[7] * inv, 1.0f, 3);
    return byte == 255 ? 0 : c;
}

// The same for elements of 16 bits, which stay as they are, two to a register: a magnitude's order is that of its bits, and the
// conversion takes pairs and divides by the scale itself.
__device__ __forceinline__ us2 magnitudes(uint32_t two) { return __builtin_bit_cast(us2, two & 0x7fff7fffu); }
__device__ __forceinline__ us2 larger2(us2 a, us2 b) { return __builtin_elementwise_max(a, b); }

template <class E>
__device__ __forceinline__ uint32_t encode_pairs(uint32_t a, uint32_t b, uint32_t d, uint32_t e, uint32_t byte)
{
    const float scale = scale_of(byte);
    uint32_t c = E::template encode2<0>(0, a, scale);
    c = E::template encode2<1>(c, b, scale);
    c = E::template encode2<2>(c, d, scale);
    c = E::template encode2<3>(c, e, scale);
    return byte == 255 ? 0 : c;
}

// what 8 codes stand for, times the scale's power of two
__device__ __forceinline__ void decode8(uint32_t c, float scale, float x[8])
{
    const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
    const v2f d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y, x[4] = d.x, x[5] = d.y, x[6] = e.x, x[7] = e.y;
}

constexpr int kFlat = 256;  // threads of the kernels of flat vectors

// A lane has 8 neighbours, a quad of lanes a block.  acc = g + r; the residual keeps what the codes do not hold, and all of
// acc where the block stands for NaN.  Bound by memory: one pass, and the block's largest magnitude goes round its quad in
// registers, so that LDS and a second look at the data are not needed.  138.4 M elements, gradient in bf16 with a residual:
// 270 us for 1.46 GB, 5.4 TB/s (a plain copy reaches 5.0); 270 thousand of fp32: 2.9 us, a launch.
template <class E, bool Residual>
__global__ __launch_bounds__(kFlat) void k_mx4_compress(const typename E::T* __restrict__ grad, float* __restrict__ residual, int64_t d,
                                                        uint32_t* __restrict__ codes, uint8_t* __restrict__ scales, int64_t groups)
{
    for (int64_t i = (int64_t)blockIdx.x * kFlat + threadIdx.x; i < groups; i += (int64_t)gridDim.x * kFlat) {
        const int64_t j = i * 8, left = d - j;
        float x[8], r[8];
        if (left >= 8) {
            load8<E>(grad + j, x);
            if (Residual) load8<F32>(residual + j, r);
        } else {
            load_few<E>(grad + j, left, x);
            if (Residual) load_few<F32>(residual + j, left, r);
        }
        if (Residual) {
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] += r[k];
        }
        const uint32_t byte = exponent_byte(largest_of_quad(largest8(x)));
        const uint32_t c = encode8(x, byte);
        codes[i] = c;
        if ((threadIdx.x & 3) == 0) scales[i >> 2] = (uint8_t)byte;
        if (Residual) {
            decode8(c, byte == 255 ? 1.0f : scale_of(byte), r);  // 255: codes of zeros, nothing is taken from acc
#pragma unroll
            for (int k = 0; k < 8; ++k) r[k] = x[k] - r[k];
            if (left >= 8)
                store8<F32>(residual + j, r);
            else
                store_few<F32>(residual + j, left, r);
        }
    }
}

// dense (+)= scale * the sum over the workers, in their order and in fp32: one thread adds all of an element, and the result is
// the same in every run.  Bound by memory: codes are read once, the dense vector is written once.  Four workers' loads are
// under way together (eight were no faster).  138.4 M elements of 8 workers: 252 us for 1.14 GB, 4.5 TB/s.
template <bool Accumulate>
__global__ __launch_bounds__(kFlat) void k_mx4_aggregate(const uint8_t* __restrict__ codes, int64_t code_stride,
                                                         const uint8_t* __restrict__ scales, int64_t scale_stride, int workers,
                                                         int64_t d, float scale, float* __restrict__ dense, int64_t groups)
{
    for (int64_t i = (int64_t)blockIdx.x * kFlat + threadIdx.x; i < groups; i += (int64_t)gridDim.x * kFlat) {
        const int64_t j = i * 8, left = d - j;
        float sum[8] = {};
#pragma unroll 4
        for (int w = 0; w < workers; ++w) {
            const uint32_t c = *(const uint32_t*)(codes + w * code_stride + i * 4);
            const uint32_t byte = scales[w * scale_stride + (i >> 2)];
            float x[8];
            decode8(c, scale_of(byte), x);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += byte == 255 ? scale_of(255) : x[k];
        }
        float old[8];
        if (Accumulate) {
            if (left >= 8)
                load8<F32>(dense + j, old);
            else
                load_few<F32>(dense + j, left, old);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] = Accumulate ? fmaf(scale, sum[k], old[k]) : scale * sum[k];
        if (left >= 8)
            store8<F32>(dense + j, sum);
        else
            store_few<F32>(dense + j, left, sum);
    }
}

// ---- matrices ----

// A launch's dimension has fewer than 2^32 threads: blocks of 512 beyond 2^20 go on in the next row of the grid.
__device__ __forceinline__ uint32_t block_number() { return blockIdx.y * gridDim.x + blockIdx.x; }
dim3 grid_of(uint32_t blocks) { return blocks <= 1u << 20 ? dim3(blocks) : dim3(1u << 20, (blocks - 1) / (1u << 20) + 1); }

constexpr int kSide = 128;       // a block quantises kSide x kSide elements
constexpr int kQuant = 512;

// Along the rows a quad of lanes has a block as above.  Along the columns a lane reads its column from LDS: 32 rows of one of
// fp32 elements, 16 of two neighbouring ones of 16 bits, two lanes then having a block.  The blocks' codes follow each other
// in the transposed row, so neighbouring lanes take the blocks of one column; their rows' columns are kept with bits 4 to 6
// changed by the block's number, so that the lanes read different banks.  x is read once for both.  Bound by memory, and more
// so by the short pieces (64 bytes of 128 rows and of 128 columns) that a square tile writes: bf16, both directions,
// 4096 x 25088 81 us for 315 MB, 3.9 TB/s; 16384 x 4096 61 us for 206 MB, 3.4 TB/s.  Tiles given to the XCDs in runs make whole
// lines of the pieces in L2 (81 to 79 us) but leave the codes elsewhere for whoever reads them next (64 us, and 6 us on two
// reads): not done.  Two loads in flight ahead of the first use cost registers and time (61 to 65 us).
template <class E, bool Along, bool Across>
__global__ __launch_bounds__(kQuant) void k_mx4_quantize(const typename E::T* __restrict__ x, int64_t rows, int64_t cols, int64_t ldx,
                                                           uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                                           uint8_t* __restrict__ codes_t, uint8_t* __restrict__ scales_t,
                                                           uint32_t across_x, uint32_t blocks)
{
    typedef typename E::T T;
    constexpr bool kHalf = sizeof(T) == 2;
    constexpr int kTurn = kHalf ? 16 : 32;  // rows whose columns are kept alike
    __shared__ __align__(16) T tile[Across ? kSide * kSide : 1];
    const uint32_t block = block_number();
    if (block >= blocks) return;
    const int64_t r0 = (int64_t)(block / across_x) * kSide, c0 = (int64_t)(block % across_x) * kSide;
    const int64_t pitch = mx4_padded(cols) / 2, pitch_t = mx4_padded(rows) / 2;
    const bool along = Along && c0 < pitch * 2, across = Across && r0 < pitch_t * 2;
#pragma unroll
    for (int k = 0; k < kSide * kSide / 8 / kQuant; ++k) {
        const int g = k * kQuant + threadIdx.x, r = g / (kSide / 8), c = g % (kSide / 8) * 8;
        const int64_t row = r0 + r, left = row < rows ? cols - (c0 + c) : 0;
        const T* p = x + row * ldx + c0 + c;
        T* to = &tile[Across ? r * kSide + (c ^ (r / kTurn * 16)) : 0];
        uint32_t byte, code;
        if constexpr (kHalf) {
            u4 v = {0, 0, 0, 0};
            if (left >= 8) {
                v = *(const u4h*)p;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < left) v[i / 2] |= (uint32_t)__builtin_bit_cast(unsigned short, p[i]) << (16 * (i % 2));
            }
            const us2 m = larger2(larger2(magnitudes(v[0]), magnitudes(v[1])), larger2(magnitudes(v[2]), magnitudes(v[3])));
            byte = exponent_byte(largest_of_quad(E::widen_bits(larger(m[0], m[1]))));
            code = encode_pairs<E>(v[0], v[1], v[2], v[3], byte);
            if (Across) *(u4*)to = v;
        } else {
            float v[8];
            if (left >= 8)
                load8<E>(p, v);
            else
                load_few<E>(p, left, v);
            byte = exponent_byte(largest_of_quad(largest8(v)));
            code = encode8(v, byte);
            if (Across) store8<E>(to, v);
        }
        if (along && row < rows) {
            *(uint32_t*)(codes + row * pitch + (c0 + c) / 2) = code;
            if ((threadIdx.x & 3) == 0) scales[row * (pitch / 16) + (c0 + c) / kMxBlock] = (uint8_t)byte;
        }
    }
    if (!Across) return;
    __syncthreads();
    if constexpr (kHalf) {
        const int c = threadIdx.x / 8 * 2, h = threadIdx.x % 8;  // columns c and c + 1, rows 16 h to 16 h + 15
        uint32_t v[16];
        us2 top = {0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            v[i] = *(const uint32_t*)&tile[(h * 16 + i) * kSide + (c ^ (h * 16))];
            top = larger2(top, magnitudes(v[i]));
        }
        const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, top), 0xb1, 0xf, 0xf, true);  // lanes 1 0 3 2
        top = larger2(top, __builtin_bit_cast(us2, other));
        if (!across) return;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (c0 + c + j >= cols) break;
            const uint32_t byte = exponent_byte(E::widen_bits(top[j])), pick = j ? 0x07060302u : 0x05040100u;
            uint32_t two[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) two[i] = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], pick);
            uint2 code = {encode_pairs<E>(two[0], two[1], two[2], two[3], byte), encode_pairs<E>(two[4], two[5], two[6], two[7], byte)};
            *(uint2*)(codes_t + (c0 + c + j) * pitch_t + r0 / 2 + h * 8) = code;
            if ((h & 1) == 0) scales_t[(c0 + c + j) * (pitch_t / 16) + r0 / kMxBlock + h / 2] = (uint8_t)byte;
        }
    } else {
        const int c = threadIdx.x / 4, b = threadIdx.x % 4;
        float v[32];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            v[i] = tile[(b * 32 + i) * kSide + (c ^ (b * 16))];
            top = larger(top, magnitude(v[i]));
        }
        if (!across || c0 + c >= cols) return;
        const uint32_t byte = exponent_byte(top);
        const u4 code = {encode8(v, byte), encode8(v + 8, byte), encode8(v + 16, byte), encode8(v + 24, byte)};
        *(u4*)(codes_t + (c0 + c) * pitch_t + r0 / 2 + b * 16) = code;
        scales_t[(c0 + c) * (pitch_t / 16) + r0 / kMxBlock + b] = (uint8_t)byte;
    }
}

// A lane has 8 neighbours of a row; a block of 2048 columns takes rows in turn.  Bound by memory: 16384 x 4096 to bf16 39 us for
// 170 MB, 4.4 TB/s; 26 us where the codes are still in the caches.
template <class E>
__global__ __launch_bounds__(kFlat) void k_mx4_dequantize(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                          int64_t rows, int64_t cols, typename E::T* __restrict__ out, int64_t ldo)
{
    const int64_t pitch = mx4_padded(cols) / 2;
    const int64_t j = ((int64_t)blockIdx.x * kFlat + threadIdx.x) * 8, left = cols - j;
    if (left <= 0) return;
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        const uint32_t byte = scales[row * (pitch / 16) + j / kMxBlock];
        float v[8];
        decode8(*(const uint32_t*)(codes + row * pitch + j / 2), scale_of(byte), v);
        if (byte == 255) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = scale_of(255);
        }
        if (left >= 8)
            store8<E>(out + row * ldo + j, v);
        else
            store_few<E>(out + row * ldo + j, left, v);
    }
}

// ---- products ----

template <class E>
__device__ __forceinline__ void store_product(const Mx4Product& p, int64_t m, int64_t n, const v4f& acc)
{
    typedef typename E::T T;
    if (m >= p.m || n >= p.n) return;
    T* c = (T*)p.c + m * p.ldc + n;
    typedef T t4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if (n + 4 <= p.n) {
        t4 v;
        if (p.accumulate) {
            const t4 old = *(const t4*)c;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = E::narrow(fmaf(p.alpha, acc[i], E::widen(old[i])));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = E::narrow(p.alpha * acc[i]);
        }
        *(t4*)c = v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.n) c[i] = E::narrow(p.accumulate ? fmaf(p.alpha, acc[i], E::widen(c[i])) : p.alpha * acc[i]);
    }
}

// Many rows on both sides: the matrix cores' time.  The instruction multiplies codes under their blocks' exponents and adds in
// fp32, so codes go from memory to it as they are; alpha and the old C are the epilogue's.  4096 x 4096 x 25088 (rows, columns,
// contraction) 190 us, 4.4 PFLOP/s; 4096 x 25088 x 4096 to bf16 256 + 19 us in two launches, 3.1, and 25088 columns to fp32
// 281 + 20 us, 2.8, where every 32 lines of a tile end with its stores; 8192 cubed 258 us, 4.3.  The matrix units are busy
// two thirds of the time and the clock falls under their load.
template <class E, class Tl>
__global__ __launch_bounds__(Tl::kThreads) void k_mx4_product(Mx4Product p, uint32_t tm, uint32_t tn, uint32_t from)
{
    __shared__ __align__(1024) char lds[Tl::kLds];
    const uint32_t pitch = (uint32_t)(mx4_padded(p.k) / 2);
    const Rows a = {p.a, p.a_scales, (uint32_t)p.m, pitch}, b = {p.b, p.b_scales, (uint32_t)p.n, pitch};
    Tl t;
    auto place = [&](uint32_t tile, uint32_t& m0, uint32_t& n0) {
        uint32_t i, j;
        tile_of(xcd_run(tile, tm * tn), tm, tn, i, j);
        m0 = i * Tl::kM;
        n0 = from + j * Tl::kN;
    };
    t.template run<1>(
        tm * tn, pitch, lds,
        [&](uint32_t tile, int) {
            uint32_t m0, n0;
            place(tile, m0, n0);
            t.take(a, b, m0, n0);
        },
        [&](uint32_t tile) {
            uint32_t m0, n0;
            place(tile, m0, n0);
            if (m0 + Tl::kM <= p.m && n0 + Tl::kN <= p.n && !p.accumulate) {
                typedef typename E::T T;
                typedef T t4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
                T* c = (T*)p.c + (int64_t)m0 * p.ldc + n0;
                t.each([&](uint32_t m, uint32_t n, const v4f& v) {
                    *(t4*)(c + (int64_t)m * p.ldc + n) = t4{E::narrow(p.alpha * v[0]), E::narrow(p.alpha * v[1]), E::narrow(p.alpha * v[2]),
                                                            E::narrow(p.alpha * v[3])};
                });
            } else {
                t.each([&](uint32_t m, uint32_t n, const v4f& v) { store_product<E>(p, (int64_t)m0 + m, (int64_t)n0 + n, v); });
            }
        });
}

__device__ __forceinline__ v4f multiply16(const v4i& a, const v4i& b, const v4f& c, int sa, int sb)
{
    const v8i wa = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, wb = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wb, c, 4, 4, 0, sa, 0, sb);  // 4: e2m1
}

// Few rows of A: the time is that of reading B once.  A block has 16 rows of B; its 8 waves take lines in turn, straight to
// registers, the next line under way while one is multiplied, and add up in LDS.  A comes in blocks, or (X other than Packed) as
// it is: then each block quantises all of it into LDS while its first lines are under way, which a launch less pays for while A
// has few elements.  1 x 4096 by 4096 x 4096: 5.0 us (8.9 MB, 1.8 TB/s: a launch's start, one trip to memory for each of two
// lines, a sum).
constexpr int kFewWaves = 8;
constexpr int kFewElements = 65536;  // of A, padding included, that LDS has room for
struct Packed {
    typedef uint8_t T;
};

template <class E, class X, int Mt>
__global__ __launch_bounds__(64 * kFewWaves) void k_mx4_few(Mx4Product p, const typename X::T* __restrict__ x, int64_t ldx)
{
    constexpr bool kPacked = sizeof(typename X::T) == 1;
    constexpr int kRowPad = 16;  // bytes after a row of codes, so that 16 rows' pieces are in different banks
    __shared__ v4f part[kFewWaves][Mt][64];
    __shared__ __align__(16) uint8_t codes[kPacked ? 16 : kFewElements / 2 + Mt * 16 * kRowPad], exps[kPacked ? 1 : kFewElements / kMxBlock];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int64_t n0 = (int64_t)block_number() * 16;
    if (n0 >= p.n) return;
    const int64_t pitch = mx4_padded(p.k) / 2;
    const int64_t nb = n0 + r < p.n ? n0 + r : p.n - 1;
    const uint8_t *b = p.b + nb * pitch + q * 16, *bs = p.b_scales + nb * (pitch / 16) + q;
    v4i fb[2], next[2];
    int sb[2], snext[2];
    auto fetch = [&](int64_t k, v4i (&f)[2], int (&sc)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f[h] = *(const v4i*)(b + k + h * 64);
            sc[h] = bs[k / 16 + h * 4];
        }
    };
    const int64_t step = kFewWaves * kLine;
    int64_t k = (int64_t)wave * kLine;
    if (k < pitch) fetch(k, fb, sb);
    if constexpr (!kPacked) {
        const int row_groups = (int)(pitch / 4), groups = (int)p.m * row_groups;  // of 8 elements; whole quads of lanes
        for (int g = threadIdx.x; g < groups; g += 64 * kFewWaves) {
            const int row = g / row_groups, at = g - row * row_groups, left = (int)p.k - at * 8;
            const typename X::T* from = x + row * ldx + at * 8;
            float v[8];
            if (left >= 8)
                load8<X>(from, v);
            else
                load_few<X>(from, left, v);
            const uint32_t byte = exponent_byte(largest_of_quad(largest8(v)));
            *(uint32_t*)(codes + row * (pitch + kRowPad) + at * 4) = encode8(v, byte);
            if ((at & 3) == 0) exps[row * (pitch / 16) + (at >> 2)] = (uint8_t)byte;
        }
        __syncthreads();
    }
    const uint8_t *a[Mt], *as[Mt];
    v4f acc[Mt];
#pragma unroll
    for (int i = 0; i < Mt; ++i) {
        const int64_t m = i * 16 + r < p.m ? i * 16 + r : p.m - 1;
        a[i] = (kPacked ? p.a + m * pitch : codes + m * (pitch + kRowPad)) + q * 16;
        as[i] = (kPacked ? p.a_scales : exps) + m * (pitch / 16) + q;
        acc[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (; k < pitch; k += step) {
        if (k + step < pitch) fetch(k + step, next, snext);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < Mt; ++i)
                acc[i] = multiply16(fb[h], *(const v4i*)(a[i] + k + h * 64), acc[i], sb[h], as[i][k / 16 + h * 4]);
#pragma unroll
        for (int h = 0; h < 2; ++h) fb[h] = next[h], sb[h] = snext[h];
    }
#pragma unroll
    for (int i = 0; i < Mt; ++i) part[wave][i][lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < Mt; i += kFewWaves) {
        v4f sum = part[0][i][lane];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) sum += part[w][i][lane];
        store_product<E>(p, i * 16 + r, n0 + 4 * q, sum);
    }
}

template <class Tl>
struct Shape {
    typedef Tl Is;
};

template <class F>
void by_type(int type, const F& f)
{
    if (type == kGradF32)
        f(F32());
    else if (type == kGradF16)
        f(F16());
    else
        f(Bf16());
}

uint32_t flat_blocks(int64_t groups)
{
    const int64_t b = (groups + kFlat - 1) / kFlat;
    return (uint32_t)(b < 8192 ? b : 8192);
}

}  // namespace

void launch_mx4_compress(const void* grad, int type, float* residual, int64_t d, uint8_t* codes, uint8_t* scales, hipStream_t s)
{
    const int64_t groups = mx4_padded(d) / 8;
    by_type(type, [&](auto e) {
        typedef decltype(e) E;
        if (residual)
            k_mx4_compress<E, true><<<flat_blocks(groups), kFlat, 0, s>>>((const typename E::T*)grad, residual, d, (uint32_t*)codes,
                                                                          scales, groups);
        else
            k_mx4_compress<E, false><<<flat_blocks(groups), kFlat, 0, s>>>((const typename E::T*)grad, residual, d, (uint32_t*)codes,
                                                                           scales, groups);
    });
}

void launch_mx4_aggregate(const uint8_t* codes, int64_t code_stride, const uint8_t* scales, int64_t scale_stride, int workers,
                          int64_t d, float scale, bool accumulate, float* dense, hipStream_t s)
{
    const int64_t groups = (d + 7) / 8;
    if (accumulate)
        k_mx4_aggregate<true><<<flat_blocks(groups), kFlat, 0, s>>>(codes, code_stride, scales, scale_stride, workers, d, scale, dense,
                                                                    groups);
    else
        k_mx4_aggregate<false><<<flat_blocks(groups), kFlat, 0, s>>>(codes, code_stride, scales, scale_stride, workers, d, scale,
                                                                     dense, groups);
}

void launch_mx4_quantize(const void* x, int type, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes, uint8_t* scales,
                         uint8_t* codes_t, uint8_t* scales_t, hipStream_t s)
{
    const uint32_t gx = (uint32_t)((codes ? mx4_padded(cols) : cols + kSide - 1) / kSide);
    const uint32_t blocks = gx * (uint32_t)((codes_t ? mx4_padded(rows) : rows + kSide - 1) / kSide);
    const dim3 grid = grid_of(blocks);
    by_type(type, [&](auto e) {
        typedef decltype(e) E;
        const typename E::T* p = (const typename E::T*)x;
        if (codes && codes_t)
            k_mx4_quantize<E, true, true><<<grid, kQuant, 0, s>>>(p, rows, cols, ldx, codes, scales, codes_t, scales_t, gx, blocks);
        else if (codes)
            k_mx4_quantize<E, true, false><<<grid, kQuant, 0, s>>>(p, rows, cols, ldx, codes, scales, codes_t, scales_t, gx, blocks);
        else
            k_mx4_quantize<E, false, true><<<grid, kQuant, 0, s>>>(p, rows, cols, ldx, codes, scales, codes_t, scales_t, gx, blocks);
    });
}

void launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* out, int type, int64_t ldo,
                           hipStream_t s)
{
    const dim3 grid((uint32_t)((cols + 8 * kFlat - 1) / (8 * kFlat)), (uint32_t)(rows < 32768 ? rows : 32768));
    by_type(type, [&](auto e) {
        typedef decltype(e) E;
        k_mx4_dequantize<E><<<grid, kFlat, 0, s>>>(codes, scales, rows, cols, (typename E::T*)out, ldo);
    });
}

namespace {

// Rows that k_mx4_few serves, two instructions' worth.
constexpr int kFewRows = 32;

// Times, us, for the choice between k_mx4_few and a tile of 64 rows, which leaves most of itself empty but has its operands
// under way ahead.  The first spreads a row of B over 8 waves and is better where rows are long and few, the second where there
// are many.  Measured, us, few / tiles, 1, 16 and 32 rows:
//   4096 x 25088 12.9 18.8 29.1 / 32.0 33.4 40.2; 4096 x 16384 11.1 16.8 23.9 / 22.6 23.8 27.1; 8192 x 8192 12.3 17.3 24.4 /
//   13.9 14.3 16.2; 25088 x 4096 17.2 27.5 39.8 / 14.3 15.7 17.9; 16384 x 16384 35.6 58.1 86.9 / 25.0 27.1 31.1;
// with 64 rows 45.8 / 53.7 for the first of these, 38.0 / 35.2 and 38.8 / 20.7 for the next.  A as it is costs each block its
// quantisation, a launch of its own 3 us; one launch / two, 1, 4 and 16 rows:
//   4096 x 4096 8.9 8.4 11.3 / 11.6 11.2 11.0; 10000 x 4096 9.1 12.0 22.4 / 11.9 11.7 12.2; 16384 x 16384 34.9 45.4 / 27.9 28.1;
//   10000 x 1500 8.7 8.3 10.1 / 11.0 10.5 11.1, with 20 rows 11.5 / 10.9, with 32 16.4 / 10.8.
struct FewTimes {
    float few, few_x, tiles;
};
FewTimes few_times(int64_t m, int64_t n, int64_t k)
{
    const float blocks = (float)((n + 15) / 16) / kCus, rounds = blocks > 1.0f ? blocks : 1.0f;
    const int64_t lines = mx4_padded(k) / 2 / kLine;
    const float few = 4.0f + rounds * (float)lines / kFewWaves * (0.9f + 0.04f * (float)m);
    return {few, few + rounds * (0.3f + 0.22f * (float)(m * mx4_padded(k)) / 4096.0f), (float)tile_time(3, (n + 63) / 64, lines)};
}

template <class X>
void few(const Mx4Product& p, const typename X::T* x, int64_t ldx, hipStream_t s)
{
    const dim3 grid = grid_of((uint32_t)((p.n + 15) / 16));
    by_type(p.type, [&](auto e) {
        typedef decltype(e) E;
        if (p.m <= 16)
            k_mx4_few<E, X, 1><<<grid, 64 * kFewWaves, 0, s>>>(p, x, ldx);
        else
            k_mx4_few<E, X, 2><<<grid, 64 * kFewWaves, 0, s>>>(p, x, ldx);
    });
}

}  // namespace

bool mx4_takes_x(int64_t m, int64_t n, int64_t k)
{
    if (m > kFewRows || m * mx4_padded(k) > kFewElements) return false;
    const FewTimes t = few_times(m, n, k);
    return t.few_x <= 3.0f + (t.few < t.tiles ? t.few : t.tiles);
}

void launch_mx4_product_x(const Mx4Product& p, const void* x, int type, int64_t ldx, hipStream_t s)
{
    by_type(type, [&](auto t) {
        typedef decltype(t) X;
        few<X>(p, (const typename X::T*)x, ldx, s);
    });
}

void launch_mx4_product(const Mx4Product& p, hipStream_t s)
{
    if (p.m <= kFewRows) {
        const FewTimes t = few_times(p.m, p.n, p.k);
        if (t.few <= t.tiles) return few<Packed>(p, nullptr, 0, s);
    }
    auto part = [&](int pick, int64_t from, int64_t columns) {
        auto go = [&](auto e, auto t) {
            typedef decltype(e) E;
            typedef typename decltype(t)::Is Tl;
            const uint32_t tm = (uint32_t)((p.m + Tl::kM - 1) / Tl::kM), tn = (uint32_t)((columns + Tl::kN - 1) / Tl::kN);
            k_mx4_product<E, Tl><<<tile_blocks(pick, (int64_t)tm * tn), Tl::kThreads, 0, s>>>(p, tm, tn, (uint32_t)from);
        };
        by_type(p.type, [&](auto e) {
            if (pick == 0)
                go(e, Shape<Tile<Mx4Core, 256, 256, 2, 2, 2>>());
            else if (pick == 1)
                go(e, Shape<Tile<Mx4Core, 192, 192, 2, 2, 3>>());
            else if (pick == 2)
                go(e, Shape<Tile<Mx4Core, 128, 128, 2, 2, 2>>());
            else
                go(e, Shape<Tile<Mx4Core, 64, 64, 2, 2, 4>>());
        });
    };
    const TilePlan plan = plan_tiles(p.m, p.n, 1, mx4_padded(p.k) / 2 / kLine);
    part(plan.pick, 0, plan.columns);
    if (plan.columns < p.n) part(plan.rest_pick, plan.columns, p.n - plan.columns);
}

}  // namespace sidco
