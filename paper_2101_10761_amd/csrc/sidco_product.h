// Tile product C = A B^T on the matrix cores, shared by the 4-bit products and by the Newton-Schulz products.
//
// Both operands are stored by rows along the contraction, and a step takes one 128-byte line of every row of the tile:
// 64 half-precision numbers, or 256 4-bit codes with the 8 exponents of their blocks.  Both kinds keep a lane's share of a
// matrix instruction at 16 bytes and the instruction at 16 cycles, so that one data path serves them.
//
// The lines go from memory to LDS without passing through registers (each lane names its own 16 bytes of memory, LDS is
// written in the order of the lanes).  A row of LDS is a line and rows follow each other, so equal columns of the 16 rows that
// an instruction reads would sit in the same banks; piece c of row r is therefore kept at place c ^ (r % 8), by choosing
// which piece a lane fetches.
#ifndef SIDCO_PRODUCT_H
#define SIDCO_PRODUCT_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sidco {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

constexpr int kLine = 128;  // bytes of a row that one step takes

// One operand: rows of `pitch` bytes, a multiple of kLine and less than 2^24, padded with zeros; for 4-bit codes also the exponents, a byte for
// each block, pitch / 16 bytes a row.
struct Rows {
    const void* data;
    const uint8_t* scales;
    uint32_t rows;
    uint32_t pitch;
};

typedef __attribute__((address_space(3))) char lds_char;

// A block's part of an operand as the loads take it: base address, bytes, raw 32-bit words.
__device__ __forceinline__ v4i resource(const void* base, uint32_t bytes)
{
    const uint64_t a = (uint64_t)base;
    return v4i{__builtin_amdgcn_readfirstlane((int)(uint32_t)a), __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xffff),
               __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
}

// Each lane's Bytes at `offset` (its own) + `at` (the wave's) of the operand go to LDS, lane by lane from `l` on.  The load
// names no register that it writes.  It is written out because the compiler, which cannot tell the stages of LDS apart, waits
// for every load made so far before the next read of LDS; wait_loads says what is waited for instead.
template <int Bytes>
__device__ __forceinline__ void to_lds(const v4i& from, uint32_t offset, uint32_t at, char* l)
{
    static_assert(Bytes == 16 || Bytes == 4, "what the load takes");
    const uint32_t place = (uint32_t)(uintptr_t)(lds_char*)l;
    if constexpr (Bytes == 16)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(place), "v"(offset), "s"(from), "s"(at)
                     : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(place), "v"(offset), "s"(from), "s"(at)
                     : "memory");
}

// Waits until at most N of this wave's loads are under way and its own LDS reads have arrived.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    static_assert(N >= 0 && N < 64, "the counter has 6 bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// The place of work item b of `total` when consecutive blocks go to the 8 XCDs in turn: each XCD gets a run of neighbours,
// whose operands meet in its L2.
__device__ __forceinline__ uint32_t xcd_run(uint32_t b, uint32_t total)
{
    const uint32_t x = b & 7, i = b >> 3, q = total >> 3, r = total & 7;
    return x * q + (x < r ? x : r) + i;
}

// Tile (row, column) number t of tm x tn: columns of 8 tile rows at a time, so that a run of tiles covers a near-square.
__device__ __forceinline__ void tile_of(uint32_t t, uint32_t tm, uint32_t tn, uint32_t& i, uint32_t& j)
{
    const uint32_t band = 8 * tn, g = t / band, first = g * 8;
    const uint32_t high = tm - first < 8 ? tm - first : 8;
    const uint32_t in = t - g * band;
    i = first + in % high;
    j = in / high;
}

// Tile number t of the lower triangle, diagonal included: row i holds i + 1 of them.
__device__ __forceinline__ void tile_of_triangle(uint32_t t, uint32_t& i, uint32_t& j)
{
    uint32_t r = (uint32_t)((__builtin_sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while (r * (r + 1) / 2 > t) --r;
    while ((r + 1) * (r + 2) / 2 <= t) ++r;
    i = r;
    j = t - r * (r + 1) / 2;
}

// What an instruction multiplies: 16 rows by 16 rows over half a line.
struct HalfCore {
    static constexpr bool kScaled = false;
    static __device__ __forceinline__ v4f mul(const v4i& a, const v4i& b, const v4f& c, int, int)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    }
};

struct Mx4Core {
    static constexpr bool kScaled = true;
    static __device__ __forceinline__ v4f mul(const v4i& a, const v4i& b, const v4f& c, int sa, int sb)
    {
        const v8i wa = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, wb = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wb, c, 4, 4, 0, sa, 0, sb);  // 4: e2m1
    }
};

// A block's tile: BM x BN by WM x WN waves, `Stages` lines deep in LDS.
template <class Core, int BM, int BN, int WM, int WN, int Stages>
struct Tile {
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int kMt = BM / WM / 16, kNt = BN / WN / 16;  // instructions' tiles of a wave
    static constexpr int kScaleBytes = Core::kScaled ? 8 * (BM + BN) : 0;
    static constexpr int kStage = (BM + BN) * kLine + kScaleBytes;
    static constexpr int kLds = Stages * kStage;
    static constexpr int kLoadsA = BM / 8 / kWaves, kLoadsB = BN / 8 / kWaves;      // 8 rows a load
    static constexpr int kLoadsS = Core::kScaled ? (BM + BN) / 32 / kWaves : 0;     // 32 rows' exponents a load
    static constexpr int kLoads = kLoadsA + kLoadsB + kLoadsS;
    static_assert(BM % (16 * WM) == 0 && BN % (16 * WN) == 0, "whole instructions");
    static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0, "whole loads");
    static_assert(!Core::kScaled || ((BM % 32 == 0) && (BM + BN) % (32 * kWaves) == 0), "whole loads of exponents");
    static_assert(kLds <= 160 * 1024, "LDS of a CU");

    v4f acc[kMt][kNt];
    v4i from_a, from_b, from_sa, from_sb;
    uint32_t src[kLoadsA + kLoadsB];  // this lane's 16 bytes of each load's rows
    uint32_t ssrc[kLoadsS + 1];
    int wave, lane;

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < kMt; ++i)
#pragma unroll
            for (int j = 0; j < kNt; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // Rows past the operand's end read its last row: their products are not stored.
    __device__ __forceinline__ void aim(const Rows& a, const Rows& b, uint32_t m0, uint32_t n0)
    {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t ra = a.rows - m0 < BM ? a.rows - m0 : BM, rb = b.rows - n0 < BN ? b.rows - n0 : BN;
        from_a = resource((const char*)a.data + (size_t)m0 * a.pitch, ra * a.pitch);
        from_b = resource((const char*)b.data + (size_t)n0 * b.pitch, rb * b.pitch);
        const uint32_t r = lane >> 3, c = (lane & 7) ^ r;
#pragma unroll
        for (int k = 0; k < kLoadsA + kLoadsB; ++k) {
            const bool first = k < kLoadsA;
            uint32_t row = (uint32_t)((first ? k : k - kLoadsA) * kWaves + wave) * 8 + r;
            const uint32_t last = (first ? ra : rb) - 1;
            src[k] = (row < last ? row : last) * (first ? a.pitch : b.pitch) + c * 16;
        }
        if (Core::kScaled) {
            from_sa = resource((const char*)a.scales + (size_t)m0 * (a.pitch / 16), ra * (a.pitch / 16));
            from_sb = resource((const char*)b.scales + (size_t)n0 * (b.pitch / 16), rb * (b.pitch / 16));
#pragma unroll
            for (int k = 0; k < kLoadsS; ++k) {
                const uint32_t at = (uint32_t)(k * kWaves + wave) * 32;  // row of the tile, B's after A's
                const uint32_t row = (at < BM ? at : at - BM) + (lane >> 1), last = (at < BM ? ra : rb) - 1;
                ssrc[k] = (row < last ? row : last) * ((at < BM ? a.pitch : b.pitch) / 16) + (lane & 1) * 4;
            }
        }
    }

    // line t of every row
    __device__ __forceinline__ void fetch(uint32_t t, char* stage)
    {
#pragma unroll
        for (int k = 0; k < kLoadsA + kLoadsB; ++k) {
            const int at = k < kLoadsA ? (k * kWaves + wave) * 1024 : BM * kLine + ((k - kLoadsA) * kWaves + wave) * 1024;
            to_lds<16>(k < kLoadsA ? from_a : from_b, src[k], t * kLine, stage + at);
        }
#pragma unroll
        for (int k = 0; k < kLoadsS; ++k) {
            const int at = k * kWaves + wave;
            to_lds<4>(at * 32 < BM ? from_sa : from_sb, ssrc[k], t * 8, stage + (BM + BN) * kLine + at * 256);
        }
    }

    __device__ __forceinline__ void multiply(const char* stage)
    {
        const int wm = wave / WN, wn = wave % WN;
        const int r = lane & 15, q = lane >> 4;
        const char* pa = stage + (wm * (BM / WM) + r) * kLine;
        const char* pb = stage + BM * kLine + (wn * (BN / WN) + r) * kLine;
        const char* ps = stage + (BM + BN) * kLine;
        uint2 sa[Core::kScaled ? kMt : 1], sb[Core::kScaled ? kNt : 1];
        if (Core::kScaled) {
#pragma unroll
            for (int i = 0; i < kMt; ++i) sa[i] = *(const uint2*)(ps + (wm * (BM / WM) + i * 16 + r) * 8);
#pragma unroll
            for (int j = 0; j < kNt; ++j) sb[j] = *(const uint2*)(ps + BM * 8 + (wn * (BN / WN) + j * 16 + r) * 8);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int piece = ((h * 4 + q) ^ (r & 7)) * 16;
            v4i fa[kMt], fb[kNt];
#pragma unroll
            for (int j = 0; j < kNt; ++j) fb[j] = *(const v4i*)(pb + j * 16 * kLine + piece);
#pragma unroll
            for (int i = 0; i < kMt; ++i) fa[i] = *(const v4i*)(pa + i * 16 * kLine + piece);
#pragma unroll
            for (int i = 0; i < kMt; ++i)
#pragma unroll
                for (int j = 0; j < kNt; ++j)
                    acc[i][j] = Core::mul(fb[j], fa[i], acc[i][j], Core::kScaled ? (int)((h ? sb[j].y : sb[j].x) >> (8 * q)) : 0,
                                          Core::kScaled ? (int)((h ? sa[i].y : sa[i].x) >> (8 * q)) : 0);
        }
    }

    // Adds the products over `steps` lines.  Every wave of the block calls it; LDS is free again when the next one fetches.
    __device__ __forceinline__ void run(const Rows& a, const Rows& b, uint32_t m0, uint32_t n0, uint32_t steps, char* lds)
    {
        aim(a, b, m0, n0);
        __syncthreads();  // the stages may still be read for what was computed before
#pragma unroll
        for (int s = 0; s < Stages - 1; ++s)
            if ((uint32_t)s < steps) fetch(s, lds + s * kStage);
        int at = 0;
        for (uint32_t t = 0; t < steps; ++t) {
            // step t's lines are there once the later steps' alone are under way, and once every wave says so
            if (t + Stages - 2 < steps)
                wait_loads<(Stages - 2) * kLoads>();
            else
                wait_loads<0>();
            __builtin_amdgcn_s_barrier();
            int next = at + Stages - 1;
            next = next >= Stages ? next - Stages : next;
            if (t + Stages - 1 < steps) fetch(t + Stages - 1, lds + next * kStage);
            multiply(lds + at * kStage);
            at = at + 1 == Stages ? 0 : at + 1;
        }
    }

    // f(row, column, 4 values): C's row and the first of four neighbouring columns, relative to the tile.
    template <class F>
    __device__ __forceinline__ void each(const F& f) const
    {
        const int wm = wave / WN, wn = wave % WN;
#pragma unroll
        for (int i = 0; i < kMt; ++i)
#pragma unroll
            for (int j = 0; j < kNt; ++j)
                f((uint32_t)(wm * (BM / WM) + i * 16 + (lane & 15)), (uint32_t)(wn * (BN / WN) + j * 16 + 4 * (lane >> 4)), acc[i][j]);
    }
};

}  // namespace sidco
#endif
