// Tile product C = A B^T on the matrix cores, shared by the 4-bit products and by the Newton-Schulz products.
//
// Both operands are stored by rows along the contraction, in pieces of 16 bytes: 8 half-precision numbers, or a block of 32
// 4-bit codes.  A matrix instruction takes four pieces of 16 rows of each operand in 16 cycles for either kind, so that one
// data path serves both.  A stage is two such fours, a line of 128 bytes of every row of the tile, and for 4-bit codes the
// exponents of these blocks.
//
// Stages go from memory to LDS without passing through registers (each lane names its own 16 bytes of memory, LDS is written
// in the order of the lanes).  Rows follow each other in LDS, so the same piece of the 16 rows that an instruction reads
// would sit in few banks; piece c of row r is therefore kept at place c ^ (r % 8), by choosing which piece a lane fetches.
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

constexpr int kLine = 128;  // a row's bytes are a multiple of this

// One operand: rows of `pitch` bytes, a multiple of kLine and less than 2^24, padded with zeros; for 4-bit codes also the exponents, a byte for
// each block, pitch / 16 bytes a row.
struct Rows {
    const void* data;
    const uint8_t* scales;
    uint32_t rows;
    uint32_t pitch;
};

// The rows' bytes from one row to the next of either operand, and the lines that are multiplied of each: all of them, or fewer,
// of a row that goes on.
struct Span {
    uint32_t pitch_a, pitch_b, lines;
};

typedef __attribute__((address_space(3))) char lds_char;

// A block's part of an operand as the loads take it: base address, bytes, raw 32-bit words.
__device__ __forceinline__ v4i resource(const void* base, uint32_t bytes)
{
    const uint64_t a = (uint64_t)base;
    return v4i{__builtin_amdgcn_readfirstlane((int)(uint32_t)a), __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xffff),
               __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
}

// Each lane's Bytes at `offset` (its own) + `at` (the wave's) of the operand go to LDS, lane by lane from `l` + More on.
// The load names no register that it writes.  It is written out because the compiler, which cannot tell the stages of LDS
// apart, waits for every load made so far before the next read of LDS; wait_loads says what is waited for instead.
template <int Bytes, int More>
__device__ __forceinline__ void to_lds(const v4i& from, uint32_t offset, uint32_t at, char* l)
{
    static_assert(Bytes == 16 || Bytes == 4, "what the load takes");
    const uint32_t to = (uint32_t)(uintptr_t)(lds_char*)l;
    if constexpr (Bytes == 16)
        asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(offset), "s"(from), "s"(at), "i"(More)
                     : "memory", "scc");
    else
        asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(to), "v"(offset), "s"(from), "s"(at), "i"(More)
                     : "memory", "scc");
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

// Four lanes with four columns of their row each come to hold four rows of one column each.
__device__ __forceinline__ v4f turned(v4f v)
{
    const int t = threadIdx.x & 3;
    auto swap1 = [](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0xb1, 0xf, 0xf, true)); };
    auto swap2 = [](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x4e, 0xf, 0xf, true)); };
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const float got = swap1(t & 1 ? v[i] : v[i + 1]);
        v[i] = t & 1 ? got : v[i];
        v[i + 1] = t & 1 ? v[i + 1] : got;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float got = swap2(t & 2 ? v[i] : v[i + 2]);
        v[i] = t & 2 ? got : v[i];
        v[i + 2] = t & 2 ? v[i + 2] : got;
    }
    return v;
}

// The same with 16-bit numbers, two to a register.
struct Four16 {
    uint32_t a, b;
};
__device__ __forceinline__ Four16 turned(Four16 v)
{
    auto swap1 = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, true); };
    auto swap2 = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, true); };
    const bool upper = threadIdx.x & 2;
    const uint32_t got = swap2(upper ? v.a : v.b);
    const uint32_t a = upper ? got : v.a, b = upper ? v.b : got;  // two columns of this row, and of the row two on
    const uint32_t pick = threadIdx.x & 1 ? 0x03020706 : 0x05040100;
    return {__builtin_amdgcn_perm(swap1(a), a, pick), __builtin_amdgcn_perm(swap1(b), b, pick)};
}

// The values as rounded to fp32.  A product rounded to fp32 and then to half is otherwise rounded once, by an instruction that
// does both, in one place and not in another: the half and what it leaves of the value would belong to different halves.
__device__ __forceinline__ v4f rounded(v4f v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x = v[i];
        asm("" : "+v"(x));
        v[i] = x;
    }
    return v;
}

// What an instruction multiplies: 16 rows by 16 rows over four pieces, lane l holding piece l / 16 of row l % 16.
//
// The instructions are written out because the sums have to stay where they are: with 64 tiles of them, all of a wave's 256
// accumulation registers, the compiler's own choice of registers moved half of them about in every step.  The waits that it
// would insert for them are written out too: settle() before instructions whose operands may just have been written by
// another kind of instruction, and rest() before the sums are read.  Nothing may move the sums between the two (the compiler
// would do it without a wait), which the one loop around all products sees to, and a test of the generated code.
struct HalfCore {
    static constexpr bool kScaled = false;
    static __device__ __forceinline__ void mul(const v4i& a, const v4i& b, v4f& c, int, int)
    {
        asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    }
};

struct Bf16Core {
    static constexpr bool kScaled = false;
    static __device__ __forceinline__ void mul(const v4i& a, const v4i& b, v4f& c, int, int)
    {
        asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    }
};

struct Mx4Core {
    static constexpr bool kScaled = true;
    static __device__ __forceinline__ void mul(const v4i& a, const v4i& b, v4f& c, int sa, int sb)  // 4: e2m1
    {
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                     : "+a"(c)
                     : "v"(a), "v"(b), "v"(sa), "v"(sb));
    }
};

__device__ __forceinline__ void settle() { asm volatile("s_nop 3" ::: "memory"); }
__device__ __forceinline__ void rest() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }

// The stages that a block fetches, in order: `stages` of each of `terms` terms of tile after tile, `step` apart.  Behind the last
// it stays at stage 0: the loads that are still made then are of a resource without bytes, whose range check subtracts the
// stage's offset from its size, and only at 0 is that no number of bytes at all.
struct Sequence {
    uint32_t tile, u;
    int term;
    // Goes on; whether to another tile's or term's first stage, or (tile >= tiles) behind the last.
    __host__ __device__ __forceinline__ bool next(uint32_t stages, int terms, uint32_t tiles, uint32_t step)
    {
        if (tile >= tiles || ++u < stages) return false;
        u = 0;
        if (++term == terms) term = 0, tile += step;
        return true;
    }
};

// A block's tile: BM x BN by WM x WN waves, `Stages` stages in LDS.
template <class Core, int BM, int BN, int WM, int WN, int Stages>
struct Tile {
    static constexpr int kM = BM, kN = BN;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int kMt = BM / WM / 16, kNt = BN / WN / 16;  // instructions' tiles of a wave
    static constexpr int kSeg = kLine, kExps = kLine / 16;        // bytes of a row in a stage, and exponents
    // a stage: exponents of A's and of B's rows, A's rows, B's rows
    static constexpr int kAtA = Core::kScaled ? (BM + BN) * kExps : 0, kAtB = kAtA + BM * kSeg, kStage = kAtB + BN * kSeg;
    static constexpr int kLds = Stages * kStage;
    static constexpr int kRowsLoad = 1024 / kSeg, kRowsExps = 256 / kExps;  // rows that a load of 16 or of 4 bytes a lane takes
    static constexpr int kLoadsA = BM / kRowsLoad / kWaves, kLoadsB = BN / kRowsLoad / kWaves;
    static constexpr int kLoadsS = Core::kScaled ? (BM + BN) / kRowsExps / kWaves : 0;
    static constexpr int kLoads = kLoadsA + kLoadsB + kLoadsS;
    static_assert(BM % (16 * WM) == 0 && BN % (16 * WN) == 0, "whole instructions");
    static_assert(BM % (kRowsLoad * kWaves) == 0 && BN % (kRowsLoad * kWaves) == 0, "whole loads");
    static_assert(!Core::kScaled || (BM % kRowsExps == 0 && (BM + BN) % (kRowsExps * kWaves) == 0), "whole loads of exponents");
    static_assert(Stages >= 2 && kLds <= 160 * 1024, "LDS of a CU");

    v4f acc[kMt][kNt];
    v4i from_a, from_b, from_s[kLoadsS + 1];
    uint32_t src[kLoadsA + kLoadsB];  // this lane's 16 bytes of each load's rows
    uint32_t ssrc[kLoadsS + 1];
    uint32_t stages;                  // of the rows
    int wave, lane;

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < kMt; ++i)
#pragma unroll
            for (int j = 0; j < kNt; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // The sums are in their registers here; nothing computed from them comes from before.
    __device__ __forceinline__ void hold()
    {
#pragma unroll
        for (int i = 0; i < kMt; ++i)
#pragma unroll
            for (int j = 0; j < kNt; ++j) asm volatile("" : "+a"(acc[i][j]));
    }

    static __device__ __forceinline__ int place(int row, int piece)
    {
        return piece ^ (row & 7);
    }

    // The lanes' places in a stage, the same for every tile.
    __device__ __forceinline__ void aim(const Span& span)
    {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        stages = span.lines;
        const int r = lane / 8, c = place(r, lane % 8);  // a load's first row is a multiple of 8
#pragma unroll
        for (int k = 0; k < kLoadsA + kLoadsB; ++k)
            src[k] = (uint32_t)(((k < kLoadsA ? k : k - kLoadsA) * kWaves + wave) * kRowsLoad + r) * (k < kLoadsA ? span.pitch_a : span.pitch_b) + c * 16;
#pragma unroll
        for (int k = 0; k < kLoadsS; ++k) {
            const uint32_t at = (uint32_t)(k * kWaves + wave) * kRowsExps;  // row of the tile, B's after A's
            ssrc[k] = ((at < BM ? at : at - BM) + lane / 2) * ((at < BM ? span.pitch_a : span.pitch_b) / 16) + lane % 2 * 4;
        }
    }

    // A tile may lie behind the last row altogether: none.
    static __device__ __forceinline__ uint32_t rows_left(uint32_t rows, uint32_t from, uint32_t most)
    {
        const uint32_t left = rows > from ? rows - from : 0;
        return left < most ? left : most;
    }

    // The tile whose stages are fetched from now on.  Rows past the operand's end are out of range: zeros come for them.
    __device__ __forceinline__ void take(const Rows& a, const Rows& b, uint32_t m0, uint32_t n0)
    {
        const uint32_t ra = rows_left(a.rows, m0, BM), rb = rows_left(b.rows, n0, BN);
        from_a = resource((const char*)a.data + (size_t)m0 * a.pitch, ra * a.pitch);
        from_b = resource((const char*)b.data + (size_t)n0 * b.pitch, rb * b.pitch);
#pragma unroll
        for (int k = 0; k < kLoadsS; ++k) {
            const bool first = (k * kWaves + wave) * kRowsExps < BM;
            const uint32_t exps = (first ? a.pitch : b.pitch) / 16;
            from_s[k] = resource((const char*)(first ? a.scales : b.scales) + (size_t)(first ? m0 : n0) * exps, (first ? ra : rb) * exps);
        }
    }
    __device__ __forceinline__ void take_nothing()
    {
        from_a[2] = from_b[2] = 0;
#pragma unroll
        for (int k = 0; k < kLoadsS; ++k) from_s[k][2] = 0;
    }

    // Load k of stage number u of the tile taken.
    template <int K>
    __device__ __forceinline__ void fetch(uint32_t u, char* stage) const
    {
        constexpr int kS = K - kLoadsA - kLoadsB;
        if constexpr (kS < 0) {
            constexpr bool kFirst = K < kLoadsA;
            constexpr int kAt = kFirst ? kAtA + K * kWaves * 1024 : kAtB + (K - kLoadsA) * kWaves * 1024;
            to_lds<16, kAt>(kFirst ? from_a : from_b, src[K], u * kSeg, stage + wave * 1024);
        } else {
            to_lds<4, kS * kWaves * 256>(from_s[kS], ssrc[kS], u * kExps, stage + wave * 256);
        }
    }
    template <int From, int To>
    __device__ __forceinline__ void fetch_range(uint32_t u, char* stage) const
    {
        if constexpr (From < To) {
            fetch<From>(u, stage);
            fetch_range<From + 1, To>(u, stage);
        }
    }

    // What a wave holds of four pieces: its rows' and their exponents.
    struct Part {
        v4i a[kMt], b[kNt];
        int sa[Core::kScaled ? kMt : 1], sb[Core::kScaled ? kNt : 1];
    };

    __device__ __forceinline__ void read_a(Part& p, const char* stage, int h, int i) const
    {
        const int r = lane & 15, row = wave / WN * (BM / WM) + r, c = 4 * h + (lane >> 4);
        p.a[i] = *(const v4i*)(stage + row * kSeg + place(r, c) * 16 + (kAtA + i * 16 * kSeg));
        if (Core::kScaled) p.sa[i] = *(const uint8_t*)(stage + row * kExps + c + i * 16 * kExps);
    }
    __device__ __forceinline__ void read_b(Part& p, const char* stage, int h, int j) const
    {
        const int r = lane & 15, row = wave % WN * (BN / WN) + r, c = 4 * h + (lane >> 4);
        p.b[j] = *(const v4i*)(stage + row * kSeg + place(r, c) * 16 + (kAtB + j * 16 * kSeg));
        if (Core::kScaled) p.sb[j] = *(const uint8_t*)(stage + row * kExps + c + (BM + j * 16) * kExps);
    }
    // reads in the order in which the products want them: a's first row, all of b, the rest of a
    __device__ __forceinline__ void read(Part& p, const char* stage, int h, int n) const
    {
        if (n == 0)
            read_a(p, stage, h, 0);
        else if (n <= kNt)
            read_b(p, stage, h, n - 1);
        else
            read_a(p, stage, h, n - kNt);
    }

    // The products of p with the reads of the next four pieces (number h of `stage`) between them, and with Fetch the loads of
    // stage number u to `to`.  A product keeps the matrix unit for 16 cycles and its wave, which is alone on its SIMD, issues
    // something every 4: up to three other instructions go between two products for nothing, a bunch of them stops the unit.
    // So each product is followed by at most one read or load, and the reads come first, for the barrier waits for them.
    template <bool Read, bool Fetch, int N = 0>
    __device__ __forceinline__ void multiply(const Part& p, Part& next, const char* stage, int h, uint32_t u, char* to)
    {
        if constexpr (N < kMt * kNt) {
            constexpr int i = N / kNt, j = N % kNt, kAll = kMt * kNt, kReads = kMt + kNt, kEvery = kAll >= 64 ? 3 : 1;
            static_assert(kReads * kEvery <= kAll || kAll < 64, "a product for each read");
            if (N == 0) settle();
            Core::mul(p.b[j], p.a[i], acc[i][j], p.sb[Core::kScaled ? j : 0], p.sa[Core::kScaled ? i : 0]);
            if (Read && kAll >= 64 && N % kEvery == 0 && N / kEvery < kReads) read(next, stage, h, N / kEvery);
            if (Read && kAll < 64) {
#pragma unroll
                for (int n = N * kReads / kAll; n < (N + 1) * kReads / kAll; ++n) read(next, stage, h, n);
            }
            if constexpr (Fetch && kAll >= 64) {
                static_assert(kLoads * 3 <= kAll + 2, "a product for each load");
                if constexpr (N % 3 == 1 && N / 3 < kLoads) fetch<N / 3>(u, to);
            } else if constexpr (Fetch) {
                fetch_range<N * kLoads / kAll, (N + 1) * kLoads / kAll>(u, to);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply<Read, Fetch, N + 1>(p, next, stage, h, u, to);
        }
    }

    // Works tile after tile of this block's: number blockIdx.x, gridDim.x after that and so on below `tiles`.  A tile's sum is
    // over `Terms` products of operands with the same pitch:
    //   operands(tile, term) takes them (take)
    //   finish(tile)         is called with the sums
    // While four pieces are multiplied the next four are read from LDS into other registers.  Once every wave has read the last
    // of a stage its place is free, and the stage after it has to be there: one barrier a stage.  The stages of all tiles are
    // one sequence: the next tile's are under way while this one's sums go out.  Long says that a
    // finish is long beside the loop's code and that its registers are not to be had from the loop's.
    template <int Terms, class Operands, class Finish>
    __device__ __forceinline__ void run(uint32_t tiles, uint32_t pitch, char* lds, const Operands& operands, const Finish& finish)
    {
        run<Terms>(tiles, Span{pitch, pitch, pitch / kLine}, lds, operands, finish);
    }
    template <int Terms, bool Long = false, class Operands, class Finish>
    __device__ __forceinline__ void run(uint32_t tiles, const Span& span, char* lds, const Operands& operands, const Finish& finish)
    {
        aim(span);
        Sequence coming = {blockIdx.x, 0, 0};  // what is fetched next
        operands(coming.tile, coming.term);
        auto advance = [&] {
            if (!coming.next(stages, Terms, tiles, gridDim.x)) return;
            if (coming.tile < tiles)
                operands(coming.tile, coming.term);
            else
                take_nothing();
        };
#pragma unroll
        for (int s = 0; s < Stages; ++s) {
            fetch_range<0, kLoads>(coming.u, lds + s * kStage);
            advance();
        }
        wait_loads<(Stages - 1) * kLoads>();
        __builtin_amdgcn_s_barrier();
        Part p0, p1;
#pragma unroll
        for (int n = 0; n < kMt + kNt; ++n) read(p0, lds, 0, n);
        char *stage = lds, *const end = lds + kLds;
        auto turn = [&](const Part& p, Part& next, uint32_t all) {
            if (Stages > 2 && !all)
                wait_loads<(Stages - 2) * kLoads>();
            else
                wait_loads<0>();
            __builtin_amdgcn_s_barrier();
            char* to = stage;
            stage = stage + kStage == end ? lds : stage + kStage;
            multiply<true, true>(p, next, stage, 0, coming.u, to);
            advance();
        };
        for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
            clear();
            hold();
            // The last turn of all reads what follows the last stage, which nothing uses.  The first turn waits for
            // everything: stores of the tile before may be counted among the loads.
            uint32_t f = 0, fresh = 1;
            do {
                multiply<true, false>(p0, p1, stage, 1, 0, nullptr);
                turn(p1, p0, fresh);
                fresh = 0;
                asm volatile("" : "+s"(fresh));  // a copy of the loop for its first turn would move the sums
            } while (Long ? __builtin_expect_with_probability(++f < Terms * stages, 1, 0.999) : ++f < Terms * stages);
            rest();
            hold();
            finish(tile);
        }
        wait_loads<0>();
    }

    // f(row, column, 4 values): C's row and the first of four neighbouring columns, relative to the tile.
    template <class F>
    __device__ __forceinline__ void each(const F& f) const
    {
        uint32_t row = wave / WN * (BM / WM) + (lane & 15), col = wave % WN * (BN / WN) + 4 * (lane >> 4);
#pragma unroll
        for (int i = 0; i < kMt; ++i) {
            asm volatile("" : "+v"(row), "+v"(col));  // addresses of later rows are not kept from here on
#pragma unroll
            for (int j = 0; j < kNt; ++j) f(row + i * 16, col + j * 16, acc[i][j]);
        }
    }

    // The sums become f(row, column, sums).
    template <class F>
    __device__ __forceinline__ void become(const F& f)
    {
        uint32_t row = wave / WN * (BM / WM) + (lane & 15), col = wave % WN * (BN / WN) + 4 * (lane >> 4);
#pragma unroll
        for (int i = 0; i < kMt; ++i) {
            asm volatile("" : "+v"(row), "+v"(col));  // addresses of later rows are not kept from here on
#pragma unroll
            for (int j = 0; j < kNt; ++j) acc[i][j] = f(row + i * 16, col + j * 16, acc[i][j]);
        }
    }

    // The lane's row of the first strip, as strips() has it.
    __device__ __forceinline__ uint32_t first_row() const { return wave / WN * (BM / WM) + (threadIdx.x & 15); }

    // f(strip, row, column, sums): the strip's number, C's row and the first of the columns of its kNt sums, which are 16
    // apart; relative to the tile.  f may change the sums.
    template <class F>
    __device__ __forceinline__ void strips(const F& f)
    {
        int lane = this->lane;
        asm volatile("" : "+v"(lane));  // places are not kept from tile to tile
        uint32_t row = wave / WN * (BM / WM) + (lane & 15), col = wave % WN * (BN / WN) + 4 * (lane >> 4);
#pragma unroll
        for (int i = 0; i < kMt; ++i) {
            asm volatile("" : "+v"(row), "+v"(col));  // addresses of later rows are not kept from here on
            f(i, row + i * 16, col, acc[i]);
        }
    }

    // ---- by way of LDS ----
    //
    // A lane holds four neighbouring columns; halves stored like that touch 16 rows with 32 bytes each.  So a wave puts 16 rows
    // (or columns, for the transpose) of its tile at a time into LDS, as S, and reads them back in 16 bytes a lane along the row.

    static constexpr int pad(int bytes) { return bytes + 16; }
    template <class S>
    static constexpr int out_bytes()  // of LDS for each wave, besides the stages
    {
        return 16 * pad((kNt > kMt ? kNt : kMt) * 16 * (int)sizeof(S));
    }

    // The tile from 16-bit numbers in registers, v[i][j] in the place of acc[i][j]; store(row, column, 16 bytes) as below.
    template <bool Turn, class Store>
    __device__ __forceinline__ void out16(char* lds, const Four16 (&v)[kMt][kNt], const Store& store) const
    {
        constexpr int kStrips = Turn ? kNt : kMt, kTiles = Turn ? kMt : kNt, kPitch = pad(kTiles * 32), kLanes = kTiles * 2;
        static_assert(16 * kLanes % 64 == 0, "whole waves");
        int lane = this->lane;
        asm volatile("" : "+v"(lane));  // nor are places kept from tile to tile
        char* mine = lds + wave * out_bytes<_Float16>();
        const int r = lane & 15, q = lane >> 4;
        uint32_t row0 = wave / WN * (BM / WM), col0 = wave % WN * (BN / WN);
#pragma unroll
        for (int x = 0; x < kStrips; ++x) {
            asm volatile("" : "+v"(row0), "+v"(col0));  // addresses of later strips are not kept from here on
#pragma unroll
            for (int y = 0; y < kTiles; ++y) {
                if (Turn)
                    *(Four16*)(mine + (4 * q + (r & 3)) * kPitch + (y * 16 + (r & ~3)) * 2) = turned(v[y][x]);
                else
                    *(Four16*)(mine + r * kPitch + (y * 16 + 4 * q) * 2) = v[x][y];
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int k = 0; k < 16 * kLanes / 64; ++k) {
                const int at = k * 64 + lane, row = at / kLanes, col = at % kLanes * 8;
                store((uint32_t)((Turn ? col0 : row0) + x * 16 + row), (uint32_t)((Turn ? row0 : col0) + col), *(const v4i*)(mine + row * kPitch + col * 2));
            }
            __builtin_amdgcn_wave_barrier();
        }
    }

    // value(row, column, sums) gives the four values of C's row from a column on; store(row, column, 16 bytes of S) takes
    // neighbours of a row - with Turn of a column: row and column are C's, exchanged.  All relative to the tile.  `lds`
    // has out_bytes<S>() for each wave.
    template <class S, bool Turn, class Value, class Store>
    __device__ __forceinline__ void out(char* lds, const Value& value, const Store& store)
    {
        hold();  // what an earlier way out has computed of them is not kept
        constexpr int kStrips = Turn ? kNt : kMt, kTiles = Turn ? kMt : kNt, kPitch = pad(kTiles * 16 * (int)sizeof(S));
        constexpr int kPer = 16 / (int)sizeof(S), kLanes = kTiles * 16 / kPer;  // lanes of a row
        static_assert(16 * kLanes % 64 == 0, "whole waves");
        typedef S s4 __attribute__((ext_vector_type(4)));
        typedef S sv __attribute__((ext_vector_type(kPer)));
        char* mine = lds + wave * out_bytes<S>();
        const int r = lane & 15, q = lane >> 4;
        uint32_t row0 = wave / WN * (BM / WM), col0 = wave % WN * (BN / WN);
#pragma unroll
        for (int x = 0; x < kStrips; ++x) {
            asm volatile("" : "+v"(row0), "+v"(col0));  // addresses of later strips are not kept from here on
#pragma unroll
            for (int y = 0; y < kTiles; ++y) {
                const int i = Turn ? y : x, j = Turn ? x : y;
                v4f v = rounded(value((uint32_t)(row0 + i * 16 + r), (uint32_t)(col0 + j * 16 + 4 * q), acc[i][j]));
                if (Turn) v = turned(v);
                const s4 w = {(S)v[0], (S)v[1], (S)v[2], (S)v[3]};
                if (Turn)
                    *(s4*)(mine + (4 * q + (r & 3)) * kPitch + (y * 16 + (r & ~3)) * (int)sizeof(S)) = w;
                else
                    *(s4*)(mine + r * kPitch + (y * 16 + 4 * q) * (int)sizeof(S)) = w;
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int k = 0; k < 16 * kLanes / 64; ++k) {
                const int at = k * 64 + lane, row = at / kLanes, col = at % kLanes * kPer;
                store((uint32_t)((Turn ? col0 : row0) + x * 16 + row), (uint32_t)((Turn ? row0 : col0) + col),
                      *(const sv*)(mine + row * kPitch + col * (int)sizeof(S)));
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
};

// ---- which tile ----
//
// A product's time is the rounds of its tiles by what a line of the rows takes in each, and what a round and the launch take
// besides (first loads, stores).  Large tiles read less for an operation, small ones leave less of the last round empty and
// are done sooner where there are few.  Measured on 4-bit products with one tile for all, us, tiles of 256, 192, 128, 64:
//   8192 x 8192 x 8192 258 313 356 605; 4096 x 4096 x 25088 185 234 270 506; 4096 x 25088 x 4096 (fp32) 281 308 392 718;
//   3000 x 3000 x 4096 35.4 27.7 39.2 46.2; 2048 x 2048 x 2048 23.1 17.9 12.1 14.7; 1024 x 1024 x 1024 16.8 12.3 8.9 8.7;
//   700 x 1500 x 6000 39.7 29.0 20.5 16.4; 6000 x 1500 x 700 18.0 15.0 15.0 15.5; 100 x 4096 x 4096 30.3 22.5 14.1 9.1.
struct TileCost {
    int side, per_cu;
    float alone, line;    // us a line of 128 bytes, one tile to a CU or per_cu of them
    float round, launch;  // us besides
};
constexpr TileCost kTileCosts[] = {{256, 1, 1.55f, 1.75f, 7.0f, 10.0f}, {192, 1, 1.05f, 1.10f, 6.0f, 8.0f}, {128, 2, 0.80f, 1.25f, 2.5f, 5.5f}, {64, 2, 0.25f, 0.58f, 2.0f, 4.5f}};
constexpr int kCus = 256;

inline double tile_time(int pick, int64_t tiles, int64_t lines)
{
    const TileCost& c = kTileCosts[pick];
    const int64_t slots = (int64_t)kCus * c.per_cu, left = tiles % slots;
    double t = c.launch + (double)(tiles / slots) * (lines * c.line + c.round);
    if (left) t += lines * (left <= kCus ? c.alone : c.line) + c.round;
    return t;
}

// count(side): tiles of the whole launch.  Returns an index of kTileCosts.
template <class Count>
inline int best_tile(const Count& count, int64_t lines, double* time = nullptr)
{
    int best = 0;
    double least = 0.0;
    for (int i = 0; i < 4; ++i) {
        const double t = tile_time(i, count(kTileCosts[i].side), lines);
        if (i == 0 || t < least) least = t, best = i;
    }
    if (time) *time = least;
    return best;
}

// Tiles on and below the diagonal of an m x m matrix, and the tile for `count` such matrices.
inline int64_t triangle_tiles(int64_t m, int64_t side)
{
    const int64_t k = (m + side - 1) / side;
    return k * (k + 1) / 2;
}
inline int best_triangle(int64_t m, int64_t count, int64_t lines)
{
    return best_tile([&](int64_t side) { return triangle_tiles(m, side) * count; }, lines);
}

// A batch of m x n products in one launch or two: the first n columns in as many large tiles as fill whole rounds, and the rest
// in tiles of its own.  4096 x 25088 in tiles of 256 is 6.1 rounds, done in 7.
struct TilePlan {
    int pick, rest_pick;
    int64_t columns;  // of the first launch
};
inline TilePlan plan_tiles(int64_t m, int64_t n, int64_t batch, int64_t lines)
{
    auto tiles = [&](int64_t cols, int64_t side) { return (m + side - 1) / side * ((cols + side - 1) / side) * batch; };
    double least = 0.0;
    TilePlan plan = {best_tile([&](int64_t side) { return tiles(n, side); }, lines, &least), 0, n};
    for (int i = 0; i < 2; ++i) {
        const int64_t side = kTileCosts[i].side, strip = (m + side - 1) / side * batch, slots = (int64_t)kCus * kTileCosts[i].per_cu;
        const int64_t columns = tiles(n, side) / slots * slots / strip * side;
        if (columns <= 0 || columns >= n) continue;
        double rest = 0.0;
        const int rest_pick = best_tile([&](int64_t s) { return tiles(n - columns, s); }, lines, &rest);
        const double t = tile_time(i, tiles(columns, side), lines) + rest;
        if (t < least) least = t, plan = {i, rest_pick, columns};
    }
    return plan;
}

// Blocks of a launch of that many tiles: each works one after the other.
inline uint32_t tile_blocks(int pick, int64_t tiles)
{
    const int64_t most = (int64_t)kCus * kTileCosts[pick].per_cu;
    return (uint32_t)(tiles < most ? tiles : most);
}

}  // namespace sidco
#endif
