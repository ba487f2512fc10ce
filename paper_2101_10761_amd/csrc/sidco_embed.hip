// The embedding: rows of a table by their words, times a scale, and the table's gradient.
//
// The gradient adds up the rows of each word.  Places are first sorted by their words, places of the same word in order, so
// that a word's sum is formed in one order whatever runs when, without atomics: a wave walks along sorted places with the sum
// of its columns in registers and writes a row when the word changes.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "sidco_elements.h"

namespace sidco {
namespace {

// ---- the lookup ----

template <class I, class T, class R>
struct Look {
    const void* words;
    int64_t n;
    uint32_t vocab;
    const T* table;
    R* rows;
    int64_t ldt, ldr, cols;
    float scale;
    int lanes;
};

// Bound by memory: 65536 rows of 4096 in bf16, of 131072, 166 us for 0.79 GB of distinct rows and results, 4.8 TB/s (a copy reaches
// 4.8 to 5.0); 700 of 1500 in fp32 4.0 us, a launch and two trips to memory.  Each: rows that a thread has under way at once, four
// where there are blocks enough for it (197 to 160 us for the first of these), else one.
template <class I, class T, class R, int Each>
__global__ __launch_bounds__(kRowBlock) void k_embedding(Look<I, T, R> p)
{
    const int lane = threadIdx.x & (p.lanes - 1);
    const int64_t per = kRowBlock / p.lanes, step = (int64_t)gridDim.x * per;
    for (int64_t i = (int64_t)blockIdx.x * per + threadIdx.x / p.lanes; i < p.n; i += step * Each) {
        uint32_t word[Each];
#pragma unroll
        for (int e = 0; e < Each; ++e) word[e] = i + e * step < p.n ? word_at<I>(p.words, i + e * step, p.vocab) : p.vocab;
        for (int64_t c = ((int64_t)blockIdx.y * p.lanes + lane) * 8; c < p.cols; c += (int64_t)gridDim.y * p.lanes * 8) {
            Eight<T> t[Each];
#pragma unroll
            for (int e = 0; e < Each; ++e)
                if (word[e] < p.vocab) t[e].load(p.table + (int64_t)word[e] * p.ldt + c, p.cols - c);
#pragma unroll
            for (int e = 0; e < Each; ++e) {
                Eight<R> r;
#pragma unroll
                for (int k = 0; k < 8; ++k) r.set(k, word[e] < p.vocab ? t[e].get(k) * p.scale : 0.0f);
                if (i + e * step < p.n) r.store(p.rows + (i + e * step) * p.ldr + c, p.cols - c);
            }
        }
    }
}

// ---- places sorted by their words ----
//
// Runs of kRun places are sorted by counting: a place's rank in its run is the number of places with a smaller word, and of
// the same word before it.  All comparisons are independent of each other, kRun a place, so that one launch of many small
// blocks does them.  Then up to kWays neighbouring runs are merged at a time: a place moves up by the number of places of
// each other run that come before it, which a search in that run finds.  65536 places 13.3 + 15.7 us.  Up to kLongRun places are one
// run: 4099 6.7 us, with runs of kRun 5.3 + 6.8.
constexpr int kRun = 2048, kLongRun = 8192, kWays = 32;
constexpr int kSortLanes = 16;  // lanes that share the comparisons of a place

struct Sorted {
    uint32_t* word;
    uint32_t* place;
};

// Each: places that a group of lanes ranks at once; Run: places of a run.
template <class I, int Each, int Run>
__global__ __launch_bounds__(256) void k_sort_run(const void* words, int64_t n, uint32_t vocab, Sorted out)
{
    constexpr int kPlaces = 256 / kSortLanes * Each;  // of a block, within one chunk of 64
    static_assert(64 % kPlaces == 0, "a block's places lie in one chunk");
    const int64_t first = (int64_t)blockIdx.x * kPlaces, run = first / Run * Run;
    const int64_t len = n - run < Run ? n - run : Run;
    __shared__ __align__(16) uint32_t keys[Run];
    uint32_t own[Run / 256];
#pragma unroll
    for (int k = 0; k < Run / 256; ++k) {
        const int j = k * 256 + threadIdx.x;
        own[k] = word_at<I>(words, run + (j < len ? j : len - 1), vocab);  // without a branch, which would wait for each
        own[k] = j < len ? own[k] : ~0u;
    }
#pragma unroll
    for (int k = 0; k < Run / 256; ++k) keys[k * 256 + threadIdx.x] = own[k];
    __syncthreads();
    const int lane = threadIdx.x % kSortLanes, group = threadIdx.x / kSortLanes;
    uint32_t mine[Each], rank[Each];
    int at[Each];
#pragma unroll
    for (int e = 0; e < Each; ++e) {
        at[e] = (int)(first - run) + group * Each + e;
        mine[e] = keys[at[e]];
        rank[e] = 0;
    }
    // chunks of 64: before the block's own the same word counts, behind it not
    const int chunk = (int)(first - run) / 64, chunks = (int)((len + 63) / 64);
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    const u4* list = (const u4*)keys + lane;
#pragma unroll 4
    for (int k = 0; k < chunk; ++k) {
        const u4 v = list[k * 16];
#pragma unroll
        for (int e = 0; e < Each; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) rank[e] += v[i] <= mine[e];
    }
    const u4 v = list[chunk * 16];
#pragma unroll
    for (int e = 0; e < Each; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) rank[e] += v[i] < mine[e] || (v[i] == mine[e] && chunk * 64 + lane * 4 + i < at[e]);
#pragma unroll 4
    for (int k = chunk + 1; k < chunks; ++k) {
        const u4 v = list[k * 16];
#pragma unroll
        for (int e = 0; e < Each; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) rank[e] += v[i] < mine[e];
    }
#pragma unroll
    for (int e = 0; e < Each; ++e) {
#pragma unroll
        for (int s = kSortLanes / 2; s > 0; s >>= 1) rank[e] += __shfl_xor(rank[e], s);
        if (lane == 0 && at[e] < len) {
            out.word[run + rank[e]] = mine[e];
            out.place[run + rank[e]] = (uint32_t)(run + at[e]);
        }
    }
}

// Runs of `len` places, kWays of them to one.  A wave searches four runs at a time for 64 neighbours of one run, whose places
// there lie close together; eight waves share the runs.  (With a lane for each run, whose probes meet no line together, 39.7 us.)
constexpr int kMergeWaves = 8, kMergeEach = kWays / kMergeWaves;
__global__ __launch_bounds__(64 * kMergeWaves) void k_merge(Sorted in, Sorted out, int64_t n, int64_t len)
{
    __shared__ uint32_t counts[kMergeWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = (int64_t)blockIdx.x * 64, all = first / (len * kWays) * (len * kWays), own = first / len * len;
    const int64_t i = first + lane < n ? first + lane : n - 1;
    const uint32_t word = in.word[i];
    // places of each run which come first: smaller words, and of runs before this one's the same word too
    const uint32_t* run[kMergeEach];
    uint32_t count[kMergeEach], below[kMergeEach], before[kMergeEach];
#pragma unroll
    for (int k = 0; k < kMergeEach; ++k) {
        const int64_t start = all + (wave * kMergeEach + k) * len, left = n - start;
        run[k] = in.word + start;
        count[k] = start == own || left <= 0 ? 0 : (uint32_t)(left < len ? left : len);
        below[k] = word + (start < own ? 1 : 0);
        before[k] = 0;
    }
    for (uint32_t step = (uint32_t)len; step > 0; step >>= 1) {  // len is a power of two
        uint32_t seen[kMergeEach];
#pragma unroll
        for (int k = 0; k < kMergeEach; ++k) {
            const uint32_t to = before[k] + step;
            seen[k] = to <= count[k] ? run[k][to - 1] : ~0u;
        }
#pragma unroll
        for (int k = 0; k < kMergeEach; ++k) before[k] += seen[k] < below[k] ? step : 0;
    }
    uint32_t sum = 0;
#pragma unroll
    for (int k = 0; k < kMergeEach; ++k) sum += before[k];
    counts[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && first + lane < n) {
        uint32_t to = (uint32_t)(i - own);
#pragma unroll
        for (int k = 0; k < kMergeWaves; ++k) to += counts[k][lane];
        out.word[all + to] = word;
        out.place[all + to] = in.place[i];
    }
}

// ---- the sums ----

constexpr int kStrip = 512;  // columns of a wave
constexpr int kFillRows = 16;
constexpr int kSumBlock = 512;  // threads of a block that adds up or fills rows
// Of one of k_sum's that only adds up: 4099 rows of 1111 fp16 19.7 us with 256 and 20.4 with 512, 8192 of 4096 bf16 onto fp32 48.9 and
// 53.5; with rows to be filled in the same launch, 65536 of 4096, 568 and 549.
constexpr int kAddBlock = 256;

template <class G, class T>
struct Sum {
    Sorted sorted;
    int64_t n;
    uint32_t vocab;
    const G* rows;
    T* table;
    int64_t ldr, ldt, cols, strips;
    float scale;
    bool accumulate;
    int chunk;        // sorted places of a wave
    int64_t chunks;
    float* partial;   // two rows of `cols` for each chunk
    int64_t sum_blocks;
};

template <class T>
__device__ __forceinline__ void put_row(T* to, const float (&sum)[8], float scale, bool accumulate, int64_t left)
{
    Eight<T> t;
    if (accumulate) t.load(to, left);
#pragma unroll
    for (int k = 0; k < 8; ++k) t.set(k, accumulate ? fmaf(scale, sum[k], t.get(k)) : scale * sum[k]);
    t.store(to, left);
}

// Zeros for those of the kFillRows rows from v0 on that are not present.  Past the caches: they are more than these hold, and with
// ordinary stores the rows that other blocks of the launch wait for came later (700 words into 10000 x 1500 fp32, whole call, 21.0
// us; so 15.1).
template <class G, class T>
__device__ __forceinline__ void fill_rows(const Sum<G, T>& p, int64_t v0, const int* present)
{
    typedef typename Eight<T>::part part;
    constexpr int kPer = Eight<T>::kPer;
    for (int r = threadIdx.x >> 6; r < kFillRows && v0 + r < p.vocab; r += kSumBlock / 64) {
        if (present[r]) continue;
        T* to = p.table + (v0 + r) * p.ldt;
        const int64_t whole = p.cols / kPer * kPer;
        const part zeros = {};
        for (int64_t c = (threadIdx.x & 63) * kPer; c < whole; c += 64 * kPer) __builtin_nontemporal_store(zeros, (part*)(to + c));
        if (whole + (threadIdx.x & 63) < p.cols) to[whole + (threadIdx.x & 63)] = (T)0.0f;
    }
}

// The same, from the sorted places: 32 lanes search for the first place of a word, 32 probes at a time.
template <class G, class T>
__device__ __forceinline__ void fill_missing(const Sum<G, T>& p, int64_t v0)
{
    constexpr int kLanes = kSumBlock / kFillRows;
    static_assert(kLanes <= 32 && 64 % kLanes == 0, "a row's lanes are a wave's");
    __shared__ int present[kFillRows];
    const int row = threadIdx.x / kLanes, lane = threadIdx.x % kLanes, shift = threadIdx.x % 64 / kLanes * kLanes;
    const uint32_t word = (uint32_t)(v0 + row);
    int64_t lo = 0, hi = p.n;  // it is in [lo, hi]
    while (__any(hi > lo)) {
        const int64_t step = (hi - lo + kLanes - 1) / kLanes, at = lo + lane * step;
        const bool less = at < hi && p.sorted.word[at] < word;
        const int count = __popc((uint32_t)(__ballot(less) >> shift) & (uint32_t)((1ull << kLanes) - 1));  // the first probes
        if (count == 0) {
            hi = lo;
        } else {
            const int64_t end = lo + count * step;
            lo += (count - 1) * step + 1;
            hi = end < hi ? end : hi;
        }
    }
    if (lane == 0) present[row] = lo < p.n && p.sorted.word[lo] == word;
    __syncthreads();
    fill_rows(p, v0, present);
    __syncthreads();
}

// The sum of the rows at `count` places, in their order; eight of them are read at a time.
template <class G, class T>
__device__ __forceinline__ void sum_rows(const Sum<G, T>& p, const uint16_t* places, int count, int64_t c, int64_t left, float (&sum)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
    if (left <= 0) return;
    for (int i = 0; i < count; i += 8) {
        Eight<G> g[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i + u < count) g[u].load(p.rows + (int64_t)places[i + u] * p.ldr + c, left);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i + u < count) {
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] += g[u].get(k);
            }
    }
}

// How many sorted places from `at` on, `stride` apart and before `end`, have that word.
__device__ __forceinline__ int64_t length_of(const uint32_t* word, int64_t at, int64_t stride, int64_t end, uint32_t of)
{
    int64_t count = 0;
    for (;;) {
        const int64_t i = at + (count + (threadIdx.x & 63)) * stride;
        const int same = __popcll(__ballot(i < end && word[i] == of));  // sorted: the first of them
        count += same;
        if (same < 64) return count;
    }
}

// The waves' sums added up in order; the whole is wave 0's.
template <int Waves = kSumBlock / 64>
__device__ __forceinline__ void join_waves(float (&sum)[8], float (*lds)[64][9])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) lds[wave][lane][k] = sum[k];
    __syncthreads();
    if (wave == 0) {
        for (int w = 1; w < Waves; ++w)
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += lds[w][lane][k];
    }
}

// Few places, in one launch and without a workspace: every block has all words in LDS.  A wave looks at a place, and if its word
// occurs at no place before it, lists the word's places and adds up their rows; a word of many places is taken by the block's
// waves together.  Bound by the table's writes and by the chain of words, list, rows: whole calls for 10000 x 1500 fp32, 1, 700, 1024 and
// 2048 words 14.3, 14.3, 16.1 and 20.8 us, where torch's zeros alone take 10.6; 2049 words, sorted, 23.8.  Onto 50000 x 1024 bf16 700, 2048
// and 2049 words 6.3, 12.4 and 14.7.
constexpr int kFewPlaces = kSumBlock / 64;     // of a block
constexpr int kAlone = 16, kListed = 64;       // of a wave, and those that it lists

// Places of `word`: their number and, in order, the first `room` of them; -1 where one lies before `at`.  Keys behind the last are
// no word.
__device__ __forceinline__ int list_places(const uint32_t* keys, int n, uint32_t word, int at, uint16_t* list, int room)
{
    const int lane = threadIdx.x & 63;
    int count = 0;
    for (int j = 0; j < n; j += 256) {
        uint64_t same[4];
        uint32_t key[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) key[k] = keys[j + k * 64 + lane];
#pragma unroll
        for (int k = 0; k < 4; ++k) same[k] = __ballot(key[k] == word);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (same[k] == 0) continue;
            if (count == 0 && j + k * 64 + __builtin_ctzll(same[k]) < at) return -1;
            const int to = count + __popcll(same[k] & ((1ull << lane) - 1));
            if (same[k] >> lane & 1 && to < room) list[to] = (uint16_t)(j + k * 64 + lane);
            count += __popcll(same[k]);
        }
    }
    return count;
}

template <class I, class G, class T>
__global__ __launch_bounds__(kSumBlock) void k_sum_few(Sum<G, T> p, const void* words)
{
    __shared__ uint32_t keys[kRun];
    __shared__ float lds[kSumBlock / 64][64][9];
    __shared__ uint16_t list[kFewPlaces][kListed], all[kRun];
    __shared__ int many[kFillRows];
    const int n = (int)p.n;
    uint32_t own[kRun / kSumBlock];
#pragma unroll
    for (int k = 0; k < kRun / kSumBlock; ++k) {
        const int j = k * kSumBlock + threadIdx.x;
        own[k] = word_at<I>(words, j < n ? j : n - 1, p.vocab);
        own[k] = j < n ? own[k] : p.vocab;
    }
    if (blockIdx.x >= p.sum_blocks) {
        for (int64_t v0 = (int64_t)(blockIdx.x - p.sum_blocks) * kFillRows; v0 < p.vocab; v0 += (int64_t)(gridDim.x - p.sum_blocks) * kFillRows) {
            if (threadIdx.x < kFillRows) many[threadIdx.x] = 0;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kRun / kSumBlock; ++k)
                if (own[k] < p.vocab && own[k] - (uint32_t)v0 < kFillRows) many[own[k] - (uint32_t)v0] = 1;
            __syncthreads();
            fill_rows(p, v0, many);
            __syncthreads();
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < kRun / kSumBlock; ++k) keys[k * kSumBlock + threadIdx.x] = own[k];
    __syncthreads();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = (int)(blockIdx.x / p.strips) * kFewPlaces, at = first + wave;
    const int64_t c = blockIdx.x % p.strips * kStrip + (threadIdx.x & 63) * 8, left = p.cols - c;
    float sum[8];
    int count = 0;
    if (at < n && keys[at] < p.vocab) {
        const uint32_t word = keys[at];
        count = list_places(keys, n, word, at, list[wave], kListed);
        __builtin_amdgcn_wave_barrier();
        if (count > 0 && count <= kAlone) {
            sum_rows(p, list[wave], count, c, left, sum);
            if (left > 0) put_row(p.table + (int64_t)word * p.ldt + c, sum, p.scale, p.accumulate, left);
        }
    }
    if ((threadIdx.x & 63) == 0) many[wave] = count > kAlone ? count : 0;
    __syncthreads();
    for (int k = 0; k < kFewPlaces; ++k) {
        const int count = many[k];
        if (count == 0) continue;
        const uint32_t word = keys[first + k];
        if (count > kListed) {
            if (wave == 0) list_places(keys, n, word, first + k, all, kRun);
            __syncthreads();
        }
        const int each = (count + kSumBlock / 64 - 1) / (kSumBlock / 64), from = wave * each, rest = count - from;
        sum_rows(p, (count > kListed ? all : list[k]) + from, rest < each ? rest : each, c, left, sum);
        join_waves(sum, lds);
        if (wave == 0 && left > 0) put_row(p.table + (int64_t)word * p.ldt + c, sum, p.scale, p.accumulate, left);
    }
}

// Many places: a wave adds up the rows of `chunk` sorted ones in one strip of columns.  A word whose places all lie in the chunk
// is done; the sums of one that began before it or goes on after it are kept for k_join.  Bound by memory: 65536 rows of 4096 in
// bf16 into 131072 in fp32, 486 to 502 us for 2.7 GB, 5.4 to 5.6 TB/s.
//
// Where waves are few it is the chain of loads that counts: the chunk's words and places come with one load of the wave, and the
// rows of eight places, and of the table if it is added to, are under way together, with nothing between them that waits: 4099 rows of
// 1111 onto a table, fp16, 8.2 us, where a wait for each word, place and row took 16.3.
// So a lane at the row's end takes its last eight columns, some of which are its neighbour's and not stored again.
template <class G, class T, bool Accumulate>
__global__ __launch_bounds__(Accumulate ? kAddBlock : kSumBlock) void k_sum(Sum<G, T> p)
{
    constexpr int kWaves = (Accumulate ? kAddBlock : kSumBlock) / 64;
    if (!Accumulate && blockIdx.x >= p.sum_blocks) {
        for (int64_t v0 = (int64_t)(blockIdx.x - p.sum_blocks) * kFillRows; v0 < p.vocab; v0 += (int64_t)(gridDim.x - p.sum_blocks) * kFillRows)
            fill_missing(p, v0);
        return;
    }
    const int64_t item = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t chunk = item / p.strips, strip = item % p.strips;
    if (chunk >= p.chunks) return;
    const int64_t from = chunk * p.chunk;
    const int lane = threadIdx.x & 63, count = (int)(from + p.chunk < p.n ? p.chunk : p.n - from);
    // of places from - 1 to from + 62
    const int64_t mine = from - 1 + lane, real = mine < 0 ? 0 : (mine < p.n ? mine : p.n - 1);
    const uint32_t words = p.sorted.word[real], places = p.sorted.place[real];
    const uint32_t kept = mine == real ? words : ~0u;
    auto word_at = [&](int k) { return (uint32_t)__builtin_amdgcn_readlane((int)kept, k + 1); };
    auto place_at = [&](int k) { return (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)places, k + 1); };
    if (word_at(0) >= p.vocab) return;  // padding comes last
    const int64_t c = strip * kStrip + lane * 8;
    auto walk = [&](auto narrow) {
        constexpr bool kNarrow = decltype(narrow)::value;  // less than eight columns
        const int64_t at = kNarrow || c < p.cols - 8 ? c : p.cols - 8, left = c < p.cols ? p.cols - c : 0;
        auto load = [&](auto& e, auto* row) {
            if constexpr (kNarrow)
                e.load(row, left);
            else
                e.load(row + at);
        };
        auto store = [&](const auto& e, auto* row) {
            if constexpr (kNarrow)
                e.store(row, left);
            else if (left >= 8)
                e.store(row + at);
            else
                e.store_last(row + at, left);
        };
        float sum[8] = {};
        bool head = word_at(0) == word_at(-1);  // the sum began in an earlier chunk
        for (int base = 0; base < count; base += 8) {
            Eight<G> g[8];
            Eight<T> old[8];
            // behind the chunk's last place, or among padding, these are rows that are not used
#pragma unroll
            for (int u = 0; u < 8; ++u) load(g[u], p.rows + place_at(base + u) * p.ldr);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (Accumulate && word_at(base + u) < p.vocab && word_at(base + u + 1) != word_at(base + u))
                    load(old[u], (const T*)p.table + (int64_t)word_at(base + u) * p.ldt);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint32_t word = word_at(base + u);
                if (base + u >= count || word >= p.vocab) return;
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] += g[u].get(k);
                const bool same = word_at(base + u + 1) == word, last = base + u + 1 == count;
                if (same && !last) continue;
                if (head || same) {
                    Eight<float> f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) f.set(k, sum[k]);
                    store(f, p.partial + (chunk * 2 + (head ? 0 : 1)) * p.cols);
                } else {
                    Eight<T> t;
#pragma unroll
                    for (int k = 0; k < 8; ++k) t.set(k, Accumulate ? fmaf(p.scale, sum[k], old[u].get(k)) : p.scale * sum[k]);
                    store(t, p.table + (int64_t)word * p.ldt);
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
                head = false;
            }
        }
    };
    if (p.cols < 8)
        walk(std::true_type());
    else
        walk(std::false_type());
}

// The sums of words whose places lie in several chunks: a block for each strip and chunk in which one begins.  Bound by the launch of
// its blocks, most of which have nothing to do: 22.7 us for the case above (35 with blocks of eight waves).
constexpr int kJoinWaves = 4;
template <class G, class T>
__global__ __launch_bounds__(64 * kJoinWaves) void k_join(Sum<G, T> p)
{
    const int64_t chunk = blockIdx.x / p.strips, from = chunk * p.chunk, to = from + p.chunk;
    const uint32_t word = p.sorted.word[to - 1], next = p.sorted.word[to], first_word = p.sorted.word[from];
    const uint32_t before = p.sorted.word[from > 0 ? from - 1 : 0];
    if (word >= p.vocab || next != word) return;                            // none goes on
    if (first_word == word && from > 0 && before == word) return;           // it began before
    __shared__ float lds[kJoinWaves][64][9];
    const int64_t c = blockIdx.x % p.strips * kStrip + (threadIdx.x & 63) * 8, left = p.cols - c;
    const int64_t count = 1 + length_of(p.sorted.word, to, p.chunk, p.n, word);  // partial sums, of this chunk the second
    const int64_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), each = (count + kJoinWaves - 1) / kJoinWaves;
    const int64_t first = wave * each, end = first + each < count ? first + each : count;
    float sum[8] = {};
    if (left > 0) {
        for (int64_t i = first; i < end; i += 4) {
            Eight<float> f[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u < end) f[u].load(p.partial + ((chunk + i + u) * 2 + (i + u == 0 ? 1 : 0)) * p.cols + c, left);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u < end) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum[k] += f[u].get(k);
                }
        }
    }
    join_waves<kJoinWaves>(sum, lds);
    if (wave == 0 && left > 0) put_row(p.table + (int64_t)word * p.ldt + c, sum, p.scale, p.accumulate, left);
}

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Sorted places of a wave: fewer where there would not be waves enough, for four times the partial sums at most.
int chunk_of(int64_t n, int64_t cols) { return n * ((cols + kStrip - 1) / kStrip) < 65536 ? 8 : 32; }

// Words and places, twice where they are merged, and the partial sums.
struct SumLayout {
    int64_t each, partial, total;
    SumLayout(int64_t n, int64_t cols)
    {
        each = up(n * 4, 256);
        const int64_t chunks = (n + chunk_of(n, cols) - 1) / chunk_of(n, cols);
        partial = up(chunks * 2 * cols * 4, 256);
        total = n > kRun ? each * 4 + partial : 0;
    }
};

}  // namespace

void launch_embedding(const Lookup& q, hipStream_t s)
{
    const RowGrid g(q.cols);
    const bool many = q.words.n / g.per >= 8192;  // blocks enough for four rows each
    const int64_t blocks = (q.words.n + g.per * (many ? 4 : 1) - 1) / (g.per * (many ? 4 : 1)), across = (q.cols + g.lanes * 8 - 1) / (g.lanes * 8);
    const dim3 grid((uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20), (uint32_t)(across < 65535 ? across : 65535));
    by_word(q.words, [&](auto i) {
        by_element(q.table.type, [&](auto t) {
            by_element(q.rows.type, [&](auto r) {
                typedef decltype(i) I;
                typedef typename decltype(t)::T T;
                typedef typename decltype(r)::T R;
                const Look<I, T, R> p = {q.words.at, q.words.n, (uint32_t)q.words.vocab, (const T*)q.table.at, (R*)q.rows.at,
                                         q.table.ld, q.rows.ld, q.cols, q.scale, g.lanes};
                if (many)
                    k_embedding<I, T, R, 4><<<grid, kRowBlock, 0, s>>>(p);
                else
                    k_embedding<I, T, R, 1><<<grid, kRowBlock, 0, s>>>(p);
            });
        });
    });
}

// A launch has less than 2^32 threads.  Blocks that fill rows, kMostFill at most, take more than kFillRows of them in a table of
// more than 33 million.
constexpr int64_t kMostBlocks = 1 << 22, kMostFill = 1 << 21;
bool embedding_grad_fits(int64_t n, int64_t cols)
{
    const int64_t chunk = n <= kRun ? kFewPlaces : chunk_of(n, cols);
    return (n + chunk - 1) / chunk * ((cols + kStrip - 1) / kStrip) <= kMostBlocks;
}

size_t embedding_grad_scratch(int64_t n, int64_t cols) { return (size_t)SumLayout(n, cols).total; }

void launch_embedding_grad(const Lookup& q, char* scratch, hipStream_t s)
{
    const int64_t n = q.words.n, strips = (q.cols + kStrip - 1) / kStrip, waves = (q.accumulate ? kAddBlock : kSumBlock) / 64;
    const int64_t fill = q.accumulate ? 0 : std::min((q.words.vocab + kFillRows - 1) / kFillRows, kMostFill);
    const bool few = n <= kRun;
    const SumLayout l(n, q.cols);
    Sorted now = {(uint32_t*)scratch, (uint32_t*)(scratch + l.each)};
    Sorted other = {(uint32_t*)(scratch + 2 * l.each), (uint32_t*)(scratch + 3 * l.each)};
    float* partial = (float*)(scratch + 4 * l.each);
    by_word(q.words, [&](auto i) {
        typedef decltype(i) I;
        if (!few && n <= kLongRun)
            k_sort_run<I, 1, kLongRun><<<(uint32_t)((n + 15) / 16), 256, 0, s>>>(q.words.at, n, (uint32_t)q.words.vocab, now);
        else if (!few)
            k_sort_run<I, 4, kRun><<<(uint32_t)((n + 63) / 64), 256, 0, s>>>(q.words.at, n, (uint32_t)q.words.vocab, now);
        for (int64_t len = n <= kLongRun ? kLongRun : kRun; len < n; len *= kWays) {
            k_merge<<<(uint32_t)((n + 63) / 64), 64 * kMergeWaves, 0, s>>>(now, other, n, len);
            std::swap(now, other);
        }
        by_element(q.rows.type, [&](auto g) {
            by_element(q.table.type, [&](auto t) {
                typedef typename decltype(g)::T G;
                typedef typename decltype(t)::T T;
                const int chunk = few ? kFewPlaces : chunk_of(n, q.cols);
                const int64_t chunks = (n + chunk - 1) / chunk, blocks = few ? chunks * strips : (chunks * strips + waves - 1) / waves;
                const Sum<G, T> p = {now, n, (uint32_t)q.words.vocab, (const G*)q.rows.at, (T*)q.table.at, q.rows.ld, q.table.ld, q.cols, strips,
                                     q.scale, q.accumulate, chunk, chunks, partial, blocks};
                if (few) {
                    k_sum_few<I, G, T><<<(uint32_t)(blocks + fill), kSumBlock, 0, s>>>(p, q.words.at);
                    return;
                }
                if (q.accumulate)
                    k_sum<G, T, true><<<(uint32_t)blocks, kAddBlock, 0, s>>>(p);
                else
                    k_sum<G, T, false><<<(uint32_t)(blocks + fill), kSumBlock, 0, s>>>(p);
                k_join<G, T><<<(uint32_t)((chunks - 1) * strips), 64 * kJoinWaves, 0, s>>>(p);
            });
        });
    });
}

}  // namespace sidco
