// The embedding: rows of a table by their words, times a scale, and the table's gradient.
//
// The gradient adds up the rows of each word.  Places are first sorted by their words, places of the same word in order, so
// that a word's sum is formed in one order whatever runs when, without atomics: a wave walks along sorted places with the sum
// of its columns in registers and writes a row when the word changes.
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

template <class I, class T, class R>
__global__ __launch_bounds__(kRowBlock) void k_embedding(Look<I, T, R> p)
{
    const int lane = threadIdx.x & (p.lanes - 1);
    const int64_t per = kRowBlock / p.lanes, row0 = threadIdx.x / p.lanes;
    for (int64_t i = (int64_t)blockIdx.x * per + row0; i < p.n; i += (int64_t)gridDim.x * per) {
        const uint32_t word = word_at<I>(p.words, i, p.vocab);
        const T* from = p.table + (int64_t)word * p.ldt;
        R* to = p.rows + i * p.ldr;
        for (int64_t c = ((int64_t)blockIdx.y * p.lanes + lane) * 8; c < p.cols; c += (int64_t)gridDim.y * p.lanes * 8) {
            Eight<T> t;
            Eight<R> r;
            if (word < p.vocab) t.load(from + c, p.cols - c);
#pragma unroll
            for (int k = 0; k < 8; ++k) r.set(k, word < p.vocab ? t.get(k) * p.scale : 0.0f);
            r.store(to + c, p.cols - c);
        }
    }
}

// ---- places sorted by their words ----
//
// Runs of kRun places are sorted by counting: a place's rank in its run is the number of places with a smaller word, and of
// the same word before it.  All comparisons are independent of each other, kRun a place, so that one launch of many small
// blocks does them.  Then up to kWays neighbouring runs are merged at a time: a place moves up by the number of places of
// each other run that come before it, which a search in that run finds.
constexpr int kRun = 2048, kWays = 32;
constexpr int kSortLanes = 16;  // lanes that share the comparisons of a place

struct Sorted {
    uint32_t* word;
    uint32_t* place;
};

// Each: places that a group of lanes ranks at once.
template <class I, int Each>
__global__ __launch_bounds__(256) void k_sort_run(const void* words, int64_t n, uint32_t vocab, Sorted out)
{
    constexpr int kPlaces = 256 / kSortLanes * Each;  // of a block, within one chunk of 64
    static_assert(64 % kPlaces == 0, "a block's places lie in one chunk");
    const int64_t first = (int64_t)blockIdx.x * kPlaces, run = first / kRun * kRun;
    const int64_t len = n - run < kRun ? n - run : kRun;
    __shared__ __align__(16) uint32_t keys[kRun];
    for (int64_t j = threadIdx.x; j < kRun; j += 256) keys[j] = j < len ? word_at<I>(words, run + j, vocab) : ~0u;
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
    const int chunk = (int)(first - run) / 64, chunks = (int)((len + 63) / 64);
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    for (int k = 0; k < chunks; ++k) {
        const u4 v = *(const u4*)(keys + k * 64 + lane * 4);
#pragma unroll
        for (int e = 0; e < Each; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool before = k < chunk || (k == chunk && k * 64 + lane * 4 + i < at[e]);
                rank[e] += v[i] < mine[e] || (before && v[i] == mine[e]);
            }
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

// Runs of `len` places, kWays of them to one.  kWays lanes share a place, each searches one run.
__global__ __launch_bounds__(256) void k_merge(Sorted in, Sorted out, int64_t n, int64_t len)
{
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kWays;
    if (i >= n) return;
    const int way = threadIdx.x % kWays;
    const int64_t all = i / (len * kWays) * (len * kWays), own = i / len * len, start = all + way * len;
    const uint32_t word = in.word[i];
    uint32_t before = 0;
    if (start == own) {
        before = (uint32_t)(i - own);
    } else if (start < n) {
        // places of that run which come first: smaller words, and of runs before this one's the same word too
        const uint32_t up = start < own ? 1 : 0;
        int64_t lo = 0, hi = n - start < len ? n - start : len;
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if (in.word[start + mid] < word + up)
                lo = mid + 1;
            else
                hi = mid;
        }
        before = (uint32_t)lo;
    }
#pragma unroll
    for (int s = kWays / 2; s > 0; s >>= 1) before += __shfl_xor(before, s);
    if (way == 0) {
        out.word[all + before] = word;
        out.place[all + before] = in.place[i];
    }
}

// ---- the sums ----

constexpr int kStrip = 512;  // columns of a wave
constexpr int kFillRows = 16;

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

// Zeros for the rows of kFillRows words from v0 on that do not occur.
template <class G, class T>
__device__ __forceinline__ void fill_rows(const Sum<G, T>& p, int64_t v0)
{
    // 16 lanes search for the first sorted place of a word, 16 probes at a time
    constexpr int kLanes = 256 / kFillRows;
    __shared__ int present[kFillRows];
    const int row = threadIdx.x / kLanes, lane = threadIdx.x % kLanes, shift = threadIdx.x % 64 / kLanes * kLanes;
    const uint32_t word = (uint32_t)(v0 + row);
    int64_t lo = 0, hi = p.n;  // it is in [lo, hi]
    while (__any(hi > lo)) {
        const int64_t step = (hi - lo + kLanes - 1) / kLanes, at = lo + lane * step;
        const bool less = at < hi && p.sorted.word[at] < word;
        const int count = __popc((uint32_t)(__ballot(less) >> shift) & ((1u << kLanes) - 1));  // the first probes
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
    for (int r = 0; r < kFillRows && v0 + r < p.vocab; ++r) {
        if (present[r]) continue;
        T* to = p.table + (v0 + r) * p.ldt;
        for (int64_t c = threadIdx.x * 8; c < p.cols; c += 256 * 8) {
            Eight<T> z;
#pragma unroll
            for (int k = 0; k < 8; ++k) z.set(k, 0.0f);
            z.store(to + c, p.cols - c);
        }
    }
}

// A wave adds up the rows of `chunk` sorted places in one strip of columns.  A word whose places all lie in the chunk is
// done; the sums of one that began before it or goes on after it are kept for k_join.
template <class G, class T>
__global__ __launch_bounds__(256) void k_sum(Sum<G, T> p)
{
    if (blockIdx.x >= p.sum_blocks) return fill_rows(p, (int64_t)(blockIdx.x - p.sum_blocks) * kFillRows);
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t chunk = item / p.strips, strip = item % p.strips;
    if (chunk >= p.chunks) return;
    const int64_t from = chunk * p.chunk, to = from + p.chunk < p.n ? from + p.chunk : p.n;
    const int64_t c = strip * kStrip + (threadIdx.x & 63) * 8, left = p.cols - c;
    const uint32_t before = from > 0 ? p.sorted.word[from - 1] : ~0u, after = to < p.n ? p.sorted.word[to] : ~0u;
    float sum[8] = {};
    uint32_t word = p.sorted.word[from];
    bool head = word == before;  // the sum began in an earlier chunk
    for (int64_t at = from; at < to; ++at) {
        if (word >= p.vocab) break;  // padding comes last
        const G* row = p.rows + (int64_t)p.sorted.place[at] * p.ldr + c;
        if (left > 0) {
            Eight<G> g;
            g.load(row, left);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += g.get(k);
        }
        const uint32_t next = at + 1 < to ? p.sorted.word[at + 1] : after;
        if (at + 1 < to && next == word) continue;
        const bool tail = at + 1 == to && next == word;
        if (left > 0) {
            if (head || tail) {
                Eight<float> f;
#pragma unroll
                for (int k = 0; k < 8; ++k) f.set(k, sum[k]);
                f.store(p.partial + (chunk * 2 + (head ? 0 : 1)) * p.cols + c, left);
            } else {
                put_row(p.table + (int64_t)word * p.ldt + c, sum, p.scale, p.accumulate, left);
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
        word = next;
        head = false;
    }
}

// The sums of words whose places lie in several chunks: a wave for each chunk in which one begins and strip.
template <class G, class T>
__global__ __launch_bounds__(256) void k_join(Sum<G, T> p)
{
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t chunk = item / p.strips, strip = item % p.strips;
    if (chunk + 1 >= p.chunks) return;  // the last one's do not go on
    const int64_t from = chunk * p.chunk, to = from + p.chunk;
    const uint32_t word = p.sorted.word[to - 1];
    if (word >= p.vocab || p.sorted.word[to] != word) return;              // none goes on
    if (p.sorted.word[from] == word && from > 0 && p.sorted.word[from - 1] == word) return;  // it began before
    const int64_t c = strip * kStrip + (threadIdx.x & 63) * 8, left = p.cols - c;
    if (left <= 0) return;
    float sum[8];
    Eight<float> f;
    f.load(p.partial + (chunk * 2 + 1) * p.cols + c, left);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = f.get(k);
    for (int64_t i = chunk + 1; i < p.chunks && p.sorted.word[i * p.chunk] == word; ++i) {
        f.load(p.partial + i * 2 * p.cols + c, left);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] += f.get(k);
    }
    put_row(p.table + (int64_t)word * p.ldt + c, sum, p.scale, p.accumulate, left);
}

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

int chunk_of(int64_t n, int64_t cols) { return n * ((cols + kStrip - 1) / kStrip) < 16384 ? 8 : 32; }

// Words and places, twice where they are merged, and the partial sums.
struct SumLayout {
    int64_t each, partial, total;
    SumLayout(int64_t n, int64_t cols)
    {
        each = up(n * 4, 256);
        const int64_t chunks = (n + chunk_of(n, cols) - 1) / chunk_of(n, cols);
        partial = up(chunks * 2 * cols * 4, 256);
        total = each * (n > kRun ? 4 : 2) + partial;
    }
};

}  // namespace

void launch_embedding(const Lookup& q, hipStream_t s)
{
    const RowGrid g(q.cols);
    const int64_t blocks = (q.words.n + g.per - 1) / g.per, across = (q.cols + g.lanes * 8 - 1) / (g.lanes * 8);
    const dim3 grid((uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20), (uint32_t)(across < 65535 ? across : 65535));
    by_word(q.words, [&](auto i) {
        by_element(q.table.type, [&](auto t) {
            by_element(q.rows.type, [&](auto r) {
                typedef decltype(i) I;
                typedef typename decltype(t)::T T;
                typedef typename decltype(r)::T R;
                const Look<I, T, R> p = {q.words.at, q.words.n, (uint32_t)q.words.vocab, (const T*)q.table.at, (R*)q.rows.at,
                                         q.table.ld, q.rows.ld, q.cols, q.scale, g.lanes};
                k_embedding<I, T, R><<<grid, kRowBlock, 0, s>>>(p);
            });
        });
    });
}

size_t embedding_grad_scratch(int64_t n, int64_t cols) { return (size_t)SumLayout(n, cols).total; }

void launch_embedding_grad(const Lookup& q, char* scratch, hipStream_t s)
{
    const int64_t n = q.words.n;
    const SumLayout l(n, q.cols);
    Sorted now = {(uint32_t*)scratch, (uint32_t*)(scratch + l.each)};
    Sorted other = {(uint32_t*)(scratch + 2 * l.each), (uint32_t*)(scratch + 3 * l.each)};
    float* partial = (float*)(scratch + l.total - l.partial);
    by_word(q.words, [&](auto i) {
        typedef decltype(i) I;
        k_sort_run<I, 4><<<(uint32_t)((n + 63) / 64), 256, 0, s>>>(q.words.at, n, (uint32_t)q.words.vocab, now);
    });
    for (int64_t len = kRun; len < n; len *= kWays) {
        k_merge<<<(uint32_t)((n + 256 / kWays - 1) / (256 / kWays)), 256, 0, s>>>(now, other, n, len);
        const Sorted t = now;
        now = other;
        other = t;
    }
    by_element(q.rows.type, [&](auto g) {
        by_element(q.table.type, [&](auto t) {
            typedef typename decltype(g)::T G;
            typedef typename decltype(t)::T T;
            const int chunk = chunk_of(n, q.cols);
            const int64_t chunks = (n + chunk - 1) / chunk, strips = (q.cols + kStrip - 1) / kStrip, blocks = (chunks * strips + 3) / 4;
            const int64_t fill = q.accumulate ? 0 : (q.words.vocab + kFillRows - 1) / kFillRows;
            const Sum<G, T> p = {now, n, (uint32_t)q.words.vocab, (const G*)q.rows.at, (T*)q.table.at, q.rows.ld, q.table.ld, q.cols, strips,
                                 q.scale, q.accumulate, chunk, chunks, partial, blocks};
            k_sum<G, T><<<(uint32_t)(blocks + fill), 256, 0, s>>>(p);
            if (chunks > 1) k_join<G, T><<<(uint32_t)blocks, 256, 0, s>>>(p);
        });
    });
}

}  // namespace sidco
