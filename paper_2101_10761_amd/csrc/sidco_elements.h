// Element types, and eight neighbours of a row that may start at any element.
#ifndef SIDCO_ELEMENTS_H
#define SIDCO_ELEMENTS_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sidco_language.h"

namespace sidco {

template <int Type>
struct ElementOf;
template <>
struct ElementOf<kGradF32> {
    typedef float T;
};
template <>
struct ElementOf<kGradF16> {
    typedef _Float16 T;
};
template <>
struct ElementOf<kGradBf16> {
    typedef __bf16 T;
};

// f(ElementOf) for an element type
template <class F>
inline void by_element(int type, const F& f)
{
    if (type == kGradF32)
        f(ElementOf<kGradF32>());
    else if (type == kGradF16)
        f(ElementOf<kGradF16>());
    else
        f(ElementOf<kGradBf16>());
}

// Eight neighbours as they are in memory.
template <class T>
struct Eight {
    typedef T part __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
    static constexpr int kParts = sizeof(T) / 2, kPer = 16 / (int)sizeof(T);
    part v[kParts];

    __device__ __forceinline__ void load(const T* p)
    {
#pragma unroll
        for (int k = 0; k < kParts; ++k) v[k] = *(const part*)(p + k * kPer);
    }
    // the first n of them, zeros for the others
    __device__ __forceinline__ void load(const T* p, int64_t n)
    {
        if (n >= 8) return load(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i / kPer][i % kPer] = i < n ? p[i] : (T)0.0f;
    }
    __device__ __forceinline__ void store(T* p) const
    {
#pragma unroll
        for (int k = 0; k < kParts; ++k) *(part*)(p + k * kPer) = v[k];
    }
    __device__ __forceinline__ void store(T* p, int64_t n) const
    {
        if (n >= 8) return store(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = v[i / kPer][i % kPer];
    }
    // the last n of them, less than eight
    __device__ __forceinline__ void store_last(T* p, int64_t n) const
    {
#pragma unroll
        for (int i = 1; i < 8; ++i)
            if (i >= 8 - n) p[i] = v[i / kPer][i % kPer];
    }
    __device__ __forceinline__ float get(int i) const { return (float)v[i / kPer][i % kPer]; }
    __device__ __forceinline__ void set(int i, float x) { v[i / kPer][i % kPer] = (T)x; }
};

// The word at place i, or for padding `vocab`.
template <class I>
__device__ __forceinline__ uint32_t word_at(const void* words, int64_t i, uint32_t vocab)
{
    const I w = ((const I*)words)[i];
    return w >= 0 && w < (I)vocab ? (uint32_t)w : vocab;
}

// The same where the type is not worth a kernel of its own.
struct WordList {
    const void* at;  // may be NULL
    bool wide;
    uint32_t vocab;
    __device__ __forceinline__ uint32_t operator[](int64_t i) const { return wide ? word_at<int64_t>(at, i, vocab) : word_at<int32_t>(at, i, vocab); }
    __device__ __forceinline__ bool none(int64_t i) const { return (*this)[i] == vocab; }
    WordList from(int64_t i) const { return {(const char*)at + i * (wide ? 8 : 4), wide, vocab}; }
};

// f(an int32_t or int64_t) for the words' type
template <class F>
inline void by_word(const Words& w, const F& f)
{
    if (w.wide)
        f((int64_t)0);
    else
        f((int32_t)0);
}

// Blocks of 256 threads over rows: a power of two of threads share a row, eight elements each at a time.
constexpr int kRowBlock = 256;
struct RowGrid {
    int lanes;     // a row's threads
    int per;       // rows of a block
    explicit RowGrid(int64_t cols)
    {
        lanes = 1;
        while (lanes < kRowBlock && lanes * 8 < cols) lanes *= 2;
        per = kRowBlock / lanes;
    }
};

}  // namespace sidco
#endif
