// Rows of activations (HIP, gfx950): element types, sixteen bytes of a row at a time whatever it is aligned to, host-side checks.
#pragma once
#include "eck_internal.h"

namespace eck {

typedef __bf16 bf16;
template <class T>
constexpr int32_t code_of = sizeof(T) == 4 ? ECK_F32 : ECK_BF16;

constexpr uint64_t MAX_ROWS = 1ull << 31;
constexpr uint64_t MAX_WIDTH = 1ull << 24;

inline uint64_t element_bytes(int32_t dtype) { return dtype == ECK_F32 ? 4 : 2; }
inline bool is_dtype(int32_t dtype) { return dtype == ECK_F32 || dtype == ECK_BF16; }
inline bool aligned(const void *p, uint64_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Elements of one access (of sixteen bytes, if not said otherwise), as an aggregate that promises no more than an element's
// alignment: the hardware takes global accesses of any alignment, the compiler only has to be told not to count on more.
template <class T, int COUNT = 16 / sizeof(T)>
struct __attribute__((packed, aligned(sizeof(T)))) Chunk {
    static constexpr int N = COUNT;
    typedef T Vector __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    Vector v;
};

// values [at, at + N) of a row of `width` as they are, zeros past its end
template <class T>
__device__ __forceinline__ Chunk<T> fetch_chunk(const T *row, uint32_t at, uint32_t width)
{
    if (at + Chunk<T>::N <= width) return *reinterpret_cast<const Chunk<T> *>(row + at);
    Chunk<T> c;
#pragma unroll
    for (int i = 0; i < Chunk<T>::N; ++i) c.v[i] = at + i < width ? row[at + i] : (T)0.0f;
    return c;
}

// values [at, at + N) as floats; `rest` past the row's end
template <class T, int N>
__device__ __forceinline__ void load_chunk(const T *row, uint32_t at, uint32_t width, float (&x)[N], float rest = 0.0f)
{
    if (at + N <= width) {
        const Chunk<T, N> c = *reinterpret_cast<const Chunk<T, N> *>(row + at);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (float)c.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = at + i < width ? (float)row[at + i] : rest;
    }
}

template <class T, int N>
__device__ __forceinline__ void store_chunk(T *row, uint32_t at, uint32_t width, const float (&x)[N])
{
    if (at + N <= width) {
        Chunk<T, N> c;
#pragma unroll
        for (int i = 0; i < N; ++i) c.v[i] = (T)x[i];
        *reinterpret_cast<Chunk<T, N> *>(row + at) = c;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (at + i < width) row[at + i] = (T)x[i];
    }
}

} // namespace eck
