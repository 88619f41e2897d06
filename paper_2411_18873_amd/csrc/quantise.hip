// Rows as 8-bit integers with a scale each (HIP, gfx950): scale = max |x| / 127, q = round(x (127 / max |x|)), to even.
//
// One pass where a row (or, of a feature matrix, a column) fits the registers of the threads that share it; the memory bounds it.
#include "activations.h"
#include "lanes.h"

namespace eck {
namespace {

constexpr uint32_t UNIT = 16;           // elements of a thread at a time: sixteen bytes of the result
constexpr uint32_t MOST_WIDTH = 131071; // as product_int8 takes
constexpr float LEAST = 7.888609e-31f;  // 2^-100: 127 over less may pass fp32's range, and there is nothing to tell apart

struct Scale {
    float scale, inverse;
};
// from the bits of the largest magnitude (those of NaN are above infinity's)
__device__ __forceinline__ Scale scale_of(uint32_t most)
{
    if (most >= 0x7F800000u) return {__builtin_nanf(""), 0.0f};
    const float m = __uint_as_float(most);
    if (m < LEAST) return {0.0f, 0.0f};
    return {m / 127.0f, 127.0f / m};
}
// (rows of zeros, and those that hold what is not finite, are zeros)
__device__ __forceinline__ int quantised(float x, float inverse) { return inverse == 0.0f ? 0 : (int)rintf(x * inverse); }

template <class T>
__device__ __forceinline__ uint32_t size_bits(T x) { return __float_as_uint((float)x) & 0x7FFFFFFFu; }

template <class T>
struct Unit {
    Chunk<T> c[UNIT / Chunk<T>::N];
    __device__ __forceinline__ T at(int i) const { return c[i / Chunk<T>::N].v[i % Chunk<T>::N]; }
    __device__ __forceinline__ void load(const T *row, uint32_t from, uint32_t width)
    {
#pragma unroll
        for (uint32_t i = 0; i < UNIT / Chunk<T>::N; ++i) {
            const uint32_t k = from + i * Chunk<T>::N;
            if (k < width) c[i] = fetch_chunk(row, k, width);
            else
#pragma unroll
                for (int j = 0; j < Chunk<T>::N; ++j) c[i].v[j] = (T)0.0f;
        }
    }
    __device__ __forceinline__ uint32_t most() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < (int)UNIT; ++i) m = max(m, size_bits(at(i)));
        return m;
    }
    __device__ __forceinline__ void store(int8_t *to, float inverse) const
    {
        uint32_t word[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            word[w] = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) word[w] |= (uint32_t)(quantised((float)at(4 * w + i), inverse) & 0xFF) << (8 * i);
        }
        *reinterpret_cast<uint4 *>(to) = make_uint4(word[0], word[1], word[2], word[3]);
    }
};

// LANES threads a row, each with up to UNITS units; longer rows (LONG) are read a second time.  8192 rows of 4096 bf16 values, 100.7 MB: 18.5 us
// (5.4 TB/s)
template <class T, int LANES, int UNITS, bool LONG>
__global__ __launch_bounds__(256) void rows_kernel(const T *x, uint64_t ld_x, uint64_t n, uint32_t width, int8_t *q, uint64_t ld_q, float *scale)
{
    const uint32_t lane = threadIdx.x % LANES, units = (width + UNIT - 1) / UNIT;
    for (uint64_t r = (uint64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES; r < n; r += (uint64_t)gridDim.x * (256 / LANES)) {
        const T *row = x + r * ld_x;
        Unit<T> held[UNITS];
        uint32_t most = 0;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) held[u].load(row, (lane + u * LANES) * UNIT, width);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) most = max(most, held[u].most());
        if (LONG)
            for (uint32_t u = lane + UNITS * LANES; u < units; u += LANES) {
                Unit<T> some;
                some.load(row, u * UNIT, width);
                most = max(most, some.most());
            }
#pragma unroll
        for (int stride = 1; stride < (LANES < 64 ? LANES : 64); stride <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, stride)); // (not all lanes go round as often)
        if (LANES == 256) {
            __shared__ uint32_t all[4];
            __syncthreads();
            if ((threadIdx.x & 63) == 0) all[threadIdx.x / 64] = most;
            __syncthreads();
            most = max(max(all[0], all[1]), max(all[2], all[3]));
        }
        const Scale s = scale_of(most);
        if (lane == 0) scale[r] = s.scale;
        int8_t *to = q + r * ld_q;
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
            if (lane + u * LANES < units) held[u].store(to + (lane + u * LANES) * UNIT, s.inverse);
        if (LONG)
            for (uint32_t u = lane + UNITS * LANES; u < units; u += LANES) {
                Unit<T> some;
                some.load(row, u * UNIT, width);
                some.store(to + u * UNIT, s.inverse);
            }
    }
}

// A matrix with a row of the result in every column.  A block takes 8 * CHUNKS columns; a thread eight of them, four rows at a time, whose
// bytes are a word of the result; words are exchanged by way of the LDS so that memory sees whole pieces of the result's rows.  A matrix of
// more rows than a block takes at a time is read a second time, out of the caches.  2^20 candidates of 64 bf16 features, 205.5 MB: 44.6 us
// (4.6 TB/s); weights of 4096 rows and 4096 columns of fp32 values, 84 MB: 45, of 4096 and 16 384, 336 MB: 154, of 16 384 and 4096: 202 (twice
// read, in 256 blocks, one a compute unit)
template <class T, int CHUNKS, bool ONCE>
__global__ __launch_bounds__(256) void columns_kernel(const T *x, uint64_t ld_x, uint64_t n, uint32_t width, int8_t *q, uint64_t ld_q,
                                                      float *scale)
{
    constexpr uint32_t GROUPS = 256 / CHUNKS, COLUMNS = 8 * CHUNKS, STEP = 4 * GROUPS, PITCH = GROUPS + 1; // words
    __shared__ uint32_t most_of[4][COLUMNS], tile[COLUMNS * PITCH];
    __shared__ float inverse_of[COLUMNS];
    const uint32_t chunk = threadIdx.x % CHUNKS, group = threadIdx.x / CHUNKS;
    const uint64_t column0 = (uint64_t)blockIdx.x * COLUMNS;
    const uint32_t columns = (uint32_t)min((uint64_t)COLUMNS, n - column0);
    const T *from = x + column0;
    const auto load = [&](uint32_t r, float(&v)[8]) {
        if (r < width) load_chunk(from + r * ld_x, chunk * 8, columns, v);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    };
    uint32_t most[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    float v[4][8];
    for (uint32_t r = 4 * group; ONCE || r < width; r += STEP) {
#pragma unroll
        for (int k = 0; k < 4; ++k) load(r + k, v[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) most[i] = max(most[i], size_bits(v[k][i]));
        if (ONCE) break;
    }
    // of a wavefront's groups, then of the four wavefronts
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int stride = CHUNKS; stride < 64; stride <<= 1) most[i] = max(most[i], lane_exchange(most[i], stride));
        if ((threadIdx.x & 63) < CHUNKS) most_of[threadIdx.x / 64][chunk * 8 + i] = most[i];
    }
    __syncthreads();
    if (threadIdx.x < columns) {
        const uint32_t c = threadIdx.x;
        const Scale s = scale_of(max(max(most_of[0][c], most_of[1][c]), max(most_of[2][c], most_of[3][c])));
        scale[column0 + c] = s.scale;
        inverse_of[c] = s.inverse;
    }
    __syncthreads();
    float inverse[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) inverse[i] = chunk * 8 + i < columns ? inverse_of[chunk * 8 + i] : 0.0f;
    const uint32_t whole = (width + UNIT - 1) / UNIT * UNIT;
    for (uint32_t r0 = 0; r0 < width; r0 += STEP) {
        if (!ONCE)
#pragma unroll
            for (int k = 0; k < 4; ++k) load(r0 + 4 * group + k, v[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t word = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) word |= (uint32_t)(quantised(v[k][i], inverse[i]) & 0xFF) << (8 * k);
            tile[(chunk * 8 + i) * PITCH + group] = word;
        }
        __syncthreads();
        constexpr uint32_t PIECES = STEP / UNIT; // of a column
        for (uint32_t p = threadIdx.x; p < columns * PIECES; p += 256) {
            const uint32_t c = p / PIECES, k = p % PIECES;
            const uint32_t *w = tile + c * PITCH + k * 4;
            if (r0 + k * UNIT < whole) *reinterpret_cast<uint4 *>(q + (column0 + c) * ld_q + r0 + k * UNIT) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        __syncthreads();
    }
}

template <class T>
int32_t launch_rows(const void *x, uint64_t ld_x, uint64_t n, uint32_t width, int8_t *q, uint64_t ld_q, float *scale, hipStream_t st)
{
    const uint32_t units = (width + UNIT - 1) / UNIT;
    const auto go = [&](auto kernel, uint32_t lanes) -> int32_t {
        const uint64_t blocks = (n + 256 / lanes - 1) / (256 / lanes);
        hipLaunchKernelGGL(kernel, dim3((uint32_t)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, st, (const T *)x, ld_x, n, width, q, ld_q, scale);
        ECK_HIP_TRY(hipGetLastError());
        return ECK_OK;
    };
    if (units <= 4) return go(rows_kernel<T, 4, 1, false>, 4);
    if (units <= 16) return go(rows_kernel<T, 16, 1, false>, 16);
    if (units <= 64) return go(rows_kernel<T, 64, 1, false>, 64);
    if (units <= 256) return go(rows_kernel<T, 256, 1, false>, 256);
    if (units <= 512) return go(rows_kernel<T, 256, 2, false>, 256);
    return go(rows_kernel<T, 256, 2, true>, 256);
}

template <class T>
int32_t launch_columns(const void *x, uint64_t ld_x, uint64_t n, uint32_t width, int8_t *q, uint64_t ld_q, float *scale, hipStream_t st)
{
    const auto go = [&](auto kernel, uint32_t columns) -> int32_t {
        const uint64_t most = (uint64_t)columns << 22; // (a launch has less than 2^32 threads)
        for (uint64_t from = 0; from < n; from += most) {
            const uint64_t some = n - from < most ? n - from : most;
            hipLaunchKernelGGL(kernel, dim3((uint32_t)((some + columns - 1) / columns)), dim3(256), 0, st, (const T *)x + from, ld_x, some, width,
                               q + from * ld_q, ld_q, scale + from);
            ECK_HIP_TRY(hipGetLastError());
        }
        return ECK_OK;
    };
    if (width <= 64) return go(columns_kernel<T, 16, true>, 128);
    // as many columns a block as leave a block for every compute unit, and with the fewer more rows at a time (a column of 2920: 60 us where a
    // block takes 128 rows of 64 columns, 9 where it takes 1024 of 8)
    if (n >= 256 * 64) return go(columns_kernel<T, 8, false>, 64);
    if (n >= 256 * 32) return go(columns_kernel<T, 4, false>, 32);
    if (n >= 256 * 16) return go(columns_kernel<T, 2, false>, 16);
    return go(columns_kernel<T, 1, false>, 8);
}

} // namespace
} // namespace eck

using namespace eck;

extern "C" int32_t quantise_rows(const void *x, int32_t x_order, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t width, int8_t *q_out,
                                 uint64_t ld_q, float *scale_out, void *stream)
{
    if (!x || !q_out || !scale_out || n == 0 || width == 0 || !is_dtype(dtype) || (x_order != ECK_ROWS && x_order != ECK_COLUMNS)) return ECK_EINVAL;
    if (ld_x < (x_order == ECK_ROWS ? width : n) || ld_q < width) return ECK_ESHAPE;
    if (n > MAX_ROWS || width > MOST_WIDTH) return ECK_EUNSUPPORTED;
    if (!aligned(x, element_bytes(dtype)) || !aligned(q_out, 16) || ld_q % 16 || !aligned(scale_out, 4)) return ECK_EALIGN;
    const hipStream_t st = as_stream(stream);
    if (x_order == ECK_ROWS) return dtype == ECK_F32 ? launch_rows<float>(x, ld_x, n, width, q_out, ld_q, scale_out, st)
                                                     : launch_rows<bf16>(x, ld_x, n, width, q_out, ld_q, scale_out, st);
    return dtype == ECK_F32 ? launch_columns<float>(x, ld_x, n, width, q_out, ld_q, scale_out, st)
                            : launch_columns<bf16>(x, ld_x, n, width, q_out, ld_q, scale_out, st);
}
