// Dropout whose mask is drawn again wherever it is needed (HIP, gfx950).
//
// out = residual + (draw < p ? 0 : x / (1 - p)), the draws halves of SplitMix64 outputs: two columns a word, a row begins with a
// word of its own, so that sixteen bytes of a row (eight bf16 values, four words) never share a word with others.
#include "activations.h"
#include "splitmix.h"

namespace eck {
namespace {

template <class T, bool RESIDUAL>
__global__ __launch_bounds__(256) void dropout_kernel(const T *x, uint64_t ld_x, uint64_t n, uint32_t width, uint32_t p, float scale,
                                                      uint64_t state, uint64_t words, const T *residual, uint64_t ld_residual, T *out,
                                                      uint64_t ld_out, uint32_t chunks, uint64_t step_rows, uint32_t step_chunks)
{
    constexpr int N = Chunk<T>::N;
    // chunk number blockIdx.x * 256 + threadIdx.x of the matrix, then every (grid's threads)-th: step_rows rows and step_chunks
    // chunks further on, so that nothing is divided on the way
    const uint32_t first = blockIdx.x * 256 + threadIdx.x;
    uint64_t r = first / chunks;
    uint32_t c = first % chunks;
    for (; r < n; r += step_rows) {
        const uint32_t at = c * N;
        float v[N], res[N];
        load_chunk(x + r * ld_x, at, width, v);
        if (RESIDUAL) load_chunk(residual + r * ld_residual, at, width, res);
        uint64_t z = state + kGamma * (r * words + at / 2);
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            z += kGamma;
            const uint64_t u = splitmix_finalise(z);
            v[i] = (uint32_t)u < p ? 0.0f : v[i] * scale;
            v[i + 1] = (uint32_t)(u >> 32) < p ? 0.0f : v[i + 1] * scale;
        }
        if (RESIDUAL)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += res[i];
        store_chunk(out + r * ld_out, at, width, v);
        c += step_chunks;
        if (c >= chunks) {
            c -= chunks;
            ++r;
        }
    }
}

template <class T>
int32_t launch(const void *x, uint64_t ld_x, uint64_t n, uint32_t width, uint32_t p, uint64_t state, uint64_t words, const void *residual,
               uint64_t ld_residual, void *out, uint64_t ld_out, hipStream_t st)
{
    const uint32_t chunks = (width + Chunk<T>::N - 1) / Chunk<T>::N;
    const uint64_t blocks = (n * chunks + 255) / 256;
    const uint32_t grid = (uint32_t)(blocks < 8192 ? blocks : 8192);
    const uint64_t threads = (uint64_t)grid * 256;
    const float scale = (float)(4294967296.0 / (4294967296.0 - (double)p));
    auto kernel = residual ? dropout_kernel<T, true> : dropout_kernel<T, false>;
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, st, (const T *)x, ld_x, n, width, p, scale, state, words, (const T *)residual,
                       ld_residual, (T *)out, ld_out, chunks, threads / chunks, (uint32_t)(threads % chunks));
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

} // namespace
} // namespace eck

using namespace eck;

extern "C" int32_t dropout_apply(const void *x, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t width, uint32_t p_drop_q32,
                                 uint64_t seed, uint32_t round, uint64_t first_row, const void *residual, uint64_t ld_residual,
                                 void *out, uint64_t ld_out, void *stream)
{
    if (!x || !out || n == 0 || width == 0 || !is_dtype(dtype)) return ECK_EINVAL;
    if (ld_x < width || ld_out < width || (residual && ld_residual < width)) return ECK_ESHAPE;
    if (n > MAX_ROWS || width > MAX_WIDTH) return ECK_EUNSUPPORTED;
    const uint64_t size = element_bytes(dtype);
    if (!aligned(x, size) || !aligned(out, size) || !aligned(residual, size)) return ECK_EALIGN;
    const uint64_t words = ((uint64_t)width + 1) / 2, state = stream_state(seed, round) + kGamma * (first_row * words);
    if (dtype == ECK_F32) return launch<float>(x, ld_x, n, width, p_drop_q32, state, words, residual, ld_residual, out, ld_out, as_stream(stream));
    return launch<bf16>(x, ld_x, n, width, p_drop_q32, state, words, residual, ld_residual, out, ld_out, as_stream(stream));
}
