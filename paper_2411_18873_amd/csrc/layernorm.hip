// Layer norm of rows of activations or of candidates' features, forward and backward (HIP, gfx950).
//
//   forward   m = sum x / w,  r = 1 / sqrt(sum (x - m)^2 / w + eps),  y = (x - m) r gamma + beta
//   backward  g = dy gamma, xh = (x - m) r:  dx = r (g - mean(g) - xh mean(g xh)),  dgamma = sum dy xh,  dbeta = sum dy
//
// Every pass is bound by memory.  A row stays in registers between its sums and its result (the two sums of the forward pass one
// after the other: the squares of differences from the mean lose nothing to a large mean), shared by as many threads as sixteen
// bytes each need: 8 to 64 lanes of a wavefront, or a block.  Threads keep their columns from row to row, so gamma and beta are
// loaded once, and the parameters' gradients grow in registers: blocks leave one partial sum per column and a second launch adds
// these in a fixed order.  Rows longer than a block's registers are read again for every pass.
#include "activations.h"
#include "lanes.h"

#include <type_traits>

namespace eck {
namespace {

constexpr int BLOCK = 256;

// sum over groups of TPR neighbouring lanes, or over the block, in every thread; all threads have to call it
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *scratch)
{
#pragma unroll
    for (uint32_t stride = 1; stride < 64 && stride < TPR; stride <<= 1)
        v += __uint_as_float(lane_exchange(__float_as_uint(v), stride));
    if (TPR > 64) {
        __syncthreads(); // (the sum before this one has been read)
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
        __syncthreads();
        v = scratch[0];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w) v += scratch[w];
    }
    return v;
}

// a thread's parameters: elements at .. at + N - 1 of gamma and beta, as ones and zeros where there are none
template <int N>
__device__ __forceinline__ void load_vector(const float *p, uint32_t at, uint32_t width, float none, float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = p && at + i < width ? p[at + i] : none;
}

template <class T, int TPR, int ITEMS>
__global__ __launch_bounds__(BLOCK) void forward_kernel(const T *x, uint64_t ld_x, uint64_t n, uint32_t width, const float *gamma,
                                                        const float *beta, float eps, T *y, uint64_t ld_y, float *mean_out, float *rstd_out)
{
    constexpr int N = Chunk<T>::N, ROWS = BLOCK / TPR;
    __shared__ float scratch[BLOCK / 64];
    const uint32_t lane = threadIdx.x % TPR;
    const float share = 1.0f / (float)width;
    float ga[ITEMS][N], be[ITEMS][N];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        load_vector(gamma, (k * TPR + lane) * N, width, 1.0f, ga[k]);
        load_vector(beta, (k * TPR + lane) * N, width, 0.0f, be[k]);
    }
    for (uint64_t r0 = (uint64_t)blockIdx.x * ROWS; r0 < n; r0 += (uint64_t)gridDim.x * ROWS) {
        const uint64_t r = r0 + threadIdx.x / TPR;
        const T *row = x + (r < n ? r : n - 1) * ld_x; // (all lanes stay, for the sums)
        float v[ITEMS][N], sum = 0.0f;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) load_chunk(row, (k * TPR + lane) * N, width, v[k]);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) sum += v[k][i];
        const float mean = row_sum<TPR>(sum, scratch) * share;
        float squares = 0.0f;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[k][i] -= mean;
                squares += (k * TPR + lane) * N + i < width ? v[k][i] * v[k][i] : 0.0f;
            }
        const float rstd = 1.0f / sqrtf(row_sum<TPR>(squares, scratch) * share + eps);
        if (r >= n) continue;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[k][i] = v[k][i] * rstd * ga[k][i] + be[k][i];
            store_chunk(y + r * ld_y, (k * TPR + lane) * N, width, v[k]);
        }
        if (mean_out && lane == 0) {
            mean_out[r] = mean;
            rstd_out[r] = rstd;
        }
    }
}

// rows of any length: a block each, read three times
template <class T>
__global__ __launch_bounds__(BLOCK) void forward_long_kernel(const T *x, uint64_t ld_x, uint64_t n, uint32_t width, const float *gamma,
                                                             const float *beta, float eps, T *y, uint64_t ld_y, float *mean_out,
                                                             float *rstd_out)
{
    constexpr int N = Chunk<T>::N;
    __shared__ float scratch[BLOCK / 64];
    const float share = 1.0f / (float)width;
    for (uint64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const T *row = x + r * ld_x;
        float sum = 0.0f, squares = 0.0f, v[N];
        for (uint32_t at = threadIdx.x * N; at < width; at += BLOCK * N) {
            load_chunk(row, at, width, v);
#pragma unroll
            for (int i = 0; i < N; ++i) sum += v[i];
        }
        const float mean = row_sum<BLOCK>(sum, scratch) * share;
        for (uint32_t at = threadIdx.x * N; at < width; at += BLOCK * N) {
            load_chunk(row, at, width, v, mean);
#pragma unroll
            for (int i = 0; i < N; ++i) squares += (v[i] - mean) * (v[i] - mean);
        }
        const float rstd = 1.0f / sqrtf(row_sum<BLOCK>(squares, scratch) * share + eps);
        for (uint32_t at = threadIdx.x * N; at < width; at += BLOCK * N) {
            float ga[N], be[N];
            load_chunk(row, at, width, v);
            load_vector(gamma, at, width, 1.0f, ga);
            load_vector(beta, at, width, 0.0f, be);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = (v[i] - mean) * rstd * ga[i] + be[i];
            store_chunk(y + r * ld_y, at, width, v);
        }
        if (mean_out && threadIdx.x == 0) {
            mean_out[r] = mean;
            rstd_out[r] = rstd;
        }
    }
}

// partial: [gridDim.x][2][width] sums of dgamma and dbeta, or NULL; dx: or NULL
template <class T, int TPR, int ITEMS>
__global__ __launch_bounds__(BLOCK) void backward_kernel(const T *x, uint64_t ld_x, const T *dy, uint64_t ld_dy, uint64_t n,
                                                         uint32_t width, const float *gamma, const float *mean, const float *rstd, T *dx,
                                                         uint64_t ld_dx, float *partial)
{
    constexpr int N = Chunk<T>::N, ROWS = BLOCK / TPR, WAVES = BLOCK / 64;
    __shared__ float scratch[WAVES];
    __shared__ float joined[TPR > 64 ? 1 : WAVES * TPR * N];
    const uint32_t lane = threadIdx.x % TPR;
    const float share = 1.0f / (float)width;
    float ga[ITEMS][N], dgamma[ITEMS][N], dbeta[ITEMS][N];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        load_vector(gamma, (k * TPR + lane) * N, width, 1.0f, ga[k]);
#pragma unroll
        for (int i = 0; i < N; ++i) dgamma[k][i] = dbeta[k][i] = 0.0f;
    }
    for (uint64_t r0 = (uint64_t)blockIdx.x * ROWS; r0 < n; r0 += (uint64_t)gridDim.x * ROWS) {
        const uint64_t r = r0 + threadIdx.x / TPR, from = r < n ? r : n - 1;
        const bool counts = r < n;
        float xh[ITEMS][N], d[ITEMS][N], sum = 0.0f, dot = 0.0f;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            load_chunk(x + from * ld_x, (k * TPR + lane) * N, width, xh[k]);
            load_chunk(dy + from * ld_dy, (k * TPR + lane) * N, width, d[k]); // zeros past the end
        }
        const float m = mean[from], s = rstd[from];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                xh[k][i] = (k * TPR + lane) * N + i < width ? (xh[k][i] - m) * s : 0.0f;
                dgamma[k][i] += counts ? d[k][i] * xh[k][i] : 0.0f;
                dbeta[k][i] += counts ? d[k][i] : 0.0f;
                d[k][i] *= ga[k][i];
                sum += d[k][i];
                dot += d[k][i] * xh[k][i];
            }
        if (!dx) continue; // (for all threads)
        sum = row_sum<TPR>(sum, scratch) * share;
        dot = row_sum<TPR>(dot, scratch) * share;
        if (!counts) continue;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
#pragma unroll
            for (int i = 0; i < N; ++i) d[k][i] = s * (d[k][i] - sum - xh[k][i] * dot);
            store_chunk(dx + r * ld_dx, (k * TPR + lane) * N, width, d[k]);
        }
    }
    if (!partial) return;
    float *mine = partial + (uint64_t)blockIdx.x * 2 * width;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            float(&v)[N] = which ? dbeta[k] : dgamma[k];
            if (TPR > 64) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if ((k * TPR + lane) * N + i < width) mine[which * width + (k * TPR + lane) * N + i] = v[i];
                continue;
            }
            // the rows of a wavefront, then of the block
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (uint32_t stride = TPR; stride < 64; stride <<= 1) v[i] += __uint_as_float(lane_exchange(__float_as_uint(v[i]), stride));
            __syncthreads();
            if ((threadIdx.x & 63) < TPR)
#pragma unroll
                for (int i = 0; i < N; ++i) joined[((threadIdx.x >> 6) * TPR + lane) * N + i] = v[i];
            __syncthreads();
            for (uint32_t c = threadIdx.x; c < TPR * N; c += BLOCK) {
                float total = joined[c];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) total += joined[w * TPR * N + c];
                if (k * TPR * N + c < width) mine[which * width + k * TPR * N + c] = total;
            }
        }
}

// dx of rows of any length: a block each, read twice
template <class T>
__global__ __launch_bounds__(BLOCK) void backward_long_kernel(const T *x, uint64_t ld_x, const T *dy, uint64_t ld_dy, uint64_t n,
                                                              uint32_t width, const float *gamma, const float *mean, const float *rstd,
                                                              T *dx, uint64_t ld_dx)
{
    constexpr int N = Chunk<T>::N;
    __shared__ float scratch[BLOCK / 64];
    const float share = 1.0f / (float)width;
    for (uint64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const float m = mean[r], s = rstd[r];
        float sum = 0.0f, dot = 0.0f, xh[N], d[N], ga[N];
        for (uint32_t at = threadIdx.x * N; at < width; at += BLOCK * N) {
            load_chunk(x + r * ld_x, at, width, xh, m);
            load_chunk(dy + r * ld_dy, at, width, d);
            load_vector(gamma, at, width, 1.0f, ga);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                sum += d[i] * ga[i];
                dot += d[i] * ga[i] * ((xh[i] - m) * s);
            }
        }
        sum = row_sum<BLOCK>(sum, scratch) * share;
        dot = row_sum<BLOCK>(dot, scratch) * share;
        for (uint32_t at = threadIdx.x * N; at < width; at += BLOCK * N) {
            load_chunk(x + r * ld_x, at, width, xh);
            load_chunk(dy + r * ld_dy, at, width, d);
            load_vector(gamma, at, width, 1.0f, ga);
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = s * (d[i] * ga[i] - sum - (xh[i] - m) * s * dot);
            store_chunk(dx + r * ld_dx, at, width, d);
        }
    }
}

// partial sums of the parameters' gradients of rows of any length: a thread per column, block row y takes every gridDim.y-th row
template <class T>
__global__ __launch_bounds__(BLOCK) void columns_long_kernel(const T *x, uint64_t ld_x, const T *dy, uint64_t ld_dy, uint64_t n,
                                                             uint32_t width, const float *mean, const float *rstd, float *partial)
{
    const uint32_t c = blockIdx.x * BLOCK + threadIdx.x;
    if (c >= width) return;
    float dgamma = 0.0f, dbeta = 0.0f;
    for (uint64_t r = blockIdx.y; r < n; r += gridDim.y) {
        const float d = (float)dy[r * ld_dy + c];
        dgamma += d * (((float)x[r * ld_x + c] - mean[r]) * rstd[r]);
        dbeta += d;
    }
    partial[(uint64_t)blockIdx.y * 2 * width + c] = dgamma;
    partial[(uint64_t)blockIdx.y * 2 * width + width + c] = dbeta;
}

// dgamma and dbeta: the blocks' partial sums, sixteen wavefronts a block of 64 columns
__global__ __launch_bounds__(1024) void join_kernel(const float *partial, uint32_t parts, uint32_t width, float *dgamma, float *dbeta)
{
    __shared__ float sums[16][64];
    const uint64_t columns = 2ull * width, c = (uint64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    float sum = 0.0f;
    if (c < columns)
        for (uint32_t p = threadIdx.x >> 6; p < parts; p += 16) sum += partial[p * columns + c];
    sums[threadIdx.x >> 6][threadIdx.x & 63] = sum;
    __syncthreads();
    if (threadIdx.x >= 64 || c >= columns) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += sums[w][threadIdx.x];
    if (c < width) dgamma[c] = sum;
    else dbeta[c - width] = sum;
}

// ------------------------------------------------------------------------------------------------ features
//
// A block takes 64 candidates.  Thread (group, chunk) holds sixteen bytes of candidates of every GROUPS-th feature; rows go
// through the LDS, because a candidate's features lie ld elements apart on one side and next to each other on the other.

constexpr int TILE = 64;
template <class T>
struct Columns {
    static constexpr int N = Chunk<T>::N, CHUNKS = TILE / N, GROUPS = BLOCK / CHUNKS; // bf16: 8 chunks, 32 groups; fp32: 16, 16
    // elements of a candidate's row in the LDS: a word more than the width, so that neighbouring candidates start on other banks
    static __host__ __device__ uint32_t pitch(uint32_t width) { return (width + 1) / 2 * 2 + 4 / sizeof(T); }
};

// sum over the features of each of a thread's N candidates, in all threads with that chunk
template <class T>
__device__ __forceinline__ void candidate_sums(float (&v)[Chunk<T>::N], float (*scratch)[TILE])
{
    using C = Columns<T>;
    const uint32_t chunk = threadIdx.x % C::CHUNKS;
#pragma unroll
    for (int i = 0; i < C::N; ++i)
#pragma unroll
        for (uint32_t stride = C::CHUNKS; stride < 64; stride <<= 1) v[i] += __uint_as_float(lane_exchange(__float_as_uint(v[i]), stride));
    __syncthreads();
    if ((threadIdx.x & 63) < C::CHUNKS)
#pragma unroll
        for (int i = 0; i < C::N; ++i) scratch[threadIdx.x >> 6][chunk * C::N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < C::N; ++i) {
        v[i] = scratch[0][chunk * C::N + i];
#pragma unroll
        for (int w = 1; w < BLOCK / 64; ++w) v[i] += scratch[w][chunk * C::N + i];
    }
}

template <class T, int ITEMS>
__global__ __launch_bounds__(BLOCK) void forward_columns_kernel(const T *x, uint64_t ld_x, uint64_t n, uint32_t width, const float *gamma,
                                                                const float *beta, float eps, T *y, uint64_t ld_y, float *mean_out,
                                                                float *rstd_out)
{
    using C = Columns<T>;
    constexpr int N = C::N;
    extern __shared__ __attribute__((aligned(16))) unsigned char dynamic[];
    T *rows = reinterpret_cast<T *>(dynamic);
    __shared__ float scratch[BLOCK / 64][TILE];
    const uint32_t chunk = threadIdx.x % C::CHUNKS, group = threadIdx.x / C::CHUNKS, pitch = C::pitch(width);
    const float share = 1.0f / (float)width;
    for (uint64_t first = (uint64_t)blockIdx.x * TILE; first < n; first += (uint64_t)gridDim.x * TILE) {
        const uint32_t here = (uint32_t)(n - first < TILE ? n - first : TILE);
        float v[ITEMS][N], mean[N], rstd[N];
#pragma unroll
        for (int i = 0; i < N; ++i) mean[i] = rstd[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const uint32_t f = k * C::GROUPS + group;
            if (f < width) load_chunk(x + f * ld_x + first, chunk * N, here, v[k]);
            else
#pragma unroll
                for (int i = 0; i < N; ++i) v[k][i] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) mean[i] += v[k][i];
        candidate_sums<T>(mean, scratch);
#pragma unroll
        for (int i = 0; i < N; ++i) mean[i] *= share;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[k][i] -= mean[i];
                rstd[i] += k * C::GROUPS + group < width ? v[k][i] * v[k][i] : 0.0f;
            }
        candidate_sums<T>(rstd, scratch);
#pragma unroll
        for (int i = 0; i < N; ++i) rstd[i] = 1.0f / sqrtf(rstd[i] * share + eps);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const uint32_t f = k * C::GROUPS + group;
            if (f >= width) continue;
            const float ga = gamma ? gamma[f] : 1.0f, be = beta ? beta[f] : 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) rows[(chunk * N + i) * pitch + f] = (T)(v[k][i] * rstd[i] * ga + be);
        }
        if (mean_out && group == 0)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (chunk * N + i < here) {
                    mean_out[first + chunk * N + i] = mean[i];
                    rstd_out[first + chunk * N + i] = rstd[i];
                }
        __syncthreads();
        const uint32_t chunks = (width + N - 1) / N;
        for (uint32_t j = threadIdx.x; j < here * chunks; j += BLOCK) {
            const uint32_t c = j / chunks, at = j % chunks * N;
            float out[N];
            load_chunk(rows + c * pitch, at, width, out);
            store_chunk(y + (first + c) * ld_y, at, width, out);
        }
        __syncthreads();
    }
}

template <class T, int ITEMS>
__global__ __launch_bounds__(BLOCK) void backward_columns_kernel(const T *x, uint64_t ld_x, const T *dy, uint64_t ld_dy, uint64_t n,
                                                                 uint32_t width, const float *gamma, const float *mean, const float *rstd,
                                                                 T *dx, uint64_t ld_dx, float *partial)
{
    using C = Columns<T>;
    constexpr int N = C::N;
    extern __shared__ __attribute__((aligned(16))) unsigned char dynamic[];
    T *rows = reinterpret_cast<T *>(dynamic);
    __shared__ float scratch[BLOCK / 64][TILE];
    const uint32_t chunk = threadIdx.x % C::CHUNKS, group = threadIdx.x / C::CHUNKS, pitch = C::pitch(width);
    const float share = 1.0f / (float)width;
    float dgamma[ITEMS], dbeta[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) dgamma[k] = dbeta[k] = 0.0f;
    for (uint64_t first = (uint64_t)blockIdx.x * TILE; first < n; first += (uint64_t)gridDim.x * TILE) {
        const uint32_t here = (uint32_t)(n - first < TILE ? n - first : TILE), chunks = (width + N - 1) / N;
        for (uint32_t j = threadIdx.x; j < here * chunks; j += BLOCK) {
            const uint32_t c = j / chunks, at = j % chunks * N;
            float in[N];
            load_chunk(dy + (first + c) * ld_dy, at, width, in);
            store_chunk(rows + c * pitch, at, width, in);
        }
        __syncthreads();
        float xh[ITEMS][N], d[ITEMS][N], m[N], s[N], sum[N], dot[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool counts = chunk * N + i < here;
            m[i] = counts ? mean[first + chunk * N + i] : 0.0f;
            s[i] = counts ? rstd[first + chunk * N + i] : 0.0f;
            sum[i] = dot[i] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const uint32_t f = k * C::GROUPS + group;
            if (f < width) load_chunk(x + f * ld_x + first, chunk * N, here, xh[k]);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const bool counts = f < width && chunk * N + i < here;
                xh[k][i] = counts ? (xh[k][i] - m[i]) * s[i] : 0.0f;
                d[k][i] = counts ? (float)rows[(chunk * N + i) * pitch + f] : 0.0f;
                dgamma[k] += d[k][i] * xh[k][i];
                dbeta[k] += d[k][i];
            }
            const float ga = gamma && f < width ? gamma[f] : 1.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                d[k][i] *= ga;
                sum[i] += d[k][i];
                dot[i] += d[k][i] * xh[k][i];
            }
        }
        if (dx) {
            candidate_sums<T>(sum, scratch);
            candidate_sums<T>(dot, scratch);
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const uint32_t f = k * C::GROUPS + group;
                if (f >= width) continue;
#pragma unroll
                for (int i = 0; i < N; ++i) d[k][i] = s[i] * (d[k][i] - sum[i] * share - xh[k][i] * (dot[i] * share));
                store_chunk(dx + f * ld_dx + first, chunk * N, here, d[k]);
            }
        }
        __syncthreads();
    }
    if (!partial) return;
    float *mine = partial + (uint64_t)blockIdx.x * 2 * width;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
#pragma unroll
        for (uint32_t stride = 1; stride < C::CHUNKS; stride <<= 1) {
            dgamma[k] += __uint_as_float(lane_exchange(__float_as_uint(dgamma[k]), stride));
            dbeta[k] += __uint_as_float(lane_exchange(__float_as_uint(dbeta[k]), stride));
        }
        const uint32_t f = k * C::GROUPS + group;
        if (chunk == 0 && f < width) {
            mine[f] = dgamma[k];
            mine[width + f] = dbeta[k];
        }
    }
}

// ------------------------------------------------------------------------------------------------ launches

// Calls f with the number of threads a row and the chunks a thread that hold a row of `width`; false if none does.  (A power of
// two below 64 lanes wastes less than half of them on short rows; a wavefront holds four chunks a lane, then a block takes over.)
template <class T, class F>
bool with_row_shape(uint32_t width, F &&f)
{
    constexpr uint32_t N = Chunk<T>::N;
#define ECK_ROW_SHAPE(tpr, items)                                                                  \
    if (width <= (tpr) * (items) * N) {                                                            \
        f(std::integral_constant<int, tpr>{}, std::integral_constant<int, items>{});               \
        return true;                                                                               \
    }
    ECK_ROW_SHAPE(8, 1)
    ECK_ROW_SHAPE(16, 1)
    ECK_ROW_SHAPE(32, 1)
    ECK_ROW_SHAPE(64, 1)
    ECK_ROW_SHAPE(64, 2)
    ECK_ROW_SHAPE(256, 1)
    ECK_ROW_SHAPE(256, 2)
    ECK_ROW_SHAPE(256, 4)
#undef ECK_ROW_SHAPE
    return false;
}

// the same for the chunks of features a thread
template <class T, class F>
void with_columns_shape(uint32_t width, F &&f)
{
    constexpr uint32_t G = Columns<T>::GROUPS;
    if (width <= G) f(std::integral_constant<int, 1>{});
    else if (width <= 2 * G) f(std::integral_constant<int, 2>{});
    else if (width <= 4 * G) f(std::integral_constant<int, 4>{});
    else if (width <= 8 * G) f(std::integral_constant<int, 8>{});
    else f(std::integral_constant<int, 16>{});
}

uint32_t at_most(uint64_t blocks, uint32_t most) { return (uint32_t)(blocks < most ? blocks : most); }

// Blocks of the backward pass, each of which leaves a partial sum per column.  Four a compute unit keep the memory busy; fewer where
// their partial sums (8 bytes a column, written and read) would be more than an eighth of what the rows move.
uint32_t backward_blocks(uint64_t n, uint32_t width, int32_t dtype, int32_t order)
{
    const uint64_t vector = 16 / element_bytes(dtype), chunks = (width + vector - 1) / vector;
    uint64_t rows = 1; // a block's at a time
    if (order == ECK_COLUMNS) rows = TILE;
    else
        for (uint64_t tpr = 8; tpr <= 64; tpr *= 2)
            if (chunks <= tpr * (tpr == 64 ? 2 : 1)) {
                rows = BLOCK / tpr;
                break;
            }
    return at_most((n + rows - 1) / rows, 1024);
}
constexpr uint32_t LONG_PARTS = 64;

template <class T>
int32_t forward(const void *x, int32_t order, uint64_t ld_x, uint64_t n, uint32_t width, const float *gamma, const float *beta, float eps,
                void *y, uint64_t ld_y, float *mean, float *rstd, hipStream_t st)
{
    if (order == ECK_COLUMNS) {
        const size_t lds = (size_t)TILE * Columns<T>::pitch(width) * sizeof(T);
        with_columns_shape<T>(width, [&](auto items) {
            hipLaunchKernelGGL((forward_columns_kernel<T, decltype(items)::value>), dim3(at_most((n + TILE - 1) / TILE, 1 << 20)), dim3(BLOCK),
                               lds, st, (const T *)x, ld_x, n, width, gamma, beta, eps, (T *)y, ld_y, mean, rstd);
        });
    } else if (!with_row_shape<T>(width, [&](auto tpr, auto items) {
                   constexpr int TPR = decltype(tpr)::value, ROWS = BLOCK / TPR;
                   hipLaunchKernelGGL((forward_kernel<T, TPR, decltype(items)::value>), dim3(at_most((n + ROWS - 1) / ROWS, 2048)), dim3(BLOCK), 0,
                                      st, (const T *)x, ld_x, n, width, gamma, beta, eps, (T *)y, ld_y, mean, rstd);
               })) {
        hipLaunchKernelGGL(forward_long_kernel<T>, dim3(at_most(n, 2048)), dim3(BLOCK), 0, st, (const T *)x, ld_x, n, width, gamma, beta, eps,
                           (T *)y, ld_y, mean, rstd);
    }
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

template <class T>
int32_t backward(const void *x_, int32_t order, uint64_t ld_x, const void *dy_, uint64_t ld_dy, uint64_t n, uint32_t width,
                 const float *gamma, const float *mean, const float *rstd, void *dx_, uint64_t ld_dx, float *dgamma, float *dbeta,
                 float *partial, hipStream_t st)
{
    const T *x = (const T *)x_, *dy = (const T *)dy_;
    T *dx = (T *)dx_;
    uint32_t parts = backward_blocks(n, width, code_of<T>, order);
    if (!dgamma) partial = nullptr;
    if (order == ECK_COLUMNS) {
        const size_t lds = (size_t)TILE * Columns<T>::pitch(width) * sizeof(T);
        with_columns_shape<T>(width, [&](auto items) {
            hipLaunchKernelGGL((backward_columns_kernel<T, decltype(items)::value>), dim3(parts), dim3(BLOCK), lds, st, x, ld_x, dy, ld_dy, n,
                               width, gamma, mean, rstd, dx, ld_dx, partial);
        });
    } else if (!with_row_shape<T>(width, [&](auto tpr, auto items) {
                   hipLaunchKernelGGL((backward_kernel<T, decltype(tpr)::value, decltype(items)::value>), dim3(parts), dim3(BLOCK), 0, st, x,
                                      ld_x, dy, ld_dy, n, width, gamma, mean, rstd, dx, ld_dx, partial);
               })) {
        // (the sums over rows first: dx may take the place of dy or x)
        parts = at_most(n, LONG_PARTS);
        if (partial)
            hipLaunchKernelGGL(columns_long_kernel<T>, dim3((width + BLOCK - 1) / BLOCK, parts), dim3(BLOCK), 0, st, x, ld_x, dy, ld_dy, n, width,
                               mean, rstd, partial);
        if (dx)
            hipLaunchKernelGGL(backward_long_kernel<T>, dim3(at_most(n, 2048)), dim3(BLOCK), 0, st, x, ld_x, dy, ld_dy, n, width, gamma, mean,
                               rstd, dx, ld_dx);
    }
    if (partial)
        hipLaunchKernelGGL(join_kernel, dim3((2 * width + 63) / 64), dim3(1024), 0, st, partial, parts, width, dgamma, dbeta);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

int32_t check(int32_t order, uint64_t ld, uint64_t n, uint32_t width)
{
    return ld < (order == ECK_COLUMNS ? n : (uint64_t)width) ? ECK_ESHAPE : ECK_OK;
}

int32_t check_sizes(int32_t order, uint64_t n, uint32_t width)
{
    if (order == ECK_COLUMNS && width > ECK_MAX_COLUMNS_WIDTH) return ECK_EUNSUPPORTED;
    return n > MAX_ROWS || width > MAX_WIDTH ? ECK_EUNSUPPORTED : ECK_OK;
}

} // namespace
} // namespace eck

using namespace eck;

extern "C" int32_t layernorm_forward(const void *x, int32_t x_order, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t width,
                                     const float *gamma, const float *beta, float eps, void *y, uint64_t ld_y, float *mean_out,
                                     float *rstd_out, void *stream)
{
    if (!x || !y || !mean_out != !rstd_out || n == 0 || width == 0 || !is_dtype(dtype)) return ECK_EINVAL;
    if ((x_order != ECK_ROWS && x_order != ECK_COLUMNS) || !(eps >= 0.0f) || eps > 3.402823466e38f) return ECK_EINVAL;
    if (check(x_order, ld_x, n, width) != ECK_OK || ld_y < width) return ECK_ESHAPE;
    if (int32_t rc = check_sizes(x_order, n, width)) return rc;
    const uint64_t size = element_bytes(dtype);
    if (!aligned(x, size) || !aligned(y, size) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean_out, 4) || !aligned(rstd_out, 4))
        return ECK_EALIGN;
    return dtype == ECK_F32 ? forward<float>(x, x_order, ld_x, n, width, gamma, beta, eps, y, ld_y, mean_out, rstd_out, as_stream(stream))
                            : forward<bf16>(x, x_order, ld_x, n, width, gamma, beta, eps, y, ld_y, mean_out, rstd_out, as_stream(stream));
}

extern "C" uint64_t layernorm_backward_workspace_bytes(uint64_t n, uint32_t width, int32_t dtype)
{
    if (n == 0 || width == 0 || n > MAX_ROWS || width > MAX_WIDTH || !is_dtype(dtype)) return 0;
    const uint64_t rows = backward_blocks(n, width, dtype, ECK_ROWS), columns = width <= ECK_MAX_COLUMNS_WIDTH ? backward_blocks(n, width, dtype, ECK_COLUMNS) : 0;
    return (rows > columns ? rows : columns) * 2 * width * sizeof(float);
}

extern "C" int32_t layernorm_backward(const void *x, int32_t x_order, int32_t dtype, uint64_t ld_x, const void *dy, uint64_t ld_dy,
                                      uint64_t n, uint32_t width, const float *gamma, const float *mean, const float *rstd, void *dx_out,
                                      uint64_t ld_dx, float *dgamma_out, float *dbeta_out, void *ws, uint64_t ws_bytes, void *stream)
{
    if (!x || !dy || !mean || !rstd || !dgamma_out != !dbeta_out || (!dx_out && !dgamma_out) || n == 0 || width == 0) return ECK_EINVAL;
    if (!is_dtype(dtype) || (x_order != ECK_ROWS && x_order != ECK_COLUMNS)) return ECK_EINVAL;
    if (check(x_order, ld_x, n, width) != ECK_OK || ld_dy < width || (dx_out && check(x_order, ld_dx, n, width) != ECK_OK)) return ECK_ESHAPE;
    if (int32_t rc = check_sizes(x_order, n, width)) return rc;
    if (dgamma_out && (!ws || ws_bytes < layernorm_backward_workspace_bytes(n, width, dtype))) return ECK_EWORKSPACE;
    const uint64_t size = element_bytes(dtype);
    if (!aligned(x, size) || !aligned(dy, size) || !aligned(dx_out, size) || !aligned(gamma, 4) || !aligned(mean, 4) || !aligned(rstd, 4) ||
        !aligned(dgamma_out, 4) || !aligned(dbeta_out, 4) || (dgamma_out && !aligned(ws, 256)))
        return ECK_EALIGN;
    return dtype == ECK_F32 ? backward<float>(x, x_order, ld_x, dy, ld_dy, n, width, gamma, mean, rstd, dx_out, ld_dx, dgamma_out, dbeta_out,
                                              (float *)ws, as_stream(stream))
                            : backward<bf16>(x, x_order, ld_x, dy, ld_dy, n, width, gamma, mean, rstd, dx_out, ld_dx, dgamma_out, dbeta_out,
                                             (float *)ws, as_stream(stream));
}
