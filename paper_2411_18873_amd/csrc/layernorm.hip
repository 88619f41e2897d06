// Layer norm of rows of activations or of candidates' features, forward and backward (HIP, gfx950).
//
//   forward   m = sum x / w,  r = 1 / sqrt(sum (x - m)^2 / w + eps),  y = (x - m) r gamma + beta
//   backward  g = dy gamma, xh = (x - m) r:  dx = r (g - mean(g) - xh mean(g xh)),  dgamma = sum dy xh,  dbeta = sum dy
//
// Every pass is bound by memory.  A row stays in registers between its sums and its result (the two sums of the forward pass one
// after the other: the squares of differences from the mean lose nothing to a large mean), shared by as many threads as sixteen
// bytes each need: 8 to 64 lanes of a wavefront, or a block.  Threads keep their columns from row to row, so gamma and beta are
// loaded once, and the parameters' gradients grow in registers: blocks leave one partial sum per column and a second launch adds
// these in a fixed order.  Rows longer than a block's registers are read again for every pass; their threads add up thousands of
// values, and do it in 64 bits, sixteen bytes' sum at a time (in 32, 4096 equal values in a row are off by 650 roundings).
#include "activations.h"
#include "lanes.h"

#include <type_traits>

namespace eck {
namespace {

constexpr int BLOCK = 256;

// Sums over groups of TPR neighbouring lanes, or over the block, in every thread; all threads have to call it.  Loads stay on their
// way across its barrier.  Two calls in a row use different halves of scratch (turn: 0 and 1), so that one barrier each will do.
template <int TPR, int COUNT>
__device__ __forceinline__ void row_sums(float (&v)[COUNT], float (*scratch)[COUNT][BLOCK / 64], int turn)
{
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
#pragma unroll
        for (uint32_t stride = 1; stride < 64 && stride < TPR; stride <<= 1) v[i] += __uint_as_float(lane_exchange(__float_as_uint(v[i]), stride));
    if (TPR <= 64) return;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < COUNT; ++i) scratch[turn][i][threadIdx.x >> 6] = v[i];
    lds_barrier();
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        v[i] = scratch[turn][i][0];
#pragma unroll
        for (int w = 1; w < BLOCK / 64; ++w) v[i] += scratch[turn][i][w];
    }
}

// the sum over the block
__device__ __forceinline__ float block_sum(float v, float (*scratch)[1][BLOCK / 64], int turn)
{
    float one[1] = {v};
    row_sums<BLOCK, 1>(one, scratch, turn);
    return one[0];
}

// a thread's parameters: elements at .. at + N - 1 of gamma or beta, ones or zeros where there are none
template <int N>
__device__ __forceinline__ void load_vector(const float *p, uint32_t at, uint32_t width, float none, float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        float some[4] = {none, none, none, none};
        if (p) load_chunk(p, at + i, width, some, none);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i + j] = some[j];
    }
}

template <class T, int TPR, int ITEMS>
__global__ __launch_bounds__(BLOCK) void forward_kernel(const T *x, uint64_t ld_x, uint64_t n, uint32_t width, const float *gamma,
                                                        const float *beta, float eps, T *y, uint64_t ld_y, float *mean_out, float *rstd_out)
{
    constexpr int N = Chunk<T>::N, ROWS = BLOCK / TPR;
    __shared__ float scratch[2][1][BLOCK / 64];
    const uint32_t lane = threadIdx.x % TPR;
    const float share = 1.0f / (float)width;
    Chunk<T> raw[ITEMS];
    const auto fetch = [&](uint64_t r) {
        const T *row = x + (r < n ? r : n - 1) * ld_x; // (all lanes stay, for the sums)
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) raw[k] = fetch_chunk(row, (k * TPR + lane) * N, width);
    };
    uint64_t r = (uint64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
    fetch(r);
    float ga[ITEMS][N], be[ITEMS][N];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        load_vector(gamma, (k * TPR + lane) * N, width, 1.0f, ga[k]);
        load_vector(beta, (k * TPR + lane) * N, width, 0.0f, be[k]);
    }
    for (uint64_t r0 = (uint64_t)blockIdx.x * ROWS; r0 < n; r0 += (uint64_t)gridDim.x * ROWS) {
        float v[ITEMS][N], sum[1] = {0.0f}, squares[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[k][i] = (float)raw[k].v[i];
                sum[0] += v[k][i];
            }
        const uint64_t here = r;
        r += (uint64_t)gridDim.x * ROWS;
        if (r0 + (uint64_t)gridDim.x * ROWS < n) fetch(r); // on its way while this row is worked out
        row_sums<TPR>(sum, scratch, 0);
        const float mean = sum[0] * share;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[k][i] -= mean;
                squares[0] += (k * TPR + lane) * N + i < width ? v[k][i] * v[k][i] : 0.0f;
            }
        row_sums<TPR>(squares, scratch, 1);
        const float rstd = 1.0f / sqrtf(squares[0] * share + eps);
        if (here >= n) continue;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[k][i] = v[k][i] * rstd * ga[k][i] + be[k][i];
            store_chunk(y + here * ld_y, (k * TPR + lane) * N, width, v[k]);
        }
        if (mean_out && lane == 0) {
            mean_out[here] = mean;
            rstd_out[here] = rstd;
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
    __shared__ float scratch[2][1][BLOCK / 64];
    const float share = 1.0f / (float)width;
    for (uint64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const T *row = x + r * ld_x;
        double sum = 0.0, squares = 0.0;
        float v[N];
        for (uint32_t at = threadIdx.x * N; at < width; at += BLOCK * N) {
            float some = 0.0f;
            load_chunk(row, at, width, v);
#pragma unroll
            for (int i = 0; i < N; ++i) some += v[i];
            sum += (double)some;
        }
        const float mean = block_sum((float)sum, scratch, 0) * share;
        for (uint32_t at = threadIdx.x * N; at < width; at += BLOCK * N) {
            float some = 0.0f;
            load_chunk(row, at, width, v, mean);
#pragma unroll
            for (int i = 0; i < N; ++i) some += (v[i] - mean) * (v[i] - mean);
            squares += (double)some;
        }
        const float rstd = 1.0f / sqrtf(block_sum((float)squares, scratch, 1) * share + eps);
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
    __shared__ float scratch[2][2][WAVES];
    __shared__ float joined[TPR > 64 ? 1 : WAVES * TPR * N];
    const uint32_t lane = threadIdx.x % TPR;
    const float share = 1.0f / (float)width;
    Chunk<T> raw_x[ITEMS], raw_d[ITEMS];
    float m, s;
    const auto fetch = [&](uint64_t r) {
        const uint64_t from = r < n ? r : n - 1;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            raw_x[k] = fetch_chunk(x + from * ld_x, (k * TPR + lane) * N, width);
            raw_d[k] = fetch_chunk(dy + from * ld_dy, (k * TPR + lane) * N, width);
        }
        m = mean[from];
        s = rstd[from];
    };
    uint64_t r = (uint64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
    fetch(r);
    float ga[ITEMS][N], dgamma[ITEMS][N], dbeta[ITEMS][N];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        load_vector(gamma, (k * TPR + lane) * N, width, 1.0f, ga[k]);
#pragma unroll
        for (int i = 0; i < N; ++i) dgamma[k][i] = dbeta[k][i] = 0.0f;
    }
    int turn = 0;
    for (uint64_t r0 = (uint64_t)blockIdx.x * ROWS; r0 < n; r0 += (uint64_t)gridDim.x * ROWS, turn ^= 1) {
        const bool counts = r < n;
        float xh[ITEMS][N], d[ITEMS][N], sums[2] = {0.0f, 0.0f}; // of g and of g xh
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                xh[k][i] = (k * TPR + lane) * N + i < width ? ((float)raw_x[k].v[i] - m) * s : 0.0f;
                d[k][i] = (float)raw_d[k].v[i];
                dgamma[k][i] += counts ? d[k][i] * xh[k][i] : 0.0f;
                dbeta[k][i] += counts ? d[k][i] : 0.0f;
                d[k][i] *= ga[k][i];
                sums[0] += d[k][i];
                sums[1] += d[k][i] * xh[k][i];
            }
        const uint64_t here = r;
        const float scale = s;
        r += (uint64_t)gridDim.x * ROWS;
        if (r0 + (uint64_t)gridDim.x * ROWS < n) fetch(r); // on its way while this row is worked out
        if (!dx) continue;                                 // (for all threads)
        row_sums<TPR>(sums, scratch, turn);
        const float from_g = sums[0] * share, from_dot = sums[1] * share;
        if (!counts) continue;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
#pragma unroll
            for (int i = 0; i < N; ++i) d[k][i] = scale * (d[k][i] - from_g - xh[k][i] * from_dot);
            store_chunk(dx + here * ld_dx, (k * TPR + lane) * N, width, d[k]);
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
                store_chunk(mine + which * width, (k * TPR + lane) * N, width, v);
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
    __shared__ float scratch[2][1][BLOCK / 64];
    const float share = 1.0f / (float)width;
    for (uint64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const float m = mean[r], s = rstd[r];
        double sums = 0.0, dots = 0.0;
        float xh[N], d[N], ga[N];
        for (uint32_t at = threadIdx.x * N; at < width; at += BLOCK * N) {
            float of_g = 0.0f, of_dot = 0.0f;
            load_chunk(x + r * ld_x, at, width, xh, m);
            load_chunk(dy + r * ld_dy, at, width, d);
            load_vector(gamma, at, width, 1.0f, ga);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                of_g += d[i] * ga[i];
                of_dot += d[i] * ga[i] * ((xh[i] - m) * s);
            }
            sums += (double)of_g;
            dots += (double)of_dot;
        }
        const float sum = block_sum((float)sums, scratch, 0) * share, dot = block_sum((float)dots, scratch, 1) * share;
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
    double dgamma = 0.0, dbeta = 0.0;
    for (uint64_t r = blockIdx.y; r < n; r += gridDim.y) {
        const float d = (float)dy[r * ld_dy + c];
        dgamma += (double)(d * (((float)x[r * ld_x + c] - mean[r]) * rstd[r]));
        dbeta += (double)d;
    }
    partial[(uint64_t)blockIdx.y * 2 * width + c] = (float)dgamma;
    partial[(uint64_t)blockIdx.y * 2 * width + width + c] = (float)dbeta;
}

// dgamma and dbeta: the blocks' partial sums; sixteen columns a block, 64 threads each
__global__ __launch_bounds__(1024) void join_kernel(const float *partial, uint32_t parts, uint32_t width, float *dgamma, float *dbeta)
{
    __shared__ float sums[64][17];
    const uint64_t columns = 2ull * width, c = (uint64_t)blockIdx.x * 16 + threadIdx.x % 16;
    const uint32_t slice = threadIdx.x / 16;
    float sum = 0.0f;
    if (c < columns) {
#pragma unroll 4
        for (uint32_t p = slice; p < parts; p += 64) sum += partial[p * columns + c];
    }
    sums[slice][threadIdx.x % 16] = sum;
    __syncthreads();
    if (threadIdx.x >= 256) return;
    // sixteen lanes a column: lane j adds rows j, j + 16, ..., then the lanes each other
    const uint32_t column = threadIdx.x / 16, j = threadIdx.x % 16;
    sum = (sums[j][column] + sums[j + 16][column]) + (sums[j + 32][column] + sums[j + 48][column]);
#pragma unroll
    for (uint32_t stride = 1; stride < 16; stride <<= 1) sum += __uint_as_float(lane_exchange(__float_as_uint(sum), stride));
    const uint64_t at = (uint64_t)blockIdx.x * 16 + column;
    if (j != 0 || at >= columns) return;
    if (at < width) dgamma[at] = sum;
    else dbeta[at - width] = sum;
}

// ------------------------------------------------------------------------------------------------ features
//
// A block takes tiles of four times CHUNKS candidates.  Thread (group, chunk) holds four candidates of four neighbouring features at
// a time; rows go through the LDS, because a candidate's features lie ld elements apart on one side and next to each other on the
// other.  In a row, sixteen bytes are stored in place p ^ chunk % 8, or all chunks would write to the same banks.  The next tile is
// on its way while one is worked out: blocks of one tile each were bound by the rate at which blocks start (2^20 candidates of 64
// bf16 features: 91 us).

template <class T, int CHUNKS_>
struct Columns {
    static constexpr int N = 4, CHUNKS = CHUNKS_, GROUPS = BLOCK / CHUNKS, TILE = CHUNKS * N, FEATURES = 4 * GROUPS;
    static constexpr int VECTOR = 16 / sizeof(T), LINE = 128 / sizeof(T); // rows are whole 128 bytes
    typedef T Granule __attribute__((ext_vector_type(4)));
    typedef T Whole __attribute__((ext_vector_type(VECTOR)));
    static __host__ __device__ uint32_t pitch(uint32_t width) { return (width + LINE - 1) / LINE * LINE; }
    // where features from f on (four from a multiple of four, or sixteen bytes from a multiple of VECTOR) of candidate c lie
    static __device__ __forceinline__ T *at(T *rows, uint32_t pitch, uint32_t c, uint32_t f)
    {
        return rows + c * pitch + (f ^ (c / N % 8 * VECTOR));
    }
};

// sums over the features of each of a thread's N candidates, in all threads with that chunk
template <class C>
__device__ __forceinline__ void candidate_sums(float (&v)[C::N], float (*scratch)[C::TILE])
{
    const uint32_t chunk = threadIdx.x % C::CHUNKS;
#pragma unroll
    for (int i = 0; i < C::N; ++i)
#pragma unroll
        for (uint32_t stride = C::CHUNKS; stride < 64; stride <<= 1) v[i] += __uint_as_float(lane_exchange(__float_as_uint(v[i]), stride));
    if ((threadIdx.x & 63) < C::CHUNKS)
#pragma unroll
        for (int i = 0; i < C::N; ++i) scratch[threadIdx.x >> 6][chunk * C::N + i] = v[i];
    lds_barrier();
#pragma unroll
    for (int i = 0; i < C::N; ++i) {
        v[i] = scratch[0][chunk * C::N + i];
#pragma unroll
        for (int w = 1; w < BLOCK / 64; ++w) v[i] += scratch[w][chunk * C::N + i];
    }
}

// a thread's features of the tile from candidate `first` on, zeros past the matrix
template <class C, class T, int ITEMS>
__device__ __forceinline__ void fetch_features(const T *x, uint64_t ld_x, uint32_t width, uint64_t first, uint64_t n,
                                               Chunk<T, C::N> (&raw)[ITEMS][4])
{
    const uint32_t f0 = threadIdx.x / C::CHUNKS * 4;
    const uint64_t c = first + threadIdx.x % C::CHUNKS * C::N;
    if (first + C::TILE <= n) { // (the same for the block)
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t f = k * C::FEATURES + f0 + j;
                raw[k][j] = {};
                if (f < width) raw[k][j] = *reinterpret_cast<const Chunk<T, C::N> *>(x + f * ld_x + c);
            }
    } else {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < C::N; ++i) {
                    const uint32_t f = k * C::FEATURES + f0 + j;
                    raw[k][j].v[i] = (T)0.0f;
                    if (f < width && c + i < n) raw[k][j].v[i] = x[f * ld_x + c + i];
                }
    }
}

template <class T, int CHUNKS, int ITEMS>
__global__ __launch_bounds__(BLOCK) void forward_columns_kernel(const T *x, uint64_t ld_x, uint64_t n, uint32_t width, const float *gamma,
                                                                const float *beta, float eps, T *y, uint64_t ld_y, float *mean_out,
                                                                float *rstd_out)
{
    using C = Columns<T, CHUNKS>;
    constexpr int N = C::N, TILE = C::TILE;
    extern __shared__ __attribute__((aligned(16))) unsigned char dynamic[];
    T *rows = reinterpret_cast<T *>(dynamic);
    __shared__ float scratch[2][BLOCK / 64][TILE];
    const uint32_t chunk = threadIdx.x % C::CHUNKS, group = threadIdx.x / C::CHUNKS, pitch = C::pitch(width), chunks = (width + C::VECTOR - 1) / C::VECTOR;
    const float share = 1.0f / (float)width;
    Chunk<T, N> raw[ITEMS][4];
    fetch_features<C, T, ITEMS>(x, ld_x, width, (uint64_t)blockIdx.x * TILE, n, raw);
    for (uint64_t first = (uint64_t)blockIdx.x * TILE; first < n; first += (uint64_t)gridDim.x * TILE) {
        const uint32_t here = (uint32_t)(n - first < TILE ? n - first : TILE);
        float v[ITEMS][4][N], mean[N], rstd[N];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) v[k][j][i] = (float)raw[k][j].v[i];
        // the next tile is on its way while this one is worked out
        fetch_features<C, T, ITEMS>(x, ld_x, width, first + (uint64_t)gridDim.x * TILE, n, raw);
#pragma unroll
        for (int i = 0; i < N; ++i) mean[i] = rstd[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) mean[i] += v[k][j][i];
        candidate_sums<C>(mean, scratch[0]);
#pragma unroll
        for (int i = 0; i < N; ++i) mean[i] *= share;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    v[k][j][i] -= mean[i];
                    rstd[i] += k * C::FEATURES + 4 * group + j < width ? v[k][j][i] * v[k][j][i] : 0.0f;
                }
        candidate_sums<C>(rstd, scratch[1]);
#pragma unroll
        for (int i = 0; i < N; ++i) rstd[i] = 1.0f / sqrtf(rstd[i] * share + eps);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const uint32_t f = k * C::FEATURES + 4 * group;
            if (f >= pitch) continue;
            float ga[4], be[4];
            load_vector(gamma, f, width, 1.0f, ga);
            load_vector(beta, f, width, 0.0f, be);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                typename C::Granule out;
#pragma unroll
                for (int j = 0; j < 4; ++j) out[j] = (T)(v[k][j][i] * rstd[i] * ga[j] + be[j]);
                *reinterpret_cast<typename C::Granule *>(C::at(rows, pitch, chunk * N + i, f)) = out;
            }
        }
        if (mean_out && group == 0)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (chunk * N + i < here) {
                    mean_out[first + chunk * N + i] = mean[i];
                    rstd_out[first + chunk * N + i] = rstd[i];
                }
        lds_barrier();
        for (uint32_t j = threadIdx.x; j < here * chunks; j += BLOCK) {
            const uint32_t c = j / chunks, at = j % chunks * C::VECTOR;
            const typename C::Whole whole = *reinterpret_cast<const typename C::Whole *>(C::at(rows, pitch, c, at));
            float out[C::VECTOR];
#pragma unroll
            for (int i = 0; i < C::VECTOR; ++i) out[i] = (float)whole[i];
            store_chunk(y + (first + c) * ld_y, at, width, out);
        }
        lds_barrier();
    }
}

template <class T, int CHUNKS, int ITEMS>
__global__ __launch_bounds__(BLOCK) void backward_columns_kernel(const T *x, uint64_t ld_x, const T *dy, uint64_t ld_dy, uint64_t n,
                                                                 uint32_t width, const float *gamma, const float *mean, const float *rstd,
                                                                 T *dx, uint64_t ld_dx, float *partial)
{
    using C = Columns<T, CHUNKS>;
    constexpr int N = C::N, TILE = C::TILE;
    extern __shared__ __attribute__((aligned(16))) unsigned char dynamic[];
    T *rows = reinterpret_cast<T *>(dynamic);
    __shared__ float scratch[2][BLOCK / 64][TILE];
    const uint32_t chunk = threadIdx.x % C::CHUNKS, group = threadIdx.x / C::CHUNKS, pitch = C::pitch(width), chunks = (width + C::VECTOR - 1) / C::VECTOR;
    const float share = 1.0f / (float)width;
    float dgamma[ITEMS][4], dbeta[ITEMS][4];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) dgamma[k][j] = dbeta[k][j] = 0.0f;
    Chunk<T, N> raw[ITEMS][4];
    fetch_features<C, T, ITEMS>(x, ld_x, width, (uint64_t)blockIdx.x * TILE, n, raw);
    for (uint64_t first = (uint64_t)blockIdx.x * TILE; first < n; first += (uint64_t)gridDim.x * TILE) {
        const uint32_t here = (uint32_t)(n - first < TILE ? n - first : TILE);
        for (uint32_t j = threadIdx.x; j < here * chunks; j += BLOCK) {
            const uint32_t c = j / chunks, at = j % chunks * C::VECTOR;
            *reinterpret_cast<typename C::Whole *>(C::at(rows, pitch, c, at)) = fetch_chunk(dy + (first + c) * ld_dy, at, width).v;
        }
        float m[N], s[N], sum[N], dot[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool counts = chunk * N + i < here;
            m[i] = counts ? mean[first + chunk * N + i] : 0.0f;
            s[i] = counts ? rstd[first + chunk * N + i] : 0.0f;
            sum[i] = dot[i] = 0.0f;
        }
        lds_barrier();
        float xh[ITEMS][4][N], d[ITEMS][4][N];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const uint32_t f = k * C::FEATURES + 4 * group;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) xh[k][j][i] = (float)raw[k][j].v[i];
            float ga[4];
            load_vector(gamma, f, width, 1.0f, ga);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                typename C::Granule in = {};
                if (f < pitch) in = *reinterpret_cast<const typename C::Granule *>(C::at(rows, pitch, chunk * N + i, f));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool counts = f + j < width && chunk * N + i < here;
                    xh[k][j][i] = counts ? (xh[k][j][i] - m[i]) * s[i] : 0.0f;
                    d[k][j][i] = counts ? (float)in[j] : 0.0f;
                    dgamma[k][j] += d[k][j][i] * xh[k][j][i];
                    dbeta[k][j] += d[k][j][i];
                    d[k][j][i] *= ga[j];
                    sum[i] += d[k][j][i];
                    dot[i] += d[k][j][i] * xh[k][j][i];
                }
            }
        }
        fetch_features<C, T, ITEMS>(x, ld_x, width, first + (uint64_t)gridDim.x * TILE, n, raw);
        if (dx) {
            candidate_sums<C>(sum, scratch[0]);
            candidate_sums<C>(dot, scratch[1]);
#pragma unroll
            for (int k = 0; k < ITEMS; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t f = k * C::FEATURES + 4 * group + j;
                    if (f >= width) continue;
#pragma unroll
                    for (int i = 0; i < N; ++i) d[k][j][i] = s[i] * (d[k][j][i] - sum[i] * share - xh[k][j][i] * (dot[i] * share));
                    store_chunk(dx + f * ld_dx + first, chunk * N, here, d[k][j]);
                }
        }
        lds_barrier();
    }
    if (!partial) return;
    float *mine = partial + (uint64_t)blockIdx.x * 2 * width;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (uint32_t stride = 1; stride < C::CHUNKS; stride <<= 1) {
                dgamma[k][j] += __uint_as_float(lane_exchange(__float_as_uint(dgamma[k][j]), stride));
                dbeta[k][j] += __uint_as_float(lane_exchange(__float_as_uint(dbeta[k][j]), stride));
            }
            const uint32_t f = k * C::FEATURES + 4 * group + j;
            if (chunk == 0 && f < width) {
                mine[f] = dgamma[k][j];
                mine[width + f] = dbeta[k][j];
            }
        }
}

// ------------------------------------------------------------------------------------------------ launches

// Calls f with the number of threads a row and the chunks a thread that hold a row of `width`; false if none does.  (A power of
// two below 64 lanes wastes less than half of them on short rows; a wavefront holds two chunks a lane, or four in the backward
// pass, then a block takes over.  16384 rows of 2000 bf16: forward 28.5 us by blocks, 30.8 by wavefronts; backward 57.3 and 48.2.)
template <class T, int WAVE_ITEMS, class F>
bool with_row_shape(uint32_t width, F &&f)
{
    constexpr uint32_t N = 16 / sizeof(T);
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
    if constexpr (WAVE_ITEMS == 4) { ECK_ROW_SHAPE(64, 4) }
    else { ECK_ROW_SHAPE(256, 1) }
    ECK_ROW_SHAPE(256, 2)
    ECK_ROW_SHAPE(256, 4)
#undef ECK_ROW_SHAPE
    return false;
}

// the same for the chunks of a tile and the fours of features a thread: as many candidates as 32 features a thread allow, 256 bytes
// of each feature at most
template <class T, class F>
void with_columns_shape(uint32_t width, F &&f)
{
    static_assert(ECK_MAX_COLUMNS_WIDTH == 256, "no width is left out");
    constexpr int MOST = 64 / sizeof(T), ONE = 1024 / MOST; // ONE: features that one four a thread holds then
    if (width <= ONE) return f(std::integral_constant<int, MOST>{}, std::integral_constant<int, 1>{});
    if constexpr (ONE < 64)
        if (width <= 64) return f(std::integral_constant<int, MOST>{}, std::integral_constant<int, 2>{});
    if (width <= 128) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
    else f(std::integral_constant<int, 8>{}, std::integral_constant<int, 2>{});
}

uint32_t at_most(uint64_t blocks, uint32_t most) { return (uint32_t)(blocks < most ? blocks : most); }

// Blocks of the backward pass, each of which leaves a partial sum per column: what keeps 32 KB on their way to a compute unit, one
// to four a unit, two at least of blocks that work on several rows at once.  (us by 1, 2, 3 and 4 a unit: 8192 rows of 4096 bf16
// 52.9, 49.0, 54.7, 67.9; of fp32 81.6, 86.2, 93.9, 93.8; 32768 of 1024 bf16 39.8, 37.6, 38.7, 46.0; 50003 of 250 fp32 66.8, 44.3,
// 37.0, 33.7; 16384 of 2000 bf16 57.4, 48.2.)  One where the partial sums, 16 bytes a column written and read, would be more than what the rows
// move (1000 rows of 4096 bf16: 16.1 for 19.3; 1967 of 3840 stay at two, 23.1 for 25.7).
uint32_t backward_blocks(uint64_t n, uint32_t width, int32_t dtype, int32_t order)
{
    if (order == ECK_COLUMNS) return at_most((n + 31) / 32, 1024); // (32 candidates: the smallest tile)
    const uint64_t size = element_bytes(dtype), vector = 16 / size, chunks = (width + vector - 1) / vector;
    uint64_t rows = 1; // a block's at a time
    for (uint64_t tpr = 8; tpr <= 64 && rows == 1; tpr *= 2)
        if (chunks <= tpr * (tpr == 64 ? 4 : 1)) rows = BLOCK / tpr;
    uint64_t a_unit = 32768 / (2 * rows * width * size);
    a_unit = a_unit > 4 ? 4 : a_unit < 1 ? 1 : a_unit;
    if (rows > 1 && a_unit < 2) a_unit = 2;
    if (16 * 256 * a_unit > n * 3 * size) a_unit = 1;
    return at_most((n + rows - 1) / rows, (uint32_t)(256 * a_unit));
}
constexpr uint32_t LONG_PARTS = 64;

template <class T>
int32_t forward(const void *x, int32_t order, uint64_t ld_x, uint64_t n, uint32_t width, const float *gamma, const float *beta, float eps,
                void *y, uint64_t ld_y, float *mean, float *rstd, hipStream_t st)
{
    if (order == ECK_COLUMNS) {
        with_columns_shape<T>(width, [&](auto chunks, auto items) {
            using C = Columns<T, decltype(chunks)::value>;
            hipLaunchKernelGGL((forward_columns_kernel<T, C::CHUNKS, decltype(items)::value>), dim3(at_most((n + C::TILE - 1) / C::TILE, 2048)),
                               dim3(BLOCK), C::TILE * C::pitch(width) * sizeof(T), st, (const T *)x, ld_x, n, width, gamma, beta, eps, (T *)y, ld_y,
                               mean, rstd);
        });
    } else if (!with_row_shape<T, 2>(width, [&](auto tpr, auto items) {
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
        with_columns_shape<T>(width, [&](auto chunks, auto items) {
            using C = Columns<T, decltype(chunks)::value>;
            hipLaunchKernelGGL((backward_columns_kernel<T, C::CHUNKS, decltype(items)::value>), dim3(parts), dim3(BLOCK),
                               C::TILE * C::pitch(width) * sizeof(T), st, x, ld_x, dy, ld_dy, n, width, gamma, mean, rstd, dx, ld_dx, partial);
        });
    } else if (!with_row_shape<T, 4>(width, [&](auto tpr, auto items) {
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
        hipLaunchKernelGGL(join_kernel, dim3((2 * width + 15) / 16), dim3(1024), 0, st, partial, parts, width, dgamma, dbeta);
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
