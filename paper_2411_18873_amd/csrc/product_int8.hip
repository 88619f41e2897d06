// Products of matrices of 8-bit integers with a scale for each row of both, and gates of pairs of them, on the matrix cores (HIP, gfx950).
//
//   y[m][c] = (sum over k of x[m][k] w[c][k]) s_x[m] s_w[c],   or a(g) u of two such
//
// Sums are 32-bit integers, so they are exact whatever the order, in any number of shares of k.  Both operands lie along k; to the
// staging of product.h two neighbouring integers are one of its elements (the sixteen bytes that a lane feeds to a matrix instruction lie
// in memory and in the LDS as eight bfloat16 values do), so stages, their swizzles and their waits are those.
#include "product.h"

namespace eck {
namespace {

using namespace product;

constexpr uint32_t MOST_IN = 131071;      // integers of magnitude 128: 131072 products of 2^14 are 2^31
constexpr uint64_t MOST_OUT = 1u << 20;
constexpr uint64_t MOST_TILES = 1u << 22; // of 64 x 64

struct Result {
    const float *x_scale, *w_scale;
    void *y;
    uint64_t ld_y;
    uint32_t n_out; // columns of y, and rows of w from a gate to its up
    int32_t act;    // ECK_ACT_*
    int32_t f32;    // y's type
};

struct Int8Product {
    const int8_t *x, *w;
    uint64_t ld_x, ld_w;
    uint32_t n, n_in;
    uint32_t tiles_m, tiles_n, shares;
    int32_t *partial; // shares > 1: sums of each, [share][n][columns]
    uint32_t columns; // of w: n_out, or twice that
    Result to;
};

// scales of eight neighbouring columns (0 past the last), and of their ups
template <bool GATE_>
struct Scales {
    float w[8], up[GATE_ ? 8 : 1];
    __device__ __forceinline__ void load(const Result &to, uint32_t c)
    {
        load_eight_of(to.w_scale, c, to.n_out, w);
        if constexpr (GATE_) load_eight_of(to.w_scale + to.n_out, c, to.n_out, up);
    }
    static __device__ __forceinline__ void load_eight_of(const float *row, uint32_t c, uint32_t n, float (&v)[8])
    {
        float low[4], high[4];
        load_chunk(row, c, n, low);
        load_chunk(row, c + 4, n, high);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = low[i], v[4 + i] = high[i];
    }
};

template <class T, bool GATE_>
__device__ __forceinline__ void finish_as(const Result &to, uint64_t m, uint32_t c, float row, const Scales<GATE_> &scales, const int (&v)[8],
                                          const int (&u)[8])
{
    float y[8], up[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y[i] = (float)v[i] * row * scales.w[i];
        if constexpr (GATE_) up[i] = (float)u[i] * row * scales.up[i];
    }
    if (GATE_)
        with_act(to.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = gate_as<decltype(act)::value, sizeof(T) == 4>(y[i]).value * up[i];
        });
    store_eight((T *)to.y + m * to.ld_y, c, to.n_out, y);
}
template <bool GATE_>
__device__ __forceinline__ void finish(const Result &to, uint64_t m, uint32_t c, float row, const Scales<GATE_> &scales, const int (&v)[8],
                                       const int (&u)[8])
{
    if (to.f32) finish_as<float, GATE_>(to, m, c, row, scales, v, u);
    else finish_as<bf16, GATE_>(to, m, c, row, scales, v, u);
}

// ------------------------------------------------------------------------------------------------ tiles

// The matrix cores bound large products (8192 rows, 4096 integers, 8192 gated columns: 472-495 us, 2220-2330 TOPS, where the library's
// ungated product of these sizes reaches 2220), the weights' bytes those of few rows (one row of the same: 12.5 us for 67 MB).
template <class S, bool GATE_, bool SHARED>
__global__ __launch_bounds__(S::THREADS) __attribute__((amdgpu_waves_per_eu(S::AT_ONCE, S::AT_ONCE))) void tiles_kernel(const Int8Product p)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    typedef Stage<S::BM, true, S::WAVES, 1> StageA;
    typedef Stage<S::BN, true, S::WAVES, 1> StageB;
    constexpr int PER_STEP = StageA::LOADS + StageB::LOADS, BK = S::BK; // BK: pairs of integers
    constexpr uint32_t STAGE = S::STAGE;
    constexpr bool PAIRED = GATE_ && !SHARED; // gates and their ups in one tile
    constexpr int COLUMNS = PAIRED ? S::BN / 2 : S::BN;

    // blocks go round the eight dies, whose blocks take neighbouring tiles, in panels eight tiles high
    const uint32_t tiles = p.tiles_m * p.tiles_n, total = gridDim.x, die = blockIdx.x & 7, left_over = total & 7;
    const uint32_t number = die * (total >> 3) + min(die, left_over) + (blockIdx.x >> 3);
    const uint32_t share = number / tiles, tile = number % tiles, panel = tile / (8 * p.tiles_n), in_panel = tile % (8 * p.tiles_n);
    const uint32_t high = min(8u, p.tiles_m - 8 * panel);
    const uint32_t m0 = (8 * panel + in_panel % high) * S::BM, c0 = in_panel / high * COLUMNS;
    const uint32_t N = PAIRED ? p.to.n_out : p.columns;

    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    StageA sa;
    StageB sb;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds;
    constexpr uint32_t HALF = S::BN / S::WN / 2; // of a wavefront's columns the first half are gates, the second the ups of the same units
    sa.init(p.ld_x / 2, lds0, [&](uint32_t r) { return m0 + r < p.n ? r : NOWHERE; });
    // (a gate's up may lie 2^32 bytes and more behind it: ups are loaded from a base of their own)
    const int8_t *at_b = p.w + c0 * p.ld_w;
    sb.init(p.ld_w / 2, lds0 + StageA::BYTES, [&](uint32_t c) {
        if (!PAIRED) return c0 + c < N ? c : NOWHERE;
        const uint32_t unit = c / (2 * HALF) * HALF + c % HALF;
        return c0 + unit < N ? unit : NOWHERE;
    });
    // which of this wavefront's loads bring ups (the same for all lanes: a load brings eight rows)
    static_assert(HALF % 8 == 0, "a load's rows are all gates or all ups");
    const uint64_t up = PAIRED ? (uint64_t)p.to.n_out * p.ld_w : 0;

    const uint32_t pairs = (p.n_in + 15) / 16 * 8, all = (pairs + BK - 1) / BK;
    const uint32_t first = (uint32_t)((uint64_t)all * share / p.shares), steps = (uint32_t)((uint64_t)all * (share + 1) / p.shares) - first;
    const int8_t *at_a = p.x + m0 * p.ld_x + (uint64_t)first * (2 * BK);
    at_b += (uint64_t)first * (2 * BK);
    uint32_t to_come = steps, left = pairs - first * BK;
    const auto load_b = [&](uint32_t some, uint32_t stage_at) {
#pragma unroll
        for (int j = 0; j < StageB::LOADS; ++j) {
            const uint32_t r = (wave * StageB::LOADS + j) * 8;
            const bool second = PAIRED && r % (2 * HALF) >= HALF;
            const uint64_t address = reinterpret_cast<uint64_t>(at_b + (second ? up : 0));
            const i32x4 where = {(int)(uint32_t)address, (int)((uint32_t)(address >> 32) & 0xFFFF), 0x7FFFFFFF, 0x00020000};
            load_to_lds(sb.lds_at + stage_at + j * 1024, sb.k_of[j] < some ? sb.offset[j] : NOWHERE, where);
        }
    };
    const auto load = [&](uint32_t slot) { // past the end: zeros
        const uint32_t some = to_come ? left : 0;
        sa.load(reinterpret_cast<const bf16 *>(at_a), some, slot * STAGE);
        load_b(some, slot * STAGE);
    };
    const auto advance = [&]() {
        to_come = to_come ? to_come - 1 : 0;
        at_a += 2 * BK;
        at_b += 2 * BK;
        left -= BK;
    };

    i32x4 sum[S::TM][S::TN];
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) sum[i][j] = i32x4{0, 0, 0, 0};
    bf16x8 a[2][S::TM], b[2][S::TN];
    const auto read = [&](uint32_t slot, int to) {
        const uint32_t at = lds0 + slot * STAGE;
#pragma unroll
        for (int j = 0; j < S::TN; ++j) b[to][j] = StageB::read(at + StageA::BYTES, wn * S::TN + j, to);
#pragma unroll
        for (int i = 0; i < S::TM; ++i) a[to][i] = StageA::read(at, wm * S::TM + i, to);
    };
    const auto multiply = [&](int from) {
        // columns as the first operand: a lane's four sums are neighbouring columns of one row
#pragma unroll
        for (int i = 0; i < S::TM; ++i)
#pragma unroll
            for (int j = 0; j < S::TN; ++j)
                sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, b[from][j]), __builtin_bit_cast(i32x4, a[from][i]), sum[i][j],
                                                                  0, 0, 0);
        constexpr int READS = S::TM + S::TN, PRODUCTS = S::TM * S::TN, EACH = PRODUCTS / READS > 0 ? PRODUCTS / READS : 1;
#pragma unroll
        for (int r = 0; r < READS; ++r) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, EACH, 0);
        }
    };

    // One half of a step's k's is multiplied from registers while the next is read from the LDS and later steps are on their way.
#pragma unroll
    for (int s = 0; s < S::STAGES; ++s) {
        load(s);
        advance();
    }
    wait_and_meet<(S::STAGES - 1) * PER_STEP>();
    read(0, 0);
    uint32_t slot = 0;
    for (uint32_t i = 0; i < steps; ++i) {
        read(slot, 1);
        multiply(0);
        wait_and_meet<(S::STAGES - 2) * PER_STEP>();
        load(slot);
        slot = slot + 1 == S::STAGES ? 0 : slot + 1;
        read(slot, 0);
        multiply(1);
        advance();
    }
    wait_and_meet<0>(); // (loads past the end have to be done writing zeros to the LDS)

    // Sums to results by way of the LDS, so that memory sees whole rows of the tile
    constexpr int HIGH = S::TM < 2 ? 1 : 2, ROWS = S::WM * 16 * HIGH, PITCH = S::BN + 4;
    constexpr int CHUNKS = COLUMNS / 8, ITEMS = ROWS * CHUNKS / S::THREADS;
    static_assert(ROWS * PITCH * 4 <= S::LDS && ITEMS * S::THREADS == ROWS * CHUNKS, "the rows fit, and every thread has as many");
    const uint32_t mine = threadIdx.x / CHUNKS, chunk = threadIdx.x % CHUNKS, c = c0 + 8 * chunk;
    int *const rows = reinterpret_cast<int *>(lds);
    const auto row_of = [&](int step, int item) {
        const uint32_t r = mine + item * (S::THREADS / CHUNKS);
        return m0 + r / (16 * HIGH) * (16 * S::TM) + step * (16 * HIGH) + r % (16 * HIGH);
    };
    // all scales that a thread needs at once: one after the other, each waited for, they took 35 us at the end of a 256 x 256 tile
    Scales<GATE_> scales;
    float row_scale[S::TM / HIGH][ITEMS];
    if constexpr (!SHARED) {
        scales.load(p.to, c);
#pragma unroll
        for (int step = 0; step < S::TM / HIGH; ++step)
#pragma unroll
            for (int item = 0; item < ITEMS; ++item) row_scale[step][item] = row_of(step, item) < p.n ? p.to.x_scale[row_of(step, item)] : 0.0f;
    }
#pragma unroll
    for (int step = 0; step < S::TM / HIGH; ++step) {
        if (step > 0) lds_barrier();
#pragma unroll
        for (int i = 0; i < HIGH; ++i)
#pragma unroll
            for (int j = 0; j < S::TN; ++j)
                *reinterpret_cast<i32x4 *>(rows + ((wm * HIGH + i) * 16 + (lane & 15)) * PITCH + (wn * S::TN + j) * 16 + 4 * (lane >> 4)) =
                    sum[step * HIGH + i][j];
        lds_barrier();
#pragma unroll
        for (int item = 0; item < ITEMS; ++item) {
            const uint32_t m = row_of(step, item);
            if (m >= p.n || c >= N) continue;
            const int *row = rows + (mine + item * (S::THREADS / CHUNKS)) * PITCH;
            const uint32_t at = PAIRED ? 8 * chunk / HALF * (2 * HALF) + 8 * chunk % HALF : 8 * chunk;
            int v[8], u[8];
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                *reinterpret_cast<i32x4 *>(v + i) = *reinterpret_cast<const i32x4 *>(row + at + i);
                if (PAIRED) *reinterpret_cast<i32x4 *>(u + i) = *reinterpret_cast<const i32x4 *>(row + at + HALF + i);
            }
            if constexpr (SHARED) {
                int *to = p.partial + ((uint64_t)share * p.n + m) * p.columns;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i < N) to[c + i] = v[i];
            } else {
                finish<GATE_>(p.to, m, c, row_scale[step][item], scales, v, u);
            }
        }
    }
}

// shares of sums added up, eight columns a thread
template <bool GATE_>
__global__ __launch_bounds__(256) void join_kernel(const Int8Product p)
{
    const uint32_t chunks = (p.to.n_out + 7) / 8;
    const uint64_t total = (uint64_t)p.n * chunks;
    for (uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (uint64_t)gridDim.x * 256) {
        const uint64_t m = at / chunks;
        const uint32_t c = (uint32_t)(at % chunks) * 8;
        int v[8] = {0, 0, 0, 0, 0, 0, 0, 0}, u[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        for (uint32_t s = 0; s < p.shares; ++s) {
            const int *row = p.partial + ((uint64_t)s * p.n + m) * p.columns;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < p.to.n_out) {
                    v[i] += row[c + i];
                    if (GATE_) u[i] += row[p.to.n_out + c + i];
                }
        }
        Scales<GATE_> scales;
        scales.load(p.to, c);
        finish<GATE_>(p.to, m, c, p.to.x_scale[m], scales, v, u);
    }
}

// ------------------------------------------------------------------------------------------------ few rows

// Up to 16 * TILES rows: the weights are read once, straight into the matrix instructions' registers.  A block has sixteen columns (GATE:
// sixteen gates and their ups); its wavefronts take the k's in turn, 128 at a time, and add their sums up in the LDS.
template <int WAVES, int TILES, bool GATE_>
__global__ __launch_bounds__(64 * WAVES) void few_rows_kernel(const Int8Product p)
{
    constexpr int SIDES = GATE_ ? 2 : 1, AHEAD = TILES == 1 && !GATE_ ? 4 : 2; // steps on their way at a time
    __shared__ __attribute__((aligned(16))) int sums[WAVES][SIDES * TILES][16 * 16];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const uint32_t c0 = blockIdx.x * 16, whole = (p.n_in + 15) / 16 * 16;
    const bool column = c0 + r < p.to.n_out;
    const int8_t *w = p.w + (uint64_t)(column ? c0 + r : 0) * p.ld_w, *w_up = w + (GATE_ ? (uint64_t)p.to.n_out * p.ld_w : 0);
    const i32x4 none = {0, 0, 0, 0};
    i32x4 sum[SIDES][TILES];
#pragma unroll
    for (int s = 0; s < SIDES; ++s)
#pragma unroll
        for (int t = 0; t < TILES; ++t) sum[s][t] = none;
    for (uint32_t k0 = wave * 128; k0 < whole; k0 += WAVES * 128 * AHEAD) {
        i32x4 a[AHEAD][2][SIDES], b[AHEAD][2][TILES];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t k = k0 + s * WAVES * 128 + h * 64 + g * 16;
                const bool there = k < whole;
                a[s][h][0] = there && column ? *reinterpret_cast<const i32x4 *>(w + k) : none;
                if (GATE_) a[s][h][SIDES - 1] = there && column ? *reinterpret_cast<const i32x4 *>(w_up + k) : none;
#pragma unroll
                for (int t = 0; t < TILES; ++t)
                    b[s][h][t] = there && t * 16 + r < p.n ? *reinterpret_cast<const i32x4 *>(p.x + (uint64_t)(t * 16 + r) * p.ld_x + k) : none;
            }
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int side = 0; side < SIDES; ++side)
#pragma unroll
                    for (int t = 0; t < TILES; ++t) sum[side][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[s][h][side], b[s][h][t], sum[side][t], 0, 0, 0);
    }
    // a lane's four sums are columns 4 g .. 4 g + 3 of row r
#pragma unroll
    for (int side = 0; side < SIDES; ++side)
#pragma unroll
        for (int t = 0; t < TILES; ++t) *reinterpret_cast<i32x4 *>(&sums[wave][side * TILES + t][r * 16 + 4 * g]) = sum[side][t];
    __syncthreads();
    // two threads a row, eight columns each
    for (uint32_t at = threadIdx.x; at < TILES * 32; at += 64 * WAVES) {
        const uint32_t m = at / 2, c = at % 2 * 8, t = m / 16;
        if (m >= p.n || c0 + c >= p.to.n_out) continue;
        Scales<GATE_> scales;
        scales.load(p.to, c0 + c);
        int v[8] = {0, 0, 0, 0, 0, 0, 0, 0}, u[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int wv = 0; wv < WAVES; ++wv)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] += sums[wv][t][m % 16 * 16 + c + i];
                if (GATE_) u[i] += sums[wv][TILES + t][m % 16 * 16 + c + i];
            }
        finish<GATE_>(p.to, m, c0 + c, p.to.x_scale[m], scales, v, u);
    }
}

// ------------------------------------------------------------------------------------------------ short rows

// Rows of up to 64 * STEPS integers, many of them: what is written bounds it, and then the activations.  A wavefront keeps the weights and scales
// of 64 columns (GATE: and of their ups) in registers and goes over rows, sixteen at a time, with no LDS and no barrier.  Matrix rows are
// handed out so that a lane's sums of four matrix instructions make pieces of sixteen bytes of one row, which lie next to those of the other
// lanes: results are written from the registers.  2^18 rows of 64, 256 columns, 152 MB in three sets of buffers in turn: 44 us (3.4 TB/s);
// gated by ReLU 48, by SiLU 50, by GELU, whose erfc is a function's length, 105; of 128 integers by SiLU 75, of 256 101.  (The gated block of
// bf16 values that is one kernel does as many SiLUs and both products in 36, and writes a quarter of the bytes.)
template <class T, bool GATE_, int STEPS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(GATE_ && STEPS > 1 ? 2 : 3))) void short_rows_kernel(const Int8Product p, uint32_t groups)
{
    constexpr int SIDES = GATE_ ? 2 : 1;
    const uint32_t lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const uint32_t id = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), step = gridDim.x * 4 / groups;
    const uint32_t c0 = id % groups * 64, tiles = (p.n + 15) / 16, whole = (p.n_in + 15) / 16 * 16;
    uint32_t tile = id / groups;
    if (tile >= step) return; // (wavefronts that are left over)
    const i32x4 none = {0, 0, 0, 0};
    i32x4 w[SIDES][4][STEPS];
    float scale[SIDES][16];
    // the column of sum number i (of sixteen) of the lanes of a quarter of the wavefront
    constexpr int N = Chunk<T>::N;
    const auto column = [&](int i, uint32_t quarter) { return c0 + i / N * (4 * N) + N * quarter + i % N; };
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const uint32_t c = column(4 * t, r >> 2) + (r & 3);
#pragma unroll
        for (int side = 0; side < SIDES; ++side)
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const uint32_t k = s * 64 + g * 16;
                const int8_t *row = p.w + ((uint64_t)side * p.to.n_out + c) * p.ld_w;
                w[side][t][s] = c < p.to.n_out && k < whole ? *reinterpret_cast<const i32x4 *>(row + k) : none;
            }
    }
#pragma unroll
    for (int side = 0; side < SIDES; ++side)
#pragma unroll
        for (int i = 0; i < 16; ++i) scale[side][i] = column(i, g) < p.to.n_out ? p.to.w_scale[side * p.to.n_out + column(i, g)] : 0.0f;

    // Rows past the last are the last one again, k's past the end the first ones (times weights of 0): no load depends on a condition, and in
    // the loop over whole tiles no store does, so that the wait for the next rows need not be one for all stores before them
    // (2^18-64-256 gate, results past the last-level cache: 56 us with conditions, 50 without).  Stores that pass the caches take 39, but the
    // next operator's reads more than that: with quantise_rows behind it 92 us for 82
    i32x4 x[STEPS], next[STEPS];
    float row_scale, next_scale;
    const auto load = [&](uint32_t of, i32x4(&to)[STEPS], float &s_to) {
        const uint32_t m = min(of * 16 + r, p.n - 1);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const uint32_t k = s * 64 + g * 16;
            to[s] = *reinterpret_cast<const i32x4 *>(p.x + (uint64_t)m * p.ld_x + (k < whole ? k : 0));
        }
        s_to = p.to.x_scale[m];
    };
    const auto rows_of = [&](uint32_t of, auto all_there) {
        constexpr bool ALL = decltype(all_there)::value;
        load(min(of + step, tiles - 1), next, next_scale);
        i32x4 sum[SIDES][4];
#pragma unroll
        for (int side = 0; side < SIDES; ++side)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                sum[side][t] = none;
#pragma unroll
                for (int s = 0; s < STEPS; ++s) sum[side][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[side][t][s], x[s], sum[side][t], 0, 0, 0);
            }
        const uint64_t m = (uint64_t)of * 16 + r;
        float y[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = (float)sum[0][i / 4][i % 4] * row_scale * scale[0][i];
        if constexpr (GATE_) {
            with_act(p.to.act, [&](auto act) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    y[i] = gate_as<decltype(act)::value, sizeof(T) == 4>(y[i]).value * ((float)sum[1][i / 4][i % 4] * row_scale * scale[1][i]);
            });
        }
        T *row = (T *)p.to.y + m * p.to.ld_y;
#pragma unroll
        for (int i = 0; i < 16; i += N) {
            if constexpr (ALL) {
                Chunk<T> some;
#pragma unroll
                for (int j = 0; j < N; ++j) some.v[j] = (T)y[i + j];
                *reinterpret_cast<Chunk<T> *>(row + column(i, g)) = some;
            } else if (m < p.n && column(i, g) < p.to.n_out) {
                float some[N];
#pragma unroll
                for (int j = 0; j < N; ++j) some[j] = y[i + j];
                store_chunk(row, column(i, g), p.to.n_out, some);
            }
        }
#pragma unroll
        for (int s = 0; s < STEPS; ++s) x[s] = next[s];
        row_scale = next_scale;
    };
    load(tile, x, row_scale);
    if (c0 + 64 <= p.to.n_out)
        for (; tile < p.n / 16; tile += step) rows_of(tile, std::true_type{});
    for (; tile < tiles; tile += step) rows_of(tile, std::false_type{});
}

// ------------------------------------------------------------------------------------------------ host

struct Sizes {
    uint64_t n;
    uint32_t n_in, n_out;
    int32_t act;
    bool gate() const { return act != ECK_ACT_NONE; }
    uint64_t columns() const { return (uint64_t)n_out * (gate() ? 2 : 1); }
};

int32_t check_sizes(const Sizes &s)
{
    if (s.n == 0 || s.n_in == 0 || s.n_out == 0 || s.act < ECK_ACT_NONE || s.act > ECK_ACT_RELU) return ECK_EINVAL;
    if (s.n > MAX_ROWS || s.n_in > MOST_IN || s.n_out > MOST_OUT || (s.n + 63) / 64 * ((s.columns() + 63) / 64) > MOST_TILES) return ECK_EUNSUPPORTED;
    return ECK_OK;
}

typedef Shapes<1>::Small Small;
typedef Shapes<1>::Medium Medium;
typedef Shapes<1>::Large Large;

// How a product is cut up, by times in us that were fitted to some 80 measured ones (1 to 2^18 rows, 64 to 131071 integers a row, 16 to 16384
// columns; the choice is within a tenth of the best, but for the smallest, which all take 3 to 5): a tile alone on a compute unit (start, end
// and a step of 128 integers), tiles of a unit that is full, and what shares of k cost (a launch, sums written and read).  Up to 32 rows the
// weights' bytes count, and reading them straight into registers takes less than tiles do, until there are tiles for all units:
// 1 x 4096 x 4096 6.7 against 10.4 us, 1 x 4096 x 16384 15.3 against 12.6.
enum Int8Shape { TILES_64, TILES_128, TILES_256, FEW, SHORT };
struct Int8Plan {
    Int8Shape shape;
    uint32_t shares;
    double time;
};
constexpr uint64_t FEW_ROWS = 32;

Int8Plan plan(const Sizes &s)
{
    static const struct {
        uint64_t side;
        double rest, step, full_rest, full_step;
    } SHAPES[3] = {{64, 3.6, 0.2, 1.05, 0.165}, {128, 5.0, 0.57, 2.55, 0.5}, {256, 10.0, 1.1, 10.5, 1.6}};
    const double steps = (double)((s.n_in + 127) / 128), columns = (double)s.columns(), n = (double)s.n;
    Int8Plan best = {FEW, 1, 1e300};
    if (s.n <= FEW_ROWS) {
        const double chain = steps / (s.gate() ? 11.0 : 16.0), bytes = columns * s.n_in / 5.4e6;
        best.time = 3.0 + (chain > bytes ? chain : bytes);
    } else if (s.n_in <= 128 || (s.n_in <= 256 && n * columns >= 33554432.0)) {
        // (rows of 256, by tiles and this way: 2^18 rows of 256 columns 55 and 47 us, gated 101 and 78; 16384 of 2048 28.4 and 28.5, gated 52 and
        // 47; 4096 of 4096 16.0 and 19.6; 2048 of 2048 gated 9.9 and 22.9.  Of 128 and less this way is never the slower)
        return {SHORT, 1, 0.0};
    }
    for (int shape = 0; shape < 3; ++shape) {
        const auto &of = SHAPES[shape];
        const uint64_t tiles = (s.n + of.side - 1) / of.side * ((s.columns() + of.side - 1) / of.side);
        for (uint32_t shares = 1; shares <= (shape == TILES_64 ? 16u : 1u); shares *= 2) {
            if (shares > 1 && (steps / shares < 4.0 || tiles * shares > 512)) break;
            const double of_share = steps / shares, a_unit = (double)((tiles * shares + 255) / 256);
            const double alone = of.rest + of.step * of_share, full = a_unit * (of.full_rest + of.full_step * of_share);
            const double time = (alone > full ? alone : full) + (shares > 1 ? 5.0 + 0.75 * shares + shares * n * columns * 8.0 / 4.0e6 : 0.0);
            if (time < best.time) best = {(Int8Shape)shape, shares, time};
        }
    }
    return best;
}

template <class S>
int32_t launch_tiles(Int8Product p, bool gate, hipStream_t st)
{
    const bool shared = p.shares > 1;
    const uint32_t across = gate && !shared ? S::BN / 2 : S::BN, N = gate && !shared ? p.to.n_out : p.columns;
    p.tiles_m = (p.n + S::BM - 1) / S::BM;
    p.tiles_n = (N + across - 1) / across;
    const auto go = [&](auto kernel) -> int32_t {
        if (S::LDS > 65536)
            ECK_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS));
        hipLaunchKernelGGL(kernel, dim3(p.tiles_m * p.tiles_n * p.shares), dim3(S::THREADS), S::LDS, st, p);
        ECK_HIP_TRY(hipGetLastError());
        return ECK_OK;
    };
    if (!shared) return gate ? go(tiles_kernel<S, true, false>) : go(tiles_kernel<S, false, false>);
    if constexpr (S::BM > 64) return ECK_EUNSUPPORTED; // (shares are of small tiles alone)
    else if (const int32_t rc = go(tiles_kernel<S, false, true>)) return rc;
    const uint64_t chunks = (uint64_t)p.n * ((p.to.n_out + 7) / 8), blocks = (chunks + 255) / 256;
    hipLaunchKernelGGL((gate ? join_kernel<true> : join_kernel<false>), dim3((uint32_t)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st, p);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

template <int WAVES, int TILES>
int32_t launch_few(const Int8Product &p, bool gate, hipStream_t st)
{
    const dim3 grid((p.to.n_out + 15) / 16), block(64 * WAVES);
    hipLaunchKernelGGL((gate ? few_rows_kernel<WAVES, TILES, true> : few_rows_kernel<WAVES, TILES, false>), grid, block, 0, st, p);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

template <class T, bool GATE_, int STEPS>
int32_t launch_short(const Int8Product &p, hipStream_t st)
{
    // as many wavefronts as the units hold, but no more than there are rows for, and the same number for every group of columns
    const uint64_t groups = (p.to.n_out + 63) / 64, tiles = (p.n + 15) / 16;
    uint64_t rows = (256 * 12 + groups - 1) / groups;
    if (rows > tiles) rows = tiles;
    hipLaunchKernelGGL((short_rows_kernel<T, GATE_, STEPS>), dim3((uint32_t)((groups * rows + 3) / 4)), dim3(256), 0, st, p, (uint32_t)groups);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}
template <class T>
int32_t launch_short_of(const Int8Product &p, bool gate, hipStream_t st)
{
    if (p.n_in <= 64) return gate ? launch_short<T, true, 1>(p, st) : launch_short<T, false, 1>(p, st);
    if (p.n_in > 128) return gate ? launch_short<T, true, 4>(p, st) : launch_short<T, false, 4>(p, st);
    return gate ? launch_short<T, true, 2>(p, st) : launch_short<T, false, 2>(p, st);
}

} // namespace
} // namespace eck

using namespace eck;

extern "C" uint64_t product_int8_workspace_bytes(uint64_t n, uint32_t n_in, uint32_t n_out, int32_t act)
{
    const Sizes s = {n, n_in, n_out, act};
    if (check_sizes(s)) return 0;
    const Int8Plan how = plan(s);
    return how.shares > 1 ? how.shares * n * s.columns() * 4 : 0;
}

extern "C" int32_t product_int8(const int8_t *x, uint64_t ld_x, const float *x_scale, uint64_t n, uint32_t n_in, uint32_t n_out, const int8_t *w,
                                uint64_t ld_w, const float *w_scale, int32_t act, int32_t dtype, void *y, uint64_t ld_y, void *ws,
                                uint64_t ws_bytes, void *stream)
{
    const Sizes s = {n, n_in, n_out, act};
    if (!x || !x_scale || !w || !w_scale || !y || !is_dtype(dtype)) return ECK_EINVAL;
    const int32_t sizes = check_sizes(s);
    if (sizes == ECK_EINVAL) return sizes;
    if (ld_x < n_in || ld_w < n_in || ld_y < n_out) return ECK_ESHAPE;
    if (sizes) return sizes;
    if (ld_x > (1u << 22) || ld_w > (1u << 22)) return ECK_EUNSUPPORTED; // offsets within a tile are of 32 bits
    const uint64_t need = product_int8_workspace_bytes(n, n_in, n_out, act);
    if (need && (!ws || ws_bytes < need)) return ECK_EWORKSPACE;
    if (!aligned(x, 16) || !aligned(w, 16) || ld_x % 16 || ld_w % 16 || !aligned(x_scale, 4) || !aligned(w_scale, 4) ||
        !aligned(y, element_bytes(dtype)) || (need && !aligned(ws, 256)))
        return ECK_EALIGN;
    Int8Product p = {x, w, ld_x, ld_w, (uint32_t)n, n_in, 0, 0, 1, (int32_t *)ws, (uint32_t)s.columns(),
                     {x_scale, w_scale, y, ld_y, n_out, act, dtype == ECK_F32}};
    const hipStream_t st = as_stream(stream);
    const Int8Plan how = plan(s);
    p.shares = how.shares;
    if (how.shape == FEW) return n <= 16 ? launch_few<8, 1>(p, s.gate(), st) : launch_few<4, 2>(p, s.gate(), st);
    if (how.shape == SHORT) return p.to.f32 ? launch_short_of<float>(p, s.gate(), st) : launch_short_of<bf16>(p, s.gate(), st);
    if (how.shape == TILES_256) return launch_tiles<Large>(p, s.gate(), st);
    if (how.shape == TILES_128) return launch_tiles<Medium>(p, s.gate(), st);
    return launch_tiles<Small>(p, s.gate(), st);
}
