// Forward passes of gated feed-forward blocks that are not two products of matrices (HIP, gfx950): few rows, bound by the weights'
// bytes, and narrow blocks of many rows, whose hidden values never leave the registers.
#pragma once
#include "lanes.h"
#include "product.h"

namespace eck {
namespace product {

// ------------------------------------------------------------------------------------------------ few rows
//
// Rows times a matrix [K][N]: every weight is read once, so the time is its bytes at the memory's rate.  A block takes a cache line of
// columns, or one of gates and one of the ups of the same units, and a share of the k's: a compute unit alone draws no more than some
// 50 GB/s, so all of them have to.  Sixteen wavefronts with eight loads of sixteen bytes each on their way (four, beside the sums of
// four rows and more), the rows in the LDS.  The shares of (g | u) are joined by who reads them, as rows of the second product.  Sums in fp32
// instructions, whatever the type and the alignment, with no copies of the weights.

// values of a row in the LDS at a time
template <int ROWS>
constexpr int VECTOR_K = ROWS <= 4 ? 4096 : 16384 / ROWS;

struct Rows {
    const void *a;         // rows of T, or NULL: a(g) u from the shares of
    const float *sums;     // [shares][n][2 K] (g | u)
    uint64_t ld;           // of a
    float *pre;            // [n][2 K], receives (g | u), or NULL
    uint32_t n, K, shares; // shares: of the sums
    int32_t act;
};

// out: T, or sums [gridDim.y][n][columns]; block (column block, share)
template <class T, bool PAIRS, int ROWS>
__global__ __launch_bounds__(1024) void vector_kernel(const Rows rows, const T *w, uint64_t ld_w, uint32_t N, uint32_t up, T *out, uint64_t ld_out,
                                                      float *sums_out)
{
    constexpr int V = Chunk<T>::N, LINE = 8 * V, LANES = PAIRS ? 16 : 8, STEP = 64 / LANES, AHEAD = ROWS >= 4 ? 4 : 8, WAVES = 16;
    constexpr int MOST = VECTOR_K<ROWS>;
    extern __shared__ __attribute__((aligned(16))) float shared[]; // [k][ROWS], then the wavefronts' sums
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane % LANES, n = rows.n, K = rows.K;
    const uint32_t c0 = blockIdx.x * LINE, mine = c0 + j % 8 * V, here = mine < N ? (N - mine < V ? N - mine : V) : 0;
    const uint32_t begin = (uint32_t)((uint64_t)K * blockIdx.y / gridDim.y), end = (uint32_t)((uint64_t)K * (blockIdx.y + 1) / gridDim.y);
    const T *column = w + mine + (PAIRS && j >= 8 ? up : 0);
    float sum[ROWS][V];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) sum[r][i] = 0.0f;
    for (uint32_t k0 = begin; k0 < end; k0 += MOST) {
        const uint32_t some = end - k0 < MOST ? end - k0 : MOST;
        __syncthreads();
#pragma unroll 4
        for (uint32_t at = threadIdx.x; at < ROWS * some; at += 1024) { // (all rows at once: their loads wait together)
            const uint32_t r = at / some, k = at % some;
            float x = 0.0f;
            if (r < n && (PAIRS || rows.a)) x = (float)((const T *)rows.a)[r * rows.ld + k0 + k];
            else if (r < n) {
                float g = 0.0f, u = 0.0f;
#pragma unroll 4
                for (uint32_t s = 0; s < rows.shares; ++s) {
                    const float *row = rows.sums + ((uint64_t)s * n + r) * 2 * K + k0 + k;
                    g += row[0];
                    u += row[K];
                }
                if (rows.pre && blockIdx.x == 0) {
                    rows.pre[(uint64_t)r * 2 * K + k0 + k] = g;
                    rows.pre[(uint64_t)r * 2 * K + K + k0 + k] = u;
                }
                with_act(rows.act, [&](auto act) { x = (float)(T)(gate_as<decltype(act)::value, sizeof(T) == 4>(g).value * u); });
            }
            shared[k * ROWS + r] = x;
        }
        __syncthreads();
        for (uint32_t k = wave * STEP + lane / LANES; k < some; k += AHEAD * WAVES * STEP) {
            Chunk<T> some_w[AHEAD];
#pragma unroll
            for (int t = 0; t < AHEAD; ++t) {
                const uint32_t at = k + t * WAVES * STEP;
                some_w[t] = {};
                const T *from = column + (uint64_t)(k0 + at) * ld_w;
                if (at < some) {
                    if (here == V) some_w[t] = *reinterpret_cast<const Chunk<T> *>(from);
                    else
#pragma unroll
                        for (int i = 0; i < V; ++i)
                            if (i < (int)here) some_w[t].v[i] = from[i];
                }
            }
#pragma unroll
            for (int t = 0; t < AHEAD; ++t) {
                const uint32_t at = k + t * WAVES * STEP;
                if (at >= some) break;
                float x[ROWS];
                __builtin_memcpy(x, __builtin_assume_aligned(shared + at * ROWS, ROWS >= 4 ? 16 : ROWS * 4), sizeof x);
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll
                    for (int i = 0; i < V; ++i) sum[r][i] = fmaf(x[r], (float)some_w[t].v[i], sum[r][i]);
            }
        }
    }
    // Over the k's of a wavefront's lanes, then over the wavefronts.  Two halves of the lanes exchange two sums each, so that each half
    // goes on with one of them: after two rounds a quarter of the lanes has a quarter of the sums (and not four exchanges for every sum,
    // which took longer than the products of a small block).
    constexpr int COUNT = ROWS * V;
    float *const flat = &sum[0][0];
#pragma unroll
    for (int i = 0; i < COUNT / 2; ++i) {
        const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(flat[i]), __float_as_uint(flat[i + COUNT / 2]), false, false);
        flat[i] = __uint_as_float(two[0]) + __uint_as_float(two[1]);
    }
#pragma unroll
    for (int i = 0; i < COUNT / 4; ++i) {
        const auto two = __builtin_amdgcn_permlane16_swap(__float_as_uint(flat[i]), __float_as_uint(flat[i + COUNT / 4]), false, false);
        flat[i] = __uint_as_float(two[0]) + __uint_as_float(two[1]);
        if (LANES == 8) flat[i] += __uint_as_float(lane_exchange(__float_as_uint(flat[i]), 8));
    }
    __syncthreads();
    if ((lane & 15) < LANES)
#pragma unroll
        for (int i = 0; i < COUNT / 4; ++i) {
            const uint32_t which = i + (lane >> 5) * (COUNT / 2) + (lane >> 4 & 1) * (COUNT / 4); // row, column of this lane's V
            shared[(wave * ROWS + which / V) * (LANES * V) + j * V + which % V] = flat[i];
        }
    __syncthreads();
    constexpr int COLUMNS = LANES * V; // gates, then ups
    for (uint32_t at = threadIdx.x; at < ROWS * COLUMNS; at += 1024) {
        const uint32_t r = at / COLUMNS, c = at % COLUMNS, to = c0 + c % LINE;
        if (r >= n || to >= N) continue;
        float total = 0.0f;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) total += shared[(v * ROWS + r) * COLUMNS + c];
        if (PAIRS) sums_out[((uint64_t)blockIdx.y * n + r) * 2 * N + (c < LINE ? 0 : N) + to] = total;
        else if (gridDim.y > 1) sums_out[((uint64_t)blockIdx.y * n + r) * ld_out + to] = total;
        else out[r * ld_out + to] = (T)total;
    }
}

// ------------------------------------------------------------------------------------------------ narrow blocks
//
// y = (a(x Wg) * (x Wu)) Wd, 32 hidden units at a time: a wavefront keeps the operands of its 32 rows of x and their sums of y in
// registers; the sums of 32 gates and ups become, lane for lane, the operand of the second product (units 4g .. 4g + 3 and 16 + 4g ..
// of row r lie in lane (g, r), and the rows of Wd are read in that order).  The weights of the next units come into the LDS
// meanwhile.  Bound by the activations' exponentials and reciprocals, a quarter of the rate of other instructions each.

struct Narrow {
    Operand x, w_gate_up, w_down;
    uint32_t n, n_in, n_hidden, n_out, up;
    bf16 *y;
    uint64_t ld_y;
};

// DK: 32 k's of x; ON: 16 columns of y
template <int DK, int ON>
struct NarrowShape {
    static constexpr int WAVES = 4, ROWS = 32 * WAVES, SLOTS = 3;
    static constexpr int PIECES_GU = 4 * DK, PIECES = PIECES_GU + ON, LOADS = PIECES / WAVES; // of 1 KB
    static constexpr int STAGE = PIECES * 1024, LDS = STAGE * SLOTS;
    static_assert(PIECES % WAVES == 0, "every wavefront issues the same number of loads");
    static constexpr uint32_t UNITS = 64; // hidden units of a turn
};

// PADDED: n_hidden is no multiple of UNITS (a kernel of its own: the branch on it costs 64-256-64 of 16384 rows 8 %)
template <int DK, int ON, int ACT, bool PADDED>
__global__ __launch_bounds__(256) void narrow_kernel(const Narrow p)
{
    using S = NarrowShape<DK, ON>;
    typedef Stage<64, false, 4, 1> StageGU; // 32 gates and 32 ups a row of k
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15;
    // rows of Wd in the LDS: units of sixteen columns, unit j of hidden unit k in place j ^ down_swizzle(k): a read takes four
    // neighbouring k's of two groups of four per half wavefront
    constexpr uint32_t DOWN_CHUNKS = 2 * ON;
    const auto down_swizzle = [](uint32_t k) { return ON >= 8 ? k & 7 : k >> 1 & 3; };

    uint32_t offset[S::LOADS], unit[S::LOADS]; // bytes from the chunk's first value, or NOWHERE; first hidden unit
#pragma unroll
    for (int j = 0; j < S::LOADS; ++j) {
        const uint32_t piece = wave * S::LOADS + j;
        if (piece < S::PIECES_GU) {
            const uint32_t k = piece * 8 + lane / 8, c = ((lane & 7) ^ StageGU::unit_swizzle(k) << 1) * 8;
            unit[j] = c % 32;
            offset[j] = k < p.n_in ? (uint32_t)(k * p.w_gate_up.ld * 2) + (c % 32 + (c >= 32 ? p.up : 0)) * 2 : NOWHERE;
        } else {
            const uint32_t k = (piece - S::PIECES_GU) * (64 / DOWN_CHUNKS) + lane / DOWN_CHUNKS, c = ((lane % DOWN_CHUNKS) ^ down_swizzle(k) << 1) * 8;
            unit[j] = k;
            offset[j] = c < p.n_out ? (uint32_t)(k * p.w_down.ld * 2) + c * 2 : NOWHERE;
        }
    }
    const auto load = [&](uint32_t first, uint32_t slot) { // hidden units from `first` on; zeros past the last
        const uint32_t left = first < p.n_hidden ? p.n_hidden - first : 0;
        const uint64_t gu = reinterpret_cast<uint64_t>(p.w_gate_up.p + first), down = reinterpret_cast<uint64_t>(p.w_down.p + first * p.w_down.ld);
#pragma unroll
        for (int j = 0; j < S::LOADS; ++j) {
            const uint32_t piece = wave * S::LOADS + j;
            const uint64_t from = piece < S::PIECES_GU ? gu : down;
            const i32x4 where = {(int)(uint32_t)from, (int)((uint32_t)(from >> 32) & 0xFFFF), 0x7FFFFFFF, 0x00020000};
            load_to_lds(lds0 + slot * S::STAGE + piece * 1024, unit[j] < left ? offset[j] : NOWHERE, where);
        }
    };

    const uint32_t m0 = blockIdx.x * S::ROWS + wave * 32;
    bf16x8 x[2][DK];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t m = m0 + 16 * i + r;
        const bf16 *row = p.x.p + (uint64_t)(m < p.n ? m : p.n - 1) * p.x.ld;
#pragma unroll
        for (int k = 0; k < DK; ++k) {
            x[i][k] = {};
            if (32 * k + 8 * g < p.n_in) x[i][k] = *reinterpret_cast<const bf16x8 *>(row + 32 * k + 8 * g);
        }
    }
    f32x4 y[2][ON];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < ON; ++j) y[i][j] = f32x4{0, 0, 0, 0};

    const auto multiply_up = [&](uint32_t slot, f32x4(&to)[4][2]) {
        const uint32_t at = lds0 + slot * S::STAGE;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) to[t][i] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < DK; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const bf16x8 w = StageGU::read(at, t, k);
#pragma unroll
                for (int i = 0; i < 2; ++i) to[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x[i][k], to[t][i], 0, 0, 0);
            }
    };
    const auto multiply_down = [&](uint32_t slot, const bf16x8(&h)[2]) {
        typedef __attribute__((address_space(3))) s16x4 *Half;
        const uint32_t at = lds0 + slot * S::STAGE + S::PIECES_GU * 1024, k = 4 * g + (r >> 2); // and 16 more
#pragma unroll
        for (int j = 0; j < ON; ++j) {
            const uint32_t from = at + k * (ON * 32) + ((j ^ down_swizzle(k)) << 5) + ((r & 3) << 3);
            const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Half)(uintptr_t)from);
            const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Half)(uintptr_t)(from + 16 * ON * 32));
            const bf16x8 w = __builtin_bit_cast(bf16x8, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int i = 0; i < 2; ++i) y[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, h[i], y[i][j], 0, 0, 0);
        }
    };

    const auto activate = [&](uint32_t first, const f32x4(&pre)[4][2], bf16x8(&h)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) h[i][e] = (bf16)(gate_as<ACT, false>(pre[e / 4][i][e % 4]).value * pre[2 + e / 4][i][e % 4]);
        if (!PADDED || first + 32 <= p.n_hidden) return;
        // (units past the last, of zero weights, are NaN in rows with an infinity, and would be in y)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (first + 4 * g + e % 4 + (e < 4 ? 0 : 16) >= p.n_hidden) h[i][e] = (bf16)0.0f;
    };

    load(0, 0);
    load(32, 1);
    wait_and_meet<S::LOADS>();
    uint32_t slot = 0;
    // The next units' gates and ups are multiplied while the activations of these are worked out, then these units' share of y (2^18
    // rows, us so and one after the other: 128-512-128 115 and 128, 64-256-64 35.5 and 37.0, 128-512-256 237 and 272; 16384 rows of
    // 64-256-64 7.7 and 8.8).  At the meeting the next units have come, and everybody is through with the ones before these.
    f32x4 pre[2][4][2]; // gates 0 .. 15, 16 .. 31, ups
    multiply_up(0, pre[0]);
    for (uint32_t first = 0; first < p.n_hidden; first += S::UNITS) {
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) { // (units past the last: zeros)
            const uint32_t next = slot == 2 ? 0 : slot + 1;
            wait_and_meet<0>();
            load(first + 32 * odd + 64, next == 2 ? 0 : next + 1);
            multiply_up(next, pre[odd ^ 1]);
            bf16x8 h[2];
            activate(first + 32 * odd, pre[odd], h);
            multiply_down(slot, h);
            slot = next;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // (zeros for units past the last end before the block does)

    // lanes (q, r) hold columns 4q .. 4q + 3 of tiles side by side: after the exchange eight columns of one of them
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t m = m0 + 16 * i + r;
#pragma unroll
        for (int j = 0; j < ON; j += 2) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const auto two = __builtin_amdgcn_permlane16_swap(__float_as_uint(y[i][j][e]), __float_as_uint(y[i][j + 1][e]), false, false);
                v[e] = __uint_as_float(two[0]);
                v[4 + e] = __uint_as_float(two[1]);
            }
            const uint32_t c = 16 * (j + (g & 1)) + 8 * (g >> 1);
            if (m < p.n && c < p.n_out) store_eight(p.y + m * p.ld_y, c, p.n_out, v);
        }
    }
}

} // namespace product
} // namespace eck
