// Products of bfloat16 matrices on the matrix cores, and what a gated feed-forward block does with their sums (HIP, gfx950).
//
// C[m][c] = sum over k of A(m, k) B(k, c).  An operand's values lie next to each other along k (K_FAST) or along m or c; both are
// staged as they lie, 32 values of k at a time, by loads that go straight into the LDS, and become matrix-core operands on the
// way out of it (the second kind by the transposing LDS reads).  A block works on a tile of C, its wavefronts on parts of it.
//
// fp32 matrices come as three bfloat16 parts each (f32_split.h): of the nine products of parts the six largest are summed, one
// after the other in the same accumulators, the smallest first.
#pragma once
#include "activations.h"

namespace eck {
namespace product {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// a(g) and a'(g)
struct Gate {
    float value, slope;
};
__device__ __forceinline__ Gate gate_of(int32_t act, float g)
{
    if (act == ECK_ACT_RELU) return {g > 0.0f ? g : g == g ? 0.0f : g, g > 0.0f ? 1.0f : 0.0f};
    if (act == ECK_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-g));
        return {g * s, s * (1.0f + g * (1.0f - s))};
    }
    const float s = 0.5f * (1.0f + erff(g * 0.70710678f));
    return {g * s, s + g * 0.39894228f * expf(-0.5f * g * g)};
}

// An operand: 16-byte aligned, ld and the extent along its rows multiples of eight elements (zeros behind the matrix)
struct Operand {
    const bf16 *p;
    uint64_t ld, part; // elements between rows, and between the parts of an fp32 matrix
};

// What becomes of the sums
enum Kind {
    STORE,   // C
    PARTIAL, // fp32 sums of a share of the k's: [share][M][ld_out]
    GATE,    // columns are pairs (g, u): h = a(g) u, and (g, u) as they are where asked for
    SLOPE    // sums are dh: dg = dh u a'(g), du = dh a(g) and h = a(g) u from the stored (g, u)
};

// STORE takes columns [0, N) to out; where columns have a gap (the padding between gate and up) only those of the two pieces
// [0, piece) and [pitch, pitch + piece) exist, and lie next to each other in out.
struct Target {
    void *out;        // STORE: element type; PARTIAL: float; GATE, SLOPE: h, an operand of the next product
    uint64_t ld_out, part_out;
    uint32_t piece, pitch;
    float *pre;       // [M][2 * n_hidden] sums (g | u): GATE writes them (or NULL), SLOPE reads them
    bf16 *d_pre;      // SLOPE: (dg | du), an operand; du from column `pitch` on
    uint64_t ld_d, part_d;
    uint32_t n_hidden;
    int32_t act;
};

struct Product {
    Operand a, b;
    uint32_t M, N, K; // GATE: N = pairs
    uint32_t b_up;    // GATE: columns from a gate's to its up column in b
    uint32_t parts;   // 1, or 3: fp32 matrices
    uint32_t tiles_m, tiles_n, shares;
    Target to;
};

// ------------------------------------------------------------------------------------------------ results
// eight neighbouring columns of a row at a time

// value of eight columns as an operand of the next product: rounded to bfloat16, or in three parts
template <int PARTS>
__device__ __forceinline__ void store_operand(bf16 *p, uint64_t part, const float (&v)[8])
{
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = v[i];
#pragma unroll
    for (int s = 0; s < PARTS; ++s) {
        bf16x8 out;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            out[i] = (bf16)rest[i];
            rest[i] -= (float)out[i];
        }
        *reinterpret_cast<bf16x8 *>(p + s * part) = out;
    }
}

template <class T>
__device__ __forceinline__ void store_eight(T *row, uint32_t at, uint32_t width, const float (&v)[8])
{
    constexpr int N = Chunk<T>::N;
#pragma unroll
    for (int i = 0; i < 8; i += N) {
        float some[N];
#pragma unroll
        for (int j = 0; j < N; ++j) some[j] = v[i + j];
        if (at + i < width) store_chunk(row, at + i, width, some);
    }
}

__device__ __forceinline__ void load_eight(const float *row, uint32_t at, uint32_t width, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
        float some[4];
        load_chunk(row, at + i, width, some);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i + j] = some[j];
    }
}

template <int PARTS>
__device__ __forceinline__ void finish_store(const Target &to, uint64_t m, uint32_t c, const float (&v)[8])
{
    // (columns of the second piece start on a multiple of eight, as all chunks do)
    const uint32_t shift = c >= to.pitch ? to.pitch : 0, base = shift ? to.piece : 0;
    if (PARTS == 1) store_eight((bf16 *)to.out + m * to.ld_out + base, c - shift, to.piece, v);
    else store_eight((float *)to.out + m * to.ld_out + base, c - shift, to.piece, v);
}

template <int PARTS>
__device__ __forceinline__ void finish_gate(const Target &to, uint64_t m, uint32_t c, const float (&g)[8], const float (&u)[8])
{
    float h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = gate_of(to.act, g[i]).value * u[i];
    store_operand<PARTS>((bf16 *)to.out + m * to.ld_out + c, to.part_out, h);
    if (to.pre) {
        float *row = to.pre + m * 2 * to.n_hidden;
        store_eight(row, c, to.n_hidden, g);
        store_eight(row + to.n_hidden, c, to.n_hidden, u);
    }
}

template <int PARTS>
__device__ __forceinline__ void finish_slope(const Target &to, uint64_t m, uint32_t c, const float (&dh)[8])
{
    float g[8], u[8], h[8], dg[8], du[8];
    const float *row = to.pre + m * 2 * to.n_hidden;
    load_eight(row, c, to.n_hidden, g); // (zeros past the end: the padding of h, dg and du is zero)
    load_eight(row + to.n_hidden, c, to.n_hidden, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const Gate gate = gate_of(to.act, g[i]);
        h[i] = gate.value * u[i];
        dg[i] = dh[i] * u[i] * gate.slope;
        du[i] = dh[i] * gate.value;
    }
    if (to.out) store_operand<PARTS>((bf16 *)to.out + m * to.ld_out + c, to.part_out, h);
    bf16 *d = to.d_pre + m * to.ld_d + c;
    store_operand<PARTS>(d, to.part_d, dg);
    store_operand<PARTS>(d + to.pitch, to.part_d, du);
}

// ------------------------------------------------------------------------------------------------ staging

constexpr int BK = 32, STAGES = 4;
constexpr uint32_t NOWHERE = 0x80000000u; // an offset outside every buffer: such loads bring zeros

// 16 bytes per lane from base + offset into the LDS, lane after lane from lds_at (the same in all lanes)
__device__ __forceinline__ void load_to_lds(uint32_t lds_at, uint32_t offset, i32x4 base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_at), "v"(offset), "s"(base) : "memory", "m0");
}

// waits until all but N of this wavefront's loads are done and its LDS reads, then for the block
template <int N>
__device__ __forceinline__ void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// How 32 k's of ROWS rows (or columns) of an operand lie in the LDS.
//   K_FAST  rows of 64 bytes, four chunks of eight k's.  Sixteen lanes read the same chunk of sixteen neighbouring rows: chunk c of
//           row r is stored in place c ^ (r / 4 % 4), which spreads them over all banks.
//   else    32 rows of k, ROWS values each, in units of sixteen.  The transposing read takes units of eight k's at a time (k % 4 and
//           k / 8 % 2 vary within half a wavefront): unit j of k is stored in place j ^ those three bits (two where a row has just
//           four units and two rows share the banks).
template <int ROWS, bool K_FAST, int WAVES>
struct Stage {
    static constexpr int BYTES = ROWS * BK * 2, LOADS = BYTES / 1024 / WAVES;
    static_assert(BYTES % (1024 * WAVES) == 0, "every wavefront issues the same number of loads");
    static constexpr int CHUNKS = ROWS / 8; // of a k's row

    static __device__ __forceinline__ uint32_t unit_swizzle(uint32_t k)
    {
        return ROWS >= 128 ? (k & 3) | (k >> 3 & 1) << 2 : (k >> 1 & 1) | (k >> 3 & 1) << 1;
    }

    uint32_t offset[LOADS], k_of[LOADS]; // bytes from the tile's first value, or NOWHERE; first k
    i32x4 base;
    uint64_t step;                       // bytes from one stage to the next
    uint32_t lds_at;

    // place(r): for row r of the tile (K_FAST), or for the eight columns from r on, where in memory that is, in rows or columns from
    // the tile's first; NOWHERE if the operand has none
    template <class F>
    __device__ __forceinline__ void init(uint64_t ld, uint32_t lds, F &&place)
    {
        const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        lds_at = lds + wave * LOADS * 1024;
        step = K_FAST ? BK * 2 : BK * 2 * ld;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const uint32_t piece = wave * LOADS + j;
            if (K_FAST) {
                const uint32_t r = piece * 16 + lane / 4, chunk = (lane & 3) ^ (r >> 2 & 3);
                const uint32_t at = place(r);
                k_of[j] = chunk * 8;
                offset[j] = at != NOWHERE ? (uint32_t)(at * ld * 2) + chunk * 16 : NOWHERE;
            } else {
                const uint32_t k = piece * (64 / CHUNKS) + lane / CHUNKS, chunk = (lane % CHUNKS) ^ unit_swizzle(k) << 1;
                const uint32_t at = place(chunk * 8);
                k_of[j] = k;
                offset[j] = at != NOWHERE ? (uint32_t)(k * ld * 2) + at * 2 : NOWHERE;
            }
        }
    }
    // from: the tile's first value at this stage's first k, of whose k's `left` are there
    __device__ __forceinline__ void load(const bf16 *from, uint32_t left, uint32_t stage_at) const
    {
        const uint64_t address = reinterpret_cast<uint64_t>(from);
        const i32x4 where = {(int)(uint32_t)address, (int)((uint32_t)(address >> 32) & 0xFFFF), 0x7FFFFFFF, 0x00020000};
#pragma unroll
        for (int j = 0; j < LOADS; ++j) load_to_lds(lds_at + stage_at + j * 1024, k_of[j] < left ? offset[j] : NOWHERE, where);
    }

    // operands of rows [16 t, 16 t + 16): lane (g = lane / 16, r) holds k's 8g .. 8g + 7 of row r.  at: LDS address of the stage
    static __device__ __forceinline__ bf16x8 read(uint32_t at, uint32_t t)
    {
        typedef __attribute__((address_space(3))) const bf16x8 *Whole;
        typedef __attribute__((address_space(3))) s16x4 *Half;
        const uint32_t lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
        if (K_FAST) return *(Whole)(uintptr_t)(at + t * 1024 + r * 64 + ((g ^ (r >> 2 & 3)) << 4));
        // sixteen lanes: four k's, four values of sixteen columns each; lane r receives the four k's of column r
        const uint32_t k = 8 * g + (r >> 2);
        const uint32_t p = at + k * (ROWS * 2) + ((t ^ unit_swizzle(k)) << 5) + ((r & 3) << 3);
        const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Half)(uintptr_t)p);
        const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Half)(uintptr_t)(p + 4 * ROWS * 2));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// ------------------------------------------------------------------------------------------------ the kernel

// Tiles of BM x BN, wavefronts in WM rows and WN columns.
template <int BM_, int BN_, int WM_, int WN_>
struct Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int TM = BM / WM / 16, TN = BN / WN / 16; // 16 x 16 tiles of a wavefront
    static constexpr int LDS = (BM + BN) * BK * 2 * STAGES;
};
typedef Shape<256, 256, 2, 4> Large;
typedef Shape<128, 128, 2, 2> Medium;
typedef Shape<64, 64, 4, 1> Small;

template <class S, bool A_FAST, bool B_FAST, int KIND, int PARTS>
__global__ __launch_bounds__(S::THREADS, 2) void product_kernel(const Product p)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    typedef Stage<S::BM, A_FAST, S::WAVES> StageA;
    typedef Stage<S::BN, B_FAST, S::WAVES> StageB;
    constexpr int PER_STEP = StageA::LOADS + StageB::LOADS;
    constexpr uint32_t STAGE = (S::BM + S::BN) * BK * 2;
    constexpr int COLUMNS = KIND == GATE ? S::BN / 2 : S::BN; // of the result

    // Blocks go round the eight dies; the blocks of a die take neighbouring tiles, in panels eight tiles high, so that its L2
    // holds the rows and columns they share.
    const uint32_t total = gridDim.x, tiles = p.tiles_m * p.tiles_n, die = blockIdx.x & 7, left_over = total & 7;
    const uint32_t number = die * (total >> 3) + min(die, left_over) + (blockIdx.x >> 3);
    const uint32_t share = number / tiles, tile = number % tiles, panel = tile / (8 * p.tiles_n), in_panel = tile % (8 * p.tiles_n);
    const uint32_t high = min(8u, p.tiles_m - 8 * panel);
    const uint32_t m0 = (8 * panel + in_panel % high) * S::BM, c0 = in_panel / high * COLUMNS;

    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    StageA sa;
    StageB sb;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds;
    // a tile of pairs: of each wavefront's columns the first half are gates, the second the ups of the same units
    constexpr uint32_t HALF = S::BN / S::WN / 2;
    sa.init(p.a.ld, lds0, [&](uint32_t r) { return m0 + r < p.M ? r : NOWHERE; });
    sb.init(p.b.ld, lds0 + S::BM * BK * 2, [&](uint32_t c) {
        if (KIND != GATE) return c0 + c < p.N ? c : NOWHERE;
        const uint32_t unit = c / (2 * HALF) * HALF + c % HALF;
        return c0 + unit < p.N ? unit + (c % (2 * HALF) >= HALF ? p.b_up : 0) : NOWHERE;
    });
    // (the tile's own place is added to the base: offsets within a tile and a step fit 32 bits)
    const bf16 *a0 = p.a.p + (A_FAST ? m0 * p.a.ld : (uint64_t)m0), *b0 = p.b.p + (B_FAST ? c0 * p.b.ld : (uint64_t)c0);

    // steps of 32 k's: all of the first pair of parts, then the next; this block's share of them
    const uint32_t steps_k = (p.K + BK - 1) / BK, pairs = p.parts == 3 ? 6 : 1;
    const uint64_t all = (uint64_t)steps_k * pairs;
    const uint32_t first = (uint32_t)(all * share / p.shares), steps = (uint32_t)(all * (share + 1) / p.shares) - first;
    uint32_t next = first, next_pair = first / steps_k, next_k = first % steps_k; // to be loaded
    const auto load = [&](uint32_t slot) {
        // x0 w2, x2 w0, x1 w1, x0 w1, x1 w0, x0 w0
        const uint32_t pair = min(next_pair, 5u);
        const uint32_t part_a = p.parts == 3 ? 0x010120u >> 4 * pair & 15 : 0, part_b = p.parts == 3 ? 0x001102u >> 4 * pair & 15 : 0;
        const uint32_t k = next_k * BK, left = next < first + steps ? p.K - k : 0;
        sa.load(a0 + part_a * p.a.part + (A_FAST ? (uint64_t)k : k * p.a.ld), left, slot * STAGE);
        sb.load(b0 + part_b * p.b.part + (B_FAST ? (uint64_t)k : k * p.b.ld), left, slot * STAGE);
        ++next;
        if (++next_k == steps_k) {
            next_k = 0;
            ++next_pair;
        }
    };

    f32x4 sum[S::TM][S::TN];
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) sum[i][j] = f32x4{0, 0, 0, 0};
    bf16x8 a[2][S::TM], b[2][S::TN];
    const auto read = [&](uint32_t slot, bf16x8(&fa)[S::TM], bf16x8(&fb)[S::TN]) {
        const uint32_t at = lds0 + slot * STAGE;
#pragma unroll
        for (int j = 0; j < S::TN; ++j) fb[j] = StageB::read(at + S::BM * BK * 2, wn * S::TN + j);
#pragma unroll
        for (int i = 0; i < S::TM; ++i) fa[i] = StageA::read(at, wm * S::TM + i);
    };
    const auto multiply = [&](const bf16x8(&fa)[S::TM], const bf16x8(&fb)[S::TN]) {
        // columns as the first operand: a lane's four sums are neighbouring columns of one row
#pragma unroll
        for (int i = 0; i < S::TM; ++i)
#pragma unroll
            for (int j = 0; j < S::TN; ++j) sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], sum[i][j], 0, 0, 0);
    };

    // Step i is multiplied from registers while step i + 1 is read from the LDS and steps i + 2 to i + 4 are on their way; at the
    // meeting at its start everybody has read step i, so step i + 4 may take its place.  Steps past the end bring zeros.
#pragma unroll
    for (int s = 0; s < STAGES; ++s) load(s);
    wait_and_meet<(STAGES - 1) * PER_STEP>();
    read(0, a[0], b[0]);
    for (uint32_t i = 0; i < steps; i += 2) {
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) {
            const uint32_t slot = (i + odd) & (STAGES - 1);
            wait_and_meet<(STAGES - 2) * PER_STEP>();
            load(slot);
            read((slot + 1) & (STAGES - 1), a[odd ^ 1], b[odd ^ 1]);
            multiply(a[odd], b[odd]);
        }
    }
    // (loads past the end are still writing zeros to the LDS, which nobody reads any more; they end before the block does)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

    // sums of two tiles side by side, lanes (q = lane / 16): 4q .. 4q + 3 of each; after the exchange eight columns of one tile
    const auto eight = [&](const f32x4 &left, const f32x4 &right, float(&v)[8]) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const auto two = __builtin_amdgcn_permlane16_swap(__float_as_uint(left[r]), __float_as_uint(right[r]), false, false);
            v[r] = __uint_as_float(two[0]);
            v[4 + r] = __uint_as_float(two[1]);
        }
    };
    const uint32_t q = lane >> 4, within = 16 * (q & 1) + 8 * (q >> 1);
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
        const uint32_t m = m0 + (wm * S::TM + i) * 16 + (lane & 15);
        if (KIND == GATE) {
#pragma unroll
            for (int j = 0; j < S::TN / 2; j += 2) {
                float g[8], u[8];
                eight(sum[i][j], sum[i][j + 1], g);
                eight(sum[i][S::TN / 2 + j], sum[i][S::TN / 2 + j + 1], u);
                const uint32_t c = c0 + wn * HALF + j * 16 + within;
                if (m < p.M && c < p.N) finish_gate<PARTS>(p.to, m, c, g, u);
            }
        } else {
#pragma unroll
            for (int j = 0; j < S::TN; j += 2) {
                float v[8];
                eight(sum[i][j], sum[i][j + 1], v);
                const uint32_t c = c0 + (wn * S::TN + j) * 16 + within;
                if (m >= p.M || c >= p.N) continue;
                if (KIND == STORE) finish_store<PARTS>(p.to, m, c, v);
                if (KIND == SLOPE) finish_slope<PARTS>(p.to, m, c, v);
                if (KIND == PARTIAL) store_eight((float *)p.to.out + ((uint64_t)share * p.M + m) * p.to.ld_out, c, (uint32_t)p.to.ld_out, v);
            }
        }
    }
}

// The shares of a product whose k's were divided, added in order; then as above.  A thread has eight columns.
template <int KIND, int PARTS>
__global__ __launch_bounds__(256) void join_kernel(const float *partial, uint32_t shares, uint32_t M, uint32_t N, uint64_t ld, uint32_t up,
                                                   const Target to)
{
    const uint32_t chunks = (N + 7) / 8;
    for (uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x; at < (uint64_t)M * chunks; at += (uint64_t)gridDim.x * 256) {
        const uint32_t m = (uint32_t)(at / chunks), c = (uint32_t)(at % chunks) * 8;
        const auto total = [&](uint32_t column, float(&v)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
            for (uint32_t s = 0; s < shares; ++s) {
                float some[8];
                load_eight(partial + ((uint64_t)s * M + m) * ld, column, (uint32_t)ld, some);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += some[i];
            }
        };
        float v[8];
        total(c, v);
        if (KIND == STORE) finish_store<PARTS>(to, m, c, v);
        if (KIND == SLOPE) finish_slope<PARTS>(to, m, c, v);
        if (KIND == GATE) {
            float u[8];
            total(up + c, u);
            finish_gate<PARTS>(to, m, c, v, u);
        }
    }
}

// ------------------------------------------------------------------------------------------------ operands

// A matrix as operands want it: rows of two pieces of `piece` columns (one, if pieces is 1), each padded with zeros to `pitch`
// (a multiple of eight); fp32 ones in three parts.  A thread has eight columns.
template <class T>
__global__ __launch_bounds__(256) void pack_kernel(const T *src, uint64_t ld, uint32_t rows, uint32_t piece, uint32_t pieces, uint32_t pitch,
                                                   bf16 *dst, uint64_t part)
{
    const uint32_t chunks = pitch / 8 * pieces;
    for (uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x; at < (uint64_t)rows * chunks; at += (uint64_t)gridDim.x * 256) {
        const uint32_t r = (uint32_t)(at / chunks), c = (uint32_t)(at % chunks) * 8, shift = c >= pitch ? pitch : 0;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i += Chunk<T>::N) {
            float some[Chunk<T>::N];
            load_chunk(src + r * ld + (shift ? piece : 0), c - shift + i, piece, some);
#pragma unroll
            for (int j = 0; j < Chunk<T>::N; ++j) v[i + j] = some[j];
        }
        store_operand<sizeof(T) == 4 ? 3 : 1>(dst + (uint64_t)r * pitch * pieces + c, part, v);
    }
}

} // namespace product
} // namespace eck
