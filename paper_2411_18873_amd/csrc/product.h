// Products of bfloat16 matrices on the matrix cores, and what a gated feed-forward block does with their sums (HIP, gfx950).
//
// C[m][c] = sum over k of A(m, k) B(k, c).  An operand's values lie next to each other along k (K_FAST) or along m or c; both are
// staged as they lie, 64 values of k at a time, by loads that go straight into the LDS, and become matrix-core operands on the
// way out of it (the second kind by the transposing LDS reads).  A block works on a tile of C, its wavefronts on parts of it.
//
// fp32 matrices come as three bfloat16 parts each (f32_split.h): of the nine products of parts the six largest are summed, the
// smallest first.  The parts of 32 neighbouring values of a row lie next to each other, so that one stage brings all of them and a
// part that enters several products is loaded once.
#pragma once
#include "activations.h"

#include <type_traits>

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
// WHOLE: of fp32 blocks, to the last bits of fp32
template <int ACT, bool WHOLE>
__device__ __forceinline__ Gate gate_as(float g)
{
    if (ACT == ECK_ACT_RELU) return {g > 0.0f ? g : g == g ? 0.0f : g, g > 0.0f ? 1.0f : 0.0f};
    if (ACT == ECK_ACT_SILU) {
        // (bf16: exponential and reciprocal as the instructions give them, within a unit of the last place each; rounding the
        // exponential's argument adds about |g| 2^-24 of the value, ten units at g = -20, all far below a bf16's.  Full ones are 25 more
        // instructions an element, which narrow blocks would wait for.)
        const float s = WHOLE ? 1.0f / (1.0f + expf(-g)) : __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f));
        return {g * s, s * (1.0f + g * (1.0f - s))};
    }
    // (1 + erf cancels far out on the left: at g = -5 a tenth of the value was lost, at -6 all)
    const float s = 0.5f * erfcf(g * -0.70710678f);
    return {g * s, s + g * 0.39894228f * expf(-0.5f * g * g)};
}
// calls f with the activation as a constant, once for all elements it works on
template <class F>
__device__ __forceinline__ void with_act(int32_t act, F &&f)
{
    if (act == ECK_ACT_SILU) f(std::integral_constant<int, ECK_ACT_SILU>{});
    else if (act == ECK_ACT_GELU) f(std::integral_constant<int, ECK_ACT_GELU>{});
    else f(std::integral_constant<int, ECK_ACT_RELU>{});
}

// An operand: 16-byte aligned, rows of a multiple of eight elements (zeros behind the matrix), or, in parts, of 32, the three parts of
// each 32 one after the other
struct Operand {
    const bf16 *p;
    uint64_t ld; // elements between rows, those of all parts
};
// where in a row column c's first part is, c a multiple of eight, and from one part to the next
template <int PARTS>
__host__ __device__ __forceinline__ uint32_t in_row(uint32_t c) { return PARTS == 1 ? c : c / 32 * 96 + c % 32; }
constexpr uint32_t PART = 32;

// What becomes of the sums
enum Kind {
    STORE, // C, or, where the k's are in several shares, fp32 sums of each: [share][M][ld_out]
    GATE,  // columns are pairs (g, u): h = a(g) u, and (g, u) as they are where asked for
    SLOPE  // sums are dh: dg = dh u a'(g), du = dh a(g) and h = a(g) u from the stored (g, u)
};

// STORE takes columns [0, N) to out; where columns have a gap (the padding between gate and up) only those of the two pieces
// [0, piece) and [pitch, pitch + piece) exist, and lie next to each other in out.
struct Target {
    void *out;        // STORE: element type, or float for shares; GATE, SLOPE: h, an operand of the next product
    uint64_t ld_out;
    uint32_t piece, pitch;
    float *pre;       // [M][2 * n_hidden] sums (g | u): GATE writes them (or NULL), SLOPE reads them
    bf16 *d_pre;      // SLOPE: (dg | du), an operand; du from column `pitch` on
    uint64_t ld_d;
    uint32_t n_hidden;
    int32_t act;
};

struct Product {
    Operand a, b;
    uint32_t M, N, K; // GATE: N = pairs
    uint32_t b_up;    // GATE: columns from a gate's to its up column in b
    uint32_t tiles_m, tiles_n, shares;
    Target to;
    __host__ __device__ uint32_t blocks() const { return tiles_m * tiles_n * shares; }
};

// ------------------------------------------------------------------------------------------------ results
// eight neighbouring columns of a row at a time

// value of eight columns as an operand of the next product: rounded to bfloat16, or in three parts
template <int PARTS>
__device__ __forceinline__ void store_operand(bf16 *row, uint32_t c, const float (&v)[8])
{
    bf16 *p = row + in_row<PARTS>(c);
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
        *reinterpret_cast<bf16x8 *>(p + s * PART) = out;
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
        float some[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (at + i + 4 <= width) {
            // read once, and not to push the operands out of the L2 (8192 x 8192 derivatives: 750 us without the hint, 635 with)
            const auto c = __builtin_nontemporal_load(reinterpret_cast<const Chunk<float>::Vector *>(row + at + i));
#pragma unroll
            for (int j = 0; j < 4; ++j) some[j] = c[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (at + i + j < width) some[j] = row[at + i + j];
        }
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

// Zeros for the columns that operands are padded with.  The products leave NaN there in rows with an infinity (times the other
// operand's padding), and it would go from there into the row's results.
__device__ __forceinline__ void clear_padding(uint32_t c, uint32_t width, float (&v)[8])
{
    if (c + 8 <= width) return;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i >= width) v[i] = 0.0f;
}

template <int PARTS>
__device__ __forceinline__ void finish_gate(const Target &to, uint64_t m, uint32_t c, const float (&g)[8], const float (&u)[8])
{
    float h[8];
    with_act(to.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = gate_as<decltype(act)::value, PARTS == 3>(g[i]).value * u[i];
    });
    clear_padding(c, to.n_hidden, h);
    store_operand<PARTS>((bf16 *)to.out + m * to.ld_out, c, h);
    if (to.pre) {
        float *row = to.pre + m * 2 * to.n_hidden;
        store_eight(row, c, to.n_hidden, g);
        store_eight(row + to.n_hidden, c, to.n_hidden, u);
    }
}

// what eight columns of dh are multiplied with (zeros past the end)
struct Pre {
    float g[8], u[8];
};
__device__ __forceinline__ void load_pre(const Target &to, uint64_t m, uint32_t c, Pre &pre)
{
    const float *row = to.pre + m * 2 * to.n_hidden;
    load_eight(row, c, to.n_hidden, pre.g);
    load_eight(row + to.n_hidden, c, to.n_hidden, pre.u);
}

template <int PARTS>
__device__ __forceinline__ void finish_slope(const Target &to, uint64_t m, uint32_t c, const float (&dh)[8], const Pre &pre)
{
    float h[8], dg[8], du[8];
    with_act(to.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Gate gate = gate_as<decltype(act)::value, PARTS == 3>(pre.g[i]);
            h[i] = gate.value * pre.u[i];
            dg[i] = dh[i] * pre.u[i] * gate.slope;
            du[i] = dh[i] * gate.value;
        }
    });
    clear_padding(c, to.n_hidden, dg);
    clear_padding(c, to.n_hidden, du);
    if (to.out) store_operand<PARTS>((bf16 *)to.out + m * to.ld_out, c, h);
    bf16 *d = to.d_pre + m * to.ld_d;
    store_operand<PARTS>(d, c, dg);
    store_operand<PARTS>(d, to.pitch + c, du);
}

// ------------------------------------------------------------------------------------------------ staging

// k's of a stage: 64, or 32 in three parts
template <int PARTS>
constexpr int STAGE_K = PARTS == 1 ? 64 : 32;
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

// How a stage of ROWS rows (or columns) of an operand lies in the LDS, each part by itself.
//   K_FAST  rows of 128 bytes (so every load takes whole cache lines: of 32 k's at a time the L1 asked the L2 for each line twice,
//           1.33e8 requests for 6.7e7 in a product of 8192^3), eight chunks of eight k's; chunk c of row r is stored in place
//           c ^ (r / 2 % 8).  In parts, rows of 64 bytes, four chunks, in place c ^ (0, 2, 3, 1)[r / 4 % 4].  A read of sixteen rows
//           takes four cycles if the lanes served in one (rows 0 .. 3 and 12 .. 15 of one chunk with 4 .. 11 of the next, or the other
//           way round) take from all banks: so found from the bank conflicts counted.
//   else    rows of k, ROWS values each, in units of sixteen.  The transposing read takes units of eight k's at a time (k % 4 and
//           k / 8 % 2 vary within half a wavefront): unit j of k is stored in place j ^ those three bits (two where a row has just
//           four units and two rows share the banks).
template <int ROWS, bool K_FAST, int WAVES, int PARTS>
struct Stage {
    static constexpr int BK = STAGE_K<PARTS>, ONE = ROWS * BK * 2, BYTES = ONE * PARTS, LOADS = BYTES / 1024 / WAVES; // ONE: a part
    static_assert(BYTES % (1024 * WAVES) == 0, "every wavefront issues the same number of loads");
    static constexpr int CHUNKS = ROWS / 8;   // of a k's row
    static constexpr int SPAN = BK / 8;       // chunks of a row of k's

    static __device__ __forceinline__ uint32_t row_swizzle(uint32_t r) { return PARTS == 1 ? r >> 1 & 7 : (r >> 2 & 1) << 1 ^ (r >> 3 & 1) * 3; }
    static __device__ __forceinline__ uint32_t unit_swizzle(uint32_t k)
    {
        return ROWS >= 128 ? (k & 3) | (k >> 3 & 1) << 2 : (k >> 1 & 1) | (k >> 3 & 1) << 1;
    }

    uint32_t offset[LOADS], k_of[LOADS]; // bytes from the tile's first value, or NOWHERE; first k
    uint32_t lds_at;

    // place(r): for row r of the tile (K_FAST), or for the eight columns from r on, where in memory that is, in rows or columns from
    // the tile's first; NOWHERE if the operand has none
    template <class F>
    __device__ __forceinline__ void init(uint64_t ld, uint32_t lds, F &&place)
    {
        const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        lds_at = lds + wave * LOADS * 1024;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const uint32_t piece = (wave * LOADS + j) % (ONE / 1024), part = (wave * LOADS + j) / (ONE / 1024);
            if (K_FAST) {
                const uint32_t r = piece * (64 / SPAN) + lane / SPAN, chunk = (lane % SPAN) ^ row_swizzle(r);
                const uint32_t at = place(r);
                k_of[j] = chunk * 8;
                offset[j] = at != NOWHERE ? (uint32_t)(at * ld * 2) + (part * PART + chunk * 8) * 2 : NOWHERE;
            } else {
                const uint32_t k = piece * (64 / CHUNKS) + lane / CHUNKS, chunk = (lane % CHUNKS) ^ unit_swizzle(k) << 1;
                const uint32_t at = place(chunk * 8);
                k_of[j] = k;
                offset[j] = at != NOWHERE ? (uint32_t)(k * ld * 2) + (in_row<PARTS>(at) + part * PART) * 2 : NOWHERE;
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

    // operands of rows [16 t, 16 t + 16): lane (g = lane / 16, r) holds 32 which + 8g .. 8g + 7 of row r's k's (in parts: 8g .. 8g + 7 of
    // part `which`).  at: LDS address of the stage
    static __device__ __forceinline__ bf16x8 read(uint32_t at, uint32_t t, uint32_t which)
    {
        typedef __attribute__((address_space(3))) const bf16x8 *Whole;
        typedef __attribute__((address_space(3))) s16x4 *Half;
        const uint32_t lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15, half = PARTS == 1 ? which : 0;
        if (PARTS > 1) at += which * ONE;
        if (K_FAST) return *(Whole)(uintptr_t)(at + (t * 16 + r) * (BK * 2) + ((half * 4 + g ^ row_swizzle(r)) << 4));
        // sixteen lanes: four k's, four values of sixteen columns each; lane r receives the four k's of column r
        const uint32_t k = 32 * half + 8 * g + (r >> 2);
        const uint32_t p = at + k * (ROWS * 2) + ((t ^ unit_swizzle(k)) << 5) + ((r & 3) << 3);
        const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Half)(uintptr_t)p);
        const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Half)(uintptr_t)(p + 4 * ROWS * 2));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// ------------------------------------------------------------------------------------------------ the kernel

// Tiles of BM x BN, wavefronts in WM rows and WN columns, STAGES in the LDS.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_, int PARTS_>
struct Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, WAVES = WM * WN, THREADS = 64 * WAVES, STAGES = STAGES_, PARTS = PARTS_;
    static constexpr int BK = STAGE_K<PARTS>, TM = BM / WM / 16, TN = BN / WN / 16; // 16 x 16 tiles of a wavefront
    static constexpr int STAGE = (BM + BN) * BK * 2 * PARTS, LDS = STAGE * STAGES;
    static constexpr int AT_ONCE = 160 * 1024 / LDS * WAVES / 4; // wavefronts a SIMD: the registers may be used up to that
};
// by type: small, medium and large ones (in parts, a large tile's stages do not fit the LDS)
template <int PARTS>
struct Shapes {
    static constexpr int COUNT = 3;
    typedef Shape<64, 64, 4, 1, 3, 1> Small;
    typedef Shape<128, 128, 2, 2, 2, 1> Medium;
    typedef Shape<256, 256, 2, 4, 2, 1> Large;
};
template <>
struct Shapes<3> {
    static constexpr int COUNT = 2;
    typedef Shape<64, 64, 4, 1, 3, 3> Small;
    typedef Shape<128, 128, 2, 4, 3, 3> Medium;
};

template <class S, bool A_FAST, bool B_FAST, int KIND>
__device__ __forceinline__ void work(const Product &p, uint32_t block, uint32_t total, unsigned char *lds)
{
    constexpr int PARTS = S::PARTS, BK = S::BK;
    typedef Stage<S::BM, A_FAST, S::WAVES, PARTS> StageA;
    typedef Stage<S::BN, B_FAST, S::WAVES, PARTS> StageB;
    constexpr int PER_STEP = StageA::LOADS + StageB::LOADS;
    constexpr uint32_t STAGE = S::STAGE;
    constexpr int COLUMNS = KIND == GATE ? S::BN / 2 : S::BN; // of the result

    // Blocks go round the eight dies; the blocks of a die take neighbouring tiles, in panels eight tiles high, so that its L2
    // holds the rows and columns they share.
    const uint32_t tiles = p.tiles_m * p.tiles_n, die = block & 7, left_over = total & 7;
    const uint32_t number = die * (total >> 3) + min(die, left_over) + (block >> 3);
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
    sb.init(p.b.ld, lds0 + StageA::BYTES, [&](uint32_t c) {
        if (KIND != GATE) return c0 + c < p.N ? c : NOWHERE;
        const uint32_t unit = c / (2 * HALF) * HALF + c % HALF;
        return c0 + unit < p.N ? unit + (c % (2 * HALF) >= HALF ? p.b_up : 0) : NOWHERE;
    });
    // steps of BK k's; this block's share of them.  (The tile's own place is added to the base: offsets within a tile and a step fit
    // 32 bits.)
    const uint32_t all = (p.K + BK - 1) / BK;
    const uint32_t first = (uint32_t)((uint64_t)all * share / p.shares), steps = (uint32_t)((uint64_t)all * (share + 1) / p.shares) - first;
    const uint64_t step_a = A_FAST ? in_row<PARTS>(BK) : BK * p.a.ld, step_b = B_FAST ? in_row<PARTS>(BK) : BK * p.b.ld;
    const bf16 *at_a = p.a.p + (A_FAST ? m0 * p.a.ld : (uint64_t)in_row<PARTS>(m0)) + first * step_a;
    const bf16 *at_b = p.b.p + (B_FAST ? c0 * p.b.ld : (uint64_t)in_row<PARTS>(c0)) + first * step_b;
    uint32_t to_come = steps, left = p.K - first * BK; // steps not yet on their way, k's from the next one on
    const auto load = [&](uint32_t slot) {             // past the end: zeros
        const uint32_t some = to_come ? left : 0;
        sa.load(at_a, some, slot * STAGE);
        sb.load(at_b, some, slot * STAGE);
    };
    const auto advance = [&]() {
        to_come = to_come ? to_come - 1 : 0;
        at_a += step_a;
        at_b += step_b;
        left -= BK; // (past the last one nothing is to come)
    };

    // the results: some rows of tiles at a time, threads with eight columns each
    constexpr int HIGH = S::TM < 2 ? 1 : 2, ROWS = S::WM * 16 * HIGH, PITCH = S::BN + 4; // four words: sixteen rows, all banks
    constexpr int CHUNKS = COLUMNS / 8, ITEMS = ROWS * CHUNKS / S::THREADS;
    static_assert(ROWS * PITCH * 4 <= S::LDS && ITEMS * S::THREADS == ROWS * CHUNKS, "the rows fit, and every thread has as many");
    const uint32_t mine = threadIdx.x / CHUNKS, chunk = threadIdx.x % CHUNKS, c = c0 + 8 * chunk;
    const auto row_of = [&](int step, int item) {
        const uint32_t r = mine + item * (S::THREADS / CHUNKS);
        return m0 + r / (16 * HIGH) * (16 * S::TM) + step * (16 * HIGH) + r % (16 * HIGH);
    };
    const uint32_t last = KIND == SLOPE ? p.to.pitch : p.N; // (derivatives: zeros up to the operand's next piece, whose k's follow)
    constexpr bool EARLY = KIND == SLOPE && S::TM == 1; // the stored sums that a small tile needs are fetched before anything else
    Pre early[EARLY ? ITEMS : 1];
    if constexpr (EARLY)
#pragma unroll
        for (int item = 0; item < ITEMS; ++item)
            if (row_of(0, item) < p.M && c < last) load_pre(p.to, row_of(0, item), c, early[item]);

    f32x4 sum[S::TM][S::TN];
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) sum[i][j] = f32x4{0, 0, 0, 0};
    // operands: of the two halves of a step's k's, or of all parts of two steps
    bf16x8 a[2][S::TM][PARTS], b[2][S::TN][PARTS];
    const auto read = [&](uint32_t slot, int to) {
        const uint32_t at = lds0 + slot * STAGE;
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
            const uint32_t which = PARTS == 1 ? to : part;
#pragma unroll
            for (int j = 0; j < S::TN; ++j) b[to][j][part] = StageB::read(at + StageA::BYTES, wn * S::TN + j, which);
#pragma unroll
            for (int i = 0; i < S::TM; ++i) a[to][i][part] = StageA::read(at, wm * S::TM + i, which);
        }
    };
    const auto multiply = [&](int from) {
        // columns as the first operand: a lane's four sums are neighbouring columns of one row
        constexpr int PAIRS = PARTS == 1 ? 1 : 6;
        constexpr int PART_A[6] = {0, 2 % PARTS, 1 % PARTS, 0, 1 % PARTS, 0}, PART_B[6] = {2 % PARTS, 0, 1 % PARTS, 1 % PARTS, 0, 0};
#pragma unroll
        for (int pair = 0; pair < PAIRS; ++pair)
#pragma unroll
            for (int i = 0; i < S::TM; ++i)
#pragma unroll
                for (int j = 0; j < S::TN; ++j)
                    sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[from][j][PART_B[pair]], a[from][i][PART_A[pair]], sum[i][j], 0, 0, 0);
        // an LDS read (of what comes next), a few products, and so on: left to itself the compiler reads every operand right before
        // its use
        constexpr int READS = PARTS * (S::TM * (A_FAST ? 1 : 2) + S::TN * (B_FAST ? 1 : 2)), PRODUCTS = PAIRS * S::TM * S::TN;
        constexpr int EACH = PRODUCTS / READS > 0 ? PRODUCTS / READS : 1;
#pragma unroll
        for (int r = 0; r < READS; ++r) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, EACH, 0);
        }
    };

    // One half of a step's k's (or, in parts, one step) is multiplied from registers while the next is read from the LDS and later
    // steps are on their way.  At a meeting everybody has read all of a step, so that its place is free, and the next step has come.
    // Steps past the end bring zeros.
#pragma unroll
    for (int s = 0; s < S::STAGES; ++s) {
        load(s);
        advance();
    }
    wait_and_meet<(S::STAGES - 1) * PER_STEP>();
    read(0, 0);
    uint32_t slot = 0;
    const auto meet = [&]() {
        wait_and_meet<(S::STAGES - 2) * PER_STEP>();
        load(slot);
        slot = slot + 1 == S::STAGES ? 0 : slot + 1;
    };
    if constexpr (PARTS == 1) {
        for (uint32_t i = 0; i < steps; ++i) {
            read(slot, 1);
            multiply(0);
            meet();
            read(slot, 0);
            multiply(1);
            advance();
        }
    } else {
        for (uint32_t i = 0; i < steps; i += 2) {
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
                meet();
                read(slot, odd ^ 1);
                multiply(odd);
                advance();
            }
        }
    }
    // Sums to results by way of the LDS, some rows of tiles at a time, so that threads next to each other work on columns next to
    // each other and memory sees whole rows of the tile (straight from the registers, in pieces of 64 bytes, 8192 x 8192 gates took
    // 1020 us for 980).
    float *const rows = reinterpret_cast<float *>(lds);
    // (loads past the end have to be done writing zeros to the LDS)
    wait_and_meet<0>();
#pragma unroll
    for (int step = 0; step < S::TM / HIGH; ++step) {
        Pre pre[ITEMS];
        if constexpr (KIND == SLOPE && !EARLY) // on their way while the sums are exchanged
#pragma unroll
            for (int item = 0; item < ITEMS; ++item)
                if (row_of(step, item) < p.M && c < last) load_pre(p.to, row_of(step, item), c, pre[item]);
        if (step > 0) lds_barrier();
#pragma unroll
        for (int i = 0; i < HIGH; ++i)
#pragma unroll
            for (int j = 0; j < S::TN; ++j)
                *reinterpret_cast<f32x4 *>(rows + ((wm * HIGH + i) * 16 + (lane & 15)) * PITCH + (wn * S::TN + j) * 16 + 4 * (lane >> 4)) =
                    sum[step * HIGH + i][j];
        lds_barrier();
#pragma unroll
        for (int item = 0; item < ITEMS; ++item) {
            const uint32_t m = row_of(step, item);
            const float *row = rows + (mine + item * (S::THREADS / CHUNKS)) * PITCH;
            if (m >= p.M || c >= last) continue;
            // (of a wavefront's columns the first half are gates, the second the ups of the same units)
            const uint32_t at = KIND == GATE ? 8 * chunk / HALF * (2 * HALF) + 8 * chunk % HALF : 8 * chunk;
            float v[8], u[8];
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                *reinterpret_cast<f32x4 *>(v + i) = *reinterpret_cast<const f32x4 *>(row + at + i);
                if (KIND == GATE) *reinterpret_cast<f32x4 *>(u + i) = *reinterpret_cast<const f32x4 *>(row + at + HALF + i);
            }
            if constexpr (KIND == STORE) {
                if (p.shares == 1) finish_store<PARTS>(p.to, m, c, v);
                else store_eight((float *)p.to.out + ((uint64_t)share * p.M + m) * p.to.ld_out, c, (uint32_t)p.to.ld_out, v);
            }
            if constexpr (KIND == GATE) finish_gate<PARTS>(p.to, m, c, v, u);
            if constexpr (KIND == SLOPE) finish_slope<PARTS>(p.to, m, c, v, EARLY ? early[item] : pre[item]);
        }
    }
}

template <class S, bool A_FAST, bool B_FAST, int KIND>
__global__ __launch_bounds__(S::THREADS) __attribute__((amdgpu_waves_per_eu(S::AT_ONCE, S::AT_ONCE))) void product_kernel(const Product p)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    work<S, A_FAST, B_FAST, KIND>(p, blockIdx.x, gridDim.x, lds);
}

// The three gradients, which wait for nothing but dg, du and h, in one launch: dx, of operands along k, then the weights', of
// operands along rows and columns.  A product of no blocks is left out.
struct Gradients {
    Product dx, dw_gate_up, dw_down;
};
template <class S>
__global__ __launch_bounds__(S::THREADS) __attribute__((amdgpu_waves_per_eu(S::AT_ONCE, S::AT_ONCE))) void gradients_kernel(const Gradients g)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const uint32_t first = g.dx.blocks(), second = g.dw_gate_up.blocks();
    if (blockIdx.x < first) {
        work<S, true, true, STORE>(g.dx, blockIdx.x, first, lds);
    } else {
        const bool up = blockIdx.x - first < second;
        work<S, false, false, STORE>(up ? g.dw_gate_up : g.dw_down, blockIdx.x - first - (up ? 0 : second), up ? second : g.dw_down.blocks(), lds);
    }
}

// The shares of products whose k's were divided, added in order; then as above.  A thread has eight columns.
struct Join {
    const float *partial;
    uint32_t shares, M, N, up; // N: columns to be written; up: from gates to ups
    uint64_t ld, first;        // first: chunk of eight columns where this one starts, of all of the launch's
    Target to;
};
struct Joins {
    Join one[3];
    uint32_t count;
    uint64_t chunks;
};
template <int KIND, int PARTS>
__global__ __launch_bounds__(256) void join_kernel(const Joins joins)
{
    for (uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x; at < joins.chunks; at += (uint64_t)gridDim.x * 256) {
        int which = 0;
        while (which + 1 < (int)joins.count && at >= joins.one[which + 1].first) ++which;
        const Join &j = joins.one[which];
        const uint32_t chunks = (j.N + 7) / 8, m = (uint32_t)((at - j.first) / chunks), c = (uint32_t)((at - j.first) % chunks) * 8;
        const auto total = [&](uint32_t column, float(&v)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
#pragma unroll 4
            for (uint32_t s = 0; s < j.shares; ++s) {
                float some[8];
                load_eight(j.partial + ((uint64_t)s * j.M + m) * j.ld, column, (uint32_t)j.ld, some);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += some[i];
            }
        };
        float v[8];
        total(c, v);
        if (KIND == STORE) finish_store<PARTS>(j.to, m, c, v);
        if (KIND == SLOPE) {
            Pre pre;
            load_pre(j.to, m, c, pre);
            finish_slope<PARTS>(j.to, m, c, v, pre);
        }
        if (KIND == GATE) {
            float u[8];
            total(j.up + c, u);
            finish_gate<PARTS>(j.to, m, c, v, u);
        }
    }
}

// ------------------------------------------------------------------------------------------------ operands

// Matrices as operands want them: rows of two pieces of `piece` columns (one, if pieces is 1), each padded with zeros to `pitch` (a
// multiple of eight, or, for fp32 ones in three parts, of 32).  A thread has eight columns.
template <class T>
struct Pack {
    const T *src;
    bf16 *dst;
    uint64_t ld, first; // first: chunk of eight columns where this one starts, of all of the launch's
    uint32_t piece, pieces, pitch;
};
template <class T>
struct Packs {
    Pack<T> one[4];
    uint32_t count;
    uint64_t chunks;
};
template <class T>
__global__ __launch_bounds__(256) void pack_kernel(const Packs<T> packs)
{
    for (uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x; at < packs.chunks; at += (uint64_t)gridDim.x * 256) {
        int which = 0;
        while (which + 1 < (int)packs.count && at >= packs.one[which + 1].first) ++which;
        const Pack<T> &p = packs.one[which];
        const uint32_t chunks = p.pitch / 8 * p.pieces;
        const uint64_t r = (at - p.first) / chunks;
        const uint32_t c = (uint32_t)((at - p.first) % chunks) * 8, shift = c >= p.pitch ? p.pitch : 0;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i += Chunk<T>::N) {
            float some[Chunk<T>::N];
            load_chunk(p.src + r * p.ld + (shift ? p.piece : 0), c - shift + i, p.piece, some);
#pragma unroll
            for (int j = 0; j < Chunk<T>::N; ++j) v[i + j] = some[j];
        }
        constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
        store_operand<PARTS>(p.dst + r * ((uint64_t)p.pitch * p.pieces * PARTS), c, v);
    }
}

} // namespace product
} // namespace eck
