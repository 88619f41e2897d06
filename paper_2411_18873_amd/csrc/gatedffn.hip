// Gated feed-forward blocks, forward and backward (HIP, gfx950).
//
//   forward   [g | u] = x Wgu,  h = a(g) u,  y = h Wd
//   backward  dh = dy Wd^T,  dg = dh u a'(g),  du = dh a(g),  dx = [dg | du] Wgu^T,  dWgu = x^T [dg | du],  dWd = h^T dy
//
// Six products; the activation, its derivative and the product of gate and up happen where a product's sums still are in registers.
#include "block_forward.h"

namespace eck {
namespace {

using namespace product;

constexpr uint64_t MAX_BLOCK_WIDTH = 1 << 20; // offsets within a tile's 256 rows of twice as many columns fit 31 bits
constexpr uint64_t MAX_TILES = 1 << 22;       // of a product
constexpr uint64_t MAX_STRAIGHT_LD = 1 << 21;
constexpr uint64_t MAX_SHARED = 1 << 27;      // sums of a product's shares

#define ECK_TRY(expr)                         \
    do {                                      \
        if (int32_t rc_ = (expr)) return rc_; \
    } while (0)

uint64_t up_to(uint64_t x, uint64_t step) { return (x + step - 1) / step * step; }
uint64_t padded(uint64_t bytes) { return up_to(bytes, 256); }

// ------------------------------------------------------------------------------------------------ which tiles

int shapes_of(uint32_t parts) { return parts == 3 ? Shapes<3>::COUNT : Shapes<1>::COUNT; }

struct Plan {
    int shape; // 0 small, 1 medium, 2 large tiles
    uint32_t shares;
    double time;
};

// The shares of k that should take a product of M x N x K (N: columns of b) least time in tiles of a shape, and that time (us).  The
// constants were fitted to 186 products of 17 blocks in bf16 and 90 of 15 blocks in parts (1 to 131072 rows, widths 7 to 8192), each in
// all shapes and up to 64 shares: the choice takes 0.7 % more than the best, on average, and 15 (in parts 21) % at most.
Plan plan_shape(int shape, uint64_t M, uint64_t N, uint64_t K, uint32_t parts)
{
    static const struct {
        uint32_t side, at_once;   // blocks a compute unit
        double step, alone, rest; // a step of a tile when the unit is full, with nothing beside them, and a tile's start and end
    } SHAPES[2][3] = {{{64, 3, 0.27, 0.31, 2.2}, {128, 2, 0.5, 0.71, 3.0}, {256, 1, 1.29, 1.58, 8.3}},
                      {{64, 2, 0.53, 0.5, 2.1}, {128, 1, 0.8, 0.88, 5.1}, {}}}; // (parts)
    const auto &of = SHAPES[parts == 3][shape];
    const uint64_t steps = parts == 3 ? (K + STAGE_K<3> - 1) / STAGE_K<3> : (K + STAGE_K<1> - 1) / STAGE_K<1>, tiles = (M + of.side - 1) / of.side * ((N + of.side - 1) / of.side);
    Plan best = {shape, 1, 1e300};
    for (uint32_t shares = 1; shares <= 64; shares *= 2) {
        if (shares > 1 && (steps / shares < 2 || tiles * shares > 2048 || shares * M * N > MAX_SHARED)) break;
        const uint64_t a_unit = (tiles * shares + 255) / 256, full = a_unit / of.at_once, last = a_unit % of.at_once;
        const auto round = [&](uint64_t blocks) {
            const double step = of.step * (double)blocks;
            return of.rest + (double)steps / shares * (step > of.alone ? step : of.alone);
        };
        double time = (double)full * round(of.at_once) + (last ? round(last) : 0.0);
        if (shares > 1) time += 3.6 + shares * (0.38 + (double)M * (double)N * 8.0 / 5.0e6); // a launch; sums written and read
        if (time < best.time) best = {shape, shares, time};
    }
    return best;
}

Plan plan(uint64_t M, uint64_t N, uint64_t K, uint32_t parts)
{
    Plan best = plan_shape(0, M, N, K, parts);
    for (int shape = 1; shape < shapes_of(parts); ++shape) {
        const Plan other = plan_shape(shape, M, N, K, parts);
        if (other.time < best.time) best = other;
    }
    return best;
}

uint64_t tiles_of(uint64_t M, uint64_t N) { return ((M + 63) / 64) * ((N + 63) / 64); } // the smallest tiles

uint64_t shares_bytes(const Plan &how, uint64_t M, uint64_t N) { return how.shares > 1 ? padded(how.shares * M * up_to(N, 8) * 4) : 0; }
uint64_t partial_bytes(uint64_t M, uint64_t N, uint64_t K, uint32_t parts) { return shares_bytes(plan(M, N, K, parts), M, N); }

// kernels take blocks of more than 64 KB of LDS once they were told so
template <class Kernel>
int32_t allow_lds(Kernel kernel, int bytes)
{
    if (bytes > 65536) ECK_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    return ECK_OK;
}

uint32_t blocks_for(uint64_t chunks)
{
    const uint64_t blocks = (chunks + 255) / 256;
    return (uint32_t)(blocks < 16384 ? blocks : 16384);
}

// Cuts a product into tiles of `side` and shares of k; shares leave their sums in `partial` (advanced past them) and a Join
template <int KIND>
void divide(Product &p, uint32_t side, uint32_t shares, char *&partial, Joins &joins)
{
    const Product whole = p;
    p.shares = shares;
    if (shares > 1) {
        if (KIND == GATE) p.N = p.b_up + p.N; // gates and ups side by side, as in memory
        p.to.out = partial;
        p.to.ld_out = up_to(p.N, 8);
        const uint32_t columns = KIND == SLOPE ? whole.to.pitch : whole.N;
        joins.one[joins.count++] = {(const float *)partial, shares, whole.M, columns, whole.b_up, p.to.ld_out, joins.chunks, whole.to};
        joins.chunks += (uint64_t)whole.M * ((columns + 7) / 8);
        partial += padded(shares * (uint64_t)p.M * p.to.ld_out * 4);
    }
    const uint32_t columns = KIND == GATE && shares == 1 ? side / 2 : side;
    p.tiles_m = (uint32_t)(((uint64_t)p.M + side - 1) / side);
    p.tiles_n = (p.N + columns - 1) / columns;
}

template <int KIND, int PARTS>
int32_t launch_joins(const Joins &joins, hipStream_t st)
{
    if (joins.count == 0) return ECK_OK;
    hipLaunchKernelGGL((join_kernel<KIND, PARTS>), dim3(blocks_for(joins.chunks)), dim3(256), 0, st, joins);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

template <class S, bool A_FAST, bool B_FAST, int KIND>
int32_t launch_tiles(const Product &p, hipStream_t st)
{
    auto kernel = product_kernel<S, A_FAST, B_FAST, KIND>;
    ECK_TRY(allow_lds(kernel, S::LDS));
    hipLaunchKernelGGL(kernel, dim3(p.blocks()), dim3(S::THREADS), S::LDS, st, p);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

template <bool A_FAST, bool B_FAST, int KIND, int PARTS>
int32_t launch_shape(int shape, const Product &p, hipStream_t st)
{
    using S = Shapes<PARTS>;
    if (shape == 0) return launch_tiles<typename S::Small, A_FAST, B_FAST, KIND>(p, st);
    if constexpr (S::COUNT == 3)
        if (shape == 2) return launch_tiles<typename S::Large, A_FAST, B_FAST, KIND>(p, st);
    return launch_tiles<typename S::Medium, A_FAST, B_FAST, KIND>(p, st);
}

constexpr uint32_t SIDES[3] = {64, 128, 256};

template <bool A_FAST, bool B_FAST, int KIND, int PARTS>
int32_t launch(Product p, const Plan &how, char *partial, hipStream_t st)
{
    Joins joins = {};
    divide<KIND>(p, SIDES[how.shape], how.shares, partial, joins);
    if (how.shares == 1) return launch_shape<A_FAST, B_FAST, KIND, PARTS>(how.shape, p, st);
    ECK_TRY((launch_shape<A_FAST, B_FAST, STORE, PARTS>(how.shape, p, st)));
    return launch_joins<KIND, PARTS>(joins, st);
}

template <class S>
int32_t launch_group(const Gradients &g, hipStream_t st)
{
    auto kernel = gradients_kernel<S>;
    ECK_TRY(allow_lds(kernel, S::LDS));
    hipLaunchKernelGGL(kernel, dim3(g.dx.blocks() + g.dw_gate_up.blocks() + g.dw_down.blocks()), dim3(S::THREADS), S::LDS, st, g);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

template <int PARTS>
int32_t launch_gradients(int shape, const Gradients &g, hipStream_t st)
{
    using S = Shapes<PARTS>;
    if (shape == 0) return launch_group<typename S::Small>(g, st);
    if constexpr (S::COUNT == 3)
        if (shape == 2) return launch_group<typename S::Large>(g, st);
    return launch_group<typename S::Medium>(g, st);
}

// ------------------------------------------------------------------------------------------------ operands

template <class T>
constexpr uint32_t parts_of = sizeof(T) == 4 ? 3 : 1;

// bytes of a matrix as an operand
uint64_t operand_bytes(uint64_t rows, uint64_t pitch, uint32_t parts) { return padded(rows * pitch * 2 * parts); }

struct Workspace {
    char *at;
    char *take(uint64_t bytes)
    {
        char *p = at;
        at += bytes;
        return p;
    }
};

// columns of a matrix of `width` as an operand
uint64_t pitch_of(uint64_t width, uint32_t parts) { return up_to(width, parts == 3 ? 32 : 8); }

template <class T>
bool is_operand(const T *src, uint64_t ld, uint32_t piece)
{
    return sizeof(T) == 2 && piece % 8 == 0 && ld % 8 == 0 && ld <= MAX_STRAIGHT_LD && aligned(src, 16);
}

// The matrix [rows][pieces * piece] as an operand: itself where it is one already, else to be copied to `room`.
template <class T>
Operand as_operand(const T *src, uint64_t ld, uint64_t rows, uint32_t piece, uint32_t pieces, char *room, Packs<T> &packs)
{
    if (is_operand(src, ld, piece)) return {(const bf16 *)src, ld};
    const uint32_t pitch = (uint32_t)pitch_of(piece, parts_of<T>);
    const uint64_t width = (uint64_t)pitch * pieces;
    packs.one[packs.count++] = {src, (bf16 *)room, ld, packs.chunks, piece, pieces, pitch};
    packs.chunks += rows * (width / 8);
    return {(const bf16 *)room, width * parts_of<T>};
}

template <class T>
int32_t launch_packs(const Packs<T> &packs, hipStream_t st)
{
    if (packs.count == 0) return ECK_OK;
    hipLaunchKernelGGL(pack_kernel<T>, dim3(blocks_for(packs.chunks)), dim3(256), 0, st, packs);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

uint32_t parts_for(int32_t dtype) { return dtype == ECK_F32 ? 3 : 1; }

struct Sizes {
    uint64_t n;
    uint32_t n_in, n_hidden, n_out;
    uint32_t parts;
    uint32_t hidden() const { return (uint32_t)pitch_of(n_hidden, parts); } // columns of h, and from gates to ups, in operands
    uint32_t pairs() const { return hidden() + n_hidden; }                  // columns of (g | u)
};

// The shape of tiles that all three gradients take, being one launch, and the shares of each: dx, dWgu, dWd, those wanted
struct GradientPlans {
    Plan of[3];
};
GradientPlans plan_gradients(const Sizes &s, bool dx, bool dw_gate_up, bool dw_down)
{
    const uint32_t parts = s.parts;
    GradientPlans best = {};
    double least = 1e300;
    for (int shape = 0; shape < shapes_of(parts); ++shape) {
        const GradientPlans now = {{plan_shape(shape, s.n, s.n_in, s.pairs(), parts), plan_shape(shape, s.n_in, s.pairs(), s.n, parts),
                                    plan_shape(shape, s.n_hidden, s.n_out, s.n, parts)}};
        const double time = (dx ? now.of[0].time : 0.0) + (dw_gate_up ? now.of[1].time : 0.0) + (dw_down ? now.of[2].time : 0.0);
        if (time < least) {
            least = time;
            best = now;
        }
    }
    return best;
}

struct Rooms { // the workspace's pieces, in order
    uint64_t x, w_gate_up, w_down, dy, d_pre, h, partial;
    uint64_t total() const { return x + w_gate_up + w_down + dy + d_pre + h + partial; }
};

uint64_t most(uint64_t a, uint64_t b) { return a > b ? a : b; }

Rooms rooms(const Sizes &s, bool backward)
{
    const uint32_t parts = s.parts;
    Rooms r = {};
    r.x = operand_bytes(s.n, pitch_of(s.n_in, parts), parts);
    r.w_gate_up = operand_bytes(s.n_in, 2ull * s.hidden(), parts);
    r.w_down = operand_bytes(s.n_hidden, pitch_of(s.n_out, parts), parts);
    r.h = operand_bytes(s.n, s.hidden(), parts);
    if (!backward) {
        r.partial = most(partial_bytes(s.n, s.pairs(), s.n_in, parts), partial_bytes(s.n, s.n_out, s.n_hidden, parts));
        return r;
    }
    r.dy = operand_bytes(s.n, pitch_of(s.n_out, parts), parts);
    r.d_pre = operand_bytes(s.n, 2ull * s.hidden(), parts);
    r.partial = partial_bytes(s.n, s.n_hidden, s.n_out, parts);
    for (int wanted = 1; wanted < 8; ++wanted) { // (the shape of tiles depends on which gradients are)
        const bool dx = wanted & 1, dw_gate_up = wanted & 2, dw_down = wanted & 4;
        const GradientPlans how = plan_gradients(s, dx, dw_gate_up, dw_down);
        r.partial = most(r.partial, (dx ? shares_bytes(how.of[0], s.n, s.n_in) : 0) + (dw_gate_up ? shares_bytes(how.of[1], s.n_in, s.pairs()) : 0) +
                                        (dw_down ? shares_bytes(how.of[2], s.n_hidden, s.n_out) : 0));
    }
    return r;
}

// ------------------------------------------------------------------------------------------------ passes

constexpr uint32_t NO_GAP = 0xFFFFFFFFu;

// Few rows: the weights' bytes (block_forward.h).  Up to how many rows that is faster than products of matrices, us, products first.
// Aligned bf16 weights, one row: 512-2048-512 15.0 and 13.1, 2048-5632-2048 24.2 and 24.0, 4096-8192-4096 53.4 and 49.6; two 15.1 and
// 14.1, 24.3 and 28.4, 53.4 and 53.2.  Where the weights have to be copied, four rows take 0.49 to 0.81 of the products' time if it is
// for their address alone (4096-8192-4096 152 and 75, 512-2048-512 21.9 and 17.8) and 0.94 on average, 0.77 to 1.13, if it is for
// widths (17 blocks: 64-257-63 13.6 and 12.9, 1000-3001-1001 28.4 and 23.0, 4096-8191-4095 171 and 143; but 500-1501-333 20.4 and
// 22.6, 256-1023-255 17.3 and 19.4, 2048-5631-2047 58 and 65: few columns' blocks, or some more than units); eight rows 18.8 and
// 24.1 at 500-1501-333, 52.5 and 74.8, 27.5 and 27.2 at 1000-3001-1001.  fp32, whose weights always have to be, sixteen rows:
// 64-257-63 14.2 and 12.8, 500-1501-333 29.1 and 23.6, 4096-8192-4096 339 and 151.
constexpr uint32_t FEW_ROWS = 1, FEW_COPIED = 4, FEW_F32 = 16;
bool few(const Sizes &s, bool straight) { return s.n <= (s.parts == 3 ? FEW_F32 : straight ? FEW_ROWS : FEW_COPIED); }

// of the k's, so that all compute units have a block if every one of them gets two rounds of loads at least
uint32_t vector_shares(uint32_t K, uint32_t N, uint32_t line)
{
    const uint32_t blocks = (N + line - 1) / line, wanted = (255 + blocks) / blocks, most = K / 256;
    return wanted < most ? wanted : most > 1 ? most : 1;
}
// bytes of the shares of (g | u), and of y
struct VectorRooms {
    uint32_t shares, shares_y;
    uint64_t sums, sums_y;
};
VectorRooms vector_rooms(const Sizes &s)
{
    const uint32_t line = s.parts == 3 ? 32 : 64;
    VectorRooms r = {vector_shares(s.n_in, s.n_hidden, line), vector_shares(s.n_hidden, s.n_out, line), 0, 0};
    r.sums = padded(r.shares * s.n * 2 * s.n_hidden * 4);
    r.sums_y = r.shares_y > 1 ? padded(r.shares_y * s.n * up_to(s.n_out, 8) * 4) : 0;
    return r;
}

template <class T, bool PAIRS, int ROWS>
int32_t launch_vector_rows(const Rows &rows, uint32_t shares, const T *w, uint64_t ld_w, uint32_t N, T *out, uint64_t ld_out, float *sums,
                           hipStream_t st)
{
    constexpr int LINE = 8 * Chunk<T>::N, SUMS = 16 * ROWS * LINE * (PAIRS ? 2 : 1), VALUES = ROWS * VECTOR_K<ROWS>;
    constexpr int LDS = (VALUES > SUMS ? VALUES : SUMS) * 4;
    auto kernel = vector_kernel<T, PAIRS, ROWS>;
    ECK_TRY(allow_lds(kernel, LDS));
    hipLaunchKernelGGL(kernel, dim3((N + LINE - 1) / LINE, shares), dim3(1024), LDS, st, rows, w, ld_w, N, N, out, ld_out, sums);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}
template <class T, bool PAIRS>
int32_t launch_vector(const Rows &rows, uint32_t shares, const T *w, uint64_t ld_w, uint32_t N, T *out, uint64_t ld_out, float *sums, hipStream_t st)
{
    if (rows.n == 1) return launch_vector_rows<T, PAIRS, 1>(rows, shares, w, ld_w, N, out, ld_out, sums, st);
    if (rows.n == 2) return launch_vector_rows<T, PAIRS, 2>(rows, shares, w, ld_w, N, out, ld_out, sums, st);
    if constexpr (sizeof(T) == 4) {
        if (rows.n > 8) return launch_vector_rows<T, PAIRS, 16>(rows, shares, w, ld_w, N, out, ld_out, sums, st);
        if (rows.n > 4) return launch_vector_rows<T, PAIRS, 8>(rows, shares, w, ld_w, N, out, ld_out, sums, st);
    }
    return launch_vector_rows<T, PAIRS, 4>(rows, shares, w, ld_w, N, out, ld_out, sums, st);
}

template <class T>
int32_t forward_few(const T *x, uint64_t ld_x, const Sizes &s, const T *w_gate_up, const T *w_down, int32_t act, T *y, uint64_t ld_y, float *pre,
                    void *ws, hipStream_t st)
{
    const VectorRooms room = vector_rooms(s);
    float *sums = (float *)ws, *sums_y = (float *)((char *)ws + room.sums);
    const uint32_t n = (uint32_t)s.n;
    ECK_TRY((launch_vector<T, true>({x, nullptr, ld_x, nullptr, n, s.n_in, 0, act}, room.shares, w_gate_up, 2ull * s.n_hidden, s.n_hidden, nullptr, 0,
                                    sums, st)));
    const Rows h = {nullptr, sums, 0, pre, n, s.n_hidden, room.shares, act};
    if (room.shares_y == 1) return launch_vector<T, false>(h, 1, w_down, s.n_out, s.n_out, y, ld_y, nullptr, st);
    const uint64_t ld = up_to(s.n_out, 8);
    ECK_TRY((launch_vector<T, false>(h, room.shares_y, w_down, s.n_out, s.n_out, nullptr, ld, sums_y, st)));
    Joins joins = {};
    joins.count = 1, joins.chunks = s.n * ((s.n_out + 7) / 8);
    joins.one[0].partial = sums_y, joins.one[0].shares = room.shares_y, joins.one[0].M = n, joins.one[0].N = s.n_out, joins.one[0].ld = ld;
    joins.one[0].to.out = y, joins.one[0].to.ld_out = ld_y, joins.one[0].to.piece = s.n_out, joins.one[0].to.pitch = NO_GAP;
    return launch_joins<STORE, parts_of<T>>(joins, st);
}

// Narrow blocks without (g | u): one kernel where it should take less time than the two products (us).  A block of it goes through all
// hidden units for 128 rows, so up to 128 rows a compute unit its time does not depend on the rows, and with more it grows by whole
// blocks a unit; a turn of 32 units is bound by the activations (GELU's are three times SiLU's), in wide blocks by the products.  The
// constants were fitted to 583 pairs of measurements (28 shapes, 200 to 131072 rows, all activations): the choice takes 0.2 % more
// than the better one, on average, and 14 % at most.  One kernel and two products, us: 64-256-64 SiLU 4096 rows 7.6 and 8.5, 16384
// 7.7 and 11.5, 131072 21 and 61; 128-2048-128 8192 rows 58 and 40, 32768 62 and 117; 64-8192-256 12288 rows 320 and 197, 65536
// 415 and 897; GELU 64-1024-64 12288 rows 71 and 38, 65536 96 and 155; 128-4096-256 12288 rows 360 and 162, 131072 1479 and 1428.
// 256-1024-256 has no kernel: on 65536 rows it took 203 for 177.
constexpr uint32_t NARROW_IN = 128, NARROW_OUT = 256;
bool narrow(const Sizes &s, int32_t act)
{
    if (s.n_in > NARROW_IN || s.n_out > NARROW_OUT) return false;
    static const struct {
        double one, more; // a turn with one block on a unit, and for each of several
    } TURNS[2][2][3] = {{{{0.60, 0.51}, {0.75, 0.61}, {1.24, 0.84}}, {{1.01, 0.71}, {1.05, 0.91}, {1.50, 1.58}}},
                        {{{2.17, 1.49}, {2.28, 1.55}, {2.62, 1.74}}, {{2.36, 1.60}, {2.31, 1.82}, {2.80, 2.88}}}}; // GELU
    const bool gelu = act == ECK_ACT_GELU;
    const auto &turn = TURNS[gelu][s.n_in > 64][s.n_out <= 64 ? 0 : s.n_out <= 128 ? 1 : 2];
    const uint64_t turns = up_to(s.n_hidden, 64) / 32, blocks = (s.n + 32767) / 32768; // (of 128 rows on 256 units)
    const double values = (double)s.n * s.n_hidden * 1e-6, ends = (double)(s.n_in + s.n_out);
    const double products = 7.8 + values * (1.28 + 1.7e-3 * ends + (gelu ? 0.88 : 0.0)) + 0.155e-6 * (double)s.n * ends;
    return (s.n_out <= 128 ? 2.8 : 5.0) + (double)turns * (blocks == 1 ? turn.one : turn.more * (double)blocks) < products;
}
template <int ACT, int DK, int ON>
int32_t launch_narrow_shape(const Narrow &p, hipStream_t st)
{
    using S = NarrowShape<DK, ON>;
    auto kernel = p.n_hidden % S::UNITS ? narrow_kernel<DK, ON, ACT, true> : narrow_kernel<DK, ON, ACT, false>;
    ECK_TRY(allow_lds(kernel, S::LDS));
    hipLaunchKernelGGL(kernel, dim3((p.n - 1) / S::ROWS + 1), dim3(64 * S::WAVES), S::LDS, st, p);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}
template <int ACT, int DK>
int32_t launch_narrow_in(const Narrow &p, hipStream_t st)
{
    if (p.n_out <= 64) return launch_narrow_shape<ACT, DK, 4>(p, st);
    if (p.n_out <= 128) return launch_narrow_shape<ACT, DK, 8>(p, st);
    return launch_narrow_shape<ACT, DK, 16>(p, st);
}
template <int ACT>
int32_t launch_narrow_as(const Narrow &p, hipStream_t st)
{
    return p.n_in <= 64 ? launch_narrow_in<ACT, 2>(p, st) : launch_narrow_in<ACT, 4>(p, st);
}
int32_t launch_narrow(const Narrow &p, int32_t act, hipStream_t st)
{
    if (act == ECK_ACT_SILU) return launch_narrow_as<ECK_ACT_SILU>(p, st);
    return act == ECK_ACT_GELU ? launch_narrow_as<ECK_ACT_GELU>(p, st) : launch_narrow_as<ECK_ACT_RELU>(p, st);
}

template <class T>
int32_t forward(const T *x, uint64_t ld_x, const Sizes &s, const T *w_gate_up, const T *w_down, int32_t act, T *y, uint64_t ld_y, float *pre,
                void *ws, hipStream_t st)
{
    constexpr uint32_t P = parts_of<T>;
    if (few(s, is_operand(w_gate_up, 2ull * s.n_hidden, s.n_hidden) && is_operand(w_down, s.n_out, s.n_out)))
        return forward_few(x, ld_x, s, w_gate_up, w_down, act, y, ld_y, pre, ws, st);
    const Rooms room = rooms(s, false);
    Workspace space = {(char *)ws};
    Packs<T> packs = {};
    const Operand ox = as_operand(x, ld_x, s.n, s.n_in, 1, space.take(room.x), packs);
    const Operand ogu = as_operand(w_gate_up, 2ull * s.n_hidden, s.n_in, s.n_hidden, 2, space.take(room.w_gate_up), packs);
    const Operand od = as_operand(w_down, s.n_out, s.n_hidden, s.n_out, 1, space.take(room.w_down), packs);
    const Operand h = {(bf16 *)space.take(room.h), (uint64_t)P * s.hidden()};
    char *partial = space.take(room.partial);
    ECK_TRY(launch_packs(packs, st));
    if constexpr (P == 1)
        if (!pre && narrow(s, act))
            return launch_narrow({ox, ogu, od, (uint32_t)s.n, s.n_in, s.n_hidden, s.n_out, s.hidden(), y, ld_y}, act, st);

    Product p = {};
    p.a = ox, p.b = ogu, p.b_up = s.hidden();
    p.M = (uint32_t)s.n, p.N = s.n_hidden, p.K = s.n_in;
    p.to.out = const_cast<bf16 *>(h.p), p.to.ld_out = h.ld, p.to.pre = pre, p.to.n_hidden = s.n_hidden, p.to.act = act;
    ECK_TRY((launch<true, false, GATE, P>(p, plan(s.n, s.pairs(), s.n_in, P), partial, st)));

    p = {};
    p.a = h, p.b = od;
    p.M = (uint32_t)s.n, p.N = s.n_out, p.K = s.n_hidden;
    p.to.out = y, p.to.ld_out = ld_y, p.to.piece = s.n_out, p.to.pitch = NO_GAP;
    return launch<true, false, STORE, P>(p, plan(s.n, s.n_out, s.n_hidden, P), partial, st);
}

template <class T>
int32_t backward(const T *x, uint64_t ld_x, const Sizes &s, const T *w_gate_up, const T *w_down, int32_t act, const float *pre, const T *dy,
                 uint64_t ld_dy, T *dx, uint64_t ld_dx, T *dw_gate_up, T *dw_down, void *ws, hipStream_t st)
{
    constexpr uint32_t P = parts_of<T>;
    const Rooms room = rooms(s, true);
    Workspace space = {(char *)ws};
    char *room_x = space.take(room.x), *room_gu = space.take(room.w_gate_up), *room_d = space.take(room.w_down), *room_dy = space.take(room.dy);
    const Operand d_pre = {(bf16 *)space.take(room.d_pre), 2ull * P * s.hidden()};
    const Operand h = {(bf16 *)space.take(room.h), (uint64_t)P * s.hidden()};
    char *partial = space.take(room.partial);
    Packs<T> packs = {};
    const Operand ody = as_operand(dy, ld_dy, s.n, s.n_out, 1, room_dy, packs);
    const Operand od = as_operand(w_down, s.n_out, s.n_hidden, s.n_out, 1, room_d, packs);
    Operand ogu = {}, ox = {};
    if (dx) ogu = as_operand(w_gate_up, 2ull * s.n_hidden, s.n_in, s.n_hidden, 2, room_gu, packs);
    if (dw_gate_up) ox = as_operand(x, ld_x, s.n, s.n_in, 1, room_x, packs);
    ECK_TRY(launch_packs(packs, st));

    Product p = {}; // dh, and from it dg, du and h
    p.a = ody, p.b = od;
    p.M = (uint32_t)s.n, p.N = s.n_hidden, p.K = s.n_out;
    p.to.out = dw_down ? const_cast<bf16 *>(h.p) : nullptr, p.to.ld_out = h.ld;
    p.to.pre = const_cast<float *>(pre), p.to.n_hidden = s.n_hidden, p.to.act = act, p.to.pitch = s.hidden();
    p.to.d_pre = const_cast<bf16 *>(d_pre.p), p.to.ld_d = d_pre.ld;
    ECK_TRY((launch<true, true, SLOPE, P>(p, plan(s.n, s.n_hidden, s.n_out, P), partial, st)));

    const GradientPlans how = plan_gradients(s, dx, dw_gate_up, dw_down);
    const uint32_t side = SIDES[how.of[0].shape];
    Gradients g = {};
    Joins joins = {};
    if (dx) {
        g.dx.a = d_pre, g.dx.b = ogu, g.dx.M = (uint32_t)s.n, g.dx.N = s.n_in, g.dx.K = s.pairs();
        g.dx.to.out = dx, g.dx.to.ld_out = ld_dx, g.dx.to.piece = s.n_in, g.dx.to.pitch = NO_GAP;
        divide<STORE>(g.dx, side, how.of[0].shares, partial, joins);
    }
    if (dw_gate_up) {
        Product &q = g.dw_gate_up;
        q.a = ox, q.b = d_pre, q.M = s.n_in, q.N = s.pairs(), q.K = (uint32_t)s.n;
        q.to.out = dw_gate_up, q.to.ld_out = 2ull * s.n_hidden, q.to.piece = s.n_hidden, q.to.pitch = s.hidden();
        divide<STORE>(q, side, how.of[1].shares, partial, joins);
    }
    if (dw_down) {
        Product &q = g.dw_down;
        q.a = h, q.b = ody, q.M = s.n_hidden, q.N = s.n_out, q.K = (uint32_t)s.n;
        q.to.out = dw_down, q.to.ld_out = s.n_out, q.to.piece = s.n_out, q.to.pitch = NO_GAP;
        divide<STORE>(q, side, how.of[2].shares, partial, joins);
    }
    ECK_TRY(launch_gradients<P>(how.of[0].shape, g, st));
    return launch_joins<STORE, P>(joins, st);
}

bool sizes_ok(const Sizes &s, bool backward)
{
    const uint64_t pairs = 2ull * s.hidden();
    if (s.n > MAX_ROWS || s.n_in > MAX_BLOCK_WIDTH || s.n_hidden > MAX_BLOCK_WIDTH || s.n_out > MAX_BLOCK_WIDTH) return false;
    if (tiles_of(s.n, pairs) > MAX_TILES || tiles_of(s.n, s.n_out) > MAX_TILES) return false;
    return !backward || (tiles_of(s.n, s.n_in) <= MAX_TILES && tiles_of(s.n_in, pairs) <= MAX_TILES && tiles_of(s.n_hidden, s.n_out) <= MAX_TILES);
}
bool act_ok(int32_t act) { return act == ECK_ACT_SILU || act == ECK_ACT_GELU || act == ECK_ACT_RELU; }
uint64_t workspace_bytes(const Sizes &s, int32_t dtype, bool backward)
{
    if (s.n == 0 || s.n_in == 0 || s.n_hidden == 0 || s.n_out == 0 || !is_dtype(dtype) || !sizes_ok(s, backward)) return 0;
    if (!backward && few(s, false)) {
        const VectorRooms room = vector_rooms(s);
        return few(s, true) ? room.sums + room.sums_y : most(room.sums + room.sums_y, rooms(s, false).total());
    }
    return rooms(s, backward).total();
}

} // namespace
} // namespace eck

using namespace eck;

extern "C" uint64_t gatedffn_forward_workspace_bytes(uint64_t n, uint32_t n_in, uint32_t n_hidden, uint32_t n_out, int32_t dtype)
{
    return workspace_bytes({n, n_in, n_hidden, n_out, parts_for(dtype)}, dtype, false);
}

extern "C" int32_t gatedffn_forward(const void *x, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t n_in, uint32_t n_hidden,
                                    uint32_t n_out, const void *w_gate_up, const void *w_down, int32_t act, void *y, uint64_t ld_y,
                                    float *pre_out, void *ws, uint64_t ws_bytes, void *stream)
{
    const Sizes s = {n, n_in, n_hidden, n_out, parts_for(dtype)};
    if (!x || !w_gate_up || !w_down || !y || n == 0 || n_in == 0 || n_hidden == 0 || n_out == 0 || !is_dtype(dtype) || !act_ok(act)) return ECK_EINVAL;
    if (ld_x < n_in || ld_y < n_out) return ECK_ESHAPE;
    if (!sizes_ok(s, false)) return ECK_EUNSUPPORTED;
    if (!ws || ws_bytes < workspace_bytes(s, dtype, false)) return ECK_EWORKSPACE;
    const uint64_t size = element_bytes(dtype);
    if (!aligned(x, size) || !aligned(w_gate_up, size) || !aligned(w_down, size) || !aligned(y, size) || !aligned(pre_out, 4) || !aligned(ws, 256))
        return ECK_EALIGN;
    if (dtype == ECK_F32)
        return forward((const float *)x, ld_x, s, (const float *)w_gate_up, (const float *)w_down, act, (float *)y, ld_y, pre_out, ws, as_stream(stream));
    return forward((const bf16 *)x, ld_x, s, (const bf16 *)w_gate_up, (const bf16 *)w_down, act, (bf16 *)y, ld_y, pre_out, ws, as_stream(stream));
}

extern "C" uint64_t gatedffn_backward_workspace_bytes(uint64_t n, uint32_t n_in, uint32_t n_hidden, uint32_t n_out, int32_t dtype)
{
    return workspace_bytes({n, n_in, n_hidden, n_out, parts_for(dtype)}, dtype, true);
}

extern "C" int32_t gatedffn_backward(const void *x, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t n_in, uint32_t n_hidden,
                                     uint32_t n_out, const void *w_gate_up, const void *w_down, int32_t act, const float *pre,
                                     const void *dy, uint64_t ld_dy, void *dx_out, uint64_t ld_dx, void *dw_gate_up_out, void *dw_down_out,
                                     void *ws, uint64_t ws_bytes, void *stream)
{
    const Sizes s = {n, n_in, n_hidden, n_out, parts_for(dtype)};
    if (!x || !w_gate_up || !w_down || !pre || !dy || n == 0 || n_in == 0 || n_hidden == 0 || n_out == 0 || !is_dtype(dtype)) return ECK_EINVAL;
    if ((!dx_out && !dw_gate_up_out && !dw_down_out) || !act_ok(act)) return ECK_EINVAL;
    if (ld_x < n_in || ld_dy < n_out || (dx_out && ld_dx < n_in)) return ECK_ESHAPE;
    if (!sizes_ok(s, true)) return ECK_EUNSUPPORTED;
    if (!ws || ws_bytes < workspace_bytes(s, dtype, true)) return ECK_EWORKSPACE;
    const uint64_t size = element_bytes(dtype);
    if (!aligned(x, size) || !aligned(w_gate_up, size) || !aligned(w_down, size) || !aligned(pre, 4) || !aligned(dy, size) ||
        !aligned(dx_out, size) || !aligned(dw_gate_up_out, size) || !aligned(dw_down_out, size) || !aligned(ws, 256))
        return ECK_EALIGN;
    if (dtype == ECK_F32)
        return backward((const float *)x, ld_x, s, (const float *)w_gate_up, (const float *)w_down, act, pre, (const float *)dy, ld_dy,
                        (float *)dx_out, ld_dx, (float *)dw_gate_up_out, (float *)dw_down_out, ws, as_stream(stream));
    return backward((const bf16 *)x, ld_x, s, (const bf16 *)w_gate_up, (const bf16 *)w_down, act, pre, (const bf16 *)dy, ld_dy, (bf16 *)dx_out,
                    ld_dx, (bf16 *)dw_gate_up_out, (bf16 *)dw_down_out, ws, as_stream(stream));
}
