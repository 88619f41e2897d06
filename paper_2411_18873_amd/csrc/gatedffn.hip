// Gated feed-forward blocks, forward and backward (HIP, gfx950).
//
//   forward   [g | u] = x Wgu,  h = a(g) u,  y = h Wd
//   backward  dh = dy Wd^T,  dg = dh u a'(g),  du = dh a(g),  dx = [dg | du] Wgu^T,  dWgu = x^T [dg | du],  dWd = h^T dy
//
// Six products; the activation, its derivative and the product of gate and up happen where a product's sums still are in registers.
#include "product.h"

namespace eck {
namespace {

using namespace product;

constexpr uint64_t MAX_BLOCK_WIDTH = 1 << 20; // offsets within a tile's 256 rows of twice as many columns fit 31 bits
constexpr uint64_t MAX_TILES = 1 << 22;       // of a product
constexpr uint64_t MAX_STRAIGHT_LD = 1 << 21;

uint64_t up_to(uint64_t x, uint64_t step) { return (x + step - 1) / step * step; }
uint64_t padded(uint64_t bytes) { return up_to(bytes, 256); }

// ------------------------------------------------------------------------------------------------ which tiles

struct Plan {
    int shape; // 0 small, 1 medium, 2 large tiles
    uint32_t shares;
};

// The tiles and shares of k that should take a product of M x N x K (N: columns of b) least time, in units of 32 k's of a large tile.
Plan plan(uint64_t M, uint64_t N, uint64_t K, uint32_t parts)
{
    static const struct {
        uint32_t bm, bn, at_once; // blocks a compute unit
        double step;              // what 32 k's of as many tiles take a compute unit
    } SHAPES[3] = {{64, 64, 4, 0.55}, {128, 128, 2, 0.65}, {256, 256, 1, 1.0}};
    const uint64_t steps = (K + BK - 1) / BK * (parts == 3 ? 6 : 1);
    Plan best = {0, 1};
    double least = 1e300;
    for (int s = 0; s < 3; ++s) {
        const uint64_t tiles = (M + SHAPES[s].bm - 1) / SHAPES[s].bm * ((N + SHAPES[s].bn - 1) / SHAPES[s].bn), slots = 256ull * SHAPES[s].at_once;
        for (uint32_t shares = 1; shares <= 64; shares *= 2) {
            if (shares > 1 && (steps / shares < 8 || tiles * shares > 2 * slots)) break;
            const double rounds = (double)((tiles * shares + slots - 1) / slots);
            // a tile's start and end: about eight steps; shares: a launch and eight bytes a sum
            const double each = ((double)steps / shares + 8) * SHAPES[s].step;
            const double join = shares > 1 ? 8.0 + 8.0 * (double)M * (double)N * shares / 2.0e6 : 0.0;
            if (rounds * each + join < least) {
                least = rounds * each + join;
                best = {s, shares};
            }
        }
    }
    return best;
}

uint64_t tiles_of(uint64_t M, uint64_t N) { return ((M + 63) / 64) * ((N + 63) / 64); } // the smallest tiles

uint64_t partial_bytes(uint64_t M, uint64_t N, uint64_t K, uint32_t parts)
{
    const Plan how = plan(M, N, K, parts);
    return how.shares > 1 ? padded(how.shares * M * up_to(N, 8) * 4) : 0;
}

template <class S, bool A_FAST, bool B_FAST, int KIND, int PARTS>
int32_t launch_shape(const Product &p, hipStream_t st)
{
    auto kernel = product_kernel<S, A_FAST, B_FAST, KIND, PARTS>;
    if (S::LDS > 65536)
        ECK_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS));
    hipLaunchKernelGGL(kernel, dim3(p.tiles_m * p.tiles_n * p.shares), dim3(S::THREADS), S::LDS, st, p);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

template <class S, bool A_FAST, bool B_FAST, int KIND, int PARTS>
int32_t launch_tiles(Product p, uint32_t shares, float *partial, hipStream_t st)
{
    constexpr uint32_t COLUMNS = KIND == GATE ? 2 : 1;
    if (shares == 1) {
        p.shares = 1;
        p.tiles_m = (uint32_t)(((uint64_t)p.M + S::BM - 1) / S::BM);
        p.tiles_n = (p.N + S::BN / COLUMNS - 1) / (S::BN / COLUMNS);
        return launch_shape<S, A_FAST, B_FAST, KIND, PARTS>(p, st);
    }
    Product q = p;
    q.N = KIND == GATE ? p.b_up + p.N : p.N; // gates and ups side by side, as in memory
    q.shares = shares;
    q.tiles_m = (uint32_t)(((uint64_t)p.M + S::BM - 1) / S::BM);
    q.tiles_n = (q.N + S::BN - 1) / S::BN;
    q.to.out = partial;
    q.to.ld_out = up_to(q.N, 8);
    if (int32_t rc = launch_shape<S, A_FAST, B_FAST, PARTIAL, PARTS>(q, st)) return rc;
    const uint64_t blocks = ((uint64_t)p.M * ((p.N + 7) / 8) + 255) / 256;
    hipLaunchKernelGGL((join_kernel<KIND, PARTS>), dim3((uint32_t)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, st, partial, shares, p.M, p.N,
                       q.to.ld_out, p.b_up, p.to);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

template <bool A_FAST, bool B_FAST, int KIND, int PARTS>
int32_t launch(const Product &p, float *partial, hipStream_t st)
{
    const Plan how = plan(p.M, KIND == GATE ? (uint64_t)p.b_up + p.N : p.N, p.K, PARTS);
    if (how.shape == 0) return launch_tiles<Small, A_FAST, B_FAST, KIND, PARTS>(p, how.shares, partial, st);
    if (how.shape == 1) return launch_tiles<Medium, A_FAST, B_FAST, KIND, PARTS>(p, how.shares, partial, st);
    return launch_tiles<Large, A_FAST, B_FAST, KIND, PARTS>(p, how.shares, partial, st);
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

// The matrix [rows][pieces * piece] as an operand: itself where it is one already, else copied to `room`.
template <class T>
int32_t as_operand(const T *src, uint64_t ld, uint64_t rows, uint32_t piece, uint32_t pieces, char *room, Operand *out, hipStream_t st)
{
    if (sizeof(T) == 2 && piece % 8 == 0 && ld % 8 == 0 && ld <= MAX_STRAIGHT_LD && aligned(src, 16)) {
        *out = {(const bf16 *)src, ld, 0};
        return ECK_OK;
    }
    const uint32_t pitch = (uint32_t)up_to(piece, 8);
    const uint64_t width = (uint64_t)pitch * pieces, blocks = (rows * (width / 8) + 255) / 256;
    *out = {(const bf16 *)room, width, rows * width};
    hipLaunchKernelGGL(pack_kernel<T>, dim3((uint32_t)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, st, src, ld, (uint32_t)rows, piece, pieces,
                       pitch, (bf16 *)room, rows * width);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

struct Sizes {
    uint64_t n;
    uint32_t n_in, n_hidden, n_out;
    uint32_t hidden() const { return (uint32_t)up_to(n_hidden, 8); } // columns of h, and from gates to ups, in operands
};

template <class T>
struct Rooms { // the workspace's pieces, in order
    uint64_t x, w_gate_up, w_down, dy, d_pre, h, partial;
    uint64_t total() const { return x + w_gate_up + w_down + dy + d_pre + h + partial; }
};

uint64_t most(uint64_t a, uint64_t b) { return a > b ? a : b; }

template <class T>
Rooms<T> rooms(const Sizes &s, bool backward)
{
    constexpr uint32_t P = parts_of<T>;
    Rooms<T> r = {};
    r.x = operand_bytes(s.n, up_to(s.n_in, 8), P);
    r.w_gate_up = operand_bytes(s.n_in, 2ull * s.hidden(), P);
    r.w_down = operand_bytes(s.n_hidden, up_to(s.n_out, 8), P);
    r.h = operand_bytes(s.n, s.hidden(), P);
    if (!backward) {
        r.partial = most(partial_bytes(s.n, s.hidden() + s.n_hidden, s.n_in, P), partial_bytes(s.n, s.n_out, s.n_hidden, P));
        return r;
    }
    r.dy = operand_bytes(s.n, up_to(s.n_out, 8), P);
    r.d_pre = operand_bytes(s.n, 2ull * s.hidden(), P);
    r.partial = most(most(partial_bytes(s.n, s.n_hidden, s.n_out, P), partial_bytes(s.n, s.n_in, s.hidden() + s.n_hidden, P)),
                     most(partial_bytes(s.n_in, s.hidden() + s.n_hidden, s.n, P), partial_bytes(s.n_hidden, s.n_out, s.n, P)));
    return r;
}

// ------------------------------------------------------------------------------------------------ passes

#define ECK_TRY(expr)                   \
    do {                                \
        if (int32_t rc_ = (expr)) return rc_; \
    } while (0)

constexpr uint32_t NO_GAP = 0xFFFFFFFFu;

template <class T>
int32_t forward(const T *x, uint64_t ld_x, const Sizes &s, const T *w_gate_up, const T *w_down, int32_t act, T *y, uint64_t ld_y, float *pre,
                void *ws, hipStream_t st)
{
    constexpr uint32_t P = parts_of<T>;
    const Rooms<T> room = rooms<T>(s, false);
    Workspace space = {(char *)ws};
    Operand ox, ogu, od;
    ECK_TRY(as_operand(x, ld_x, s.n, s.n_in, 1, space.take(room.x), &ox, st));
    ECK_TRY(as_operand(w_gate_up, 2ull * s.n_hidden, s.n_in, s.n_hidden, 2, space.take(room.w_gate_up), &ogu, st));
    ECK_TRY(as_operand(w_down, s.n_out, s.n_hidden, s.n_out, 1, space.take(room.w_down), &od, st));
    const Operand h = {(bf16 *)space.take(room.h), s.hidden(), s.n * s.hidden()};
    float *partial = (float *)space.take(room.partial);

    Product p = {};
    p.a = ox, p.b = ogu, p.b_up = s.hidden();
    p.M = (uint32_t)s.n, p.N = s.n_hidden, p.K = s.n_in;
    p.to.out = const_cast<bf16 *>(h.p), p.to.ld_out = h.ld, p.to.part_out = h.part, p.to.pre = pre, p.to.n_hidden = s.n_hidden, p.to.act = act;
    ECK_TRY((launch<true, false, GATE, P>(p, partial, st)));

    p = {};
    p.a = h, p.b = od;
    p.M = (uint32_t)s.n, p.N = s.n_out, p.K = s.n_hidden;
    p.to.out = y, p.to.ld_out = ld_y, p.to.piece = s.n_out, p.to.pitch = NO_GAP;
    return launch<true, false, STORE, P>(p, partial, st);
}

template <class T>
int32_t backward(const T *x, uint64_t ld_x, const Sizes &s, const T *w_gate_up, const T *w_down, int32_t act, const float *pre, const T *dy,
                 uint64_t ld_dy, T *dx, uint64_t ld_dx, T *dw_gate_up, T *dw_down, void *ws, hipStream_t st)
{
    constexpr uint32_t P = parts_of<T>;
    const Rooms<T> room = rooms<T>(s, true);
    Workspace space = {(char *)ws};
    char *room_x = space.take(room.x), *room_gu = space.take(room.w_gate_up), *room_d = space.take(room.w_down), *room_dy = space.take(room.dy);
    const Operand d_pre = {(bf16 *)space.take(room.d_pre), 2ull * s.hidden(), s.n * 2 * s.hidden()};
    const Operand h = {(bf16 *)space.take(room.h), s.hidden(), s.n * s.hidden()};
    float *partial = (float *)space.take(room.partial);
    Operand ody, od, other;
    ECK_TRY(as_operand(dy, ld_dy, s.n, s.n_out, 1, room_dy, &ody, st));
    ECK_TRY(as_operand(w_down, s.n_out, s.n_hidden, s.n_out, 1, room_d, &od, st));

    Product p = {}; // dh, and from it dg, du and h
    p.a = ody, p.b = od;
    p.M = (uint32_t)s.n, p.N = s.n_hidden, p.K = s.n_out;
    p.to.out = dw_down ? const_cast<bf16 *>(h.p) : nullptr, p.to.ld_out = h.ld, p.to.part_out = h.part;
    p.to.pre = const_cast<float *>(pre), p.to.n_hidden = s.n_hidden, p.to.act = act, p.to.pitch = s.hidden();
    p.to.d_pre = const_cast<bf16 *>(d_pre.p), p.to.ld_d = d_pre.ld, p.to.part_d = d_pre.part;
    ECK_TRY((launch<true, true, SLOPE, P>(p, partial, st)));
    if (dx) {
        ECK_TRY(as_operand(w_gate_up, 2ull * s.n_hidden, s.n_in, s.n_hidden, 2, room_gu, &other, st));
        p = {};
        p.a = d_pre, p.b = other;
        p.M = (uint32_t)s.n, p.N = s.n_in, p.K = s.hidden() + s.n_hidden;
        p.to.out = dx, p.to.ld_out = ld_dx, p.to.piece = s.n_in, p.to.pitch = NO_GAP;
        ECK_TRY((launch<true, true, STORE, P>(p, partial, st)));
    }
    if (dw_gate_up) {
        ECK_TRY(as_operand(x, ld_x, s.n, s.n_in, 1, room_x, &other, st));
        p = {};
        p.a = other, p.b = d_pre;
        p.M = s.n_in, p.N = s.hidden() + s.n_hidden, p.K = (uint32_t)s.n;
        p.to.out = dw_gate_up, p.to.ld_out = 2ull * s.n_hidden, p.to.piece = s.n_hidden, p.to.pitch = s.hidden();
        ECK_TRY((launch<false, false, STORE, P>(p, partial, st)));
    }
    if (dw_down) {
        p = {};
        p.a = h, p.b = ody;
        p.M = s.n_hidden, p.N = s.n_out, p.K = (uint32_t)s.n;
        p.to.out = dw_down, p.to.ld_out = s.n_out, p.to.piece = s.n_out, p.to.pitch = NO_GAP;
        ECK_TRY((launch<false, false, STORE, P>(p, partial, st)));
    }
    return ECK_OK;
}

bool sizes_ok(const Sizes &s)
{
    const uint64_t hidden = s.hidden();
    return s.n <= MAX_ROWS && s.n_in <= MAX_BLOCK_WIDTH && s.n_hidden <= MAX_BLOCK_WIDTH && s.n_out <= MAX_BLOCK_WIDTH &&
           tiles_of(s.n, 2 * hidden) <= MAX_TILES && tiles_of(s.n, s.n_out) <= MAX_TILES && tiles_of(s.n, s.n_in) <= MAX_TILES &&
           tiles_of(s.n_in, 2 * hidden) <= MAX_TILES && tiles_of(s.n_hidden, s.n_out) <= MAX_TILES;
}
bool act_ok(int32_t act) { return act == ECK_ACT_SILU || act == ECK_ACT_GELU || act == ECK_ACT_RELU; }
uint64_t workspace_bytes(const Sizes &s, int32_t dtype, bool backward)
{
    if (s.n == 0 || s.n_in == 0 || s.n_hidden == 0 || s.n_out == 0 || !is_dtype(dtype) || !sizes_ok(s)) return 0;
    return dtype == ECK_F32 ? rooms<float>(s, backward).total() : rooms<bf16>(s, backward).total();
}

} // namespace
} // namespace eck

using namespace eck;

extern "C" uint64_t gatedffn_forward_workspace_bytes(uint64_t n, uint32_t n_in, uint32_t n_hidden, uint32_t n_out, int32_t dtype)
{
    return workspace_bytes({n, n_in, n_hidden, n_out}, dtype, false);
}

extern "C" int32_t gatedffn_forward(const void *x, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t n_in, uint32_t n_hidden,
                                    uint32_t n_out, const void *w_gate_up, const void *w_down, int32_t act, void *y, uint64_t ld_y,
                                    float *pre_out, void *ws, uint64_t ws_bytes, void *stream)
{
    const Sizes s = {n, n_in, n_hidden, n_out};
    if (!x || !w_gate_up || !w_down || !y || n == 0 || n_in == 0 || n_hidden == 0 || n_out == 0 || !is_dtype(dtype) || !act_ok(act)) return ECK_EINVAL;
    if (ld_x < n_in || ld_y < n_out) return ECK_ESHAPE;
    if (!sizes_ok(s)) return ECK_EUNSUPPORTED;
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
    return workspace_bytes({n, n_in, n_hidden, n_out}, dtype, true);
}

extern "C" int32_t gatedffn_backward(const void *x, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t n_in, uint32_t n_hidden,
                                     uint32_t n_out, const void *w_gate_up, const void *w_down, int32_t act, const float *pre,
                                     const void *dy, uint64_t ld_dy, void *dx_out, uint64_t ld_dx, void *dw_gate_up_out, void *dw_down_out,
                                     void *ws, uint64_t ws_bytes, void *stream)
{
    const Sizes s = {n, n_in, n_hidden, n_out};
    if (!x || !w_gate_up || !w_down || !pre || !dy || n == 0 || n_in == 0 || n_hidden == 0 || n_out == 0 || !is_dtype(dtype)) return ECK_EINVAL;
    if ((!dx_out && !dw_gate_up_out && !dw_down_out) || !act_ok(act)) return ECK_EINVAL;
    if (ld_x < n_in || ld_dy < n_out || (dx_out && ld_dx < n_in)) return ECK_ESHAPE;
    if (!sizes_ok(s)) return ECK_EUNSUPPORTED;
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
