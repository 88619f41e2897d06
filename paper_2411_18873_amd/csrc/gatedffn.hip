// Gated feed-forward blocks, forward and backward (HIP, gfx950).
//
//   forward   [g | u] = x Wgu,  h = a(g) u,  y = h Wd
//   backward  dh = dy Wd^T,  dg = dh u a'(g),  du = dh a(g),  dx = [dg | du] Wgu^T,  dWgu = x^T [dg | du],  dWd = h^T dy
//
// Six products; the activation, its derivative and the product of gate and up happen where a product's sums still are in registers.
#include "activations.h"

namespace eck {
namespace {

// a(g) and a'(g)
struct Gate {
    float value, slope;
};
template <int ACT>
__device__ __forceinline__ Gate gate_of(float g)
{
    if (ACT == ECK_ACT_RELU) return {g > 0.0f ? g : g == g ? 0.0f : g, g > 0.0f ? 1.0f : 0.0f};
    if (ACT == ECK_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-g));
        return {g * s, s * (1.0f + g * (1.0f - s))};
    }
    const float s = 0.5f * (1.0f + erff(g * 0.70710678f));
    return {g * s, s + g * 0.39894228f * expf(-0.5f * g * g)};
}

// what becomes of element (m, c) of a product
enum { STORE, GATE, SLOPE };
template <class T>
struct Product {
    const T *a, *b;              // a(m, k) = a[m * am + k * ak], b(k, c) = b[k * bk + c * bc]
    uint64_t am, ak, bk, bc;
    uint64_t M, K;
    uint32_t C;
    uint64_t b_up;               // GATE: b of the up projection is this far behind the gate's
    T *out;                      // STORE: [M][ld_out]; GATE, SLOPE: h
    uint64_t ld_out;
    float *pre;                  // GATE: written where not NULL; SLOPE: read; [M][2 C]
    T *d_pre;                    // SLOPE: [M][ld_d]: dg, and du from column `half` on
    uint64_t ld_d, half;
    uint64_t tiles_c, tiles;
};

template <class T, int KIND, int ACT>
__global__ __launch_bounds__(256) void product_kernel(Product<T> p)
{
    constexpr int TILE = 32, KS = 16;
    __shared__ float a[KS][TILE + 1], b[KS][TILE + 1], b2[KS][TILE + 1];
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (uint64_t tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
        const uint64_t m0 = tile / p.tiles_c * TILE, c0 = tile % p.tiles_c * TILE;
        float s[2][2] = {}, s2[2][2] = {};
        for (uint64_t k0 = 0; k0 < p.K; k0 += KS) {
            for (int i = threadIdx.x; i < KS * TILE; i += 256) {
                const int k = i / TILE, j = i % TILE;
                a[k][j] = k0 + k < p.K && m0 + j < p.M ? (float)p.a[(m0 + j) * p.am + (k0 + k) * p.ak] : 0.0f;
                const bool in = k0 + k < p.K && c0 + j < p.C;
                b[k][j] = in ? (float)p.b[(k0 + k) * p.bk + (c0 + j) * p.bc] : 0.0f;
                if (KIND == GATE) b2[k][j] = in ? (float)p.b[p.b_up + (k0 + k) * p.bk + (c0 + j) * p.bc] : 0.0f;
            }
            __syncthreads();
            for (int k = 0; k < KS; ++k)
                for (int i = 0; i < 2; ++i)
                    for (int j = 0; j < 2; ++j) {
                        s[i][j] = fmaf(a[k][ty + 16 * i], b[k][tx + 16 * j], s[i][j]);
                        if (KIND == GATE) s2[i][j] = fmaf(a[k][ty + 16 * i], b2[k][tx + 16 * j], s2[i][j]);
                    }
            __syncthreads();
        }
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j) {
                const uint64_t m = m0 + ty + 16 * i, c = c0 + tx + 16 * j;
                if (m >= p.M || c >= p.C) continue;
                if (KIND == STORE) p.out[m * p.ld_out + c] = (T)s[i][j];
                if (KIND == GATE) {
                    p.out[m * p.ld_out + c] = (T)(gate_of<ACT>(s[i][j]).value * s2[i][j]);
                    if (p.pre) {
                        p.pre[m * 2 * p.C + c] = s[i][j];
                        p.pre[m * 2 * p.C + p.C + c] = s2[i][j];
                    }
                }
                if (KIND == SLOPE) {
                    const float u = p.pre[m * 2 * p.C + p.C + c];
                    const Gate gate = gate_of<ACT>(p.pre[m * 2 * p.C + c]);
                    p.out[m * p.ld_out + c] = (T)(gate.value * u);
                    p.d_pre[m * p.ld_d + c] = (T)(s[i][j] * u * gate.slope);
                    p.d_pre[m * p.ld_d + p.half + c] = (T)(s[i][j] * gate.value);
                }
            }
    }
}

template <class T, int KIND>
void launch(Product<T> p, int32_t act, hipStream_t st)
{
    p.tiles_c = ((uint64_t)p.C + 31) / 32;
    p.tiles = (p.M + 31) / 32 * p.tiles_c;
    auto kernel = KIND == STORE || act == ECK_ACT_SILU ? product_kernel<T, KIND, ECK_ACT_SILU>
                  : act == ECK_ACT_GELU                ? product_kernel<T, KIND, KIND == STORE ? ECK_ACT_SILU : ECK_ACT_GELU>
                                                       : product_kernel<T, KIND, KIND == STORE ? ECK_ACT_SILU : ECK_ACT_RELU>;
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(p.tiles < (1u << 20) ? p.tiles : (1u << 20))), dim3(256), 0, st, p);
}

uint64_t padded(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

template <class T>
int32_t forward(const T *x, uint64_t ld_x, uint64_t n, uint32_t n_in, uint32_t n_hidden, uint32_t n_out, const T *w_gate_up,
                const T *w_down, int32_t act, T *y, uint64_t ld_y, float *pre, void *ws, hipStream_t st)
{
    T *h = (T *)ws;
    Product<T> p = {};
    p.a = x, p.am = ld_x, p.ak = 1, p.b = w_gate_up, p.bk = 2ull * n_hidden, p.bc = 1, p.b_up = n_hidden;
    p.M = n, p.K = n_in, p.C = n_hidden, p.out = h, p.ld_out = n_hidden, p.pre = pre;
    launch<T, GATE>(p, act, st);
    p.a = h, p.am = n_hidden, p.b = w_down, p.bk = n_out, p.K = n_hidden, p.C = n_out, p.out = y, p.ld_out = ld_y;
    launch<T, STORE>(p, act, st);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

template <class T>
int32_t backward(const T *x, uint64_t ld_x, uint64_t n, uint32_t n_in, uint32_t n_hidden, uint32_t n_out, const T *w_gate_up,
                 const T *w_down, int32_t act, const float *pre, const T *dy, uint64_t ld_dy, T *dx, uint64_t ld_dx, T *dw_gate_up,
                 T *dw_down, void *ws, hipStream_t st)
{
    T *h = (T *)ws, *d_pre = (T *)((char *)ws + padded(n * n_hidden * sizeof(T)));
    Product<T> p = {};
    p.a = dy, p.am = ld_dy, p.ak = 1, p.b = w_down, p.bk = 1, p.bc = n_out, p.M = n, p.K = n_out, p.C = n_hidden;
    p.out = h, p.ld_out = n_hidden, p.pre = const_cast<float *>(pre), p.d_pre = d_pre, p.ld_d = 2ull * n_hidden, p.half = n_hidden;
    launch<T, SLOPE>(p, act, st);
    if (dx) {
        p.a = d_pre, p.am = 2ull * n_hidden, p.ak = 1, p.b = w_gate_up, p.bk = 1, p.bc = 2ull * n_hidden;
        p.M = n, p.K = 2ull * n_hidden, p.C = n_in, p.out = dx, p.ld_out = ld_dx;
        launch<T, STORE>(p, act, st);
    }
    if (dw_gate_up) {
        p.a = x, p.am = 1, p.ak = ld_x, p.b = d_pre, p.bk = 2ull * n_hidden, p.bc = 1;
        p.M = n_in, p.K = n, p.C = 2 * n_hidden, p.out = dw_gate_up, p.ld_out = 2ull * n_hidden;
        launch<T, STORE>(p, act, st);
    }
    if (dw_down) {
        p.a = h, p.am = 1, p.ak = n_hidden, p.b = dy, p.bk = ld_dy, p.bc = 1;
        p.M = n_hidden, p.K = n, p.C = n_out, p.out = dw_down, p.ld_out = n_out;
        launch<T, STORE>(p, act, st);
    }
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

bool sizes_ok(uint64_t n, uint32_t n_in, uint32_t n_hidden, uint32_t n_out)
{
    return n <= MAX_ROWS && n_in <= MAX_WIDTH && n_hidden <= MAX_WIDTH && n_out <= MAX_WIDTH;
}

} // namespace
} // namespace eck

using namespace eck;

extern "C" uint64_t gatedffn_forward_workspace_bytes(uint64_t n, uint32_t n_in, uint32_t n_hidden, uint32_t n_out, int32_t dtype)
{
    if (n == 0 || n_in == 0 || n_hidden == 0 || n_out == 0 || !is_dtype(dtype) || !sizes_ok(n, n_in, n_hidden, n_out)) return 0;
    return padded(n * n_hidden * element_bytes(dtype));
}

extern "C" int32_t gatedffn_forward(const void *x, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t n_in, uint32_t n_hidden,
                                    uint32_t n_out, const void *w_gate_up, const void *w_down, int32_t act, void *y, uint64_t ld_y,
                                    float *pre_out, void *ws, uint64_t ws_bytes, void *stream)
{
    if (!x || !w_gate_up || !w_down || !y || n == 0 || n_in == 0 || n_hidden == 0 || n_out == 0 || !is_dtype(dtype)) return ECK_EINVAL;
    if (act != ECK_ACT_SILU && act != ECK_ACT_GELU && act != ECK_ACT_RELU) return ECK_EINVAL;
    if (ld_x < n_in || ld_y < n_out) return ECK_ESHAPE;
    if (!sizes_ok(n, n_in, n_hidden, n_out)) return ECK_EUNSUPPORTED;
    if (!ws || ws_bytes < gatedffn_forward_workspace_bytes(n, n_in, n_hidden, n_out, dtype)) return ECK_EWORKSPACE;
    const uint64_t size = element_bytes(dtype);
    if (!aligned(x, size) || !aligned(w_gate_up, size) || !aligned(w_down, size) || !aligned(y, size) || !aligned(pre_out, 4) || !aligned(ws, 256))
        return ECK_EALIGN;
    if (dtype == ECK_F32)
        return forward<float>((const float *)x, ld_x, n, n_in, n_hidden, n_out, (const float *)w_gate_up, (const float *)w_down, act, (float *)y,
                              ld_y, pre_out, ws, as_stream(stream));
    return forward<bf16>((const bf16 *)x, ld_x, n, n_in, n_hidden, n_out, (const bf16 *)w_gate_up, (const bf16 *)w_down, act, (bf16 *)y, ld_y,
                         pre_out, ws, as_stream(stream));
}

extern "C" uint64_t gatedffn_backward_workspace_bytes(uint64_t n, uint32_t n_in, uint32_t n_hidden, uint32_t n_out, int32_t dtype)
{
    if (n == 0 || n_in == 0 || n_hidden == 0 || n_out == 0 || !is_dtype(dtype) || !sizes_ok(n, n_in, n_hidden, n_out)) return 0;
    return padded(n * n_hidden * element_bytes(dtype)) + padded(2 * n * n_hidden * element_bytes(dtype));
}

extern "C" int32_t gatedffn_backward(const void *x, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t n_in, uint32_t n_hidden,
                                     uint32_t n_out, const void *w_gate_up, const void *w_down, int32_t act, const float *pre,
                                     const void *dy, uint64_t ld_dy, void *dx_out, uint64_t ld_dx, void *dw_gate_up_out, void *dw_down_out,
                                     void *ws, uint64_t ws_bytes, void *stream)
{
    if (!x || !w_gate_up || !w_down || !pre || !dy || n == 0 || n_in == 0 || n_hidden == 0 || n_out == 0 || !is_dtype(dtype)) return ECK_EINVAL;
    if ((!dx_out && !dw_gate_up_out && !dw_down_out) || (act != ECK_ACT_SILU && act != ECK_ACT_GELU && act != ECK_ACT_RELU)) return ECK_EINVAL;
    if (ld_x < n_in || ld_dy < n_out || (dx_out && ld_dx < n_in)) return ECK_ESHAPE;
    if (!sizes_ok(n, n_in, n_hidden, n_out)) return ECK_EUNSUPPORTED;
    if (!ws || ws_bytes < gatedffn_backward_workspace_bytes(n, n_in, n_hidden, n_out, dtype)) return ECK_EWORKSPACE;
    const uint64_t size = element_bytes(dtype);
    if (!aligned(x, size) || !aligned(w_gate_up, size) || !aligned(w_down, size) || !aligned(pre, 4) || !aligned(dy, size) ||
        !aligned(dx_out, size) || !aligned(dw_gate_up_out, size) || !aligned(dw_down_out, size) || !aligned(ws, 256))
        return ECK_EALIGN;
    if (dtype == ECK_F32)
        return backward<float>((const float *)x, ld_x, n, n_in, n_hidden, n_out, (const float *)w_gate_up, (const float *)w_down, act, pre,
                               (const float *)dy, ld_dy, (float *)dx_out, ld_dx, (float *)dw_gate_up_out, (float *)dw_down_out, ws,
                               as_stream(stream));
    return backward<bf16>((const bf16 *)x, ld_x, n, n_in, n_hidden, n_out, (const bf16 *)w_gate_up, (const bf16 *)w_down, act, pre,
                          (const bf16 *)dy, ld_dy, (bf16 *)dx_out, ld_dx, (bf16 *)dw_gate_up_out, (bf16 *)dw_down_out, ws,
                          as_stream(stream));
}
