// A step of AdamW over many tensors, with states of 32 bits or of 8, and the norm of their gradients (HIP, gfx950).
//
//   g = s grad,  m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g g,
//   w <- w (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
//
// Everything is read and written once, so memory bounds it: 100.7 million parameters with bf16 gradients and copies, 2.82 GB, take 534 us
// (5.3 TB/s; a copy of 1 GiB 5.1), 96 million with 8-bit states, 1.54 GB, 315 (4.9 TB/s; the states' arithmetic takes nearly as long as their
// way).  The tensors' addresses travel as kernel arguments, so that a step needs no
// table on the device and a captured one holds its own; arguments are not free, so a launch has room for 12, 48 or 200 tensors, whichever does
// (steps of 12, 48, 49 and 200 tensors of 1024 elements: 5.1, 5.5, 5.7 and 6.1 us; of 16 384 elements 5.2, 7.4, 7.6 and 15.5).  Blocks of
// threads take stretches of a tensor.
//
// 8-bit states.  m is held in e4m3 and v in e5m2, each with a power of two for every 128 elements that brings the largest into
// [2^7, 2^8) and [2^14, 2^15): steps of at most an eighth and a quarter of a number, down to 2^-17 and 2^-31 of the block's largest.
// A step moves v by a thousandth, so rounding to nearest would leave it where it is for ever; it is rounded up with the probability of
// what is missing (16-bit draws of the generator of the genes), which is right on average.  A positive v never becomes 0, since m / eps
// would be the next step's size.  The step itself is made with m and v before they are rounded.
#include "activations.h"
#include "lanes.h"
#include "splitmix.h"

#include <math.h>

#include <type_traits>

namespace eck {
namespace {

constexpr uint32_t THREADS = 256, EACH = 4;          // elements of a thread at a time: 32 lanes share an 8-bit block
constexpr uint32_t ROUND = THREADS * EACH;           // of a block of threads at a time
constexpr uint64_t MOST_ELEMENTS = 1ull << 34, MOST_BLOCKS = (1u << 24) - 1; // (a launch has less than 2^32 threads)
static_assert(ECK_STATE_BLOCK == 32 * EACH, "a block of an 8-bit state is half a wavefront's");

template <bool EIGHT>
struct Tensor;
template <>
struct Tensor<false> {
    float *param;
    const void *grad;
    void *m, *v;
    bf16 *copy;
    uint64_t n;
    uint32_t first; // block of threads that starts it
    float keep;     // 1 - lr decay
};
template <>
struct Tensor<true> {
    float *param;
    const void *grad;
    void *m, *v;
    bf16 *copy;
    uint64_t n;
    uint32_t first;
    float keep;
    uint8_t *m_scale, *v_scale;
    uint64_t number; // of the first element, for the draws
};
constexpr uint64_t OF_BF16 = 1ull << 63; // the highest bit of a number of elements: gradients of bf16
struct Step {
    float beta1, beta2, one_beta1, one_beta2, eps, rate, inverse; // rate: lr / (1 - b1^t); inverse: 1 / (1 - b2^t)
    double lr, beta1_wide, beta2_wide;
    uint64_t seed, state;
    uint32_t t;
    const uint32_t *more;    // or NULL: rate, inverse and state are those of t
    const float *grad_scale; // or NULL: 1
};
// arguments of one launch
template <bool EIGHT, int ROOM>
struct Tensors {
    Step step;
    uint32_t count, rounds; // rounds: of a block of threads
    Tensor<EIGHT> one[ROOM];
};

// which tensor a block of threads works on: the last whose first block, first(i), is not behind it
template <class F>
__device__ __forceinline__ uint32_t tensor_of(uint32_t count, uint32_t block, F &&first)
{
    uint32_t lo = 0, hi = count;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (first(mid) <= block) lo = mid;
        else hi = mid;
    }
    return lo;
}

// the largest of 32 lanes' values, none of them negative or NaN
__device__ __forceinline__ float half_most(float v)
{
    uint32_t bits = __float_as_uint(v);
#pragma unroll
    for (int stride = 1; stride < 32; stride <<= 1) bits = max(bits, lane_exchange(bits, stride));
    return __uint_as_float(bits);
}

template <class T>
__device__ __forceinline__ void fetch(const T *from, uint64_t at, uint64_t n, T (&x)[EACH])
{
    if (at + EACH <= n) {
        const Chunk<T, EACH> c = *reinterpret_cast<const Chunk<T, EACH> *>(from + at);
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) x[i] = c.v[i];
    } else {
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) x[i] = at + i < n ? from[at + i] : (T)0;
    }
}
template <class T>
__device__ __forceinline__ void put(T *to, uint64_t at, uint64_t n, const T (&x)[EACH])
{
    if (at + EACH <= n) {
        Chunk<T, EACH> c;
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) c.v[i] = x[i];
        *reinterpret_cast<Chunk<T, EACH> *>(to + at) = c;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i)
            if (at + i < n) to[at + i] = x[i];
    }
}

__device__ __forceinline__ float power_of_two(int exponent) { return __uint_as_float((uint32_t)(exponent + 127) << 23); }

// An 8-bit state of EACH elements a thread.  FRACTION bits: 3 (e4m3, signed) or 2 (e5m2, never negative)
template <int FRACTION>
struct Eight {
    static constexpr int TOP = FRACTION == 3 ? 7 : 14, LOW = FRACTION == 3 ? -6 : -14, DROP = 23 - FRACTION;

    static __device__ __forceinline__ void decode(const uint8_t (&code)[EACH], uint8_t scale, float (&x)[EACH])
    {
        const float power = __uint_as_float((uint32_t)scale << 23);
        const int word = code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24;
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        f32x2 lo, hi;
        if (FRACTION == 3) {
            lo = __builtin_amdgcn_cvt_pk_f32_fp8(word, false);
            hi = __builtin_amdgcn_cvt_pk_f32_fp8(word, true);
        } else {
            lo = __builtin_amdgcn_cvt_pk_f32_bf8(word, false);
            hi = __builtin_amdgcn_cvt_pk_f32_bf8(word, true);
        }
        x[0] = lo[0] * power, x[1] = lo[1] * power, x[2] = hi[0] * power, x[3] = hi[1] * power;
    }
    // draws: 16 bits for each element.  Numbers that are not finite become NaN and count nothing in the block's power of two.
    static __device__ __forceinline__ uint8_t encode(const float (&x)[EACH], const uint32_t (&draw)[EACH], uint8_t (&code)[EACH])
    {
        float most = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) {
            const float size = __builtin_fabsf(x[i]);
            most = fmaxf(most, size < __builtin_inff() ? size : 0.0f);
        }
        most = half_most(most);
        const int exponent = (int)(__float_as_uint(most) >> 23) - 127;
        const int power = max(exponent - TOP, -100);
        const float down = power_of_two(-power), least = power_of_two(LOW);
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) {
            const float y = x[i] * down, size = __builtin_fabsf(y);
            // below the normal numbers steps are of one size: those of [least, 2 least), where these are taken to
            const bool small = size < least;
            const uint32_t raised = __float_as_uint(small ? size + least : size) + (draw[i] << (DROP - 16));
            uint32_t c = (raised >> DROP) - ((uint32_t)(LOW + (small ? 127 : 126)) << FRACTION);
            if (FRACTION == 2) c = max(c, x[i] > 0.0f ? 1u : 0u);
            c = size < __builtin_inff() ? c : 0x7Fu;
            if (FRACTION == 3) c |= __float_as_uint(y) >> 24 & 0x80;
            code[i] = (uint8_t)c;
        }
        return (uint8_t)(power + 127);
    }
};

// what a thread holds of its tensor
template <bool EIGHT, class G>
struct Hold {
    typedef typename std::conditional<EIGHT, uint8_t, float>::type S;
    float w[EACH];
    G g[EACH];
    S m[EACH], v[EACH];
    uint8_t m_scale, v_scale;

    __device__ __forceinline__ void load(const Tensor<EIGHT> &t, uint64_t n, uint64_t at)
    {
        fetch(t.param, at, n, w);
        fetch((const G *)t.grad, at, n, g);
        fetch((const S *)t.m, at, n, m);
        fetch((const S *)t.v, at, n, v);
        if constexpr (EIGHT) {
            const bool there = at < n;
            m_scale = there ? t.m_scale[at / ECK_STATE_BLOCK] : 0;
            v_scale = there ? t.v_scale[at / ECK_STATE_BLOCK] : 0;
        }
    }
};

template <bool EIGHT, class G>
__device__ __forceinline__ void advance(const Tensor<EIGHT> &t, uint64_t n, uint64_t at, const Hold<EIGHT, G> &had, const Step &step, float rate, float inverse,
                                        float scale, uint64_t state)
{
    float w[EACH], m[EACH], v[EACH];
    if constexpr (EIGHT) {
        Eight<3>::decode(had.m, had.m_scale, m);
        Eight<2>::decode(had.v, had.v_scale, v);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) m[i] = had.m[i], v[i] = had.v[i];
    }
#pragma unroll
    for (uint32_t i = 0; i < EACH; ++i) {
        const float g = (float)had.g[i] * scale;
        // (32 bits: rounded where torch's elementwise operations round, so that refits made with those are repeated bit for bit.  8 bits:
        // without contraction, which any IEEE arithmetic repeats, as the borders between two of a format's numbers want it)
        if (EIGHT) {
            m[i] = m[i] * step.beta1 + g * step.one_beta1;
            v[i] = v[i] * step.beta2 + g * step.one_beta2 * g;
        } else {
            m[i] = fmaf(step.one_beta1, g, m[i] * step.beta1);
            v[i] = fmaf(step.one_beta2, g * g, v[i] * step.beta2);
        }
    }
    if (EIGHT && step.eps >= 0x1p-39f) {
        // (8 bits: root and quotient as the instructions give them, within a unit of the last place each; full ones are two dozen
        // instructions, and instructions bound this kernel.  They take numbers below 2^-126 for 0: of roots, which are below 2^-63, that is within a
        // rounding beside such an eps, but not beside a smaller one, with which the smallest gradients' steps would be infinite)
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i)
            w[i] = fmaf(-rate, m[i] * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[i] * inverse) + step.eps), had.w[i] * t.keep);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) w[i] = fmaf(-rate, m[i] / (sqrtf(v[i] * inverse) + step.eps), had.w[i] * t.keep);
    }
    put(t.param, at, n, w);
    if (t.copy) {
        bf16 c[EACH];
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) c[i] = (bf16)w[i];
        put(t.copy, at, n, c);
    }
    if constexpr (EIGHT) {
        uint32_t for_m[EACH], for_v[EACH];
        const uint64_t number = (t.number + at) / 2;
#pragma unroll
        for (uint32_t i = 0; i < EACH; i += 2) {
            const uint64_t u = splitmix_finalise(state + kGamma * (number + i / 2 + 1));
            for_m[i] = (uint32_t)u & 0xFFFF, for_v[i] = (uint32_t)u >> 16;
            for_m[i + 1] = (uint32_t)(u >> 32) & 0xFFFF, for_v[i + 1] = (uint32_t)(u >> 48);
        }
        // (elements past the end are zeros with zero gradients: they count nothing)
        uint8_t code_m[EACH], code_v[EACH];
        const uint8_t scale_m = Eight<3>::encode(m, for_m, code_m), scale_v = Eight<2>::encode(v, for_v, code_v);
        put((uint8_t *)t.m, at, n, code_m);
        put((uint8_t *)t.v, at, n, code_v);
        if (at % ECK_STATE_BLOCK == 0 && at < n) {
            t.m_scale[at / ECK_STATE_BLOCK] = scale_m;
            t.v_scale[at / ECK_STATE_BLOCK] = scale_v;
        }
    } else {
        put((float *)t.m, at, n, m);
        put((float *)t.v, at, n, v);
    }
}

template <bool EIGHT, class G>
__device__ __forceinline__ void work(const Tensor<EIGHT> &t, uint64_t n, uint32_t block, uint32_t rounds, const Step &step, float rate,
                                     float inverse, float scale, uint64_t state)
{
    const uint64_t first = (uint64_t)block * rounds * ROUND + threadIdx.x * EACH;
    // (whole wavefronts stay together: 8-bit blocks are exchanged between lanes)
    for (uint32_t r = 0; r < rounds && first - threadIdx.x * EACH + r * ROUND < n; ++r) {
        const uint64_t at = first + r * ROUND;
        Hold<EIGHT, G> had;
        had.load(t, n, at);
        advance<EIGHT, G>(t, n, at, had, step, rate, inverse, scale, state);
    }
}

template <bool EIGHT, int ROOM>
__global__ __launch_bounds__(THREADS) void adamw_kernel(const Tensors<EIGHT, ROOM> a)
{
    const Tensor<EIGHT> &t = a.one[tensor_of(a.count, blockIdx.x, [&](uint32_t i) { return a.one[i].first; })];
    const float scale = a.step.grad_scale ? *a.step.grad_scale : 1.0f;
    if (!(__builtin_fabsf(scale) < __builtin_inff())) return; // gradients that are not finite: nothing changes
    float rate = a.step.rate, inverse = a.step.inverse;
    uint64_t state = a.step.state;
    if (a.step.more) {
        const uint32_t now = a.step.t + *a.step.more;
        if (now == 0) return; // (there is no step before the first)
        double power1 = 1.0, power2 = 1.0, square1 = a.step.beta1_wide, square2 = a.step.beta2_wide;
        for (uint32_t k = now; k; k >>= 1) {
            if (k & 1) {
                power1 *= square1;
                power2 *= square2;
            }
            square1 *= square1;
            square2 *= square2;
        }
        rate = (float)(a.step.lr / (1.0 - power1));
        inverse = (float)(1.0 / (1.0 - power2));
        state = splitmix_finalise(a.step.seed + kGamma * ((uint64_t)now + 1));
    }
    const uint32_t block = blockIdx.x - t.first;
    const uint64_t n = t.n & ~OF_BF16;
    if (t.n & OF_BF16) work<EIGHT, bf16>(t, n, block, a.rounds, a.step, rate, inverse, scale, state);
    else work<EIGHT, float>(t, n, block, a.rounds, a.step, rate, inverse, scale, state);
}

// ------------------------------------------------------------------------------------------------ norm

// Sums of squares of stretches of tensors, a block of threads each, then one block adds them up in a fixed order.  Memory bounds the first
// (37.3 million bf16 gradients in 194 tensors: 16 us for 74.6 MB), the launches themselves small lists (18 us for these, 9 for 99 thousand in ten)
template <int ROOM>
struct GradientList {
    double *sums;
    uint32_t count, stretch; // stretch: elements of a block of threads, a multiple of THREADS * 8
    const void *grad[ROOM];
    uint64_t n[ROOM];
    uint32_t first[ROOM];
};

__device__ __forceinline__ double block_sum(double x, double *lds)
{
#pragma unroll
    for (int stride = 1; stride < 64; stride <<= 1) x += lane_exchange(x, stride);
    const uint32_t waves = blockDim.x / 64;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0.0;
    for (uint32_t w = 0; w < waves; ++w) x += lds[w];
    return x;
}

// squares are exact and summed in 64 bits: no gradient is too large or too small for them
template <class G>
__device__ __forceinline__ double squares(const G *grad, uint64_t from, uint64_t to)
{
    constexpr int AHEAD = 4, N = Chunk<G>::N;
    double sum = 0.0;
    for (uint64_t at = from + threadIdx.x * 8; at < to; at += THREADS * 8 * AHEAD) {
        Chunk<G> c[AHEAD][8 / N];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const uint64_t here = at + (uint64_t)k * (THREADS * 8);
#pragma unroll
            for (int i = 0; i < 8 / N; ++i) {
                if (here + (i + 1) * N <= to) c[k][i] = *reinterpret_cast<const Chunk<G> *>(grad + here + i * N);
                else
#pragma unroll
                    for (int j = 0; j < N; ++j) c[k][i].v[j] = here + i * N + j < to ? grad[here + i * N + j] : (G)0.0f;
            }
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int i = 0; i < 8 / N; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const double x = (double)(float)c[k][i].v[j];
                    sum += x * x;
                }
    }
    return sum;
}

template <int ROOM>
__global__ __launch_bounds__(THREADS) void squares_kernel(const GradientList<ROOM> a)
{
    __shared__ double lds[THREADS / 64];
    const uint32_t t = tensor_of(a.count, blockIdx.x, [&](uint32_t i) { return a.first[i]; });
    const uint64_t n = a.n[t] & ~OF_BF16, from = (uint64_t)(blockIdx.x - a.first[t]) * a.stretch, to = min(n, from + a.stretch);
    const double sum = a.n[t] & OF_BF16 ? squares((const bf16 *)a.grad[t], from, to) : squares((const float *)a.grad[t], from, to);
    const double all = block_sum(sum, lds);
    if (threadIdx.x == 0) a.sums[blockIdx.x] = all;
}

__global__ __launch_bounds__(1024) void norm_kernel(const double *sums, uint32_t count, float max_norm, float *norm_out, float *scale_out)
{
    __shared__ double lds[16];
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < count; i += 1024) sum += sums[i];
    const double norm = sqrt(block_sum(sum, lds));
    if (threadIdx.x != 0) return;
    if (norm_out) *norm_out = (float)norm;
    if (scale_out) *scale_out = !(norm < __builtin_inf()) ? __builtin_nanf("") : norm > max_norm ? (float)(max_norm / norm) : 1.0f;
}

// ------------------------------------------------------------------------------------------------ host

uint64_t gradient_bytes(int32_t dtype) { return dtype == ECK_F32 ? 4 : 2; }

// what both calls want of their list
int32_t check_list(const eck_parameter *p, uint32_t count, bool norm)
{
    if (!p || count == 0) return ECK_EINVAL;
    bool some = false;
    for (uint32_t i = 0; i < count; ++i) {
        if (!is_dtype(p[i].grad_dtype)) return ECK_EINVAL;
        if (p[i].n == 0) continue;
        some = true;
        if (!p[i].grad || (!norm && (!p[i].param || !p[i].m || !p[i].v))) return ECK_EINVAL;
        if (p[i].n > MOST_ELEMENTS) return ECK_EUNSUPPORTED;
        if (!aligned(p[i].grad, gradient_bytes(p[i].grad_dtype))) return ECK_EALIGN;
    }
    return some ? ECK_OK : ECK_EINVAL;
}

// elements of one block of threads, and blocks of all, in a norm of that list: at most 16384 and one for each tensor
uint64_t norm_stretch(const eck_parameter *p, uint32_t count)
{
    uint64_t total = 0;
    for (uint32_t i = 0; i < count; ++i) total += p[i].n;
    const uint64_t unit = THREADS * 8;
    return ((total + 16383) / 16384 + 4 * unit - 1) / (4 * unit) * (4 * unit);
}
uint64_t norm_blocks(const eck_parameter *p, uint32_t count, uint64_t stretch)
{
    uint64_t blocks = 0;
    for (uint32_t i = 0; i < count; ++i) blocks += (p[i].n + stretch - 1) / stretch;
    return blocks;
}

// tensors from `from` on, as many as there is room for, in one launch; advances `from` and the elements' number
template <bool EIGHT, int ROOM>
int32_t step_some(const eck_parameter *p, uint32_t count, uint32_t &from, uint64_t &number, const Step &step, hipStream_t st)
{
    Tensors<EIGHT, ROOM> a;
    a.step = step;
    a.count = 0;
    a.rounds = 2;
    uint64_t blocks = 0;
    for (; from < count && a.count < ROOM; ++from) {
        const eck_parameter &t = p[from];
        if (t.n == 0) continue;
        const uint64_t mine = (t.n + a.rounds * ROUND - 1) / (a.rounds * ROUND);
        if (blocks + mine > MOST_BLOCKS) break;
        Tensor<EIGHT> &to = a.one[a.count++];
        to.param = t.param, to.grad = t.grad, to.m = t.m, to.v = t.v, to.copy = (bf16 *)t.bf16_out;
        to.n = t.n | (t.grad_dtype == ECK_BF16 ? OF_BF16 : 0);
        to.first = (uint32_t)blocks;
        to.keep = (float)(1.0 - step.lr * t.weight_decay);
        if constexpr (EIGHT) to.m_scale = t.m_scale, to.v_scale = t.v_scale, to.number = number;
        blocks += mine;
        number += (t.n + ECK_STATE_BLOCK - 1) / ECK_STATE_BLOCK * ECK_STATE_BLOCK;
    }
    if (a.count == 0) return ECK_OK;
    hipLaunchKernelGGL((adamw_kernel<EIGHT, ROOM>), dim3((uint32_t)blocks), dim3(THREADS), 0, st, a);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}
template <bool EIGHT>
int32_t step_all(const eck_parameter *p, uint32_t count, const Step &step, hipStream_t st)
{
    uint64_t number = 0;
    for (uint32_t from = 0; from < count;) {
        const uint32_t left = count - from;
        const int32_t rc = left <= 12   ? step_some<EIGHT, 12>(p, count, from, number, step, st)
                           : left <= 48 ? step_some<EIGHT, 48>(p, count, from, number, step, st)
                                        : step_some<EIGHT, 200>(p, count, from, number, step, st);
        if (rc) return rc;
    }
    return ECK_OK;
}

template <int ROOM>
int32_t squares_of_some(const eck_parameter *p, uint32_t count, uint32_t &from, double *&sums, uint64_t stretch, hipStream_t st)
{
    GradientList<ROOM> a;
    a.sums = sums;
    a.count = 0;
    a.stretch = (uint32_t)stretch;
    uint64_t blocks = 0;
    for (; from < count && a.count < ROOM; ++from) {
        const eck_parameter &t = p[from];
        if (t.n == 0) continue;
        a.grad[a.count] = t.grad;
        a.n[a.count] = t.n | (t.grad_dtype == ECK_BF16 ? OF_BF16 : 0);
        a.first[a.count++] = (uint32_t)blocks;
        blocks += (t.n + stretch - 1) / stretch;
    }
    if (a.count == 0) return ECK_OK;
    hipLaunchKernelGGL(squares_kernel<ROOM>, dim3((uint32_t)blocks), dim3(THREADS), 0, st, a);
    ECK_HIP_TRY(hipGetLastError());
    sums += blocks;
    return ECK_OK;
}

} // namespace
} // namespace eck

using namespace eck;

extern "C" int32_t adamw_step(const eck_parameter *parameters, uint32_t count, int32_t state, double lr, double beta1, double beta2, double eps,
                              uint32_t step, const uint32_t *step_more, const float *grad_scale, uint64_t seed, void *stream)
{
    if (state != ECK_STATE_F32 && state != ECK_STATE_8BIT) return ECK_EINVAL;
    if (!(lr >= 0.0 && lr <= 3e38) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0 && eps <= 3e38)) return ECK_EINVAL;
    if (step == 0 && !step_more) return ECK_EINVAL;
    if (const int32_t rc = check_list(parameters, count, false)) return rc;
    const bool eight = state == ECK_STATE_8BIT;
    for (uint32_t i = 0; i < count; ++i) {
        const eck_parameter &p = parameters[i];
        if (p.n == 0) continue;
        if (!(p.weight_decay >= 0.0f && p.weight_decay <= 3e38f) || (eight && (!p.m_scale || !p.v_scale))) return ECK_EINVAL;
        if (!aligned(p.param, 4) || !aligned(p.bf16_out, 2) || (!eight && (!aligned(p.m, 4) || !aligned(p.v, 4)))) return ECK_EALIGN;
    }
    if (!aligned(step_more, 4) || !aligned(grad_scale, 4)) return ECK_EALIGN;

    Step of = {(float)beta1, (float)beta2, (float)(1.0 - beta1), (float)(1.0 - beta2), (float)eps, 0.0f, 0.0f, lr, beta1, beta2, seed, 0, step,
               step_more, grad_scale};
    if (!step_more) {
        of.rate = (float)(lr / (1.0 - pow(beta1, step)));
        of.inverse = (float)(1.0 / (1.0 - pow(beta2, step)));
        of.state = stream_state(seed, step);
    }
    if (eight) return step_all<true>(parameters, count, of, as_stream(stream));
    return step_all<false>(parameters, count, of, as_stream(stream));
}

extern "C" uint64_t gradients_norm_workspace_bytes(const eck_parameter *parameters, uint32_t count)
{
    if (check_list(parameters, count, true)) return 0;
    return norm_blocks(parameters, count, norm_stretch(parameters, count)) * sizeof(double);
}

extern "C" int32_t gradients_norm(const eck_parameter *parameters, uint32_t count, float max_norm, float *norm_out, float *scale_out, void *ws,
                                  uint64_t ws_bytes, void *stream)
{
    if ((!norm_out && !scale_out) || !(max_norm > 0.0f)) return ECK_EINVAL;
    if (const int32_t rc = check_list(parameters, count, true)) return rc;
    const uint64_t stretch = norm_stretch(parameters, count), total = norm_blocks(parameters, count, stretch);
    if (stretch > 0x7FFFFFFF || total > MOST_BLOCKS) return ECK_EUNSUPPORTED;
    if (!ws || ws_bytes < total * sizeof(double)) return ECK_EWORKSPACE;
    if (!aligned(ws, 256) || !aligned(norm_out, 4) || !aligned(scale_out, 4)) return ECK_EALIGN;
    double *sums = (double *)ws;
    for (uint32_t from = 0; from < count;) {
        const uint32_t left = count - from;
        const int32_t rc = left <= 16   ? squares_of_some<16>(parameters, count, from, sums, stretch, as_stream(stream))
                           : left <= 64 ? squares_of_some<64>(parameters, count, from, sums, stretch, as_stream(stream))
                                        : squares_of_some<256>(parameters, count, from, sums, stretch, as_stream(stream));
        if (rc) return rc;
    }
    hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(1024), 0, as_stream(stream), (const double *)ws, (uint32_t)total, max_norm, norm_out, scale_out);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}
