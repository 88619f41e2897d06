// Selection by drawing: parents of the next generation from the predicted energies and given random numbers (HIP, gfx950).
//
// Candidate i of a segment has weight w = exp(-(E - E_min) / T).  In order of energy, equal ones by index, the kept are a prefix: the k
// least, of these the fewest that have the share top_p of their weight, of these the ones of weight min_p and more.  A draw u takes the
// first kept candidate, by index, at which the sum of weights passes u times all of it.
//
// Nothing is sorted.  The end of a prefix is found in a histogram of the energies' order keys over the range in question, count and weight
// of every bin, then again within the bin where the end lies, down to a single key: eleven bits at a time, three times at most.  Weights
// are 64-bit floating point, and in histograms whole multiples of 2^-60, held as two numbers of thirty bits, whose sums do not depend on
// the order in which the atomics come.  Of equal energies that the prefix ends among, the index of the last is found by counting.
#include "activations.h"

namespace eck {
namespace {

constexpr uint32_t BINS = 2048, BIN_BITS = 11, STRIPS = 1024, NO_KEY = 0xFFFFFFFFu;
constexpr uint64_t MOST_CANDIDATES = 1ull << 31;
constexpr uint32_t NOBODY = 0xFFFFFFFFu;

struct Draws {
    const float *energy;
    const uint8_t *legal;
    uint64_t n; // of a segment
    const float *uniform;
    uint32_t draws, k;
    double top_p, min_p, per_temperature;
    uint32_t *idx;
    float *logprob;
    uint32_t *count;
};

// order key of a candidate that may be drawn (finite and legal), equal for both zeros; NO_KEY of the others
__device__ __forceinline__ uint32_t key_of(float e, bool legal)
{
    return legal && __builtin_fabsf(e) < __builtin_inff() ? score_order_key(e + 0.0f) : NO_KEY;
}
__device__ __forceinline__ float energy_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
__device__ __forceinline__ double weight_of(uint32_t key, double least, double per_temperature)
{
    return exp(-((double)energy_of(key) - least) * per_temperature);
}

// a sum of weights: high * 2^-30 + low * 2^-60
struct Mass {
    uint64_t high, low;
    __device__ __forceinline__ double value() const { return (double)high * 0x1p-30 + (double)low * 0x1p-60; }
    __device__ __forceinline__ Mass operator+(const Mass &o) const { return {high + o.high, low + o.low}; }
};
__device__ __forceinline__ Mass mass_of(double w)
{
    const double t = w * 0x1p30;
    const uint64_t high = (uint64_t)t;
    return {high, (uint64_t)((t - (double)high) * 0x1p30)};
}

// four candidates from `at` on, as keys
__device__ __forceinline__ void load_keys(const float *energy, const uint8_t *legal, uint64_t at, uint64_t n, uint32_t (&key)[4])
{
    if (at + 4 <= n) {
        const Chunk<float, 4> e = *reinterpret_cast<const Chunk<float, 4> *>(energy + at);
        Chunk<uint8_t, 4> l;
        if (legal) l = *reinterpret_cast<const Chunk<uint8_t, 4> *>(legal + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) key[i] = key_of(e.v[i], !legal || l.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) key[i] = at + i < n ? key_of(energy[at + i], !legal || legal[at + i]) : NO_KEY;
    }
}

// ------------------------------------------------------------------------------------------------ blocks

// sums over a block's threads up to and including each
template <int THREADS, class V>
__device__ __forceinline__ V block_prefix(V v, V *of_waves)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64;
#pragma unroll
    for (int stride = 1; stride < 64; stride <<= 1) {
        const V other = __shfl_up(v, stride);
        if ((int)lane >= stride) v += other;
    }
    __syncthreads(); // (of_waves may still be read from the last time)
    if (lane == 63) of_waves[wave] = v;
    __syncthreads();
    V before = 0;
    for (uint32_t w = 0; w < wave; ++w) before += of_waves[w];
    return before + v;
}

struct Histogram {
    uint32_t count[BINS];
    unsigned long long high[BINS], low[BINS];
};

// where a prefix ends: with `kept` of the candidates of this key, of which there are `all`
struct End {
    uint32_t key, kept, all;
};

struct Search {
    uint32_t lo, hi;     // keys in question
    uint32_t shift;
    uint32_t before;     // candidates below lo, and their weight
    Mass mass;
};
__device__ __forceinline__ uint32_t shift_for(uint32_t lo, uint32_t hi)
{
    const int bits = 32 - __builtin_clz((hi - lo) | 1);
    return bits > (int)BIN_BITS ? bits - BIN_BITS : 0;
}

template <int THREADS>
struct Shared {
    Histogram bins;
    uint32_t small[THREADS / 64];
    unsigned long long wide[2][THREADS / 64];
    double real[THREADS / 64];
    Search found;
    uint32_t number, least, most;
    double sums[STRIPS], sums_to[STRIPS]; // of strips, and up to and including each
    uint32_t counts[STRIPS];
};

template <int THREADS>
__device__ __forceinline__ void clear_bins(Shared<THREADS> &s, bool weights)
{
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < BINS; b += THREADS) {
        s.bins.count[b] = 0;
        if (weights) s.bins.high[b] = s.bins.low[b] = 0;
    }
    __syncthreads();
}

__device__ __forceinline__ void add_to_bins(Histogram &bins, uint32_t bin, const double *weight)
{
    atomicAdd(&bins.count[bin], 1u);
    if (weight) {
        const Mass m = mass_of(*weight);
        atomicAdd(&bins.high[bin], (unsigned long long)m.high);
        atomicAdd(&bins.low[bin], (unsigned long long)m.low);
    }
}

// The bin where the prefix of `need` candidates (or, by weight, of `target`) ends, and the search within it.  `weights`: whether the bins
// hold weights
template <int THREADS>
__device__ __forceinline__ void narrow(Shared<THREADS> &s, Search &at, bool by_weight, uint32_t need, double target, bool weights)
{
    constexpr uint32_t EACH = BINS / THREADS;
    uint32_t count = 0;
    Mass mass = {0, 0};
    for (uint32_t i = 0; i < EACH; ++i) {
        const uint32_t b = threadIdx.x * EACH + i;
        count += s.bins.count[b];
        if (weights) mass = mass + Mass{s.bins.high[b], s.bins.low[b]};
    }
    const uint32_t count_to = block_prefix<THREADS>(count, s.small);
    Mass mass_to = {0, 0};
    if (weights) mass_to = {block_prefix<THREADS>((unsigned long long)mass.high, s.wide[0]), block_prefix<THREADS>((unsigned long long)mass.low, s.wide[1])};
    // up to the last bin, whatever roundings say
    uint32_t before = at.before + count_to - count;
    Mass mass_before = {at.mass.high + mass_to.high - mass.high, at.mass.low + mass_to.low - mass.low};
    const auto reached = [&](uint32_t c, const Mass &m) { return by_weight ? m.value() >= target : c >= need; };
    const bool mine = !reached(before, mass_before) && reached(before + count, mass_before + mass);
    __syncthreads();
    if (mine || (threadIdx.x == 0 && reached(before, mass_before))) {
        uint32_t b = threadIdx.x * EACH;
        for (; b < threadIdx.x * EACH + EACH - 1; ++b) {
            const uint32_t c = s.bins.count[b];
            const Mass m = weights ? Mass{s.bins.high[b], s.bins.low[b]} : Mass{0, 0};
            if (reached(before + c, mass_before + m)) break;
            before += c;
            mass_before = mass_before + m;
        }
        Search next;
        next.lo = at.lo + (b << at.shift);
        next.hi = min(at.hi, next.lo + ((1u << at.shift) - 1));
        next.before = before;
        next.mass = mass_before;
        next.shift = shift_for(next.lo, next.hi);
        s.found = next;
        s.number = s.bins.count[b];
    }
    __syncthreads();
}

// how many of `all` candidates of weight w each, behind `before`, it takes to `target`
__device__ __forceinline__ uint32_t enough(double before, double w, uint32_t all, double target)
{
    if (!(w > 0.0)) return all;
    double j = ceil((target - before) / w);
    j = fmin(fmax(j, 1.0), (double)all);
    while (j > 1.0 && before + (j - 1.0) * w >= target) j -= 1.0;
    while (j < (double)all && before + j * w < target) j += 1.0;
    return (uint32_t)j;
}

// A block a segment.  HELD: its keys stay in registers, sixteen a thread
template <int THREADS, bool HELD>
__global__ __launch_bounds__(THREADS) void segment_kernel(const Draws a)
{
    __shared__ Shared<THREADS> s;
    const uint64_t n = a.n;
    const float *energy = a.energy + blockIdx.x * n;
    const uint8_t *legal = a.legal ? a.legal + blockIdx.x * n : nullptr;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, waves = THREADS / 64;

    constexpr int HOLD = HELD ? 4 : 1;
    uint32_t held[HOLD][4];
    if (HELD)
#pragma unroll
        for (int h = 0; h < HOLD; ++h) load_keys(energy, legal, ((uint64_t)h * THREADS + threadIdx.x) * 4, n, held[h]);
    const auto each = [&](auto &&f) { // of the candidates that may be drawn
        if (HELD) {
#pragma unroll
            for (int h = 0; h < HOLD; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (held[h][i] != NO_KEY) f(held[h][i]);
        } else {
            for (uint64_t at = threadIdx.x * 4; at < n; at += THREADS * 4) {
                uint32_t key[4];
                load_keys(energy, legal, at, n, key);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (key[i] != NO_KEY) f(key[i]);
            }
        }
    };

    // the range of keys
    if (threadIdx.x == 0) {
        s.least = NO_KEY;
        s.most = 0;
        s.number = 0;
    }
    __syncthreads();
    {
        uint32_t least = NO_KEY, most = 0, number = 0;
        each([&](uint32_t key) {
            least = min(least, key);
            most = max(most, key);
            ++number;
        });
#pragma unroll
        for (int stride = 1; stride < 64; stride <<= 1) {
            least = min(least, (uint32_t)__shfl_xor((int)least, stride));
            most = max(most, (uint32_t)__shfl_xor((int)most, stride));
            number += (uint32_t)__shfl_xor((int)number, stride);
        }
        if (lane == 0) {
            atomicMin(&s.least, least);
            atomicMax(&s.most, most);
            atomicAdd(&s.number, number);
        }
    }
    __syncthreads();
    const uint32_t number = s.number;
    const Search whole = {s.least, s.most, shift_for(s.least, s.most), 0, {0, 0}};
    uint32_t *const idx = a.idx + (uint64_t)blockIdx.x * a.draws;
    float *const logprob = a.logprob ? a.logprob + (uint64_t)blockIdx.x * a.draws : nullptr;
    if (number == 0) {
        for (uint32_t d = threadIdx.x; d < a.draws; d += THREADS) {
            idx[d] = NOBODY;
            if (logprob) logprob[d] = -__builtin_inff();
        }
        if (threadIdx.x == 0 && a.count) a.count[blockIdx.x] = 0;
        return;
    }
    const double least = (double)energy_of(whole.lo);

    const bool weights = a.top_p < 1.0;
    End end = {whole.hi, 1, 1};
    double total = 0.0; // of the k least
    const auto find = [&](bool by_weight, uint32_t need, double target) { // narrowed down to one key
        Search at = whole;
        at.hi = by_weight ? end.key : at.hi;
        at.shift = shift_for(at.lo, at.hi);
        for (int round = 0; round < 3; ++round) { // (32 bits, 21, 10)
            clear_bins(s, weights);
            each([&](uint32_t key) {
                if (key < at.lo || key > at.hi) return;
                const double w = weights ? weight_of(key, least, a.per_temperature) : 0.0;
                add_to_bins(s.bins, (key - at.lo) >> at.shift, weights ? &w : nullptr);
            });
            __syncthreads();
            narrow(s, at, by_weight, need, target, weights);
            const uint32_t shift = at.shift;
            at = s.found;
            if (shift == 0) break;
        }
        const uint32_t all = s.number;
        __syncthreads();
        end.key = at.lo;
        end.all = all;
        return at;
    };
    bool cut = false;
    if (a.k && a.k < number) {
        const Search at = find(false, a.k, 0.0);
        end.kept = a.k - at.before;
        cut = true;
        if (weights) {
            const Mass each_one = mass_of(weight_of(end.key, least, a.per_temperature));
            total = Mass{at.mass.high + end.kept * each_one.high, at.mass.low + end.kept * each_one.low}.value();
        }
    } else if (weights) {
        clear_bins(s, true);
        unsigned long long high = 0, low = 0;
        each([&](uint32_t key) {
            const Mass m = mass_of(weight_of(key, least, a.per_temperature));
            high += m.high;
            low += m.low;
        });
#pragma unroll
        for (int stride = 1; stride < 64; stride <<= 1) {
            high += __shfl_xor(high, stride);
            low += __shfl_xor(low, stride);
        }
        if (lane == 0) {
            atomicAdd(&s.bins.high[0], high);
            atomicAdd(&s.bins.low[0], low);
        }
        __syncthreads();
        total = Mass{s.bins.high[0], s.bins.low[0]}.value();
        __syncthreads();
    }
    if (weights) {
        const double target = a.top_p * total;
        const uint32_t at_most = cut ? end.kept : 0, key_most = end.key;
        const Search at = find(true, 0, target);
        uint32_t most = end.all;
        if (cut && end.key == key_most) most = at_most; // (of the k least's last ones)
        end.kept = enough(at.mass.value(), weight_of(end.key, least, a.per_temperature), most, target);
        cut = true;
    }

    // strips of candidates, a wavefront each at a time
    const uint64_t strip = (n + STRIPS - 1) / STRIPS <= 64 ? 64 : ((n + STRIPS - 1) / STRIPS + 63) / 64 * 64;
    const uint32_t strips = (uint32_t)((n + strip - 1) / strip);
    const auto key_at = [&](uint64_t i) { return i < n ? key_of(energy[i], !legal || legal[i]) : NO_KEY; };
    uint64_t last = n; // of the candidates of the last key, those before it stay
    if (cut && end.kept < end.all) {
        for (uint32_t t = wave; t < strips; t += waves) {
            uint32_t some = 0;
            for (uint64_t i = t * strip; i < min(n, (t + 1) * strip); i += 64) some += __builtin_popcountll(__ballot(key_at(i + lane) == end.key));
            if (lane == 0) s.counts[t] = some;
        }
        __syncthreads();
        if (wave == 0) {
            uint32_t left = end.kept;
            for (uint32_t t = 0; t < strips; t += 64) {
                const uint32_t mine = t + lane < strips ? s.counts[t + lane] : 0;
                uint32_t to = mine;
#pragma unroll
                for (int stride = 1; stride < 64; stride <<= 1) {
                    const uint32_t other = __shfl_up(to, stride);
                    if ((int)lane >= stride) to += other;
                }
                const uint64_t there = __ballot(to >= left);
                if (there == 0) {
                    left -= __shfl(to, 63);
                    continue;
                }
                const int l = __builtin_ctzll(there);
                left -= __shfl(to - mine, l);
                uint64_t i = (t + l) * strip;
                for (const uint64_t to_here = i + strip; i < to_here; i += 64) {
                    uint64_t equal = __ballot(key_at(i + lane) == end.key);
                    const uint32_t some = __builtin_popcountll(equal);
                    if (some < left) {
                        left -= some;
                        continue;
                    }
                    while (--left) equal &= equal - 1;
                    i += __builtin_ctzll(equal) + 1;
                    break;
                }
                if (lane == 0) {
                    s.found.lo = (uint32_t)i;
                    s.found.hi = (uint32_t)(i >> 32);
                }
                break;
            }
        }
        __syncthreads();
        last = (uint64_t)s.found.hi << 32 | s.found.lo;
    }
    const auto kept_weight = [&](uint64_t i, bool &kept) {
        const uint32_t key = key_at(i);
        kept = key < end.key || (key == end.key && i < last);
        if (!kept) return 0.0;
        const double w = weight_of(key, least, a.per_temperature);
        kept = w >= a.min_p;
        return kept ? w : 0.0;
    };

    for (uint32_t t = wave; t < STRIPS; t += waves) {
        double sum = 0.0;
        uint32_t some = 0;
        if (t < strips)
            for (uint64_t i = t * strip; i < min(n, (t + 1) * strip); i += 64) {
                bool kept;
                sum += kept_weight(i + lane, kept);
                some += __builtin_popcountll(__ballot(kept));
            }
#pragma unroll
        for (int stride = 1; stride < 64; stride <<= 1) sum += __shfl_xor(sum, stride);
        if (lane == 0) {
            s.sums[t] = sum;
            s.counts[t] = some;
        }
    }
    __syncthreads();
    // sums up to and including each strip
    {
        constexpr uint32_t EACH = STRIPS / THREADS;
        double to[EACH], sum = 0.0;
        uint32_t some = 0;
        for (uint32_t i = 0; i < EACH; ++i) {
            sum += s.sums[threadIdx.x * EACH + i];
            some += s.counts[threadIdx.x * EACH + i];
            to[i] = sum;
        }
        const double up_to = block_prefix<THREADS>(sum, s.real) - sum;
        const uint32_t all = block_prefix<THREADS>(some, s.small);
        for (uint32_t i = 0; i < EACH; ++i) s.sums_to[threadIdx.x * EACH + i] = up_to + to[i];
        if (threadIdx.x == THREADS - 1 && a.count) a.count[blockIdx.x] = all;
    }
    __syncthreads();
    const double of_all = s.sums_to[STRIPS - 1];
    for (uint32_t d = wave; d < a.draws; d += waves) {
        const double target = fmax((double)a.uniform[(uint64_t)blockIdx.x * a.draws + d] * of_all, 0.0);
        // the first strip that adds something and passes it, or the last that adds anything
        uint32_t t = STRIPS, last_one = 0;
        for (uint32_t t0 = 0; t0 < STRIPS; t0 += 64) {
            const bool some = s.sums[t0 + lane] > 0.0;
            const uint64_t passes = __ballot(some && s.sums_to[t0 + lane] > target), adds = __ballot(some);
            if (adds) last_one = t0 + 63 - __builtin_clzll(adds);
            if (passes) {
                t = t0 + __builtin_ctzll(passes);
                break;
            }
        }
        const bool past = t == STRIPS;
        if (past) t = last_one;
        double left = past ? __builtin_inf() : target - (t ? s.sums_to[t - 1] : 0.0), w_found = 0.0;
        uint64_t found = 0;
        for (uint64_t i = t * strip; i < min(n, (t + 1) * strip); i += 64) {
            bool kept;
            const double w = kept_weight(i + lane, kept);
            double to = w;
#pragma unroll
            for (int stride = 1; stride < 64; stride <<= 1) {
                const double other = __shfl_up(to, stride);
                if ((int)lane >= stride) to += other;
            }
            const uint64_t some = __ballot(w > 0.0), passes = __ballot(w > 0.0 && to > left);
            if (some) { // where roundings leave none that passes, the last
                const int l = passes ? __builtin_ctzll(passes) : 63 - __builtin_clzll(some);
                found = i + l;
                w_found = __shfl(w, l);
            }
            if (passes) break;
            left -= __shfl(to, 63);
        }
        if (lane == 0) {
            idx[d] = (uint32_t)found;
            if (logprob) logprob[d] = (float)log(w_found / of_all);
        }
    }
}

} // namespace
} // namespace eck

using namespace eck;

extern "C" uint64_t sample_select_workspace_bytes(uint64_t n, uint32_t n_segments, uint32_t draws)
{
    return 0;
}

extern "C" int32_t sample_select(const float *energy, const uint8_t *legal, uint64_t n, uint32_t n_segments, const float *uniform, uint32_t draws,
                                 float temperature, uint32_t k, float top_p, float min_p, uint32_t *idx_out, float *logprob_out,
                                 uint32_t *count_out, void *ws, uint64_t ws_bytes, void *stream)
{
    if (!energy || !uniform || !idx_out || n == 0 || n_segments == 0 || draws == 0) return ECK_EINVAL;
    if (!(temperature >= 0.0f && temperature < __builtin_inff()) || !(top_p > 0.0f && top_p <= 1.0f) || !(min_p >= 0.0f && min_p <= 1.0f)) return ECK_EINVAL;
    if (n % n_segments) return ECK_ESHAPE;
    if (n / n_segments > MOST_CANDIDATES) return ECK_EUNSUPPORTED;
    if (!aligned(energy, 4) || !aligned(uniform, 4) || !aligned(idx_out, 4) || !aligned(logprob_out, 4) || !aligned(count_out, 4)) return ECK_EALIGN;
    const uint64_t need = sample_select_workspace_bytes(n, n_segments, draws);
    if (need && (!ws || ws_bytes < need)) return ECK_EWORKSPACE;
    if (need && !aligned(ws, 256)) return ECK_EALIGN;
    Draws a = {energy, legal, n / n_segments, uniform, draws, k, top_p, min_p, 0.0, idx_out, logprob_out, count_out};
    if (temperature > 0.0f) {
        a.per_temperature = 1.0 / (double)temperature;
    } else { // the least, and of equal ones the first
        a.per_temperature = 1.0;
        a.k = 1;
        a.top_p = 1.0;
        a.min_p = 0.0;
    }
    const dim3 grid(n_segments);
    const hipStream_t st = as_stream(stream);
    if (a.n <= 256 * 16) hipLaunchKernelGGL((segment_kernel<256, true>), grid, dim3(256), 0, st, a);
    else if (a.n <= 1024 * 16) hipLaunchKernelGGL((segment_kernel<1024, true>), grid, dim3(1024), 0, st, a);
    else hipLaunchKernelGGL((segment_kernel<1024, false>), grid, dim3(1024), 0, st, a);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}
