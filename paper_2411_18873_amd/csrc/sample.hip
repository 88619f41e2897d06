// Selection by drawing: parents of the next generation from the predicted energies and given random numbers (HIP, gfx950).
//
// Candidate i of a segment has weight w = exp(-(E - E_min) / T).  In order of energy, equal ones by index, the kept are a prefix: the k
// least, of these the fewest that have the share top_p of their weight, of these the ones of weight min_p and more.  A draw u takes the
// first kept candidate, by index, at which the sum of weights passes u times all of it.
//
// Nothing is sorted but a few.  The end of a prefix is looked for in a histogram of the energies' order keys over the range in question,
// count and weight of every bin, then in the bin where it lies, until that holds so few candidates that they can be put in order, or equal
// ones alone, which are counted by index.  (Keys are close to logarithms of energies, so a range over both signs, or one outlier, leaves
// most candidates in a few bins: a second histogram is what that costs.)  Weights are 64-bit floating point, and in histograms, which find the
// ends of shares, whole multiples of 2^-60 (of a largest weight of 1; rounded down), held as two numbers of thirty bits, whose sums do not
// depend on the order in which the atomics come.
//
// Segments of up to 16 384 candidates: a block each, keys in registers, one launch.  Longer ones: blocks by the piece, a launch for each
// time that all of a segment has to be known (range, histogram, histogram, candidates at the ends, ends, sums, draws; where few are kept,
// range, histogram, list, draws).  Short ones are bound by a block's chain of phases between barriers (6400 candidates, k = 64, all
// limits: 10 us), long ones by the passes over their candidates (64 segments of 2^18, k = 4096, all three limits: 83 us in four launches, one
// reading of the 84 MB is 16.5; 16 of 2^20 by share alone: 179 us in nine, of which the first histogram, an exponential and three LDS atomics a
// candidate, takes 49; 122 of 92 987, k = 4345 and a share 297 in eleven; 16 of 2^20 without limits 66 in four, the sums 41 of them).
#include "activations.h"
#include "lanes.h"

namespace eck {
namespace {

constexpr uint32_t BINS = 2048, BIN_BITS = 11, NO_KEY = 0xFFFFFFFFu, NOBODY = 0xFFFFFFFFu;
constexpr uint64_t MOST_CANDIDATES = 1ull << 31;
constexpr uint32_t MOST_SEGMENTS = 1u << 20, MOST_DRAWS = 1u << 31; // (draws are counted in 32 bits, a launch's threads at a time)

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
__device__ __forceinline__ Mass mass_of(double w) // (of at most 1: both parts fit 32 bits, to which one instruction converts)
{
    const double t = w * 0x1p30;
    const uint32_t high = (uint32_t)t;
    return {high, (uint32_t)((t - (double)high) * 0x1p30)};
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

// sums over a wavefront's lanes up to and including each
__device__ __forceinline__ uint32_t wave_sums(uint32_t v) { return wave_prefix_sum(v); }
__device__ __forceinline__ unsigned long long wave_sums(unsigned long long v) { return (unsigned long long)wave_prefix_sum((int64_t)v); }
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved_real(double v) { return __builtin_bit_cast(double, moved<CTRL, ROWS>(__builtin_bit_cast(int64_t, v))); }
__device__ __forceinline__ double wave_sums(double v) // (the steps of wave_prefix_sum)
{
    v += moved_real<0x111, 0xF>(v);
    v += moved_real<0x112, 0xF>(v);
    v += moved_real<0x114, 0xF>(v);
    v += moved_real<0x118, 0xF>(v);
    v += moved_real<0x142, 0xA>(v);
    v += moved_real<0x143, 0xC>(v);
    return v;
}
__device__ __forceinline__ uint32_t of_lane(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ unsigned long long of_lane(unsigned long long v, int lane) { return (unsigned long long)lane_value((int64_t)v, lane); }
__device__ __forceinline__ double of_lane(double v, int lane) { return __builtin_bit_cast(double, lane_value(__builtin_bit_cast(int64_t, v), lane)); }

// sums over a block's threads up to and including each (of at most sixteen wavefronts)
template <int THREADS, class V>
__device__ __forceinline__ V block_prefix(V v, V *of_waves)
{
    v = wave_sums(v);
    if (THREADS == 64) return v;
    constexpr int WAVES = THREADS / 64;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    __syncthreads(); // (of_waves may still be read from the last time)
    if (lane == 63) of_waves[wave] = v;
    __syncthreads();
    const V to = wave_sums(lane < WAVES ? of_waves[lane] : (V)0);
    return wave ? of_lane(to, wave - 1) + v : v;
}

typedef unsigned long long u64;

struct Histogram {
    u64 high[BINS], low[BINS];
    uint32_t count[BINS];
};

// Keys lo .. hi, `number` candidates of them; how many are below, and their weight
struct Range {
    uint32_t lo, hi, number, before;
    Mass mass;
};
__device__ __forceinline__ uint32_t shift_of(const Range &r)
{
    const int bits = 32 - __builtin_clz((r.hi - r.lo) | 1);
    return bits > (int)BIN_BITS ? bits - BIN_BITS : 0;
}

// what a prefix ends with: a key, and of the candidates of that key the index of the last
struct Cut {
    uint32_t key, index;
};
__device__ __forceinline__ bool within(uint32_t key, uint32_t index, const Cut &cut) { return key < cut.key || (key == cut.key && index <= cut.index); }

template <int THREADS, int LIST_>
struct Scratch { // of a block that looks for ends
    static constexpr int LIST = LIST_;
    u64 list[LIST], sorted[LIST];
    u64 wide[2][THREADS / 64];
    uint32_t small[THREADS / 64];
    Range found[2];
    Cut cut;
    Mass total;
    uint32_t listed;
};

// of all threads
template <int THREADS, class S>
__device__ __forceinline__ Mass block_total(S &s, const Mass &mine)
{
    const u64 high = block_prefix<THREADS>((u64)mine.high, s.wide[0]), low = block_prefix<THREADS>((u64)mine.low, s.wide[1]);
    __syncthreads();
    if (threadIdx.x == THREADS - 1) s.total = {high, low};
    __syncthreads();
    return s.total;
}

// which prefix: the `need` least candidates, or the fewest of a weight of `target` (from and up to, while that is not known)
struct Goal {
    bool by_weight;
    uint32_t need;
    double target[2];
    double share = 0.0; // above 0: the targets are this share of all weight, which find_cut_of takes from its first histogram
    __device__ __forceinline__ bool reached(int which, uint32_t count, const Mass &mass) const
    {
        return by_weight ? mass.value() >= target[which] : count >= need;
    }
};

template <int THREADS>
__device__ __forceinline__ void clear_bins(Histogram &bins, bool weights)
{
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < BINS; b += THREADS) {
        bins.count[b] = 0;
        if (weights) bins.high[b] = bins.low[b] = 0;
    }
    __syncthreads();
}

__device__ __forceinline__ void add_to_bins(Histogram &bins, uint32_t bin, bool weights, double w)
{
    atomicAdd(&bins.count[bin], 1u);
    if (weights) {
        const Mass m = mass_of(w);
        atomicAdd(&bins.high[bin], (u64)m.high);
        atomicAdd(&bins.low[bin], (u64)m.low);
    }
}

// The bins of `at` in which the prefix ends, or may end: s.found[0] from the first of them to the last.  All threads get the result.
// weights: whether the bins hold any.
template <int THREADS, class S>
__device__ __forceinline__ Range narrow(S &s, const Histogram &bins, const Range &at, const Goal &goal, bool weights)
{
    constexpr uint32_t EACH = BINS / THREADS;
    const uint32_t first = threadIdx.x * EACH, shift = shift_of(at);
    uint32_t count = 0;
    Mass mass = {0, 0};
#pragma unroll
    for (uint32_t i = 0; i < EACH; ++i) {
        count += bins.count[first + i];
        if (weights) mass = mass + Mass{bins.high[first + i], bins.low[first + i]};
    }
    const uint32_t to = at.before + block_prefix<THREADS>(count, s.small);
    Mass mass_to = at.mass;
    if (weights) mass_to = mass_to + Mass{block_prefix<THREADS>((u64)mass.high, s.wide[0]), block_prefix<THREADS>((u64)mass.low, s.wide[1])};
    const uint32_t from = to - count;
    const Mass mass_from = {mass_to.high - mass.high, mass_to.low - mass.low};
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        // (the last thread's, should none reach it)
        const bool mine = (threadIdx.x == 0 || !goal.reached(which, from, mass_from)) && (threadIdx.x == THREADS - 1 || goal.reached(which, to, mass_to));
        if (mine) {
            uint32_t c = from, b = first;
            Mass m = mass_from;
            for (; b < first + EACH - 1; ++b) {
                const Mass next = weights ? m + Mass{bins.high[b], bins.low[b]} : m;
                if (goal.reached(which, c + bins.count[b], next)) break;
                c += bins.count[b];
                m = next;
            }
            const uint32_t lo = at.lo + (b << shift);
            s.found[which] = {lo, min(at.hi, lo + ((1u << shift) - 1)), bins.count[b], c, m};
        }
    }
    __syncthreads();
    Range r = s.found[0];
    const Range last = s.found[1];
    if (last.lo > r.lo) { // (by weight, of which the end is not known yet)
        r.hi = last.hi;
        r.number = last.before + last.number - r.before;
    }
    __syncthreads();
    return r;
}

// s.sorted = the `c` first of s.list, least first (no two are equal)
template <int THREADS, class S>
__device__ __forceinline__ void sort_list(S &s, uint32_t c)
{
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < c; i += THREADS) {
        const u64 mine = s.list[i];
        uint32_t rank = 0;
#pragma unroll 4
        for (uint32_t j = 0; j < c; ++j) rank += s.list[j] < mine;
        s.sorted[rank] = mine;
    }
    __syncthreads();
}

// Where the prefix ends among the range's candidates, all of them in s.sorted: s.cut; and the weight up to there: s.total
template <int THREADS, class S, class W>
__device__ __forceinline__ void cut_sorted(S &s, const Range &at, const Goal &goal, bool weights, W &&weight)
{
    constexpr uint32_t EACH = (S::LIST + THREADS - 1) / THREADS;
    const uint32_t c = at.number, first = threadIdx.x * EACH;
    Mass mass[EACH], sum = {0, 0};
#pragma unroll
    for (uint32_t i = 0; i < EACH; ++i) {
        mass[i] = weights && first + i < c ? mass_of(weight((uint32_t)(s.sorted[first + i] >> 32))) : Mass{0, 0};
        sum = sum + mass[i];
    }
    Mass to = at.mass;
    if (weights) {
        to = to + Mass{block_prefix<THREADS>((u64)sum.high, s.wide[0]), block_prefix<THREADS>((u64)sum.low, s.wide[1])};
        to = {to.high - sum.high, to.low - sum.low};
    }
#pragma unroll
    for (uint32_t i = 0; i < EACH; ++i) {
        if (first + i >= c) break;
        const Mass next = to + mass[i];
        const uint32_t count = at.before + first + i;
        // (the last one, should none reach it)
        if ((first + i == 0 || !goal.reached(0, count, to)) && (first + i == c - 1 || goal.reached(0, count + 1, next))) {
            s.cut = {(uint32_t)(s.sorted[first + i] >> 32), (uint32_t)s.sorted[first + i]};
            s.total = next;
        }
        to = next;
    }
    __syncthreads();
}

// how many of `all` candidates of weight w each, behind `before`, it takes to `target`
__device__ __forceinline__ uint32_t enough(double before, double w, uint32_t all, double target)
{
    if (!(w > 0.0)) return all;
    double j = ceil((target - before) / w);
    j = fmin(fmax(j, 1.0), (double)all);
    if (j > 1.0 && before + (j - 1.0) * w >= target) j -= 1.0;
    if (j < (double)all && before + j * w < target) j += 1.0;
    return (uint32_t)j;
}

// Of candidates of one key, the number of the last in the prefix (from 1), and the weight up to there: s.total
template <class S>
__device__ __forceinline__ uint32_t last_of_equal(S &s, const Range &at, const Goal &goal, double w)
{
    const uint32_t j = goal.by_weight ? enough(at.mass.value(), w, at.number, goal.target[0]) : min(max(goal.need - at.before, 1u), at.number);
    const Mass one = mass_of(w);
    __syncthreads();
    if (threadIdx.x == 0) s.total = at.mass + Mass{j * one.high, j * one.low};
    __syncthreads();
    return j;
}

// energies from the least up to a bound, in bins of one width
struct Linear {
    float least, last, scale;
    __device__ __forceinline__ Linear(uint32_t from, uint32_t to) : least(energy_of(from)), last(energy_of(to))
    {
        const float width = last - least;
        scale = width > 0.0f ? (float)BINS / width : 0.0f;
        if (!(scale < __builtin_inff())) scale = 0.0f;
    }
    __device__ __forceinline__ bool holds(float e) const { return e >= least && e <= last; } // (no NaN)
    // the bin is this rounded down: every step keeps the order of energies (a width past fp32's range times 0 is taken for the last bin's)
    __device__ __forceinline__ float place(float e) const { return fminf((e - least) * scale, (float)(BINS - 1)); }
    __device__ __forceinline__ uint32_t bin(float e) const { return (uint32_t)place(e); }
};

// The end of a prefix within the range `at`, from the candidates themselves: source.each(f) calls f(key, index) for those that may be drawn,
// source.nth(key, j) is the index of the j-th one of a key; Source::FITS: a list takes all there can be.  Sets s.cut and s.total.
template <int THREADS, class S, class Source, class W>
__device__ void find_cut(S &s, Histogram &bins, Range at, const Goal &goal, bool weights, const Source &source, W &&weight)
{
    for (int round = 0; round < 4; ++round) { // (three rounds leave one key)
        if (Source::FITS || at.number <= (uint32_t)S::LIST) {
            __syncthreads();
            if (threadIdx.x == 0) s.listed = 0;
            __syncthreads();
            source.each([&](uint32_t key, uint32_t index) {
                if (key < at.lo || key > at.hi) return;
                const uint32_t place = atomicAdd(&s.listed, 1u);
                if (place < (uint32_t)S::LIST) s.list[place] = (u64)key << 32 | index;
            });
            sort_list<THREADS>(s, at.number);
            cut_sorted<THREADS>(s, at, goal, weights, weight);
            return;
        }
        if constexpr (!Source::FITS) {
            if (at.lo == at.hi) {
                const uint32_t j = last_of_equal(s, at, goal, weight(at.lo)), index = source.nth(at.lo, j);
                if (threadIdx.x == 0) s.cut = {at.lo, index};
                __syncthreads();
                return;
            }
            clear_bins<THREADS>(bins, weights);
            const uint32_t shift = shift_of(at);
            source.each([&](uint32_t key, uint32_t) {
                if (key >= at.lo && key <= at.hi) add_to_bins(bins, (key - at.lo) >> shift, weights, weights ? weight(key) : 0.0);
            });
            __syncthreads();
            at = narrow<THREADS>(s, bins, at, goal, weights);
        }
    }
}

// The same over all keys from..to of the source, `number` candidates, most of them far from each other: a first histogram linear in energy has
// few of them in a bin, and none that all threads add to at once
template <int THREADS, class S, class Source, class W>
__device__ void find_cut_of(S &s, Histogram &bins, uint32_t from, uint32_t to, uint32_t number, Goal goal, bool weights, const Source &source, W &&weight)
{
    if (!Source::FITS && number > (uint32_t)S::LIST) {
        const Linear linear(from, to);
        clear_bins<THREADS>(bins, weights);
        source.each([&](uint32_t key, uint32_t) { add_to_bins(bins, linear.bin(energy_of(key)), weights, weights ? weight(key) : 0.0); });
        __syncthreads();
        if (goal.share > 0.0) {
            constexpr uint32_t EACH = BINS / THREADS;
            Mass sum = {0, 0};
#pragma unroll
            for (uint32_t i = 0; i < EACH; ++i) sum = sum + Mass{bins.high[threadIdx.x * EACH + i], bins.low[threadIdx.x * EACH + i]};
            goal.target[0] = goal.target[1] = goal.share * block_total<THREADS>(s, sum).value();
        }
        const Range bin = narrow<THREADS>(s, bins, {0, BINS - 1, number, 0, {0, 0}}, goal, weights);
        if (bin.number <= (uint32_t)S::LIST && bin.lo == bin.hi) {
            if (threadIdx.x == 0) s.listed = 0;
            __syncthreads();
            source.each([&](uint32_t key, uint32_t index) {
                if (linear.bin(energy_of(key)) != bin.lo) return;
                const uint32_t place = atomicAdd(&s.listed, 1u);
                if (place < (uint32_t)S::LIST) s.list[place] = (u64)key << 32 | index;
            });
            sort_list<THREADS>(s, bin.number);
            cut_sorted<THREADS>(s, bin, goal, weights, weight);
            return;
        }
    }
    find_cut<THREADS>(s, bins, {from, to, number, 0, {0, 0}}, goal, weights, source, weight);
}

__device__ __forceinline__ void nothing_to_draw(const Draws &a, uint64_t segment, uint32_t first, uint32_t step)
{
    for (uint32_t d = first; d < a.draws; d += step) {
        a.idx[segment * a.draws + d] = NOBODY;
        if (a.logprob) a.logprob[segment * a.draws + d] = -__builtin_inff();
    }
}

// ------------------------------------------------------------------------------------------------ short segments

// Keys of a block's candidates, EACH neighbouring ones a thread; those up to a cut
template <int THREADS, int EACH, class S>
struct Held {
    static constexpr bool FITS = THREADS * EACH <= S::LIST; // all of them in a list
    uint32_t (&key)[EACH];
    S &s;
    const Cut &cut;
    template <class F>
    __device__ __forceinline__ void each(F &&f) const
    {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (within(key[i], threadIdx.x * EACH + i, cut)) f(key[i], threadIdx.x * EACH + i); // (NO_KEY is above any)
    }
    __device__ uint32_t nth(uint32_t of, uint32_t j) const
    {
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) mine += key[i] == of;
        uint32_t before = block_prefix<THREADS>(mine, s.small) - mine;
        __syncthreads();
        if (before < j && before + mine >= j)
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (key[i] == of && ++before == j) s.listed = threadIdx.x * EACH + i;
        __syncthreads();
        return s.listed;
    }
};

template <int THREADS, int EACH>
struct Short {
    // few candidates are put in order at once, more are binned first
    static constexpr bool BINNED = THREADS * EACH > 256;
    typedef Scratch<THREADS, 256> S;
    struct Ends {
        S s;
        Histogram bins[BINNED ? 1 : 0];
    };
    union {
        Ends ends;
        // sums of weights up to and including each candidate; a place between threads' keeps their lanes off each other's banks (16 384 by a least
        // weight alone: 14 us, 25 without it)
        double to[THREADS * (EACH + 1)];
    };
    static __device__ __forceinline__ uint32_t place(uint32_t i) { return i + i / EACH; }
    double of_waves[THREADS / 64];
    uint32_t least[THREADS / 64], most[THREADS / 64], number[THREADS / 64];
};

// The least of a short segment, where so few are kept that a list takes all up to the end's bin: put in order once, after which one wavefront
// has all ends and sums without a barrier.  False (and nothing written) where the bin holds too many for that.  6400 candidates, k = 64, all
// limits: 9.8 us by this, 18.3 by the ends one after the other.
template <int THREADS, int EACH, class S, class W>
__device__ __forceinline__ bool draw_from_few(const Draws &a, S &s, Histogram &bins, const uint32_t (&key)[EACH], uint32_t least, uint32_t most,
                                              uint32_t number, W &&weight)
{
    constexpr int OF_LANE = S::LIST / 64;
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t segment = blockIdx.x;
    const Linear linear(least, most);
    clear_bins<THREADS>(bins, false);
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (key[i] != NO_KEY) atomicAdd(&bins.count[linear.bin(energy_of(key[i]))], 1u);
    if (threadIdx.x == 0) s.listed = 0;
    __syncthreads();
    const Range end = narrow<THREADS>(s, bins, {0, BINS - 1, number, 0, {0, 0}}, {false, a.k, {0.0, 0.0}}, false); // (one bin)
    const uint32_t listed = end.before + end.number;
    if (listed > (uint32_t)S::LIST) return false;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (key[i] != NO_KEY && linear.bin(energy_of(key[i])) <= end.lo) s.list[atomicAdd(&s.listed, 1u)] = (u64)key[i] << 32 | (threadIdx.x * EACH + i);
    sort_list<THREADS>(s, listed);

    u64 *const w_of = bins.high, *const sum_to = bins.low; // (by index; bits of fp64)
    if (threadIdx.x < 64) {
        const auto meet = [] { // what the wavefront has written is there for all its lanes
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
        u64 one[OF_LANE];
        double w[OF_LANE];
        uint32_t kept = a.k;
#pragma unroll
        for (int i = 0; i < OF_LANE; ++i) {
            const uint32_t e = lane * OF_LANE + i;
            one[i] = e < kept ? s.sorted[e] : 0;
            w[i] = e < kept ? weight((uint32_t)(one[i] >> 32)) : 0.0;
        }
        if (a.top_p < 1.0) {
            Mass sum = {0, 0};
#pragma unroll
            for (int i = 0; i < OF_LANE; ++i) sum = sum + mass_of(w[i]);
            Mass to = {wave_sums((u64)sum.high), wave_sums((u64)sum.low)};
            const double target = a.top_p * Mass{of_lane((u64)to.high, 63), of_lane((u64)to.low, 63)}.value();
            to = {to.high - sum.high, to.low - sum.low};
            uint32_t before = 0; // how many leave the sum below the target
#pragma unroll
            for (int i = 0; i < OF_LANE; ++i) {
                to = to + mass_of(w[i]);
                before += lane * OF_LANE + i < kept && to.value() < target;
            }
            kept = min(kept, of_lane(wave_sums(before), 63) + 1);
        }
        uint32_t mine[OF_LANE], rank[OF_LANE];
#pragma unroll
        for (int i = 0; i < OF_LANE; ++i) {
            const bool stays = lane * OF_LANE + i < kept && w[i] >= a.min_p;
            mine[i] = stays ? (uint32_t)one[i] : NOBODY;
            rank[i] = 0;
            s.list[lane * OF_LANE + i] = mine[i];
        }
        meet();
#pragma unroll 4
        for (uint32_t j = 0; j < kept; ++j) {
            const uint32_t other = (uint32_t)s.list[j];
#pragma unroll
            for (int i = 0; i < OF_LANE; ++i) rank[i] += other < mine[i];
        }
        uint32_t number_kept = 0;
#pragma unroll
        for (int i = 0; i < OF_LANE; ++i) {
            number_kept += __builtin_popcountll(__ballot(mine[i] != NOBODY));
            if (mine[i] == NOBODY) continue;
            s.sorted[rank[i]] = mine[i];
            w_of[rank[i]] = __builtin_bit_cast(u64, w[i]);
        }
        meet();
        double up_to[OF_LANE], sum = 0.0;
#pragma unroll
        for (int i = 0; i < OF_LANE; ++i) {
            sum += lane * OF_LANE + i < number_kept ? __builtin_bit_cast(double, w_of[lane * OF_LANE + i]) : 0.0;
            up_to[i] = sum;
        }
        const double before = wave_sums(sum) - sum;
#pragma unroll
        for (int i = 0; i < OF_LANE; ++i) sum_to[lane * OF_LANE + i] = __builtin_bit_cast(u64, before + up_to[i]);
        if (lane == 0) {
            s.listed = number_kept;
            if (a.count) a.count[segment] = number_kept;
        }
    }
    __syncthreads();
    const uint32_t kept = s.listed;
    const auto sum_of = [&](uint32_t i) { return __builtin_bit_cast(double, sum_to[i]); };
    const auto weight_at = [&](uint32_t i) { return __builtin_bit_cast(double, w_of[i]); };
    const double all = sum_of(kept - 1);
    for (uint32_t d = threadIdx.x; d < a.draws; d += THREADS) {
        const double target = fmax((double)a.uniform[segment * a.draws + d] * all, 0.0);
        uint32_t lo = 0, hi = kept - 1;
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (sum_of(mid) > target) hi = mid;
            else lo = mid + 1;
        }
        while (!(weight_at(lo) > 0.0) && lo + 1 < kept && all > target) ++lo;
        while (!(weight_at(lo) > 0.0) && lo > 0) --lo;
        a.idx[segment * a.draws + d] = (uint32_t)s.sorted[lo];
        if (a.logprob) a.logprob[segment * a.draws + d] = (float)log(weight_at(lo) / all);
    }
    return true;
}

template <int THREADS, int EACH, bool FEWEST>
__global__ __launch_bounds__(THREADS) void short_kernel(const Draws a)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    typedef Short<THREADS, EACH> Lds;
    Lds &s = *reinterpret_cast<Lds *>(lds);
    const uint32_t n = (uint32_t)a.n, lane = threadIdx.x & 63, wave = threadIdx.x / 64, first = threadIdx.x * EACH;
    const uint64_t segment = blockIdx.x;
    const float *energy = a.energy + segment * n;
    const uint8_t *legal = a.legal ? a.legal + segment * n : nullptr;
    uint32_t key[EACH], least = NO_KEY, most = 0, number = 0;
#pragma unroll
    for (int i = 0; i < EACH; i += 4) {
        uint32_t four[4] = {NO_KEY, NO_KEY, NO_KEY, NO_KEY};
        if (first + i < n) load_keys(energy, legal, first + i, n, four);
#pragma unroll
        for (int j = 0; j < 4; ++j) key[i + j] = four[j];
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        least = min(least, key[i]);
        most = key[i] != NO_KEY ? max(most, key[i]) : most;
        number += key[i] != NO_KEY;
    }
#pragma unroll
    for (int stride = 1; stride < 64; stride <<= 1) {
        least = min(least, lane_exchange(least, stride));
        most = max(most, lane_exchange(most, stride));
        number += lane_exchange(number, stride);
    }
    if (THREADS > 64) {
        if (lane == 0) s.least[wave] = least, s.most[wave] = most, s.number[wave] = number;
        __syncthreads();
        number = 0;
        for (int w = 0; w < THREADS / 64; ++w) {
            least = min(least, s.least[w]);
            most = max(most, s.most[w]);
            number += s.number[w];
        }
    }
    if (number == 0) {
        nothing_to_draw(a, segment, threadIdx.x, THREADS);
        if (threadIdx.x == 0 && a.count) a.count[segment] = 0;
        return;
    }
    const double best = (double)energy_of(least);
    const auto weight = [&](uint32_t k) { return weight_of(k, best, a.per_temperature); };

    if constexpr (FEWEST) {
        if (a.k < number) {
            if (draw_from_few<THREADS, EACH>(a, s.ends.s, s.ends.bins[0], key, least, most, number, weight)) return;
            __syncthreads();
        }
    }
    Cut cut = {most, n};
    {
        typename Lds::S &sc = s.ends.s;
        Histogram &bins = s.ends.bins[0];
        const Held<THREADS, EACH, typename Lds::S> held = {key, sc, cut};
        uint32_t kept = number;
        if (a.k && a.k < number) {
            Cut found;
            if (a.k == 1) { // the first of the least
                found = {least, held.nth(least, 1)};
            } else {
                find_cut_of<THREADS>(sc, bins, least, most, number, {false, a.k, {0.0, 0.0}}, false, held, weight);
                found = sc.cut;
                __syncthreads();
            }
            cut = found; // (`held` goes by it from here on)
            kept = a.k;
        }
        if (a.top_p < 1.0 && kept > 1) {
            Goal goal = {true, 0, {0.0, 0.0}, a.top_p};
            if (decltype(held)::FITS || kept <= (uint32_t)Lds::S::LIST) { // (no histogram will be made)
                Mass mine = {0, 0};
                held.each([&](uint32_t k, uint32_t) { mine = mine + mass_of(weight(k)); });
                goal.target[0] = goal.target[1] = a.top_p * block_total<THREADS>(sc, mine).value();
            }
            find_cut_of<THREADS>(sc, bins, least, cut.key, kept, goal, true, held, weight);
            cut = sc.cut;
        }
    }
    __syncthreads(); // (what is written now lies where that was)

    double sum = 0.0;
    uint32_t kept = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (within(key[i], first + i, cut)) { // (NO_KEY is above any)
            const double w = weight(key[i]);
            if (w >= a.min_p) {
                sum += w;
                ++kept;
            }
        }
        if (first + i < n) s.to[Lds::place(first + i)] = sum;
    }
    const double before = block_prefix<THREADS>(sum, s.of_waves) - sum;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (first + i < n) s.to[Lds::place(first + i)] += before;
#pragma unroll
    for (int stride = 1; stride < 64; stride <<= 1) kept += lane_exchange(kept, stride);
    if (lane == 0) s.number[wave] = kept;
    __syncthreads();
    if (threadIdx.x == 0 && a.count) {
        for (int o = 1; o < THREADS / 64; ++o) kept += s.number[o];
        a.count[segment] = kept;
    }
    const double all = s.to[Lds::place(n - 1)];
    const auto kept_weight = [&](uint32_t i) {
        const uint32_t k = key_of(energy[i], !legal || legal[i]);
        const double x = k != NO_KEY && within(k, i, cut) ? weight(k) : 0.0;
        return x >= a.min_p ? x : 0.0;
    };
    for (uint32_t d = threadIdx.x; d < a.draws; d += THREADS) {
        const double target = fmax((double)a.uniform[segment * a.draws + d] * all, 0.0);
        uint32_t lo = 0, hi = n - 1; // the first sum that passes the target, or the last
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (s.to[Lds::place(mid)] > target) hi = mid;
            else lo = mid + 1;
        }
        // (between two threads' candidates sums may differ in their last bit where nothing is added; and past the end the last one is wanted)
        double x = kept_weight(lo);
        while (!(x > 0.0) && lo + 1 < n && s.to[Lds::place(n - 1)] > target) x = kept_weight(++lo);
        while (!(x > 0.0) && lo > 0) x = kept_weight(--lo);
        a.idx[segment * a.draws + d] = lo;
        if (a.logprob) a.logprob[segment * a.draws + d] = (float)log(x / all);
    }
}

// ------------------------------------------------------------------------------------------------ long segments

constexpr int LONG_THREADS = 1024;
constexpr uint32_t LIST = 4096;       // candidates at the ends that are listed, of a segment
constexpr uint32_t MOST_PIECES = 512; // blocks of a segment
typedef Scratch<LONG_THREADS, 1024> LongScratch;

struct Bounds { // of a block's piece; gate: the largest of its threads' least keys, threads: of those that have any
    uint32_t least, most, number, gate, threads;
};
struct Equal { // candidates of a range in a block's piece: their least and largest key, and how many
    uint32_t least, most, number, unused;
};
struct Segment {
    uint32_t least, most, number, listed, listed_below;
    uint32_t need, before, at_end; // how many are kept, below the end's bin and in it
    Range by_count, by_weight;
    double total; // weight of all, where no k least are taken
    Cut cut;
};
struct Long {
    Draws a;
    uint64_t segments;
    uint32_t pieces;     // blocks a segment
    uint64_t piece;      // candidates of a block: a multiple of 4096
    uint64_t strip;      // candidates of a strip: a multiple of 64; 64 strips are a chunk
    uint32_t chunks;     // of a segment
    Bounds *bounds;      // [segments][pieces]
    Histogram *parts;    // [2][segments][pieces]
    Histogram *whole;    // [2][segments], of several pieces; else parts
    Segment *segment;    // [segments]
    u64 *list;           // [segments][LIST]
    Equal *equal;        // [2][segments][pieces]: by count, by weight
    double *strip_sums;  // [segments][chunks][64]
    double *chunk_sums;  // [segments][chunks]
    uint32_t *chunk_counts;
    __device__ __forceinline__ Histogram *histogram(int which, uint64_t s) const
    {
        return pieces > 1 ? whole + which * segments + s : parts + which * segments + s;
    }
};

__device__ __forceinline__ bool by_count(const Long &p, uint32_t number) { return p.a.k && p.a.k < number; }

template <class F>
__device__ __forceinline__ void each_of_piece(const Draws &a, uint64_t segment, uint64_t from, uint64_t to, F &&f)
{
    const float *energy = a.energy + segment * a.n;
    const uint8_t *legal = a.legal ? a.legal + segment * a.n : nullptr;
    constexpr int AHEAD = 4;
    for (uint64_t at = from + threadIdx.x * 4; at < to; at += LONG_THREADS * 4 * AHEAD) {
        uint32_t key[AHEAD][4];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const uint64_t here = at + (uint64_t)k * LONG_THREADS * 4;
            if (here < to) load_keys(energy, legal, here, to, key[k]);
            else key[k][0] = key[k][1] = key[k][2] = key[k][3] = NO_KEY;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (key[k][i] != NO_KEY) f(key[k][i], (uint32_t)(at + (uint64_t)k * LONG_THREADS * 4 + i));
    }
}

// least and largest key and how many, over a block
__device__ __forceinline__ Bounds block_bounds(Bounds b, Bounds *of_waves)
{
#pragma unroll
    for (int stride = 1; stride < 64; stride <<= 1) {
        b.least = min(b.least, lane_exchange(b.least, stride));
        b.most = max(b.most, lane_exchange(b.most, stride));
        b.number += lane_exchange(b.number, stride);
        b.gate = max(b.gate, lane_exchange(b.gate, stride));
        b.threads += lane_exchange(b.threads, stride);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) of_waves[threadIdx.x / 64] = b;
    __syncthreads();
    b = of_waves[threadIdx.x % (LONG_THREADS / 64)];
#pragma unroll
    for (int stride = 1; stride < LONG_THREADS / 64; stride <<= 1) {
        b.least = min(b.least, lane_exchange(b.least, stride));
        b.most = max(b.most, lane_exchange(b.most, stride));
        b.number += lane_exchange(b.number, stride);
        b.gate = max(b.gate, lane_exchange(b.gate, stride));
        b.threads += lane_exchange(b.threads, stride);
    }
    return b;
}

__global__ __launch_bounds__(LONG_THREADS) void bounds_kernel(const Long p)
{
    __shared__ Bounds of_waves[LONG_THREADS / 64];
    const uint64_t segment = blockIdx.x / p.pieces, from = blockIdx.x % p.pieces * p.piece, to = min(p.a.n, from + p.piece);
    Bounds b = {NO_KEY, 0, 0, 0, 0};
    each_of_piece(p.a, segment, from, to, [&](uint32_t key, uint32_t) {
        b.least = min(b.least, key);
        b.most = max(b.most, key);
        ++b.number;
    });
    b = block_bounds(b, of_waves);
    if (threadIdx.x == 0) p.bounds[blockIdx.x] = b;
}

// of all pieces of a segment
__device__ __forceinline__ Bounds segment_bounds(const Long &p, uint64_t segment, Bounds *of_waves)
{
    Bounds b = {NO_KEY, 0, 0, 0, 0};
    if (threadIdx.x < p.pieces) b = p.bounds[segment * p.pieces + threadIdx.x];
    return block_bounds(b, of_waves);
}

// Places of energies on a scale of 32 bits, linear from the least up to where weights are below e^-64 or energies end: what the share of the
// weight is looked for with.  (Of order keys a range over both signs has eight bins a binade, which all threads add to at once: first
// histograms of 2^24 candidates took 51 us.)
struct Scale {
    float least, factor;
    static constexpr uint32_t LAST = 0xFFFFFF00u; // the largest that a float holds
    __device__ __forceinline__ Scale(const Draws &a, uint32_t least_key, uint32_t most_key) : least(energy_of(least_key))
    {
        const float far = (float)((double)least + 64.0 / a.per_temperature), most = energy_of(most_key), last = far < most ? far : most;
        factor = last > least ? (float)LAST / (last - least) : 0.0f;
        if (!(last > least) && most > least) factor = __builtin_inff(); // nothing but the least has a weight
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t key) const
    {
        const float e = energy_of(key);
        return e == least ? 0 : (uint32_t)fminf((e - least) * factor, (float)LAST);
    }
};
constexpr Range SCALE = {0, 0xFFFFFFFFu, 0, 0, {0, 0}};

__device__ __forceinline__ void write_bins(Histogram &to, const Histogram &from, bool weights)
{
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < BINS; b += LONG_THREADS) {
        to.count[b] = from.count[b];
        if (!weights) continue;
        to.high[b] = from.high[b];
        to.low[b] = from.low[b];
    }
}

// By key for the k least, by weight for a share: one of the two or both
__global__ __launch_bounds__(LONG_THREADS) __attribute__((amdgpu_waves_per_eu(8))) void first_bins_kernel(const Long p)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    Histogram *const bins = reinterpret_cast<Histogram *>(lds);
    __shared__ Bounds of_waves[LONG_THREADS / 64];
    const uint64_t segment = blockIdx.x / p.pieces, from = blockIdx.x % p.pieces * p.piece, to = min(p.a.n, from + p.piece);
    const Bounds b = segment_bounds(p, segment, of_waves);
    if (b.number == 0) return;
    const bool weights = p.a.top_p < 1.0;
    const double best = (double)energy_of(b.least);
    const Range whole = {b.least, b.most, b.number, 0, {0, 0}};
    const Scale scale(p.a, b.least, b.most);
    const uint32_t shift = shift_of(whole), shift_weight = shift_of(SCALE);
    const bool limited = by_count(p, b.number);
    clear_bins<LONG_THREADS>(bins[0], weights);
    if (limited && weights) clear_bins<LONG_THREADS>(bins[1], weights);
    Histogram &by_weight = bins[limited ? 1 : 0];
    each_of_piece(p.a, segment, from, to, [&](uint32_t key, uint32_t) {
        const double w = weights ? weight_of(key, best, p.a.per_temperature) : 0.0;
        if (limited) add_to_bins(bins[0], (key - whole.lo) >> shift, weights, w);
        if (weights) add_to_bins(by_weight, scale(key) >> shift_weight, true, w);
    });
    if (limited) write_bins(p.parts[blockIdx.x], bins[0], weights);
    if (weights) write_bins(p.parts[p.segments * p.pieces + blockIdx.x], by_weight, true);
}

// histograms of a segment's pieces added up: a block has 64 bins, each wavefront some of the pieces
constexpr uint32_t JOIN_BLOCKS = BINS / 64;
__global__ __launch_bounds__(LONG_THREADS) void join_bins_kernel(const Long p, int which)
{
    __shared__ Mass masses[LONG_THREADS / 64][64];
    __shared__ uint32_t counts[LONG_THREADS / 64][64];
    const uint64_t segment = blockIdx.x / JOIN_BLOCKS;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, b = blockIdx.x % JOIN_BLOCKS * 64 + lane;
    const Histogram *from = p.parts + (which * p.segments + segment) * p.pieces;
    const bool weights = p.a.top_p < 1.0;
    uint32_t count = 0;
    Mass mass = {0, 0};
#pragma unroll 4
    for (uint32_t i = wave; i < p.pieces; i += LONG_THREADS / 64) {
        count += from[i].count[b];
        if (weights) mass = mass + Mass{from[i].high[b], from[i].low[b]};
    }
    counts[wave][lane] = count;
    masses[wave][lane] = mass;
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < LONG_THREADS / 64; ++w) {
        count += counts[w][lane];
        mass = mass + masses[w][lane];
    }
    Histogram &to = p.whole[which * p.segments + segment];
    to.count[b] = count;
    to.high[b] = mass.high;
    to.low[b] = mass.low;
}

__device__ __forceinline__ void read_bins(Histogram &to, const Histogram &from, bool weights)
{
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < BINS; b += LONG_THREADS) {
        to.count[b] = from.count[b];
        if (!weights) continue;
        to.high[b] = from.high[b];
        to.low[b] = from.low[b];
    }
    __syncthreads();
}

// Where the weight's share ends: between those of the least and the largest sum that the k least may have
__device__ __forceinline__ Goal weight_goal(const Draws &a, bool limited, const Range &by_count, const Mass &of_range, double total)
{
    const double from = limited ? by_count.mass.value() : total, to = limited ? (by_count.mass + of_range).value() : total;
    return {true, 0, {a.top_p * from, a.top_p * to}};
}

// weight of the bin that narrow() found within `at`
__device__ __forceinline__ Mass mass_in(const Histogram &bins, const Range &at, const Range &found)
{
    const uint32_t b = (found.lo - at.lo) >> shift_of(at);
    return {bins.high[b], bins.low[b]};
}

// The ranges that the ends lie in, from the histogram over all keys, and a histogram of each
__global__ __launch_bounds__(LONG_THREADS) __attribute__((amdgpu_waves_per_eu(8))) void second_bins_kernel(const Long p)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    Histogram *const bins = reinterpret_cast<Histogram *>(lds);
    __shared__ LongScratch s;
    __shared__ Bounds of_waves[LONG_THREADS / 64];
    const uint64_t segment = blockIdx.x / p.pieces, from = blockIdx.x % p.pieces * p.piece, to = min(p.a.n, from + p.piece);
    const Bounds b = segment_bounds(p, segment, of_waves);
    Segment &of = p.segment[segment];
    const bool weights = p.a.top_p < 1.0, limited = by_count(p, b.number), first = blockIdx.x % p.pieces == 0 && threadIdx.x == 0;
    if (first) of.least = b.least, of.most = b.most, of.number = b.number, of.listed = 0;
    if (b.number == 0) return;
    const double best = (double)energy_of(b.least);
    const Range whole = {b.least, b.most, b.number, 0, {0, 0}};
    const Scale scale(p.a, b.least, b.most);
    Range at[2] = {whole, SCALE};
    at[1].number = b.number;
    double total = 0.0;
    Mass of_range = {0, 0};
    if (limited) {
        read_bins(bins[0], *p.histogram(0, segment), weights);
        at[0] = narrow<LONG_THREADS>(s, bins[0], whole, {false, p.a.k, {0.0, 0.0}}, weights);
        if (weights) of_range = mass_in(bins[0], whole, at[0]);
    }
    if (weights) {
        read_bins(bins[0], *p.histogram(1, segment), true);
        if (!limited) {
            u64 high = 0, low = 0;
            for (uint32_t i = threadIdx.x; i < BINS; i += LONG_THREADS) high += bins[0].high[i], low += bins[0].low[i];
            high = block_prefix<LONG_THREADS>(high, s.wide[0]);
            low = block_prefix<LONG_THREADS>(low, s.wide[1]);
            __syncthreads();
            if (threadIdx.x == LONG_THREADS - 1) s.total = {high, low};
            __syncthreads();
            total = s.total.value();
        }
        at[1] = narrow<LONG_THREADS>(s, bins[0], at[1], weight_goal(p.a, limited, at[0], of_range, total), true);
    }
    if (first) of.by_count = at[0], of.by_weight = at[1], of.total = total;
    // (one histogram where one is wanted: with both in the LDS a compute unit has room for one block, not two)
    Histogram &of_count = bins[0], &of_weight = bins[p.a.k ? 1 : 0];
    if (limited) clear_bins<LONG_THREADS>(of_count, weights);
    if (weights) clear_bins<LONG_THREADS>(of_weight, true);
    const uint32_t shift[2] = {shift_of(at[0]), shift_of(at[1])};
    each_of_piece(p.a, segment, from, to, [&](uint32_t key, uint32_t) {
        const uint32_t place[2] = {key, scale(key)};
        const bool in[2] = {limited && key >= at[0].lo && key <= at[0].hi, weights && place[1] >= at[1].lo && place[1] <= at[1].hi};
        if (!in[0] && !in[1]) return;
        const double w = weights ? weight_of(key, best, p.a.per_temperature) : 0.0;
        if (in[0]) add_to_bins(of_count, (place[0] - at[0].lo) >> shift[0], weights, w);
        if (in[1]) add_to_bins(of_weight, (place[1] - at[1].lo) >> shift[1], true, w);
    });
    __syncthreads();
    if (limited) write_bins(p.parts[blockIdx.x], of_count, weights); // (the first ones are not needed again)
    if (weights) write_bins(p.parts[p.segments * p.pieces + blockIdx.x], of_weight, true);
}

// The ranges again, by the second histograms, and the candidates in them
__global__ __launch_bounds__(LONG_THREADS) __attribute__((amdgpu_waves_per_eu(8))) void list_kernel(const Long p)
{
    __shared__ Histogram bins;
    __shared__ LongScratch s;
    __shared__ Bounds of_waves[LONG_THREADS / 64];
    const uint64_t segment = blockIdx.x / p.pieces, from = blockIdx.x % p.pieces * p.piece, to = min(p.a.n, from + p.piece);
    Segment &of = p.segment[segment];
    const uint32_t number = of.number;
    if (number == 0) return;
    const bool weights = p.a.top_p < 1.0, limited = by_count(p, number);
    Range at[2] = {of.by_count, of.by_weight};
    Mass of_range = {0, 0};
    const Scale scale(p.a, of.least, of.most);
    if (limited) {
        read_bins(bins, *p.histogram(0, segment), weights);
        const Range within_it = at[0];
        at[0] = narrow<LONG_THREADS>(s, bins, within_it, {false, p.a.k, {0.0, 0.0}}, weights);
        if (weights) of_range = mass_in(bins, within_it, at[0]);
    }
    if (weights) {
        read_bins(bins, *p.histogram(1, segment), true);
        at[1] = narrow<LONG_THREADS>(s, bins, at[1], weight_goal(p.a, limited, at[0], of_range, of.total), true);
    }
    Bounds found[2] = {{NO_KEY, 0, 0, 0, 0}, {NO_KEY, 0, 0, 0, 0}};
    each_of_piece(p.a, segment, from, to, [&](uint32_t key, uint32_t index) {
        const uint32_t place_of = scale(key);
        const bool in[2] = {limited && key >= at[0].lo && key <= at[0].hi, weights && place_of >= at[1].lo && place_of <= at[1].hi};
        if (!in[0] && !in[1]) return;
#pragma unroll
        for (int r = 0; r < 2; ++r)
            if (in[r]) {
                found[r].least = min(found[r].least, key);
                found[r].most = max(found[r].most, key);
                ++found[r].number;
            }
        // (a place in the list for all of a wavefront's lanes that are here at once)
        const u64 here = __ballot(true);
        const int leader = __builtin_ctzll(here);
        uint32_t place = 0;
        if ((int)(threadIdx.x & 63) == leader) place = atomicAdd(&of.listed, (uint32_t)__builtin_popcountll(here));
        place = __shfl(place, leader) + __builtin_popcountll(here & ((1ull << (threadIdx.x & 63)) - 1));
        if (place < LIST) p.list[segment * LIST + place] = (u64)key << 32 | index;
    });
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const Bounds all = block_bounds(found[r], of_waves);
        if (threadIdx.x == 0) p.equal[r * p.segments * p.pieces + blockIdx.x] = {all.least, all.most, all.number, 0};
    }
    // the next kernel works on from here; blocks of this one read it no more once the last has counted its candidates, which is why the
    // ranges go to a place of their own
    if (blockIdx.x % p.pieces == 0 && threadIdx.x == 0) {
        Segment &next = p.segment[p.segments + segment];
        next.by_count = at[0];
        next.by_weight = at[1];
    }
}

// All of a segment, for a block by itself
struct Stream {
    static constexpr bool FITS = false;
    const Draws &a;
    uint64_t segment;
    template <class F>
    __device__ __forceinline__ void each(F &&f) const { each_of_piece(a, segment, 0, a.n, f); }
    // by index, a block's threads at a time
    __device__ uint32_t nth_from(uint64_t from, uint64_t to, uint32_t of, uint32_t j) const
    {
        const float *energy = a.energy + segment * a.n;
        const uint8_t *legal = a.legal ? a.legal + segment * a.n : nullptr;
        __shared__ uint32_t small[LONG_THREADS / 64], found;
        uint32_t passed = 0;
        if (threadIdx.x == 0) found = (uint32_t)(to - 1);
        for (uint64_t at = from; at < to; at += LONG_THREADS * 4) {
            uint32_t key[4] = {NO_KEY, NO_KEY, NO_KEY, NO_KEY}, mine = 0;
            const uint64_t here = at + threadIdx.x * 4;
            if (here < to) load_keys(energy, legal, here, to, key);
#pragma unroll
            for (int i = 0; i < 4; ++i) mine += key[i] == of;
            uint32_t up_to = passed + block_prefix<LONG_THREADS>(mine, small);
            uint32_t before = up_to - mine;
            if (before < j && up_to >= j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (key[i] == of && ++before == j) found = (uint32_t)(here + i);
            __syncthreads();
            for (int w = 0; w < LONG_THREADS / 64; ++w) passed += small[w];
            if (passed >= j) break;
        }
        __syncthreads();
        return found;
    }
    __device__ uint32_t nth(uint32_t of, uint32_t j) const { return nth_from(0, a.n, of, j); }
};

// The ends of both prefixes, a block a segment
__global__ __launch_bounds__(LONG_THREADS) void ends_kernel(const Long p)
{
    __shared__ Histogram bins;
    __shared__ LongScratch s;
    __shared__ Bounds of_waves[LONG_THREADS / 64];
    __shared__ uint32_t which_piece, left_there;
    const uint64_t segment = blockIdx.x;
    Segment &of = p.segment[segment];
    const bool weights = p.a.top_p < 1.0, any = p.a.k || weights;
    if (!any) { // (nothing went before but the bounds)
        const Bounds b = segment_bounds(p, segment, of_waves);
        if (threadIdx.x == 0) {
            of.least = b.least, of.most = b.most, of.number = b.number;
            of.cut = {b.most, 0xFFFFFFFFu};
        }
        return;
    }
    const uint32_t number = of.number, listed = of.listed;
    if (number == 0) return;
    const bool limited = by_count(p, number);
    const double best = (double)energy_of(of.least);
    const auto weight = [&](uint32_t key) { return weight_of(key, best, p.a.per_temperature); };
    const Stream stream = {p.a, segment};
    const Segment &ranges = p.segment[p.segments + segment];
    const Scale scale(p.a, of.least, of.most);

    const auto find = [&](const Range &at, const Goal &goal, int r) {
        if (listed <= LIST && at.number <= (uint32_t)LongScratch::LIST) {
            __syncthreads();
            if (threadIdx.x == 0) s.listed = 0;
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < listed; i += LONG_THREADS) {
                const u64 one = p.list[segment * LIST + i];
                const uint32_t key = (uint32_t)(one >> 32), place_of = r ? scale(key) : key;
                if (place_of < at.lo || place_of > at.hi) continue;
                const uint32_t place = atomicAdd(&s.listed, 1u);
                if (place < (uint32_t)LongScratch::LIST) s.list[place] = one;
            }
            sort_list<LONG_THREADS>(s, at.number);
            cut_sorted<LONG_THREADS>(s, at, goal, weights, weight);
            return;
        }
        const Equal *equal = p.equal + (r * p.segments + segment) * p.pieces;
        Bounds b = {NO_KEY, 0, 0, 0, 0};
        if (threadIdx.x < p.pieces) b = {equal[threadIdx.x].least, equal[threadIdx.x].most, equal[threadIdx.x].number, 0, 0};
        const uint32_t mine = b.number;
        b = block_bounds(b, of_waves);
        if (b.least != b.most) { // many, and not equal
            find_cut<LONG_THREADS>(s, bins, {of.least, of.most, number, 0, {0, 0}}, goal, weights, stream, weight);
            return;
        }
        Range one = at;
        one.lo = one.hi = b.least;
        const uint32_t j = last_of_equal(s, one, goal, weight(b.least));
        if (threadIdx.x == 0) which_piece = 0, left_there = 1;
        const uint32_t to = block_prefix<LONG_THREADS>(mine, s.small); // (and a barrier)
        if (to >= j && to - mine < j) {
            which_piece = threadIdx.x;
            left_there = j - (to - mine);
        }
        __syncthreads();
        const uint64_t from = which_piece * p.piece;
        const uint32_t index = stream.nth_from(from, min(p.a.n, from + p.piece), b.least, left_there);
        if (threadIdx.x == 0) s.cut = {b.least, index};
        __syncthreads();
    };

    Cut cut = {of.most, 0xFFFFFFFFu};
    double total = of.total;
    if (limited) {
        find(ranges.by_count, {false, p.a.k, {0.0, 0.0}}, 0);
        cut = s.cut;
        total = s.total.value();
        __syncthreads();
    }
    if (weights) {
        find(ranges.by_weight, {true, 0, {p.a.top_p * total, p.a.top_p * total}}, 1);
        if (within(s.cut.key, s.cut.index, cut)) cut = s.cut;
    }
    if (threadIdx.x == 0) of.cut = cut;
}

// Sums of the kept candidates' weights over strips, and over chunks of 64 strips: a wavefront a chunk
__global__ __launch_bounds__(256) void sums_kernel(const Long p)
{
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t chunk = (uint64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (chunk >= p.segments * p.chunks) return;
    const uint64_t segment = chunk / p.chunks, from = chunk % p.chunks * (64 * p.strip);
    const Segment &of = p.segment[segment];
    if (of.number == 0) return;
    const Cut cut = of.cut;
    const double best = (double)energy_of(of.least);
    const float *energy = p.a.energy + segment * p.a.n;
    const uint8_t *legal = p.a.legal ? p.a.legal + segment * p.a.n : nullptr;
    // sixteen lanes a strip, four strips at a time
    double all = 0.0;
    uint32_t kept = 0;
    for (uint32_t t = 0; t < 64; t += 4) {
        const uint64_t begin = from + (t + lane / 16) * p.strip, end = min(p.a.n, begin + p.strip);
        double sum = 0.0;
        for (uint64_t i = begin + lane % 16 * 4; i < end; i += 64) {
            uint32_t key[4];
            load_keys(energy, legal, i, end, key);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (key[k] == NO_KEY || !within(key[k], (uint32_t)(i + k), cut)) continue;
                const double w = weight_of(key[k], best, p.a.per_temperature);
                if (w >= p.a.min_p) {
                    sum += w;
                    ++kept;
                }
            }
        }
#pragma unroll
        for (int stride = 1; stride < 16; stride <<= 1) sum += lane_exchange(sum, stride);
        if (lane % 16 == 0) p.strip_sums[chunk * 64 + t + lane / 16] = sum;
        all += lane % 16 == 0 ? sum : 0.0;
    }
#pragma unroll
    for (int stride = 1; stride < 64; stride <<= 1) {
        all += lane_exchange(all, stride);
        kept += lane_exchange(kept, stride);
    }
    if (lane == 0) {
        p.chunk_sums[chunk] = all;
        p.chunk_counts[chunk] = kept;
    }
}

constexpr int DRAW_THREADS = 512, MOST_CHUNKS = 4096;

// Of a wavefront's lanes with a weight, the first whose sum passes the target, or the last
__device__ __forceinline__ int lane_of(double w, double to, double target)
{
    const u64 some = __ballot(w > 0.0), passes = __ballot(w > 0.0 && to > target);
    return passes ? __builtin_ctzll(passes) : some ? 63 - __builtin_clzll(some) : -1;
}

// A wavefront a draw: its chunk, its strip, its candidate
__global__ __launch_bounds__(DRAW_THREADS) void draws_kernel(const Long p, uint32_t blocks)
{
    __shared__ double to[MOST_CHUNKS];
    __shared__ double of_waves[DRAW_THREADS / 64];
    __shared__ uint32_t small[DRAW_THREADS / 64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, waves = DRAW_THREADS / 64;
    const uint64_t segment = blockIdx.x / blocks;
    const uint32_t first = blockIdx.x % blocks;
    const Segment &of = p.segment[segment];
    if (of.number == 0) {
        nothing_to_draw(p.a, segment, first * DRAW_THREADS + threadIdx.x, blocks * DRAW_THREADS);
        if (first == 0 && threadIdx.x == 0 && p.a.count) p.a.count[segment] = 0;
        return;
    }
    const double *sums = p.chunk_sums + segment * p.chunks;
    constexpr uint32_t EACH = MOST_CHUNKS / DRAW_THREADS;
    {
        double mine[EACH], sum = 0.0;
        uint32_t kept = 0;
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) {
            const uint32_t c = threadIdx.x * EACH + i;
            mine[i] = c < p.chunks ? sums[c] : 0.0;
            kept += c < p.chunks ? p.chunk_counts[segment * p.chunks + c] : 0;
            sum += mine[i];
        }
        double up_to = block_prefix<DRAW_THREADS>(sum, of_waves) - sum;
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) {
            up_to += mine[i];
            to[threadIdx.x * EACH + i] = up_to;
        }
        kept = block_prefix<DRAW_THREADS>(kept, small);
        if (first == 0 && threadIdx.x == DRAW_THREADS - 1 && p.a.count) p.a.count[segment] = kept;
    }
    __syncthreads();
    const Cut cut = of.cut;
    const double best = (double)energy_of(of.least), all = to[MOST_CHUNKS - 1];
    const float *energy = p.a.energy + segment * p.a.n;
    const uint8_t *legal = p.a.legal ? p.a.legal + segment * p.a.n : nullptr;
    for (uint32_t d = first * waves + wave; d < p.a.draws; d += blocks * waves) {
        const double target = fmax((double)p.a.uniform[segment * p.a.draws + d] * all, 0.0);
        uint32_t lo = 0, hi = p.chunks - 1;
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (to[mid] > target) hi = mid;
            else lo = mid + 1;
        }
        // (between two threads' chunks sums may differ in their last bit where nothing is added; and past the end the last one is wanted)
        while (!(sums[lo] > 0.0) && lo + 1 < p.chunks && all > target) ++lo;
        while (!(sums[lo] > 0.0) && lo > 0) --lo;
        double left = all > target ? target - (lo ? to[lo - 1] : 0.0) : __builtin_inf();
        const uint64_t chunk = segment * p.chunks + lo;
        const double of_strip = p.strip_sums[chunk * 64 + lane], strips_to = wave_sums(of_strip);
        const int t = max(lane_of(of_strip, strips_to, left), 0);
        left -= t ? __shfl(strips_to, t - 1) : 0.0;
        const uint64_t begin = ((uint64_t)lo * 64 + t) * p.strip, end = min(p.a.n, begin + p.strip);
        uint64_t found = begin;
        double of_found = 0.0;
        for (uint64_t i = begin; i < end; i += 64) {
            const uint32_t key = i + lane < end ? key_of(energy[i + lane], !legal || legal[i + lane]) : NO_KEY;
            double w = key != NO_KEY && within(key, (uint32_t)(i + lane), cut) ? weight_of(key, best, p.a.per_temperature) : 0.0;
            w = w >= p.a.min_p ? w : 0.0;
            const double up_to = wave_sums(w);
            const int l = lane_of(w, up_to, left);
            if (l >= 0) {
                found = i + l;
                of_found = __shfl(w, l);
            }
            if (__ballot(w > 0.0 && up_to > left)) break;
            left -= of_lane(up_to, 63);
        }
        if (lane == 0) {
            p.a.idx[segment * p.a.draws + d] = (uint32_t)found;
            if (p.a.logprob) p.a.logprob[segment * p.a.draws + d] = (float)log(of_found / all);
        }
    }
}

// ------------------------------------------------------------------------------------------------ long segments, few kept
//
// Where k is at most FEW, the k least of a segment fit a block's LDS.  The largest of all threads' least candidates is an upper bound for the
// k-th least once k threads have any (at 2^18 candidates a third of them lie below it), so one histogram of counts, linear in energy from the
// least up to that, has bins of some dozens where the k-th lies; what lies below goes to a list, which one block finishes, draws included.
// 64 segments of 2^18, k = 4096: range 16.6 us (the stream of energies and flags), histogram 15.9 (the same, out of the last-level cache, and
// the LDS atomics of a third of the candidates), list 31.5 (the same and places in the list, which all blocks of a segment take from one
// counter), draws 21 (one block a segment, a quarter of the compute units: its phases).

constexpr uint32_t FEW = 4096;

struct Few {
    Draws a;
    uint64_t segments;
    uint32_t pieces;
    uint64_t piece;
    Bounds *bounds;   // [segments][pieces]
    uint32_t *bins;   // [segments][pieces][BINS]
    uint32_t *joined; // [segments][BINS], of many pieces
    Segment *segment; // [segments]
    u64 *below, *at;  // [segments][FEW] each: candidates of the bins below the end's, and of that
    Equal *equal;     // [segments][pieces]: of the end's bin
};

// how many are kept, and the bound of the range that holds them
__device__ __forceinline__ uint32_t needed(const Few &p, const Bounds &b) { return min(p.a.k, b.number); }
__device__ __forceinline__ Linear range_of(const Few &p, const Bounds &b) { return Linear(b.least, b.threads >= needed(p, b) ? b.gate : b.most); }

// energies of a thread's share of a piece, so many at a time, and NaN where there is no legal candidate
constexpr int FEW_AHEAD = 4;
constexpr uint64_t FEW_ROUND = (uint64_t)LONG_THREADS * 4 * FEW_AHEAD; // of a block
struct Some {
    Chunk<float, 4> four[FEW_AHEAD];
    Chunk<uint8_t, 4> flags[FEW_AHEAD];
    // from candidate `at` of a segment on, up to `to`
    __device__ __forceinline__ void load(const float *energy, const uint8_t *legal, uint64_t at, uint64_t to)
    {
#pragma unroll
        for (int k = 0; k < FEW_AHEAD; ++k) {
            const uint64_t here = at + ((uint64_t)k * LONG_THREADS + threadIdx.x) * 4;
            if (here + 4 <= to) {
                four[k] = *reinterpret_cast<const Chunk<float, 4> *>(energy + here);
                if (legal) flags[k] = *reinterpret_cast<const Chunk<uint8_t, 4> *>(legal + here);
                else flags[k].v = 1;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool there = here + i < to;
                    four[k].v[i] = there ? energy[here + i] : 0.0f;
                    flags[k].v[i] = there && (!legal || legal[here + i]);
                }
            }
        }
    }
    __device__ __forceinline__ float energy(int k, int i) const { return flags[k].v[i] ? four[k].v[i] : __builtin_nanf(""); }
};

__global__ __launch_bounds__(LONG_THREADS) void few_bounds_kernel(const Few p)
{
    __shared__ Bounds of_waves[LONG_THREADS / 64];
    const uint64_t segment = blockIdx.x / p.pieces, from = blockIdx.x % p.pieces * p.piece, to = min(p.a.n, from + p.piece);
    Bounds b = {NO_KEY, 0, 0, 0, 0};
    each_of_piece(p.a, segment, from, to, [&](uint32_t key, uint32_t) {
        b.least = min(b.least, key);
        b.most = max(b.most, key);
        ++b.number;
    });
    if (b.number) b.gate = b.least, b.threads = 1;
    b = block_bounds(b, of_waves);
    if (threadIdx.x == 0) p.bounds[blockIdx.x] = b;
}

__device__ __forceinline__ Bounds few_bounds(const Few &p, uint64_t segment, Bounds *of_waves)
{
    Bounds b = {NO_KEY, 0, 0, 0, 0};
    if (threadIdx.x < p.pieces) b = p.bounds[segment * p.pieces + threadIdx.x];
    return block_bounds(b, of_waves);
}

__global__ __launch_bounds__(LONG_THREADS) void few_bins_kernel(const Few p)
{
    __shared__ uint32_t bins[BINS];
    __shared__ Bounds of_waves[LONG_THREADS / 64];
    const uint64_t segment = blockIdx.x / p.pieces, from = blockIdx.x % p.pieces * p.piece, to = min(p.a.n, from + p.piece);
    const float *energy = p.a.energy + segment * p.a.n;
    const uint8_t *legal = p.a.legal ? p.a.legal + segment * p.a.n : nullptr;
    Some now; // (on its way while the range is worked out)
    now.load(energy, legal, from, to);
    for (uint32_t b = threadIdx.x; b < BINS; b += LONG_THREADS) bins[b] = 0;
    const Bounds b = few_bounds(p, segment, of_waves); // (and barriers)
    if (blockIdx.x % p.pieces == 0 && threadIdx.x == 0) {
        Segment &of = p.segment[segment];
        of.least = b.least, of.most = b.most, of.number = b.number, of.listed = 0, of.listed_below = 0;
    }
    if (b.number == 0) return;
    const Linear range = range_of(p, b);
    for (uint64_t at = from;;) {
#pragma unroll
        for (int k = 0; k < FEW_AHEAD; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = now.energy(k, i);
                if (range.holds(e)) atomicAdd(&bins[range.bin(e)], 1u);
            }
        at += FEW_ROUND;
        if (at >= to) break;
        now.load(energy, legal, at, to);
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < BINS; i += LONG_THREADS) p.bins[(uint64_t)blockIdx.x * BINS + i] = bins[i];
}

constexpr uint32_t JOINED_ABOVE = 16; // pieces whose bins are not added up by every block that reads them

__global__ __launch_bounds__(LONG_THREADS) void few_join_kernel(const Few p)
{
    __shared__ uint32_t counts[LONG_THREADS / 64][64];
    const uint64_t segment = blockIdx.x / JOIN_BLOCKS;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, b = blockIdx.x % JOIN_BLOCKS * 64 + lane;
    uint32_t count = 0;
#pragma unroll 8
    for (uint32_t i = wave; i < p.pieces; i += LONG_THREADS / 64) count += p.bins[(segment * p.pieces + i) * BINS + b];
    counts[wave][lane] = count;
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < LONG_THREADS / 64; ++w) count += counts[w][lane];
    p.joined[segment * BINS + b] = count;
}

__global__ __launch_bounds__(LONG_THREADS) __attribute__((amdgpu_waves_per_eu(8))) void few_list_kernel(const Few p)
{
    __shared__ Bounds of_waves[LONG_THREADS / 64];
    __shared__ uint32_t small[LONG_THREADS / 64], found[3];
    const uint64_t segment = blockIdx.x / p.pieces, from = blockIdx.x % p.pieces * p.piece, to = min(p.a.n, from + p.piece);
    const float *energy = p.a.energy + segment * p.a.n;
    const uint8_t *legal = p.a.legal ? p.a.legal + segment * p.a.n : nullptr;
    Some now; // (on its way while the end's bin is looked for)
    now.load(energy, legal, from, to);
    // the bin of the last that is kept
    static_assert(BINS == 2 * LONG_THREADS, "two bins a thread");
    uint32_t two[2] = {0, 0};
    if (p.pieces > JOINED_ABOVE) {
        two[0] = p.joined[segment * BINS + 2 * threadIdx.x], two[1] = p.joined[segment * BINS + 2 * threadIdx.x + 1];
    } else {
        for (uint32_t first = 0; first < p.pieces; first += 4) {
            uint2 some[4];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                some[i] = first + i < p.pieces ? *reinterpret_cast<const uint2 *>(p.bins + (segment * p.pieces + first + i) * BINS + 2 * threadIdx.x)
                                               : make_uint2(0, 0);
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) two[0] += some[i].x, two[1] += some[i].y;
        }
    }
    const Bounds b = few_bounds(p, segment, of_waves);
    if (b.number == 0) return;
    const uint32_t need = needed(p, b);
    const uint32_t up_to = block_prefix<LONG_THREADS>(two[0] + two[1], small), before = up_to - two[0] - two[1];
    if (before < need && up_to >= need) {
        const bool second = before + two[0] < need;
        found[0] = 2 * threadIdx.x + second;
        found[1] = before + (second ? two[0] : 0);
        found[2] = two[second];
    }
    __syncthreads();
    const uint32_t end = found[0];
    Segment &of = p.segment[segment];
    if (blockIdx.x % p.pieces == 0 && threadIdx.x == 0) of.before = found[1], of.at_end = found[2], of.need = need;
    // (found is written again after the next barrier)

    const Linear range = range_of(p, b);
    Bounds equal = {NO_KEY, 0, 0, 0, 0};
    const float from_here = (float)end, to_here = end == BINS - 1 ? __builtin_inff() : (float)(end + 1);
    for (uint64_t here = from;;) {
        const uint32_t first = (uint32_t)here + threadIdx.x * 4;
        // which are below the end's bin and which in it: a place in a list for each of a block's at once
        uint32_t below = 0, at = 0;
        static_assert(FEW_AHEAD * 4 <= 32, "a bit a candidate");
#pragma unroll
        for (int k = 0; k < FEW_AHEAD; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = now.energy(k, i), place = range.place(e);
                const bool held = range.holds(e);
                below |= (uint32_t)(held && place < from_here) << (4 * k + i);
                at |= (uint32_t)(held && !(place < from_here) && place < to_here) << (4 * k + i);
            }
        static_assert(FEW_ROUND < 65536, "both counts in a word");
        const uint32_t counts = __builtin_popcount(below) << 16 | __builtin_popcount(at), counted = block_prefix<LONG_THREADS>(counts, small);
        __syncthreads();
        if (threadIdx.x == LONG_THREADS - 1) {
            found[1] = counted >> 16 ? atomicAdd(&of.listed_below, counted >> 16) : 0;
            found[2] = counted & 0xFFFF ? atomicAdd(&of.listed, counted & 0xFFFF) : 0;
        }
        __syncthreads();
        uint32_t place_below = found[1] + (counted >> 16) - (counts >> 16), place_at = found[2] + (counted & 0xFFFF) - (counts & 0xFFFF);
        // few of a thread's are listed; they are read again, some at once
        for (uint32_t both = below | at; both;) {
            uint32_t bit[4];
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                bit[i] = both ? __builtin_ctz(both) : 32;
                both &= both - (both != 0);
                e[i] = bit[i] < 32 ? energy[first + bit[i] / 4 * (LONG_THREADS * 4) + bit[i] % 4] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (bit[i] == 32) break;
                const uint32_t key = key_of(e[i], true);
                const u64 one = (u64)key << 32 | (first + bit[i] / 4 * (LONG_THREADS * 4) + bit[i] % 4);
                if (below >> bit[i] & 1) {
                    if (place_below < FEW) p.below[segment * FEW + place_below] = one;
                    ++place_below;
                } else {
                    if (place_at < FEW) p.at[segment * FEW + place_at] = one;
                    ++place_at;
                    equal.least = min(equal.least, key);
                    equal.most = max(equal.most, key);
                    ++equal.number;
                }
            }
        }
        here += FEW_ROUND;
        if (here >= to) break;
        now.load(energy, legal, here, to);
    }
    equal = block_bounds(equal, of_waves);
    if (threadIdx.x == 0) p.equal[blockIdx.x] = {equal.least, equal.most, equal.number, 0};
}

struct FewLds {
    LongScratch s;
    Bounds of_waves[LONG_THREADS / 64];
    double real[LONG_THREADS / 64];
    uint32_t entries, which_piece, left_there;
    u64 kept[FEW];
    double to[FEW];
    union {
        Histogram bins;
        struct {
            u64 scattered[FEW];
            uint32_t start[BINS + 1];
        };
    };
};

// Candidates in the LDS, in any order, up to a cut
struct Listed {
    static constexpr bool FITS = false;
    const u64 *kept;
    uint32_t number;
    uint32_t &found;
    template <class F>
    __device__ __forceinline__ void each(F &&f) const
    {
        for (uint32_t i = threadIdx.x; i < number; i += LONG_THREADS) f((uint32_t)(kept[i] >> 32), (uint32_t)kept[i]);
    }
    __device__ uint32_t nth(uint32_t of, uint32_t j) const
    {
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < number; i += LONG_THREADS) {
            if ((uint32_t)(kept[i] >> 32) != of) continue;
            uint32_t rank = 1;
            for (uint32_t o = 0; o < number; ++o) rank += (uint32_t)(kept[o] >> 32) == of && (uint32_t)kept[o] < (uint32_t)kept[i];
            if (rank == j) found = (uint32_t)kept[i];
        }
        __syncthreads();
        return found;
    }
};

__global__ __launch_bounds__(LONG_THREADS) void few_draws_kernel(const Few p)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    FewLds &l = *reinterpret_cast<FewLds *>(lds);
    LongScratch &s = l.s;
    const Draws &a = p.a;
    const uint64_t segment = blockIdx.x;
    const Segment &of = p.segment[segment];
    if (of.number == 0) {
        nothing_to_draw(a, segment, threadIdx.x, LONG_THREADS);
        if (threadIdx.x == 0 && a.count) a.count[segment] = 0;
        return;
    }
    const uint32_t need = of.need, at_end = of.at_end, below = of.before;
    const double best = (double)energy_of(of.least);
    const auto weight = [&](uint32_t key) { return weight_of(key, best, a.per_temperature); };
    const Stream stream = {a, segment};

    // the k least
    const u64 *list = p.at + segment * FEW;
    if (at_end <= (uint32_t)LongScratch::LIST) {
        for (uint32_t i = threadIdx.x; i < at_end; i += LONG_THREADS) s.list[i] = list[i];
        sort_list<LONG_THREADS>(s, at_end);
        if (threadIdx.x == 0) {
            const u64 one = s.sorted[min(max(need - below, 1u), at_end) - 1];
            s.cut = {(uint32_t)(one >> 32), (uint32_t)one};
        }
    } else {
        const Equal *equal = p.equal + segment * p.pieces;
        Bounds b = {NO_KEY, 0, 0, 0, 0};
        if (threadIdx.x < p.pieces) b = {equal[threadIdx.x].least, equal[threadIdx.x].most, equal[threadIdx.x].number, 0, 0};
        const uint32_t mine = b.number, j = need - below;
        b = block_bounds(b, l.of_waves);
        if (b.least == b.most) { // all equal: by index, from the piece that holds the last one
            if (threadIdx.x == 0) l.which_piece = 0, l.left_there = 1;
            const uint32_t to = block_prefix<LONG_THREADS>(mine, s.small); // (and a barrier)
            if (to >= j && to - mine < j) {
                l.which_piece = threadIdx.x;
                l.left_there = j - (to - mine);
            }
            __syncthreads();
            const uint64_t from = l.which_piece * p.piece;
            const uint32_t index = stream.nth_from(from, min(a.n, from + p.piece), b.least, l.left_there);
            if (threadIdx.x == 0) s.cut = {b.least, index};
        } else {
            // so many next to each other, or one candidate so far below all others that these share a bin: this block goes over the segment again
            // (64 segments of 2^18, k = 4096, with such a candidate in each: 333 us, 84 without; one of 2^24 10.9 ms, 83 us without)
            find_cut<LONG_THREADS>(s, l.bins, {of.least, of.most, of.number, 0, {0, 0}}, {false, need, {0.0, 0.0}}, false, stream, weight);
        }
    }
    if (threadIdx.x == 0) l.entries = 0;
    __syncthreads();
    Cut cut = s.cut;
    const auto keep = [&](u64 one) {
        const uint32_t place = atomicAdd(&l.entries, 1u);
        if (place < FEW) l.kept[place] = one;
    };
    if (at_end <= FEW) {
        for (uint32_t i = threadIdx.x; i < below; i += LONG_THREADS) keep(p.below[segment * FEW + i]);
        for (uint32_t i = threadIdx.x; i < at_end; i += LONG_THREADS)
            if (within((uint32_t)(list[i] >> 32), (uint32_t)list[i], cut)) keep(list[i]);
    } else { // (more than the list takes: from the candidates themselves)
        stream.each([&](uint32_t key, uint32_t index) {
            if (within(key, index, cut)) keep((u64)key << 32 | index);
        });
    }
    __syncthreads();
    const uint32_t entries = min(l.entries, FEW);

    // a share of their weight
    if (a.top_p < 1.0 && entries > 1) {
        Goal goal = {true, 0, {0.0, 0.0}, a.top_p};
        if (entries <= (uint32_t)LongScratch::LIST) { // (no histogram will be made)
            Mass mine = {0, 0};
            for (uint32_t i = threadIdx.x; i < entries; i += LONG_THREADS) mine = mine + mass_of(weight((uint32_t)(l.kept[i] >> 32)));
            goal.target[0] = goal.target[1] = a.top_p * block_total<LONG_THREADS>(s, mine).value();
        }
        const Listed listed = {l.kept, entries, s.listed};
        find_cut_of<LONG_THREADS>(s, l.bins, of.least, cut.key, entries, goal, true, listed, weight);
        cut = s.cut;
        __syncthreads();
    }

    // by index: into buckets of neighbouring ones, and in order within each
    const uint32_t shift = 64 - __builtin_clzll((a.n - 1) | 1) > (int)BIN_BITS ? 64 - __builtin_clzll((a.n - 1) | 1) - BIN_BITS : 0;
    for (uint32_t i = threadIdx.x; i <= BINS; i += LONG_THREADS) l.start[i] = 0;
    __syncthreads();
    const auto stays = [&](u64 one) {
        const uint32_t key = (uint32_t)(one >> 32);
        return within(key, (uint32_t)one, cut) && (a.min_p <= 0.0 || weight(key) >= a.min_p);
    };
    constexpr int EACH = FEW / LONG_THREADS;
    u64 mine[EACH];
    uint32_t bucket[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const uint32_t e = threadIdx.x + i * LONG_THREADS;
        bucket[i] = BINS;
        if (e < entries) {
            mine[i] = l.kept[e];
            if (stays(mine[i])) {
                bucket[i] = (uint32_t)mine[i] >> shift;
                atomicAdd(&l.start[bucket[i]], 1u);
            }
        }
    }
    __syncthreads();
    const uint32_t count[2] = {l.start[2 * threadIdx.x], l.start[2 * threadIdx.x + 1]};
    const uint32_t up_to = block_prefix<LONG_THREADS>(count[0] + count[1], s.small); // (and barriers)
    l.start[2 * threadIdx.x] = up_to - count[1] - count[0];
    l.start[2 * threadIdx.x + 1] = up_to - count[1];
    if (threadIdx.x == LONG_THREADS - 1) l.entries = up_to;
    __syncthreads();
    const uint32_t kept = l.entries;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (bucket[i] < BINS) l.scattered[atomicAdd(&l.start[bucket[i]], 1u)] = (u64)(uint32_t)mine[i] << 32 | (uint32_t)(mine[i] >> 32);
    __syncthreads();
    // (a bucket's start is now its end)
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (bucket[i] == BINS) continue;
        const uint32_t from = bucket[i] ? l.start[bucket[i] - 1] : 0, to = l.start[bucket[i]];
        uint32_t place = from;
        for (uint32_t o = from; o < to; ++o) place += (uint32_t)(l.scattered[o] >> 32) < (uint32_t)mine[i];
        l.kept[place] = mine[i];
    }
    __syncthreads();

    double w[EACH], sum = 0.0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const uint32_t e = threadIdx.x * EACH + i;
        w[i] = e < kept ? weight((uint32_t)(l.kept[e] >> 32)) : 0.0;
        sum += w[i];
    }
    double to = block_prefix<LONG_THREADS>(sum, l.real) - sum;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        to += w[i];
        l.to[threadIdx.x * EACH + i] = to;
    }
    if (threadIdx.x == 0 && a.count) a.count[segment] = kept;
    __syncthreads();
    const double all = l.to[kept - 1];
    for (uint32_t d = threadIdx.x; d < a.draws; d += LONG_THREADS) {
        const double target = fmax((double)a.uniform[segment * a.draws + d] * all, 0.0);
        uint32_t lo = 0, hi = kept - 1;
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (l.to[mid] > target) hi = mid;
            else lo = mid + 1;
        }
        double x = weight((uint32_t)(l.kept[lo] >> 32));
        while (!(x > 0.0) && lo + 1 < kept && all > target) x = weight((uint32_t)(l.kept[++lo] >> 32));
        while (!(x > 0.0) && lo > 0) x = weight((uint32_t)(l.kept[--lo] >> 32));
        a.idx[segment * a.draws + d] = (uint32_t)l.kept[lo];
        if (a.logprob) a.logprob[segment * a.draws + d] = (float)log(x / all);
    }
}

// k = 1: the first of the least, in every draw
__global__ __launch_bounds__(LONG_THREADS) void least_kernel(const Few p)
{
    __shared__ u64 of_waves[LONG_THREADS / 64];
    const uint64_t segment = blockIdx.x / p.pieces, from = blockIdx.x % p.pieces * p.piece, to = min(p.a.n, from + p.piece);
    u64 least = ~0ull;
    each_of_piece(p.a, segment, from, to, [&](uint32_t key, uint32_t index) { least = min(least, (u64)key << 32 | index); });
#pragma unroll
    for (int stride = 1; stride < 64; stride <<= 1) least = min(least, (u64)lane_exchange((uint64_t)least, stride));
    if ((threadIdx.x & 63) == 0) of_waves[threadIdx.x / 64] = least;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < LONG_THREADS / 64; ++w) least = min(least, of_waves[w]);
    p.below[blockIdx.x] = least;
}
__global__ __launch_bounds__(256) void least_draws_kernel(const Few p)
{
    const uint64_t segment = blockIdx.x;
    __shared__ u64 of_waves[4];
    u64 least = ~0ull;
    for (uint32_t i = threadIdx.x; i < p.pieces; i += 256) least = min(least, p.below[segment * p.pieces + i]);
#pragma unroll
    for (int stride = 1; stride < 64; stride <<= 1) least = min(least, (u64)lane_exchange((uint64_t)least, stride));
    if ((threadIdx.x & 63) == 0) of_waves[threadIdx.x / 64] = least;
    __syncthreads();
    least = min(min(of_waves[0], of_waves[1]), min(of_waves[2], of_waves[3]));
    if (threadIdx.x == 0 && p.a.count) p.a.count[segment] = least != ~0ull;
    if (least == ~0ull) {
        nothing_to_draw(p.a, segment, threadIdx.x, 256);
        return;
    }
    for (uint32_t d = threadIdx.x; d < p.a.draws; d += 256) {
        p.a.idx[segment * p.a.draws + d] = (uint32_t)least;
        if (p.a.logprob) p.a.logprob[segment * p.a.draws + d] = 0.0f;
    }
}

// ------------------------------------------------------------------------------------------------ host

constexpr uint64_t SHORT = 16384;

uint64_t padded(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

// sizes of a call on long segments, and the places in its workspace
uint64_t lay_out(Long &p, void *ws)
{
    const uint64_t n = p.a.n, s = p.segments;
    uint64_t pieces = (MOST_PIECES + s - 1) / s;
    if (pieces > (n + 16383) / 16384) pieces = (n + 16383) / 16384;
    p.piece = ((n + pieces - 1) / pieces + 4095) / 4096 * 4096;
    p.pieces = (uint32_t)((n + p.piece - 1) / p.piece);
    p.strip = 64;
    while ((n + 64 * p.strip - 1) / (64 * p.strip) > MOST_CHUNKS) p.strip *= 2;
    p.chunks = (uint32_t)((n + 64 * p.strip - 1) / (64 * p.strip));
    char *at = (char *)ws;
    const auto take = [&](uint64_t bytes) {
        char *here = at;
        at += padded(bytes);
        return (void *)here;
    };
    p.segment = (Segment *)take(2 * s * sizeof(Segment));
    p.bounds = (Bounds *)take(s * p.pieces * sizeof(Bounds));
    p.parts = (Histogram *)take(2 * s * p.pieces * sizeof(Histogram));
    p.whole = (Histogram *)take(p.pieces > 1 ? 2 * s * sizeof(Histogram) : 0);
    p.list = (u64 *)take(s * LIST * sizeof(u64));
    p.equal = (Equal *)take(2 * s * p.pieces * sizeof(Equal));
    p.strip_sums = (double *)take(s * p.chunks * 64 * sizeof(double));
    p.chunk_sums = (double *)take(s * p.chunks * sizeof(double));
    p.chunk_counts = (uint32_t *)take(s * p.chunks * sizeof(uint32_t));
    return (uint64_t)(at - (char *)ws);
}

uint64_t lay_out_few(Few &p, void *ws)
{
    const uint64_t n = p.a.n, s = p.segments;
    uint64_t pieces = (MOST_PIECES + s - 1) / s;
    if (pieces > (n + 32767) / 32768) pieces = (n + 32767) / 32768;
    p.piece = ((n + pieces - 1) / pieces + 4095) / 4096 * 4096;
    p.pieces = (uint32_t)((n + p.piece - 1) / p.piece);
    char *at = (char *)ws;
    const auto take = [&](uint64_t bytes) {
        char *here = at;
        at += padded(bytes);
        return (void *)here;
    };
    p.segment = (Segment *)take(s * sizeof(Segment));
    p.bounds = (Bounds *)take(s * p.pieces * sizeof(Bounds));
    p.bins = (uint32_t *)take(s * p.pieces * BINS * 4);
    p.joined = (uint32_t *)take(p.pieces > JOINED_ABOVE ? s * BINS * 4 : 0);
    p.below = (u64 *)take(s * FEW * sizeof(u64));
    p.at = (u64 *)take(s * FEW * sizeof(u64));
    p.equal = (Equal *)take(s * p.pieces * sizeof(Equal));
    return (uint64_t)(at - (char *)ws);
}

// Whether the least of a segment are put in order first: not so many that a list would seldom take the end's bin too, and few where the other way
// is short, for k alone (1024 segments of 6400: k = 16 32 us by this, 36 otherwise, k = 64 41 and 36; 512 of 16 384, k = 64, 59 and 39; 4096 of
// 1000 51 and 40) and long segments (with a share 512 of 16 384, k = 64, 59 us by this, k = 192 67; k = 300, the other way, 64).  Of others with a
// share k = 192 takes 56 (1024 of 6400) and 65 (4096 of 1000), k = 300 the other way 75 and 86.  A kernel of its own: both in one take more
// registers than there are (16 384 by share alone twice the time).
bool is_fewest(const Draws &a)
{
    const uint32_t most = a.top_p < 1.0 ? (a.n <= 8192 ? 192 : 64) : a.n > 1024 && a.n <= 8192 ? 48 : 0;
    return a.n > 256 && a.k > 1 && a.k <= most;
}

template <int THREADS, int EACH, bool FEWEST>
int32_t launch_short_of(const Draws &a, uint32_t segments, hipStream_t st)
{
    constexpr int bytes = sizeof(Short<THREADS, EACH>);
    const auto kernel = short_kernel<THREADS, EACH, FEWEST>;
    if (bytes > 65536) ECK_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    hipLaunchKernelGGL(kernel, dim3(segments), dim3(THREADS), bytes, st, a);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}
template <int THREADS, int EACH>
int32_t launch_short(const Draws &a, uint32_t segments, hipStream_t st)
{
    if constexpr (Short<THREADS, EACH>::BINNED)
        if (is_fewest(a)) return launch_short_of<THREADS, EACH, true>(a, segments, st);
    return launch_short_of<THREADS, EACH, false>(a, segments, st);
}

int32_t launch_few(const Draws &a, uint32_t segments, void *ws, hipStream_t st)
{
    Few p;
    p.a = a;
    p.segments = segments;
    lay_out_few(p, ws);
    const dim3 pieces(segments * p.pieces), threads(LONG_THREADS);
    if (a.k == 1) {
        hipLaunchKernelGGL(least_kernel, pieces, threads, 0, st, p);
        hipLaunchKernelGGL(least_draws_kernel, dim3(segments), dim3(256), 0, st, p);
    } else {
        ECK_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(few_draws_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(FewLds)));
        hipLaunchKernelGGL(few_bounds_kernel, pieces, threads, 0, st, p);
        hipLaunchKernelGGL(few_bins_kernel, pieces, threads, 0, st, p);
        if (p.pieces > JOINED_ABOVE) hipLaunchKernelGGL(few_join_kernel, dim3(segments * JOIN_BLOCKS), threads, 0, st, p);
        hipLaunchKernelGGL(few_list_kernel, pieces, threads, 0, st, p);
        hipLaunchKernelGGL(few_draws_kernel, dim3(segments), threads, sizeof(FewLds), st, p);
    }
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

int32_t launch_long(const Draws &a, uint32_t segments, void *ws, hipStream_t st)
{
    Long p;
    p.a = a;
    p.segments = segments;
    lay_out(p, ws);
    const dim3 pieces(segments * p.pieces), threads(LONG_THREADS);
    const bool weights = a.top_p < 1.0;
    hipLaunchKernelGGL(bounds_kernel, pieces, threads, 0, st, p);
    if (a.k || weights) {
        const auto join = [&](int which) {
            if (p.pieces > 1) hipLaunchKernelGGL(join_bins_kernel, dim3(segments * JOIN_BLOCKS), threads, 0, st, p, which);
        };
        constexpr int one = sizeof(Histogram);
        const int bins = a.k && weights ? 2 * one : one;
        ECK_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(first_bins_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bins));
        ECK_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(second_bins_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bins));
        hipLaunchKernelGGL(first_bins_kernel, pieces, threads, bins, st, p);
        if (a.k) join(0);
        if (weights) join(1);
        hipLaunchKernelGGL(second_bins_kernel, pieces, threads, bins, st, p);
        if (a.k) join(0);
        if (weights) join(1);
        hipLaunchKernelGGL(list_kernel, pieces, threads, 0, st, p);
    }
    hipLaunchKernelGGL(ends_kernel, dim3(segments), threads, 0, st, p);
    hipLaunchKernelGGL(sums_kernel, dim3((uint32_t)((p.segments * p.chunks + 3) / 4)), dim3(256), 0, st, p);
    // some draws a wavefront, so that a block's sums over chunks serve several
    const uint32_t most = (a.draws + DRAW_THREADS / 64 - 1) / (DRAW_THREADS / 64), wanted = (1024 + segments - 1) / segments;
    const uint32_t blocks = most < wanted ? most : wanted;
    hipLaunchKernelGGL(draws_kernel, dim3(segments * blocks), dim3(DRAW_THREADS), 0, st, p, blocks);
    ECK_HIP_TRY(hipGetLastError());
    return ECK_OK;
}

} // namespace
} // namespace eck

using namespace eck;

extern "C" uint64_t sample_select_workspace_bytes(uint64_t n, uint32_t n_segments, uint32_t draws)
{
    if (n == 0 || n_segments == 0 || draws == 0 || n % n_segments || n / n_segments > MOST_CANDIDATES || n_segments > MOST_SEGMENTS || draws > MOST_DRAWS)
        return 0;
    if (n / n_segments <= SHORT) return 0;
    Long p; // (the query does not know k: room for either way)
    p.a.n = n / n_segments;
    p.segments = n_segments;
    Few f;
    f.a.n = p.a.n;
    f.segments = n_segments;
    const uint64_t all = lay_out(p, nullptr), few = lay_out_few(f, nullptr);
    return all > few ? all : few;
}

extern "C" int32_t sample_select(const float *energy, const uint8_t *legal, uint64_t n, uint32_t n_segments, const float *uniform, uint32_t draws,
                                 float temperature, uint32_t k, float top_p, float min_p, uint32_t *idx_out, float *logprob_out,
                                 uint32_t *count_out, void *ws, uint64_t ws_bytes, void *stream)
{
    if (!energy || !uniform || !idx_out || n == 0 || n_segments == 0 || draws == 0) return ECK_EINVAL;
    if (!(temperature >= 0.0f && temperature < __builtin_inff()) || !(top_p > 0.0f && top_p <= 1.0f) || !(min_p >= 0.0f && min_p <= 1.0f)) return ECK_EINVAL;
    if (n % n_segments) return ECK_ESHAPE;
    if (n / n_segments > MOST_CANDIDATES || n_segments > MOST_SEGMENTS || draws > MOST_DRAWS) return ECK_EUNSUPPORTED;
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
    const hipStream_t st = as_stream(stream);
    if (a.n <= 256) return launch_short<64, 4>(a, n_segments, st);
    if (a.n <= 1024) return launch_short<256, 4>(a, n_segments, st);
    if (a.n <= 4096) return launch_short<512, 8>(a, n_segments, st);
    if (a.n <= 8192) return launch_short<1024, 8>(a, n_segments, st);
    if (a.n <= SHORT) return launch_short<1024, 16>(a, n_segments, st);
    if (a.k && a.k <= FEW) return launch_few(a, n_segments, ws, st);
    return launch_long(a, n_segments, ws, st);
}
