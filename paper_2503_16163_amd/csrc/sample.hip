// Choice of a token per row of logits: temperature, top-k, top-p, min-p, from a given random number.
//
// All three limits keep a prefix of the row in the order of its logits (the lower index first among equals), and so is the
// choice a place in that order: the first element at which a count, or the running sum of the weights, reaches a target.  Nothing
// of the row's length is sorted for it.
//   - Few tokens kept: those that can be are listed in LDS, sorted there, and their weights summed in order.  With top_k the list is what
//     is not below the k-th largest of the threads' own maxima, or of the 16-byte vectors' (there are k such elements at least, and hardly more);
//     without it, what a histogram over the logarithm of the weights puts in or before the bin where the kept mass ends.
//   - Many: the elements of the histogram's bins that hold the targets are listed; a bin that holds too many is taken apart further, by the bits
//     of its logits.
// An element's weight is r 2^(-bin / 64): the power of the bin, of which there are 64 per power of two, and a whole number r of units 2^-R,
// so that a bin's sum is exact in whatever order it is made; sums of bins and of listed elements are binary64 in a fixed order.
#include "operators.h"
#include "wave_ops.h"

#include <algorithm>
#include <cmath>

namespace specache {
namespace {

constexpr int kThreads = 1024, kWavesPerRow = kThreads / 64;
constexpr int kBins = 2048;            // two per thread
constexpr float kBinsPerLog2 = 64.0f;  // 32 powers of two of the weights; what is lighter shares the last bin
constexpr int kList = 2048;            // elements that are sorted at once
constexpr int kFew = 256;              // a list so short is sorted by comparing each with all the others,
constexpr int kRanked = 1024;          // of a bin's so many each is compared with all the others
constexpr int kTable = 32768;          // vectors of a row whose largest logits are kept (32 of each thread)
// top_k by the threads' largest logits, by the vectors': us, 256 rows of 128256 / 17 of 49999 in fp32, top_k 100 by the one 22.3 / 13.0, by the other 23.8 / 14.4;
// 200 24.6 / 15.7 and 25.7 / 16.3; 400 25.9 / 15.7 by the vectors', 1400 36 / 20.
constexpr int kFewMaxima = 256, kMostByMaxima = 1536;
constexpr int kMostVocab = 1 << 20;

struct SampleArgs {
    const void* logits;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t* top_k;
    int32_t* tokens;
    int64_t row_stride;
    int vocab;
    int unit_log2, count_shift;        // R; a bin is its elements' number << count_shift | the sum of their r
};

struct Shared {
    uint64_t bins[kBins + 64];         // the last ones take what is not allowed, a lane each
    uint64_t list[kList];              // descending_key << 32 | index: ascending is the order of the row
    uint64_t sorted[kList];
    double wave_mass[kWavesPerRow];
    uint32_t wave_count[kWavesPerRow];
    float wave_most[kWavesPerRow];
    int wave_first[kWavesPerRow];
    uint32_t list_n, key_low, key_high, found_bin, found_count;
    double found_mass;
    int found_index;
    double mark_mass[3];
    uint32_t mark_count[3];
    uint64_t border_units;
    double power[64];                  // 2^(-i / 64) / 2^R
    uint16_t vector_most[kTable];      // of a thread's own vectors: the largest logit's key, its upper half rounded up
    uint32_t places[kBins];            // sort_list: elements of a bin, then the place of its first
    uint32_t crowded;
};

template <typename T> __device__ __forceinline__ float logit_of(T x) { return (float)x; }

// f(vector, first index, elements, number of the vector or -1) over a row: 16-byte loads between the first and the last aligned address, four ahead, single elements
// before and behind.  A thread's calls come in ascending order of the index.
template <typename T, typename F>
__device__ __forceinline__ void each_vector(const T* row, int n, F&& f) {
    constexpr int kVec = 16 / sizeof(T), kAhead = 4;
    typedef T Vec __attribute__((ext_vector_type(kVec)));
    const int head = min(n, (int)((16 - (uintptr_t)row % 16) % 16 / sizeof(T)));
    const int vecs = (n - head) / kVec, tail = head + vecs * kVec;
    if ((int)threadIdx.x < head) {
        Vec x{};
        x[0] = row[threadIdx.x];
        f(x, (int)threadIdx.x, 1, -1);
    }
    const Vec* body = (const Vec*)(row + head);
    int v = threadIdx.x;
    for (; v + (kAhead - 1) * kThreads < vecs; v += kAhead * kThreads) {
        Vec x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) x[i] = body[v + i * kThreads];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) f(x[i], head + (v + i * kThreads) * kVec, kVec, v + i * kThreads);
    }
    if (v < vecs) {
        Vec x[kAhead - 1];
#pragma unroll
        for (int i = 0; i < kAhead - 1; ++i) x[i] = body[min(v + i * kThreads, vecs - 1)];
#pragma unroll
        for (int i = 0; i < kAhead - 1; ++i)
            if (v + i * kThreads < vecs) f(x[i], head + (v + i * kThreads) * kVec, kVec, v + i * kThreads);
    }
    if (tail + (int)threadIdx.x < n) {
        Vec x{};
        x[0] = row[tail + threadIdx.x];
        f(x, tail + (int)threadIdx.x, 1, -1);
    }
}
// f(logit, index) for every allowed token
template <typename T, typename F>
__device__ __forceinline__ void each(const T* row, int n, F&& f) {
    constexpr int kVec = 16 / sizeof(T);
    each_vector(row, n, [&](const auto& x, int i, int elements, int) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const float l = logit_of(x[e]);
            if (l > -INFINITY && e < elements) f(l, i + e);   // (false for NaN as well)
        }
    });
}

// f(logit, index) for every allowed token inside (hardly any: a vector without one costs its comparisons)
template <typename T, typename Inside, typename F>
__device__ __forceinline__ void each_where(const T* row, int n, Inside&& inside, F&& f) {
    constexpr int kVec = 16 / sizeof(T);
    each_vector(row, n, [&](const auto& x, int i, int elements, int) {
        bool any = false;
#pragma unroll
        for (int e = 0; e < kVec; ++e) any |= inside(logit_of(x[e]));
        if (any)
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const float l = logit_of(x[e]);
                if (inside(l) && l > -INFINITY && e < elements) f(l, i + e);
            }
    });
}
// The same for the tokens that are not below `least`; vectors that hold none are not read again where the row's table says so.
template <typename T, typename F>
__device__ __forceinline__ void each_from(const Shared& s, const T* row, int n, float least, F&& f) {
    constexpr int kVec = 16 / sizeof(T);
    typedef T Vec __attribute__((ext_vector_type(kVec)));
    const int head = min(n, (int)((16 - (uintptr_t)row % 16) % 16 / sizeof(T)));
    const int vecs = (n - head) / kVec, tail = head + vecs * kVec;
    if (vecs > kTable) {
        each_where(row, n, [&](float l) { return l >= least; }, f);
        return;
    }
    const auto one = [&](T x, int i) {
        const float l = logit_of(x);
        if (l >= least && l > -INFINITY) f(l, i);
    };
    if ((int)threadIdx.x < head) one(row[threadIdx.x], threadIdx.x);
    if (tail + (int)threadIdx.x < n) one(row[tail + threadIdx.x], tail + threadIdx.x);
    const uint32_t from = float_to_key(least) >> 16;
    uint32_t wanted = 0;
    for (int v = threadIdx.x, i = 0; v < vecs; v += kThreads, ++i) wanted |= (uint32_t)(s.vector_most[v] >= from) << i;
    constexpr int kAhead = 4;
    while (wanted) {
        Vec x[kAhead];
        int v[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j, wanted &= wanted - 1) {
            v[j] = wanted ? threadIdx.x + __builtin_ctz(wanted) * kThreads : -1;
            if (wanted) x[j] = ((const Vec*)(row + head))[v[j]];
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (v[j] >= 0)
#pragma unroll
                for (int e = 0; e < kVec; ++e) one(x[j][e], head + v[j] * kVec + e);
    }
}
struct Range {
    float least, most;
    __device__ __forceinline__ bool operator()(float l) const { return l >= least && l <= most; }
};

struct Weights {
    float most, bins_per_logit, unit;      // bins_per_logit: above 0; unit: 2^R
    const double* power;
    // bins below the largest logit: never falls as the logit does (0 for the difference of two infinities)
    __device__ __forceinline__ float depth(float l) const { return fmaxf((most - l) * bins_per_logit, 0.0f); }
    __device__ __forceinline__ uint32_t bin_of(float depth) const { return (uint32_t)fminf(depth, kBins - 1.0f); }
    // logits between which all elements of bins first to last lie (and few others): the depth is turned round with room for its roundings
    __device__ __forceinline__ float below(uint32_t last) const {
        if (last >= kBins - 1 || !(most < INFINITY)) return -INFINITY;
        const float d = ((float)last + 1.01f) / bins_per_logit;
        return most - d - (d * 0x1p-16f + fabsf(most) * 0x1p-20f);
    }
    __device__ __forceinline__ float above(uint32_t first) const {
        if (!first || !(most < INFINITY)) return INFINITY;
        const float d = ((float)first - 0.01f) / bins_per_logit;
        return most - d + (d * 0x1p-16f + fabsf(most) * 0x1p-20f);
    }
    // 2^(-f / 64) for a place f from 0 to 1 in a bin: 1 + f (c1 + f c2), off by 2^-26.8 at most (the best such polynomial)
    __device__ __forceinline__ uint32_t units_of_place(float f) const {
        return (uint32_t)fmaf(f, fmaf(f, 0x1.e984d6p-15f, -0x1.62e36cp-7f) * unit, unit + 0.5f);
    }
    __device__ __forceinline__ uint32_t units(float depth, uint32_t bin) const {
        if (bin < kBins - 1) return units_of_place(depth - (float)bin);
        return (uint32_t)fmaf(__builtin_amdgcn_exp2f(((float)bin - depth) * (1.0f / kBinsPerLog2)), unit, 0.5f);
    }
    __device__ __forceinline__ double of_bin(uint64_t units, uint32_t bin) const {
        return __builtin_amdgcn_ldexp((double)units * power[bin % 64], -(int)(bin / 64));
    }
    __device__ __forceinline__ double of(float l) const {
        const float d = depth(l);
        const uint32_t b = bin_of(d);
        return of_bin(units(d, b), b);
    }
};

__device__ __forceinline__ uint32_t descending_key(float l) { return ~float_to_key(l); }
__device__ __forceinline__ float logit_of_key(uint32_t descending) {
    const uint32_t k = ~descending;
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

// the sums of (count, mass) over the threads before this one, in the threads' order
__device__ __forceinline__ void sums_before(Shared& s, uint32_t& count, double& mass) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t c = count;
    double m = mass;
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t cc = __shfl_up(c, d);
        const double mm = __shfl_up(m, d);
        if (lane >= d) c += cc, m += mm;
    }
    if (lane == 63) s.wave_count[wave] = c, s.wave_mass[wave] = m;
    const uint32_t c_before = __shfl_up(c, 1);
    const double m_before = __shfl_up(m, 1);
    count = lane ? c_before : 0, mass = lane ? m_before : 0.0;
    __syncthreads();
    uint32_t cw = 0;
    double mw = 0.0;
    for (int w = 0; w < wave; ++w) cw += s.wave_count[w], mw += s.wave_mass[w];
    count += cw, mass = mw + mass;
    __syncthreads();
}

// What is looked for: the element that makes the count reach `count`, or the first whose running mass reaches (or passes) `mass`.
struct Target {
    bool by_count, pass;
    uint32_t count;
    double mass;
    __device__ __forceinline__ bool reached(uint32_t c, double m) const { return by_count ? c >= count : pass ? m > mass : m >= mass; }
};

struct Place { uint32_t count; double mass; int index; };   // an element: elements and weights up to and with it

// The elements and the mass of the bins before every bin: [bin] for this thread's two and all together.
struct BinSums {
    uint32_t count[3];
    double mass[3];
};
// weight_bin < 0: the bins are those of the weights; else they are parts of that one
template <bool MASS = true>
__device__ __forceinline__ BinSums sum_bins(Shared& s, const Weights& w, int count_shift, int weight_bin) {
    BinSums b;
    const uint64_t mask = (1ull << count_shift) - 1;
    uint32_t c[2];
    double m[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint64_t bin = s.bins[2 * threadIdx.x + i];
        c[i] = (uint32_t)(bin >> count_shift);
        m[i] = MASS && bin ? w.of_bin(bin & mask, weight_bin < 0 ? 2 * threadIdx.x + i : weight_bin) : 0.0;
    }
    b.count[0] = c[0] + c[1], b.mass[0] = m[0] + m[1];
    sums_before(s, b.count[0], b.mass[0]);
#pragma unroll
    for (int i = 0; i < 2; ++i) b.count[i + 1] = b.count[i] + c[i], b.mass[i + 1] = b.mass[i] + m[i];
    return b;
}
// The bin in which the target is reached and what lies before it; where it is not (sums made in another order can fall short at the very end):
// the last one that holds anything, or kBins.
template <bool OR_LAST>
__device__ __forceinline__ uint32_t find_bin(Shared& s, const BinSums& b, const Target& t, uint32_t& before_count, double& before_mass) {
    if (threadIdx.x == 0) s.found_bin = kBins;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)   // (exactly one bin: reached with it and not before it; an empty bin changes nothing)
        if (!t.reached(before_count + b.count[i], before_mass + b.mass[i]) && t.reached(before_count + b.count[i + 1], before_mass + b.mass[i + 1]))
            s.found_bin = 2 * threadIdx.x + i, s.found_count = before_count + b.count[i], s.found_mass = before_mass + b.mass[i];
    __syncthreads();
    uint32_t bin = s.found_bin;
    if (OR_LAST && bin == kBins) {
        __syncthreads();
        if (threadIdx.x == 0) s.found_bin = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (b.count[i + 1] > b.count[i]) atomicMax(&s.found_bin, 2 * threadIdx.x + i);
        __syncthreads();
        bin = s.found_bin;
        if (threadIdx.x == bin / 2) s.found_count = before_count + (bin % 2 ? b.count[1] : b.count[0]), s.found_mass = before_mass + (bin % 2 ? b.mass[1] : b.mass[0]);
        __syncthreads();
    }
    before_count = s.found_count, before_mass = s.found_mass;
    __syncthreads();
    return bin;
}

__device__ __forceinline__ void clear_bins(Shared& s) {
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kThreads) s.bins[i] = 0;
    __syncthreads();
}

// One more listed element; what does not fit is counted.
__device__ __forceinline__ void list_one(Shared& s, float l, int i) {
    const uint32_t at = atomicAdd(&s.list_n, 1u);
    if (at < kList) s.list[at] = (uint64_t)descending_key(l) << 32 | (uint32_t)i;
}

// The listed elements (n of them, at most kList), sorted: few are compared with each other, more put to their bins' places and there compared
// with their bin's others; where a bin holds very many, by exchanges (66 steps for 2048).  us, a row of 32000 by exchanges / so: top_k 1000 33 / 25, top_p 0.9 29 /
// 22; 50 by their bins' places 11.9, compared with each other 11.
__device__ __forceinline__ const uint64_t* sort_list(Shared& s, const Weights& w, uint32_t n) {
    if (n <= kFew) {
        if (threadIdx.x < n) {
            const uint64_t x = s.list[threadIdx.x];
            uint32_t rank = 0;
#pragma unroll 8
            for (uint32_t j = 0; j < n; ++j) rank += s.list[j] < x;
            s.sorted[rank] = x;
        }
        __syncthreads();
        return s.sorted;
    }
    const uint32_t first = 2 * threadIdx.x;
    s.places[first] = s.places[first + 1] = 0;
    if (threadIdx.x == 0) s.crowded = 0;
    __syncthreads();
    uint64_t x[2];
    uint32_t bin[2], place[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t at = threadIdx.x + i * kThreads;
        if (at < n) {
            x[i] = s.list[at];
            bin[i] = w.bin_of(w.depth(logit_of_key((uint32_t)(x[i] >> 32))));
            place[i] = atomicAdd(&s.places[bin[i]], 1u);
        }
    }
    __syncthreads();
    const uint32_t c0 = s.places[first], c1 = s.places[first + 1];
    if (c0 > kRanked || c1 > kRanked) s.crowded = 1;
    uint32_t before = c0 + c1;
    double unused = 0.0;
    sums_before(s, before, unused);
    s.places[first] = before, s.places[first + 1] = before + c0;
    __syncthreads();
    if (!s.crowded) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (threadIdx.x + i * kThreads < n) s.sorted[s.places[bin[i]] + place[i]] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (threadIdx.x + i * kThreads < n) {
                const uint32_t from = s.places[bin[i]], to = bin[i] + 1 < kBins ? s.places[bin[i] + 1] : n;
                uint32_t rank = from;
#pragma unroll 8
                for (uint32_t j = from; j < to; ++j) rank += s.sorted[j] < x[i];
                s.list[rank] = x[i];
            }
        __syncthreads();
        return s.list;
    }
    uint32_t all = 2;
    while (all < n) all *= 2;
    for (uint32_t i = n + threadIdx.x; i < all; i += kThreads) s.list[i] = ~0ull;
    for (uint32_t size = 2; size <= all; size *= 2)
        for (uint32_t apart = size / 2; apart; apart /= 2) {
            // (a wave's 128 elements are its own until two threads of different waves meet)
            if (apart >= 128 || (apart == 64 && size >= 256) || size == 2) __syncthreads();
            else wave_sync();
            const uint32_t t = threadIdx.x;
            if (t < all / 2) {
                const uint32_t i = 2 * apart * (t / apart) + t % apart, j = i + apart;
                const uint64_t p = s.list[i], q = s.list[j];
                if ((p > q) == !(i & size)) s.list[i] = q, s.list[j] = p;
            }
        }
    __syncthreads();
    return s.list;
}

// this thread's two places in the sorted list: counts and masses up to and with them, beginning with what lies before the list
__device__ __forceinline__ void sum_list(Shared& s, const Weights& w, const uint64_t* list, uint32_t n, uint32_t before_count, double before_mass,
                                         uint32_t (&count)[3], double (&mass)[3]) {
    double m[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) m[i] = 2 * threadIdx.x + i < n ? w.of(logit_of_key((uint32_t)(list[2 * threadIdx.x + i] >> 32))) : 0.0;
    count[0] = 0, mass[0] = m[0] + m[1];
    sums_before(s, count[0], mass[0]);
    mass[0] = before_mass + mass[0];
#pragma unroll
    for (int i = 0; i < 2; ++i) mass[i + 1] = mass[i] + m[i];
#pragma unroll
    for (int i = 0; i < 3; ++i) count[i] = before_count + min(2 * threadIdx.x + i, n);
}

// The element at which t is reached, from the weights' histogram in s.bins; kept is false where that had to make room.
template <typename T>
__device__ __forceinline__ Place find(Shared& s, const T* row, const SampleArgs& a, const Weights& w, const Target& t, bool& kept) {
    const int n = a.vocab;
    uint32_t before_count = 0;
    double before_mass = 0.0;
    uint32_t bin = find_bin<true>(s, sum_bins(s, w, a.count_shift, -1), t, before_count, before_mass);
    const uint32_t weight_bin = bin;
    const Range range{w.below(bin), w.above(bin)};
    uint32_t low = 0, high = 0xFFFFFFFFu;
    const auto inside = [&](float l) {
        const uint32_t k = descending_key(l);
        return w.bin_of(w.depth(l)) == weight_bin && k >= low && k <= high;
    };
    uint32_t here = (uint32_t)(s.bins[bin] >> a.count_shift);
    bool equal = false;
    while (here > kList && !equal) {
        kept = false;
        if (threadIdx.x == 0) s.key_low = 0xFFFFFFFFu, s.key_high = 0;
        clear_bins(s);
        uint32_t k_min = 0xFFFFFFFFu, k_max = 0;
        each_where(row, n, range, [&](float l, int) {
            if (inside(l)) k_min = min(k_min, descending_key(l)), k_max = max(k_max, descending_key(l));
        });
        atomicMin(&s.key_low, k_min);
        atomicMax(&s.key_high, k_max);
        __syncthreads();
        const uint32_t from = s.key_low, span = s.key_high - from;
        equal = span == 0;   // (key_low is theirs)
        if (equal) break;
        const int shift = span < kBins ? 0 : 21 - __builtin_clz(span);
        each_where(row, n, range, [&](float l, int) {
            if (inside(l)) atomicAdd((unsigned long long*)&s.bins[(descending_key(l) - from) >> shift], 1ull << a.count_shift | w.units(w.depth(l), weight_bin));
        });
        __syncthreads();
        bin = find_bin<true>(s, sum_bins(s, w, a.count_shift, weight_bin), t, before_count, before_mass);
        low = from + (bin << shift);
        high = low + ((1u << shift) - 1);
        here = (uint32_t)(s.bins[bin] >> a.count_shift);
        __syncthreads();
    }
    if (equal) {
        // which of them it is, and that one in the order of their indices: every thread counts a stretch of the row
        const double one = w.of(logit_of_key(s.key_low));
        uint32_t k = here;
        if (t.by_count) k = t.count - before_count;
        else if (one > 0.0) k = (uint32_t)fmin(fmax((t.mass - before_mass) / one, 1.0), (double)here);
        while (k < here && !t.reached(before_count + k, before_mass + k * one)) ++k;
        while (k > 1 && t.reached(before_count + k - 1, before_mass + (k - 1) * one)) --k;
        const int per = (n + kThreads - 1) / kThreads, begin = min(n, (int)threadIdx.x * per), end = min(n, begin + per);
        const auto same = [&](int i) {
            const float l = logit_of(row[i]);
            return l > -INFINITY && inside(l);
        };
        uint32_t c = 0;
        for (int i = begin; i < end; ++i) c += same(i);
        uint32_t place = c;
        double unused = 0.0;
        sums_before(s, place, unused);
        if (place < k && k <= place + c)
            for (int i = begin; i < end; ++i)
                if (same(i) && ++place == k) s.found_index = i;
        __syncthreads();
        const Place p{before_count + k, before_mass + k * one, s.found_index};
        __syncthreads();
        return p;
    }
    if (threadIdx.x == 0) s.list_n = 0;
    __syncthreads();
    each_where(row, n, range, [&](float l, int i) {
        if (inside(l)) list_one(s, l, i);   // (here of them)
    });
    __syncthreads();
    const uint32_t have = s.list_n;
    const uint64_t* list = sort_list(s, w, have);
    uint32_t count[3];
    double mass[3];
    sum_list(s, w, list, have, before_count, before_mass, count, mass);
    // the first that reaches it, or the last one
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (2 * threadIdx.x + i < have && !t.reached(count[i], mass[i]) && (t.reached(count[i + 1], mass[i + 1]) || 2 * threadIdx.x + i + 1 == have))
            s.found_count = count[i + 1], s.found_mass = mass[i + 1], s.found_index = (int)(uint32_t)list[2 * threadIdx.x + i];
    __syncthreads();
    const Place p{s.found_count, s.found_mass, s.found_index};
    __syncthreads();
    return p;
}

// What limits a row's choice; a limit that is off: count = all, mass_part >= 1, depth < 0.
struct Limits {
    uint32_t count;
    float mass_part, depth, u;
};

// The choice from a sorted list that holds all kept elements.  total: the mass of which mass_part is kept; < 0: that of the first lim.count.
__device__ __forceinline__ int choose(Shared& s, const Weights& w, const uint64_t* list, uint32_t n, const Limits& lim, double total) {
    uint32_t count[3];
    double mass[3];
    sum_list(s, w, list, n, 0, 0.0, count, mass);
    const uint32_t first = 2 * threadIdx.x, n_count = min(lim.count, n);
    if (threadIdx.x == 0) s.mark_count[0] = s.mark_count[1] = n_count, s.mark_count[2] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (first + i + 1 == n_count) s.mark_mass[0] = mass[i + 1];
    __syncthreads();
    if (lim.mass_part < 1.0f) {
        const double need = (double)lim.mass_part * (total < 0.0 ? s.mark_mass[0] : total);
#pragma unroll
        for (int i = 0; i < 2; ++i)   // (one place at most)
            if (first + i < n_count && (first + i == 0 || mass[i] < need) && mass[i + 1] >= need) s.mark_count[0] = first + i + 1;
    }
    if (lim.depth >= 0.0f) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (first + i < n) {
                const bool here = w.depth(logit_of_key((uint32_t)(list[first + i] >> 32))) <= lim.depth;
                const bool next = first + i + 1 < n && w.depth(logit_of_key((uint32_t)(list[first + i + 1] >> 32))) <= lim.depth;
                if (here && !next) s.mark_count[1] = first + i + 1;
            }
    }
    __syncthreads();
    const uint32_t kept = min(s.mark_count[0], s.mark_count[1]);
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (first + i + 1 == kept) s.mark_mass[1] = mass[i + 1], s.mark_count[2] = first + i;
    __syncthreads();
    const double need = (double)lim.u * s.mark_mass[1];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (first + i < kept && mass[i] <= need && mass[i + 1] > need) s.mark_count[2] = first + i;
    __syncthreads();
    return (int)(uint32_t)list[s.mark_count[2]];
}

// A workgroup per row: it reads the row once for its largest logits (256 rows of 128256 in bfloat16, 66 MB: greedy choices take 13.5 us, where the bytes need
// 11), and again what it cannot leave out.  The same rows with top_k 50 21 us (of the second reading only the vectors whose largest logit
// counts; 28 with all of it), 1000 31 (51 from the threads' largest logits, of which the 1000th is no limit), without a limit 51, top_p 0.9 53, at a
// temperature of 0.7 49 (65 with every element that falls to the last bin added there): the histogram of a whole row, some 18 us of vector instructions and
// LDS additions on its compute unit (20 with an exponential for every element), and a third reading.  Two rows of 32000: 4.3, 11, 17, 19, 20, 19 us, a chain
// of some 20 barriers and as many exchanges.  A row to a workgroup, not to several: with as many rows as compute units nothing is gained, and few
// rows would pay a launch (3 us) for each reading.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
    __shared__ Shared s;
    const int r = blockIdx.x, n = a.vocab;
    const T* row = (const T*)a.logits + r * a.row_stride;
    constexpr int kVec = 16 / sizeof(T);

    // the largest logit; a thread keeps where its own largest one is first
    float own_most = -INFINITY;
    int own_at = 0;
    each_vector(row, n, [&](const auto& x, int i, int elements, int v) {
        float most = logit_of(x[0]);
#pragma unroll
        for (int e = 1; e < kVec; ++e) most = fmaxf(most, e < elements ? logit_of(x[e]) : -INFINITY);
        if (most > own_most) own_most = most, own_at = i;
        if (v >= 0 && v < kTable) {
            const uint32_t key = float_to_key(most);
            s.vector_most[v] = (uint16_t)min((key >> 16) + (key % 65536 != 0), 0xFFFFu);
        }
    });
    float most = own_most;
    for (int d = 32; d; d /= 2) most = fmaxf(most, __shfl_xor(most, d));
    if (threadIdx.x % 64 == 0) s.wave_most[threadIdx.x / 64] = most;
    if (threadIdx.x == 0) s.key_low = 0x7FFFFFFFu, s.key_high = 0, s.list_n = 0;
    if (threadIdx.x < 64) s.power[threadIdx.x] = exp2(-(double)threadIdx.x / 64 - a.unit_log2);
    __syncthreads();
    for (int w = 0; w < kWavesPerRow; ++w) most = fmaxf(most, s.wave_most[w]);
    float temperature = a.temperature ? a.temperature[r] : 1.0f;
    if (temperature != temperature) temperature = 1.0f;
    if (temperature <= 0.0f || most == -INFINITY) {
        if (own_most == most && most > -INFINITY)
            for (int i = own_at; i < min(own_at + kVec, n); ++i)
                if (logit_of(row[i]) == most) {
                    atomicMin(&s.key_low, (uint32_t)i);
                    break;
                }
        __syncthreads();
        if (threadIdx.x == 0) a.tokens[r] = most == -INFINITY ? -1 : (int)s.key_low;
        return;
    }
    const Weights w{most, fmaxf(kBinsPerLog2 * 1.44269504088896340736f / temperature, 0x1p-126f), __builtin_amdgcn_ldexpf(1.0f, a.unit_log2), s.power};
    const int top_k = a.top_k ? a.top_k[r] : 0;
    const float top_p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p ? a.min_p[r] : 0.0f;
    Limits lim;
    lim.count = top_k > 0 && top_k < n ? top_k : 0xFFFFFFFFu;
    if (top_p <= 0.0f) lim.count = 1;
    lim.mass_part = top_p > 0.0f && top_p < 1.0f ? top_p : 1.0f;
    lim.depth = min_p > 0.0f ? fmaxf(-kBinsPerLog2 * log2f(min_p), 0.0f) : -1.0f;
    lim.u = fminf(fmaxf(a.u[r], 0.0f), 0x1.fffffep-1f);

    const bool by_vector = lim.count > kFewMaxima && n / kVec <= kTable;
    if (lim.count <= (by_vector ? kMostByMaxima : kThreads / 2)) {
        clear_bins(s);
        uint32_t before_count = 0, end = kBins;
        double before_mass = 0.0;
        float least = -INFINITY;
        const Target last{true, false, lim.count, 0.0};
        if (!by_vector) {
            // the bin of the count-th largest of the threads' own largest; the least of those up to there
            const uint32_t own_bin = w.bin_of(w.depth(own_most));
            if (own_most > -INFINITY) atomicAdd((unsigned long long*)&s.bins[own_bin], 1ull << a.count_shift);
            __syncthreads();
            const uint32_t bin = find_bin<false>(s, sum_bins<false>(s, w, a.count_shift, -1), last, before_count, before_mass);
            if (own_most > -INFINITY && own_bin <= bin) atomicMax(&s.key_high, descending_key(own_most));
            __syncthreads();
            if (bin < kBins) least = logit_of_key(s.key_high);
        } else {
            // the bin of the count-th largest of the vectors' largest, each taken for what is surely not above it
            const int head = min(n, (int)((16 - (uintptr_t)row % 16) % 16 / sizeof(T)));
            for (int v = threadIdx.x; v < (n - head) / kVec; v += kThreads) {
                const float l = logit_of_key(~((uint32_t)(s.vector_most[v] - 1) << 16));
                if (l > -INFINITY) atomicAdd((unsigned long long*)&s.bins[w.bin_of(w.depth(l))], 1ull << a.count_shift);
            }
            __syncthreads();
            end = find_bin<false>(s, sum_bins<false>(s, w, a.count_shift, -1), last, before_count, before_mass);
            if (end < kBins) least = w.below(end);
        }
        each_from(s, row, n, least, [&](float l, int i) {
            if (w.bin_of(w.depth(l)) <= end) list_one(s, l, i);
        });
        __syncthreads();
        const uint32_t listed = s.list_n;
        if (listed <= kList) {
            const int token = choose(s, w, sort_list(s, w, listed), listed, lim, -1.0);
            if (threadIdx.x == 0) a.tokens[r] = token;
            return;
        }
    }

    const auto histogram = [&]() {
        clear_bins(s);
        // The last bin takes many of a row where the temperature is low, so every thread sums its own there (and a row whose largest logit is
        // infinite has all but those); without branches else: what is not of the other bins is added where nobody looks.
        const uint64_t one = (uint64_t)(1u << (a.count_shift - 32)) << 32;
        uint64_t light = 0;
        each_vector(row, n, [&](const auto& x, int, int elements, int) {
            bool rest = false;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const float d = (w.most - logit_of(x[e])) * w.bins_per_logit;
                const bool in = d < kBins - 1.0f && e < elements;
                rest |= !in;
                atomicAdd((unsigned long long*)&s.bins[in ? (uint32_t)d : kBins + threadIdx.x % 64], one | w.units_of_place(__builtin_amdgcn_fractf(d)));
            }
            if (rest)
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    const float l = logit_of(x[e]), d = w.depth(l);
                    if (!((w.most - l) * w.bins_per_logit < kBins - 1.0f) && l > -INFINITY && e < elements) {
                        if (d < kBins - 1.0f) atomicAdd((unsigned long long*)&s.bins[0], one | w.units(d, 0));   // (infinite)
                        else light += one | w.units(d, kBins - 1);
                    }
                }
        });
        for (int d = 32; d; d /= 2) light += __shfl_xor((unsigned long long)light, d);
        if (threadIdx.x % 64 == 0 && light) atomicAdd((unsigned long long*)&s.bins[kBins - 1], (unsigned long long)light);
        __syncthreads();
    };
    histogram();
    const BinSums bins = sum_bins(s, w, a.count_shift, -1);
    if (threadIdx.x == kThreads - 1) s.mark_count[0] = bins.count[2], s.mark_mass[0] = bins.mass[2];
    __syncthreads();
    const uint32_t all = s.mark_count[0];
    const double all_mass = s.mark_mass[0];
    const bool count_on = lim.count < all, mass_on = lim.mass_part < 1.0f, depth_on = lim.depth >= 0.0f;
    // the bin behind which nothing is kept
    uint32_t end = kBins - 1;
    uint32_t before_count = 0;
    double before_mass = 0.0;
    if (count_on) end = min(end, find_bin<false>(s, bins, Target{true, false, lim.count, 0.0}, before_count, before_mass));
    else if (mass_on) end = min(end, find_bin<false>(s, bins, Target{false, false, 0, (double)lim.mass_part * all_mass}, before_count, before_mass));
    if (depth_on && !(count_on && mass_on)) end = min(end, w.bin_of(lim.depth));
    if (threadIdx.x == end / 2) s.mark_count[1] = end % 2 ? bins.count[2] : bins.count[1];
    if (threadIdx.x == 0) s.list_n = 0;
    __syncthreads();
    const uint32_t candidates = s.mark_count[1];
    __syncthreads();                   // (thread 0 clears that word further down: all have it before)
    if (candidates <= kList) {
        each_from(s, row, n, w.below(end), [&](float l, int i) {
            if (w.bin_of(w.depth(l)) <= end) list_one(s, l, i);
        });
        __syncthreads();
        const uint32_t listed = s.list_n;
        const int token = choose(s, w, sort_list(s, w, listed), listed, lim, count_on ? -1.0 : all_mass);
        if (threadIdx.x == 0) a.tokens[r] = token;
        return;
    }

    uint32_t kept = all;
    double mass = all_mass;
    bool whole = true;                 // s.bins are still those of the row
    if (depth_on) {
        // whole bins, and of the one that holds the border what is not behind it
        const uint32_t border = w.bin_of(lim.depth);
        uint32_t c = 0;
        uint64_t units = 0;
        each(row, n, [&](float l, int) {
            const float d = w.depth(l);
            if (!(d <= lim.depth)) return;
            ++c;
            if (w.bin_of(d) == border) units += w.units(d, border);
        });
        if (threadIdx.x == 0) s.mark_count[1] = 0, s.border_units = 0;
        if (threadIdx.x == border / 2) s.mark_mass[1] = border % 2 ? bins.mass[1] : bins.mass[0];
        __syncthreads();
        atomicAdd(&s.mark_count[1], c);
        atomicAdd((unsigned long long*)&s.border_units, (unsigned long long)units);
        __syncthreads();
        if (threadIdx.x == 0) s.mark_mass[1] += w.of_bin(s.border_units, border);
        __syncthreads();
    }
    const uint32_t heavy = depth_on ? s.mark_count[1] : all;
    const double heavy_mass = depth_on ? s.mark_mass[1] : all_mass;
    // Without top_k the end of the kept mass and the choice are looked for together: the bin of the first is known, and so is, but for that bin's own
    // mass, the choice's, hardly ever more than one; their elements are listed side by side.
    if (mass_on && !count_on) {
        const double need = (double)lim.mass_part * all_mass;
        uint32_t c_end = 0, c_low = 0, c_high = 0;
        double m_end = 0.0, m_low = 0.0, m_high = 0.0;
        const uint32_t b_end = find_bin<true>(s, bins, Target{false, false, 0, need}, c_end, m_end);
        const double m_most = m_end + w.of_bin(s.bins[b_end] & ((1ull << a.count_shift) - 1), b_end);
        const double least = heavy < c_end ? heavy_mass : m_end, most_kept = heavy < c_end ? heavy_mass : m_most;
        const uint32_t b_low = find_bin<true>(s, bins, Target{false, true, 0, (double)lim.u * least}, c_low, m_low);
        const uint32_t b_high = find_bin<true>(s, bins, Target{false, true, 0, (double)lim.u * most_kept}, c_high, m_high);
        if (threadIdx.x == b_high / 2) s.mark_count[2] = (b_high % 2 ? bins.count[2] : bins.count[1]) - c_low;
        if (threadIdx.x == 0) s.list_n = 0;
        __syncthreads();
        const uint32_t n_low = s.mark_count[2], n_end = b_end > b_high ? (uint32_t)(s.bins[b_end] >> a.count_shift) : 0;
        if (b_low <= b_high && b_high <= b_end && n_low + n_end <= kList) {
            const Range choice{w.below(b_high), w.above(b_low)}, border{w.below(b_end), w.above(b_end)};
            each_where(row, n, [&](float l) { return choice(l) || border(l); }, [&](float l, int i) {
                const uint32_t bin = w.bin_of(w.depth(l));
                if ((bin >= b_low && bin <= b_high) || bin == b_end) list_one(s, l, i);
            });
            __syncthreads();
            const uint32_t listed = s.list_n;
            const uint64_t* list = sort_list(s, w, listed);
            uint32_t count[3];
            double mass[3];
            sum_list(s, w, list, listed, c_low, m_low, count, mass);
            // the elements of b_end, where it is not among the others, begin with what lies before that bin
            const uint32_t first = 2 * threadIdx.x;
            if (threadIdx.x == 0) s.mark_mass[0] = m_low, s.found_index = -1;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (first + i + 1 == n_low) s.mark_mass[0] = mass[i + 1];
            __syncthreads();
            const double moved = n_end ? m_end - s.mark_mass[0] : 0.0;
            double before[2], after[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bool in_end = first + i >= n_low;
                before[i] = mass[i] + (in_end ? moved : 0.0), after[i] = mass[i + 1] + (in_end ? moved : 0.0);
                count[i] = in_end ? c_end + first + i + 1 - n_low : c_low + first + i + 1;
                if (first + i < listed && before[i] < need && (after[i] >= need || first + i + 1 == listed)) s.found_count = count[i], s.found_mass = after[i];
            }
            __syncthreads();
            const uint32_t kept_count = s.found_count;
            const double aim = (double)lim.u * (heavy < kept_count ? heavy_mass : s.found_mass);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (first + i < listed && before[i] <= aim && after[i] > aim && count[i] <= kept_count) s.found_index = (int)(uint32_t)list[first + i];
            __syncthreads();
            if (s.found_index >= 0) {
                if (threadIdx.x == 0) a.tokens[r] = s.found_index;
                return;
            }
            __syncthreads();
        }
    }
    // the end of the first top_k, of the mass that is kept of them, and the choice
    for (int stage = count_on ? 0 : mass_on ? 1 : 2; stage < 3; ++stage) {
        if (stage == 1 && !mass_on) continue;
        if (stage == 2 && heavy < kept) mass = heavy_mass;
        Target t;
        t.by_count = stage == 0, t.pass = stage == 2, t.count = lim.count;
        t.mass = (stage == 1 ? (double)lim.mass_part : (double)lim.u) * mass;
        if (!whole) histogram();
        whole = true;
        const Place p = find(s, row, a, w, t, whole);
        if (stage == 2) {
            if (threadIdx.x == 0) a.tokens[r] = p.index;
        } else if (p.count < kept) {
            kept = p.count, mass = p.mass;
        }
    }
}

int check(const specache_sample_config* c) {
    if (!c) return fail_without_context(SPECACHE_EINVAL, "null configuration");
    if (c->rows < 0 || c->vocab < 1 || c->vocab > kMostVocab) return fail_without_context(SPECACHE_EINVAL, "rows must not be negative, vocab 1 to 2^20");
    if (c->dtype != SPECACHE_FP16 && c->dtype != SPECACHE_BF16 && c->dtype != SPECACHE_FP32)
        return fail_without_context(SPECACHE_EINVAL, "dtype must be SPECACHE_FP16, SPECACHE_BF16 or SPECACHE_FP32");
    if (c->row_stride < 0) return fail_without_context(SPECACHE_EINVAL, "row_stride must not be negative");
    return SPECACHE_OK;
}

}  // namespace
}  // namespace specache

using namespace specache;

extern "C" {

int specache_sample_scratch(const specache_sample_config* cfg, int64_t* bytes) {
    if (int rc = check(cfg)) return rc;
    if (!bytes) return fail_without_context(SPECACHE_EINVAL, "null output");
    *bytes = 0;
    return SPECACHE_OK;
}

int specache_sample(const specache_sample_config* cfg, const void* logits, const float* u, const float* temperature,
                    const int32_t* top_k, const float* top_p, const float* min_p, int32_t* tokens, void* scratch,
                    int64_t scratch_bytes, void* stream) {
    if (int rc = check(cfg)) return rc;
    if (!cfg->rows) return SPECACHE_OK;
    const size_t size = cfg->dtype == SPECACHE_FP32 ? 4 : 2;
    if (!logits || (uintptr_t)logits % size) return fail_without_context(SPECACHE_EINVAL, "logits must be aligned to their type");
    for (const void* x : {(const void*)u, (const void*)tokens, (const void*)temperature, (const void*)top_k, (const void*)top_p, (const void*)min_p})
        if ((uintptr_t)x % 4) return fail_without_context(SPECACHE_EINVAL, "u, tokens and parameters must be 4-byte aligned");
    if (!u || !tokens) return fail_without_context(SPECACHE_EINVAL, "null u or tokens");
    SampleArgs a{logits, u, temperature, top_p, min_p, top_k, tokens, cfg->row_stride, cfg->vocab, 0, 0};
    // 2^bits >= vocab elements: bits + 1 bits for their number, bits + R + 1 for the sum of their r <= 2^R
    int bits = 0;
    while ((1 << bits) < cfg->vocab) ++bits;
    a.unit_log2 = 62 - 2 * bits < 28 ? 62 - 2 * bits : 28;
    a.count_shift = bits + a.unit_log2 + 1 > 32 ? bits + a.unit_log2 + 1 : 32;   // (the upper word's, for a cheap sum of the two)
    const auto kernel = cfg->dtype == SPECACHE_FP32 ? sample_kernel<float> : cfg->dtype == SPECACHE_BF16 ? sample_kernel<__bf16> : sample_kernel<_Float16>;
    // (a launch's threads are counted in 32 bits)
    for (int64_t first = 0, at_once = (1ll << 31) / kThreads; first < cfg->rows; first += at_once) {
        SampleArgs some = a;
        some.logits = (const char*)logits + first * cfg->row_stride * (int64_t)size;
        some.u += first, some.tokens += first;
        if (temperature) some.temperature += first;
        if (top_k) some.top_k += first;
        if (top_p) some.top_p += first;
        if (min_p) some.min_p += first;
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(at_once, cfg->rows - first)), dim3(kThreads), 0, (hipStream_t)stream, some);
        if (int rc = launched()) return rc;
    }
    return SPECACHE_OK;
}

}  // extern "C"
