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
// A running sum next to a border between two tokens decides, so weights and sums have 64 bits.  A weight is the power of its bin's middle, of which
// there are 64 per power of two, times a binary64 polynomial; in the histogram that is rounded to whole units of 2^-R, R = 62 less the vocabulary's bits (42 at least,
// 46 at most), so that a bin's sum is exact in whatever order it is made.  What weighs less than 2^-63 of the largest is left out: u and top_p
// are binary32 numbers below 1, so the last 2^-24 of a row's mass holds neither the end of what top_p keeps nor the choice, and 2^20 such tokens have 2^-43.
// Together the running sums are off by 2^-41 of the row's at most: 2^-43 by the units' halves, 2^-43 by what is left out, 2^-45 by an
// exponent of up to 44 off by 2^-51 of itself, 2^-48 by the polynomial and by the sums over bins each.
#include "operators.h"
#include "wave_ops.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

namespace specache {
namespace {

constexpr int kThreads = 1024, kWavesPerRow = kThreads / 64;
constexpr int kBins = 4096, kOwn = kBins / kThreads;   // a thread's own bins
constexpr double kBinsPerLog2 = 64.0;  // 64 powers of two of the weights
constexpr int kList = 2048;            // elements that are sorted at once
constexpr int kFew = 256;              // a list so short is sorted by comparing each with all the others,
constexpr int kRanked = 1024;          // of a bin's so many each is compared with all the others
constexpr int kTable = 32768;          // vectors of a row whose largest logits are kept (32 of each thread)
// top_k by the threads' largest logits, by the vectors': us, 256 rows of 128256 / 17 of 49999 in fp32, top_k 100 by the one 23.3 / 15.1, by the other 24.9 / 16.2;
// 200 25.5 / 17.3 and 26.3 / 18.0; 400 26.6 / 18.1 by either, 1400 36.8 / 21.9 by the vectors'.
constexpr int kFewMaxima = 256, kMostByMaxima = 1536;
constexpr int kMostVocab = 1 << 20;
constexpr double kRounder = 0x1.8p52;  // added to a number below 2^31: the sum's lower word is its nearest whole number

struct SampleArgs {
    const void* logits;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t* top_k;
    int32_t* tokens;
    int64_t row_stride;
    int vocab, unit_log2;              // R
    double unit, weight[4];            // 2^R, and of 2^R (2^(-f / 64) - 1), a polynomial in f, the coefficients
};

struct Found { uint32_t place, count; double mass; };   // a place in a row's order with a count and a mass

struct Shared {
    uint64_t bins[kBins + 64];         // the last ones take what is left out, a lane each
    uint64_t list[kList];              // descending_key << 32 | index: ascending is the order of the row
    uint64_t sorted[kList];
    double wave_mass[kWavesPerRow];
    uint32_t wave_count[kWavesPerRow];
    float wave_most[kWavesPerRow];
    uint32_t list_n, key_low, key_high, last_bin, found_index;
    Found found[kWavesPerRow];
    uint32_t wave_found[kWavesPerRow];
    double mark_mass[2];
    uint32_t mark_count[3];
    double power[64];                  // 2^(-i / 64) / 2^R
    uint16_t vector_most[kTable];      // of a thread's own vectors: the largest logit's key, its upper half rounded up
    uint32_t places[kBins];            // elements of a bin; sort_list: then the place of its first
    uint32_t crowded;
};

template <typename T> __device__ __forceinline__ float logit_of(T x) { return (float)x; }

// The thread's number, anew at every call: what follows from it is worked out where it is used, not kept in registers (or scratch memory) from phase to phase.
__device__ __forceinline__ uint32_t thread() {
    uint32_t t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// f(vector, first index, number of the vector or -1) over a row: 16-byte loads between the first and the last aligned address, four ahead, single elements
// before and behind, as vectors whose others are -infinity.
template <typename T, typename F>
__device__ __forceinline__ void each_vector(const T* row, int n, F&& f) {
    const uint32_t tid = thread();
    constexpr int kVec = 16 / sizeof(T), kAhead = 4;
    typedef T Vec __attribute__((ext_vector_type(kVec)));
    const int head = min(n, (int)((16 - (uintptr_t)row % 16) % 16 / sizeof(T)));
    const int vecs = (n - head) / kVec, tail = head + vecs * kVec;
    const Vec* body = (const Vec*)(row + head);
    for (int v = tid; v < vecs; v += kAhead * kThreads) {
        Vec x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) x[i] = body[min(v + i * kThreads, vecs - 1)];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (v + i * kThreads < vecs) f(x[i], head + (v + i * kThreads) * kVec, v + i * kThreads);
    }
    if ((int)tid < head + n - tail) {
        const int i = (int)tid < head ? tid : tail + tid - head;
        Vec x = (T)-INFINITY;
        x[0] = row[i];
        f(x, i, -1);
    }
}
// f(logit, index) for every token inside, which is false for what is not allowed (hardly any are: a vector without one costs its comparisons)
template <typename T, typename Inside, typename F>
__device__ __forceinline__ void each_where(const T* row, int n, Inside&& inside, F&& f) {
    constexpr int kVec = 16 / sizeof(T);
    each_vector(row, n, [&](const auto& x, int i, int) {
        bool any = false;
#pragma unroll
        for (int e = 0; e < kVec; ++e) any |= inside(logit_of(x[e]));
        if (any)
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const float l = logit_of(x[e]);
                if (inside(l)) f(l, i + e);
            }
    });
}
// The same for the tokens that are not below `least` (a finite number); vectors that hold none are not read again where the row's table says so.
template <typename T, typename F>
__device__ __forceinline__ void each_from(const Shared& s, const T* row, int n, float least, F&& f) {
    const uint32_t tid = thread();
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
        if (l >= least) f(l, i);
    };
    if ((int)tid < head) one(row[tid], tid);
    if (tail + (int)tid < n) one(row[tail + tid], tail + tid);
    const uint32_t from = float_to_key(least) >> 16;
    uint32_t wanted = 0;
    for (int v = tid, i = 0; v < vecs; v += kThreads, ++i) wanted |= (uint32_t)(s.vector_most[v] >= from) << i;
    constexpr int kAhead = 4;
    while (wanted) {
        Vec x[kAhead];
        int v[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j, wanted &= wanted - 1) {
            v[j] = wanted ? tid + __builtin_ctz(wanted) * kThreads : -1;
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

__device__ __forceinline__ uint32_t descending_key(float l) { return ~float_to_key(l); }
__device__ __forceinline__ float logit_of_key(uint32_t descending) {
    const uint32_t k = ~descending;
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
// the least binary32 number that is not below x, of the finite ones (x is below the largest)
__device__ __forceinline__ float not_below(double x) {
    float f = fmaxf((float)x, -FLT_MAX);
    if ((double)f < x) f = logit_of_key(descending_key(f) - 1);
    return f;
}

// A row's weights.  Logits from `floor` on count (a finite number, so that no NaN and no -infinity does); those below `split` (-infinity: none) go one bin further on,
// so that the bins up to split_bin are all that min_p keeps.
struct Weights {
    float most, floor, split;
    uint32_t split_bin;
    double scale;                      // bins per logit
    const double* power;
    const double* weight;
    double unit;                       // 2^R
    int unit_log2;

    // the bin of a logit from floor on, before the split, and where in it, from -0.5 to 0.5
    __device__ __forceinline__ uint32_t weight_bin(float l, double& place) const {
        const double d = (double)most - (double)l, r = fma(d, scale, kRounder);
        place = fma(d, scale, -(r - kRounder));
        return (uint32_t)__builtin_bit_cast(uint64_t, r);
    }
    __device__ __forceinline__ uint32_t weight_bin(float l) const {
        double unused;
        return weight_bin(l, unused);
    }
    __device__ __forceinline__ uint32_t bin_of(float l) const { return weight_bin(l) + (l < split); }
    __device__ __forceinline__ uint32_t weight_bin_of(uint32_t bin) const { return bin - (bin > split_bin); }
    // logits between which all elements of the bins up to last, or from first on, lie (and few others)
    __device__ __forceinline__ float below(uint32_t last) const {
        const float l = not_below((double)most - ((double)weight_bin_of(last) + 0.51) / scale);
        return l > floor ? fmaxf(logit_of_key(descending_key(l) + 2), floor) : floor;
    }
    __device__ __forceinline__ float above(uint32_t first) const {
        if (!weight_bin_of(first)) return most;
        const float l = not_below((double)most - ((double)weight_bin_of(first) - 0.51) / scale);
        return l < most ? fminf(logit_of_key(descending_key(l) - 2), most) : most;
    }
    // 2^R 2^(-place / 64), with `first` in place of 2^R: the Taylor polynomial whose fifth power is replaced by what it adds to the third and the first (T5 less its
    // fifth power), off by 2^-48.5.  first = 2^R + 2^52 leaves the nearest whole number in the lower bits.
    __device__ __forceinline__ double polynomial(double place, double first) const {
        return fma(place, fma(place, fma(place, fma(place, weight[3], weight[2]), weight[1]), weight[0]), first);
    }
    __device__ __forceinline__ uint64_t units(double place) const { return __builtin_bit_cast(uint64_t, polynomial(place, unit + 0x1p52)) - 0x4330000000000000ull; }
    __device__ __forceinline__ double of_bin(uint64_t units, uint32_t bin) const {
        const uint32_t b = weight_bin_of(bin);
        return __builtin_amdgcn_ldexp((double)units * power[b % 64], -(int)(b / 64));
    }
    // no fewer than the elements of so many units: each has 2^R 2^(-1 / 128) at least
    __device__ __forceinline__ uint32_t most_elements(uint64_t units) const { return units ? (uint32_t)((units + (units >> 7)) >> unit_log2) + 1 : 0; }
    __device__ __forceinline__ double of(float l) const {
        double place;
        const uint32_t b = weight_bin(l, place);
        return __builtin_amdgcn_ldexp(polynomial(place, unit) * power[b % 64], -(int)(b / 64));
    }
};

// the sums of (count, mass) over the threads before this one, in the threads' order
template <bool COUNT, bool MASS>
__device__ __forceinline__ void sums_before(Shared& s, uint32_t& count, double& mass) {
    const uint32_t tid = thread();
    const int lane = tid % 64, wave = tid / 64;
    uint32_t c = count;
    double m = mass;
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t cc = COUNT ? __shfl_up(c, d) : 0;
        const double mm = MASS ? __shfl_up(m, d) : 0.0;
        if (lane >= d) c += cc, m += mm;
    }
    if (lane == 63) s.wave_count[wave] = c, s.wave_mass[wave] = m;
    const uint32_t c_before = COUNT ? __shfl_up(c, 1) : 0;
    const double m_before = MASS ? __shfl_up(m, 1) : 0.0;
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

struct Place { double mass; int index; };   // an element: the weights up to and with it

// The elements and the mass of the bins before every bin: [bin] for this thread's own and all together.
struct BinSums {
    uint32_t count[kOwn + 1];
    double mass[kOwn + 1];
};
// counted: the elements are counted in s.places; else (as many as there can be) by their units.  part_of < kBins: the bins are parts of that one
template <bool MASS>
__device__ __forceinline__ BinSums sum_bins(Shared& s, const Weights& w, bool counted, uint32_t part_of = kBins) {
    const uint32_t tid = thread();
    BinSums b;
    uint32_t c[kOwn];
    double m[kOwn];
    b.count[0] = 0, b.mass[0] = 0.0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const uint32_t bin = kOwn * tid + i;
        const uint64_t units = MASS ? s.bins[bin] : 0;
        c[i] = counted ? s.places[bin] : w.most_elements(units);
        m[i] = MASS && units ? w.of_bin(units, part_of < kBins ? part_of : bin) : 0.0;
        b.count[0] += c[i], b.mass[0] += m[i];
    }
    sums_before<true, MASS>(s, b.count[0], b.mass[0]);
#pragma unroll
    for (int i = 0; i < kOwn; ++i) b.count[i + 1] = b.count[i] + c[i], b.mass[i + 1] = b.mass[i] + m[i];
    return b;
}
// What the first thread with one has found, in the threads' order; false where none has.  (Sums next to a border between two threads are added in different
// orders, so the one's last can lie below the other's first: a place is the first at whose end the target is reached, whatever its beginning.)
__device__ __forceinline__ bool first_found(Shared& s, bool here, Found& f) {
    const uint32_t tid = thread(), lane = tid % 64, wave = tid / 64;
    const uint64_t lanes = __ballot(here);
    if (lanes ? lane == (uint32_t)__builtin_ctzll(lanes) : lane == 0) {
        s.found[wave] = f;
        s.wave_found[wave] = lanes != 0;
    }
    __syncthreads();
    const uint64_t waves = __ballot(lane < kWavesPerRow && s.wave_found[lane % kWavesPerRow]);
    if (waves) f = s.found[__builtin_ctzll(waves)];
    __syncthreads();
    return waves != 0;
}
// The first bin with elements at whose end the target is reached, and what lies before it; where there is none (sums made in another order can fall short at
// the very end): the last one with elements, or kBins.
template <bool OR_LAST>
__device__ __forceinline__ uint32_t find_bin(Shared& s, const BinSums& b, const Target& t, uint32_t& before_count, double& before_mass) {
    const uint32_t tid = thread();
    Found f{kBins, 0, 0.0};
#pragma unroll
    for (int i = kOwn - 1; i >= 0; --i)
        if (b.count[i + 1] > b.count[i] && t.reached(before_count + b.count[i + 1], before_mass + b.mass[i + 1]))
            f = Found{kOwn * tid + i, before_count + b.count[i], before_mass + b.mass[i]};
    if (!first_found(s, f.place < kBins, f)) {
        if (!OR_LAST) return kBins;
        if (tid == 0) s.last_bin = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
            if (b.count[i + 1] > b.count[i]) atomicMax(&s.last_bin, kOwn * tid + i);
        __syncthreads();
        const uint32_t last = s.last_bin;
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
            if (last == kOwn * tid + i) f = Found{last, before_count + b.count[i], before_mass + b.mass[i]};
        first_found(s, tid == last / kOwn, f);
    }
    before_count = f.count, before_mass = f.mass;
    return f.place;
}

template <bool COUNTS, bool MASS>
__device__ __forceinline__ void clear_bins(Shared& s) {
    const uint32_t tid = thread();
    __syncthreads();
    for (int i = tid; i < kBins; i += kThreads) {
        if (COUNTS) s.places[i] = 0;
        if (MASS) s.bins[i] = 0;
    }
    __syncthreads();
}

// One more listed element; what does not fit is counted.
__device__ __forceinline__ void list_one(Shared& s, float l, int i) {
    const uint32_t at = atomicAdd(&s.list_n, 1u);
    if (at < kList) s.list[at] = (uint64_t)descending_key(l) << 32 | (uint32_t)i;
}
__device__ __forceinline__ float listed_logit(uint64_t x) { return logit_of_key((uint32_t)(x >> 32)); }

// The listed elements (n of them, at most kList), sorted: few are compared with each other, more put to their bins' places and there compared
// with their bin's others; where a bin holds very many, by exchanges (66 steps for 2048).  us, two rows of 32000 by exchanges / so: top_k 1000 31.1 / 17.9, top_p 0.9 26.4 /
// 20.0; 50 by their bins' places 12.7, compared with each other 11.5, 200 (longer lists) 14.5 and 15.5.
__device__ __forceinline__ const uint64_t* sort_list(Shared& s, const Weights& w, uint32_t n) {
    const uint32_t tid = thread();
    if (n <= kFew) {
        if (tid < n) {
            const uint64_t x = s.list[tid];
            uint32_t rank = 0;
#pragma unroll 8
            for (uint32_t j = 0; j < n; ++j) rank += s.list[j] < x;
            s.sorted[rank] = x;
        }
        __syncthreads();
        return s.sorted;
    }
    const uint32_t first = kOwn * tid;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) s.places[first + i] = 0;
    if (tid == 0) s.crowded = 0;
    __syncthreads();
    uint64_t x[2];
    uint32_t bin[2], place[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t at = tid + i * kThreads;
        if (at < n) {
            x[i] = s.list[at];
            bin[i] = w.weight_bin(listed_logit(x[i]));
            place[i] = atomicAdd(&s.places[bin[i]], 1u);
        }
    }
    __syncthreads();
    uint32_t c[kOwn], before = 0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        c[i] = s.places[first + i];
        before += c[i];
        if (c[i] > kRanked) s.crowded = 1;
    }
    double unused = 0.0;
    sums_before<true, false>(s, before, unused);
#pragma unroll
    for (int i = 0; i < kOwn; before += c[i++]) s.places[first + i] = before;
    __syncthreads();
    if (!s.crowded) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (tid + i * kThreads < n) s.sorted[s.places[bin[i]] + place[i]] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (tid + i * kThreads < n) {
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
    for (uint32_t i = n + tid; i < all; i += kThreads) s.list[i] = ~0ull;
    for (uint32_t size = 2; size <= all; size *= 2)
        for (uint32_t apart = size / 2; apart; apart /= 2) {
            // (a wave's 128 elements are its own until two threads of different waves meet)
            if (apart >= 128 || (apart == 64 && size >= 256) || size == 2) __syncthreads();
            else wave_sync();
            const uint32_t t = tid;
            if (t < all / 2) {
                const uint32_t i = 2 * apart * (t / apart) + t % apart, j = i + apart;
                const uint64_t p = s.list[i], q = s.list[j];
                if ((p > q) == !(i & size)) s.list[i] = q, s.list[j] = p;
            }
        }
    __syncthreads();
    return s.list;
}

// this thread's two places in the sorted list: masses up to and with them, beginning with what lies before the list
__device__ __forceinline__ void sum_list(Shared& s, const Weights& w, const uint64_t* list, uint32_t n, double before_mass, double (&mass)[3]) {
    const uint32_t tid = thread();
    double m[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) m[i] = 2 * tid + i < n ? w.of(listed_logit(list[2 * tid + i])) : 0.0;
    uint32_t unused = 0;
    mass[0] = m[0] + m[1];
    sums_before<false, true>(s, unused, mass[0]);
    mass[0] = before_mass + mass[0];
#pragma unroll
    for (int i = 0; i < 2; ++i) mass[i + 1] = mass[i] + m[i];
}

// The index of the k-th token, from 1, for which same(index) holds: every thread counts a stretch of the row.
template <typename Same>
__device__ __forceinline__ int index_of_place(Shared& s, int n, uint32_t k, Same&& same) {
    const uint32_t tid = thread();
    const int per = (n + kThreads - 1) / kThreads, begin = min(n, (int)tid * per), end = min(n, begin + per);
    uint32_t c = 0;
    for (int i = begin; i < end; ++i) c += same(i);
    uint32_t place = c;
    double unused = 0.0;
    sums_before<true, false>(s, place, unused);
    if (place < k && k <= place + c)
        for (int i = begin; i < end; ++i)
            if (same(i) && ++place == k) s.found_index = i;
    __syncthreads();
    return (int)s.found_index;
}

// The element at which t is reached, from the histogram in s.bins (t by count: and s.places); kept is false where that had to make room.
template <typename T>
__device__ __forceinline__ Place find(Shared& s, const T* row, int n, const Weights& w, bool counted, const Target& t, bool& kept) {
    const uint32_t tid = thread();
    uint32_t before_count = 0;
    double before_mass = 0.0;
    const uint32_t whole = find_bin<true>(s, sum_bins<true>(s, w, counted), t, before_count, before_mass);
    const Range range{w.below(whole), w.above(whole)};
    uint32_t low = 0, high = 0xFFFFFFFFu;
    const auto inside = [&](float l) {
        const uint32_t k = descending_key(l);
        return w.bin_of(l) == whole && k >= low && k <= high;
    };
    uint32_t here = counted ? s.places[whole] : w.most_elements(s.bins[whole]);
    bool equal = false;
    while (here > kList && !equal) {
        kept = false;
        if (tid == 0) s.key_low = 0xFFFFFFFFu, s.key_high = 0;
        clear_bins<true, true>(s);
        uint32_t k_min = 0xFFFFFFFFu, k_max = 0;
        each_where(row, n, range, [&](float l, int) {
            if (inside(l)) k_min = min(k_min, descending_key(l)), k_max = max(k_max, descending_key(l));
        });
        atomicMin(&s.key_low, k_min);
        atomicMax(&s.key_high, k_max);
        __syncthreads();
        const uint32_t from = s.key_low, span = s.key_high - from;
        const int shift = span < kBins ? 0 : 20 - __builtin_clz(span);
        each_where(row, n, range, [&](float l, int) {
            if (!inside(l)) return;
            const uint32_t part = (descending_key(l) - from) >> shift;
            double place;
            w.weight_bin(l, place);
            atomicAdd((unsigned long long*)&s.bins[part], w.units(place));
            atomicAdd(&s.places[part], 1u);
        });
        __syncthreads();
        const uint32_t part = find_bin<true>(s, sum_bins<true>(s, w, true, whole), t, before_count, before_mass);
        low = from + (part << shift);
        high = low + ((1u << shift) - 1);
        here = s.places[part];
        equal = shift == 0;
        __syncthreads();
    }
    if (equal && here > kList) {
        // which of them it is, and that one in the order of their indices
        const double one = w.of(logit_of_key(low));
        uint32_t k = here;
        if (t.by_count) k = t.count - before_count;
        else if (one > 0.0) k = (uint32_t)fmin(fmax((t.mass - before_mass) / one, 1.0), (double)here);
        while (k < here && !t.reached(before_count + k, before_mass + k * one)) ++k;
        while (k > 1 && t.reached(before_count + k - 1, before_mass + (k - 1) * one)) --k;
        const Place p{before_mass + k * one, index_of_place(s, n, k, [&](int i) {
            const float l = logit_of(row[i]);
            return range(l) && inside(l);
        })};
        __syncthreads();
        return p;
    }
    if (tid == 0) s.list_n = 0;
    __syncthreads();
    each_where(row, n, range, [&](float l, int i) {
        if (inside(l)) list_one(s, l, i);   // (here of them at most)
    });
    __syncthreads();
    const uint32_t have = s.list_n;
    const uint64_t* list = sort_list(s, w, have);
    double mass[3];
    sum_list(s, w, list, have, before_mass, mass);
    // the first that reaches it, or the last one
    Found f{0, 0, 0.0};
    bool here_too = false;
#pragma unroll
    for (int i = 1; i >= 0; --i) {
        const uint32_t at = 2 * tid + i;
        if (at < have && (at + 1 == have || t.reached(before_count + at + 1, mass[i + 1]))) f = Found{at, 0, mass[i + 1]}, here_too = true;
    }
    first_found(s, here_too, f);
    const Place p{f.mass, (int)(uint32_t)list[f.place]};
    __syncthreads();
    return p;
}

// What limits a row's choice; a limit that is off: count = all, mass_part >= 1, least = -infinity.
struct Limits {
    uint32_t count;
    float mass_part, least, u;         // least: the least logit that min_p keeps
};

// The choice from a sorted list that holds all kept elements.  total: the mass of which mass_part is kept; < 0: that of the first lim.count.
__device__ __forceinline__ int choose(Shared& s, const Weights& w, const uint64_t* list, uint32_t n, const Limits& lim, double total) {
    const uint32_t tid = thread();
    double mass[3];
    sum_list(s, w, list, n, 0.0, mass);
    const uint32_t first = 2 * tid, n_count = min(lim.count, n);
    if (tid == 0) s.mark_count[1] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (first + i < n) {
            if (first + i + 1 == n_count) s.mark_mass[0] = mass[i + 1];
            const bool here = listed_logit(list[first + i]) >= lim.least;
            const bool next = first + i + 1 < n && listed_logit(list[first + i + 1]) >= lim.least;
            if (here && !next) s.mark_count[1] = first + i + 1;
        }
    __syncthreads();
    uint32_t kept = n_count;
    if (lim.mass_part < 1.0f) {
        const double need = (double)lim.mass_part * (total < 0.0 ? s.mark_mass[0] : total);
        Found f{kBins, 0, 0.0};
#pragma unroll
        for (int i = 1; i >= 0; --i)
            if (first + i < n_count && (first + i + 1 == n_count || mass[i + 1] >= need)) f.place = first + i;
        first_found(s, f.place < kBins, f);
        kept = f.place + 1;
    }
    kept = max(1u, min(kept, s.mark_count[1]));
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (first + i + 1 == kept) s.mark_mass[1] = mass[i + 1];
    __syncthreads();
    const double need = (double)lim.u * s.mark_mass[1];
    Found f{kBins, 0, 0.0};
#pragma unroll
    for (int i = 1; i >= 0; --i)
        if (first + i < kept && (first + i + 1 == kept || mass[i + 1] > need)) f.place = first + i;
    first_found(s, f.place < kBins, f);
    return (int)(uint32_t)list[f.place];
}

// Of a row with infinite logits those weigh the same, and all others nothing.
template <typename T>
__device__ __forceinline__ int choose_infinite(Shared& s, const T* row, int n, const Limits& lim) {
    const auto infinite = [](float l) { return l == INFINITY; };
    uint32_t c = 0;
    each_where(row, n, infinite, [&](float, int) { ++c; });
    if (c) atomicAdd(&s.list_n, c);
    __syncthreads();
    uint32_t kept = min(s.list_n, lim.count);
    if (lim.mass_part < 1.0f) kept = min(kept, max(1u, (uint32_t)ceil((double)lim.mass_part * kept)));
    return index_of_place(s, n, (uint32_t)((double)lim.u * kept) + 1, [&](int i) { return infinite(logit_of(row[i])); });
}

// A workgroup per row: it reads the row once for its largest logits (256 rows of 128256 in bfloat16, 66 MB: greedy choices take 14.0 us, where the bytes need
// 11), and again what it cannot leave out.  The same rows with top_k 50 22.0 us (of the second reading only the vectors whose largest logit
// counts), 1000 32.1, without a limit 59.0, top_p 0.9 57.0, at a temperature of 0.7 48.9: the histogram of a whole row, some 19 us of vector
// instructions and LDS additions on its compute unit (16 with binary32 weights, whose sums chose another token once in some thousand draws), and a third reading.  Two rows of
// 32000: 4.0, 11.2, 17.7, 19.3, 22.9, 19.3 us, a chain of some 20 barriers and as many exchanges.  A row to a workgroup, not to several: where every
// row needs a histogram and there are as many as compute units nothing is gained, and few rows would pay a launch (3 us) for each reading.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
    __shared__ Shared s;
    const int r = blockIdx.x, n = a.vocab;
    const T* row = (const T*)a.logits + r * a.row_stride;
    constexpr int kVec = 16 / sizeof(T);

    float temperature = a.temperature ? a.temperature[r] : 1.0f;
    if (temperature != temperature) temperature = 1.0f;
    const int top_k = a.top_k ? a.top_k[r] : 0;
    const float top_p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p ? a.min_p[r] : 0.0f, u = a.u[r];

    // the largest logit; a thread keeps where its own largest one is first
    float own_most = -INFINITY;
    int own_at = 0;
    each_vector(row, n, [&](const auto& x, int i, int v) {
        float most = logit_of(x[0]);
#pragma unroll
        for (int e = 1; e < kVec; ++e) most = fmaxf(most, logit_of(x[e]));
        if (most > own_most || (v < 0 && most == own_most && i < own_at)) own_most = most, own_at = i;
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
    Limits lim;
    lim.count = top_k > 0 && top_k < n ? top_k : 0xFFFFFFFFu;
    if (top_p <= 0.0f || min_p > 1.0f) lim.count = 1;   // (no token reaches either: one at least is kept)
    lim.mass_part = top_p > 0.0f && top_p < 1.0f ? top_p : 1.0f;
    lim.u = fminf(fmaxf(u, 0.0f), 0x1.fffffep-1f);
    lim.least = -INFINITY;
    if (most == INFINITY) {
        const int token = choose_infinite(s, row, n, lim);
        if (threadIdx.x == 0) a.tokens[r] = token;
        return;
    }
    if (min_p >= 1.0f) lim.least = most;
    else if (min_p > 0.0f && temperature < INFINITY) lim.least = not_below((double)most + (double)temperature * log((double)min_p));
    Weights w{most, 0.0f, -INFINITY, kBins, kBinsPerLog2 * 1.44269504088896340736 / temperature, s.power, a.weight, a.unit, a.unit_log2};
    w.floor = not_below((double)most - (kBins - 1.75) / w.scale);   // (the last bin is left for what is split off)
    // where top_p does not ask for the whole row's mass, nothing that min_p leaves out counts
    const bool mass_on = lim.mass_part < 1.0f;
    if (!mass_on) w.floor = fmaxf(w.floor, lim.least);

    const bool by_vector = lim.count > kFewMaxima && n / kVec <= kTable;
    if (lim.count <= (by_vector ? kMostByMaxima : kThreads / 2)) {
        clear_bins<true, false>(s);
        uint32_t before_count = 0, end = kBins;
        double before_mass = 0.0;
        float least = w.floor;
        const Target last{true, false, lim.count, 0.0};
        if (!by_vector) {
            // the bin of the count-th largest of the threads' own largest; the least of those up to there
            const bool counts = own_most >= w.floor;
            const uint32_t own_bin = counts ? w.weight_bin(own_most) : 0;
            if (counts) atomicAdd(&s.places[own_bin], 1u);
            __syncthreads();
            const uint32_t bin = find_bin<false>(s, sum_bins<false>(s, w, true), last, before_count, before_mass);
            if (counts && own_bin <= bin) atomicMax(&s.key_high, descending_key(own_most));
            __syncthreads();
            if (bin < kBins) least = logit_of_key(s.key_high);
        } else {
            // the bin of the count-th largest of the vectors' largest, each taken for what is surely not above it
            const int head = min(n, (int)((16 - (uintptr_t)row % 16) % 16 / sizeof(T)));
            for (int v = threadIdx.x; v < (n - head) / kVec; v += kThreads) {
                const float l = logit_of_key(~((uint32_t)(s.vector_most[v] - 1) << 16));
                if (l >= w.floor && l <= most) atomicAdd(&s.places[w.weight_bin(l)], 1u);
            }
            __syncthreads();
            end = find_bin<false>(s, sum_bins<false>(s, w, true), last, before_count, before_mass);
            if (end < kBins) least = w.below(end);
        }
        each_from(s, row, n, least, [&](float l, int i) {
            if (w.weight_bin(l) <= end) list_one(s, l, i);
        });
        __syncthreads();
        const uint32_t listed = s.list_n;
        if (listed <= kList) {
            const int token = choose(s, w, sort_list(s, w, listed), listed, lim, -1.0);
            if (threadIdx.x == 0) a.tokens[r] = token;
            return;
        }
    }

    // (most rows' histograms need no split and no counts)
    if (mass_on && lim.least > w.floor) w.split = lim.least, w.split_bin = w.weight_bin(lim.least);
    const bool limited = lim.count != 0xFFFFFFFFu;
    const auto fill = [&](auto with_split, auto with_counts) __attribute__((always_inline)) {
        constexpr bool SPLIT = decltype(with_split)::value, COUNTS = decltype(with_counts)::value;
        clear_bins<COUNTS, true>(s);
        // without branches: what does not count is added where nobody looks
        each_vector(row, n, [&](const auto& x, int, int) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const float l = logit_of(x[e]);
                double place;
                uint32_t bin = w.weight_bin(l, place);
                if (SPLIT) bin += l < w.split;
                bin = l >= w.floor ? bin : kBins + threadIdx.x % 64;
                atomicAdd((unsigned long long*)&s.bins[bin], w.units(place));
                if (COUNTS && l >= w.floor) atomicAdd(&s.places[bin], 1u);
            }
        });
        __syncthreads();
    };
    if (limited) fill(std::true_type{}, std::true_type{});
    else if (w.split_bin < kBins) fill(std::true_type{}, std::false_type{});
    else fill(std::false_type{}, std::false_type{});
    const uint32_t last = min(w.split_bin, (uint32_t)kBins - 1);   // behind it nothing is kept
    const BinSums bins = sum_bins<true>(s, w, limited);
    // what lies before the end of a bin
    const auto mark = [&](uint32_t bin, int at) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
            if (bin == kOwn * threadIdx.x + i) s.mark_count[at] = bins.count[i + 1], s.mark_mass[at] = bins.mass[i + 1];
    };
    mark(kBins - 1, 0);
    mark(last, 1);
    __syncthreads();
    double mass = s.mark_mass[0];
    const double heavy_mass = s.mark_mass[1];
    const bool count_on = limited && lim.count < s.mark_count[0];
    uint32_t end = kBins, before_count = 0;
    double before_mass = 0.0;
    if (count_on) end = find_bin<false>(s, bins, Target{true, false, lim.count, 0.0}, before_count, before_mass);
    else if (mass_on) end = find_bin<false>(s, bins, Target{false, false, 0, (double)lim.mass_part * mass}, before_count, before_mass);
    end = min(end, count_on && mass_on ? (uint32_t)kBins - 1 : last);
    __syncthreads();
    mark(end, 0);
    if (threadIdx.x == 0) s.list_n = 0;
    __syncthreads();
    const uint32_t candidates = s.mark_count[0];
    __syncthreads();           // (the word is used again)
    if (candidates <= kList) {
        each_from(s, row, n, w.below(end), [&](float l, int i) {
            if (w.bin_of(l) <= end) list_one(s, l, i);
        });
        __syncthreads();
        const uint32_t listed = s.list_n;
        const int token = choose(s, w, sort_list(s, w, listed), listed, lim, count_on ? -1.0 : mass);
        if (threadIdx.x == 0) a.tokens[r] = token;
        return;
    }
    int stage = count_on ? 0 : mass_on ? 1 : 2;
    // Without top_k the end of the kept mass and the choice are looked for together: the bin of the first is known, and so is, but for that bin's own
    // mass, the choice's, hardly ever more than one; their elements are listed side by side.
    if (stage == 1) {
        const double need = (double)lim.mass_part * mass;
        uint32_t c_end = 0, c_low = 0, c_high = 0;
        double m_end = 0.0, m_low = 0.0, m_high = 0.0;
        const uint32_t b_end = find_bin<true>(s, bins, Target{false, false, 0, need}, c_end, m_end);
        if (b_end > last) stage = 2;   // min_p keeps less
        else {
            const double m_most = m_end + w.of_bin(s.bins[b_end], b_end);
            const uint32_t b_low = find_bin<true>(s, bins, Target{false, true, 0, (double)lim.u * m_end}, c_low, m_low);
            const uint32_t b_high = find_bin<true>(s, bins, Target{false, true, 0, (double)lim.u * m_most}, c_high, m_high);
            mark(b_high, 0);
            __syncthreads();
            const uint32_t n_end = b_end > b_high ? w.most_elements(s.bins[b_end]) : 0;
            if (b_low <= b_high && b_high <= b_end && s.mark_count[0] - c_low + n_end <= kList) {
                const Range choice{w.below(b_high), w.above(b_low)}, border{w.below(b_end), w.above(b_end)};
                each_where(row, n, [&](float l) { return choice(l) || border(l); }, [&](float l, int i) {
                    const uint32_t bin = w.bin_of(l);
                    if ((bin >= b_low && bin <= b_high) || bin == b_end) list_one(s, l, i);
                });
                __syncthreads();
                const uint32_t listed = s.list_n;
                const uint64_t* list = sort_list(s, w, listed);
                double sums[3];
                sum_list(s, w, list, listed, m_low, sums);
                // the elements of b_end, where it is not among the others, begin with what lies before that bin
                const uint32_t first = 2 * threadIdx.x;
                bool in_end[3];
#pragma unroll
                for (int i = 0; i < 3; ++i) in_end[i] = first + i >= listed || w.bin_of(listed_logit(list[first + i])) > b_high;
                if (threadIdx.x == 0) s.mark_mass[0] = m_low;
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (!in_end[i] && in_end[i + 1]) s.mark_mass[0] = sums[i + 1];
                __syncthreads();
                const double moved = m_end - s.mark_mass[0];
                double before[2], after[2];
                Found f{kBins, 0, 0.0};
#pragma unroll
                for (int i = 1; i >= 0; --i) {
                    before[i] = sums[i] + (in_end[i] ? moved : 0.0), after[i] = sums[i + 1] + (in_end[i] ? moved : 0.0);
                    if (first + i < listed && (first + i + 1 == listed || after[i] >= need)) f = Found{first + i, 0, after[i]};
                }
                first_found(s, f.place < kBins, f);
                const uint32_t last_kept = f.place;
                const double aim = (double)lim.u * f.mass;
                f.place = kBins;
#pragma unroll
                for (int i = 1; i >= 0; --i)   // (what lies between the two groups is not listed)
                    if (first + i < listed && first + i <= last_kept && after[i] > aim && (!in_end[i] || before[i] <= aim)) f.place = first + i;
                if (first_found(s, f.place < kBins, f)) {
                    if (threadIdx.x == 0) a.tokens[r] = (int)(uint32_t)list[f.place];
                    return;
                }
            }
        }
    }
    // the end of the first top_k, of the mass that is kept of them, and the choice
    bool whole = true;                 // s.bins are those of the row
    for (;; ++stage) {
        if (stage == 1 && !mass_on) continue;
        if (stage == 2) mass = fmin(mass, heavy_mass);
        Target t;
        t.by_count = stage == 0, t.pass = stage == 2, t.count = lim.count;
        t.mass = (stage == 1 ? (double)lim.mass_part : (double)lim.u) * mass;
        if (!whole) fill(std::true_type{}, std::false_type{});
        whole = true;
        const Place p = find(s, row, n, w, limited && stage == 0, t, whole);   // (sorting takes the room of the counts)
        if (stage == 2) {
            if (threadIdx.x == 0) a.tokens[r] = p.index;
            return;
        }
        mass = fmin(mass, p.mass);
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
    SampleArgs a{logits, u, temperature, top_p, min_p, top_k, tokens, cfg->row_stride, cfg->vocab, 0, 0.0, {}};
    // 2^bits >= vocab elements of hardly more than 2^R units each
    int bits = 0;
    while ((1 << bits) < cfg->vocab) ++bits;
    a.unit_log2 = std::min(62 - bits, 46);
    // e^y = 1 + y + y^2 / 2 + y^3 / 6 + y^4 / 24 + y^5 / 120 for y = -x f, x = ln 2 / 64, up to h = x / 2; y^5 taken for (20 h^2 y^3 - 5 h^4 y) / 16
    const double x = 0.69314718055994530942 / kBinsPerLog2, h2 = x * x / 4;
    a.unit = std::ldexp(1.0, a.unit_log2);
    a.weight[0] = -x * (1 - 5 * h2 * h2 / (16 * 120)) * a.unit;
    a.weight[1] = x * x / 2 * a.unit;
    a.weight[2] = -x * x * x * (1.0 / 6 + 20 * h2 / (16 * 120)) * a.unit;
    a.weight[3] = x * x * x * x / 24 * a.unit;
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
