// Choice of a token per row of logits: temperature, top-k, top-p, min-p, from a given random number.
//
// All three limits keep a prefix of the row in the order of its logits (the lower index first among equals), and so is the
// choice a place in that order: the first element at which a count, or the running sum of the weights, reaches a target.  Nothing
// is sorted for it.  A histogram over the logarithm of the weights gives every bin's count and sum; the bin that holds the target is taken
// apart further, by the bits of its logits, until its elements fit in LDS, where they are ranked.  Weights are whole numbers
// (a binary32 exponential in units of 2^-E of the largest weight), so sums are exact in any order and every way to an element meets the
// same ones.
#include "operators.h"

#include <cmath>

namespace specache {
namespace {

constexpr int kThreads = 1024, kWavesPerRow = kThreads / 64;
constexpr int kBins = 2048;            // two per thread
constexpr float kBinsPerLog2 = 64.0f;  // 32 powers of two of the weights; what is lighter shares the last bin
constexpr int kFits = 1024;            // elements that are ranked at once

struct SampleArgs {
    const void* logits;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t* top_k;
    int32_t* tokens;
    int64_t row_stride;
    int vocab, unit_log2;              // weights in 2^-unit_log2
};

struct Place {                         // an element in the order: elements and weights up to and with it
    uint32_t count;
    uint64_t mass;
    int index;
};

struct Shared {
    uint32_t count[kBins];
    uint64_t mass[kBins];
    uint32_t wave_count[kWavesPerRow];
    uint64_t wave_mass[kWavesPerRow];
    float list_value[kFits];
    int list_index[kFits];
    uint32_t list_n, key_low, key_high, found_bin;
    uint32_t found_count;
    uint64_t found_mass;
    int found_index;
};

template <typename T> __device__ __forceinline__ float logit_of(T x);
template <> __device__ __forceinline__ float logit_of<float>(float x) { return x; }
template <> __device__ __forceinline__ float logit_of<_Float16>(_Float16 x) { return (float)x; }
template <> __device__ __forceinline__ float logit_of<__bf16>(__bf16 x) { return (float)x; }

// f(logit, index) for every allowed token of a row, in no order.  16-byte loads between the first and the last aligned address.
template <typename T, typename F>
__device__ __forceinline__ void each(const T* row, int n, F&& f) {
    constexpr int kVec = 16 / sizeof(T);
    const auto one = [&](T x, int i) {
        const float l = logit_of(x);
        if (l > -INFINITY) f(l, i);   // (false for NaN as well)
    };
    const int head = min(n, (int)((16 - (uintptr_t)row % 16) % 16 / sizeof(T)));
    const int vecs = (n - head) / kVec;
    for (int i = threadIdx.x; i < head; i += kThreads) one(row[i], i);
    typedef T Vec __attribute__((ext_vector_type(kVec)));
    const Vec* body = (const Vec*)(row + head);
#pragma unroll 2
    for (int v = threadIdx.x; v < vecs; v += kThreads) {
        const Vec x = body[v];
#pragma unroll
        for (int e = 0; e < kVec; ++e) one(x[e], head + v * kVec + e);
    }
    for (int i = head + vecs * kVec + threadIdx.x; i < n; i += kThreads) one(row[i], i);
}

struct Weights {
    float most, per_log2;
    int unit_log2;
    // log2 of the weight: never rises as the logit falls
    __device__ __forceinline__ float log2_of(float l) const { return l == most ? 0.0f : (l - most) * per_log2; }
    __device__ __forceinline__ uint64_t of_log2(float a) const {
        const float w = __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(a), unit_log2 - 32);
        const uint32_t hi = (uint32_t)w;
        return (uint64_t)hi << 32 | (uint32_t)((w - (float)hi) * 4294967296.0f);
    }
    __device__ __forceinline__ uint64_t of(float l) const { return of_log2(log2_of(l)); }
};

__device__ __forceinline__ uint32_t wave_add(uint32_t v) {
    for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ uint64_t wave_add(uint64_t v) {
    for (int d = 32; d; d /= 2) v += __shfl_xor((unsigned long long)v, d);
    return v;
}

// the sums of (count, mass) over the threads before this one
__device__ __forceinline__ void sums_before(Shared& s, uint32_t& count, uint64_t& mass) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t c = count;
    uint64_t m = mass;
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t cc = __shfl_up(c, d);
        const uint64_t mm = __shfl_up((unsigned long long)m, d);
        if (lane >= d) c += cc, m += mm;
    }
    if (lane == 63) s.wave_count[wave] = c, s.wave_mass[wave] = m;
    __syncthreads();
    c -= count, m -= mass;
    for (int w = 0; w < wave; ++w) c += s.wave_count[w], m += s.wave_mass[w];
    count = c, mass = m;
    __syncthreads();
}

// What is looked for: the element that makes the count reach `count`, or the first whose running mass reaches (or passes) `mass`.
struct Target {
    bool by_count, pass;
    uint32_t count;
    double mass;
    __device__ __forceinline__ bool reached(uint32_t c, uint64_t m) const {
        return by_count ? c >= count : pass ? (double)m > mass : (double)m >= mass;
    }
};

// Bins in the order of the elements: the one in which the target is reached, with what lies before it.
__device__ __forceinline__ void find_bin(Shared& s, const Target& t, uint32_t& before_count, uint64_t& before_mass, uint32_t& bin) {
    const uint32_t c0 = s.count[2 * threadIdx.x], c1 = s.count[2 * threadIdx.x + 1];
    const uint64_t m0 = s.mass[2 * threadIdx.x], m1 = s.mass[2 * threadIdx.x + 1];
    uint32_t c = c0 + c1;
    uint64_t m = m0 + m1;
    sums_before(s, c, m);
    c += before_count, m += before_mass;
    if (threadIdx.x == 0) s.found_bin = kBins;
    __syncthreads();
    // (exactly one bin: reached with it and not before it; an empty bin changes nothing)
    const bool r0 = t.reached(c, m), r1 = t.reached(c + c0, m + m0), r2 = t.reached(c + c0 + c1, m + m0 + m1);
    if (!r0 && r1 && c0) s.found_bin = 2 * threadIdx.x, s.found_count = c, s.found_mass = m;
    if (!r1 && r2 && c1) s.found_bin = 2 * threadIdx.x + 1, s.found_count = c + c0, s.found_mass = m + m0;
    __syncthreads();
    bin = s.found_bin;
    before_count = s.found_count, before_mass = s.found_mass;
    __syncthreads();
}

__device__ __forceinline__ uint32_t descending_key(float l) { return ~float_to_key(l); }

// The element at which t is reached; the histogram of all elements by log2 of the weights is in s.count, s.mass on entry and
// may be gone on return.
template <typename T>
__device__ Place find(Shared& s, const T* row, int n, const Weights& w, const Target& t) {
    uint32_t before_count = 0, bin;
    uint64_t before_mass = 0;
    find_bin(s, t, before_count, before_mass, bin);
    if (bin == kBins) return Place{0, 0, -1};   // the target is not reached
    bool by_log2 = true;
    uint32_t low = 0, high = 0xFFFFFFFFu;
    const auto inside = [&](float l) {
        if (by_log2) return (uint32_t)fminf(-w.log2_of(l) * kBinsPerLog2, kBins - 1.0f) == bin;
        const uint32_t k = descending_key(l);
        return k >= low && k <= high;
    };
    uint32_t here = s.count[bin];
    __syncthreads();
    while (here > kFits) {
        if (threadIdx.x == 0) s.key_low = 0xFFFFFFFFu, s.key_high = 0;
        __syncthreads();
        uint32_t k_min = 0xFFFFFFFFu, k_max = 0;
        each(row, n, [&](float l, int) {
            if (inside(l)) {
                const uint32_t k = descending_key(l);
                k_min = min(k_min, k), k_max = max(k_max, k);
            }
        });
        atomicMin(&s.key_low, k_min);
        atomicMax(&s.key_high, k_max);
        __syncthreads();
        const uint32_t new_low = s.key_low, new_high = s.key_high;
        if (new_low == new_high) break;         // all equal
        const uint32_t span = new_high - new_low;
        const int shift = span < kBins ? 0 : 32 - __builtin_clz(span) - 11;
        for (int i = threadIdx.x; i < kBins; i += kThreads) s.count[i] = 0, s.mass[i] = 0;
        __syncthreads();
        each(row, n, [&](float l, int) {
            if (inside(l)) {
                const uint32_t at = (descending_key(l) - new_low) >> shift;
                atomicAdd(&s.count[at], 1u);
                atomicAdd((unsigned long long*)&s.mass[at], (unsigned long long)w.of(l));
            }
        });
        __syncthreads();
        find_bin(s, t, before_count, before_mass, bin);
        by_log2 = false;
        low = new_low + (bin << shift);
        high = low + ((1u << shift) - 1);
        here = s.count[bin];
        __syncthreads();
    }
    if (here > kFits) {
        // equal ones, in the order of their indices: every thread counts a stretch of the row
        const int per = (n + kThreads - 1) / kThreads, from = min(n, (int)threadIdx.x * per), to = min(n, from + per);
        const auto same = [&](int i) {
            const float l = logit_of(row[i]);
            return l > -INFINITY && inside(l);
        };
        uint32_t c = 0;
        float value = 0;
        for (int i = from; i < to; ++i)
            if (same(i)) ++c, value = logit_of(row[i]);
        const uint64_t each_one = c ? w.of(value) : 0;
        uint32_t place = c;
        uint64_t mass = c * each_one;
        sums_before(s, place, mass);
        place += before_count, mass += before_mass;
        if (c && !t.reached(place, mass) && t.reached(place + c, mass + c * each_one))
            for (int i = from; i < to; ++i)
                if (same(i)) {
                    ++place, mass += each_one;
                    if (t.reached(place, mass)) {
                        s.found_count = place, s.found_mass = mass, s.found_index = i;
                        break;
                    }
                }
        __syncthreads();
        const Place p{s.found_count, s.found_mass, s.found_index};
        __syncthreads();
        return p;
    }
    if (threadIdx.x == 0) s.list_n = 0;
    __syncthreads();
    each(row, n, [&](float l, int i) {
        if (inside(l)) {
            const uint32_t at = atomicAdd(&s.list_n, 1u);
            if (at < kFits) s.list_value[at] = l, s.list_index[at] = i;
        }
    });
    __syncthreads();
    // every element's rank and the weights ahead of it
    const uint32_t have = min(s.list_n, (uint32_t)kFits);
    if (threadIdx.x < have) {
        const float l = s.list_value[threadIdx.x];
        const int i = s.list_index[threadIdx.x];
        uint32_t c = before_count + 1;
        uint64_t m = before_mass + w.of(l);
        for (uint32_t j = 0; j < have; ++j) {
            const float lj = s.list_value[j];
            if (lj > l || (lj == l && s.list_index[j] < i)) ++c, m += w.of(lj);
        }
        if (t.reached(c, m) && !t.reached(c - 1, m - w.of(l))) s.found_count = c, s.found_mass = m, s.found_index = i;
    }
    __syncthreads();
    const Place p{s.found_count, s.found_mass, s.found_index};
    __syncthreads();
    return p;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
    __shared__ Shared s;
    const int r = blockIdx.x, n = a.vocab;
    const T* row = (const T*)a.logits + r * a.row_stride;

    // the largest logit and its first place
    float most = -INFINITY;
    int first = 0x7FFFFFFF;
    each(row, n, [&](float l, int i) {
        if (l > most || (l == most && i < first)) most = l, first = i;
    });
    for (int d = 32; d; d /= 2) {
        const float l = __shfl_xor(most, d);
        const int i = __shfl_xor(first, d);
        if (l > most || (l == most && i < first)) most = l, first = i;
    }
    if (threadIdx.x % 64 == 0) s.list_value[threadIdx.x / 64] = most, s.list_index[threadIdx.x / 64] = first;
    __syncthreads();
    for (int w = 0; w < kWavesPerRow; ++w) {
        const float l = s.list_value[w];
        const int i = s.list_index[w];
        if (l > most || (l == most && i < first)) most = l, first = i;
    }
    float temperature = a.temperature ? a.temperature[r] : 1.0f;
    if (temperature != temperature) temperature = 1.0f;
    if (temperature <= 0.0f || most == -INFINITY) {
        if (threadIdx.x == 0) a.tokens[r] = most == -INFINITY ? -1 : first;
        return;
    }
    const Weights w{most, 1.44269504088896340736f / temperature, a.unit_log2};
    const int top_k = a.top_k ? a.top_k[r] : 0;
    const float top_p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p ? a.min_p[r] : 0.0f;
    const float min_log2 = min_p > 0.0f ? fminf(log2f(min_p), 0.0f) : -INFINITY;
    const float u = fminf(fmaxf(a.u[r], 0.0f), 0x1.fffffep-1f);

    uint32_t all = 0, heavy = 0;
    uint64_t all_mass = 0, heavy_mass = 0;
    const auto histogram = [&]() {
        __syncthreads();
        for (int i = threadIdx.x; i < kBins; i += kThreads) s.count[i] = 0, s.mass[i] = 0;
        __syncthreads();
        uint32_t c = 0, hc = 0;
        uint64_t m = 0, hm = 0;
        each(row, n, [&](float l, int) {
            const float at = w.log2_of(l);
            const uint64_t mass = w.of_log2(at);
            const uint32_t bin = (uint32_t)fminf(-at * kBinsPerLog2, kBins - 1.0f);
            atomicAdd(&s.count[bin], 1u);
            atomicAdd((unsigned long long*)&s.mass[bin], (unsigned long long)mass);
            ++c, m += mass;
            if (at >= min_log2) ++hc, hm += mass;
        });
        all = c, all_mass = m, heavy = hc, heavy_mass = hm;
        __syncthreads();
    };
    const auto over_the_row = [&](uint32_t& c, uint64_t& m) {
        c = wave_add(c), m = wave_add(m);
        if (threadIdx.x % 64 == 0) s.wave_count[threadIdx.x / 64] = c, s.wave_mass[threadIdx.x / 64] = m;
        __syncthreads();
        c = 0, m = 0;
        for (int i = 0; i < kWavesPerRow; ++i) c += s.wave_count[i], m += s.wave_mass[i];
        __syncthreads();
    };
    histogram();
    over_the_row(all, all_mass);
    over_the_row(heavy, heavy_mass);
    uint32_t kept = all;
    uint64_t mass = all_mass;
    const uint32_t heavy_count = heavy;
    const uint64_t heavy_sum = heavy_mass;
    if (top_k > 0 && (uint32_t)top_k < all) {
        const Place p = find(s, row, n, w, Target{true, false, (uint32_t)top_k, 0.0});
        kept = p.count, mass = p.mass;
        histogram();
    }
    if (top_p < 1.0f) {
        const Place p = find(s, row, n, w, top_p > 0.0f ? Target{false, false, 0, (double)top_p * (double)mass} : Target{true, false, 1, 0.0});
        if (p.count && p.count < kept) kept = p.count, mass = p.mass;
        histogram();
    }
    if (heavy_count < kept) mass = heavy_sum;
    const Place p = find(s, row, n, w, Target{false, true, 0, (double)u * (double)mass});
    if (threadIdx.x == 0) a.tokens[r] = p.index;
}

int check(const specache_sample_config* c) {
    if (!c) return fail_without_context(SPECACHE_EINVAL, "null configuration");
    if (c->rows < 0 || c->vocab < 1 || c->vocab > (1 << 24)) return fail_without_context(SPECACHE_EINVAL, "rows must not be negative, vocab 1 to 2^24");
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
    SampleArgs a{logits, u, temperature, top_p, min_p, top_k, tokens, cfg->row_stride, cfg->vocab, 0};
    int bits = 0;
    while ((1 << bits) < cfg->vocab) ++bits;
    a.unit_log2 = 62 - bits < 46 ? 62 - bits : 46;   // the sum of a row stays below 2^63
    const auto kernel = cfg->dtype == SPECACHE_FP32 ? sample_kernel<float> : cfg->dtype == SPECACHE_BF16 ? sample_kernel<__bf16> : sample_kernel<_Float16>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)cfg->rows), dim3(kThreads), 0, (hipStream_t)stream, a);
    return launched();
}

}  // extern "C"
