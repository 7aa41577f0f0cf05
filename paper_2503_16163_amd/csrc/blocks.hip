// Choice of blocks of a paged cache by a cheap score: for every query row of a KV head, the blocks whose bounds promise most.
//
// score(block) = max over the KV head's query heads of  max(q, 0) . most + min(q, 0) . least, where least and most are the block's bounds: a product over 256
// channels, [max(q, 0), min(q, 0)] by [most, least].  Which block is the last chosen depends on scores next to each other, and a sum in
// 32 bits would choose differently from one order of additions to another, so the choice is that of sums in 64 bits.  Hardly a block needs them: score_kernel
// makes all scores on the matrix cores in 32 bits, together with the sums of the addends' magnitudes, which bound their error; select_kernel, a workgroup
// to a row, finds the last chosen one by its bits from the top, and only where others are nearer to it than the error are those
// made again in 64 bits.  (All scores in 64 bits on the matrix cores: 19 us instead of 5 for 16 sequences of up to 512 blocks and 8 heads of 4, 52 instead of 12
// for 256 rows of 313 blocks and 8 heads of 8.)
#include "pages.h"
#include "wave_ops.h"

#include <algorithm>
#include <cmath>

namespace specache {
namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef __bf16 bfloat8v __attribute__((ext_vector_type(8)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));

constexpr int kTile = 16;             // blocks, and rows, of a product
constexpr int kScoreWaves = 4;

struct BlockArgs {
    specache_view q;
    PageArgs pages;
    const int32_t* q_lengths;
    const int32_t* kv_lengths;
    int32_t* blocks;
    float* scores;                    // [batch][KV head][token][row_blocks]
    float* sizes;                     // [batch][KV head][token][row_blocks / 16]: the largest sum of magnitudes of 16 blocks
    uint64_t* keys;                   // [batch][KV head][token][row_blocks]: where a row's scores are all made again
    int batch, G, q_tokens, kv_tokens, top, first, recent;
    int row_blocks;                   // whole tiles
    int tokens_here, passes, token_groups, splits;
};

template <bool BF16>
__device__ __forceinline__ float4v mfma16(short8v a, short8v b, float4v c) {
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfloat8v, a), __builtin_bit_cast(bfloat8v, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

// A wave's rows are up to 16 query heads at a time: of as many tokens as fit, or of a part of one token.  It keeps 16 blocks' bounds and walks the rows of its
// tokens.  Lane l has, of row and of block l % 16, the channels 32 s + 8 (l / 16) + e: 16-byte accesses, four neighbouring lanes' 64 bytes for every s.
template <bool BF16>
__global__ __launch_bounds__(64 * kScoreWaves) void score_kernel(BlockArgs a) {
    __shared__ float2 room[kScoreWaves][kTile][kTile + 1];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int split = blockIdx.x % a.splits, unit = blockIdx.x / a.splits;
    const int token0 = unit % a.token_groups * a.tokens_here * a.passes, h = unit / a.token_groups % a.pages.n_kv_heads, b = unit / a.token_groups / a.pages.n_kv_heads;
    const int n = length_of(a.q_lengths, b, a.q_tokens), N = length_of(a.kv_lengths, b, a.kv_tokens);
    const int tokens = min(a.tokens_here * a.passes, n - token0), last = N - n + token0 + tokens - 1;   // the last row's position
    if (tokens <= 0 || last < 0) return;
    const int tiles = (last >> a.pages.log2) / kTile + 1;
    const int column = lane % 16, quarter = lane / 16;
    const int32_t* table = a.pages.table + b * a.pages.table_stride;
    const uint16_t* base = (const uint16_t*)a.pages.bounds.data + h * a.pages.bounds.head + 8 * quarter;
    const int64_t row0 = ((int64_t)b * a.pages.n_kv_heads + h) * a.q_tokens;
    for (int tile = split * kScoreWaves + wave; tile < tiles; tile += a.splits * kScoreWaves) {
        const int block = tile * kTile + column;
        int page = block < a.pages.table_pages ? table[block] : -1;
        const bool there = (uint32_t)page < (uint32_t)a.pages.n_pages;
        if (!there) page = 0;
        const uint16_t* from = base + page * a.pages.bounds.batch;
        short8v least[4], most[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            least[s] = *(const short8v*)(from + 32 * s);
            most[s] = *(const short8v*)(from + a.pages.bounds.token + 32 * s);
        }
        for (int t0 = 0; t0 < tokens; t0 += a.tokens_here) {
            const int here = min(a.tokens_here, tokens - t0), rows = here * a.G;
            float best[4], size[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) best[i] = -INFINITY, size[i] = 0.0f;
            for (int r0 = 0; r0 < rows; r0 += kTile) {
                const int r = min(r0 + column, rows - 1);
                const uint16_t* q = (const uint16_t*)a.q.data + b * a.q.batch + (h * a.G + r % a.G) * a.q.head + (token0 + t0 + r / a.G) * a.q.token + 8 * quarter;
                float4v sum = {0.0f, 0.0f, 0.0f, 0.0f}, magnitude = sum;
                constexpr short8v kZero = {0, 0, 0, 0, 0, 0, 0, 0}, kNoSign = {0x7FFF, 0x7FFF, 0x7FFF, 0x7FFF, 0x7FFF, 0x7FFF, 0x7FFF, 0x7FFF};
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const short8v x = *(const short8v*)(q + 32 * s);
                    const short8v plus = __builtin_elementwise_max(x, kZero), minus = __builtin_elementwise_min(x, kZero);   // (a negative number's bits are one)
                    sum = mfma16<BF16>(plus, most[s], sum);
                    sum = mfma16<BF16>(minus, least[s], sum);
                    magnitude = mfma16<BF16>(plus, most[s] & kNoSign, magnitude);
                    magnitude = mfma16<BF16>(minus & kNoSign, least[s] & kNoSign, magnitude);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) room[wave][4 * quarter + i][column] = float2{sum[i], magnitude[i]};
                wave_sync();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = quarter + 4 * i, end = min(min((t + 1) * a.G, r0 + kTile), rows);   // the token's heads among these rows
                    for (int g = max(t * a.G, r0); g < end; ++g) {
                        const float2 x = room[wave][g - r0][column];
                        best[i] = fmaxf(best[i], x.x);
                        size[i] = x.y <= size[i] ? size[i] : x.y == x.y ? x.y : INFINITY;
                    }
                }
                wave_sync();
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = quarter + 4 * i;
                if (4 * i >= here) break;
                const bool candidate = t < here && there && block <= (N - n + token0 + t0 + t) >> a.pages.log2;
                float largest = candidate ? size[i] : 0.0f;
#pragma unroll
                for (int d = 1; d < 16; d *= 2) largest = fmaxf(largest, __shfl_xor(largest, d));
                if (t >= here) continue;
                const int64_t row = row0 + token0 + t0 + t;
                a.scores[row * a.row_blocks + block] = best[i];
                if (column == 0) a.sizes[row * (a.row_blocks / kTile) + tile] = largest;
            }
        }
    }
}

// 32-bit sums are off by 2^-23 of the magnitudes per addition at most, of which there are 256 with the products; twice that, as the magnitudes are
// such a sum as well, and what is lost below the smallest numbers.
__device__ __forceinline__ double error_of(float size) { return 0x1p-14 * (double)size + 0x1p-110; }

// Order of whole numbers for that of scores: the larger the later, 0 below all of them.
__device__ __forceinline__ uint32_t key_of(float x) {
    if (!(x == x)) x = -INFINITY;
    const uint32_t u = __float_as_uint(x + 0.0f);       // (of the two zeros the positive one)
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float score_of(uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7FFFFFFFu : ~key); }
__device__ __forceinline__ uint64_t key_of(double x) {
    if (!(x == x)) x = -INFINITY;
    const uint64_t u = __double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

// A block's score in 64 bits, by 16 lanes of 8 channels each.
template <bool BF16>
__device__ __forceinline__ uint64_t exact_key(const BlockArgs& a, int b, int h, int token, int page) {
    const int part = threadIdx.x % 16;
    const uint16_t* bounds = (const uint16_t*)a.pages.bounds.data + page * a.pages.bounds.batch + h * a.pages.bounds.head + 8 * part;
    const short8v least = *(const short8v*)bounds, most = *(const short8v*)(bounds + a.pages.bounds.token);
    double best = -INFINITY;
    for (int g = 0; g < a.G; ++g) {
        const short8v q = *(const short8v*)((const uint16_t*)a.q.data + b * a.q.batch + (h * a.G + g) * a.q.head + token * a.q.token + 8 * part);
        double sum = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double x = widen16<BF16>((uint16_t)q[e]);
            sum += (x < 0.0 ? 0.0 : x) * (double)widen16<BF16>((uint16_t)most[e]) + (x > 0.0 ? 0.0 : x) * (double)widen16<BF16>((uint16_t)least[e]);
        }
#pragma unroll
        for (int d = 1; d < 16; d *= 2) sum += __shfl_xor(sum, d);
        best = fmax(best, sum);
    }
    return key_of(best);
}

constexpr int kBand = 256;            // blocks so near to the last chosen one that are told apart in LDS
template <int THREADS>
struct Select {
    static constexpr int kWaves = THREADS / 64, kBins = 1024;
    uint32_t bins[kBins];
    uint32_t of_wave[kWaves];
    uint32_t least[kWaves], most[kWaves];
    float size[kWaves];
    uint32_t found[2], band_n, band_index[kBand];
    uint64_t band_key[kBand];
    bool band_chosen[kBand];

    // sum over the threads before this one; total: over all
    __device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t& total) {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
        uint32_t run = x;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t y = __shfl_up(run, d);
            if (lane >= d) run += y;
        }
        __syncthreads();              // (what was there has been read)
        if (lane == 63) of_wave[wave] = run;
        __syncthreads();
        uint32_t before = 0;
        total = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) before += of_wave[w];
            total += of_wave[w];
        }
        return before + run - x;
    }
    // the least and the largest over all threads
    __device__ __forceinline__ void extremes(uint32_t& lo, uint32_t& hi, float& sz) {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            lo = min(lo, (uint32_t)__shfl_xor(lo, d));
            hi = max(hi, (uint32_t)__shfl_xor(hi, d));
            sz = fmaxf(sz, __shfl_xor(sz, d));
        }
        __syncthreads();
        if (lane == 0) least[wave] = lo, most[wave] = hi, size[wave] = sz;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) lo = min(lo, least[w]), hi = max(hi, most[w]), sz = fmaxf(sz, size[w]);
    }
    // The bin of the `left`th element, counted from the last bin (every thread has counted its elements); returns its number of elements, takes those behind it from `left`.
    __device__ __forceinline__ uint32_t find(uint32_t& left, uint32_t& bin) {
        constexpr int kOwn = kBins / THREADS;
        __syncthreads();
        uint32_t c[kOwn], sum = 0, total;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) sum += c[i] = bins[kBins - 1 - (int)threadIdx.x * kOwn - i];
        uint32_t before = sum_before(sum, total);
        if (before < left && before + sum >= left) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                if (before < left && before + c[i] >= left) found[0] = kBins - 1 - threadIdx.x * kOwn - i, found[1] = before;
                before += c[i];
            }
        }
        __syncthreads();
        bin = found[0];
        left -= found[1];
        return bins[bin];
    }
    __device__ __forceinline__ void clear() {
        __syncthreads();
        for (int i = threadIdx.x; i < kBins; i += THREADS) bins[i] = 0;
        __syncthreads();
    }
};

// The choice by 64-bit keys in memory, where too many scores are alike: chosen(key) and, of those that match the last chosen one's bits, the first ones.
struct Exact {
    uint64_t edge;
    int shift;
    uint32_t equal;                   // of the matching ones
    __device__ __forceinline__ bool above(uint64_t k) const { return k >> shift > edge >> shift; }
    __device__ __forceinline__ bool matches(uint64_t k) const { return k >> shift == edge >> shift; }
};

// Thread t has the blocks t * own .. t * own + own - 1 of the row.  KEEP: their scores stay in registers (as many at most); 0: they are read again in every pass.
template <bool BF16, int THREADS, int KEEP>
__global__ __launch_bounds__(THREADS) void select_kernel(BlockArgs a) {
    __shared__ Select<THREADS> s;
    const int tid = threadIdx.x, token = blockIdx.x % a.q_tokens, h = blockIdx.x / a.q_tokens % a.pages.n_kv_heads, b = blockIdx.x / a.q_tokens / a.pages.n_kv_heads;
    const int n = length_of(a.q_lengths, b, a.q_tokens), N = length_of(a.kv_lengths, b, a.kv_tokens);
    if (token >= n) return;
    const int slots = a.first + a.top + a.recent;
    int32_t* list = a.blocks + (int64_t)blockIdx.x * slots;
    const int position = N - n + token, mine = position >= 0 ? position >> a.pages.log2 : -1;
    const int blocks = mine + 1, own = (blocks + THREADS - 1) / THREADS, first = tid * own;
    const int32_t* table = a.pages.table + b * a.pages.table_stride;
    const float* scores = a.scores + (int64_t)blockIdx.x * a.row_blocks;
    const auto has_page = [&](int c) { return c < blocks && (uint32_t)table[c] < (uint32_t)a.pages.n_pages; };
    const auto always = [&](int c) { return c < a.first || c > mine - a.recent; };
    // 0: not in the choice (nothing is where there is no choice, and no scores either)
    const auto read = [&](int i) -> uint32_t { return a.top > 0 && i < own && has_page(first + i) && !always(first + i) ? key_of(scores[first + i]) : 0; };
    uint32_t kept[KEEP ? KEEP : 1];
    if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i) kept[i] = read(i);
    }
    const auto each = [&](auto&& f) {
        if constexpr (KEEP) {
#pragma unroll
            for (int i = 0; i < KEEP; ++i) f(i, kept[i]);
        } else {
            for (int i = 0; i < own; ++i) f(i, read(i));
        }
    };

    uint32_t there = 0, total, least = ~0u, most = 0;
    float size = 0.0f;
    if (a.top > 0)
        for (int i = tid; i < (blocks + kTile - 1) / kTile; i += THREADS) size = fmaxf(size, a.sizes[(int64_t)blockIdx.x * (a.row_blocks / kTile) + i]);
    each([&](int, uint32_t k) {
        if (!k) return;
        ++there;
        least = min(least, k);
        most = max(most, k);
    });
    s.sum_before(there, total);
    s.extremes(least, most, size);

    // Chosen are: all of the choice; or the keys from `least + edge` on; or those above a band of scores, and the band's best.
    enum { kAll, kNone, kAbove, kNear, kExact } how;
    uint32_t left = min((uint32_t)a.top, total), edge = 0;
    float low = 0.0f, high = 0.0f;                       // the band
    Exact exact{0, 0, 0};
    const auto is_near = [&](uint32_t k) { const float x = score_of(k); return !(x > high) && !(x < low); };
    const uint64_t* keys = a.keys + (int64_t)blockIdx.x * a.row_blocks;
    if (left == total) how = kAll;
    else if (!left) how = kNone;
    else {
        const uint32_t wanted = left;
        int shift = least == most ? 0 : 32 - __builtin_clz(most - least);   // bits of the keys' distances from the least
        uint32_t here = total;
        while (shift > 0 && here != left) {
            const int above = shift;
            shift = max(0, shift - 10);
            s.clear();
            each([&](int, uint32_t k) {
                if (k && (above == 32 || ((k - least) ^ edge) >> above == 0)) atomicAdd(&s.bins[((k - least) >> shift) & ((1 << (above - shift)) - 1)], 1u);
            });
            uint32_t bin;
            here = s.find(left, bin);
            edge |= bin << shift;
        }
        // the last chosen score, and the best that is not
        uint32_t worst = ~0u, next = 0;
        float unused = 0.0f;
        each([&](int, uint32_t k) {
            if (!k) return;
            if (k - least >= edge) worst = min(worst, k);
            else next = max(next, k);
        });
        s.extremes(worst, next, unused);
        const double error = 2.0 * error_of(size);
        how = here == left && (double)score_of(worst) - (double)score_of(next) > error ? kAbove : kNear;
        if (how == kNear) {
            // (rounded away from each other; infinite or NaN, everything is near)
            low = (float)((double)score_of(worst) - error), high = (float)((double)score_of(worst) + error);
            low = low - fabsf(low) * 0x1p-23f, high = high + fabsf(high) * 0x1p-23f;
            uint32_t above = 0, above_all;
            each([&](int, uint32_t k) { above += k && score_of(k) > high; });
            s.sum_before(above, above_all);
            if (tid == 0) s.band_n = 0;
            __syncthreads();
            each([&](int i, uint32_t k) {
                if (!k || !is_near(k)) return;
                const uint32_t at = atomicAdd(&s.band_n, 1u);
                if (at < kBand) s.band_index[at] = first + i;
            });
            __syncthreads();
            const int band = s.band_n;
            left = wanted - above_all;
            if (band <= kBand) {
                for (int e = tid / 16; e < band; e += THREADS / 16) {
                    const uint64_t k = exact_key<BF16>(a, b, h, token, table[s.band_index[e]]);
                    if (tid % 16 == 0) s.band_key[e] = k;
                }
                __syncthreads();
                for (int e = tid; e < band; e += THREADS) {
                    uint32_t better = 0;
                    for (int o = 0; o < band; ++o)
                        better += s.band_key[o] > s.band_key[e] || (s.band_key[o] == s.band_key[e] && s.band_index[o] < s.band_index[e]);
                    s.band_chosen[e] = better < left;
                }
                __syncthreads();
            } else {
                how = kExact;
                uint64_t* to = a.keys + (int64_t)blockIdx.x * a.row_blocks;
                for (int c = tid / 16; c < blocks; c += THREADS / 16) {
                    const uint64_t k = has_page(c) && !always(c) ? exact_key<BF16>(a, b, h, token, table[c]) : 0;
                    if (tid % 16 == 0) to[c] = k;
                }
                left = wanted;
                here = total;
                int at = 64;
                while (at > 0 && here != left) {
                    const int above = at;
                    at = max(0, at - 10);
                    s.clear();
                    for (int i = 0; i < own; ++i) {
                        const uint64_t k = first + i < blocks ? keys[first + i] : 0;
                        if (k && (above == 64 || (k ^ exact.edge) >> above == 0)) atomicAdd(&s.bins[(k >> at) & ((1ull << (above - at)) - 1)], 1u);
                    }
                    uint32_t bin;
                    here = s.find(left, bin);
                    exact.edge |= (uint64_t)bin << at;
                }
                exact.shift = at;
                exact.equal = left;
                __syncthreads();
            }
        }
    }
    uint32_t tie_at = 0;
    if (how == kExact) {
        uint32_t matching = 0, unused;
        for (int i = 0; i < own; ++i) matching += first + i < blocks && keys[first + i] && exact.matches(keys[first + i]);
        tie_at = s.sum_before(matching, unused);
    }
    const auto chosen = [&](int i, uint32_t k, uint32_t& tie) {
        const int c = first + i;
        if (i >= own) return false;
        if (!k) return always(c) && has_page(c);
        if (how == kAll) return true;
        if (how == kNone) return false;
        if (how == kAbove) return k - least >= edge;
        if (how == kExact) return exact.matches(keys[c]) ? tie++ < exact.equal : exact.above(keys[c]);
        if (!is_near(k)) return score_of(k) > high;
        for (uint32_t e = 0; e < s.band_n; ++e)
            if (s.band_index[e] == (uint32_t)c) return (bool)s.band_chosen[e];
        return false;
    };
    uint32_t number = 0, tie = tie_at;
    each([&](int i, uint32_t k) { number += chosen(i, k, tie); });
    uint32_t at = s.sum_before(number, total);
    tie = tie_at;
    each([&](int i, uint32_t k) {
        if (chosen(i, k, tie)) list[at++] = first + i;
    });
    for (int i = total + tid; i < slots; i += THREADS) list[i] = -1;
}

constexpr int64_t kMostGroups = INT32_MAX / 1024;

struct Plan {
    BlockArgs a{};
    int64_t groups = 0, rows = 0, bytes = 0;
};

int plan_of(const specache_pages* cache, const specache_block_config* c, Plan& p) {
    if (int rc = check_blocks(cache, c)) return rc;
    BlockArgs& a = p.a;
    a.G = c->n_q_heads / cache->n_kv_heads;
    const int64_t blocks = ((int64_t)c->kv_tokens + cache->page_tokens - 1) / cache->page_tokens, tiles = (blocks + kTile - 1) / kTile;
    a.row_blocks = (int)(tiles * kTile);
    a.tokens_here = std::max(1, kTile / a.G);
    p.rows = (int64_t)c->batch * cache->n_kv_heads * c->q_tokens;
    const int64_t heads = (int64_t)c->batch * cache->n_kv_heads, groups = (c->q_tokens + a.tokens_here - 1) / a.tokens_here;
    // a wave's bounds are read for up to 8 products' rows, where there are rows enough for 4096 waves all the same
    a.passes = (int)std::max<int64_t>(1, std::min<int64_t>(8, heads * groups * tiles / 4096));
    a.token_groups = (int)((groups + a.passes - 1) / a.passes);
    const int64_t units = heads * a.token_groups;
    a.splits = units ? (int)std::max<int64_t>(1, std::min<int64_t>((tiles + kScoreWaves - 1) / kScoreWaves, (1024 + units - 1) / units)) : 1;
    p.groups = a.row_blocks ? units * a.splits : 0;
    if (p.rows > kMostGroups || p.groups > kMostGroups) return fail_without_context(SPECACHE_EINVAL, "too many rows");
    p.bytes = c->top > 0 ? p.rows * (a.row_blocks * (int64_t)(sizeof(uint64_t) + sizeof(float)) + tiles * (int64_t)sizeof(float)) : 0;
    return SPECACHE_OK;
}

template <bool BF16>
void launch(const Plan& p, const BlockArgs& a, hipStream_t stream) {
    if (a.top > 0 && p.groups && a.pages.n_pages) hipLaunchKernelGGL((score_kernel<BF16>), dim3((unsigned)p.groups), dim3(64 * kScoreWaves), 0, stream, a);
    const int threads = a.row_blocks > 1024 ? 1024 : 256;
    const auto kernel = a.row_blocks <= 512 ? select_kernel<BF16, 256, 2> : a.row_blocks <= 1024 ? select_kernel<BF16, 256, 4> : a.row_blocks <= 4096 ? select_kernel<BF16, 1024, 4>
                        : a.row_blocks <= 16384 ? select_kernel<BF16, 1024, 16> : select_kernel<BF16, 1024, 0>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.rows), dim3(threads), 0, stream, a);
}

}  // namespace
}  // namespace specache

using namespace specache;

extern "C" {

int specache_block_scratch(const specache_pages* cache, const specache_block_config* cfg, int64_t* bytes) {
    Plan p;
    int64_t attend_bytes;
    if (int rc = plan_of(cache, cfg, p)) return rc;
    if (int rc = block_attend_scratch(*cache, *cfg, &attend_bytes)) return rc;
    if (!bytes) return fail_without_context(SPECACHE_EINVAL, "null output");
    *bytes = std::max(p.bytes, attend_bytes);
    return SPECACHE_OK;
}

int specache_block_select(const specache_pages* cache, const specache_block_config* cfg, const specache_view* q, int32_t* blocks, const int32_t* q_lengths,
                          const int32_t* kv_lengths, void* scratch, int64_t scratch_bytes, void* stream) {
    Plan p;
    if (int rc = plan_of(cache, cfg, p)) return rc;
    if (!p.rows) return SPECACHE_OK;
    if (!q || !view_fits(*q)) return fail_without_context(SPECACHE_EINVAL, "q must be a view whose address is 16-byte aligned, its strides multiples of 8");
    if (!blocks || (uintptr_t)blocks % 4) return fail_without_context(SPECACHE_EINVAL, "null or misaligned blocks");
    if ((uintptr_t)q_lengths % 4 || (uintptr_t)kv_lengths % 4) return fail_without_context(SPECACHE_EINVAL, "misaligned lengths");
    if (cfg->kv_tokens)
        if (int rc = check_page_views(*cache, false, cfg->top > 0)) return rc;
    if (p.bytes) {
        if (!scratch || (uintptr_t)scratch % 16) return fail_without_context(SPECACHE_EINVAL, "scratch must be 16-byte aligned");
        if (scratch_bytes < p.bytes) return fail_without_context(SPECACHE_ECAPACITY, "scratch is smaller than specache_block_scratch says");
    }
    BlockArgs& a = p.a;
    a.q = *q;
    a.pages = page_args(*cache);
    a.q_lengths = q_lengths;
    a.kv_lengths = kv_lengths;
    a.blocks = blocks;
    a.keys = (uint64_t*)scratch;
    a.scores = (float*)(a.keys + p.rows * a.row_blocks);
    a.sizes = a.scores + p.rows * a.row_blocks;
    a.batch = cfg->batch;
    a.q_tokens = cfg->q_tokens;
    a.kv_tokens = cfg->kv_tokens;
    a.top = cfg->top;
    a.first = cfg->first;
    a.recent = cfg->recent;
    if (cache->dtype == SPECACHE_BF16) launch<true>(p, a, (hipStream_t)stream);
    else launch<false>(p, a, (hipStream_t)stream);
    return launched();
}

}  // extern "C"
