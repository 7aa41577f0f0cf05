// Choice of blocks of a paged cache by a cheap score: for every query row of a KV head, the blocks whose bounds promise most.
//
// score(block) = max over the KV head's query heads of  max(q, 0) . most + min(q, 0) . least, where least and most are the block's bounds: a product over 256
// channels, [max(q, 0), min(q, 0)] by [most, least].  Which block is the last chosen depends on scores next to each other, and a sum in
// 32 bits would choose differently from one order of additions to another, so the choice is that of sums in 64 bits.  Hardly a block needs them: score_kernel
// makes all scores on the matrix cores in 32 bits, together with a bound of the sums of the addends' magnitudes, which bounds their error; select_kernel, a workgroup to a
// row, counts them in bins and makes those around the last chosen one again in 64 bits.
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
    int unit0, row0;                  // a launch's first unit (what the workgroups of a token group make) and its first row [batch][KV head][token]
    float* scores;                    // [row of the launch][row_blocks]
    float* sizes;                     // [row of the launch][row_blocks / 16]: the largest sum of magnitudes of 16 blocks
    uint64_t* keys;                   // [row of the launch][row_blocks]: where a row's scores are all made again
    int batch, G, q_tokens, kv_tokens, top, first, recent;
    int row_blocks;                   // whole tiles
    int tokens_here;                  // tokens whose heads make a product's rows
    int passes, token_groups;         // of those to a workgroup; workgroups to a sequence
    int splits;
};

template <bool BF16>
__device__ __forceinline__ float4v mfma16(short8v a, short8v b, float4v c) {
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfloat8v, a), __builtin_bit_cast(bfloat8v, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

__device__ __forceinline__ int page_of(const BlockArgs& a, int b, int tile) {
    const int block = tile * kTile + threadIdx.x % 16;
    return block < a.pages.table_pages ? a.pages.table[b * a.pages.table_stride + block] : -1;
}

// The scores of 16 blocks for the tokens token0 .. token0 + tokens - 1 of a KV head, by a wave.  Its rows are up to 16 query heads at a time: of as many tokens as
// fit, or of a part of one token.  It keeps the blocks' bounds and walks the rows.  Lane l has, of row and of block l % 16, the channels 32 s + 8 (l / 16) + e:
// 16-byte accesses, four neighbouring lanes' 64 bytes for every s.  Every s has a sum of its own, so that none has more than 64 addends in a row.
// page: the lane's block's, as page_of has it.  emit(token, block, score, the largest sum of magnitudes of these blocks as far as the token's candidates go)
template <bool BF16, typename Emit>
__device__ __forceinline__ void tile_scores(const BlockArgs& a, int b, int h, int first_position, int token0, int tokens, int tile, int page, float2 (*room)[kTile + 1], Emit&& emit) {
    const int lane = threadIdx.x % 64, column = lane % 16, quarter = lane / 16, block = tile * kTile + column;
    const bool there = (uint32_t)page < (uint32_t)a.pages.n_pages;
    if (!there) page = 0;
    const uint16_t* from = (const uint16_t*)a.pages.bounds.data + page * a.pages.bounds.batch + h * a.pages.bounds.head + 8 * quarter;
    constexpr short8v kZero = {0, 0, 0, 0, 0, 0, 0, 0}, kNoSign = {0x7FFF, 0x7FFF, 0x7FFF, 0x7FFF, 0x7FFF, 0x7FFF, 0x7FFF, 0x7FFF};
    short8v least[4], most[4], largest[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        least[s] = *(const short8v*)(from + 32 * s);
        most[s] = *(const short8v*)(from + a.pages.bounds.token + 32 * s);
    }
    const auto query = [&](int t0, int r0, int s) {
        const int r = min(r0 + column, min(a.tokens_here, tokens - t0) * a.G - 1);
        return *(const short8v*)((const uint16_t*)a.q.data + b * a.q.batch + (h * a.G + r % a.G) * a.q.head + (token0 + t0 + r / a.G) * a.q.token + 8 * quarter + 32 * s);
    };
    short8v next[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) next[s] = query(0, 0, s);
#pragma unroll
    for (int s = 0; s < 4; ++s) largest[s] = __builtin_elementwise_max(most[s] & kNoSign, least[s] & kNoSign);   // (magnitudes' bits are in their order)
    // Where heads are 1, 2, 4, 8 or whole products to a token its rows are in a lane's registers and in those of the lanes 16, 32 and 48 away: value i of a lane is token
    // first_of + i then; else they meet in LDS, and it is token quarter + 4 i.
    const bool even = (a.G & (a.G - 1)) == 0;
    const int values = !even ? 4 : a.G == 1 ? 4 : a.G == 2 ? 2 : 1, step = even ? 1 : 4;
    const int first_of = !even ? quarter : a.G == 1 ? 4 * quarter : a.G == 2 ? 2 * quarter : a.G == 4 ? quarter : a.G == 8 ? quarter / 2 : 0;
    for (int t0 = 0; t0 < tokens; t0 += a.tokens_here) {
        const int here = min(a.tokens_here, tokens - t0), rows = here * a.G;
        float best[4], size[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) best[i] = -INFINITY, size[i] = 0.0f;
        const auto take = [](float& best, float& size, float score, float magnitude) {
            best = fmaxf(best, score);
            size = magnitude <= size ? size : magnitude == magnitude ? magnitude : INFINITY;
        };
        for (int r0 = 0; r0 < rows; r0 += kTile) {
            constexpr float4v kNone = {0.0f, 0.0f, 0.0f, 0.0f};
            float4v sum[4], magnitude = kNone;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const short8v x = next[s];
                const short8v plus = __builtin_elementwise_max(x, kZero), minus = __builtin_elementwise_min(x, kZero);   // (a negative number's bits are one)
                sum[s] = mfma16<BF16>(minus, least[s], mfma16<BF16>(plus, most[s], kNone));
                magnitude = mfma16<BF16>(x & kNoSign, largest[s], magnitude);
            }
            // (the next rows are on their way meanwhile)
            const bool same = r0 + kTile < rows;
            if (same || t0 + a.tokens_here < tokens)
#pragma unroll
                for (int s = 0; s < 4; ++s) next[s] = query(same ? t0 : t0 + a.tokens_here, same ? r0 + kTile : 0, s);
            sum[0] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
            if (even) {                                  // (rows behind the last are that one again, of whose token nothing is kept, or which adds nothing)
                float score[4], of[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) score[i] = sum[0][i], of[i] = magnitude[i] == magnitude[i] ? magnitude[i] : INFINITY;
                if (a.G > 1) score[0] = fmaxf(score[0], score[1]), of[0] = fmaxf(of[0], of[1]), score[1] = fmaxf(score[2], score[3]), of[1] = fmaxf(of[2], of[3]);
                if (a.G > 2) score[0] = fmaxf(score[0], score[1]), of[0] = fmaxf(of[0], of[1]);
                if (a.G > 4) score[0] = fmaxf(score[0], __shfl_xor(score[0], 16)), of[0] = fmaxf(of[0], __shfl_xor(of[0], 16));
                if (a.G > 8) score[0] = fmaxf(score[0], __shfl_xor(score[0], 32)), of[0] = fmaxf(of[0], __shfl_xor(of[0], 32));
#pragma unroll
                for (int i = 0; i < 4; ++i) take(best[i], size[i], score[i], of[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) room[4 * quarter + i][column] = float2{sum[0][i], magnitude[i]};
                wave_sync();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = quarter + 4 * i, end = min(min((t + 1) * a.G, r0 + kTile), rows);   // the token's heads among these rows
                    for (int g = max(t * a.G, r0); g < end; ++g) take(best[i], size[i], room[g - r0][column].x, room[g - r0][column].y);
                }
                wave_sync();
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i >= values) break;
            const int t = first_of + step * i;
            const bool candidate = t < here && there && block <= (first_position + t0 + t) >> a.pages.log2;
            float most_of = candidate ? size[i] : 0.0f;
            most_of = fmaxf(most_of, dpp_move<kDppXor1>(most_of));
            most_of = fmaxf(most_of, dpp_move<kDppXor2>(most_of));
            most_of = fmaxf(most_of, dpp_move<kDppHalfMirror>(most_of));
            most_of = fmaxf(most_of, dpp_move<kDppMirror>(most_of));
            if (t < here) emit(t0 + t, block, best[i], most_of);   // (several lanes the same, of many heads)
        }
    }
}

template <bool BF16>
__global__ __launch_bounds__(64 * kScoreWaves) void score_kernel(BlockArgs a) {
    __shared__ float2 room[kScoreWaves][kTile][kTile + 1];
    const int wave = threadIdx.x / 64, split = blockIdx.x % a.splits, unit = a.unit0 + blockIdx.x / a.splits;
    const int token0 = unit % a.token_groups * a.tokens_here * a.passes, h = unit / a.token_groups % a.pages.n_kv_heads, b = unit / a.token_groups / a.pages.n_kv_heads;
    const int tile0 = split * kScoreWaves + wave;
    int page = page_of(a, b, tile0);                     // (on its way while the lengths are)
    const int n = length_of(a.q_lengths, b, a.q_tokens), first_position = length_of(a.kv_lengths, b, a.kv_tokens) - n + token0;
    const int tokens = min(a.tokens_here * a.passes, n - token0), last = first_position + tokens - 1;
    if (tokens <= 0 || last < 0) return;
    const int tiles = (last >> a.pages.log2) / kTile + 1;
    const int64_t row0 = ((int64_t)b * a.pages.n_kv_heads + h) * a.q_tokens + token0 - a.row0;
    for (int tile = tile0; tile < tiles; tile += a.splits * kScoreWaves) {
        const int here = page;
        page = page_of(a, b, tile + a.splits * kScoreWaves);
        tile_scores<BF16>(a, b, h, first_position, token0, tokens, tile, here, room[wave], [&](int t, int block, float score, float size) {
            a.scores[(row0 + t) * a.row_blocks + block] = score;
            if (block % kTile == 0) a.sizes[(row0 + t) * (a.row_blocks / kTile) + tile] = size;
        });
    }
}

// 32-bit sums are off by 2^-23 of the magnitudes per addition at most, of which 64 and 2 make a score: 2^-16.9.  The rest to 2^-16 is more than what the magnitudes are off
// by, as sums of 128 (2^-16 of themselves); and what is lost below the smallest numbers.
__device__ __forceinline__ double error_of(float size) { return 0x1p-16 * (double)size + 0x1p-110; }
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

// A query head's score of a block in 64 bits, by 16 lanes of 8 channels each.
template <bool BF16>
__device__ __forceinline__ uint64_t exact_key(const BlockArgs& a, int b, int h, int token, int g, int page) {
    const int part = threadIdx.x % 16;
    const uint16_t* bounds = (const uint16_t*)a.pages.bounds.data + page * a.pages.bounds.batch + h * a.pages.bounds.head + 8 * part;
    const short8v least = *(const short8v*)bounds, most = *(const short8v*)(bounds + a.pages.bounds.token);
    const short8v q = *(const short8v*)((const uint16_t*)a.q.data + b * a.q.batch + (h * a.G + g) * a.q.head + token * a.q.token + 8 * part);
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double x = widen16<BF16>((uint16_t)q[e]);
        sum += (x < 0.0 ? 0.0 : x) * (double)widen16<BF16>((uint16_t)most[e]) + (x > 0.0 ? 0.0 : x) * (double)widen16<BF16>((uint16_t)least[e]);
    }
#pragma unroll
    for (int d = 1; d < 16; d *= 2) sum += __shfl_xor(sum, d);
    return key_of(sum);
}

__device__ __forceinline__ uint32_t wave_min_bits(uint32_t v) { return ~wave_max_bits(~v); }
// the sum over the lanes up to this one
__device__ __forceinline__ uint32_t wave_sum_to(uint32_t x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);   // lanes 1, 2, 4, 8 before in a row of 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);   // the last of rows 0 and 2 to rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);   // the last of row 1 to rows 2 and 3
    return x;
}

constexpr int kBand = 256;            // blocks around the last chosen one that are told apart in LDS
template <int THREADS>
struct Select {
    static constexpr int kWaves = THREADS / 64, kBins = 1024;
    uint32_t bins[kBins];
    uint32_t of_wave[2][kWaves];
    uint32_t least[kWaves], most[kWaves], size[kWaves], there[kWaves];
    uint32_t found[3], above, band_n, band_index[kBand];
    int band_page[kBand];
    unsigned long long band_key[kBand];
    bool band_chosen[kBand];

    // sum over the threads before this one; total: over all (turn: 0 and 1 in turn, as what one call left is read until the next one's barrier)
    __device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t& total, int turn) {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
        const uint32_t run = wave_sum_to(x);
        if (lane == 63) of_wave[turn][wave] = run;
        __syncthreads();
        uint32_t before = 0;
        total = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) before += of_wave[turn][w];
            total += of_wave[turn][w];
        }
        return before + run - x;
    }
    // The bin of the `left`th element, counted from the last bin (every thread has counted its elements, and a barrier is behind); the number of its elements, and of those
    // behind it.
    __device__ __forceinline__ void find(uint32_t left, uint32_t& bin, uint32_t& here, uint32_t& behind, int turn) {
        constexpr int kOwn = kBins / THREADS;
        uint32_t c[kOwn], sum = 0, total;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) sum += c[i] = bins[kBins - 1 - (int)threadIdx.x * kOwn - i];
        uint32_t before = sum_before(sum, total, turn);
        if (before < left && before + sum >= left) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                if (before < left && before + c[i] >= left) found[0] = kBins - 1 - threadIdx.x * kOwn - i, found[1] = before, found[2] = c[i];
                before += c[i];
            }
        }
        __syncthreads();
        bin = found[0];
        behind = found[1];
        here = found[2];
    }
    __device__ __forceinline__ void clear() {
        for (int i = threadIdx.x; i < kBins; i += THREADS) bins[i] = 0;
    }
};

// Thread t has the blocks t * own .. t * own + own - 1 of the row.  KEEP: their scores stay in registers (as many at most); 0: they are read again in every pass.
template <bool BF16, int THREADS, int KEEP>
__global__ __launch_bounds__(THREADS) void select_kernel(BlockArgs a) {
    __shared__ Select<THREADS> s;
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const int row = a.row0 + blockIdx.x, token = row % a.q_tokens, h = row / a.q_tokens % a.pages.n_kv_heads, b = row / a.q_tokens / a.pages.n_kv_heads;
    const int n = length_of(a.q_lengths, b, a.q_tokens), N = length_of(a.kv_lengths, b, a.kv_tokens);
    if (token >= n) return;
    const int slots = a.first + a.top + a.recent;
    int32_t* list = a.blocks + (int64_t)row * slots;
    const int position = N - n + token, mine = position >= 0 ? position >> a.pages.log2 : -1;
    const int blocks = mine + 1, own = (blocks + THREADS - 1) / THREADS, first = tid * own;
    const int32_t* table = a.pages.table + b * a.pages.table_stride;
    const float* scores = a.scores + (int64_t)blockIdx.x * a.row_blocks;
    const auto has_page = [&](int c) { return c < blocks && (uint32_t)table[c] < (uint32_t)a.pages.n_pages; };
    const auto always = [&](int c) { return c < a.first || c > mine - a.recent; };
    // 0: not in the choice (nothing is where there is no choice, and no scores either)
    const auto read = [&](int i) -> uint32_t {
        if (a.top <= 0 || i >= own) return 0;
        const int c = first + i, page = table[min(c, blocks - 1)];       // (both loads at once)
        const float score = scores[min(c, blocks - 1)];
        return c < blocks && (uint32_t)page < (uint32_t)a.pages.n_pages && !always(c) ? key_of(score) : 0;
    };
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

    // how many there are, the range of their keys and the largest sum of magnitudes
    uint32_t there = 0, least = ~0u, most = 0, size = 0;
    if (a.top > 0)
        for (int i = tid; i < (blocks + kTile - 1) / kTile; i += THREADS) size = max(size, __float_as_uint(a.sizes[(int64_t)blockIdx.x * (a.row_blocks / kTile) + i]));
    s.clear();
    each([&](int, uint32_t k) {
        if (!k) return;
        ++there;
        least = min(least, k);
        most = max(most, k);
    });
    least = wave_min_bits(least), most = wave_max_bits(most), size = wave_max_bits(size), there = wave_sum_to(there);
    if (lane == 63) s.least[wave] = least, s.most[wave] = most, s.size[wave] = size, s.there[wave] = there;
    if (tid == 0) s.above = s.band_n = 0;
    __syncthreads();
    uint32_t total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) least = min(least, s.least[w]), most = max(most, s.most[w]), size = max(size, s.size[w]), total += s.there[w];

    // Chosen are: all of the choice; none; those above a band of scores, and the band's best; or, where too many are alike, the best by 64-bit keys in memory.
    enum { kAll, kNone, kNear, kExact } how;
    const uint32_t wanted = min((uint32_t)a.top, total);
    float low = 0.0f, high = 0.0f;                       // the band
    uint64_t cut = 0;                                    // kExact: the last chosen key, of whose equals the first ones are chosen
    uint32_t equal = 0, tie_at = 0;
    const auto is_near = [&](uint32_t k) { const float x = score_of(k); return !(x > high) && !(x < low); };
    uint64_t* const keys = a.keys + (int64_t)blockIdx.x * a.row_blocks;
    if (wanted == total) how = kAll;
    else if (!wanted) how = kNone;
    else {
        how = kNear;
        const double error = 2.0 * error_of(__uint_as_float(size));
        const int bits = least == most ? 1 : 32 - __builtin_clz(most - least);   // of the keys' distances from the least
        int shift = max(0, bits - 10);
        uint32_t edge = 0, here, bin, behind, left = wanted;   // the bin's first distance
        each([&](int, uint32_t k) {
            if (k) atomicAdd(&s.bins[(k - least) >> shift], 1u);
        });
        __syncthreads();
        s.find(left, bin, here, behind, 0);
        edge = bin << shift;
        left -= behind;
        // a bin of many is taken apart once
        if (here > kBand / 2 && shift) {
            const int above = shift;
            shift = max(0, shift - 10);
            s.clear();
            __syncthreads();
            each([&](int, uint32_t k) {
                if (k && ((k - least) ^ edge) >> above == 0) atomicAdd(&s.bins[((k - least) ^ edge) >> shift], 1u);
            });
            __syncthreads();
            s.find(left, bin, here, behind, 1);
            edge |= bin << shift;
        }
        // Scores beyond twice the error of the bin that holds the last chosen one are sure (rounded away from it; where the error is infinite or NaN, none is).
        const uint32_t last = edge + ((1u << shift) - 1);
        low = (float)((double)score_of(least + edge) - error), high = (float)((double)score_of(min(last, most - least) + least) + error);
        low -= fabsf(low) * 0x1p-23f, high += fabsf(high) * 0x1p-23f;
        each([&](int i, uint32_t k) {
            const uint64_t sure = __ballot(k && score_of(k) > high);
            if (sure && lane == 0) atomicAdd(&s.above, (uint32_t)__builtin_popcountll(sure));
            if (!k || !is_near(k)) return;
            const uint32_t at = atomicAdd(&s.band_n, 1u);
            if (at < kBand) s.band_index[at] = first + i, s.band_page[at] = table[first + i], s.band_key[at] = 0;
        });
        __syncthreads();
        const int band = s.band_n;
        left = wanted - s.above;
        if (band <= kBand) {
            if ((uint32_t)band != left) {                // (else all of it)
                for (int x = tid / 16; x < band * a.G; x += THREADS / 16) {
                    const uint64_t k = exact_key<BF16>(a, b, h, token, x % a.G, s.band_page[x / a.G]);
                    if (tid % 16 == 0) atomicMax(&s.band_key[x / a.G], (unsigned long long)k);
                }
                __syncthreads();
            }
            for (int e = tid; e < band; e += THREADS) {
                uint32_t better = 0;
                for (int o = 0; o < band; ++o)
                    better += s.band_key[o] > s.band_key[e] || (s.band_key[o] == s.band_key[e] && s.band_index[o] < s.band_index[e]);
                s.band_chosen[e] = better < left;
            }
            __syncthreads();
        } else {
            how = kExact;
            for (int c = tid / 16; c < blocks; c += THREADS / 16) {
                uint64_t best = 0;
                if (has_page(c) && !always(c))
                    for (int g = 0; g < a.G; ++g) {
                        const uint64_t k = exact_key<BF16>(a, b, h, token, g, table[c]);
                        best = k > best ? k : best;
                    }
                if (tid % 16 == 0) keys[c] = best;
            }
            left = wanted;
            int at = 64;
            here = total;
            for (int turn = 0; at > 0 && here != left; turn ^= 1) {
                const int above = at;
                at = max(0, at - 10);
                __syncthreads();
                s.clear();
                __syncthreads();
                for (int i = 0; i < own; ++i) {
                    const uint64_t k = first + i < blocks ? keys[first + i] : 0;
                    if (k && (above == 64 || (k ^ cut) >> above == 0)) atomicAdd(&s.bins[(k >> at) & ((1ull << (above - at)) - 1)], 1u);
                }
                __syncthreads();
                s.find(left, bin, here, behind, turn);
                left -= behind;
                cut |= (uint64_t)bin << at;
            }
            // (where all of a bin are chosen, so is all from its first key on)
            if (here == left) equal = ~0u, cut -= cut ? 1 : 0;
            else equal = left;
            __syncthreads();
            uint32_t matching = 0, unused;
            for (int i = 0; i < own; ++i) matching += first + i < blocks && keys[first + i] && keys[first + i] == cut;
            tie_at = s.sum_before(matching, unused, 0);
            if (equal == ~0u) equal = 0;
            __syncthreads();
        }
    }
    const auto chosen = [&](int i, uint32_t k, uint32_t& tie) {
        const int c = first + i;
        if (i >= own) return false;
        if (!k) return always(c) && has_page(c);
        if (how == kAll) return true;
        if (how == kNone) return false;
        if (how == kExact) return keys[c] == cut ? tie++ < equal : keys[c] > cut;
        if (!is_near(k)) return score_of(k) > high;
        for (uint32_t e = 0; e < s.band_n; ++e)
            if (s.band_index[e] == (uint32_t)c) return (bool)s.band_chosen[e];
        return false;
    };
    uint32_t number = 0, tie = tie_at, picked = 0;
    each([&](int i, uint32_t k) {
        const bool yes = chosen(i, k, tie);
        number += yes;
        if (KEEP) picked |= (uint32_t)yes << i;
    });
    uint32_t at = s.sum_before(number, total, 1);
    tie = tie_at;
    each([&](int i, uint32_t k) {
        if (KEEP ? picked >> i & 1 : chosen(i, k, tie)) list[at++] = first + i;
    });
    for (int i = total + tid; i < slots; i += THREADS) list[i] = -1;
}

constexpr int64_t kMostGroups = INT32_MAX / 1024;
// What the scores of a launch take at most, so that a long prompt's choice does not ask for its tokens times its blocks (32768 tokens of 8 KV heads behind 8192 blocks: 26 GB);
// the units go in slices, alike in size.  ms, all at once / slices of 1 GiB / of 256 MiB:
// 4096 tokens of 8 KV heads of 8 behind 8192 blocks 7.53 / 7.66 / 8.23, 1024 of 32 heads behind 4096 1.73 / 1.73 / 1.79, 512 of 8 of 8 behind 8192 0.97 / 0.98 / 1.08.
constexpr int64_t kSliceBytes = 1 << 30;

struct Plan {
    BlockArgs a{};
    int64_t rows = 0, units = 0, slice_units = 0, slice_rows = 0, bytes = 0;
    int64_t first_row(int64_t unit) const { return unit == units ? rows : unit / a.token_groups * a.q_tokens + unit % a.token_groups * a.tokens_here * a.passes; }
};

int plan_of(const specache_pages* cache, const specache_block_config* c, Plan& p) {
    if (int rc = check_blocks(cache, c)) return rc;
    BlockArgs& a = p.a;
    a.G = c->n_q_heads / cache->n_kv_heads;
    a.q_tokens = c->q_tokens;
    const int64_t blocks = ((int64_t)c->kv_tokens + cache->page_tokens - 1) / cache->page_tokens, tiles = (blocks + kTile - 1) / kTile;
    a.row_blocks = (int)(tiles * kTile);
    a.tokens_here = std::max(1, kTile / a.G);
    p.rows = (int64_t)c->batch * cache->n_kv_heads * c->q_tokens;
    const int64_t heads = (int64_t)c->batch * cache->n_kv_heads, groups = (c->q_tokens + a.tokens_here - 1) / a.tokens_here;
    const int64_t row_bytes = c->top > 0 ? a.row_blocks * (int64_t)(sizeof(uint64_t) + sizeof(float)) + tiles * (int64_t)sizeof(float) : 0;
    // a wave's bounds are read for up to 8 products' rows, where there are rows enough for 4096 waves all the same
    a.passes = (int)std::max<int64_t>(1, std::min<int64_t>(8, heads * groups * tiles / 4096));
    while (a.passes > 1 && a.tokens_here * a.passes * row_bytes > kSliceBytes) --a.passes;
    a.token_groups = (int)((groups + a.passes - 1) / a.passes);
    p.units = heads * a.token_groups;
    const int64_t unit_rows = std::max<int64_t>(1, std::min<int64_t>(c->q_tokens, a.tokens_here * a.passes));
    p.slice_units = std::min(p.units, kMostGroups / unit_rows);
    if (row_bytes) p.slice_units = std::min(p.slice_units, std::max<int64_t>(1, kSliceBytes / (unit_rows * row_bytes)));
    if (p.units) {
        const int64_t slices = (p.units + p.slice_units - 1) / p.slice_units;
        p.slice_units = (p.units + slices - 1) / slices;
    }
    p.slice_rows = std::min(p.rows, p.slice_units * unit_rows);
    a.splits = p.units ? (int)std::max<int64_t>(1, std::min<int64_t>((tiles + kScoreWaves - 1) / kScoreWaves, (1024 + p.slice_units - 1) / p.slice_units)) : 1;
    p.bytes = p.slice_rows * row_bytes;
    return SPECACHE_OK;
}

template <bool BF16>
void launch(const Plan& p, BlockArgs& a, hipStream_t stream) {
    const int threads = a.row_blocks > 1024 ? 1024 : 256;
    const auto kernel = a.row_blocks <= 512 ? select_kernel<BF16, 256, 2> : a.row_blocks <= 1024 ? select_kernel<BF16, 256, 4> : a.row_blocks <= 4096 ? select_kernel<BF16, 1024, 4>
                        : a.row_blocks <= 16384 ? select_kernel<BF16, 1024, 16> : select_kernel<BF16, 1024, 0>;
    for (int64_t unit = 0; unit < p.units; unit += p.slice_units) {
        const int64_t units = std::min(p.slice_units, p.units - unit);
        a.unit0 = (int)unit;
        a.row0 = (int)p.first_row(unit);
        if (a.top > 0 && a.row_blocks && a.pages.n_pages)
            hipLaunchKernelGGL((score_kernel<BF16>), dim3((unsigned)(units * a.splits)), dim3(64 * kScoreWaves), 0, stream, a);
        hipLaunchKernelGGL(kernel, dim3((unsigned)(p.first_row(unit + units) - a.row0)), dim3(threads), 0, stream, a);
    }
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
    a.scores = (float*)(a.keys + p.slice_rows * a.row_blocks);
    a.sizes = a.scores + p.slice_rows * a.row_blocks;
    a.batch = cfg->batch;
    a.kv_tokens = cfg->kv_tokens;
    a.top = cfg->top;
    a.first = cfg->first;
    a.recent = cfg->recent;
    if (cache->dtype == SPECACHE_BF16) launch<true>(p, a, (hipStream_t)stream);
    else launch<false>(p, a, (hipStream_t)stream);
    return launched();
}

}  // extern "C"
