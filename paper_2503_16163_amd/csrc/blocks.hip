// Choice of blocks of a paged cache by a cheap score: for every query row of a KV head, the blocks whose bounds promise most.
//
// score(block) = max over the KV head's query heads of  max(q, 0) . most + min(q, 0) . least, where least and most are the block's bounds: a product over 256
// channels, [max(q, 0), min(q, 0)] by [most, least].  Which block is the last chosen depends on scores next to each other, and a sum in
// 32 bits would choose differently from one order of additions to another; so products and sums have 64 bits, on the matrix cores.  (Products of
// 16-bit numbers have at most 22 bits, so that the sums are exact but where addends differ by more than 2^31.)
//
// score_kernel leaves a row's scores in scratch memory as whole numbers that are in order as the scores are; select_kernel, a workgroup to a row, finds the last chosen
// one by its bits from the top and writes the list.
#include "pages.h"
#include "wave_ops.h"

#include <algorithm>

namespace specache {
namespace {

typedef double double4v __attribute__((ext_vector_type(4)));

struct BlockArgs {
    specache_view q;
    PageArgs pages;
    const int32_t* q_lengths;
    const int32_t* kv_lengths;
    int32_t* blocks;
    uint64_t* keys;                   // [batch][KV head][token][most_blocks]
    int batch, G, q_tokens, kv_tokens, top, first, recent;
    int most_blocks;
    int tokens_here, token_groups, splits;
};

// Order of whole numbers for that of scores: the larger the later, 0 below all of them.
__device__ __forceinline__ uint64_t key_of(double x) {
    if (!(x == x)) x = -INFINITY;
    const uint64_t u = __double_as_longlong(x + 0.0);   // (of the two zeros the positive one)
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

constexpr int kScoreWaves = 4, kTile = 16;   // blocks, and rows, of a product
template <bool BF16>
__device__ __forceinline__ double element(const uint4 (&x)[4], int i) {
    const uint4& u = x[i / 8];
    const uint32_t w = i / 2 % 4 == 0 ? u.x : i / 2 % 4 == 1 ? u.y : i / 2 % 4 == 2 ? u.z : u.w;
    return (double)widen16<BF16>(i % 2 ? w >> 16 : w & 0xFFFFu);
}

// A wave's rows are up to 16 query heads: of as many tokens as fit, or of one token 16 at a time.  It walks tiles of 16 blocks: lane l has, of row and of block
// l % 16, the channels 32 s + 8 (l / 16) + e, which are two 16-byte accesses of four neighbouring lanes' 64 bytes for every s.
template <bool BF16>
__global__ __launch_bounds__(64 * kScoreWaves) void score_kernel(BlockArgs a) {
    __shared__ double scores[kScoreWaves][kTile][kTile + 1];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int split = blockIdx.x % a.splits, unit = blockIdx.x / a.splits;
    const int token0 = unit % a.token_groups * a.tokens_here, h = unit / a.token_groups % a.pages.n_kv_heads, b = unit / a.token_groups / a.pages.n_kv_heads;
    const int n = length_of(a.q_lengths, b, a.q_tokens), N = length_of(a.kv_lengths, b, a.kv_tokens);
    const int tokens = min(a.tokens_here, n - token0), last = N - n + token0 + tokens - 1;   // the last row's position
    if (tokens <= 0 || last < 0) return;
    const int tiles = (last >> a.pages.log2) / kTile + 1, rows = tokens * a.G;
    const int column = lane % 16, quarter = lane / 16;
    const int32_t* table = a.pages.table + b * a.pages.table_stride;
    const uint16_t* base = (const uint16_t*)a.pages.bounds.data + h * a.pages.bounds.head + 8 * quarter;
    for (int tile = split * kScoreWaves + wave; tile < tiles; tile += a.splits * kScoreWaves) {
        const int block = tile * kTile + column;
        int page = block < a.pages.table_pages ? table[block] : 0;
        if ((uint32_t)page >= (uint32_t)a.pages.n_pages) page = 0;
        const uint16_t* from = base + page * a.pages.bounds.batch;
        uint4 least[4], most[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            least[s] = *(const uint4*)(from + 32 * s);
            most[s] = *(const uint4*)(from + a.pages.bounds.token + 32 * s);
        }
        double of_token[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        for (int row0 = 0; row0 < rows; row0 += kTile) {
            const int r = min(row0 + column, rows - 1);
            const uint16_t* q = (const uint16_t*)a.q.data + b * a.q.batch + (h * a.G + r % a.G) * a.q.head + (token0 + r / a.G) * a.q.token + 8 * quarter;
            uint4 x[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) x[s] = *(const uint4*)(q + 32 * s);
            double4v sum[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const double y = element<BF16>(x, i);
                sum[0] = __builtin_amdgcn_mfma_f64_16x16x4f64(y < 0.0 ? 0.0 : y, element<BF16>(most, i), sum[0], 0, 0, 0);
                sum[1] = __builtin_amdgcn_mfma_f64_16x16x4f64(y > 0.0 ? 0.0 : y, element<BF16>(least, i), sum[1], 0, 0, 0);
            }
            // sum[.][i]: row 4 i + quarter, block column
#pragma unroll
            for (int i = 0; i < 4; ++i) scores[wave][4 * i + quarter][column] = sum[0][i] + sum[1][i];
            wave_sync();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = quarter + 4 * i;                           // the token's heads among these rows
                for (int g = max(t * a.G, row0); g < min(min((t + 1) * a.G, row0 + kTile), rows); ++g) of_token[i] = fmax(of_token[i], scores[wave][g - row0][column]);
            }
            wave_sync();
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = quarter + 4 * i;
            if (t < tokens && block < a.most_blocks)
                a.keys[(((int64_t)b * a.pages.n_kv_heads + h) * a.q_tokens + token0 + t) * a.most_blocks + block] = key_of(of_token[i]);
        }
    }
}

// Sum over the lanes before this one, of a workgroup; total: over all.
constexpr int kSelectThreads = 256, kSelectWaves = kSelectThreads / 64;
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t* room, uint32_t& total) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t run = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t y = __shfl_up(run, d);
        if (lane >= d) run += y;
    }
    __syncthreads();                  // (what was there has been read)
    if (lane == 63) room[wave] = run;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
        if (w < wave) before += room[w];
        total += room[w];
    }
    return before + run - x;
}

// Thread t has the blocks t * own .. t * own + own - 1 of the row.  KEEP: their keys stay in registers (as many at most); 0: they are read again in every pass.
template <int KEEP>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(BlockArgs a) {
    __shared__ uint32_t room[kSelectWaves], count[256], found[2];
    __shared__ uint64_t extremes[kSelectWaves][2];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, tid = threadIdx.x;
    const int token = blockIdx.x % a.q_tokens, b = blockIdx.x / a.q_tokens / a.pages.n_kv_heads;
    const int n = length_of(a.q_lengths, b, a.q_tokens), N = length_of(a.kv_lengths, b, a.kv_tokens);
    if (token >= n) return;
    const int slots = a.first + a.top + a.recent;
    int32_t* list = a.blocks + (int64_t)blockIdx.x * slots;
    const int position = N - n + token, mine = position >= 0 ? position >> a.pages.log2 : -1;
    const int blocks = mine + 1, own = (blocks + kSelectThreads - 1) / kSelectThreads, first = tid * own;
    const int32_t* table = a.pages.table + b * a.pages.table_stride;
    const uint64_t* keys = a.keys + (int64_t)blockIdx.x * a.most_blocks;
    const auto has_page = [&](int c) { return c < blocks && (uint32_t)table[c] < (uint32_t)a.pages.n_pages; };
    const auto always = [&](int c) { return c < a.first || c > mine - a.recent; };
    // 0: not in the choice (nothing is where there is no choice, and no scores either)
    const auto read = [&](int i) -> uint64_t { return a.top > 0 && i < own && has_page(first + i) && !always(first + i) ? keys[first + i] : 0; };
    uint64_t kept[KEEP ? KEEP : 1];
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

    // how many there are, and the bits in which they differ
    uint32_t there = 0, total;
    uint64_t least = ~0ull, most = 0;
    each([&](int, uint64_t k) {
        if (!k) return;
        ++there;
        least = k < least ? k : least;
        most = k > most ? k : most;
    });
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint64_t x = __shfl_xor(least, d), y = __shfl_xor(most, d);
        least = x < least ? x : least;
        most = y > most ? y : most;
    }
    if (lane == 0) extremes[wave][0] = least, extremes[wave][1] = most;
    sum_before(there, room, total);
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
        least = extremes[w][0] < least ? extremes[w][0] : least;
        most = extremes[w][1] > most ? extremes[w][1] : most;
    }

    // Chosen are keys above `edge` and the first `equal` ones of those that match it in the bits from `shift` on.
    uint32_t left = min((uint32_t)a.top, total), equal = 0;
    uint64_t edge = 0;
    int shift = 0;
    bool all = left == total, ties = false;
    if (!all && left) {
        int top = least == most ? 0 : 64 - __builtin_clzll(least ^ most);   // bits above are the same in all
        edge = top < 64 ? most >> top << top : 0;
        shift = top;
        uint32_t here = total;
        while (shift > 0 && here != left) {
            const int bits = min(8, shift), above = shift;
            shift -= bits;
            __syncthreads();
            count[tid] = 0;
            __syncthreads();
            each([&](int, uint64_t k) {
                if (k && (above == 64 || (k ^ edge) >> above == 0)) atomicAdd(&count[(k >> shift) & ((1 << bits) - 1)], 1u);
            });
            __syncthreads();
            if (wave == 0) {                                             // the bin that holds the last one, from the top: lane l has bins 255 - 4 l and the three below
                uint32_t c[4], sum = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += c[i] = count[255 - 4 * lane - i];
                uint32_t run = sum;
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const uint32_t y = __shfl_up(run, d);
                    if (lane >= d) run += y;
                }
                uint32_t before = run - sum;
                if (before < left && run >= left) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (before < left && before + c[i] >= left) found[0] = 255 - 4 * lane - i, found[1] = before;
                        before += c[i];
                    }
                }
            }
            __syncthreads();
            const uint32_t bin = found[0];
            left -= found[1];
            here = count[bin];
            edge |= (uint64_t)bin << shift;
        }
        equal = left;
        ties = here != left;
    }
    const auto matches = [&](uint64_t k) { return !all && left && k && k >> shift == edge >> shift; };
    const auto above = [&](uint64_t k) { return k && (all || (left && k >> shift > edge >> shift)); };
    uint32_t tie_at = 0;
    if (ties) {
        uint32_t mine_ties = 0, unused;
        each([&](int, uint64_t k) { mine_ties += matches(k); });
        tie_at = sum_before(mine_ties, room, unused);
    }
    const auto chosen = [&](int i, uint64_t k, uint32_t& tie) {
        if (i >= own) return false;
        if (matches(k)) return !ties || tie++ < equal;
        return above(k) || (always(first + i) && has_page(first + i));
    };
    uint32_t number = 0, tie = tie_at;
    each([&](int i, uint64_t k) { number += chosen(i, k, tie); });
    uint32_t at = sum_before(number, room, total);
    tie = tie_at;
    each([&](int i, uint64_t k) {
        if (chosen(i, k, tie)) list[at++] = first + i;
    });
    for (int i = total + tid; i < slots; i += kSelectThreads) list[i] = -1;
}

constexpr int64_t kMostGroups = INT32_MAX / 256;

int plan_of(const specache_pages* cache, const specache_block_config* c, BlockArgs& a, int64_t& score_groups, int64_t& rows, int64_t& bytes) {
    if (int rc = check_blocks(cache, c)) return rc;
    a.G = c->n_q_heads / cache->n_kv_heads;
    a.most_blocks = (c->kv_tokens + cache->page_tokens - 1) / cache->page_tokens;
    a.tokens_here = std::max(1, kTile / a.G);
    a.token_groups = (c->q_tokens + a.tokens_here - 1) / a.tokens_here;
    rows = (int64_t)c->batch * cache->n_kv_heads * c->q_tokens;
    const int64_t units = (int64_t)c->batch * cache->n_kv_heads * a.token_groups, tiles = (a.most_blocks + kTile - 1) / kTile;
    a.splits = units ? (int)std::max<int64_t>(1, std::min<int64_t>((tiles + kScoreWaves - 1) / kScoreWaves, (1024 + units - 1) / units)) : 1;
    score_groups = a.most_blocks ? units * a.splits : 0;
    if (rows > kMostGroups || score_groups > kMostGroups) return fail_without_context(SPECACHE_EINVAL, "too many rows");
    bytes = c->top > 0 ? rows * a.most_blocks * (int64_t)sizeof(uint64_t) : 0;
    return SPECACHE_OK;
}

}  // namespace
}  // namespace specache

using namespace specache;

extern "C" {

int specache_block_scratch(const specache_pages* cache, const specache_block_config* cfg, int64_t* bytes) {
    BlockArgs a{};
    int64_t groups, rows, select_bytes, attend_bytes;
    if (int rc = plan_of(cache, cfg, a, groups, rows, select_bytes)) return rc;
    if (int rc = block_attend_scratch(*cache, *cfg, &attend_bytes)) return rc;
    if (!bytes) return fail_without_context(SPECACHE_EINVAL, "null output");
    *bytes = std::max(select_bytes, attend_bytes);
    return SPECACHE_OK;
}

int specache_block_select(const specache_pages* cache, const specache_block_config* cfg, const specache_view* q, int32_t* blocks, const int32_t* q_lengths,
                          const int32_t* kv_lengths, void* scratch, int64_t scratch_bytes, void* stream) {
    BlockArgs a{};
    int64_t groups, rows, bytes;
    if (int rc = plan_of(cache, cfg, a, groups, rows, bytes)) return rc;
    if (!rows) return SPECACHE_OK;
    if (!q || !view_fits(*q)) return fail_without_context(SPECACHE_EINVAL, "q must be a view whose address is 16-byte aligned, its strides multiples of 8");
    if (!blocks || (uintptr_t)blocks % 4) return fail_without_context(SPECACHE_EINVAL, "null or misaligned blocks");
    if ((uintptr_t)q_lengths % 4 || (uintptr_t)kv_lengths % 4) return fail_without_context(SPECACHE_EINVAL, "misaligned lengths");
    if (cfg->kv_tokens)
        if (int rc = check_page_views(*cache, false, cfg->top > 0)) return rc;
    if (bytes) {
        if (!scratch || (uintptr_t)scratch % 16) return fail_without_context(SPECACHE_EINVAL, "scratch must be 16-byte aligned");
        if (scratch_bytes < bytes) return fail_without_context(SPECACHE_ECAPACITY, "scratch is smaller than specache_block_scratch says");
    }
    a.q = *q;
    a.pages = page_args(*cache);
    a.q_lengths = q_lengths;
    a.kv_lengths = kv_lengths;
    a.blocks = blocks;
    a.keys = (uint64_t*)scratch;
    a.batch = cfg->batch;
    a.q_tokens = cfg->q_tokens;
    a.kv_tokens = cfg->kv_tokens;
    a.top = cfg->top;
    a.first = cfg->first;
    a.recent = cfg->recent;
    hipStream_t s = (hipStream_t)stream;
    if (cfg->top > 0 && groups && cache->n_pages) {
        if (cache->dtype == SPECACHE_BF16) hipLaunchKernelGGL((score_kernel<true>), dim3((unsigned)groups), dim3(64 * kScoreWaves), 0, s, a);
        else hipLaunchKernelGGL((score_kernel<false>), dim3((unsigned)groups), dim3(64 * kScoreWaves), 0, s, a);
    }
    const auto select = a.most_blocks <= 2 * kSelectThreads ? select_kernel<2> : a.most_blocks <= 8 * kSelectThreads ? select_kernel<8>
                        : a.most_blocks <= 32 * kSelectThreads ? select_kernel<32> : select_kernel<0>;
    hipLaunchKernelGGL(select, dim3((unsigned)rows), dim3(kSelectThreads), 0, s, a);
    return launched();
}

}  // extern "C"
