// Appending to a paged cache with the rotation on the way: queries to their rows, keys and values into pages, the pages' bounds, in one launch.
//
// The first workgroups take the keys and values, the others the queries.  A workgroup of keys holds what one call brings to one page (a segment), so that
// the page's bounds need no atomics: it walks the segment's tokens head by head, keeps the running minimum and maximum of its lanes' channels in registers,
// and joins them across rows in the waves and between waves in LDS.  Memory is what bounds it; a step's tokens, one to a page, are spread over heads instead.
#include <cmath>

#include "pages.h"
#include "rotate16.h"
#include "wave_ops.h"

namespace specache {
namespace {

constexpr int kThreads = 256, kSlots = kThreads / kParts;   // rows that a workgroup has in hand at a time
constexpr int kAhead = 4, kAheadPairs = 2;   // rows whose loads a lane has in flight: queries, and keys with their values
constexpr int64_t kMostGroups = INT32_MAX / kThreads;   // of a launch, whose threads are counted in 32 bits

struct AppendArgs {
    specache_rotary plan;
    specache_view q, q_out, k, v;
    PageArgs pages;
    const int32_t *starts, *lengths, *positions;
    int turns;                         // there is a plan
    int batch, tokens, n_q_heads;
    int segments;                      // of a sequence, at most
    int64_t first_group;               // of this launch
    int key_groups, key_splits;        // workgroups of keys and values; of them to a segment
    int key_tile_log2, q_tile_log2;    // tokens among the rows in hand
    int q_splits;
};

// The least and the largest of what a lane has had of a head, channels 8 part and 64 + 8 part on: as signed whole numbers of 16 bits that are in order as the numbers are (all
// bits but the sign's turned over where that is set), which a register has two of.
typedef short short8v __attribute__((ext_vector_type(8)));
__device__ __forceinline__ short8v in_order(short8v x) { return x ^ ((x >> (short)15) & (short)0x7FFF); }   // (and back)
template <bool BF16>
struct Bounds {
    static constexpr short kInfinity = BF16 ? 0x7F80 : 0x7C00;
    short8v least[2], most[2];         // of the two accesses
    static __device__ __forceinline__ short8v numbers(const uint4& x) { return __builtin_bit_cast(short8v, x); }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 2; ++i) least[i] = kInfinity, most[i] = (short)~kInfinity;
    }
    __device__ __forceinline__ void take(const uint4 (&u)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const short8v x = numbers(u[i]), y = in_order(x), odd = (x & (short)0x7FFF) > kInfinity;   // a NaN (all ones there) is passed over
            least[i] = __builtin_elementwise_min(least[i], (y & ~odd) | (kInfinity & odd));
            most[i] = __builtin_elementwise_max(most[i], (y & ~odd) | ((short)~kInfinity & odd));
        }
    }
    // by the bounds that were: the least's two accesses, the most's
    __device__ __forceinline__ void widen(const uint4 (&old)[4]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            least[i] = __builtin_elementwise_min(least[i], in_order(numbers(old[i])));
            most[i] = __builtin_elementwise_max(most[i], in_order(numbers(old[2 + i])));
        }
    }
    // with those of the lanes 8 ROWS away
    template <int ROWS>
    __device__ __forceinline__ void meet() {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4v l = __builtin_bit_cast(uint4v, least[i]), m = __builtin_bit_cast(uint4v, most[i]);
            uint4v a[2], b[2];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                both<ROWS>(l[c], a, c);
                both<ROWS>(m[c], b, c);
            }
            least[i] = __builtin_elementwise_min(__builtin_bit_cast(short8v, a[0]), __builtin_bit_cast(short8v, a[1]));
            most[i] = __builtin_elementwise_max(__builtin_bit_cast(short8v, b[0]), __builtin_bit_cast(short8v, b[1]));
        }
    }
    // a lane's own and the other's, in some order
    template <int ROWS, typename V>
    static __device__ __forceinline__ void both(uint32_t x, V (&y)[2], int c) {
        if constexpr (ROWS == 1) {
            y[0][c] = x, y[1][c] = dpp_move_u32<kDppRowRor8>(x);
        } else {
            const auto p = ROWS == 2 ? __builtin_amdgcn_permlane16_swap(x, x, false, false) : __builtin_amdgcn_permlane32_swap(x, x, false, false);
            y[0][c] = p[0], y[1][c] = p[1];
        }
    }
    // of `rows` neighbouring rows of a wave: 1, 2, 4 or 8
    __device__ __forceinline__ void meet_rows(int rows) {
        if (rows > 1) meet<1>();
        if (rows > 2) meet<2>();
        if (rows > 4) meet<4>();
    }
};

template <bool BF16, bool HALF, bool PART, bool STREAM>
__device__ __forceinline__ void append_queries(const AppendArgs& a, int group) {
    const int part = threadIdx.x % kParts, slot = threadIdx.x / kParts;
    const int tile = 1 << a.q_tile_log2, tiles = (a.tokens + tile - 1) >> a.q_tile_log2;
    const int split = group % a.q_splits, place = group / a.q_splits;
    const int b = place / tiles, t = place % tiles * tile + (slot & (tile - 1));
    const int n = length_of(a.lengths, b, a.tokens);
    if (t >= n) return;
    const RowParts<HALF> parts(part, a.plan.rotary_dim);
    Turn<BF16, HALF> turn;
    const bool turns = a.turns && parts.turns[0];
    if (turns) turn.set(a.plan, part, a.positions ? a.positions[(int64_t)b * a.tokens + t] : (int64_t)(a.starts ? a.starts[b] : 0) + t);
    const uint16_t* from = (const uint16_t*)a.q.data + b * a.q.batch + t * a.q.token;
    uint16_t* to = (uint16_t*)a.q_out.data + b * a.q_out.batch + t * a.q_out.token;
    const int heads_here = kSlots >> a.q_tile_log2, step = heads_here * a.q_splits;
    for (int h0 = split * heads_here + (slot >> a.q_tile_log2); h0 < a.n_q_heads; h0 += kAhead * step) {
        uint4 u[kAhead][2];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int h = min(h0 + i * step, a.n_q_heads - 1);           // (of the last one again nothing is kept)
            u[i][0] = *(const uint4*)(from + h * a.q.head + parts.c0);
            u[i][1] = *(const uint4*)(from + h * a.q.head + parts.c1);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (turns) turn.apply(u[i][0], u[i][1], parts.turns[1]);
        if constexpr (PART) deal_lines(u, part, a.plan.rotary_dim);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int h = h0 + i * step;
            if (h >= a.n_q_heads) continue;
            store16<STREAM>(to + h * a.q_out.head + 8 * part, u[i][0]);
            store16<STREAM>(to + h * a.q_out.head + kD / 2 + 8 * part, u[i][1]);
        }
    }
}

template <bool BF16, bool HALF, bool PART, bool STREAM, bool BOUNDS>
__device__ __forceinline__ void append_pairs(const AppendArgs& a, int group, uint4v (*joined)[BOUNDS ? kThreads / 64 : 1][2][2][kParts]) {
    const int part = threadIdx.x % kParts, slot = threadIdx.x / kParts, tile = 1 << a.key_tile_log2;
    const int split = group % a.key_splits, segment = group / a.key_splits % a.segments, b = group / a.key_splits / a.segments;
    const int n = length_of(a.lengths, b, a.tokens);
    const int64_t start = a.starts ? a.starts[b] : 0, end = start + n;
    // the page's positions, and those of the tokens among them
    const int64_t index = (start >> a.pages.log2) + segment, at0 = index << a.pages.log2;
    const int64_t low = max(start, at0), high = min(end, at0 + (1 << a.pages.log2));
    if (low >= high || index < 0 || index >= a.pages.table_pages) return;
    const int page = a.pages.table[b * a.pages.table_stride + index];
    if ((uint32_t)page >= (uint32_t)a.pages.n_pages) return;

    const RowParts<HALF> parts(part, a.plan.rotary_dim);
    const bool turns = a.turns && parts.turns[0];
    Turn<BF16, HALF> turn;
    const int heads_here = kSlots >> a.key_tile_log2, step = heads_here * a.key_splits;
    const int tokens = (int)(high - low), passes = (tokens + tile - 1) >> a.key_tile_log2, t0 = (int)(low - start), place0 = (int)(low - at0);
    const uint16_t* from_k = (const uint16_t*)a.k.data + b * a.k.batch + t0 * a.k.token;
    const uint16_t* from_v = (const uint16_t*)a.v.data + b * a.v.batch + t0 * a.v.token;
    uint16_t* to_k = (uint16_t*)a.pages.k.data + page * a.pages.k.batch + place0 * a.pages.k.token;
    uint16_t* to_v = (uint16_t*)a.pages.v.data + page * a.pages.v.batch + place0 * a.pages.v.token;
    int turned = -1, turn_of_heads = 0;
    // The rows of up to 8 tokens are in one wave: their bounds meet there, and the page's own ones travel with the rows (a step's 16 tokens 4.4 us against 5.9 through LDS).
    const bool few = tile <= 8;
    const int heads = (a.pages.n_kv_heads - split * heads_here + step - 1) / step;    // of these lanes
    Bounds<BF16> bounds;
    uint16_t* kept = nullptr;
    // kAheadPairs rows at a time, head by head and in them pass by pass: all loads, then all stores, as a load behind a store waits for that as well
    for (int f0 = 0; f0 < heads * passes; f0 += kAheadPairs) {
        uint4 u[kAheadPairs][2], w[kAheadPairs][2];
#pragma unroll
        for (int x = 0; x < kAheadPairs; ++x) {
            const int f = min(f0 + x, heads * passes - 1), i = min(f % passes * tile + (slot & (tile - 1)), tokens - 1);
            const int h = min(split * heads_here + f / passes * step + (slot >> a.key_tile_log2), a.pages.n_kv_heads - 1);
            u[x][0] = *(const uint4*)(from_k + h * a.k.head + i * a.k.token + parts.c0);
            u[x][1] = *(const uint4*)(from_k + h * a.k.head + i * a.k.token + parts.c1);
            w[x][0] = *(const uint4*)(from_v + h * a.v.head + i * a.v.token + 8 * part);
            w[x][1] = *(const uint4*)(from_v + h * a.v.head + i * a.v.token + kD / 2 + 8 * part);
        }
        uint4 old[4] = {};
        if (BOUNDS && few && place0) {                   // (kAheadPairs heads at most: one by one)
            const int h = min(split * heads_here + f0 * step + (slot >> a.key_tile_log2), a.pages.n_kv_heads - 1);
            const uint16_t* from = (const uint16_t*)a.pages.bounds.data + page * a.pages.bounds.batch + h * a.pages.bounds.head + 8 * part;
            old[0] = *(const uint4*)from;
            old[1] = *(const uint4*)(from + kD / 2);
            old[2] = *(const uint4*)(from + a.pages.bounds.token);
            old[3] = *(const uint4*)(from + a.pages.bounds.token + kD / 2);
        }
#pragma unroll
        for (int x = 0; x < kAheadPairs; ++x) {
            const int pass = (f0 + x) % passes;
            if (turns) {
                const int i = min(pass * tile + (slot & (tile - 1)), tokens - 1);
                if (turned != pass) turn.set(a.plan, part, a.positions ? a.positions[(int64_t)b * a.tokens + t0 + i] : low + i);
                turned = pass;
                turn.apply(u[x][0], u[x][1], parts.turns[1]);
            }
        }
        if constexpr (PART) deal_lines(u, part, a.plan.rotary_dim);
#pragma unroll
        for (int x = 0; x < kAheadPairs; ++x) {
            const int f = f0 + x, i = f % passes * tile + (slot & (tile - 1)), h = split * heads_here + f / passes * step + (slot >> a.key_tile_log2);
            if (f >= heads * passes || i >= tokens || h >= a.pages.n_kv_heads) continue;
            uint16_t* k = to_k + h * a.pages.k.head + i * a.pages.k.token + 8 * part;
            uint16_t* v = to_v + h * a.pages.v.head + i * a.pages.v.token + 8 * part;
            store16<STREAM>(k, u[x][0]);
            store16<STREAM>(k + kD / 2, u[x][1]);
            store16<STREAM>(v, w[x][0]);
            store16<STREAM>(v + kD / 2, w[x][1]);
        }
        if constexpr (BOUNDS) {
#pragma unroll
            for (int x = 0; x < kAheadPairs; ++x) {
                const int f = f0 + x, pass = f % passes, i = pass * tile + (slot & (tile - 1)), hh = split * heads_here + f / passes * step;
                const int h = hh + (slot >> a.key_tile_log2);
                if (f >= heads * passes) break;
                if (pass == 0) bounds.clear();
                if (i < tokens && h < a.pages.n_kv_heads) bounds.take(u[x]);
                if (pass + 1 < passes) continue;
                if (few) {
                    kept = (uint16_t*)a.pages.bounds.data + page * a.pages.bounds.batch + h * a.pages.bounds.head + 8 * part;
                    const bool writes = (slot & (tile - 1)) == 0 && h < a.pages.n_kv_heads;
                    if (place0 && writes) {
                        if (x) {                         // (only the first head's were asked for ahead)
                            old[0] = *(const uint4*)kept;
                            old[1] = *(const uint4*)(kept + kD / 2);
                            old[2] = *(const uint4*)(kept + a.pages.bounds.token);
                            old[3] = *(const uint4*)(kept + a.pages.bounds.token + kD / 2);
                        }
                        bounds.widen(old);
                    }
                    bounds.meet_rows(tile);
                    if (writes) {
                        *(short8v*)kept = in_order(bounds.least[0]);
                        *(short8v*)(kept + kD / 2) = in_order(bounds.least[1]);
                        *(short8v*)(kept + a.pages.bounds.token) = in_order(bounds.most[0]);
                        *(short8v*)(kept + a.pages.bounds.token + kD / 2) = in_order(bounds.most[1]);
                    }
                    continue;
                }
                // a wave's 8 rows meet in it, the waves of a head in LDS (by turns in one of two places: a barrier is between a place's reads and its next writes)
                bounds.meet_rows(8);
                auto place = joined[turn_of_heads];
                turn_of_heads ^= 1;
                if (slot % 8 == 0) {
#pragma unroll
                    for (int access = 0; access < 2; ++access) {
                        place[slot / 8][0][access][part] = __builtin_bit_cast(uint4v, bounds.least[access]);
                        place[slot / 8][1][access][part] = __builtin_bit_cast(uint4v, bounds.most[access]);
                    }
                }
                __syncthreads();
                // one thread to a head, part and bound's access of 8 channels
                const int waves = tile / 8, y = threadIdx.x, p = y % kParts, which = y / kParts % 2, access = y / kParts / 2 % 2, head = hh + y / kParts / 4;
                if (y < heads_here * kParts * 4 && head < a.pages.n_kv_heads) {
                    uint4v* const to = (uint4v*)((uint16_t*)a.pages.bounds.data + page * a.pages.bounds.batch + head * a.pages.bounds.head + which * a.pages.bounds.token + access * (kD / 2) + 8 * p);
                    const int wave0 = y / kParts / 4 * waves;
                    short8v z = __builtin_bit_cast(short8v, place[wave0][which][access][p]);
                    for (int s = 1; s < waves; ++s) {
                        const short8v v = __builtin_bit_cast(short8v, place[wave0 + s][which][access][p]);
                        z = which ? __builtin_elementwise_max(z, v) : __builtin_elementwise_min(z, v);
                    }
                    if (place0) {
                        const short8v v = in_order(__builtin_bit_cast(short8v, *to));
                        z = which ? __builtin_elementwise_max(z, v) : __builtin_elementwise_min(z, v);
                    }
                    *to = __builtin_bit_cast(uint4v, in_order(z));
                }
            }
        }
    }
}

// HALF: pairs of channels are halves of what is turned; PART: which is less than the head
// (With both and bounds it spills 3 registers, which costs nothing that shows: 32768 tokens of 32 and 8 heads to pages of 64 take 156.5 us with 64 channels turned, without bounds
// 157.0, all 128 turned 154.6.)
template <bool BF16, bool HALF, bool PART, bool STREAM, bool BOUNDS>
__global__ __launch_bounds__(kThreads, 4) void paged_append_kernel(AppendArgs a) {
    __shared__ uint4v joined[2][BOUNDS ? kThreads / 64 : 1][2][2][kParts];   // [turn][wave][least, most][access][part]
    const int64_t group = a.first_group + blockIdx.x;
    if (group < a.key_groups) append_pairs<BF16, HALF, PART, STREAM, BOUNDS>(a, (int)group, joined);
    else append_queries<BF16, HALF, PART, STREAM>(a, (int)(group - a.key_groups));
}

template <bool BF16, bool HALF, bool PART>
void launch(AppendArgs& a, int64_t groups, bool stream_out, bool bounds, hipStream_t stream) {
    const auto kernel = stream_out ? (bounds ? paged_append_kernel<BF16, HALF, PART, true, true> : paged_append_kernel<BF16, HALF, PART, true, false>)
                                   : (bounds ? paged_append_kernel<BF16, HALF, PART, false, true> : paged_append_kernel<BF16, HALF, PART, false, false>);
    for (a.first_group = 0; a.first_group < groups; a.first_group += kMostGroups)
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(groups - a.first_group, kMostGroups)), dim3(kThreads), 0, stream, a);
}
template <bool BF16>
void launch(AppendArgs& a, int64_t groups, bool stream_out, bool bounds, hipStream_t stream) {
    if (a.turns && a.plan.layout == SPECACHE_ROTARY_INTERLEAVED) launch<BF16, false, false>(a, groups, stream_out, bounds, stream);
    else if (a.plan.rotary_dim == kD) launch<BF16, true, false>(a, groups, stream_out, bounds, stream);
    else launch<BF16, true, true>(a, groups, stream_out, bounds, stream);
}

}  // namespace
}  // namespace specache

using namespace specache;

extern "C" int specache_paged_append(const specache_pages* cache, const specache_rotary* plan, int32_t batch, int32_t tokens, int32_t n_q_heads,
                                     const specache_view* q, const specache_view* q_out, const specache_view* k, const specache_view* v,
                                     const int32_t* starts, const int32_t* lengths, const int32_t* positions, void* stream) {
    if (int rc = check_pages(cache)) return rc;
    if (plan && !is_plan(*plan)) return fail_without_context(SPECACHE_EINVAL, "plan is not one that specache_rotary_plan wrote");
    if (batch < 0 || tokens < 0 || n_q_heads < 0) return fail_without_context(SPECACHE_EINVAL, "counts must not be negative");
    if (n_q_heads > (1 << 20)) return fail_without_context(SPECACHE_EINVAL, "too many heads");
    if ((int64_t)batch * tokens > (1 << 30)) return fail_without_context(SPECACHE_EINVAL, "too many tokens");
    if (!batch || !tokens) return SPECACHE_OK;
    if ((uintptr_t)starts % 4 || (uintptr_t)lengths % 4 || (uintptr_t)positions % 4) return fail_without_context(SPECACHE_EINVAL, "misaligned starts, lengths or positions");
    AppendArgs a{};
    if (n_q_heads) {
        if (!q || !q_out) return fail_without_context(SPECACHE_EINVAL, "null view");
        a.q = *q;
        a.q_out = *q_out;
        if (!view_fits(a.q) || !view_fits(a.q_out)) return fail_without_context(SPECACHE_EINVAL, "a view's address must be 16-byte aligned, its strides multiples of 8");
        if (!rows_apart(a.q_out, batch, n_q_heads, tokens)) return fail_without_context(SPECACHE_EINVAL, "an output's rows share memory");
        if (!in_place_or_apart(a.q, a.q_out)) return fail_without_context(SPECACHE_EINVAL, "in place, the output's strides are the input's");
    }
    if (!k || !v) return fail_without_context(SPECACHE_EINVAL, "null view");
    a.k = *k;
    a.v = *v;
    if (!view_fits(a.k) || !view_fits(a.v)) return fail_without_context(SPECACHE_EINVAL, "a view's address must be 16-byte aligned, its strides multiples of 8");
    const bool bounds = cache->bounds.data != nullptr;
    if (int rc = check_page_views(*cache, true, bounds)) return rc;
    if (!rows_apart(cache->k, cache->n_pages, cache->n_kv_heads, cache->page_tokens) || !rows_apart(cache->v, cache->n_pages, cache->n_kv_heads, cache->page_tokens) ||
        (bounds && !rows_apart(cache->bounds, cache->n_pages, cache->n_kv_heads, 2)))
        return fail_without_context(SPECACHE_EINVAL, "the pages' rows share memory");
    if (plan) a.plan = *plan;
    else a.plan.rotary_dim = kD;
    a.turns = plan != nullptr;
    a.pages = page_args(*cache);
    a.starts = starts;
    a.lengths = lengths;
    a.positions = positions;
    a.batch = batch;
    a.tokens = tokens;
    a.n_q_heads = n_q_heads;
    const int page = cache->page_tokens;
    a.segments = starts ? (tokens + page - 2) / page + 1 : (tokens + page - 1) / page;
    while (a.key_tile_log2 < 5 && (1 << a.key_tile_log2) < std::min(tokens, page)) ++a.key_tile_log2;
    while (a.q_tile_log2 < 2 && (1 << a.q_tile_log2) < tokens) ++a.q_tile_log2;
    const int64_t q_tiles = (int64_t)batch * (((int64_t)tokens + (1 << a.q_tile_log2) - 1) >> a.q_tile_log2);   // (2^30 of these and of segments at most)
    // 16 workgroups per compute unit, if there are heads to split
    const auto splits = [](int64_t groups, int heads, int tile_log2) {
        const int64_t most = (heads + (kSlots >> tile_log2) - 1) / (kSlots >> tile_log2);
        return (int)std::min(std::max<int64_t>((4096 + groups - 1) / groups, 1), std::max<int64_t>(most, 1));
    };
    const int64_t key_tiles = cache->n_pages ? (int64_t)batch * a.segments : 0, q_tiles_n = n_q_heads ? q_tiles : 0;
    a.key_splits = key_tiles ? splits(key_tiles, cache->n_kv_heads, a.key_tile_log2) : 1;
    a.q_splits = q_tiles_n ? splits(q_tiles_n, n_q_heads, a.q_tile_log2) : 1;
    const int64_t key_groups = key_tiles * a.key_splits, groups = key_groups + q_tiles_n * a.q_splits;
    if (!groups) return SPECACHE_OK;
    a.key_groups = (int)key_groups;
    const bool stream_out = (int64_t)batch * tokens * (n_q_heads + 2 * cache->n_kv_heads) * kD * 2 > kCached;
    if (cache->dtype == SPECACHE_BF16) launch<true>(a, groups, stream_out, bounds, (hipStream_t)stream);
    else launch<false>(a, groups, stream_out, bounds, (hipStream_t)stream);
    return launched();
}
