// Appending to a paged cache with the rotation on the way: queries to their rows, keys and values into pages, the pages' bounds, in one launch.
//
// The first workgroups take the keys and values, the others the queries.  A workgroup of keys holds what one call brings to one page (a segment), so that
// the page's bounds need no atomics: it walks the segment's tokens head by head, keeps the running minimum and maximum of its lanes' channels in registers,
// and joins them in LDS.  Memory is what bounds it; a step's tokens, one to a page, are spread over heads instead.
#include <cmath>

#include "pages.h"
#include "rotate16.h"

namespace specache {
namespace {

constexpr int kThreads = 256, kSlots = kThreads / kParts;   // rows that a workgroup has in hand at a time
constexpr int kAhead = 4;
constexpr int64_t kMostGroups = (1ll << 32) / kThreads - 1;

struct AppendArgs {
    specache_rotary plan;
    specache_view q, q_out, k, v;
    PageArgs pages;
    const int32_t *starts, *lengths, *positions;
    int turns;                         // there is a plan
    int batch, tokens, n_q_heads;
    int segments;                      // of a sequence, at most
    int key_groups, key_splits;        // workgroups of keys and values; of them to a segment
    int key_tile_log2, q_tile_log2;    // tokens among the rows in hand
    int q_splits;
};

// kThreads lanes; the least and the largest of what the lanes of a part (and of a head, where HEADS share the workgroup) hold
struct Bounds {
    float least[16], most[16];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 16; ++i) least[i] = INFINITY, most[i] = -INFINITY;
    }
    template <bool BF16>
    __device__ __forceinline__ void take(const uint4& u0, const uint4& u1) {
        float x[2][8];
        unpack8<BF16>(u0, x[0]);
        unpack8<BF16>(u1, x[1]);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            least[i] = fminf(least[i], x[i / 8][i % 8]);
            most[i] = fmaxf(most[i], x[i / 8][i % 8]);
        }
    }
};

template <bool BF16, bool HALF, bool STREAM>
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
            const int h = h0 + i * step;
            if (h >= a.n_q_heads) continue;
            u[i][0] = *(const uint4*)(from + h * a.q.head + parts.c0);
            u[i][1] = *(const uint4*)(from + h * a.q.head + parts.c1);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int h = h0 + i * step;
            if (h >= a.n_q_heads) continue;
            if (turns) turn.apply(u[i][0], u[i][1], parts.turns[1]);
            store16<STREAM>(to + h * a.q_out.head + parts.c0, u[i][0]);
            store16<STREAM>(to + h * a.q_out.head + parts.c1, u[i][1]);
        }
    }
}

template <bool BF16, bool HALF, bool STREAM, bool BOUNDS>
__device__ __forceinline__ void append_pairs(const AppendArgs& a, int group, float (*joined)[kParts][2][16]) {
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
    int turned = -1;
    for (int hh = split * heads_here; hh < a.pages.n_kv_heads; hh += step) {
        const int h = hh + (slot >> a.key_tile_log2);
        Bounds bounds;
        bounds.clear();
        for (int pass = 0; pass < passes; ++pass) {
            const int i = pass * tile + (slot & (tile - 1));
            if (i >= tokens || h >= a.pages.n_kv_heads) continue;
            uint4 u[2], w[2];
            u[0] = *(const uint4*)(from_k + h * a.k.head + i * a.k.token + parts.c0);
            u[1] = *(const uint4*)(from_k + h * a.k.head + i * a.k.token + parts.c1);
            w[0] = *(const uint4*)(from_v + h * a.v.head + i * a.v.token + parts.c0);
            w[1] = *(const uint4*)(from_v + h * a.v.head + i * a.v.token + parts.c1);
            if (turns) {
                if (turned != pass) turn.set(a.plan, part, a.positions ? a.positions[(int64_t)b * a.tokens + t0 + i] : low + i);
                turned = pass;
                turn.apply(u[0], u[1], parts.turns[1]);
            }
            store16<STREAM>(to_k + h * a.pages.k.head + i * a.pages.k.token + parts.c0, u[0]);
            store16<STREAM>(to_k + h * a.pages.k.head + i * a.pages.k.token + parts.c1, u[1]);
            store16<STREAM>(to_v + h * a.pages.v.head + i * a.pages.v.token + parts.c0, w[0]);
            store16<STREAM>(to_v + h * a.pages.v.head + i * a.pages.v.token + parts.c1, w[1]);
            if constexpr (BOUNDS) bounds.take<BF16>(u[0], u[1]);
        }
        if constexpr (BOUNDS) {
            __syncthreads();           // (what the head before left there has been read)
#pragma unroll
            for (int c = 0; c < 16; ++c) joined[slot][part][0][c] = bounds.least[c], joined[slot][part][1][c] = bounds.most[c];
            __syncthreads();
            // one thread to a head, part and bound's access of 8 channels
            for (int x = threadIdx.x; x < heads_here * kParts * 4; x += kThreads) {
                const int p = x % kParts, which = x / kParts % 2, access = x / kParts / 2 % 2, head = hh + x / kParts / 4;
                if (head >= a.pages.n_kv_heads) continue;
                const RowParts<HALF> places(p, a.plan.rotary_dim);
                uint16_t* to = (uint16_t*)a.pages.bounds.data + page * a.pages.bounds.batch + head * a.pages.bounds.head + which * a.pages.bounds.token + (access ? places.c1 : places.c0);
                float y[8];
                if (place0 == 0) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) y[c] = which ? -INFINITY : INFINITY;
                } else unpack8<BF16>(*(const uint4*)to, y);
                const int slot0 = (x / kParts / 4) << a.key_tile_log2;
                for (int s = 0; s < min(tile, tokens); ++s)
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const float v = joined[slot0 + s][p][which][8 * access + c];
                        y[c] = which ? fmaxf(y[c], v) : fminf(y[c], v);
                    }
                *(uint4*)to = pack8<BF16>(y);
            }
        }
    }
}

template <bool BF16, bool HALF, bool STREAM, bool BOUNDS>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(AppendArgs a) {
    __shared__ float joined[BOUNDS ? kSlots : 1][kParts][2][16];
    if ((int)blockIdx.x < a.key_groups) append_pairs<BF16, HALF, STREAM, BOUNDS>(a, blockIdx.x, joined);
    else append_queries<BF16, HALF, STREAM>(a, blockIdx.x - a.key_groups);
}

template <bool BF16, bool HALF>
void launch(const AppendArgs& a, int64_t groups, bool stream_out, bool bounds, hipStream_t stream) {
    const auto kernel = stream_out ? (bounds ? paged_append_kernel<BF16, HALF, true, true> : paged_append_kernel<BF16, HALF, true, false>)
                                   : (bounds ? paged_append_kernel<BF16, HALF, false, true> : paged_append_kernel<BF16, HALF, false, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(kThreads), 0, stream, a);
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
    const auto q_tiles = [&] { return (int64_t)batch * (((int64_t)tokens + (1 << a.q_tile_log2) - 1) >> a.q_tile_log2); };
    while (n_q_heads && a.q_tile_log2 < 5 && q_tiles() >= kMostGroups / 4) ++a.q_tile_log2;
    // 16 workgroups per compute unit, if there are heads to split
    const auto splits = [](int64_t groups, int heads, int tile_log2) {
        const int64_t most = (heads + (kSlots >> tile_log2) - 1) / (kSlots >> tile_log2);
        return (int)std::min(std::max<int64_t>((4096 + groups - 1) / groups, 1), std::max<int64_t>(most, 1));
    };
    const int64_t key_tiles = cache->n_pages ? (int64_t)batch * a.segments : 0, q_tiles_n = n_q_heads ? q_tiles() : 0;
    if (key_tiles >= kMostGroups / 2 || q_tiles_n >= kMostGroups / 2) return fail_without_context(SPECACHE_EINVAL, "too many tokens");
    a.key_splits = key_tiles ? splits(key_tiles, cache->n_kv_heads, a.key_tile_log2) : 1;
    a.q_splits = q_tiles_n ? splits(q_tiles_n, n_q_heads, a.q_tile_log2) : 1;
    const int64_t key_groups = key_tiles * a.key_splits, groups = key_groups + q_tiles_n * a.q_splits;
    if (!groups) return SPECACHE_OK;
    if (groups >= kMostGroups) return fail_without_context(SPECACHE_EINVAL, "too many tokens");
    a.key_groups = (int)key_groups;
    const bool half = !plan || plan->layout == SPECACHE_ROTARY_HALF;
    const bool stream_out = (int64_t)batch * tokens * (n_q_heads + 2 * cache->n_kv_heads) * kD * 2 > kCached && (!half || a.plan.rotary_dim == kD);
    if (cache->dtype == SPECACHE_BF16) half ? launch<true, true>(a, groups, stream_out, bounds, (hipStream_t)stream) : launch<true, false>(a, groups, stream_out, bounds, (hipStream_t)stream);
    else half ? launch<false, true>(a, groups, stream_out, bounds, (hipStream_t)stream) : launch<false, false>(a, groups, stream_out, bounds, (hipStream_t)stream);
    return launched();
}
