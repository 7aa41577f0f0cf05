// Rotary positions: from a projection's rows to the rows that the cache's calls take, q and k turned, v as it is, in one launch.
//
// An angle is position * turns[i] modulo 2^64, in whole numbers: turns come in 2^-64, positions have 31 bits, so nothing is
// rounded until the top 32 bits become the binary32 argument (in turns, which is what v_sin_f32 and v_cos_f32 take).
// Far positions cost no more than near ones, and no table is read.
#include <cmath>

#include "operators.h"

namespace specache {
namespace {

struct RotateArgs {
    specache_rotary plan;
    specache_view in[3], out[3];   // q, k, v
    int heads[3];
    int batch, tokens, first;
    const int32_t* positions;
    int tile_log2;                 // tokens of a workgroup's tile
};

constexpr int kThreads = 256, kParts = 8;   // a row is 8 lanes' work: 8 pairs of channels each, two 16-byte accesses
constexpr int kAhead = 4;                   // rows whose loads a lane has in flight
constexpr int64_t kMostGroups = (1ll << 32) / kThreads;   // a launch's threads are counted in 32 bits
constexpr int64_t kCached = 32 << 20;       // bytes that the L2s of the 8 XCDs hold

typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
template <bool STREAM>
__device__ __forceinline__ void store16(uint16_t* to, const uint4& v) {
    if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(uint4v, v), (uint4v*)to);
    else *(uint4*)to = v;
}
template <bool BF16>
__device__ __forceinline__ void unpack8(const uint4& u, float (&x)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = widen16<BF16>(w[i] & 0xFFFFu);
        x[2 * i + 1] = widen16<BF16>(w[i] >> 16);
    }
}
template <bool BF16>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    return uint4{pack16<BF16>(x[0], x[1]), pack16<BF16>(x[2], x[3]), pack16<BF16>(x[4], x[5]), pack16<BF16>(x[6], x[7])};
}

// A workgroup holds a tile of up to 4 tokens times the other factor of 32 in heads at a time and walks the heads: a lane works out its 8
// angles once for all of them.  Memory is what bounds it.  The tile weighs reads, in which a token's heads lie side by side, against writes, in
// which a head's tokens do: rotating 32k tokens of 32 + 8 heads and copying 8 (805 MB, 163 us at the rate of a large copy) takes 193 us with 1
// token, 178 with 2, 172 with 4, 173 with 8, 178 with 16, 184 with 32.
// STREAM: stores that leave the caches to others, for outputs that would not stay in them (the same 172 -> 164 us), where every access of a row's 8 lanes is a
// line's 128 bytes; halves of less than the whole head, whose lines two accesses share, are written through the caches instead
// (16k tokens of 32 + 32 heads, 32 of 128 channels turned, 197 us; past them 249).
template <bool BF16, bool HALF, bool STREAM>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a) {
    const int part = threadIdx.x % kParts, slot = threadIdx.x / kParts;
    const int tile = 1 << a.tile_log2, tiles = (a.tokens + tile - 1) >> a.tile_log2;
    const int b = blockIdx.x / tiles, t = (blockIdx.x % tiles) * tile + (slot & (tile - 1));
    const int d = a.plan.rotary_dim, heads_here = (kThreads / kParts) >> a.tile_log2;
    if (t >= a.tokens) return;

    // Halves: pair e of this part joins element e of both accesses.  Neighbours: pairs 0 to 3 are the first access's, 4 to 7 the second's.  Channels that
    // stay are dealt like the others, so that an access of neighbouring lanes is in few pieces.
    const bool turns[2] = {(HALF ? 16 : 8) * part < d, HALF ? 16 * part < d : 8 * part + kD / 2 < d};
    const int c0 = HALF && !turns[0] ? d / 2 + 8 * part : 8 * part;
    const int c1 = c0 + (!HALF ? kD / 2 : turns[0] ? d / 2 : (kD - d) / 2);
    float cosine[8], sine[8];
    if (turns[0]) {
        const int64_t p = a.positions ? a.positions[(int64_t)b * a.tokens + t] : a.first + t;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int pair = HALF ? 8 * part + e : 4 * part + e % 4 + e / 4 * (kD / 4);
            const uint64_t angle = (uint64_t)p * a.plan.turns[pair];   // (0 for pairs that there are not)
            const float x = (float)(int32_t)(angle >> 32) * 0x1p-32f;
            cosine[e] = __builtin_amdgcn_cosf(x) * a.plan.gain;
            sine[e] = __builtin_amdgcn_sinf(x) * a.plan.gain;
        }
    }
    const int n_q = a.heads[0], n_k = a.heads[1], n = n_q + n_k + a.heads[2];
    const int step = heads_here * gridDim.y;
    for (int h0 = blockIdx.y * heads_here + (slot >> a.tile_log2); h0 < n; h0 += kAhead * step) {
        uint4 u[kAhead][2];
        uint16_t* to[kAhead];
        bool is_v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int h = h0 + i * step;
            to[i] = nullptr;
            if (h >= n) continue;
            const int which = h < n_q ? 0 : h < n_q + n_k ? 1 : 2;
            const int hh = which == 0 ? h : which == 1 ? h - n_q : h - n_q - n_k;
            const specache_view in = which == 0 ? a.in[0] : which == 1 ? a.in[1] : a.in[2];
            const specache_view out = which == 0 ? a.out[0] : which == 1 ? a.out[1] : a.out[2];
            const uint16_t* from = (const uint16_t*)in.data + b * in.batch + hh * in.head + t * in.token;
            to[i] = (uint16_t*)out.data + b * out.batch + hh * out.head + t * out.token;
            is_v[i] = which == 2;
            u[i][0] = *(const uint4*)(from + c0);
            u[i][1] = *(const uint4*)(from + c1);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (!to[i]) continue;
            if (turns[0] && !is_v[i]) {
                float x[2][8], y[2][8];
                unpack8<BF16>(u[i][0], x[0]);
                unpack8<BF16>(u[i][1], x[1]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int r0 = HALF ? 0 : e / 4, e0 = HALF ? e : 2 * (e % 4), r1 = HALF ? 1 : r0, e1 = HALF ? e : e0 + 1;
                    const float p = x[r0][e0], q = x[r1][e1];
                    y[r0][e0] = fmaf(p, cosine[e], -(q * sine[e]));
                    y[r1][e1] = fmaf(q, cosine[e], p * sine[e]);
                }
                u[i][0] = pack8<BF16>(y[0]);
                if (turns[1]) u[i][1] = pack8<BF16>(y[1]);
            }
            store16<STREAM>(to[i] + c0, u[i][0]);
            store16<STREAM>(to[i] + c1, u[i][1]);
        }
    }
}

bool in_place_or_apart(const specache_view& in, const specache_view& out) { return in.data != out.data || same_view(in, out); }

}  // namespace
}  // namespace specache

using namespace specache;

extern "C" {

int specache_rotary_plan(const specache_rotary_config* cfg, specache_rotary* out) {
    if (!cfg || !out) return fail_without_context(SPECACHE_EINVAL, "null configuration or output");
    const specache_rotary_config& c = *cfg;
    const int d = c.rotary_dim;
    if (d < 16 || d > kD || d % 16) return fail_without_context(SPECACHE_EINVAL, "rotary_dim must be a multiple of 16 up to 128");
    if (c.layout != SPECACHE_ROTARY_HALF && c.layout != SPECACHE_ROTARY_INTERLEAVED)
        return fail_without_context(SPECACHE_EINVAL, "layout must be SPECACHE_ROTARY_HALF or SPECACHE_ROTARY_INTERLEAVED");
    if (c.scaling < SPECACHE_ROTARY_UNSCALED || c.scaling > SPECACHE_ROTARY_RAMP) return fail_without_context(SPECACHE_EINVAL, "unknown scaling");
    if (!(c.base > 1.0) || !std::isfinite(c.base)) return fail_without_context(SPECACHE_EINVAL, "base must be above 1");
    if (c.scaling != SPECACHE_ROTARY_UNSCALED && (!(c.factor >= 1.0) || !std::isfinite(c.factor)))
        return fail_without_context(SPECACHE_EINVAL, "factor must be at least 1");
    const bool blended = c.scaling == SPECACHE_ROTARY_BANDS || c.scaling == SPECACHE_ROTARY_RAMP;
    if (blended && (c.original_tokens < 1 || !(c.low > 0.0) || !(c.high > c.low) || !std::isfinite(c.high)))
        return fail_without_context(SPECACHE_EINVAL, "original_tokens must be positive and 0 < low < high");
    if (!std::isfinite(c.gain)) return fail_without_context(SPECACHE_EINVAL, "gain must be finite");

    // in the widest type of the host: a frequency's error is multiplied by the position
    const long double two_pi = 2 * acosl(-1.0L);
    long double base = c.base, lowest = 0, highest = 0;
    if (c.scaling == SPECACHE_ROTARY_BASE) base *= powl((long double)c.factor, (long double)d / (d - 2));
    if (c.scaling == SPECACHE_ROTARY_RAMP) {
        const auto pair_of = [&](long double turns) { return d * logl(c.original_tokens / (two_pi * turns)) / (2 * logl(base)); };
        lowest = fmaxl(0.0L, floorl(pair_of(c.high)));
        highest = fminl((long double)(d - 1), ceill(pair_of(c.low)));
    }
    specache_rotary r{};
    for (int i = 0; i < d / 2; ++i) {
        long double f = powl(base, -2.0L * i / d), keep = 1;
        if (c.scaling == SPECACHE_ROTARY_LINEAR) keep = 0;
        if (c.scaling == SPECACHE_ROTARY_BANDS) keep = (c.original_tokens * f / two_pi - c.low) / ((long double)c.high - c.low);
        if (c.scaling == SPECACHE_ROTARY_RAMP) keep = 1 - (i - lowest) / fmaxl(highest - lowest, 0.001L);
        keep = fminl(fmaxl(keep, 0.0L), 1.0L);
        if (c.scaling != SPECACHE_ROTARY_UNSCALED && c.scaling != SPECACHE_ROTARY_BASE) f = keep * f + (1 - keep) * f / c.factor;
        r.turns[i] = (uint64_t)(ldexpl(f / two_pi, 64) + 0.5L);   // f <= 1: below 2^62
    }
    r.gain = (float)(c.gain > 0.0 ? c.gain : c.scaling == SPECACHE_ROTARY_RAMP ? 0.1 * std::log(c.factor) + 1.0 : 1.0);
    r.rotary_dim = d;
    r.layout = c.layout;
    *out = r;
    return SPECACHE_OK;
}

int specache_rotate(const specache_rotary* plan, int32_t dtype, int32_t batch, int32_t tokens, int32_t n_q_heads,
                    const specache_view* q, const specache_view* q_out, int32_t n_kv_heads, const specache_view* k,
                    const specache_view* k_out, const specache_view* v, const specache_view* v_out, const int32_t* positions,
                    int32_t first_position, void* stream) {
    if (!plan || plan->rotary_dim < 16 || plan->rotary_dim > kD || plan->rotary_dim % 16 ||
        (plan->layout != SPECACHE_ROTARY_HALF && plan->layout != SPECACHE_ROTARY_INTERLEAVED))
        return fail_without_context(SPECACHE_EINVAL, "plan is not one that specache_rotary_plan wrote");
    if (dtype != SPECACHE_FP16 && dtype != SPECACHE_BF16) return fail_without_context(SPECACHE_EINVAL, "dtype must be SPECACHE_FP16 or SPECACHE_BF16");
    if (batch < 0 || tokens < 0 || n_q_heads < 0 || n_kv_heads < 0) return fail_without_context(SPECACHE_EINVAL, "counts must not be negative");
    if (tokens > (1 << 30)) return fail_without_context(SPECACHE_EINVAL, "too many tokens");
    if (!positions && (int64_t)first_position + tokens > INT32_MAX) return fail_without_context(SPECACHE_EINVAL, "positions pass 2^31");
    if ((k == nullptr) != (k_out == nullptr) || (v == nullptr) != (v_out == nullptr))
        return fail_without_context(SPECACHE_EINVAL, "a tensor and its output are given or left out together");
    RotateArgs a{};
    a.plan = *plan;
    const specache_view* from[3] = {q, k, v};
    const specache_view* to[3] = {q_out, k_out, v_out};
    const int heads[3] = {n_q_heads, k ? n_kv_heads : 0, v ? n_kv_heads : 0};
    int64_t n = 0;
    for (int i = 0; i < 3; ++i) {
        a.heads[i] = heads[i];
        n += heads[i];
        if (!heads[i]) continue;
        if (!from[i] || !to[i]) return fail_without_context(SPECACHE_EINVAL, "null view");
        a.in[i] = *from[i];
        a.out[i] = *to[i];
        if (batch && tokens && (!view_fits(a.in[i]) || !view_fits(a.out[i])))
            return fail_without_context(SPECACHE_EINVAL, "a view's address must be 16-byte aligned, its strides multiples of 8");
        if (!rows_apart(a.out[i], batch, heads[i], tokens)) return fail_without_context(SPECACHE_EINVAL, "an output's rows share memory");
        if (!in_place_or_apart(a.in[i], a.out[i])) return fail_without_context(SPECACHE_EINVAL, "in place, the output's strides are the input's");
    }
    if (!batch || !tokens || !n) return SPECACHE_OK;
    if (n > (1 << 20)) return fail_without_context(SPECACHE_EINVAL, "too many heads");
    a.batch = batch;
    a.tokens = tokens;
    a.first = first_position;
    a.positions = positions;
    while (a.tile_log2 < 2 && (1 << a.tile_log2) < tokens) ++a.tile_log2;
    const auto tiles_of = [&](int log2) { return (int64_t)batch * (((int64_t)tokens + (1 << log2) - 1) >> log2); };
    while (a.tile_log2 < 5 && tiles_of(a.tile_log2) >= kMostGroups) ++a.tile_log2;
    const int64_t tiles = tiles_of(a.tile_log2);
    if (tiles >= kMostGroups) return fail_without_context(SPECACHE_EINVAL, "too many tokens");
    const int64_t passes = (n + (32 >> a.tile_log2) - 1) / (32 >> a.tile_log2);   // of a workgroup that walks all heads
    // 16 workgroups per compute unit, if there are heads to split (32k tokens in tiles of 32: 197 us with 1024 workgroups, 192 with 2048, 184 with 4096)
    int64_t split = (4096 + tiles - 1) / tiles;
    if (split < 1) split = 1;
    if (split > passes) split = passes;
    const dim3 grid((unsigned)tiles, (unsigned)split);
    const bool half = plan->layout == SPECACHE_ROTARY_HALF;
    const bool stream_out = (int64_t)batch * tokens * n * kD * 2 > kCached && (!half || plan->rotary_dim == kD);
    const auto kernel = dtype == SPECACHE_BF16
                            ? (half ? (stream_out ? rotate_kernel<true, true, true> : rotate_kernel<true, true, false>)
                                    : (stream_out ? rotate_kernel<true, false, true> : rotate_kernel<true, false, false>))
                            : (half ? (stream_out ? rotate_kernel<false, true, true> : rotate_kernel<false, true, false>)
                                    : (stream_out ? rotate_kernel<false, false, true> : rotate_kernel<false, false, false>));
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
    return launched();
}

}  // extern "C"
