// Attention over 16-bit keys and values with a sliding window and sinks.
//
// The rows of a KV head are its queries token by token, the heads that share it side by side: row r is query r / G of head
// r % G.  A workgroup takes 128 of them, 32 per wave, and walks the tiles of 64 positions that any of them sees, with the
// running maximum and sum of a softmax (the weights of a tile are rounded to the inputs' type for the product with the values, maximum,
// sum and both products are binary32).
//
// Both products run with the positions as the matrix cores' rows: S^T = K Q^T leaves a lane 16 scores of ONE query row, so
// that maximum, sum and rescaling need no exchange but one between the two halves of a wave, and what the lane holds of
// S^T is, rounded, already the operand that O^T = V^T P^T wants, if the contraction takes the positions in the order in which
// the first product leaves them (4 of the lower half, 4 of the upper, ...).  The values' operand in that order, channel by
// channel, comes from LDS through its transposing read.
#include "operators.h"

#include <algorithm>
#include <cmath>

namespace specache {
namespace {

typedef float float16v __attribute__((ext_vector_type(16)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __bf16 bfloat8v __attribute__((ext_vector_type(8)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));

constexpr int kTile = 64;             // positions of a tile
constexpr int kWaves = 4, kWaveRows = 32, kRows = kWaves * kWaveRows;
constexpr int kTileBytes = kTile * kD * 2;
constexpr float kNever = -1e30f;      // a maximum below every score: nothing seen yet
constexpr float kLazy = 8.0f;         // the maximum moves when a score exceeds it by more than this (in powers of two)
constexpr float kLog2e = 1.44269504088896340736f;

struct WindowArgs {
    specache_view q, k, v, out;
    const int32_t* q_lengths;
    const int32_t* kv_lengths;
    float* part_o;                    // [row tile][chunk][kRows][kD], not divided by the sum
    float* part_ml;                   // [row tile][chunk][kRows][2]: maximum (in powers of two), sum
    int n_kv_heads, G, q_tokens, kv_tokens, window, sinks;
    int row_tiles, chunks;
    float scale;                      // sm_scale in powers of two
};

template <bool BF16>
__device__ __forceinline__ float16v mfma32(uint4v a, uint4v b, float16v c) {
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bfloat8v, a), __builtin_bit_cast(bfloat8v, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

__device__ __forceinline__ float other_half(float v) {   // the value of the lane 32 away
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(threadIdx.x & 32 ? p[0] : p[1]);
}

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

// Where 16-byte piece c (8 channels) of position r of a tile is, in bytes.  A wave's key reads take one piece of 32 positions at a
// time, its value reads 64 bytes of 4 positions: either spreads over all banks.
__device__ __forceinline__ int key_swizzle(int r) { return r & 15; }
__device__ __forceinline__ int value_swizzle(int r) { return (r & 3) << 2 | (r >> 2 & 1) << 1; }

// One wave's quarter of a tile of keys or values: 16 positions, four at a time.  The LDS side is in order of lanes, so the pieces are
// exchanged on the way from memory.
template <bool KEYS>
struct Fetch {
    const uint16_t* base;             // position 0 of the head
    int64_t stride;
    uint32_t at[4];                   // bytes from the tile's first position to this lane's pieces
    int wave, lane;
    __device__ __forceinline__ int position(int i) const { return 16 * wave + 4 * i + lane / 16; }
    __device__ __forceinline__ uint32_t piece(int i) const {
        const int r = position(i);
        return ((lane % 16) ^ (KEYS ? key_swizzle(r) : value_swizzle(r))) * 16;
    }
    __device__ __forceinline__ void start() {
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = (uint32_t)position(i) * (uint32_t)stride * 2 + piece(i);
    }
    // Positions from `last` on are that one again (no row sees them, but they are finite if it is).
    __device__ __forceinline__ void operator()(int first, int last, char* lds) const {
        const char* tile = (const char*)(base + first * stride);
        if (first + kTile - 1 <= last) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                __builtin_amdgcn_global_load_lds((global_void*)(tile + at[i]), (lds_void*)(lds + (16 * wave + 4 * i) * kD * 2), 16, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t r = min(position(i), last - first);
                __builtin_amdgcn_global_load_lds((global_void*)(tile + (r * (uint32_t)stride * 2 + piece(i))), (lds_void*)(lds + (16 * wave + 4 * i) * kD * 2), 16, 0, 0);
            }
        }
    }
};

template <bool BF16> constexpr uint32_t kExponents = BF16 ? 0x7F807F80u : 0x7C007C00u;        // of two values: all ones where one is not finite
template <bool BF16> constexpr uint32_t kAboveExponents = BF16 ? 0x00800080u : 0x04000400u;   // added to them, it then sets the sign's bit

// What a row of queries sees: positions up to `last`, of these the sinks and those from `low` on.
struct Seen {
    int last, low, sinks;
    __device__ __forceinline__ bool operator()(int j) const { return (j <= last) & ((j < sinks) | (j >= low)); }
};

template <bool BF16, bool SPLIT>
__global__ __launch_bounds__(256, 2) void window_kernel(WindowArgs a) {
    // (arrays of their own: the compiler then sees that what is fetched into one and what is read from another do not meet)
    __shared__ __align__(1024) char keys_even[kTileBytes];
    __shared__ __align__(1024) char keys_odd[kTileBytes];
    __shared__ __align__(1024) char values_even[kTileBytes];
    __shared__ __align__(1024) char values_odd[kTileBytes];
    __shared__ int any_dropped;

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    // the row tiles of a KV head follow each other on one XCD, the longest first
    const int total = gridDim.x, per_xcd = total / 8, rest = total % 8, xcd = blockIdx.x % 8;
    const int id = xcd * per_xcd + min(xcd, rest) + blockIdx.x / 8;
    const int chunk = SPLIT ? id % a.chunks : 0;
    const int item = SPLIT ? id / a.chunks : id;
    const int head_row = item / a.row_tiles, row_tile = a.row_tiles - 1 - item % a.row_tiles;
    const int b = head_row / a.n_kv_heads, h = head_row % a.n_kv_heads;

    const int n = a.q_lengths ? min(max(a.q_lengths[b], 0), a.q_tokens) : a.q_tokens;
    const int N = a.kv_lengths ? min(max(a.kv_lengths[b], 0), a.kv_tokens) : a.kv_tokens;
    const int rows = n * a.G;
    if (row_tile * kRows >= rows) return;

    const int r = row_tile * kRows + wave * kWaveRows + lane % 32;
    const bool row_exists = r < rows;
    const int r_here = min(r, rows - 1);
    const int token = r_here / a.G, q_head = h * a.G + r_here % a.G;
    Seen seen;
    seen.last = N - n + token;
    seen.low = a.window ? seen.last - a.window + 1 : 0;
    seen.sinks = a.sinks;

    // positions that the workgroup's rows see: tiles from 0 (sinks), then tiles from low_tile on
    const int tile_last_row = min(rows, (row_tile + 1) * kRows) - 1;
    const int first_pos = N - n + row_tile * kRows / a.G, last_pos = N - n + tile_last_row / a.G;
    const int low_tile = a.window ? max(0, first_pos - a.window + 1) / kTile : 0;
    const int end_tile = last_pos < 0 ? 0 : last_pos / kTile + 1;
    const int sink_tiles = min((min(a.sinks, last_pos + 1) + kTile - 1) / kTile, low_tile);
    const int n_tiles = max(0, sink_tiles) + max(0, end_tile - low_tile);
    const auto tile_at = [&](int i) { return i < sink_tiles ? i : i - max(0, sink_tiles) + low_tile; };
    int i_begin = 0, i_end = n_tiles;
    if constexpr (SPLIT) {
        const int per = (n_tiles + a.chunks - 1) / a.chunks;
        i_begin = min(chunk * per, n_tiles);
        i_end = min(i_begin + per, n_tiles);
    }
    // the wave's own bounds, for tiles that all of its rows see
    const int wave_first = N - n + min(row_tile * kRows + wave * kWaveRows, rows - 1) / a.G;
    const int wave_last = N - n + min(row_tile * kRows + wave * kWaveRows + kWaveRows - 1, rows - 1) / a.G;
    const int wave_low = a.window ? wave_last - a.window + 1 : 0;
    const int wave_first_low = a.window ? wave_first - a.window + 1 : 0;

    uint4v qf[8];
    {
        const uint16_t* qrow = (const uint16_t*)a.q.data + b * a.q.batch + q_head * a.q.head + token * a.q.token;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) qf[kk] = *(const uint4v*)(qrow + 16 * kk + 8 * half);
    }
    Fetch<true> fetch_keys{(const uint16_t*)a.k.data + b * a.k.batch + h * a.k.head, a.k.token, {}, wave, lane};
    Fetch<false> fetch_values{(const uint16_t*)a.v.data + b * a.v.batch + h * a.v.head, a.v.token, {}, wave, lane};
    fetch_keys.start();
    fetch_values.start();

    float16v o[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.0f;
    float m = kNever, l = 0.0f;       // l: of this lane's half of the positions

    if (threadIdx.x == 0) any_dropped = 0;
    __syncthreads();
    if (i_begin < i_end) {
        fetch_keys(tile_at(i_begin) * kTile, N - 1, keys_even);
        fetch_values(tile_at(i_begin) * kTile, N - 1, values_even);
    }
    const auto is_edge = [&](int tile0) {   // some row of the workgroup does not see all of the tile
        return tile0 + kTile - 1 > first_pos || (a.window && tile0 < last_pos - a.window + 1 && tile0 + kTile > a.sinks);
    };
    const auto step = [&](int it, char* keys, char* values, char* next_keys, char* next_values) {
        const int tile0 = tile_at(it) * kTile;
        __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
        if (is_edge(tile0)) {
            // A row that does not see a value has it times zero, so values that are not finite are dropped here, by the wave that
            // fetched them, and given to the rows that see them after the walk.
            uint4v* own = (uint4v*)(values + wave * 16 * kD * 2);
            bool dropped = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint4v x = own[i * 64 + lane];
                uint32_t odd = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) odd |= (x[e] & kExponents<BF16>) + kAboveExponents<BF16>;
                if (odd & 0x80008000u) {
                    dropped = true;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t y = (x[e] & kExponents<BF16>) + kAboveExponents<BF16>;
                        x[e] &= (y & 0x8000u ? 0u : 0xFFFFu) | (y & 0x80000000u ? 0u : 0xFFFF0000u);
                    }
                    own[i * 64 + lane] = x;
                }
            }
            if (dropped) any_dropped = 1;
        }
        __syncthreads();
        if (it + 1 < i_end) {
            fetch_keys(tile_at(it + 1) * kTile, N - 1, next_keys);
            fetch_values(tile_at(it + 1) * kTile, N - 1, next_values);
        }
        // none of the wave's rows sees the tile
        if (tile0 > wave_last || (tile0 + kTile <= wave_first_low && tile0 >= a.sinks)) return;

        float16v s[2];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[hf][i] = 0.0f;
            const int row = 32 * hf + lane % 32;
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) {
                const uint4v kf = *(const uint4v*)(keys + row * kD * 2 + (((2 * kk + half) ^ key_swizzle(row)) * 16));
                s[hf] = mfma32<BF16>(kf, qf[kk], s[hf]);
            }
        }
        if (tile0 + kTile - 1 > wave_first || (tile0 < wave_low && tile0 + kTile > a.sinks)) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!seen(tile0 + 32 * hf + 8 * (i / 4) + 4 * half + i % 4)) s[hf][i] = -INFINITY;
        }
        float most = s[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) most = fmaxf(most, s[i / 16][i % 16]);
        most = fmaxf(most, other_half(most)) * a.scale;
        if (__ballot(most > m + kLazy)) {
            const float to = fmaxf(m, most), factor = __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= factor;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[dt][i] *= factor;
        }
        uint4v p[4];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[i / 16][i % 16], a.scale, -m)), y = __builtin_amdgcn_exp2f(fmaf(s[i / 16][i % 16 + 1], a.scale, -m));
            l += x;
            l += y;
            p[i / 8][i % 8 / 2] = pack16<BF16>(x, y);
        }
        // the 4 x 4 block of a lane group: position 4 half + (lane % 16) / 4, channels 16 (lane / 16 % 2) + 4 (lane % 4)
        const int vr = 4 * half + lane % 16 / 4, vc = 16 * (lane / 16 % 2) + 4 * (lane % 4);
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
                uint4v f;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int row = 16 * st + 8 * j + vr, col = 32 * dt + vc;
                    const char* at = values + row * kD * 2 + ((col / 8) ^ value_swizzle(row)) * 16 + col % 8 * 2;
                    const uint2v w = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)at));
                    f[2 * j] = w[0];
                    f[2 * j + 1] = w[1];
                }
                o[dt] = mfma32<BF16>(f, p[st], o[dt]);
            }
    };
    for (int it = i_begin; it < i_end; it += 2) {
        step(it, keys_even, values_even, keys_odd, values_odd);
        if (it + 1 < i_end) step(it + 1, keys_odd, values_odd, keys_even, values_even);
    }
    __syncthreads();
    if (any_dropped) {
        for (int it = i_begin; it < i_end; ++it) {
            const int tile0 = tile_at(it) * kTile;
            if (!is_edge(tile0)) continue;
            for (int j = tile0; j < min(tile0 + kTile, N); ++j)
#pragma unroll
                for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint32_t x = fetch_values.base[j * a.v.token + 32 * dt + 8 * (i / 4) + 4 * half + i % 4];
                        if ((x & kExponents<BF16> & 0xFFFFu) == (kExponents<BF16> & 0xFFFFu) && seen(j)) o[dt][i] += widen16<BF16>(x);
                    }
        }
    }

    l += other_half(l);
    if constexpr (SPLIT) {
        const int64_t place = ((int64_t)(item / a.row_tiles * a.row_tiles + row_tile) * a.chunks + chunk) * kRows + wave * kWaveRows + lane % 32;
        if (half == 0) {
            a.part_ml[2 * place] = m;
            a.part_ml[2 * place + 1] = l;
        }
        if (i_begin >= i_end) return;   // nothing to add, and nothing that the merge reads
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(float4*)(a.part_o + place * kD + 32 * dt + 8 * i + 4 * half) = float4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
    } else {
        if (!row_exists) return;
        const float by = l == 0.0f ? 0.0f : 1.0f / l;
        uint16_t* to = (uint16_t*)a.out.data + b * a.out.batch + q_head * a.out.head + token * a.out.token;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(uint2v*)(to + 32 * dt + 8 * i + 4 * half) =
                    uint2v{pack16<BF16>(o[dt][4 * i] * by, o[dt][4 * i + 1] * by), pack16<BF16>(o[dt][4 * i + 2] * by, o[dt][4 * i + 3] * by)};
    }
}

// The chunks of a row, joined: a wave per row, two channels per lane.
template <bool BF16>
__global__ __launch_bounds__(256) void window_merge_kernel(WindowArgs a) {
    const int lane = threadIdx.x % 64;
    const int64_t id = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    const int row = id % kRows, item = id / kRows;
    const int row_tile = item % a.row_tiles, b = item / a.row_tiles / a.n_kv_heads, h = item / a.row_tiles % a.n_kv_heads;
    const int n = a.q_lengths ? min(max(a.q_lengths[b], 0), a.q_tokens) : a.q_tokens;
    const int r = row_tile * kRows + row;
    if (r >= n * a.G) return;
    const float* ml = a.part_ml + 2 * ((int64_t)item * a.chunks * kRows + row);
    const float* po = a.part_o + ((int64_t)item * a.chunks * kRows + row) * kD + 2 * lane;
    float m = kNever;
    for (int c = 0; c < a.chunks; ++c) m = fmaxf(m, ml[(int64_t)c * kRows * 2]);
    float l = 0.0f, x = 0.0f, y = 0.0f;
    for (int c = 0; c < a.chunks; ++c) {
        const float lc = ml[(int64_t)c * kRows * 2 + 1];
        if (lc == 0.0f) continue;
        const float w = __builtin_amdgcn_exp2f(ml[(int64_t)c * kRows * 2] - m);
        const float2 oc = *(const float2*)(po + (int64_t)c * kRows * kD);
        l = fmaf(w, lc, l);
        x = fmaf(w, oc.x, x);
        y = fmaf(w, oc.y, y);
    }
    const float by = l == 0.0f ? 0.0f : 1.0f / l;
    uint16_t* to = (uint16_t*)a.out.data + b * a.out.batch + (h * a.G + r % a.G) * a.out.head + r / a.G * a.out.token;
    *(uint32_t*)(to + 2 * lane) = pack16<BF16>(x * by, y * by);
}

struct Plan {
    int row_tiles = 0, chunks = 1;
    int64_t items = 0, scratch = 0;
};

int check(const specache_window_config* c) {
    if (!c) return fail_without_context(SPECACHE_EINVAL, "null configuration");
    if (c->batch < 0 || c->q_tokens < 0 || c->kv_tokens < 0 || c->window < 0 || c->sinks < 0)
        return fail_without_context(SPECACHE_EINVAL, "batch, q_tokens, kv_tokens, window and sinks must not be negative");
    if (c->n_kv_heads < 1 || c->n_q_heads < 1 || c->n_q_heads % c->n_kv_heads || c->n_q_heads / c->n_kv_heads > 64)
        return fail_without_context(SPECACHE_EINVAL, "n_q_heads must be a multiple of n_kv_heads, up to 64 of it");
    if (c->head_dim != kD) return fail_without_context(SPECACHE_EINVAL, "head_dim must be 128");
    if (c->dtype != SPECACHE_FP16 && c->dtype != SPECACHE_BF16) return fail_without_context(SPECACHE_EINVAL, "dtype must be SPECACHE_FP16 or SPECACHE_BF16");
    if (!std::isfinite(c->sm_scale)) return fail_without_context(SPECACHE_EINVAL, "sm_scale must be finite");
    if (c->kv_tokens > (1 << 30) || (int64_t)c->q_tokens * (c->n_q_heads / c->n_kv_heads) > (1 << 30))
        return fail_without_context(SPECACHE_EINVAL, "too many tokens");
    return SPECACHE_OK;
}

// Row tiles that are too few to fill the chip (two workgroups per compute unit) have their positions split into chunks, of at least
// four tiles each.
int plan_of(const specache_window_config& c, Plan& p) {
    const int G = c.n_q_heads / c.n_kv_heads;
    p.row_tiles = (int)(((int64_t)c.q_tokens * G + kRows - 1) / kRows);
    p.items = (int64_t)c.batch * c.n_kv_heads * p.row_tiles;
    int64_t most = c.kv_tokens;
    if (c.window) most = std::min<int64_t>(most, (int64_t)c.window + c.sinks + kRows);
    const int64_t tiles = (most + kTile - 1) / kTile;
    int64_t chunks = p.items ? 512 / p.items : 1;
    chunks = std::min(chunks, tiles / 4);
    p.chunks = (int)std::max<int64_t>(chunks, 1);
    if (p.items * p.chunks > INT32_MAX / 64) return fail_without_context(SPECACHE_EINVAL, "too many rows");
    p.scratch = p.chunks > 1 ? p.items * p.chunks * kRows * (kD + 2) * (int64_t)sizeof(float) : 0;
    return SPECACHE_OK;
}

}  // namespace
}  // namespace specache

using namespace specache;

extern "C" {

int specache_window_scratch(const specache_window_config* cfg, int64_t* bytes) {
    if (int rc = check(cfg)) return rc;
    if (!bytes) return fail_without_context(SPECACHE_EINVAL, "null output");
    Plan p;
    if (int rc = plan_of(*cfg, p)) return rc;
    *bytes = p.scratch;
    return SPECACHE_OK;
}

int specache_window_attend(const specache_window_config* cfg, const specache_view* q, const specache_view* k,
                           const specache_view* v, const specache_view* out, const int32_t* q_lengths, const int32_t* kv_lengths,
                           void* scratch, int64_t scratch_bytes, void* stream) {
    if (int rc = check(cfg)) return rc;
    Plan p;
    if (int rc = plan_of(*cfg, p)) return rc;
    if (!p.items) return SPECACHE_OK;
    if (!q || !k || !v || !out) return fail_without_context(SPECACHE_EINVAL, "null view");
    if (!view_fits(*q) || !view_fits(*out) || (cfg->kv_tokens && (!view_fits(*k) || !view_fits(*v))))
        return fail_without_context(SPECACHE_EINVAL, "a view's address must be 16-byte aligned, its strides multiples of 8");
    if (k->token > (1 << 24) || v->token > (1 << 24)) return fail_without_context(SPECACHE_EINVAL, "token strides of k and v go up to 2^24");
    if (!rows_apart(*out, cfg->batch, cfg->n_q_heads, cfg->q_tokens)) return fail_without_context(SPECACHE_EINVAL, "the output's rows share memory");
    if (p.scratch) {
        if (!scratch || (uintptr_t)scratch % 16) return fail_without_context(SPECACHE_EINVAL, "scratch must be 16-byte aligned");
        if (scratch_bytes < p.scratch) return fail_without_context(SPECACHE_ECAPACITY, "scratch is smaller than specache_window_scratch says");
    }
    WindowArgs a{};
    a.q = *q;
    a.k = *k;
    a.v = *v;
    a.out = *out;
    a.q_lengths = q_lengths;
    a.kv_lengths = kv_lengths;
    a.part_o = (float*)scratch;
    a.part_ml = a.part_o + p.items * p.chunks * kRows * kD;
    a.n_kv_heads = cfg->n_kv_heads;
    a.G = cfg->n_q_heads / cfg->n_kv_heads;
    a.q_tokens = cfg->q_tokens;
    a.kv_tokens = cfg->kv_tokens;
    a.window = cfg->window;
    a.sinks = cfg->sinks;
    a.row_tiles = p.row_tiles;
    a.chunks = p.chunks;
    a.scale = (cfg->sm_scale > 0.0f ? cfg->sm_scale : 0.08838834764831845f) * kLog2e;
    const bool bf16 = cfg->dtype == SPECACHE_BF16, split = p.chunks > 1;
    const auto kernel = bf16 ? (split ? window_kernel<true, true> : window_kernel<true, false>)
                             : (split ? window_kernel<false, true> : window_kernel<false, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(p.items * p.chunks)), dim3(256), 0, (hipStream_t)stream, a);
    if (split)
        hipLaunchKernelGGL(bf16 ? window_merge_kernel<true> : window_merge_kernel<false>, dim3((unsigned)(p.items * kRows / 4)), dim3(256), 0,
                           (hipStream_t)stream, a);
    return launched();
}

}  // extern "C"
