// Attention over 16-bit keys and values with a sliding window and sinks.
//
// The rows of a KV head are its queries token by token, the heads that share it side by side: row r is query r / G of head
// r % G.  A wave takes 32 rows and walks the tiles of positions that any of them sees, with the running maximum and sum of a softmax (the
// weights of a tile are rounded to the inputs' type for the product with the values; maximum, sum and both products are binary32).
//
// Both products run with the positions as the matrix cores' rows: S^T = K Q^T leaves a lane 16 scores of ONE query row, so
// that maximum, sum and rescaling need no exchange but one between the two halves of a wave, and what the lane holds of
// S^T is, rounded, already the operand that O^T = V^T P^T wants, if the contraction takes the positions in the order in which
// the first product leaves them (4 of the lower half, 4 of the upper, ...).  The values' operand in that order, channel by
// channel, comes from LDS through its transposing read.  Keys and values go to LDS without passing registers.
//
// Two kernels.  tile_kernel, for prompts and parts of prompts: the 4 or 8 waves of a workgroup have rows of their own and share the
// tiles.  step_kernel, for up to 32 rows per KV head: a wave by itself, with tiles of its own; memory bounds it, so that
// the rows that a short step leaves empty cost nothing.  Where rows are few, either splits the positions into chunks, whose partial
// results (as fractions of the chunk's own maximum) merge_kernel joins.
#include "operators.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

namespace specache {
namespace {

typedef float float16v __attribute__((ext_vector_type(16)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __bf16 bfloat8v __attribute__((ext_vector_type(8)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));

constexpr int kWaveRows = 32;
constexpr int kRowBytes16 = kD * 2;   // a position's keys, or its values
constexpr float kNever = -FLT_MAX;    // a maximum that no finite score is below: nothing seen yet
constexpr float kFar = 0x1p20f;       // of maxima beyond it, products are rounded before the maximum is taken off
constexpr float kLazy = 8.0f;         // the maximum moves when a score exceeds it by more than this (in powers of two)
// binary16 holds all bits of numbers down to 2^-14 only, so that its weights are taken 2^7 times: up to 2^15, and those below 2^-21 of the largest lose bits, below
// 2^-32 all.  The factor is one of sums and weights alike.
template <bool BF16> constexpr float kLift = BF16 ? 0.0f : 7.0f;
constexpr float kLog2e = 1.44269504088896340736f;

struct WindowArgs {
    specache_view q, k, v, out;
    const int32_t* q_lengths;
    const int32_t* kv_lengths;
    float* part_o;                    // [item][chunk][item_rows][kD], not divided by the sum
    float* part_ml;                   // [item][chunk][item_rows][2]: maximum (in powers of two), sum
    int n_kv_heads, G, q_tokens, kv_tokens, window, sinks;
    int merge_rows;                   // items * item_rows
    int row_tiles, item_rows, chunks; // an item is a tile of item_rows rows of a KV head of a sequence
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

// Where 16-byte piece c (8 channels) of position r of a tile is: at piece c ^ swizzle(r) of the position's 16.  A wave's key reads take
// one piece of 32 positions at a time, its value reads 64 bytes of 4 positions: either spreads over all banks (no conflicts counted).
__device__ __forceinline__ int key_swizzle(int r) { return r & 15; }
__device__ __forceinline__ int value_swizzle(int r) { return (r & 3) << 2 | (r >> 2 & 1) << 1; }

// One wave's share of a tile of keys or values: FETCHES times 4 positions from position 4 * FETCHES * part on.  The LDS side is in order of
// lanes, so the pieces are exchanged on the way from memory.  A lane's places are worked out once: a tile then costs a uniform
// address and the loads (by 64-bit arithmetic per tile a prompt of 16k tokens with 32 heads took 2476 us instead of 2282).
template <bool KEYS, int FETCHES>
struct Fetch {
    const uint16_t* base;             // position 0 of the head
    int64_t stride;
    int part, lane;
    uint32_t at[FETCHES];             // bytes from the tile's first position to this lane's pieces
    __device__ __forceinline__ int position(int i) const { return 4 * (FETCHES * part + i) + lane / 16; }
    __device__ __forceinline__ uint32_t piece(int i) const {
        const int r = position(i);
        return ((lane % 16) ^ (KEYS ? key_swizzle(r) : value_swizzle(r))) * 16;
    }
    __device__ __forceinline__ Fetch(const specache_view& v, int b, int h, int part_, int lane_)
        : base((const uint16_t*)v.data + b * v.batch + h * v.head), stride(v.token), part(part_), lane(lane_) {
#pragma unroll
        for (int i = 0; i < FETCHES; ++i) at[i] = (uint32_t)position(i) * (uint32_t)stride * 2 + piece(i);
    }
    // Positions from `last` on are that one again (no row sees them, but they are finite if it is).
    __device__ __forceinline__ void operator()(int first, int tile, int last, char* lds) const {
        const char* from = (const char*)(base + first * stride);
        char* to = lds + 4 * FETCHES * part * kRowBytes16;
        if (first + tile - 1 <= last) {
#pragma unroll
            for (int i = 0; i < FETCHES; ++i)
                __builtin_amdgcn_global_load_lds((global_void*)(from + at[i]), (lds_void*)(to + 4 * i * kRowBytes16), 16, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < FETCHES; ++i) {
                const uint32_t r = min(position(i), last - first);
                __builtin_amdgcn_global_load_lds((global_void*)(from + (r * (uint32_t)stride * 2 + piece(i))), (lds_void*)(to + 4 * i * kRowBytes16), 16, 0, 0);
            }
        }
    }
};

template <bool BF16> constexpr uint32_t kExponents = BF16 ? 0x7F807F80u : 0x7C007C00u;        // of two values: all ones where one is not finite
template <bool BF16> constexpr uint32_t kAboveExponents = BF16 ? 0x00800080u : 0x04000400u;   // added to them, it then sets the sign's bit

// A row that does not see a value has it times zero.  Of tiles that some row does not see all of, values that are not finite are therefore dropped
// (by the wave that fetched them) and given to the rows that see them after the walk.  True where something was dropped.
template <bool BF16, int FETCHES>
__device__ __forceinline__ bool drop_odd_values(char* values, int part, int lane) {
    uint4v* own = (uint4v*)(values + part * FETCHES * 4 * kRowBytes16);
    bool dropped = false;
#pragma unroll
    for (int i = 0; i < FETCHES; ++i) {
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
    return dropped;
}

// What a row's sums are divided by.  No weight at all: a row that sees nothing gives zeros; one that sees scores of -infinity alone has no softmax.
__device__ __forceinline__ float divisor_of(float l, bool sees) { return l != 0.0f ? 1.0f / l : sees ? NAN : 0.0f; }

// What a row of queries sees: positions up to `last`, of these the sinks and those from `low` on.
struct Seen {
    int last, low, sinks;
    __device__ __forceinline__ bool operator()(int j) const { return (j <= last) & ((j < sinks) | (j >= low)); }
};

// The tiles of TILE positions that the rows from position `first` to `last` see between them: those with sinks, then those from the first
// row's window to the last row's own position.
template <int TILE>
struct Walk {
    int sink_tiles, low_tile, n;
    __device__ __forceinline__ Walk(int first, int last, int window, int sinks) {
        low_tile = window ? max(0, first - window + 1) / TILE : 0;
        const int end = last < 0 ? 0 : last / TILE + 1;
        sink_tiles = max(0, min((min(sinks, last + 1) + TILE - 1) / TILE, low_tile));
        n = sink_tiles + max(0, end - low_tile);
    }
    __device__ __forceinline__ int position(int i) const { return (i < sink_tiles ? i : i - sink_tiles + low_tile) * TILE; }
};
// Some row from `first` to `last` does not see all of the tile.
template <int TILE>
__device__ __forceinline__ bool is_edge(int tile0, int first, int last, int window, int sinks) {
    return tile0 + TILE - 1 > first || (window && tile0 < last - window + 1 && tile0 + TILE > sinks);
}

// A wave's 32 rows (lane l and l + 32 hold row l) and their softmax over tiles of 32 * BLOCKS positions.
template <bool BF16, int BLOCKS>
struct Rows {
    uint4v q[8];
    float16v s[BLOCKS], o[4];
    float m, l;                       // l: of this lane's half of the positions
    float by, less;                   // a weight is 2^(score by - less)
    bool far, any_far;                // the row's maximum is beyond kFar; some row's of the wave
    uint4v p[2 * BLOCKS];
    Seen seen;
    int lane, half;

    __device__ __forceinline__ void start(const uint16_t* row, int lane_, float scale) {
        lane = lane_, half = lane / 32;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) q[kk] = *(const uint4v*)(row + 16 * kk + 8 * half);
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] = 0.0f;
        m = kNever, l = 0.0f, by = scale, less = -kLift<BF16>, far = any_far = false;
    }
    __device__ __forceinline__ void scores(const char* keys) {
#pragma unroll
        for (int i = 0; i < 16 * BLOCKS; ++i) s[i / 16][i % 16] = 0.0f;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
#pragma unroll
            for (int blk = 0; blk < BLOCKS; ++blk) {
                const int r = 32 * blk + lane % 32;
                s[blk] = mfma32<BF16>(*(const uint4v*)(keys + r * kRowBytes16 + (((2 * kk + half) ^ key_swizzle(r)) * 16)), q[kk], s[blk]);
            }
    }
    // position of s[i / 16][i % 16] in a tile, less 4 * half
    static __device__ __forceinline__ constexpr int place(int i) { return 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4; }
    __device__ __forceinline__ void mask(int tile0) {
        const Seen here{seen.last - tile0 - 4 * half, seen.low - tile0 - 4 * half, seen.sinks - tile0 - 4 * half};
#pragma unroll
        for (int i = 0; i < 16 * BLOCKS; ++i) {
            if (!here(place(i))) s[i / 16][i % 16] = -INFINITY;
            if (i % 2) __builtin_amdgcn_sched_barrier(0);   // few conditions at a time: they live in scalar registers
        }
    }
    // The maximum moves rarely, so that the sums do (each row's by its own scores alone): weights up to 2^kLazy of a row's own maximum keep all their bits.
    // A weight's exponent is the exact product of score and scale less the rounded one that the maximum is: half a step of the maximum is a factor of all of a
    // row's weights, which does not count while the maximum is small; of one beyond kFar the products are rounded as the maximum was.
    __device__ __forceinline__ void move_maximum(float scale) {
        float most = s[0][0];
#pragma unroll
        for (int i = 1; i < 16 * BLOCKS; ++i) most = fmaxf(most, s[i / 16][i % 16]);
        most = fmaxf(most, other_half(most)) * scale;
        if (__ballot(most > m + kLazy)) {
            const float to = most > m + kLazy ? most : m, factor = __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= factor;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[dt][i] *= factor;
            far = fabsf(m) > kFar && m != kNever;
            any_far = __ballot(far);
            by = far ? 1.0f : scale, less = (far || m == kNever ? 0.0f : m) - kLift<BF16>;
        }
        if (any_far)
#pragma unroll
            for (int i = 0; i < 16 * BLOCKS; ++i) s[i / 16][i % 16] = far ? s[i / 16][i % 16] * scale - m : s[i / 16][i % 16];
    }
    __device__ __forceinline__ void weights() {
#pragma unroll
        for (int i = 0; i < 16 * BLOCKS; i += 2) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[i / 16][i % 16], by, -less)), y = __builtin_amdgcn_exp2f(fmaf(s[i / 16][i % 16 + 1], by, -less));
            l += x;
            l += y;
            p[i / 8][i % 8 / 2] = pack16<BF16>(x, y);
        }
    }
    __device__ __forceinline__ void add_values(const char* values) {
        // the 4 x 4 block of a lane group: position 4 half + (lane % 16) / 4, channels 16 (lane / 16 % 2) + 4 (lane % 4)
        const int vr = 4 * half + lane % 16 / 4, vc = 16 * (lane / 16 % 2) + 4 * (lane % 4);
#pragma unroll
        for (int st = 0; st < 2 * BLOCKS; ++st)
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
                uint4v f;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int r = 16 * st + 8 * j + vr, c = 32 * dt + vc;
                    const char* at = values + r * kRowBytes16 + ((c / 8) ^ value_swizzle(r)) * 16 + c % 8 * 2;
                    const uint2v w = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)at));
                    f[2 * j] = w[0];
                    f[2 * j + 1] = w[1];
                }
                o[dt] = mfma32<BF16>(f, p[st], o[dt]);
            }
    }
    // what drop_odd_values dropped of positions tile0 to end - 1
    __device__ void give_odd_values(const uint16_t* values, int64_t stride, int tile0, int end) {
        for (int j = tile0; j < end; ++j)
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t x = values[j * stride + 32 * dt + 8 * (i / 4) + 4 * half + i % 4];
                    if ((x & kExponents<BF16> & 0xFFFFu) == (kExponents<BF16> & 0xFFFFu) && seen(j)) o[dt][i] += widen16<BF16>(x);
                }
    }
    __device__ __forceinline__ void store(uint16_t* to) {
        const float by = divisor_of(l, seen.last >= 0);
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(uint2v*)(to + 32 * dt + 8 * i + 4 * half) =
                    uint2v{pack16<BF16>(o[dt][4 * i] * by, o[dt][4 * i + 1] * by), pack16<BF16>(o[dt][4 * i + 2] * by, o[dt][4 * i + 3] * by)};
    }
    // something: the chunk had a tile; without one the merge reads no sums of this chunk
    __device__ __forceinline__ void store_part(float* part_o, float* part_ml, int64_t place, bool something) {
        if (half == 0) *(float2*)(part_ml + 2 * place) = float2{m, l};
        if (!something) return;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(float4*)(part_o + place * kD + 32 * dt + 8 * i + 4 * half) = float4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
    }
};

__device__ __forceinline__ int length_of(const int32_t* lengths, int b, int most) { return lengths ? min(max(lengths[b], 0), most) : most; }

// The workgroups of a KV head of a sequence (per_head) follow each other on one XCD (workgroups go to the 8 XCDs in turn), whose L2 they share. Heads
// are dealt to the XCDs in turn, so that a long sequence of a batch is everybody's (5 prompts of up to 3001 tokens, in stretches of heads 194 us, so 141); of the last ones, fewer
// than 8, each XCD has a stretch.
__device__ __forceinline__ int on_one_xcd(int per_head) {
    const int xcd = blockIdx.x % 8, dealt = gridDim.x / per_head / 8 * 8 * per_head;
    if ((int)blockIdx.x < dealt) {
        const int at = blockIdx.x / 8;
        return (at / per_head * 8 + xcd) * per_head + at % per_head;
    }
    const int total = gridDim.x - dealt, per_xcd = total / 8, rest = total % 8;
    return dealt + xcd * per_xcd + min(xcd, rest) + (blockIdx.x - dealt) / 8;
}

// Tiles of 64 positions travel to LDS while the one before is worked on; a wave takes 1/WAVES of a tile's keys and values.
// us, 32 heads over a prompt of 16k tokens: 2165 (1.02 PFLOP/s, the matrix cores busy 0.52 of the time at the clock that random inputs leave; 2130 to 2230 from one card to
// another), 8 heads of 4 queries over 32k through a window of 4096 1950 to 2140, 256 tokens of 8 heads of 8 behind 32k 250 to 267 and the merge.
template <bool BF16, bool SPLIT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void tile_kernel(WindowArgs a) {
    constexpr int TILE = 64, ROWS = WAVES * kWaveRows, FETCHES = 16 / WAVES;
    // (arrays of their own: the compiler then sees that what is fetched into one and what is read from another do not meet, and
    // does not wait for the next tile in front of a tile's reads)
    __shared__ __align__(1024) char keys_even[TILE * kRowBytes16];
    __shared__ __align__(1024) char keys_odd[TILE * kRowBytes16];
    __shared__ __align__(1024) char values_even[TILE * kRowBytes16];
    __shared__ __align__(1024) char values_odd[TILE * kRowBytes16];
    __shared__ int any_dropped;

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int id = on_one_xcd(SPLIT ? a.row_tiles * a.chunks : a.row_tiles), chunk = SPLIT ? id % a.chunks : 0, item = SPLIT ? id / a.chunks : id;
    const int b = item / a.row_tiles / a.n_kv_heads, h = item / a.row_tiles % a.n_kv_heads;
    const int row_tile = a.row_tiles - 1 - item % a.row_tiles;   // the longest first
    const int n = length_of(a.q_lengths, b, a.q_tokens), N = length_of(a.kv_lengths, b, a.kv_tokens);
    const int rows = n * a.G, row0 = row_tile * ROWS, wave_row0 = row0 + wave * kWaveRows;
    if (row0 >= rows) return;

    const int row = wave_row0 + lane % 32, r = min(row, rows - 1), token = r / a.G, q_head = h * a.G + r % a.G;
    const int first = N - n + row0 / a.G, last = N - n + min(row0 + ROWS - 1, rows - 1) / a.G;
    const int wave_first = N - n + min(wave_row0, rows - 1) / a.G, wave_last = N - n + min(wave_row0 + kWaveRows - 1, rows - 1) / a.G;
    const int wave_first_low = a.window ? wave_first - a.window + 1 : 0;
    const Walk<TILE> walk(first, last, a.window, a.sinks);
    int i_begin = 0, i_end = walk.n;
    if constexpr (SPLIT) {
        i_begin = (int)((int64_t)walk.n * chunk / a.chunks);
        i_end = (int)((int64_t)walk.n * (chunk + 1) / a.chunks);
    }

    Rows<BF16, TILE / 32> rs;
    rs.seen = Seen{N - n + token, a.window ? N - n + token - a.window + 1 : 0, a.sinks};
    rs.start((const uint16_t*)a.q.data + b * a.q.batch + q_head * a.q.head + token * a.q.token, lane, a.scale);
    const Fetch<true, FETCHES> fetch_keys(a.k, b, h, wave, lane);
    const Fetch<false, FETCHES> fetch_values(a.v, b, h, wave, lane);

    if (threadIdx.x == 0) any_dropped = 0;
    __syncthreads();
    if (i_begin < i_end) {
        fetch_keys(walk.position(i_begin), TILE, N - 1, keys_even);
        fetch_values(walk.position(i_begin), TILE, N - 1, values_even);
    }
    const auto step = [&](int it, char* keys, char* values, char* next_keys, char* next_values) __attribute__((always_inline)) {
        const int tile0 = walk.position(it);
        __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
        if (is_edge<TILE>(tile0, first, last, a.window, a.sinks) && drop_odd_values<BF16, FETCHES>(values, wave, lane)) any_dropped = 1;
        __syncthreads();
        if (it + 1 < i_end) {
            fetch_keys(walk.position(it + 1), TILE, N - 1, next_keys);
            fetch_values(walk.position(it + 1), TILE, N - 1, next_values);
        }
        // none of the wave's rows sees the tile
        if (tile0 > wave_last || (tile0 + TILE <= wave_first_low && tile0 >= a.sinks)) return;
        rs.scores(keys);
        // the first reads ahead of the products, then one beside each
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int i = 0; i < 10; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 6, 0);
        if (is_edge<TILE>(tile0, wave_first, wave_last, a.window, a.sinks)) rs.mask(tile0);
        rs.move_maximum(a.scale);
        rs.weights();
        rs.add_values(values);
        // the first step's weights, then the others' beside the products
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 28, 0);
#pragma unroll
        for (int i = 0; i < 12; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 7, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    };
    for (int it = i_begin; it < i_end; it += 2) {
        step(it, keys_even, values_even, keys_odd, values_odd);
        if (it + 1 < i_end) step(it + 1, keys_odd, values_odd, keys_even, values_even);
    }
    __syncthreads();
    if (any_dropped)
        for (int it = i_begin; it < i_end; ++it) {
            const int tile0 = walk.position(it);
            if (is_edge<TILE>(tile0, first, last, a.window, a.sinks)) rs.give_odd_values(fetch_values.base, a.v.token, tile0, min(tile0 + TILE, N));
        }
    rs.l += other_half(rs.l);
    if constexpr (SPLIT)
        rs.store_part(a.part_o, a.part_ml, ((int64_t)item * a.chunks + chunk) * ROWS + wave * kWaveRows + lane % 32, i_begin < i_end);
    else if (row < rows)
        rs.store((uint16_t*)a.out.data + b * a.out.batch + q_head * a.out.head + token * a.out.token);
}

// Waves by themselves: 32 positions at a time, the next ones on their way while a wave works on these; the waves of a workgroup take a chunk's
// tiles in turn and join their results in LDS at its end.  Memory is what bounds it, latency where a wave has few tiles (1.0 us each: 64, 128, 192
// and 256 positions of 32 heads without chunks take 5.4, 6.4, 7.4 and 8.4 us, the launch among them).  32 heads and two rows over 2048, 4096 and 8192 positions, not in
// the caches, take 13.3, 19.0 and 30.0 us: 8 for two launches, their first loads and the join, and the bytes at 6 TB/s.  By
// workgroups of 1, 2 and 4 waves, with one round of them, us (the time of reading once at 6.2 TB/s): 32 heads over 32768 positions 98, 100, 115
// (87), 4 of 32 on 8 heads and two rows over 8192 33, 32, 32 (22), one sequence of 1 head over 100000 35, 28, 24 (8), 32 heads and two rows through a
// window of 4096 22, 23, 23 (11); 16 ragged sequences of 8 heads up to 32768 265, 251, 262 (203), and 236 with workgroups dealt to the XCDs
// as they come instead of a sequence's together.
template <bool BF16, bool SPLIT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void step_kernel(WindowArgs a) {
    constexpr int TILE = 32, FETCHES = 8, BYTES = TILE * kRowBytes16;
    __shared__ __align__(1024) char keys_even[WAVES * BYTES];
    __shared__ __align__(1024) char keys_odd[WAVES * BYTES];
    __shared__ __align__(1024) char values_even[WAVES * BYTES];
    __shared__ __align__(1024) char values_odd[WAVES * BYTES];
    __shared__ float2 joined[WAVES][kWaveRows];

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int id = blockIdx.x, chunk = SPLIT ? id % a.chunks : 0, item = SPLIT ? id / a.chunks : id;
    const int b = item / a.n_kv_heads, h = item % a.n_kv_heads;
    const int n = length_of(a.q_lengths, b, a.q_tokens), N = length_of(a.kv_lengths, b, a.kv_tokens);
    const int rows = n * a.G;
    if (!rows) return;

    const int row = lane % 32, r = min(row, rows - 1), token = r / a.G, q_head = h * a.G + r % a.G;
    const int first = N - n, last = N - 1;
    const Walk<TILE> walk(first, last, a.window, a.sinks);
    int i_begin = 0, i_end = walk.n;
    if constexpr (SPLIT) {
        i_begin = (int)((int64_t)walk.n * chunk / a.chunks);
        i_end = (int)((int64_t)walk.n * (chunk + 1) / a.chunks);
    }
    const int i_first = i_begin + wave;

    Rows<BF16, 1> rs;
    rs.seen = Seen{N - n + token, a.window ? N - n + token - a.window + 1 : 0, a.sinks};
    const Fetch<true, FETCHES> fetch_keys(a.k, b, h, 0, lane);
    const Fetch<false, FETCHES> fetch_values(a.v, b, h, 0, lane);
    bool dropped = false;
    if (i_first < i_end) {
        fetch_keys(walk.position(i_first), TILE, N - 1, keys_even + wave * BYTES);
        fetch_values(walk.position(i_first), TILE, N - 1, values_even + wave * BYTES);
    }
    rs.start((const uint16_t*)a.q.data + b * a.q.batch + q_head * a.q.head + token * a.q.token, lane, a.scale);
    const auto step = [&](int it, char* keys, char* values, char* next_keys, char* next_values) __attribute__((always_inline)) {
        const int tile0 = walk.position(it);
        const bool more = it + WAVES < i_end;
        asm volatile("" ::: "memory");        // (the buffers' last reads are behind)
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
        if (more) {
            fetch_keys(walk.position(it + WAVES), TILE, N - 1, next_keys + wave * BYTES);
            fetch_values(walk.position(it + WAVES), TILE, N - 1, next_values + wave * BYTES);
            __builtin_amdgcn_s_waitcnt(0x4F78);   // vmcnt(24): this tile's keys are there
        } else {
            __builtin_amdgcn_s_waitcnt(0x0F78);   // vmcnt(8)
        }
        asm volatile("" ::: "memory");
        rs.scores(keys + wave * BYTES);
        const bool edge = is_edge<TILE>(tile0, first, last, a.window, a.sinks);
        if (edge) rs.mask(tile0);
        rs.move_maximum(a.scale);
        rs.weights();
        asm volatile("" ::: "memory");
        if (more) __builtin_amdgcn_s_waitcnt(0x4F70);   // vmcnt(16): and its values
        else __builtin_amdgcn_s_waitcnt(0x0F70);
        asm volatile("" ::: "memory");
        if (edge) dropped |= drop_odd_values<BF16, FETCHES>(values + wave * BYTES, 0, lane);
        rs.add_values(values + wave * BYTES);
    };
    for (int it = i_first; it < i_end; it += 2 * WAVES) {
        step(it, keys_even, values_even, keys_odd, values_odd);
        if (it + WAVES < i_end) step(it + WAVES, keys_odd, values_odd, keys_even, values_even);
    }
    if (__ballot(dropped))
        for (int it = i_first; it < i_end; it += WAVES) {
            const int tile0 = walk.position(it);
            if (is_edge<TILE>(tile0, first, last, a.window, a.sinks)) rs.give_odd_values(fetch_values.base, a.v.token, tile0, min(tile0 + TILE, N));
        }
    rs.l += other_half(rs.l);

    // every wave's sums to LDS (a row's channels turned by 4 per row: no two rows of a group of lanes meet in a bank), then four channels per thread
    __syncthreads();
    char* const room = wave == 0 ? keys_even : wave == 1 ? keys_odd : wave == 2 ? values_even : values_odd;
    if (row < rows) {
        if (lane < 32) joined[wave][row] = float2{rs.m, rs.l};
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(float4*)(room + (row * kD + (32 * dt + 8 * i + 4 * rs.half + 4 * row) % kD) * 4) =
                    float4{rs.o[dt][4 * i], rs.o[dt][4 * i + 1], rs.o[dt][4 * i + 2], rs.o[dt][4 * i + 3]};
    }
    __syncthreads();
    for (int at = threadIdx.x; at < rows * (kD / 4); at += 64 * WAVES) {
        const int row = at / (kD / 4), c = at % (kD / 4) * 4;
        float m = kNever, l = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, joined[w][row].x);
        float4 o{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float2 ml = joined[w][row];
            const float f = __builtin_amdgcn_exp2f(ml.x - m);
            const char* from = w == 0 ? keys_even : w == 1 ? keys_odd : w == 2 ? values_even : values_odd;
            const float4 x = *(const float4*)(from + (row * kD + (c + 4 * row) % kD) * 4);
            l = fmaf(f, ml.y, l);
            o.x = fmaf(f, x.x, o.x), o.y = fmaf(f, x.y, o.y), o.z = fmaf(f, x.z, o.z), o.w = fmaf(f, x.w, o.w);
        }
        if constexpr (SPLIT) {
            const int64_t place = ((int64_t)item * a.chunks + chunk) * a.item_rows + row;
            if (c == 0) *(float2*)(a.part_ml + 2 * place) = float2{m, l};
            *(float4*)(a.part_o + place * kD + c) = o;
        } else {
            const float by = divisor_of(l, first + row / a.G >= 0);
            uint16_t* to = (uint16_t*)a.out.data + b * a.out.batch + (h * a.G + row % a.G) * a.out.head + row / a.G * a.out.token;
            *(uint2v*)(to + c) = uint2v{pack16<BF16>(o.x * by, o.y * by), pack16<BF16>(o.z * by, o.w * by)};
        }
    }
}

// The chunks of a row, joined: two channels per lane, the chunks dealt to the waves of a workgroup.  What it takes is latency, so every load of a
// wave's first chunks is asked for at once, and each wave goes by its own chunks' maximum (4.9 us of a step of one short sequence
// with the loads behind the row's maximum, 4.5 so).
// Up to kFewChunks a wave takes a row by itself, without LDS: 4 chunks of 16384 rows, 34 MB, 9.8 us (3.4 TB/s) against 39 with four waves to a
// row, three of them for one chunk each.
constexpr int kMergeWaves = 4, kFewChunks = 4;
template <bool BF16, int WAVES>
__global__ __launch_bounds__(64 * kMergeWaves) void merge_kernel(WindowArgs a) {
    __shared__ float part[WAVES][kD];
    __shared__ float2 joined[WAVES];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64 % WAVES;
    const int place_of_row = blockIdx.x * (kMergeWaves / WAVES) + threadIdx.x / (64 * WAVES);
    const int row = place_of_row % a.item_rows, item = place_of_row / a.item_rows;
    if (WAVES < kMergeWaves && place_of_row >= a.merge_rows) return;
    const int b = item / a.row_tiles / a.n_kv_heads, h = item / a.row_tiles % a.n_kv_heads;
    const int r = (a.row_tiles - 1 - item % a.row_tiles) * a.item_rows + row;
    const int n = length_of(a.q_lengths, b, a.q_tokens);
    const int64_t place = (int64_t)item * a.chunks * a.item_rows + row;
    const float2* ml = (const float2*)a.part_ml + place;
    const float* po = a.part_o + place * kD + 2 * lane;
    float m = kNever, l = 0.0f, x = 0.0f, y = 0.0f;
    constexpr int kAhead = WAVES == 1 ? kFewChunks : 8;
    for (int c0 = wave; c0 < a.chunks; c0 += kAhead * WAVES) {
        float2 one[kAhead], oc[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t at = (int64_t)min(c0 + i * WAVES, a.chunks - 1) * a.item_rows;
            one[i] = ml[at];
            oc[i] = *(const float2*)(po + at * kD);
        }
        if (r >= n * a.G) return;      // (no row: nothing was stored, and nothing is asked of what was loaded)
        float most = m;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) most = fmaxf(most, one[i].x);
        const float moved = __builtin_amdgcn_exp2f(m - most);
        l *= moved, x *= moved, y *= moved;
        m = most;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (c0 + i * WAVES >= a.chunks || one[i].y == 0.0f) continue;   // (an empty chunk stored no sums)
            const float w = __builtin_amdgcn_exp2f(one[i].x - m);
            l = fmaf(w, one[i].y, l);
            x = fmaf(w, oc[i].x, x);
            y = fmaf(w, oc[i].y, y);
        }
    }
    if constexpr (WAVES > 1) {
        *(float2*)&part[wave][2 * lane] = float2{x, y};
        if (lane == 0) joined[wave] = float2{m, l};
        __syncthreads();
        if (wave || r >= n * a.G) return;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, joined[w].x);
        l = x = y = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(joined[w].x - m);
            const float2 o = *(const float2*)&part[w][2 * lane];
            l = fmaf(f, joined[w].y, l);
            x = fmaf(f, o.x, x);
            y = fmaf(f, o.y, y);
        }
    }
    const float by = divisor_of(l, length_of(a.kv_lengths, b, a.kv_tokens) - n + r / a.G >= 0);
    uint16_t* to = (uint16_t*)a.out.data + b * a.out.batch + (h * a.G + r % a.G) * a.out.head + r / a.G * a.out.token;
    *(uint32_t*)(to + 2 * lane) = pack16<BF16>(x * by, y * by);
}

constexpr int kStepWaves = 2;
enum { kStep, kTile4, kTile8 };
struct Plan {
    int kernel = kStep, row_tiles = 1, item_rows = 0, chunks = 1;
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
    // (positions, and their distances from a window's or a tile's edge, then keep to 32 bits)
    if (c->kv_tokens > (1 << 28) || (int64_t)c->q_tokens * (c->n_q_heads / c->n_kv_heads) > (1 << 28))
        return fail_without_context(SPECACHE_EINVAL, "too many tokens");
    return SPECACHE_OK;
}

// a window that holds every position is none
int window_of(const specache_window_config& c) { return c.window < c.kv_tokens ? c.window : 0; }

// Steps: one round of workgroups (two on a compute unit by their LDS), chunks of at most 64 tiles (2048 positions) so that a ragged batch's lengths
// even out, a tile for every wave at least, and no more than 256 chunks of a row to merge unless they are that long.  us, by chunks: one sequence of 8
// KV heads, 131072 positions, 64 chunks 98, 80 chunks (a second round) 116, 128 101; 16 ragged sequences of 8 heads up to 32768 positions, chunks of 64 tiles 236, of 128
// 261; 1 head, 100000 positions, 128 chunks 28, 256 26, 512 33.  Up to 4 tiles per wave no chunks at all, as a merge is a launch more: 192
// positions of 32 heads 7.4 us against 8.4 with them, 256 8.4 either way, 320 9.4 against 8.8, 512 12.4 against 8.7.
// Prompts: 8 waves to a workgroup where a row tile walks 2048 positions or more (8 waves / 4: a prompt of 16k tokens 2148 / 2225 us, through a
// window of 4096 1974 / 2014, but ragged ones of up to 3001 tokens through 512 145 / 134, 8 prompts of 1000 tokens
// 106 / 98: first tiles and edges are then most of a walk);
// row tiles that are too few for the chip have their positions split, at least four tiles to a chunk.
constexpr int64_t kStepsAtOnce = 512;
int plan_of(const specache_window_config& c, Plan& p) {
    const int G = c.n_q_heads / c.n_kv_heads;
    const int64_t rows = (int64_t)c.q_tokens * G;
    int64_t most = c.kv_tokens;                     // positions that a row tile walks
    if (window_of(c)) most = std::min<int64_t>(most, (int64_t)c.window + c.sinks + 128);
    const int64_t heads = (int64_t)c.batch * c.n_kv_heads;
    int64_t chunks = 1;
    if (rows <= kWaveRows) {
        p.kernel = kStep;
        p.item_rows = (int)rows;
        p.items = heads * (rows > 0);
        const int64_t tiles = (most + 31) / 32;
        if (p.items && tiles > 4 * kStepWaves) {
            chunks = std::max(kStepsAtOnce / p.items, tiles / 64);
            chunks = std::min({chunks, tiles / kStepWaves, std::max<int64_t>(256, tiles / 64)});
        }
    } else {
        p.kernel = most >= 2048 && rows > 128 ? kTile8 : kTile4;
        p.item_rows = p.kernel == kTile8 ? 256 : 128;
        p.row_tiles = (int)((rows + p.item_rows - 1) / p.item_rows);
        p.items = heads * p.row_tiles;
        if (p.items) chunks = std::min<int64_t>((p.kernel == kTile8 ? 256 : 512) / p.items, (most + 63) / 64 / 4);
    }
    if (p.items * p.item_rows >= (1ll << 32) / (64 * kMergeWaves)) chunks = 1;   // (the merge's threads, counted in 32 bits)
    p.chunks = (int)std::max<int64_t>(chunks, 1);
    if (p.items * p.chunks > INT32_MAX / 256) return fail_without_context(SPECACHE_EINVAL, "too many rows");
    p.scratch = p.chunks > 1 ? p.items * p.chunks * p.item_rows * (kD + 2) * (int64_t)sizeof(float) : 0;
    return SPECACHE_OK;
}

template <bool BF16>
void launch(const Plan& p, const WindowArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)(p.items * p.chunks));
    const bool split = p.chunks > 1;
    if (p.kernel == kStep) hipLaunchKernelGGL((split ? step_kernel<BF16, true, kStepWaves> : step_kernel<BF16, false, kStepWaves>), grid, dim3(64 * kStepWaves), 0, stream, a);
    else if (p.kernel == kTile4) hipLaunchKernelGGL((split ? tile_kernel<BF16, true, 4> : tile_kernel<BF16, false, 4>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((split ? tile_kernel<BF16, true, 8> : tile_kernel<BF16, false, 8>), grid, dim3(512), 0, stream, a);
    if (split && p.chunks <= kFewChunks) hipLaunchKernelGGL((merge_kernel<BF16, 1>), dim3((unsigned)((a.merge_rows + kMergeWaves - 1) / kMergeWaves)), dim3(64 * kMergeWaves), 0, stream, a);
    else if (split) hipLaunchKernelGGL((merge_kernel<BF16, kMergeWaves>), dim3((unsigned)a.merge_rows), dim3(64 * kMergeWaves), 0, stream, a);
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
    a.part_ml = a.part_o + p.items * p.chunks * p.item_rows * kD;
    a.n_kv_heads = cfg->n_kv_heads;
    a.G = cfg->n_q_heads / cfg->n_kv_heads;
    a.q_tokens = cfg->q_tokens;
    a.kv_tokens = cfg->kv_tokens;
    a.window = window_of(*cfg);
    a.sinks = std::min(cfg->sinks, cfg->kv_tokens);
    a.merge_rows = (int)(p.items * p.item_rows);
    a.row_tiles = p.row_tiles;
    a.item_rows = p.item_rows;
    a.chunks = p.chunks;
    a.scale = (cfg->sm_scale > 0.0f ? cfg->sm_scale : 0.08838834764831845f) * kLog2e;
    if (cfg->dtype == SPECACHE_BF16) launch<true>(p, a, (hipStream_t)stream);
    else launch<false>(p, a, (hipStream_t)stream);
    return launched();
}

}  // extern "C"
