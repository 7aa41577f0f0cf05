// What the kernels of 16-bit attention share: a wave's 32 query rows and their softmax over tiles of keys and values in LDS.
#pragma once
#include <cfloat>
#include <cmath>

#include "operators.h"

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

// Of `total` workgroups, `per_head` that read the same keys and values (a KV head of a sequence) follow each other on one XCD (workgroups go to the 8 XCDs in
// turn), whose L2 they share.  Heads are dealt to the XCDs in turn, so that a long sequence of a batch is everybody's (5 prompts of up to 3001 tokens, in
// stretches of heads 194 us, so 141); of the last ones, fewer than 8, each XCD has a stretch.
__device__ __forceinline__ int on_one_xcd(int index, int total, int per_head) {
    const int xcd = index % 8, dealt = total / per_head / 8 * 8 * per_head;
    if (index < dealt) {
        const int at = index / 8;
        return (at / per_head * 8 + xcd) * per_head + at % per_head;
    }
    const int left = total - dealt, per_xcd = left / 8, rest = left % 8;
    return dealt + xcd * per_xcd + min(xcd, rest) + (index - dealt) / 8;
}

}  // namespace
}  // namespace specache
