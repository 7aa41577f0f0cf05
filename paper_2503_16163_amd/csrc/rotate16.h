// What the kernels that turn 16-bit rows by their rotary positions share: 8 channels to a 16-byte access.
#pragma once
#include "operators.h"

namespace specache {
namespace {

constexpr int kParts = 8;               // a row is 8 lanes' work: 8 pairs of channels each, two 16-byte accesses
constexpr int64_t kCached = 32 << 20;   // bytes that the L2s of the 8 XCDs hold

typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
template <bool STREAM>
__device__ __forceinline__ void store16(uint16_t* to, const uint4& v) {
    if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(uint4v, v), (uint4v*)to);
    else *(uint4v*)to = __builtin_bit_cast(uint4v, v);
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

// The channels of a lane's two accesses.  Halves: pair e of this part joins element e of both accesses.  Neighbours: pairs 0 to 3 are the first access's, 4 to 7 the
// second's.  Channels that stay are dealt like the others, so that an access of neighbouring lanes is in few pieces.
template <bool HALF>
struct RowParts {
    bool turns[2];
    int c0, c1;
    __device__ __forceinline__ RowParts(int part, int d)
        : turns{(HALF ? 16 : 8) * part < d, HALF ? 16 * part < d : 8 * part + kD / 2 < d},
          c0(HALF && !turns[0] ? d / 2 + 8 * part : 8 * part),
          c1(c0 + (!HALF ? kD / 2 : turns[0] ? d / 2 : (kD - d) / 2)) {}
};

// A lane's 8 angles at a position, and two accesses turned by them.
template <bool BF16, bool HALF>
struct Turn {
    float cosine[8], sine[8];
    __device__ __forceinline__ void set(const specache_rotary& plan, int part, int64_t p) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int pair = HALF ? 8 * part + e : 4 * part + e % 4 + e / 4 * (kD / 4);
            const uint64_t angle = (uint64_t)p * plan.turns[pair];   // (0 for pairs that there are not)
            const float x = (float)(int32_t)(angle >> 32) * 0x1p-32f;
            cosine[e] = __builtin_amdgcn_cosf(x) * plan.gain;
            sine[e] = __builtin_amdgcn_sinf(x) * plan.gain;
        }
    }
    __device__ __forceinline__ void apply(uint4& u0, uint4& u1, bool second) const {
        float x[2][8], y[2][8];
        unpack8<BF16>(u0, x[0]);
        unpack8<BF16>(u1, x[1]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int r0 = HALF ? 0 : e / 4, e0 = HALF ? e : 2 * (e % 4), r1 = HALF ? 1 : r0, e1 = HALF ? e : e0 + 1;
            const float p = x[r0][e0], q = x[r1][e1];
            y[r0][e0] = fmaf(p, cosine[e], -(q * sine[e]));
            y[r1][e1] = fmaf(q, cosine[e], p * sine[e]);
        }
        u0 = pack8<BF16>(y[0]);
        if (second) u1 = pack8<BF16>(y[1]);
    }
};

// Where a head's halves of less than all of it are turned, either of a lane's accesses shares its lines with the other.  This deals the 8 lanes' channels of ROWS rows
// anew, 8 part and 64 + 8 part on, so that a row is two whole lines: of the 16 pieces of 8 channels lane p has p and p + e where it turns them (p < e = d / 16),
// else p + e and p + 8.
template <int E>
__device__ __forceinline__ void deal_piece(uint32_t& u0, uint32_t& u1, int part) {
    const uint32_t gone = part < E ? u1 : u0;
    const uint32_t lower = __builtin_amdgcn_update_dpp(0, gone, 0x110 + E, 0xF, 0xF, false);       // of lane - E, in a row of 16
    const uint32_t upper = __builtin_amdgcn_update_dpp(0, gone, 0x100 + 8 - E, 0xF, 0xF, false);   // of lane + 8 - E
    if (part < E) u1 = upper;
    else u0 = lower;
}
template <int E, int ROWS>
__device__ __forceinline__ void deal_rows(uint4 (&u)[ROWS][2], int part) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        deal_piece<E>(u[i][0].x, u[i][1].x, part);
        deal_piece<E>(u[i][0].y, u[i][1].y, part);
        deal_piece<E>(u[i][0].z, u[i][1].z, part);
        deal_piece<E>(u[i][0].w, u[i][1].w, part);
    }
}
template <int ROWS>
__device__ __forceinline__ void deal_lines(uint4 (&u)[ROWS][2], int part, int d) {
    switch (d / 16) {
        case 1: return deal_rows<1>(u, part);
        case 2: return deal_rows<2>(u, part);
        case 3: return deal_rows<3>(u, part);
        case 4: return deal_rows<4>(u, part);
        case 5: return deal_rows<5>(u, part);
        case 6: return deal_rows<6>(u, part);
        case 7: return deal_rows<7>(u, part);
    }
}

inline bool in_place_or_apart(const specache_view& in, const specache_view& out) { return in.data != out.data || same_view(in, out); }

inline bool is_plan(const specache_rotary& p) {
    return p.rotary_dim >= 16 && p.rotary_dim <= kD && p.rotary_dim % 16 == 0 && (p.layout == SPECACHE_ROTARY_HALF || p.layout == SPECACHE_ROTARY_INTERLEAVED);
}

}  // namespace
}  // namespace specache
