// What the calls without a context share: their errors, the checks of views, 16-bit packing.
#pragma once
#include "../../include/specache.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "layout.h"

namespace specache {

// The calling thread's message for specache_last_error(NULL); returns code.
int fail_without_context(int code, const char* msg) noexcept;

// What the launches of a call left behind.
inline int launched() noexcept {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return SPECACHE_OK;
    return fail_without_context(SPECACHE_EHIP, hipGetErrorString(e));
}

// 16-byte loads of 8 channels: the address and every stride keep to them.
inline bool view_fits(const specache_view& v) {
    return v.data && (uintptr_t)v.data % 16 == 0 && v.batch >= 0 && v.head >= 0 && v.token >= 0 && v.batch % 8 == 0 && v.head % 8 == 0 &&
           v.token % 8 == 0;
}
// an output's rows are places of their own
inline bool rows_apart(const specache_view& v, int64_t batch, int64_t heads, int64_t tokens) {
    return (batch <= 1 || v.batch) && (heads <= 1 || v.head) && (tokens <= 1 || v.token);
}
inline bool same_view(const specache_view& a, const specache_view& b) {
    return a.batch == b.batch && a.head == b.head && a.token == b.token;
}

#if defined(__HIPCC__)
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bfloat2v __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));

// a sequence's length, held to 0 .. most (NULL: most)
__device__ __forceinline__ int length_of(const int32_t* lengths, int b, int most) { return lengths ? min(max(lengths[b], 0), most) : most; }

// two binary32 numbers as two 16-bit ones, each rounded to the nearest (even)
template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    const float2v f = {lo, hi};
    if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bfloat2v));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, half2v));
}
#endif

}  // namespace specache
