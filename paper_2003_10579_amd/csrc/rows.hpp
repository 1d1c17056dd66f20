// Rows of a norm and their weights, eight columns to a thread.
#pragma once
#include "ops.hpp"

namespace ssgd {

__device__ __forceinline__ void load_weight(const void* w, int bf16, int64_t at, int64_t left, float (&x)[8]) {
    if (bf16) load_vec<8>(static_cast<const bf16_t*>(w) + at, left, x);
    else load_vec<8>(static_cast<const float*>(w) + at, left, x);
}

__device__ __forceinline__ float as_stored(const float*, float x) { return x; }
__device__ __forceinline__ float as_stored(const bf16_t*, float x) { return bf16_to_f32(f32_to_bf16(x)); }
// Numbers in fp64 on their way to bfloat16 through fp32.  Where `near`, the fp32 number, is the middle of two neighbours in bfloat16 and not the number itself, the fp32 number beside the
// middle on its side goes on instead; in all other places both roundings together are the one.  `is_middle` is zero at a middle: its last 16 bits are 0x8000 (an infinity's and NaN's are not).
__device__ __forceinline__ uint32_t is_middle(float near) { return (__builtin_bit_cast(uint32_t, near) << 16) + 0x80000000u; }
__device__ __forceinline__ float beside_middle(float near, double x) {
    uint32_t w = __builtin_bit_cast(uint32_t, near);
    if (is_middle(near) == 0u && (double)near != x) w += __builtin_fabs(x) > __builtin_fabs((double)near) ? 1u : ~0u;
    return __builtin_bit_cast(float, w);
}

// Eight columns of a row up to `end`, read and, when they have arrived, as numbers; SHORT: rows of less than eight columns are among them.
template <bool SHORT, typename T>
__device__ __forceinline__ void read(Eight<T>& to, const void* rows, int64_t row, int64_t pitch, int col, int end, int d) {
    const T* from = static_cast<const T*>(rows) + row * pitch;
    if (!SHORT || d >= 8) to.load(from, col, end);
    else to.load_few(from, col, end);
}
template <bool SHORT, typename T>
__device__ __forceinline__ void numbers(Eight<T>& x, int col, int end, int d, float (&to)[8]) {
    if (!SHORT || d >= 8) x.settle(col, end);
    x.numbers(to);
}

}  // namespace ssgd
