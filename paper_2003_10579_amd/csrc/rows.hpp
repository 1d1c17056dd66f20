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
