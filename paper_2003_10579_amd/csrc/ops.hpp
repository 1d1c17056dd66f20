// Shared by the operators of a low-precision training step (adamw.hip, rmsnorm.hip, mx_quantize.hip, mx_matmul.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <exception>
#include <new>
#include <string>

#include "../../include/ssgd.h"
#include "common.hpp"

namespace ssgd {

// ---- host ------------------------------------------------------------------------------------------------------------
inline ssgd_status op_fail(ssgd_status st, const char* what) {
    try { set_global_error(what); } catch (...) {}
    return st;
}
inline ssgd_status op_hip(hipError_t e, const char* what) {
    if (e == hipSuccess) return SSGD_OK;
    try { set_global_error(std::string(what) + ": " + hipGetErrorString(e)); } catch (...) {}
    return e == hipErrorOutOfMemory ? SSGD_ENOMEM : SSGD_EDEVICE;
}
// Nothing throws across the ABI.
template <typename F>
ssgd_status op_entry(F&& body) {
    try { return body(); }
    catch (const std::bad_alloc&) { return op_fail(SSGD_ENOMEM, "out of host memory"); }
    catch (...) { return op_fail(SSGD_EDEVICE, "unexpected error"); }
}
inline bool dtype_ok(int32_t t) { return t == SSGD_F32 || t == SSGD_BF16; }
inline int64_t dtype_bytes(int32_t t) { return t == SSGD_F32 ? 4 : 2; }
inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

constexpr int64_t kMostBlocks = (int64_t(1) << 23) - 1;      // workgroups of up to 512: a launch ends at 2^32 threads

constexpr int kMxBlock = 32;      // columns per scale
constexpr int kMxPad = 128;       // rows of a quantised matrix are padded to so many columns: what one matrix instruction contracts
constexpr int64_t mx_padded(int64_t cols) { return (cols + kMxPad - 1) / kMxPad * kMxPad; }
constexpr int64_t mx_row_bytes(int fmt, int64_t cols) { return fmt == SSGD_MX_FP4 ? mx_padded(cols) / 2 : mx_padded(cols); }

// ---- device ----------------------------------------------------------------------------------------------------------
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t words2 __attribute__((ext_vector_type(2)));
typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef uint16_t bf16_t;          // bits of a bfloat16

__device__ __forceinline__ float bf16_to_f32(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }
// Nearest even; NaN stays NaN (one instruction for two values).
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ uint32_t f32_to_bf16(float x) { return pack_bf16(x, 0.0f) & 0xFFFFu; }

// V consecutive values (4 or 8) at p; `left` of them exist, the rest are zero.  Global loads and stores of 16 bytes need no more alignment
// than the element's (the types say so, and the compiler then splits nothing), so rows at odd places take the same path.
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef words4 words4_any __attribute__((aligned(2)));
typedef words2 words2_any __attribute__((aligned(2)));
template <int V>
__device__ __forceinline__ void load_vec(const float* p, int64_t left, float (&x)[V]) {
    if (left >= V) {
#pragma unroll
        for (int q = 0; q < V; q += 4) {
            const f32x4 v = *reinterpret_cast<const f32x4_any*>(p + q);
            x[q] = v.x; x[q + 1] = v.y; x[q + 2] = v.z; x[q + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int q = 0; q < V; ++q) x[q] = q < left ? p[q] : 0.0f;
    }
}
template <int V>
__device__ __forceinline__ void load_vec(const bf16_t* p, int64_t left, float (&x)[V]) {
    if (left >= V) {
        uint32_t w[V / 2];
        if constexpr (V == 8) {
            const words4 v = *reinterpret_cast<const words4_any*>(p);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            const words2 v = *reinterpret_cast<const words2_any*>(p);
            w[0] = v.x; w[1] = v.y;
        }
#pragma unroll
        for (int q = 0; q < V / 2; ++q) { x[2 * q] = bf16_to_f32(w[q] & 0xFFFFu); x[2 * q + 1] = __builtin_bit_cast(float, w[q] & 0xFFFF0000u); }
    } else {
#pragma unroll
        for (int q = 0; q < V; ++q) x[q] = q < left ? bf16_to_f32(p[q]) : 0.0f;
    }
}
template <int V>
__device__ __forceinline__ void store_vec(float* p, int64_t left, const float (&x)[V]) {
    if (left >= V) {
#pragma unroll
        for (int q = 0; q < V; q += 4) *reinterpret_cast<f32x4_any*>(p + q) = f32x4{x[q], x[q + 1], x[q + 2], x[q + 3]};
    } else {
#pragma unroll
        for (int q = 0; q < V; ++q) if (q < left) p[q] = x[q];
    }
}
template <int V>
__device__ __forceinline__ void store_vec(bf16_t* p, int64_t left, const float (&x)[V]) {
    if (left >= V) {
        if constexpr (V == 8) *reinterpret_cast<words4_any*>(p) = words4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
        else *reinterpret_cast<words2_any*>(p) = words2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    } else {
#pragma unroll
        for (int q = 0; q < V; ++q) if (q < left) p[q] = (bf16_t)f32_to_bf16(x[q]);
    }
}

// Moves within rows of 16 lanes, without LDS.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true); }
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
// Largest of 4 and of 16 adjacent lanes.  On the bits of magnitudes: infinities and NaN are the largest, so they carry.
__device__ __forceinline__ uint32_t max_of_4(uint32_t x) { x = umax(x, dpp<kXor1>(x)); return umax(x, dpp<kXor2>(x)); }
__device__ __forceinline__ uint32_t max_of_16(uint32_t x) {
    x = max_of_4(x);
    x = umax(x, dpp<kHalfMirror>(x));
    return umax(x, dpp<kMirror>(x));
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu; }

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) x += __shfl_xor(x, m);
    return x;
}
__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) x += __shfl_xor(x, m);
    return x;
}

// ---- microscaled formats ---------------------------------------------------------------------------------------------
// A block of 32 values shares the scale 2^(byte - 127), the exponent of its largest magnitude less that of the format's largest
// value (E2M1: 6 = 1.5 x 2^2, E4M3: 448 = 1.75 x 2^8), so that the largest value lands in the top binade and saturates in its
// upper part.  Byte 255 stands for NaN: a block with an infinity or a NaN has no scale.
template <int FMT>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t largest) {
    const uint32_t e = largest >> 23, top = FMT == SSGD_MX_FP4 ? 2u : 8u;
    return e == 255u ? 255u : (e > top ? e - top : 0u);
}
// Eight values at a scale -> 4 (E2M1, low nibble first) or 8 bytes, nearest, ties to even, saturating.  The conversions divide by a scale
// themselves, whose exponent field is the byte; past E4M3's largest value they give NaN, so those values are cut off before: at 448 times the
// scale, 1.75 x 2^(byte + 8 - 127), which bfloat16 holds as well.  (The byte is 246 at most in 8 bits, and 252 in 4.)
typedef short shorts2 __attribute__((ext_vector_type(2)));
typedef uint16_t half2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float mx_scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }
__device__ __forceinline__ uint32_t mx_limit(uint32_t byte) { return ((byte + 8u) << 23) | 0x600000u; }
__device__ __forceinline__ uint32_t mx_pack_fp4(const float (&x)[8], uint32_t byte) {
    const float s = mx_scale_of(byte);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
    return byte == 255u ? 0u : r;
}
__device__ __forceinline__ words2 mx_pack_fp8(const float (&x)[8], uint32_t byte) {
    const float s = mx_scale_of(byte), most = __builtin_bit_cast(float, mx_limit(byte));
    float y[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) y[q] = __builtin_amdgcn_fmed3f(x[q], -most, most);
    shorts2 lo = {0, 0}, hi = {0, 0};
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, y[0], y[1], s, false); lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, y[2], y[3], s, true);
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, y[4], y[5], s, false); hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, y[6], y[7], s, true);
    return byte == 255u ? words2{0u, 0u} : words2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}
// The same from eight bfloat16, two to a word, as they are.
// (A bit cast of a vector's element reads its first one: copies are taken.)
__device__ __forceinline__ bf16x2 as_pair(uint32_t w) { return __builtin_bit_cast(bf16x2, w); }
__device__ __forceinline__ half2 as_halves(uint32_t w) { return __builtin_bit_cast(half2, w); }
__device__ __forceinline__ uint32_t mx_pack_fp4(const words4& w, uint32_t byte) {
    const float s = mx_scale_of(byte);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, as_pair(w.x), s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, as_pair(w.y), s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, as_pair(w.z), s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, as_pair(w.w), s, 3);
    return byte == 255u ? 0u : r;
}
__device__ __forceinline__ bf16x2 cut_off(uint32_t w, uint32_t limit) {       // magnitudes as whole numbers
    const half2 m = __builtin_elementwise_min(as_halves(w & 0x7FFF7FFFu), as_halves(limit));
    return __builtin_bit_cast(bf16x2, __builtin_bit_cast(uint32_t, m) | (w & 0x80008000u));
}
__device__ __forceinline__ words2 mx_pack_fp8(const words4& w, uint32_t byte) {
    const float s = mx_scale_of(byte);
    const uint32_t half = mx_limit(byte) >> 16, limit = half | half << 16;
    shorts2 lo = {0, 0}, hi = {0, 0};
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, cut_off(w.x, limit), s, false); lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, cut_off(w.y, limit), s, true);
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, cut_off(w.z, limit), s, false); hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, cut_off(w.w, limit), s, true);
    return byte == 255u ? words2{0u, 0u} : words2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// Eight columns of a row, in their own type: what quantisation and the norm take.  `load` reads the row's last eight where fewer are left, so it
// has no branch and nothing waits between the loads of several places; `settle`, when they have arrived, moves them to the front and puts zeros
// behind the row's end.  (In fp32 the loads at a row's end do not wait for each other by themselves.)  Rows of less than eight columns: `load_few`.
// `load_own` reads no other columns than the eight, and settles itself; AT_ONCE: loads past the end read the last column, since one that is left
// out would wait for those before.  `largest`: the largest magnitude as the bits of an fp32 number.
template <typename T> struct Eight;
template <> struct Eight<float> {
    float x[8];
    __device__ __forceinline__ void load(const float* row, int64_t col, int64_t cols) { load_vec<8>(row + col, cols - col, x); }
    __device__ __forceinline__ void load_few(const float* row, int64_t col, int64_t cols) { load(row, col, cols); }
    template <bool> __device__ __forceinline__ void load_own(const float* row, int64_t col, int64_t cols) { load(row, col, cols); }
    __device__ __forceinline__ void settle(int64_t, int64_t) {}
    __device__ __forceinline__ uint32_t largest() const {
        uint32_t most = 0;
#pragma unroll
        for (int q = 0; q < 8; ++q) most = umax(most, magnitude(x[q]));
        return most;
    }
    __device__ __forceinline__ const float (&values() const)[8] { return x; }
    __device__ __forceinline__ void numbers(float (&y)[8]) const {
#pragma unroll
        for (int q = 0; q < 8; ++q) y[q] = x[q];
    }
};
template <> struct Eight<bf16_t> {
    words4 w;
    __device__ __forceinline__ void load(const bf16_t* row, int64_t col, int64_t cols) {
        w = *reinterpret_cast<const words4_any*>(row + (col < cols - 8 ? col : cols - 8));
    }
    __device__ __forceinline__ void load_few(const bf16_t* row, int64_t col, int64_t cols) {
        uint32_t v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = (col + 2 * q < cols ? row[col + 2 * q] : 0u) | (col + 2 * q + 1 < cols ? (uint32_t)row[col + 2 * q + 1] << 16 : 0u);
        w = words4{v[0], v[1], v[2], v[3]};
    }
    template <bool AT_ONCE> __device__ __forceinline__ void load_own(const bf16_t* row, int64_t col, int64_t cols) {
        const int64_t left = cols - col;
        if (left >= 8) { w = *reinterpret_cast<const words4_any*>(row + col); return; }
        if constexpr (!AT_ONCE) { load_few(row, col, cols); return; }
        w = words4{0u, 0u, 0u, 0u};
        if (left <= 0) return;
        uint32_t v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = row[q < left ? col + q : cols - 1];
#pragma unroll
        for (int q = 1; q < 8; ++q) if (q >= left) v[q] = 0u;
        w = words4{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16};
    }
    __device__ __forceinline__ void settle(int64_t col, int64_t cols) {
        if (col + 8 <= cols) return;
        const int gone = col < cols ? (int)(col + 8 - cols) : 8;
        if (gone & 4) w = words4{w.z, w.w, 0u, 0u};
        if (gone & 2) w = words4{w.y, w.z, w.w, 0u};
        if (gone & 1) w = words4{w.x >> 16 | w.y << 16, w.y >> 16 | w.z << 16, w.z >> 16 | w.w << 16, w.w >> 16};
        if (gone == 8) w = words4{0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ uint32_t largest() const {
        constexpr uint32_t kMagnitudes = 0x7FFF7FFFu;
        const half2 a = __builtin_elementwise_max(as_halves(w.x & kMagnitudes), as_halves(w.y & kMagnitudes));
        const half2 b = __builtin_elementwise_max(as_halves(w.z & kMagnitudes), as_halves(w.w & kMagnitudes));
        const half2 m = __builtin_elementwise_max(a, b);
        return (uint32_t)(m.x > m.y ? m.x : m.y) << 16;
    }
    __device__ __forceinline__ const words4& values() const { return w; }
    __device__ __forceinline__ void numbers(float (&y)[8]) const {
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) { y[2 * q] = bf16_to_f32(v[q] & 0xFFFFu); y[2 * q + 1] = __builtin_bit_cast(float, v[q] & 0xFFFF0000u); }
    }
};

}  // namespace ssgd
