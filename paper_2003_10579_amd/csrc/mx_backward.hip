// What lies between the products of a backward pass in few bits: the gradient of a dense layer's or a gated block's activation from its checkpoint, quantised
// along its rows and along its columns; and a checkpoint in few bits quantised again along its columns.
//
//   dp = dy act'(p),   h = act(p)          gated, in pairs of columns g, u:   dg = dy u act'(g),   du = dy act(g),   h = act(g) u
#include "activations.hpp"
#include "column_sums.hpp"

using namespace ssgd;

namespace {

constexpr int kTile = 128, kThreads = 256;

struct Target { uint8_t *values, *scales; int64_t row_bytes, scale_bytes; int32_t fmt; };   // values == nullptr: not wanted
struct Gradient {
    const void *dy, *p;
    const uint8_t *p_values, *p_scales;
    float* partial;                          // sums of dp over the rows of a tile [tiles down][columns], nullptr: not wanted
    int64_t rows, cols, p_cols, dy_pitch, p_pitch, p_bytes, p_scale_bytes, across;
    int32_t p_bf16, activation;
    Target along, columns, hidden;
};

// A wave has 32 rows of the 128 columns of a tile: of every sixteen lanes, four side by side have a block of 32 columns, eight each, and the next four
// the eight rows below.  So a block along a row is four lanes', and one along a column eight registers of the lanes four, eight and twelve further on.
constexpr int kTurn4 = 0x124, kTurn8 = 0x128;
__device__ __forceinline__ uint32_t max_of_turns(uint32_t x) { x = umax(x, dpp<kTurn4>(x)); return umax(x, dpp<kTurn8>(x)); }
__device__ __forceinline__ float sum_of_turns(float x) {
    x += __builtin_bit_cast(float, dpp<kTurn4>(__builtin_bit_cast(uint32_t, x)));
    return x + __builtin_bit_cast(float, dpp<kTurn8>(__builtin_bit_cast(uint32_t, x)));
}
struct Place {
    int64_t row, col;       // the lane's first
    int turn;               // of its rows
    __device__ __forceinline__ Place(int64_t r0, int64_t c0) {
        const int lane = threadIdx.x & 63;
        turn = (lane >> 2) & 3;
        row = r0 + (threadIdx.x >> 6) * 32 + turn * 8;
        col = c0 + (lane >> 4) * 32 + (lane & 3) * 8;
    }
};

// Eight columns of a row of the matrix that is quantised along its rows.
__device__ __forceinline__ void store_along(const Target& t, int64_t row, int64_t col, bool live, const float (&x)[8]) {
    uint32_t most = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) most = umax(most, magnitude(x[q]));
    most = max_of_4(most);
    const uint32_t byte = t.fmt == SSGD_MX_FP4 ? mx_scale_byte<SSGD_MX_FP4>(most) : mx_scale_byte<SSGD_MX_FP8>(most);
    if (!live) return;
    uint8_t* to = t.values + row * t.row_bytes;
    if (t.fmt == SSGD_MX_FP4) *reinterpret_cast<uint32_t*>(to + col / 2) = mx_pack_fp4(x, byte);
    else *reinterpret_cast<words2*>(to + col) = mx_pack_fp8(x, byte);
    if ((threadIdx.x & 3) == 0) t.scales[row * t.scale_bytes + col / kMxBlock] = (uint8_t)byte;
}
// Eight rows of a column as a part of the transposed matrix's row `col`.
__device__ __forceinline__ void store_column(const Target& t, const Place& at, int64_t col, bool live, const float (&x)[8]) {
    uint32_t most = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) most = umax(most, magnitude(x[q]));
    most = max_of_turns(most);
    const uint32_t byte = t.fmt == SSGD_MX_FP4 ? mx_scale_byte<SSGD_MX_FP4>(most) : mx_scale_byte<SSGD_MX_FP8>(most);
    if (!live) return;
    uint8_t* to = t.values + col * t.row_bytes;
    if (t.fmt == SSGD_MX_FP4) *reinterpret_cast<uint32_t*>(to + at.row / 2) = mx_pack_fp4(x, byte);
    else *reinterpret_cast<words2*>(to + at.row) = mx_pack_fp8(x, byte);
    if (at.turn == 0) t.scales[col * t.scale_bytes + at.row / kMxBlock] = (uint8_t)byte;
}

// In place: p becomes dp (gated) or act(p), dy becomes h or dp.
template <int ACT, bool GATED, int W>
__device__ __forceinline__ void differentiate(float (&p)[8][8], float (&dy)[8][W]) {
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int q = 0; q < W; ++q) {
            float y, slope;
            if constexpr (GATED) {
                const float up = p[r][2 * q + 1];
                activation_and_slope(ACT, p[r][2 * q], y, slope);
                p[r][2 * q] = dy[r][q] * up * slope;
                p[r][2 * q + 1] = dy[r][q] * y;
                dy[r][q] = y * up;
            } else {
                activation_and_slope(ACT, p[r][q], y, slope);
                dy[r][q] = ACT == SSGD_ACT_RELU ? (slope > 0.0f ? dy[r][q] : 0.0f) : dy[r][q] * slope;
                p[r][q] = y;
            }
        }
}

template <typename T, bool GATED>
__global__ __launch_bounds__(kThreads) void gradient_kernel(Gradient a) {
    constexpr int W = GATED ? 4 : 8;
    __shared__ float sums[4][kTile];
    const int64_t tile_row = blockIdx.x / a.across, c0 = (blockIdx.x - tile_row * a.across) * kTile;
    const Place at(tile_row * kTile, c0);
    const int64_t own_col = GATED ? at.col / 2 : at.col;
    float p[8][8], dy[8][W];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int64_t row = at.row + r;
        const bool live = row < a.rows;
        load_vec<W>(static_cast<const T*>(a.dy) + row * a.dy_pitch + own_col, live ? a.cols - own_col : 0, dy[r]);
        if (a.p_values != nullptr) {
            words2 w = {0u, 0u};
            uint32_t byte = 0;
            if (live) {
                w = *reinterpret_cast<const words2*>(a.p_values + row * a.p_bytes + at.col);
                byte = a.p_scales[row * a.p_scale_bytes + at.col / kMxBlock];
            }
            mx_unpack_fp8(w, mx_scale_value(byte), p[r]);
            // (a block that is NaN has columns past the last one too)
#pragma unroll
            for (int q = 0; q < 8; ++q) if (at.col + q >= a.p_cols) p[r][q] = 0.0f;
        } else if (a.p == nullptr) {
#pragma unroll
            for (int q = 0; q < 8; ++q) p[r][q] = 0.0f;
        } else if (a.p_bf16) load_vec<8>(static_cast<const bf16_t*>(a.p) + row * a.p_pitch + at.col, live ? a.p_cols - at.col : 0, p[r]);
        else load_vec<8>(static_cast<const float*>(a.p) + row * a.p_pitch + at.col, live ? a.p_cols - at.col : 0, p[r]);
    }
    if (a.activation == SSGD_ACT_RELU) differentiate<SSGD_ACT_RELU, GATED>(p, dy);
    else if (a.activation == SSGD_ACT_GELU) differentiate<SSGD_ACT_GELU, GATED>(p, dy);
    else if (a.activation == SSGD_ACT_SILU) differentiate<SSGD_ACT_SILU, GATED>(p, dy);
    else differentiate<SSGD_ACT_NONE, GATED>(p, dy);
    auto gradient = [&]() -> float (&)[8][8] { if constexpr (GATED) return p; else return dy; };
    auto output = [&]() -> float (&)[8][W] { if constexpr (GATED) return dy; else return p; };
    float (&d)[8][8] = gradient();
    float (&h)[8][W] = output();
    if (a.along.values != nullptr) {
#pragma unroll
        for (int r = 0; r < 8; ++r) store_along(a.along, at.row + r, at.col, at.row + r < a.rows, d[r]);
    }
    if (a.columns.values != nullptr) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float x[8] = {d[0][q], d[1][q], d[2][q], d[3][q], d[4][q], d[5][q], d[6][q], d[7][q]};
            store_column(a.columns, at, at.col + q, at.col + q < a.p_cols, x);
        }
    }
    if (a.hidden.values != nullptr) {
#pragma unroll
        for (int q = 0; q < W; ++q) {
            const float x[8] = {h[0][q], h[1][q], h[2][q], h[3][q], h[4][q], h[5][q], h[6][q], h[7][q]};
            store_column(a.hidden, at, own_col + q, own_col + q < a.cols, x);
        }
    }
    if constexpr (!GATED) {
        if (a.partial == nullptr) return;
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 8; ++r) sum += d[r][q];
            sum = sum_of_turns(sum);
            if (at.turn == 0) sums[threadIdx.x >> 6][(lane >> 4) * 32 + (lane & 3) * 8 + q] = sum;
        }
        __syncthreads();
        const int64_t col = c0 + threadIdx.x;
        if (threadIdx.x < kTile && col < a.cols)
            a.partial[tile_row * a.cols + col] = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
    }
}

template <int FMT>
__global__ __launch_bounds__(kThreads) void transpose_kernel(const uint8_t* values, const uint8_t* scales, int64_t row_bytes, int64_t scale_bytes, int64_t rows, int64_t cols, Target t,
                                                             int64_t across) {
    const int64_t tile_row = blockIdx.x / across;
    const Place at(tile_row * kTile, (blockIdx.x - tile_row * across) * kTile);
    float x[8][8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int64_t row = at.row + r;
        uint32_t byte = 0;
        words2 w = {0u, 0u};
        if (row < rows) {
            byte = scales[row * scale_bytes + at.col / kMxBlock];
            if constexpr (FMT == SSGD_MX_FP8) w = *reinterpret_cast<const words2*>(values + row * row_bytes + at.col);
            else w.x = *reinterpret_cast<const uint32_t*>(values + row * row_bytes + at.col / 2);
        }
        if constexpr (FMT == SSGD_MX_FP8) mx_unpack_fp8(w, mx_scale_value(byte), x[r]);
        else mx_unpack_fp4(w.x, mx_scale_value(byte), x[r]);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const float y[8] = {x[0][q], x[1][q], x[2][q], x[3][q], x[4][q], x[5][q], x[6][q], x[7][q]};
        store_column(t, at, at.col + q, at.col + q < cols, y);
    }
}

bool format_ok(int32_t f) { return f == SSGD_MX_FP4 || f == SSGD_MX_FP8; }
constexpr int64_t kMost = int64_t(1) << 31, kMostSums = int64_t(1) << 25;
bool target_ok(const void* values, const void* scales, int32_t fmt) {
    return (values != nullptr) == (scales != nullptr) && (values == nullptr || (format_ok(fmt) && aligned(values, 16) && aligned(scales, 16)));
}
Target target_of(void* values, void* scales, int32_t fmt, int64_t cols) {
    return {static_cast<uint8_t*>(values), static_cast<uint8_t*>(scales), mx_row_bytes(fmt, cols), mx_padded(cols) / kMxBlock, fmt};
}
int64_t tiles_of(int64_t n) { return (n + kTile - 1) / kTile; }

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int64_t ssgd_mx_activation_backward_work_floats(int64_t rows, int64_t cols) { return rows < 0 || cols < 0 || rows >= kMost || cols >= kMostSums ? -1 : tiles_of(rows) * cols; }

ssgd_status ssgd_mx_activation_backward(const void* dy, int32_t dtype, int64_t dy_pitch, int64_t rows, int64_t cols, int32_t gated, int32_t activation, const void* p, int32_t p_dtype,
                                        int64_t p_pitch, const void* p_values, const void* p_scales, int32_t fmt, void* values, void* scales, int32_t fmt_t, void* values_t,
                                        void* scales_t, int32_t fmt_h, void* values_h, void* scales_h, float* dbias, float* work, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        const char* name = "mx activation backward: ";
        auto no = [&](const char* what) { return op_fail(SSGD_EINVAL, (std::string(name) + what).c_str()); };
        if (!dtype_ok(dtype) || rows < 0 || cols < 0 || rows >= kMost || cols >= kMost / 2) return no("a type of the enumeration, rows from zero to 2^31, columns to 2^30");
        if ((gated != 0 && gated != 1) || activation < SSGD_ACT_NONE || activation > SSGD_ACT_SILU) return no("an activation of the enumeration, gated or not");
        if (gated && dbias != nullptr) return no("a gated block has no bias");
        if (dbias != nullptr && (cols >= kMostSums || !aligned(dbias, 4) || (rows > 0 && cols > 0 && (!work || !aligned(work, 16))))) return no("dbias needs less than 2^25 columns and a 16-byte aligned work area");
        if (!target_ok(values, scales, fmt) || !target_ok(values_t, scales_t, fmt_t) || !target_ok(values_h, scales_h, fmt_h)) return no("outputs are 16-byte aligned arrays of values and scales, formats of the enumeration");
        const int64_t p_cols = gated ? 2 * cols : cols;
        const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        if (cols == 0) return SSGD_OK;
        if (rows > 0) {
            if (!values && !values_t && !values_h && !dbias) return no("no output");
            if (!dy || !aligned(dy, (uintptr_t)dtype_bytes(dtype)) || dy_pitch < cols) return no("dy, pitch >= columns");
            const bool needed = gated || activation != SSGD_ACT_NONE || values_h != nullptr;
            if ((p_values != nullptr) != (p_scales != nullptr) || (p != nullptr && p_values != nullptr) || (needed && !p && !p_values)) return no("p is a matrix, or values and scales");
            if (p != nullptr && (!dtype_ok(p_dtype) || !aligned(p, (uintptr_t)dtype_bytes(p_dtype)) || p_pitch < p_cols)) return no("p, pitch >= its columns");
            if (p_values != nullptr && (!aligned(p_values, 16) || !aligned(p_scales, 16))) return no("values and scales are 16-byte aligned");
            if (tiles_of(rows) > kMostBlocks / tiles_of(p_cols)) return no("too many elements");
            Gradient a{};
            a.dy = dy; a.p = p; a.p_values = static_cast<const uint8_t*>(p_values); a.p_scales = static_cast<const uint8_t*>(p_scales);
            a.rows = rows; a.cols = cols; a.p_cols = p_cols; a.dy_pitch = dy_pitch; a.p_pitch = p_pitch; a.p_bytes = mx_row_bytes(SSGD_MX_FP8, p_cols); a.p_scale_bytes = mx_padded(p_cols) / kMxBlock;
            a.across = tiles_of(p_cols); a.p_bf16 = p_dtype == SSGD_BF16; a.activation = activation;
            a.along = target_of(values, scales, fmt, p_cols); a.columns = target_of(values_t, scales_t, fmt_t, rows); a.hidden = target_of(values_h, scales_h, fmt_h, rows);
            a.partial = dbias != nullptr ? work : nullptr;
            const dim3 grid((unsigned)(tiles_of(rows) * a.across));
#define SSGD_GRADIENT(T, G) hipLaunchKernelGGL((gradient_kernel<T, G>), grid, dim3(kThreads), 0, stream, a)
            if (dtype == SSGD_F32) { if (gated) SSGD_GRADIENT(float, true); else SSGD_GRADIENT(float, false); }
            else { if (gated) SSGD_GRADIENT(bf16_t, true); else SSGD_GRADIENT(bf16_t, false); }
#undef SSGD_GRADIENT
        }
        if (dbias != nullptr) launch_column_sums(work, tiles_of(rows), cols, dbias, stream);
        return op_hip(hipGetLastError(), "mx activation backward");
    });
}

ssgd_status ssgd_mx_transpose(const void* values, const void* scales, int32_t fmt, int64_t rows, int64_t cols, int32_t fmt_t, void* values_t, void* scales_t, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        if (!format_ok(fmt) || !format_ok(fmt_t) || rows < 0 || cols < 0 || rows >= kMost || cols >= kMost) return op_fail(SSGD_EINVAL, "mx transpose: formats of the enumeration, rows and columns from zero to 2^31");
        if (rows == 0 || cols == 0) return SSGD_OK;
        if (!values || !scales || !values_t || !scales_t || !aligned(values, 16) || !aligned(scales, 16) || !aligned(values_t, 16) || !aligned(scales_t, 16))
            return op_fail(SSGD_EINVAL, "mx transpose: values and scales are 16-byte aligned arrays");
        const int64_t across = tiles_of(cols);
        if (tiles_of(rows) > kMostBlocks / across) return op_fail(SSGD_EINVAL, "mx transpose: too many elements");
        const Target t = target_of(values_t, scales_t, fmt_t, rows);
        const dim3 grid((unsigned)(tiles_of(rows) * across));
        const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
#define SSGD_TRANSPOSE(F) hipLaunchKernelGGL((transpose_kernel<F>), grid, dim3(kThreads), 0, stream, static_cast<const uint8_t*>(values), static_cast<const uint8_t*>(scales), \
                                             mx_row_bytes(fmt, cols), mx_padded(cols) / kMxBlock, rows, cols, t, across)
        if (fmt == SSGD_MX_FP4) SSGD_TRANSPOSE(SSGD_MX_FP4); else SSGD_TRANSPOSE(SSGD_MX_FP8);
#undef SSGD_TRANSPOSE
        return op_hip(hipGetLastError(), "mx transpose");
    });
}

}  // extern "C"
#pragma GCC visibility pop
