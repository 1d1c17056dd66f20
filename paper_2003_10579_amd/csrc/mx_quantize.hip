// Microscaled quantisation along the rows, along the columns (the transposed matrix), or both from one read, and back.
//
// A value is read once and half a byte or one (and 1/32 of one for the scale) is written per direction: bound by memory.
// Along the rows a lane holds eight columns and four lanes a block, whose largest magnitude takes two lane moves.  For the
// columns a workgroup of 512 holds 128 x 128 values in LDS, in their own type, and a lane takes the 32 rows of one block, so the maximum
// needs no other lane; four lanes side by side take the four blocks of a column, whose bytes are then 64 (4 bits) or 128 next to each
// other.
#include "ops.hpp"

using namespace ssgd;

namespace {

constexpr int kTile = 128;
constexpr int kThreads = 256, kTileThreads = 512;

struct Source { const void* x; int64_t rows, cols, pitch; };
struct Target { uint8_t *values, *scales; int64_t row_bytes, scale_bytes; };   // values == nullptr: not wanted

// Eight columns of a row (zeros where there are none) -> values and, from the first of four lanes, the scale.
template <int FMT, typename T>
__device__ __forceinline__ void store_block(const Target& t, int64_t row, int64_t col, const Eight<T>& x) {
    const uint32_t byte = mx_scale_byte<FMT>(max_of_4(x.largest()));
    uint8_t* to = t.values + row * t.row_bytes;
    if constexpr (FMT == SSGD_MX_FP4) *reinterpret_cast<uint32_t*>(to + col / 2) = mx_pack_fp4(x.values(), byte);
    else *reinterpret_cast<words2*>(to + col) = mx_pack_fp8(x.values(), byte);
    if ((threadIdx.x & 3) == 0) t.scales[row * t.scale_bytes + col / kMxBlock] = (uint8_t)byte;
}

// Rows alone: a thread per eight columns of the padded matrix (8192 x 8192 bf16 to 4 bits: 36 us, 4.7 TB/s).
template <typename T, int FMT>
__global__ __launch_bounds__(kThreads) void rows_kernel(Source s, Target t, int64_t groups, int64_t groups_per_row) {
    const int64_t g = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (g >= groups) return;                 // (groups is a multiple of 16: whole blocks)
    const int64_t row = g / groups_per_row, col = (g - row * groups_per_row) * 8;
    Eight<T> x;
    const T* from = static_cast<const T*>(s.x) + row * s.pitch;
    if (s.cols >= 8) { x.load(from, col, s.cols); x.settle(col, s.cols); }
    else x.load_few(from, col, s.cols);
    store_block<FMT>(t, row, col, x);
}

// A tile of 128 x 128 (8192 x 6144 fp32 to 4 bits both ways: 60 us, 4.2 TB/s; 4001 x 2100 bf16 to 8 bits: 12.7 us, 2.7 TB/s, two tiles to a CU).  The
// rows of a column's block begin 16 columns further on than those of the block before, so that four lanes on
// one column and sixteen on the next ones meet in no bank.
__device__ __forceinline__ int place(int row, int col) { return row * kTile + (row >> 5) * 16 + col; }
__device__ __forceinline__ void put(float* t, const Eight<float>& x) {
    *reinterpret_cast<f32x4*>(t) = f32x4{x.x[0], x.x[1], x.x[2], x.x[3]};
    *reinterpret_cast<f32x4*>(t + 4) = f32x4{x.x[4], x.x[5], x.x[6], x.x[7]};
}
__device__ __forceinline__ void put(bf16_t* t, const Eight<bf16_t>& x) { *reinterpret_cast<words4*>(t) = x.w; }
// Eight rows of a column.
__device__ __forceinline__ void take(const float* t, Eight<float>& x) {
#pragma unroll
    for (int q = 0; q < 8; ++q) x.x[q] = t[q * kTile];
}
__device__ __forceinline__ void take(const bf16_t* t, Eight<bf16_t>& x) {
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = t[2 * q * kTile] | (uint32_t)t[(2 * q + 1) * kTile] << 16;
    x.w = words4{w[0], w[1], w[2], w[3]};
}

template <typename T, int ROWS, int COLS>       // formats; ROWS < 0: columns alone
__global__ __launch_bounds__(kTileThreads) void tile_kernel(Source s, Target t, Target tt, int64_t tiles_across) {
    __shared__ __attribute__((aligned(16))) T tile[kTile * kTile + 3 * 16];
    const int64_t r0 = (int64_t)(blockIdx.x / tiles_across) * kTile, c0 = (int64_t)(blockIdx.x % tiles_across) * kTile;
    const int lane_col = (threadIdx.x & 15) * 8;
    Eight<T> x[kTile / 32];
#pragma unroll
    for (int q = 0; q < kTile / 32; ++q) {
        const int64_t row = r0 + q * 32 + (threadIdx.x >> 4);
        if constexpr (sizeof(T) == 4) {
            load_vec<8>(static_cast<const T*>(s.x) + row * s.pitch + c0 + lane_col, row < s.rows ? s.cols - c0 - lane_col : 0, x[q].x);
        } else {
            const T* from = static_cast<const T*>(s.x) + (row < s.rows ? row : s.rows - 1) * s.pitch;
            const int64_t col = row < s.rows ? c0 + lane_col : s.cols;       // (past the last row: zeros)
            if (s.cols >= 8) x[q].load(from, col, s.cols);
            else x[q].load_few(from, col, s.cols);
        }
    }
#pragma unroll
    for (int q = 0; q < kTile / 32; ++q) {
        const int r = q * 32 + (threadIdx.x >> 4);
        if (sizeof(T) == 2 && s.cols >= 8) x[q].settle(r0 + r < s.rows ? c0 + lane_col : s.cols, s.cols);
        put(&tile[place(r, lane_col)], x[q]);
        if constexpr (ROWS >= 0) { if (r0 + r < s.rows) store_block<ROWS>(t, r0 + r, c0 + lane_col, x[q]); }
    }
    __syncthreads();
    const int block = threadIdx.x & 3, c = threadIdx.x >> 2;
    const int64_t col = c0 + c;
    if (col >= s.cols) return;
    uint32_t most = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) { take(&tile[place(block * 32 + q * 8, c)], x[q]); most = umax(most, x[q].largest()); }
    const uint32_t byte = mx_scale_byte<COLS>(most);
    uint8_t* to = tt.values + col * tt.row_bytes + (r0 + block * 32) * (COLS == SSGD_MX_FP4 ? 1 : 2) / 2;
    if constexpr (COLS == SSGD_MX_FP4) {
        *reinterpret_cast<words4*>(to) = words4{mx_pack_fp4(x[0].values(), byte), mx_pack_fp4(x[1].values(), byte), mx_pack_fp4(x[2].values(), byte), mx_pack_fp4(x[3].values(), byte)};
    } else {
        const words2 a = mx_pack_fp8(x[0].values(), byte), b = mx_pack_fp8(x[1].values(), byte), d = mx_pack_fp8(x[2].values(), byte), e = mx_pack_fp8(x[3].values(), byte);
        *reinterpret_cast<words4*>(to) = words4{a.x, a.y, b.x, b.y};
        *reinterpret_cast<words4*>(to + 16) = words4{d.x, d.y, e.x, e.y};
    }
    tt.scales[col * tt.scale_bytes + r0 / kMxBlock + block] = (uint8_t)byte;
}

// Eight columns of a row from their values and scale (8192 x 6144, 4 bits to bf16: 24 us, 5.3 TB/s).
template <int FMT, typename T>
__global__ __launch_bounds__(kThreads) void back_kernel(const uint8_t* values, const uint8_t* scales, int64_t row_bytes, int64_t scale_bytes, T* out,
                                                        int64_t cols, int64_t pitch, int64_t groups, int64_t groups_per_row) {
    const int64_t g = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (g >= groups) return;
    const int64_t row = g / groups_per_row, col = (g - row * groups_per_row) * 8;
    const uint32_t byte = scales[row * scale_bytes + col / kMxBlock];
    const float scale = mx_scale_value(byte);
    float x[8];
    if constexpr (FMT == SSGD_MX_FP4) mx_unpack_fp4(*reinterpret_cast<const uint32_t*>(values + row * row_bytes + col / 2), scale, x);
    else mx_unpack_fp8(*reinterpret_cast<const words2*>(values + row * row_bytes + col), scale, x);
    store_vec<8>(out + row * pitch + col, cols - col, x);
}

bool format_ok(int32_t f) { return f == SSGD_MX_FP4 || f == SSGD_MX_FP8; }
constexpr int64_t kMostRows = int64_t(1) << 40, kMostCols = int64_t(1) << 31;

template <typename T>
void launch_rows(const Source& s, const Target& t, int fmt, hipStream_t stream) {
    const int64_t per_row = mx_padded(s.cols) / 8, groups = s.rows * per_row;
    const dim3 grid((unsigned)((groups + kThreads - 1) / kThreads));
    if (fmt == SSGD_MX_FP4) hipLaunchKernelGGL((rows_kernel<T, SSGD_MX_FP4>), grid, dim3(kThreads), 0, stream, s, t, groups, per_row);
    else hipLaunchKernelGGL((rows_kernel<T, SSGD_MX_FP8>), grid, dim3(kThreads), 0, stream, s, t, groups, per_row);
}

template <typename T>
void launch_tiles(const Source& s, const Target& t, int fmt, const Target& tt, int tfmt, hipStream_t stream) {
    const int64_t across = mx_padded(s.cols) / kTile, tiles = across * (mx_padded(s.rows) / kTile);
    const dim3 grid((unsigned)tiles);
#define SSGD_TILES(R, C) hipLaunchKernelGGL((tile_kernel<T, R, C>), grid, dim3(kTileThreads), 0, stream, s, t, tt, across)
    if (!t.values) { if (tfmt == SSGD_MX_FP4) SSGD_TILES(-1, SSGD_MX_FP4); else SSGD_TILES(-1, SSGD_MX_FP8); }
    else if (fmt == SSGD_MX_FP4) { if (tfmt == SSGD_MX_FP4) SSGD_TILES(SSGD_MX_FP4, SSGD_MX_FP4); else SSGD_TILES(SSGD_MX_FP4, SSGD_MX_FP8); }
    else { if (tfmt == SSGD_MX_FP4) SSGD_TILES(SSGD_MX_FP8, SSGD_MX_FP4); else SSGD_TILES(SSGD_MX_FP8, SSGD_MX_FP8); }
#undef SSGD_TILES
}

// rows x groups of eight columns in one launch (as a quotient: the product may pass 64 bits)
bool fits(int64_t rows, int64_t per_row) { return rows <= kMostBlocks * kThreads / per_row; }

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int64_t ssgd_mx_row_bytes(int32_t fmt, int64_t cols) { return format_ok(fmt) && cols >= 0 && cols < kMostCols ? mx_row_bytes(fmt, cols) : -1; }

ssgd_status ssgd_mx_quantize(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t pitch, int32_t fmt, void* values, void* scales,
                             int32_t fmt_t, void* values_t, void* scales_t, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        if (!dtype_ok(dtype) || rows < 0 || cols < 0 || rows >= kMostRows || cols >= kMostCols || pitch < cols)
            return op_fail(SSGD_EINVAL, "mx quantize: a type of the enumeration, rows and columns of zero or more, pitch >= columns");
        const bool along = values != nullptr || scales != nullptr, across = values_t != nullptr || scales_t != nullptr;
        if (rows == 0 || cols == 0) return SSGD_OK;
        if (!along && !across) return op_fail(SSGD_EINVAL, "mx quantize: no output");
        if ((along && (!format_ok(fmt) || !values || !scales || !aligned(values, 16) || !aligned(scales, 16))) ||
            (across && (!format_ok(fmt_t) || !values_t || !scales_t || !aligned(values_t, 16) || !aligned(scales_t, 16))))
            return op_fail(SSGD_EINVAL, "mx quantize: outputs are 16-byte aligned arrays of values and scales, formats of the enumeration");
        if (!x || !aligned(x, (uintptr_t)dtype_bytes(dtype))) return op_fail(SSGD_EINVAL, "mx quantize: the matrix is null or misaligned");
        if (across && rows >= kMostCols) return op_fail(SSGD_EINVAL, "mx quantize: too many rows to be columns");
        if (across ? mx_padded(cols) / kTile * (mx_padded(rows) / kTile) > kMostBlocks : !fits(rows, mx_padded(cols) / 8)) return op_fail(SSGD_EINVAL, "mx quantize: too many elements");
        const Source s{x, rows, cols, pitch};
        const Target t{static_cast<uint8_t*>(values), static_cast<uint8_t*>(scales), mx_row_bytes(fmt, cols), mx_padded(cols) / kMxBlock};
        const Target tt{static_cast<uint8_t*>(values_t), static_cast<uint8_t*>(scales_t), mx_row_bytes(fmt_t, rows), mx_padded(rows) / kMxBlock};
        const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        if (!across) { if (dtype == SSGD_F32) launch_rows<float>(s, t, fmt, stream); else launch_rows<bf16_t>(s, t, fmt, stream); }
        else if (dtype == SSGD_F32) launch_tiles<float>(s, t, fmt, tt, fmt_t, stream);
        else launch_tiles<bf16_t>(s, t, fmt, tt, fmt_t, stream);
        return op_hip(hipGetLastError(), "mx quantize");
    });
}

ssgd_status ssgd_mx_dequantize(const void* values, const void* scales, int32_t fmt, int64_t rows, int64_t cols, void* out, int32_t dtype, int64_t pitch,
                               void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        if (!dtype_ok(dtype) || !format_ok(fmt) || rows < 0 || cols < 0 || rows >= kMostRows || cols >= kMostCols || pitch < cols)
            return op_fail(SSGD_EINVAL, "mx dequantize: a type and a format of the enumerations, rows and columns of zero or more, pitch >= columns");
        if (rows == 0 || cols == 0) return SSGD_OK;
        if (!values || !scales || !out || !aligned(values, 16) || !aligned(scales, 16) || !aligned(out, (uintptr_t)dtype_bytes(dtype)))
            return op_fail(SSGD_EINVAL, "mx dequantize: a buffer is null or misaligned");
        const int64_t per_row = (cols + 7) / 8;
        if (!fits(rows, per_row)) return op_fail(SSGD_EINVAL, "mx dequantize: too many elements");
        const int64_t groups = rows * per_row;
        const int64_t rb = mx_row_bytes(fmt, cols), sb = mx_padded(cols) / kMxBlock;
        const dim3 grid((unsigned)((groups + kThreads - 1) / kThreads));
        const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
#define SSGD_BACK(F, T) hipLaunchKernelGGL((back_kernel<F, T>), grid, dim3(kThreads), 0, stream, static_cast<const uint8_t*>(values), static_cast<const uint8_t*>(scales), \
                                           rb, sb, static_cast<T*>(out), cols, pitch, groups, per_row)
        if (fmt == SSGD_MX_FP4) { if (dtype == SSGD_F32) SSGD_BACK(SSGD_MX_FP4, float); else SSGD_BACK(SSGD_MX_FP4, bf16_t); }
        else { if (dtype == SSGD_F32) SSGD_BACK(SSGD_MX_FP8, float); else SSGD_BACK(SSGD_MX_FP8, bf16_t); }
#undef SSGD_BACK
        return op_hip(hipGetLastError(), "mx dequantize");
    });
}

}  // extern "C"
#pragma GCC visibility pop
