// What lies between the products of a backward pass in few bits: the gradient of a dense layer's or a gated block's activation from its checkpoint, quantised
// along its rows and along its columns; and a checkpoint in few bits quantised again along its columns.
//
//   dp = dy act'(p),   h = act(p)          gated, in pairs of columns g, u:   dg = dy u act'(g),   du = dy act(g),   h = act(g) u
//
// Per pair from 8-bit checkpoints 4.1 bytes are read and 4.1 written for both quantisations of dp, 0.5 to 1 more for h's (8192 x 8192 pairs, dy in bf16, h in 8 bits: 141 us, 4.4 TB/s; p in bf16 172 us, 4.4 TB/s; not gated 85 us;
// a bias alone 53 us).  A wave has 1370 vector instructions for 64 values of dp, most of them of their two quantisations: 54 % of the time.  Large outputs go past the caches'
// replacement (7 us more otherwise).  Measured and not kept: four rows to a lane, for twice the waves (190 us: rows in pieces of 64 bytes), registers for three waves by force (173),
// workgroups of an XCD side by side (185), two, four or eight tiles of a column in turn (151 to 160 against 151), loads past the replacement (transposition of
// 8192 x 8192 to 4 bits 31 us instead of 22).  Rows in 4 bits leave a lane in four bytes and take the same time past the replacement or not (148 and 152 us).
#include <type_traits>

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

// A wave has 32 rows of the 128 columns of a tile: sixteen lanes side by side have eight columns each, the next sixteen the eight rows below.  So a block along a row is
// four lanes', and one along a column eight registers of the four lanes with the same place in a row of sixteen.
struct Place {
    int64_t row, col;       // the lane's first
    int32_t wave, turn, own;      // turn: of its rows, own: its first column in the tile
    __device__ __forceinline__ Place(int64_t r0, int64_t c0) {
        const int lane = threadIdx.x & 63;
        wave = threadIdx.x >> 6;
        turn = lane >> 4;
        own = (lane & 15) * 8;
        row = r0 + wave * 32 + turn * 8;
        col = c0 + own;
    }
};

// Eight columns of rows of the matrix that is quantised along its rows; `to`: the tile's first row (128 rows are less than 2^31 bytes).
struct Along {
    uint8_t *values, *scales;
    uint32_t at, scale_at;
    __device__ __forceinline__ Along(const Target& t, const Place& p, int64_t tile_row)
        : values(t.values + tile_row * kTile * t.row_bytes), scales(t.scales + tile_row * kTile * t.scale_bytes),
          at((uint32_t)(p.wave * 32 + p.turn * 8) * (uint32_t)t.row_bytes + (uint32_t)(t.fmt == SSGD_MX_FP4 ? p.col / 2 : p.col)),
          scale_at((uint32_t)(p.wave * 32 + p.turn * 8) * (uint32_t)t.scale_bytes + (uint32_t)(p.col / kMxBlock)) {}
    __device__ __forceinline__ void store(const Target& t, int r, bool live, const float (&x)[8]) const {
        const uint32_t most = max_of_4(largest_of(x)), to = at + (uint32_t)r * (uint32_t)t.row_bytes;
        uint32_t byte;
        if (t.fmt == SSGD_MX_FP4) {
            byte = mx_scale_byte<SSGD_MX_FP4>(most);
            if (live) *reinterpret_cast<uint32_t*>(values + to) = mx_pack_fp4(x, byte);
        } else {
            const words2 w = mx_quantize_fp8(x, most, byte);
            if (live) __builtin_nontemporal_store(w, reinterpret_cast<words2*>(values + to));
        }
        if (!live) return;
        if ((threadIdx.x & 3) == 0) scales[scale_at + (uint32_t)r * (uint32_t)t.scale_bytes] = (uint8_t)byte;
    }
};

// The columns of a tile, quantised, on their way to the transposed matrix: 128 rows of one are 128 or 64 bytes side by side there, of which a lane has eight or four
// (stored by the lanes themselves, in pieces of 32 bytes: 8192 x 8192 pairs in 8 bits 227 us instead of 158).  The 16-byte parts of a column, and columns next to each
// other, change places by the column's number, so that the lanes that write at a time, and those that read, meet in no bank.
template <int COLS> struct Columns {
    uint32_t values[COLS * 32];
    uint8_t scales[COLS * 4];
    static __device__ __forceinline__ int part8(int col, int part) { return ((col ^ ((col >> 6) & 1)) * 8 + (part ^ ((col >> 3) & 7))) * 4; }
    static __device__ __forceinline__ int part4(int col, int part) { return ((col ^ ((col >> 5) & 3)) * 4 + (part ^ ((col >> 3) & 3))) * 4; }
    // Eight rows of column `own + q` of the tile, q < 8 and own a multiple of eight.  (All that depends on the lane is the same for all q but which of two neighbours it is,
    // so the compiler has two addresses and constants.)
    __device__ __forceinline__ void put(int32_t fmt, const Place& at, int own, int q, const float (&x)[8]) {
        const uint32_t most = max_of_rows(largest_of(x));
        uint32_t byte;
        if (fmt == SSGD_MX_FP4) {
            byte = mx_scale_byte<SSGD_MX_FP4>(most);
            values[part4(own + q, at.wave) + at.turn] = mx_pack_fp4(x, byte);
        } else {
            const int flip = (own >> 6) & 1, part = (at.wave * 2 + (at.turn >> 1)) ^ ((own >> 3) & 7);
            const int first = (own * 8 + part) * 4 + (at.turn & 1) * 2 + (q % 2 ? -flip : flip) * 32;
            *reinterpret_cast<words2*>(&values[first + q * 32]) = mx_quantize_fp8(x, most, byte);
        }
        if (at.turn == 0) scales[(own + q) * 4 + at.wave] = (uint8_t)byte;
    }
    // The same for any column.
    __device__ __forceinline__ void put_at(int32_t fmt, const Place& at, int col, const float (&x)[8]) { put(fmt, at, col & ~7, col & 7, x); }
    // All of them, when all waves have met: column 0 is row `first` of the transposed matrix, of `rows`.
    __device__ __forceinline__ void store(const Target& t, int64_t first, int64_t rows, int64_t r0) const {
        const int parts = t.fmt == SSGD_MX_FP4 ? 4 : 8, shift = t.fmt == SSGD_MX_FP4 ? 2 : 3;
        const int64_t at = t.fmt == SSGD_MX_FP4 ? r0 / 2 : r0;
        for (int u = threadIdx.x; u < COLS * parts; u += kThreads) {
            const int col = u >> shift, part = u & (parts - 1);
            if (first + col >= rows) continue;
            const words4 w = *reinterpret_cast<const words4*>(&values[t.fmt == SSGD_MX_FP4 ? part4(col, part) : part8(col, part)]);
            __builtin_nontemporal_store(w, reinterpret_cast<words4*>(t.values + (first + col) * t.row_bytes + at + part * 16));
        }
        if ((int)threadIdx.x < COLS && first + threadIdx.x < rows)
            *reinterpret_cast<uint32_t*>(t.scales + (first + threadIdx.x) * t.scale_bytes + r0 / kMxBlock) = *reinterpret_cast<const uint32_t*>(&scales[threadIdx.x * 4]);
    }
};

// Eight rows of W columns as they come, two columns at a time as numbers.  (Values in few bits stay packed until they are used: with all of a lane's 64 numbers of
// p and dy in registers beside those of dp a SIMD had two waves.)
struct Fp8 {};       // with scales
template <typename T, int W> struct Raw;
template <int W> struct Raw<float, W> {
    float x[8][W];
    __device__ __forceinline__ void load_all(int r, const float* row) { load_vec<W>(row, W, x[r]); }
    __device__ __forceinline__ void settle(int r, int gone) {
        if (gone == 0) return;
#pragma unroll
        for (int step = W / 2; step > 0; step /= 2) {
            if (gone & step) {
#pragma unroll
                for (int q = 0; q < W; ++q) x[r][q] = q + step < W ? x[r][q + step] : 0.0f;
            }
        }
        if (gone >= W) clear(r);
    }
    __device__ __forceinline__ void load(int r, const float* row, int64_t left) { load_vec<W>(row, left, x[r]); }
    __device__ __forceinline__ void clear(int r) {
#pragma unroll
        for (int q = 0; q < W; ++q) x[r][q] = 0.0f;
    }
    __device__ __forceinline__ f32x2 pair(int r, int k) const { return f32x2{x[r][2 * k], x[r][2 * k + 1]}; }
};
template <int W> struct Raw<bf16_t, W> {
    uint32_t x[8][W / 2];
    __device__ __forceinline__ void load_all(int r, const bf16_t* row) {
        if constexpr (W == 8) {
            const words4 v = *reinterpret_cast<const words4_any*>(row);
            x[r][0] = v.x; x[r][1] = v.y; x[r][2] = v.z; x[r][3] = v.w;
        } else {
            const words2 v = *reinterpret_cast<const words2_any*>(row);
            x[r][0] = v.x; x[r][1] = v.y;
        }
    }
    __device__ __forceinline__ void settle(int r, int gone) {
        if (gone == 0) return;
#pragma unroll
        for (int step = W / 4; step > 0; step /= 2) {
            if (gone & (2 * step)) {
#pragma unroll
                for (int k = 0; k < W / 2; ++k) x[r][k] = k + step < W / 2 ? x[r][k + step] : 0u;
            }
        }
        if (gone & 1) {
#pragma unroll
            for (int k = 0; k < W / 2; ++k) x[r][k] = x[r][k] >> 16 | (k + 1 < W / 2 ? x[r][k + 1] << 16 : 0u);
        }
        if (gone >= W) clear(r);
    }
    __device__ __forceinline__ void load(int r, const bf16_t* row, int64_t left) {
        if (left >= W) load_all(r, row);
        else {
#pragma unroll
            for (int k = 0; k < W / 2; ++k) x[r][k] = (2 * k < left ? (uint32_t)row[2 * k] : 0u) | (2 * k + 1 < left ? (uint32_t)row[2 * k + 1] << 16 : 0u);
        }
    }
    __device__ __forceinline__ void clear(int r) {
#pragma unroll
        for (int k = 0; k < W / 2; ++k) x[r][k] = 0u;
    }
    __device__ __forceinline__ f32x2 pair(int r, int k) const { return f32x2{bf16_to_f32(x[r][k] & 0xFFFFu), __builtin_bit_cast(float, x[r][k] & 0xFFFF0000u)}; }
};
template <> struct Raw<Fp8, 8> {
    words2 x[8];
    float scale[8];
    __device__ __forceinline__ f32x2 pair(int r, int k) const {
        const int w = (int)(k < 2 ? x[r].x : x[r].y);
        const f32x2 v = k % 2 ? __builtin_amdgcn_cvt_pk_f32_fp8(w, true) : __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
        return f32x2{v.x * scale[r], v.y * scale[r]};
    }
};
// Rows of a matrix in a tile: `whole`: all of the tile's rows and columns are there.  Where they are not, rows past the last one read that one and columns past the end
// the row's last ones, which move to the front or are cleared when all have arrived: a load that may be left out waits for those before it (129 x 777: 14.7 us instead of 13.2, of which most is the code's
// first way through the instruction cache).
template <typename T, int W>
__device__ __forceinline__ void load_rows(Raw<T, W>& to, const void* matrix, int64_t pitch, int64_t rows, int64_t cols, int64_t row, int64_t col, bool whole) {
    const T* from = static_cast<const T*>(matrix);
    if (whole) {
        from += row * pitch + col;
#pragma unroll
        for (int r = 0; r < 8; ++r) to.load_all(r, from + r * pitch);
    } else if (cols >= W) {
        const int64_t at = col <= cols - W ? col : cols - W;
#pragma unroll
        for (int r = 0; r < 8; ++r) to.load_all(r, from + (row + r < rows ? row + r : rows - 1) * pitch + at);
        const int gone = col - at < W ? (int)(col - at) : W;
#pragma unroll
        for (int r = 0; r < 8; ++r) to.settle(r, row + r < rows ? gone : W);
    } else {
        from += row * pitch + col;
#pragma unroll
        for (int r = 0; r < 8; ++r) to.load(r, from + r * pitch, row + r < rows ? cols - col : 0);
    }
}
template <typename P>
__device__ __forceinline__ void load_kept(const Gradient& a, const Place& at, bool whole, Raw<P, 8>& p) {
    if constexpr (std::is_same_v<P, Fp8>) {
        uint32_t byte[8];
        // (from the tile's first row on: 128 rows are less than 2^31 bytes)
        const int64_t r0 = at.row - (at.wave * 32 + at.turn * 8);
        const uint8_t *values = a.p_values + r0 * a.p_bytes, *scales = a.p_scales + r0 * a.p_scale_bytes;
        const uint32_t pitch = (uint32_t)a.p_bytes, scale_pitch = (uint32_t)a.p_scale_bytes, row = (uint32_t)(at.wave * 32 + at.turn * 8);
        // (rows past the last one read that one, and are cleared)
        const uint32_t last = (uint32_t)(a.rows - 1 - r0 < kTile ? a.rows - 1 - r0 : kTile), cols_at = (uint32_t)at.col, block_at = (uint32_t)(at.col / kMxBlock);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const uint32_t own = row + r < last ? row + r : last;
            byte[r] = scales[own * scale_pitch + block_at];
            p.x[r] = *reinterpret_cast<const words2*>(values + (own * pitch + cols_at));
        }
        if (!whole) {
#pragma unroll
            for (int r = 0; r < 8; ++r) if (row + r > last) { byte[r] = 0u; p.x[r] = words2{0u, 0u}; }
        }
        // (columns past the last one in a block that is NaN are NaN too: what the formulas make of them is what they make of the block's others)
#pragma unroll
        for (int r = 0; r < 8; ++r) p.scale[r] = mx_scale_value(byte[r]);
    } else {
        if (a.p == nullptr) {
#pragma unroll
            for (int r = 0; r < 8; ++r) p.clear(r);
            return;
        }
        load_rows<P, 8>(p, a.p, a.p_pitch, a.rows, a.p_cols, at.row, at.col, whole);
    }
}

// Two columns of p, and of dy (gated: one), at a time: their part of dp, and their columns, which need no other.
template <int ACT, bool GATED, typename T, typename P>
__device__ __forceinline__ void differentiate(const Gradient& a, const Place& at, const Raw<P, 8>& p, const Raw<T, GATED ? 4 : 8>& dy, float (&d)[8][8], Columns<kTile>& columns,
                                              Columns<GATED ? kTile / 2 : kTile>& hidden) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float h[GATED ? 1 : 2][8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const f32x2 x = p.pair(r, k);
            float y, slope;
            if constexpr (GATED) {
                const f32x2 both = dy.pair(r, k / 2);
                const float g = k % 2 ? both.y : both.x;
                activation_and_slope(ACT, x.x, y, slope);
                // (relu selects, here as below: where its slope is zero, a product past fp32's range is no part of the gradient)
                d[r][2 * k] = ACT == SSGD_ACT_RELU ? (slope > 0.0f ? g * x.y : 0.0f) : g * x.y * slope;
                d[r][2 * k + 1] = g * y;
                h[0][r] = y * x.y;
            } else {
                const f32x2 g = dy.pair(r, k);
                activation_and_slope(ACT, x.x, y, slope);
                d[r][2 * k] = ACT == SSGD_ACT_RELU ? (slope > 0.0f ? g.x : 0.0f) : g.x * slope;
                h[0][r] = y;
                activation_and_slope(ACT, x.y, y, slope);
                d[r][2 * k + 1] = ACT == SSGD_ACT_RELU ? (slope > 0.0f ? g.y : 0.0f) : g.y * slope;
                h[1][r] = y;
            }
        }
        if (a.columns.values != nullptr) {
#pragma unroll
            for (int q = 2 * k; q < 2 * k + 2; ++q) {
                const float x[8] = {d[0][q], d[1][q], d[2][q], d[3][q], d[4][q], d[5][q], d[6][q], d[7][q]};
                columns.put(a.columns.fmt, at, at.own, q, x);
            }
        }
        if (a.hidden.values != nullptr) {
            if constexpr (GATED) hidden.put_at(a.hidden.fmt, at, at.own / 2 + k, h[0]);
            else {
                hidden.put(a.hidden.fmt, at, at.own, 2 * k, h[0]);
                hidden.put(a.hidden.fmt, at, at.own, 2 * k + 1, h[1]);
            }
        }
    }
}

template <typename T, typename P, bool GATED>
__global__ __launch_bounds__(kThreads) void gradient_kernel(Gradient a) {
    constexpr int W = GATED ? 4 : 8;
    __shared__ __attribute__((aligned(16))) Columns<kTile> columns;
    __shared__ __attribute__((aligned(16))) Columns<GATED ? kTile / 2 : kTile> hidden;
    __shared__ float sums[GATED ? 1 : 4][kTile];
    const int64_t tile_row = blockIdx.x / a.across, c0 = (blockIdx.x - tile_row * a.across) * kTile;
    const Place at(tile_row * kTile, c0);
    const int64_t own_col = GATED ? at.col / 2 : at.col;
    conversions_saturate();
    Raw<P, 8> p;
    Raw<T, W> dy;
    float d[8][8];
    const bool whole = (tile_row + 1) * kTile <= a.rows && c0 + kTile <= a.p_cols;
    load_rows<T, W>(dy, a.dy, a.dy_pitch, a.rows, a.cols, at.row, own_col, whole);
    load_kept(a, at, whole, p);
    if (a.activation == SSGD_ACT_RELU) differentiate<SSGD_ACT_RELU, GATED>(a, at, p, dy, d, columns, hidden);
    else if (a.activation == SSGD_ACT_GELU) differentiate<SSGD_ACT_GELU, GATED>(a, at, p, dy, d, columns, hidden);
    else if (a.activation == SSGD_ACT_SILU) differentiate<SSGD_ACT_SILU, GATED>(a, at, p, dy, d, columns, hidden);
    else differentiate<SSGD_ACT_NONE, GATED>(a, at, p, dy, d, columns, hidden);
    if (a.along.values != nullptr) {
        const Along to(a.along, at, tile_row);
#pragma unroll
        for (int r = 0; r < 8; ++r) to.store(a.along, r, whole || at.row + r < a.rows, d[r]);
    }
    if constexpr (!GATED) {
        if (a.partial != nullptr) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                float sum = 0.0f;
#pragma unroll
                for (int r = 0; r < 8; ++r) sum += d[r][q];
                sum = sum_of_rows(sum);
                if (at.turn == 0) sums[at.wave][at.own + q] = sum;
            }
        }
    }
    __syncthreads();
    if (a.columns.values != nullptr) columns.store(a.columns, c0, a.p_cols, tile_row * kTile);
    if (a.hidden.values != nullptr) hidden.store(a.hidden, GATED ? c0 / 2 : c0, a.cols, tile_row * kTile);
    if constexpr (!GATED) {
        const int64_t col = c0 + threadIdx.x;
        if (a.partial != nullptr && threadIdx.x < kTile && col < a.cols)
            a.partial[tile_row * a.cols + col] = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
    }
}

template <int FMT>
__global__ __launch_bounds__(kThreads) void transpose_kernel(const uint8_t* values, const uint8_t* scales, int64_t row_bytes, int64_t scale_bytes, int64_t rows, int64_t cols, Target t,
                                                             int64_t across) {
    __shared__ __attribute__((aligned(16))) Columns<kTile> columns;
    const int64_t tile_row = blockIdx.x / across, c0 = (blockIdx.x - tile_row * across) * kTile;
    const Place at(tile_row * kTile, c0);
    conversions_saturate();
    float x[8][8];
    uint32_t byte[8];
    words2 w[8];
    // (rows past the last one read that one, and are cleared)
    auto load = [&](int r) {
        const int64_t row = at.row + r < rows ? at.row + r : rows - 1;
        const uint8_t* from = values + row * row_bytes + (FMT == SSGD_MX_FP8 ? at.col : at.col / 2);
        byte[r] = scales[row * scale_bytes + at.col / kMxBlock];
        if constexpr (FMT == SSGD_MX_FP8) w[r] = *reinterpret_cast<const words2*>(from);
        else w[r] = words2{*reinterpret_cast<const uint32_t*>(from), 0u};
    };
#pragma unroll
    for (int r = 0; r < 8; ++r) load(r);
    if ((tile_row + 1) * kTile > rows) {
#pragma unroll
        for (int r = 0; r < 8; ++r) if (at.row + r >= rows) { byte[r] = 0u; w[r] = words2{0u, 0u}; }
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        if constexpr (FMT == SSGD_MX_FP8) mx_unpack_fp8(w[r], mx_scale_value(byte[r]), x[r]);
        else mx_unpack_fp4(w[r].x, mx_scale_value(byte[r]), x[r]);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const float y[8] = {x[0][q], x[1][q], x[2][q], x[3][q], x[4][q], x[5][q], x[6][q], x[7][q]};
        columns.put(t.fmt, at, at.own, q, y);
    }
    __syncthreads();
    columns.store(t, c0, cols, tile_row * kTile);
}

bool format_ok(int32_t f) { return f == SSGD_MX_FP4 || f == SSGD_MX_FP8; }
constexpr int64_t kMost = int64_t(1) << 31, kMostColumns = (int64_t(1) << 24) - kMxPad;      // of p: what a product contracts
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

int64_t ssgd_mx_activation_backward_work_floats(int64_t rows, int64_t cols) { return rows < 0 || cols < 0 || rows >= kMost || cols > kMostColumns ? -1 : (rows <= kTile && rows > 0 ? 0 : tiles_of(rows) * cols); }      // (one tile of rows leaves its sums where they belong)

ssgd_status ssgd_mx_activation_backward(const void* dy, int32_t dtype, int64_t dy_pitch, int64_t rows, int64_t cols, int32_t gated, int32_t activation, const void* p, int32_t p_dtype,
                                        int64_t p_pitch, const void* p_values, const void* p_scales, int32_t fmt, void* values, void* scales, int32_t fmt_t, void* values_t,
                                        void* scales_t, int32_t fmt_h, void* values_h, void* scales_h, float* dbias, float* work, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        const char* name = "mx activation backward: ";
        auto no = [&](const char* what) { return op_fail(SSGD_EINVAL, (std::string(name) + what).c_str()); };
        if (!dtype_ok(dtype) || rows < 0 || cols < 0 || rows >= kMost || cols > kMostColumns || (gated == 1 && 2 * cols > kMostColumns)) return no("a type of the enumeration, rows from zero to 2^31, columns of p to 2^24 - 128");
        if ((gated != 0 && gated != 1) || activation < SSGD_ACT_NONE || activation > SSGD_ACT_SILU) return no("an activation of the enumeration, gated or not");
        if (gated && dbias != nullptr) return no("a gated block has no bias");
        if (dbias != nullptr && (!aligned(dbias, 4) || (rows > kTile && cols > 0 && (!work || !aligned(work, 16))))) return no("dbias, a gradient of a bias, needs a 16-byte aligned work area");
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
            a.across = tiles_of(p_cols); a.p_bf16 = p == nullptr || p_dtype == SSGD_BF16; a.activation = activation;
            a.along = target_of(values, scales, fmt, p_cols); a.columns = target_of(values_t, scales_t, fmt_t, rows); a.hidden = target_of(values_h, scales_h, fmt_h, rows);
            a.partial = dbias != nullptr && rows > kTile ? work : dbias;
            const dim3 grid((unsigned)(tiles_of(rows) * a.across));
#define SSGD_GRADIENT(T, P) do { if (gated) hipLaunchKernelGGL((gradient_kernel<T, P, true>), grid, dim3(kThreads), 0, stream, a); \
                                  else hipLaunchKernelGGL((gradient_kernel<T, P, false>), grid, dim3(kThreads), 0, stream, a); } while (0)
            if (dtype == SSGD_F32) { if (p_values) SSGD_GRADIENT(float, Fp8); else if (a.p_bf16) SSGD_GRADIENT(float, bf16_t); else SSGD_GRADIENT(float, float); }
            else { if (p_values) SSGD_GRADIENT(bf16_t, Fp8); else if (a.p_bf16) SSGD_GRADIENT(bf16_t, bf16_t); else SSGD_GRADIENT(bf16_t, float); }
#undef SSGD_GRADIENT
        }
        if (dbias != nullptr && (rows > kTile || rows == 0)) launch_column_sums(work, tiles_of(rows), cols, dbias, stream);
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
