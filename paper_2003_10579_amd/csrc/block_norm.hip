// What lies between two blocks of a residual stream: the norm behind the first, its gate, the scaled residual, and the norm in front of the second.
//
//   s' = scale s + gate (o rstd_o) w_post      (rounded to the rows' type: what the stream keeps is what is normalised, forward and backward)
//   y = (s' rstd) w                            rstd_o = (mean o^2 + eps)^(-1/2),   rstd = (mean s'^2 + eps)^(-1/2)
//
//   G = rstd (dy w - shat mean(dy w shat)) + dsum,   shat = s' rstd,   ohat = o rstd_o                (the gradient of s')
//   ds = scale G,   do = rstd_o (G gate w_post - ohat mean(G gate w_post ohat))
//   dw = sum dy shat,   S = sum over a gate's rows of G ohat:   dgate = w_post S,   dw_post = sum over gates of gate S
//
// Bound by memory (16384 x 4096 in bf16, a gate for each of 8 runs: forward with 8-bit output 85 us, 5.5 TB/s; backward 159 us and its sums 7, 4.8 TB/s; 4000 x 8192: 43 and 79 us; 65536 x 512:
// 42 and 76).  Rows of 8193 to 16384 columns leave 1024 threads no registers for the next one, and some of their own go to scratch memory (forward 4 to 17 of 128, backward 34 in bf16 and 94 in
// fp32): 2000 x 16000 in bf16 3.6 and 2.4 TB/s; so do backward rows of 4097 to 8192 in fp32 (31 of 256; 4000 x 8192: 234 us, 3.4 TB/s, forward 86 us, 5.0).  A row stays in the registers of its threads, eight or sixteen columns each, through both sums.  The sum s' is taken in fp64,
// rounded to fp32 and from there to the rows' type, as torch brings fp64 to bfloat16: what it is rounded to decides all that follows, and a sum of three products in fp32 is a few units off before
// it is rounded (of bfloat16 rows three sums in 10^5 are on the other side of a border then; through fp32 seven in 10^6 are not the nearest to the sum in fp64).
#include <cmath>

#include "rows.hpp"

using namespace ssgd;

namespace {

constexpr int kMostKept = 16384;      // columns that fit the registers of 1024 threads
constexpr int64_t kMostColumns = int64_t(1) << 24;     // 16 to a workgroup of 1024 in the sums, of two kinds: a launch ends at 2^32 threads

struct Forward {
    const void *o, *s, *post, *w, *gate;
    void *sum, *y;
    uint8_t *values, *scales;
    float *rstd_o, *rstd;
    int64_t rows, per_gate, chunk, o_pitch, s_pitch, sum_pitch, y_pitch, gate_pitch, row_bytes, scale_bytes;
    int32_t d, post_bf16, w_bf16, gate_bf16;
    double scale, eps, per_column;        // per_column: 1 / d
};

struct Backward {
    const void *dy, *o, *sum, *post, *w, *gate, *dsum;
    const float *rstd_o, *rstd;
    void *grad_o, *grad_s;
    float *dw_parts, *s_parts;            // [units][d], nullptr: not wanted
    int64_t rows, per_gate, chunk, chunks, dy_pitch, o_pitch, sum_pitch, gate_pitch, dsum_pitch, grad_o_pitch, grad_s_pitch;
    int32_t d, post_bf16, w_bf16, gate_bf16;
    float scale;
    double per_column;                    // 1 / d
};

// Sum over the threads of a row, in fp64, by moves between lanes that do not go through LDS.  A row has two of them with an array each, and all waves have read one when
// they meet for the other: one meeting to a sum.
template <int CTRL>
__device__ __forceinline__ double plus_moved(double x) {
    const uint64_t w = __builtin_bit_cast(uint64_t, x);
    const uint64_t v = (uint64_t)dpp<CTRL>((uint32_t)(w >> 32)) << 32 | dpp<CTRL>((uint32_t)w);
    return x + __builtin_bit_cast(double, v);
}
__device__ __forceinline__ double sum_of_pair(uint32_t lo0, uint32_t hi0, uint32_t lo1, uint32_t hi1) {
    return __builtin_bit_cast(double, (uint64_t)hi0 << 32 | lo0) + __builtin_bit_cast(double, (uint64_t)hi1 << 32 | lo1);
}
__device__ __forceinline__ double sum_of_wave(double x) {
    x = plus_moved<kMirror>(plus_moved<kHalfMirror>(plus_moved<kXor2>(plus_moved<kXor1>(x))));
    uint64_t w = __builtin_bit_cast(uint64_t, x);
    const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)w, (uint32_t)w, false, false), hi = __builtin_amdgcn_permlane16_swap((uint32_t)(w >> 32), (uint32_t)(w >> 32), false, false);
    w = __builtin_bit_cast(uint64_t, sum_of_pair(lo[0], hi[0], lo[1], hi[1]));
    const auto lo2 = __builtin_amdgcn_permlane32_swap((uint32_t)w, (uint32_t)w, false, false), hi2 = __builtin_amdgcn_permlane32_swap((uint32_t)(w >> 32), (uint32_t)(w >> 32), false, false);
    return sum_of_pair(lo2[0], hi2[0], lo2[1], hi2[1]);
}
template <int LANES>
__device__ __forceinline__ double team_sum(double x, double* part) {
    x = sum_of_wave(x);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0.0;
#pragma unroll
        for (int q = 0; q < LANES / 64; ++q) x += part[q];
    }
    return x;
}
// The sum of squares of a row's numbers.  (In fp64 from the squares on: what is a unit of 2^-24 off in rstd_o is one in the sum that is rounded.)
template <int LANES, int NV>
__device__ __forceinline__ double sum_of_squares(const float (&x)[NV][8], double* part) {
    double sum = 0.0;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int q = 0; q < 8; ++q) sum += (double)x[v][q] * (double)x[v][q];
    return team_sum<LANES>(sum, part);
}

template <typename T>
__device__ __forceinline__ void load_row(const void* rows, int64_t row, int64_t pitch, int col, int d, float (&x)[8]) { load_vec<8>(static_cast<const T*>(rows) + row * pitch + col, d - col, x); }

// (mean + eps)^(-1/2) from the sum of squares: an estimate of 2^-26 or so, and one step of Newton's that doubles its digits (a root and a quotient in fp64 are a hundred
// instructions for every thread of a row).
__device__ __forceinline__ double inverse_root(double squares, double per_column, double eps) {
    const double x = __builtin_fma(squares, per_column, eps), r = __builtin_amdgcn_rsq(x);
    const double better = __builtin_fma(r, __builtin_fma(-0.5 * x * r, r, 0.5), r);
    return x > 0.0 && x < __builtin_inf() ? better : r;
}

// w_post times the gate of a row: what the normalised output is multiplied by.
__device__ __forceinline__ void factor_of(const Forward& a, int64_t gate, int col, double (&f)[8]) {
    float x[8];
    load_weight(a.post, a.post_bf16, col, a.d - col, x);
#pragma unroll
    for (int q = 0; q < 8; ++q) f[q] = x[q];
    if (a.gate == nullptr) return;
    load_weight(a.gate, a.gate_bf16, gate * a.gate_pitch + col, a.d - col, x);
#pragma unroll
    for (int q = 0; q < 8; ++q) f[q] *= x[q];
}
template <typename T>
__device__ __forceinline__ void join(const Forward& a, const float (&o)[8], const float (&s)[8], const double (&f)[8], double rstd_o, float (&sum)[8]) {
#pragma unroll
    for (int q = 0; q < 8; ++q) sum[q] = as_stored(static_cast<const T*>(nullptr), (float)((double)s[q] * a.scale + ((double)o[q] * rstd_o) * f[q]));
}
template <typename T, bool FP8>
__device__ __forceinline__ void store_normed(const Forward& a, int64_t row, int col, const float (&s)[8], float rstd, const float (&w)[8]) {
    float y[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) y[q] = (s[q] * rstd) * w[q];
    if constexpr (FP8) {
        const uint32_t byte = mx_scale_byte<SSGD_MX_FP8>(max_of_4(largest_of(y)));
        __builtin_nontemporal_store(mx_pack_fp8(y, byte), reinterpret_cast<words2*>(a.values + row * a.row_bytes + col));
        if ((threadIdx.x & 3) == 0) a.scales[row * a.scale_bytes + col / kMxBlock] = (uint8_t)byte;
    } else {
        stream_vec(static_cast<T*>(a.y) + row * a.y_pitch + col, a.d - col, y);
    }
}

// (The weights and the gate stay in registers, and the next row is on its way while a row's sums are taken; sixteen columns to each of 1024 threads leave no registers
// for either: they read both again for every row, from L2.)
template <typename T, bool FP8, int LANES, int NV>
__global__ __launch_bounds__(LANES == 64 ? 256 : LANES) void forward_kernel(Forward a) {
    constexpr int kRows = LANES == 64 ? 4 : 1;         // teams of a workgroup
    constexpr bool kKept = LANES < 1024 || NV == 1, kShort = LANES == 64 && NV == 1;
    __shared__ double part[2][LANES / 64];
    const int lane = threadIdx.x & (LANES - 1);
    const int64_t team = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES, first = team * a.chunk, end = first + a.chunk < a.rows ? first + a.chunk : a.rows;
    const int wide = FP8 ? (int)mx_padded(a.d) : a.d;
    int64_t gate = first / a.per_gate, next_gate = (gate + 1) * a.per_gate;
    double f[NV][8];
    float w[NV][8];
    auto col_of = [&](int v) { return (v * LANES + lane) * 8; };
    auto end_of = [&](int v) { return v < NV - 1 ? col_of(v) + 8 : a.d; };          // (kernels with NV > 1 have rows that long)
    Eight<T> next_o[NV], next_s[NV];
    auto load = [&](int64_t row) {
        if (row >= end) return;
#pragma unroll
        for (int v = 0; v < NV; ++v) read<kShort>(next_o[v], a.o, row, a.o_pitch, col_of(v), end_of(v), a.d);
#pragma unroll
        for (int v = 0; v < NV; ++v) read<kShort>(next_s[v], a.s, row, a.s_pitch, col_of(v), end_of(v), a.d);
    };
    if (first >= end) return;              // (the whole team; teams of several waves have their workgroup to themselves)
    if constexpr (kKept) {
        load(first);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            load_weight(a.w, a.w_bf16, col_of(v), end_of(v) - col_of(v), w[v]);
            factor_of(a, gate, col_of(v), f[v]);
        }
    }
    for (int64_t row = first; row < end; ++row) {
        if (row == next_gate) {
            ++gate;
            next_gate += a.per_gate;
            if constexpr (kKept) {
#pragma unroll
                for (int v = 0; v < NV; ++v) factor_of(a, gate, col_of(v), f[v]);
            }
        }
        if constexpr (!kKept) load(row);
        float o[NV][8], s[NV][8];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            numbers<kShort>(next_o[v], col_of(v), end_of(v), a.d, o[v]);
            numbers<kShort>(next_s[v], col_of(v), end_of(v), a.d, s[v]);
        }
        if constexpr (kKept) load(row + 1);
        const double rstd_o = inverse_root(sum_of_squares<LANES, NV>(o, part[0]), a.per_column, a.eps);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (!kKept) factor_of(a, gate, col_of(v), f[v]);
            join<T>(a, o[v], s[v], f[v], rstd_o, o[v]);
            stream_vec(static_cast<T*>(a.sum) + row * a.sum_pitch + col_of(v), end_of(v) - col_of(v), o[v]);
        }
        const float rstd = (float)inverse_root(sum_of_squares<LANES, NV>(o, part[1]), a.per_column, a.eps);
        if (lane == 0) { a.rstd_o[row] = (float)rstd_o; a.rstd[row] = rstd; }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (!kKept) load_weight(a.w, a.w_bf16, col_of(v), end_of(v) - col_of(v), w[v]);
            if (v < NV - 1 || col_of(v) < wide) store_normed<T, FP8>(a, row, col_of(v), o[v], rstd, w[v]);
        }
    }
}

// Rows that registers do not hold: o a second time, and the sum, which its own threads have written.
template <typename T, bool FP8>
__global__ __launch_bounds__(1024) void forward_long_kernel(Forward a) {
    __shared__ double part[2][16];
    const int wide = FP8 ? (int)mx_padded(a.d) : a.d;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t gate = row / a.per_gate;
        double squares = 0.0;
        for (int col = threadIdx.x * 8; col < a.d; col += 8192) {
            float o[8];
            load_row<T>(a.o, row, a.o_pitch, col, a.d, o);
#pragma unroll
            for (int q = 0; q < 8; ++q) squares += (double)o[q] * (double)o[q];
        }
        const double rstd_o = inverse_root(team_sum<1024>(squares, part[0]), a.per_column, a.eps);
        squares = 0.0;
        for (int col = threadIdx.x * 8; col < a.d; col += 8192) {
            float o[8], s[8];
            double f[8];
            load_row<T>(a.o, row, a.o_pitch, col, a.d, o);
            load_row<T>(a.s, row, a.s_pitch, col, a.d, s);
            factor_of(a, gate, col, f);
            join<T>(a, o, s, f, rstd_o, s);
#pragma unroll
            for (int q = 0; q < 8; ++q) squares += (double)s[q] * (double)s[q];
            stream_vec(static_cast<T*>(a.sum) + row * a.sum_pitch + col, a.d - col, s);
        }
        const float rstd = (float)inverse_root(team_sum<1024>(squares, part[1]), a.per_column, a.eps);
        if (threadIdx.x == 0) { a.rstd_o[row] = (float)rstd_o; a.rstd[row] = rstd; }
        for (int col = threadIdx.x * 8; col < wide; col += 8192) {
            float s[8], w[8];
            load_row<T>(a.sum, row, a.sum_pitch, col, a.d, s);
            load_weight(a.w, a.w_bf16, col, a.d - col, w);
            store_normed<T, FP8>(a, row, col, s, rstd, w);
        }
    }
}

__device__ __forceinline__ void factor_of(const Backward& a, int64_t gate, int col, float (&f)[8]) {
    load_weight(a.post, a.post_bf16, col, a.d - col, f);
    if (a.gate == nullptr) return;
    float x[8];
    load_weight(a.gate, a.gate_bf16, gate * a.gate_pitch + col, a.d - col, x);
#pragma unroll
    for (int q = 0; q < 8; ++q) f[q] *= x[q];
}
template <typename T>
__device__ __forceinline__ void load_dsum(const Backward& a, int64_t row, int col, float (&x)[8]) {
    if (a.dsum != nullptr) load_row<T>(a.dsum, row, a.dsum_pitch, col, a.d, x);
    else {
#pragma unroll
        for (int q = 0; q < 8; ++q) x[q] = 0.0f;
    }
}

// A workgroup takes a unit: up to `chunk` rows that share a gate, whose sums of dw and S it leaves.
template <typename T, int LANES, int NV>
__global__ __launch_bounds__(LANES == 64 ? 256 : LANES) void backward_kernel(Backward a) {
    constexpr int kRows = LANES == 64 ? 4 : 1;
    constexpr bool kKept = LANES < 1024 || NV == 1, kShort = LANES == 64 && NV == 1;
    __shared__ double part[2][LANES / 64];
    __shared__ float others[kRows > 1 ? kRows - 1 : 1][kRows > 1 ? LANES * NV * 16 : 1];
    const int lane = threadIdx.x & (LANES - 1), team = threadIdx.x / LANES;
    const int64_t gate = blockIdx.x / a.chunks, begin = (blockIdx.x - gate * a.chunks) * a.chunk, rows = a.per_gate - begin < a.chunk ? a.per_gate - begin : a.chunk;
    const int64_t first = gate * a.per_gate + begin, end = first + rows;
    auto col_of = [&](int v) { return (v * LANES + lane) * 8; };
    auto end_of = [&](int v) { return v < NV - 1 ? col_of(v) + 8 : a.d; };
    float w[NV][8], f[NV][8], dw[NV][8], S[NV][8];
    auto load_sides = [&](int v) {
        load_weight(a.w, a.w_bf16, col_of(v), end_of(v) - col_of(v), w[v]);
        factor_of(a, gate, col_of(v), f[v]);
    };
    Eight<T> next_dy[NV], next_sum[NV], next_o[NV], next_more[NV];
    float next_rstd = 0.0f, next_rstd_o = 0.0f;
    auto load = [&](int64_t row) {
        if (row >= end) return;
        next_rstd = a.rstd[row];
        next_rstd_o = a.rstd_o[row];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            read<kShort>(next_dy[v], a.dy, row, a.dy_pitch, col_of(v), end_of(v), a.d);
            read<kShort>(next_sum[v], a.sum, row, a.sum_pitch, col_of(v), end_of(v), a.d);
            read<kShort>(next_o[v], a.o, row, a.o_pitch, col_of(v), end_of(v), a.d);
        }
        if (a.dsum != nullptr) {
#pragma unroll
            for (int v = 0; v < NV; ++v) read<kShort>(next_more[v], a.dsum, row, a.dsum_pitch, col_of(v), end_of(v), a.d);
        }
    };
    if constexpr (kKept) load(first + team);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if constexpr (kKept) load_sides(v);
#pragma unroll
        for (int q = 0; q < 8; ++q) dw[v][q] = S[v][q] = 0.0f;
    }
    for (int64_t row = first + team; row < end; row += kRows) {
        if constexpr (!kKept) load(row);
        const float rstd = next_rstd, rstd_o = next_rstd_o;
        float g[NV][8], x[NV][8];
        // (o and what is added past the sum stay as they came until they are used)
        Eight<T> raw_o[NV], raw_more[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            numbers<kShort>(next_dy[v], col_of(v), end_of(v), a.d, g[v]);
            numbers<kShort>(next_sum[v], col_of(v), end_of(v), a.d, x[v]);
            raw_o[v] = next_o[v];
            if (a.dsum != nullptr) raw_more[v] = next_more[v];
        }
        if constexpr (kKept) load(row + kRows);
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (!kKept) load_sides(v);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                x[v][q] *= rstd;
                dw[v][q] += g[v][q] * x[v][q];
                g[v][q] *= w[v][q];
                sum += g[v][q] * x[v][q];
            }
        }
        const float c = (float)(team_sum<LANES>((double)sum, part[0]) * a.per_column);
        sum = 0.0f;
        float oh[NV][8];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            numbers<kShort>(raw_o[v], col_of(v), end_of(v), a.d, oh[v]);
#pragma unroll
            for (int q = 0; q < 8; ++q) g[v][q] = rstd * (g[v][q] - x[v][q] * c);
            if (a.dsum != nullptr) {
                numbers<kShort>(raw_more[v], col_of(v), end_of(v), a.d, x[v]);
#pragma unroll
                for (int q = 0; q < 8; ++q) g[v][q] += x[v][q];
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                oh[v][q] *= rstd_o;
                S[v][q] += g[v][q] * oh[v][q];
                x[v][q] = g[v][q] * f[v][q];
                sum += x[v][q] * oh[v][q];
            }
        }
        const float c_o = (float)(team_sum<LANES>((double)sum, part[1]) * a.per_column);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (v == NV - 1 && col_of(v) >= a.d) break;
#pragma unroll
            for (int q = 0; q < 8; ++q) { oh[v][q] = rstd_o * (x[v][q] - oh[v][q] * c_o); g[v][q] *= a.scale; }
            stream_vec(static_cast<T*>(a.grad_o) + row * a.grad_o_pitch + col_of(v), end_of(v) - col_of(v), oh[v]);
            stream_vec(static_cast<T*>(a.grad_s) + row * a.grad_s_pitch + col_of(v), end_of(v) - col_of(v), g[v]);
        }
    }
    if (a.dw_parts == nullptr) return;
    if constexpr (kRows > 1) {
        // the rows of a workgroup's waves, in their order
        if (team > 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                store_vec<8>(&others[team - 1][(v * LANES + lane) * 16], 8, dw[v]);
                store_vec<8>(&others[team - 1][(v * LANES + lane) * 16 + 8], 8, S[v]);
            }
        }
        __syncthreads();
        if (team > 0) return;
#pragma unroll
        for (int t = 0; t < kRows - 1; ++t)
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float x[8], y[8];
                load_vec<8>(&others[t][(v * LANES + lane) * 16], 8, x);
                load_vec<8>(&others[t][(v * LANES + lane) * 16 + 8], 8, y);
#pragma unroll
                for (int q = 0; q < 8; ++q) { dw[v][q] += x[q]; S[v][q] += y[q]; }
            }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        store_vec<8>(a.dw_parts + (int64_t)blockIdx.x * a.d + col_of(v), end_of(v) - col_of(v), dw[v]);
        store_vec<8>(a.s_parts + (int64_t)blockIdx.x * a.d + col_of(v), end_of(v) - col_of(v), S[v]);
    }
}

// The same for rows that registers do not hold: what is read is read again for each sum, and the unit's sums are read and written for every row.
template <typename T>
__global__ __launch_bounds__(1024) void backward_long_kernel(Backward a) {
    __shared__ double part[2][16];
    const int64_t gate = blockIdx.x / a.chunks, begin = (blockIdx.x - gate * a.chunks) * a.chunk, rows = a.per_gate - begin < a.chunk ? a.per_gate - begin : a.chunk;
    const int64_t first = gate * a.per_gate + begin;
    for (int64_t row = first; row < first + rows; ++row) {
        const float rstd = a.rstd[row], rstd_o = a.rstd_o[row];
        double sum = 0.0;
        for (int col = threadIdx.x * 8; col < a.d; col += 8192) {
            float g[8], x[8], w[8];
            load_row<T>(a.dy, row, a.dy_pitch, col, a.d, g);
            load_row<T>(a.sum, row, a.sum_pitch, col, a.d, x);
            load_weight(a.w, a.w_bf16, col, a.d - col, w);
            float few = 0.0f;
#pragma unroll
            for (int q = 0; q < 8; ++q) few += g[q] * w[q] * (x[q] * rstd);
            sum += few;
        }
        const float c = (float)(team_sum<1024>(sum, part[0]) * a.per_column);
        // G and what is multiplied with it, of eight columns
        auto gradient = [&](int col, float (&g)[8], float (&oh)[8], float (&f)[8], float (&dw)[8]) {
            float x[8], w[8], more[8];
            load_row<T>(a.dy, row, a.dy_pitch, col, a.d, g);
            load_row<T>(a.sum, row, a.sum_pitch, col, a.d, x);
            load_row<T>(a.o, row, a.o_pitch, col, a.d, oh);
            load_dsum<T>(a, row, col, more);
            load_weight(a.w, a.w_bf16, col, a.d - col, w);
            factor_of(a, gate, col, f);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                x[q] *= rstd;
                dw[q] = g[q] * x[q];
                g[q] = rstd * (g[q] * w[q] - x[q] * c) + more[q];
                oh[q] *= rstd_o;
            }
        };
        sum = 0.0;
        for (int col = threadIdx.x * 8; col < a.d; col += 8192) {
            float g[8], oh[8], f[8], dw[8];
            gradient(col, g, oh, f, dw);
            float few = 0.0f;
#pragma unroll
            for (int q = 0; q < 8; ++q) few += g[q] * f[q] * oh[q];
            sum += few;
        }
        const float c_o = (float)(team_sum<1024>(sum, part[1]) * a.per_column);
        for (int col = threadIdx.x * 8; col < a.d; col += 8192) {
            float g[8], oh[8], f[8], dw[8], S[8], x[8];
            gradient(col, g, oh, f, dw);
#pragma unroll
            for (int q = 0; q < 8; ++q) { S[q] = g[q] * oh[q]; x[q] = rstd_o * (g[q] * f[q] - oh[q] * c_o); g[q] *= a.scale; }
            stream_vec(static_cast<T*>(a.grad_o) + row * a.grad_o_pitch + col, a.d - col, x);
            stream_vec(static_cast<T*>(a.grad_s) + row * a.grad_s_pitch + col, a.d - col, g);
            if (a.dw_parts == nullptr) continue;
            float *dw_to = a.dw_parts + (int64_t)blockIdx.x * a.d + col, *s_to = a.s_parts + (int64_t)blockIdx.x * a.d + col;
            if (row > first) {
                load_vec<8>(dw_to, a.d - col, x);
#pragma unroll
                for (int q = 0; q < 8; ++q) dw[q] += x[q];
                load_vec<8>(s_to, a.d - col, x);
#pragma unroll
                for (int q = 0; q < 8; ++q) S[q] += x[q];
            }
            store_vec<8>(dw_to, a.d - col, dw);
            store_vec<8>(s_to, a.d - col, S);
        }
    }
}

// The units' sums of 16 columns, in fp64 and in order: dw by the workgroups of blockIdx.y = 0; by the others S, for each gate by its own 64 / `slots` of the 64 quarter
// waves, with dgate, and over the gates dw_post.
struct Sums { const float *dw_parts, *s_parts; const void *post, *gate; float *dw, *dw_post, *dgate; int64_t gates, chunks, gate_pitch, dgate_pitch; int32_t d, post_bf16, gate_bf16, slots; };
__device__ __forceinline__ float side_at(const void* w, int bf16, int64_t at) { return bf16 ? bf16_to_f32(static_cast<const bf16_t*>(w)[at]) : static_cast<const float*>(w)[at]; }
__global__ __launch_bounds__(1024) void sums_kernel(Sums a) {
    __shared__ double part[64][17];
    const int c = threadIdx.x & 15, quarter = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    const bool live = col < a.d;
    auto strided = [&](const float* from, int64_t n, int begin, int step) {
        double sum = 0.0;
        if (!live) return sum;
        for (int64_t t = begin; t < n; t += (int64_t)step * 8) {
            float x[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = from[(t + (int64_t)step * q < n ? t + (int64_t)step * q : n - 1) * a.d + col];
#pragma unroll
            for (int q = 0; q < 8; ++q) sum += t + (int64_t)step * q < n ? (double)x[q] : 0.0;
        }
        return sum;
    };
    if (blockIdx.y == 0) {
        part[quarter][c] = strided(a.dw_parts, a.gates * a.chunks, quarter, 64);
        __syncthreads();
        if (quarter != 0 || !live) return;
        double sum = 0.0;
        for (int q = 0; q < 64; ++q) sum += part[q][c];
        a.dw[col] = (float)sum;
        return;
    }
    const int each = 64 / a.slots;
    const float post = live ? side_at(a.post, a.post_bf16, col) : 0.0f;
    double total = 0.0;
    for (int64_t base = 0; base < a.gates; base += a.slots) {
        const int64_t gate = base + quarter / each;
        double sum = 0.0;
        if (gate < a.gates) sum = strided(a.s_parts + gate * a.chunks * a.d, a.chunks, quarter % each, each);
        __syncthreads();
        part[quarter][c] = sum;
        __syncthreads();
        if (quarter < a.slots && base + quarter < a.gates && live) {
            sum = 0.0;
            for (int q = 0; q < each; ++q) sum += part[quarter * each + q][c];
            if (a.dgate != nullptr) a.dgate[(base + quarter) * a.dgate_pitch + col] = (float)(sum * post);
            total += a.gate != nullptr ? sum * side_at(a.gate, a.gate_bf16, (base + quarter) * a.gate_pitch + col) : sum;
        }
    }
    __syncthreads();
    part[quarter][c] = total;
    __syncthreads();
    if (quarter != 0 || !live) return;
    double sum = 0.0;
    for (int q = 0; q < a.slots; ++q) sum += part[q][c];
    a.dw_post[col] = (float)sum;
}

// Threads of a row.  (16384 x 4096 in bf16, forward: 256 with sixteen columns each 85 us, 512 with eight 91 to 95; backward with its sums, which has more to keep: 166 either way.  4000 x 8192,
// 512 and 1024: 43 and 51 us, 79 and 99.  In fp32 16384 x 4096 takes 223 and 198 us forward, 429 and 399 backward.)
int lanes_for(int64_t d) { return d <= 1024 ? 64 : (d <= 4096 ? 256 : (d <= 8192 ? 512 : 1024)); }
int lanes_backward(int64_t d) { return d <= 1024 ? 64 : (d <= 2048 ? 256 : (d <= 8192 ? 512 : 1024)); }

template <typename T, bool FP8>
void launch_forward(Forward a, hipStream_t s) {
    const int lanes = lanes_for(a.d), teams = lanes == 64 ? 4 : 1;
    if (a.d > kMostKept) {
        hipLaunchKernelGGL((forward_long_kernel<T, FP8>), dim3((unsigned)(a.rows < 512 ? a.rows : 512)), dim3(1024), 0, s, a);
        return;
    }
    // rows next to each other to a team: they share a gate as a rule
    // as many workgroups as are resident, or twice or nearly three times as many where rows are short or two to four thousand columns (65536 x 512: 41 us with 2048, 45 with 1024;
    // 16384 x 4096: 87 with 2048, 96 with 768; 4000 x 8192: 40 with 256, 47 with 1024; 30000 x 2000: 73 with 1024, 75 with 2048)
    const int64_t most = (a.d <= 512 ? 2048 : (a.d <= 1024 ? 768 : (a.d <= 2048 ? 1024 : (a.d <= 4096 ? 2048 : 256)))) * (int64_t)teams;
    a.chunk = (a.rows + most - 1) / most;
    const int64_t blocks = ((a.rows + a.chunk - 1) / a.chunk + teams - 1) / teams;
    const dim3 grid((unsigned)blocks), group(lanes == 64 ? 256 : lanes);
    if (a.d <= 512) hipLaunchKernelGGL((forward_kernel<T, FP8, 64, 1>), grid, group, 0, s, a);
    else if (a.d <= 1024) hipLaunchKernelGGL((forward_kernel<T, FP8, 64, 2>), grid, group, 0, s, a);
    else if (a.d <= 2048) hipLaunchKernelGGL((forward_kernel<T, FP8, 256, 1>), grid, group, 0, s, a);
    else if (a.d <= 4096) hipLaunchKernelGGL((forward_kernel<T, FP8, 256, 2>), grid, group, 0, s, a);
    else if (a.d <= 8192) hipLaunchKernelGGL((forward_kernel<T, FP8, 512, 2>), grid, group, 0, s, a);
    else hipLaunchKernelGGL((forward_kernel<T, FP8, 1024, 2>), grid, group, 0, s, a);
}

// Rows of a unit: as many units as are resident (16384 x 4096: 162 us with 256, 166 with 512), at most 64 rows to a team, whose sums are in fp32.
constexpr int64_t kChain = 64;
int64_t chunk_for(int64_t rows, int64_t per_gate, int64_t d) {
    const int lanes = lanes_backward(d);
    const int64_t teams = lanes == 64 ? 4 : 1, most = d > 2048 ? 256 : (d > 1024 ? 768 : (d > 512 ? 512 : 1024));
    int64_t chunk = (rows + most - 1) / most;
    if (chunk < teams) chunk = teams;
    if (chunk > kChain * teams) chunk = kChain * teams;
    return chunk < per_gate ? chunk : (per_gate < 1 ? 1 : per_gate);
}
int64_t units_for(int64_t rows, int64_t per_gate, int64_t d) {
    if (rows == 0) return 0;
    const int64_t chunk = chunk_for(rows, per_gate, d);
    return rows / per_gate * ((per_gate + chunk - 1) / chunk);
}

template <typename T>
void launch_backward(const Backward& a, int64_t units, hipStream_t s) {
    const int lanes = lanes_backward(a.d);
    const dim3 grid((unsigned)units), group(lanes == 64 ? 256 : lanes);
    if (a.d > kMostKept) hipLaunchKernelGGL((backward_long_kernel<T>), grid, dim3(1024), 0, s, a);
    else if (a.d <= 512) hipLaunchKernelGGL((backward_kernel<T, 64, 1>), grid, group, 0, s, a);
    else if (a.d <= 1024) hipLaunchKernelGGL((backward_kernel<T, 64, 2>), grid, group, 0, s, a);
    else if (a.d <= 2048) hipLaunchKernelGGL((backward_kernel<T, 256, 1>), grid, group, 0, s, a);
    else if (a.d <= 4096) hipLaunchKernelGGL((backward_kernel<T, 512, 1>), grid, group, 0, s, a);
    else if (a.d <= 8192) hipLaunchKernelGGL((backward_kernel<T, 512, 2>), grid, group, 0, s, a);
    else hipLaunchKernelGGL((backward_kernel<T, 1024, 2>), grid, group, 0, s, a);
}

bool there(const void* p, int32_t dtype) { return p != nullptr && aligned(p, (uintptr_t)dtype_bytes(dtype)); }
const char* shape_refused(int32_t dtype, int32_t post_dtype, int32_t w_dtype, int64_t rows, int64_t d, const void* gate, int32_t gate_dtype, int64_t gates, int64_t gate_pitch, double scale) {
    if (!dtype_ok(dtype) || !dtype_ok(post_dtype) || !dtype_ok(w_dtype) || rows < 0 || rows >= int64_t(1) << 31 || d < 1 || d >= kMostColumns)
        return "block norm: types of the enumeration, rows from zero to 2^31, 1 <= d < 2^24";
    if (!std::isfinite(scale) || !std::isfinite((float)scale)) return "block norm: a finite scale";
    if (gate != nullptr && (!there(gate, gate_dtype) || !dtype_ok(gate_dtype) || gates < 1 || rows % gates != 0 || (gates > 1 && gate_pitch < d)))
        return "block norm: a gate of a type of the enumeration, as many rows to each, pitch >= d";
    return nullptr;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

ssgd_status ssgd_block_norm(const void* o, int64_t o_pitch, const void* s, int64_t s_pitch, const void* post_weight, int32_t post_dtype, const void* weight, int32_t weight_dtype,
                            const void* gate, int32_t gate_dtype, int64_t gates, int64_t gate_pitch, double scale, double eps, int32_t dtype, int64_t rows, int64_t d, void* sum, int64_t sum_pitch,
                            void* y, int64_t y_pitch, void* values, void* scales, float* rstd_o, float* rstd, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        if (const char* why = shape_refused(dtype, post_dtype, weight_dtype, rows, d, gate, gate_dtype, gates, gate_pitch, scale)) return op_fail(SSGD_EINVAL, why);
        if (!(eps >= 0) || !std::isfinite(eps)) return op_fail(SSGD_EINVAL, "block norm: eps of zero or more");
        if (rows == 0) return SSGD_OK;
        if (!there(o, dtype) || !there(s, dtype) || !there(post_weight, post_dtype) || !there(weight, weight_dtype) || !there(sum, dtype) || !there(rstd_o, SSGD_F32) || !there(rstd, SSGD_F32) ||
            o_pitch < d || s_pitch < d || sum_pitch < d)
            return op_fail(SSGD_EINVAL, "block norm: o, s, both weights, sum and both rstd, pitch >= d");
        if ((y == nullptr) == (values == nullptr) || (values == nullptr) != (scales == nullptr)) return op_fail(SSGD_EINVAL, "block norm: either y, or values and scales");
        if (y != nullptr && (!there(y, dtype) || y_pitch < d)) return op_fail(SSGD_EINVAL, "block norm: y, pitch >= d");
        if (values != nullptr && (!aligned(values, 16) || !aligned(scales, 16))) return op_fail(SSGD_EINVAL, "block norm: values and scales are 16-byte aligned");
        Forward a{};
        a.o = o; a.s = s; a.post = post_weight; a.w = weight; a.gate = gate; a.sum = sum; a.y = y;
        a.values = static_cast<uint8_t*>(values); a.scales = static_cast<uint8_t*>(scales); a.rstd_o = rstd_o; a.rstd = rstd;
        a.rows = rows; a.per_gate = gate != nullptr ? rows / gates : rows; a.o_pitch = o_pitch; a.s_pitch = s_pitch; a.sum_pitch = sum_pitch; a.y_pitch = y_pitch; a.gate_pitch = gate_pitch;
        a.row_bytes = mx_row_bytes(SSGD_MX_FP8, d); a.scale_bytes = mx_padded(d) / kMxBlock;
        a.d = (int32_t)d; a.post_bf16 = post_dtype == SSGD_BF16; a.w_bf16 = weight_dtype == SSGD_BF16; a.gate_bf16 = gate_dtype == SSGD_BF16; a.scale = scale; a.eps = eps; a.per_column = 1.0 / (double)d;
        const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        if (dtype == SSGD_F32) { if (values) launch_forward<float, true>(a, stream); else launch_forward<float, false>(a, stream); }
        else { if (values) launch_forward<bf16_t, true>(a, stream); else launch_forward<bf16_t, false>(a, stream); }
        return op_hip(hipGetLastError(), "block norm");
    });
}

int64_t ssgd_block_norm_work_floats(int64_t rows, int64_t d, int64_t gates) {
    if (rows < 0 || rows >= int64_t(1) << 31 || d < 1 || d >= kMostColumns || gates < 1 || rows % gates != 0) return -1;
    return 2 * units_for(rows, rows / gates, d) * d;
}

ssgd_status ssgd_block_norm_backward(const void* dy, int64_t dy_pitch, const void* o, int64_t o_pitch, const void* sum, int64_t sum_pitch, const void* post_weight, int32_t post_dtype,
                                     const void* weight, int32_t weight_dtype, const void* gate, int32_t gate_dtype, int64_t gates, int64_t gate_pitch, double scale, const float* rstd_o,
                                     const float* rstd, const void* dsum, int64_t dsum_pitch, int32_t dtype, int64_t rows, int64_t d, void* grad_o, int64_t grad_o_pitch, void* grad_s,
                                     int64_t grad_s_pitch, float* dpost, float* dweight, float* dgate, float* work, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        if (const char* why = shape_refused(dtype, post_dtype, weight_dtype, rows, d, gate, gate_dtype, gates, gate_pitch, scale)) return op_fail(SSGD_EINVAL, why);
        if ((dpost != nullptr) != (dweight != nullptr) || (dgate != nullptr && (gate == nullptr || dpost == nullptr))) return op_fail(SSGD_EINVAL, "block norm backward: the weights' gradients go together, a gate's with them");
        if (dpost != nullptr && (!aligned(dpost, 4) || !aligned(dweight, 4) || !aligned(dgate, 4) || (rows > 0 && (!work || !aligned(work, 16)))))
            return op_fail(SSGD_EINVAL, "block norm backward: the weights' gradients need a 16-byte aligned work area");
        const int64_t per_gate = gate != nullptr ? rows / gates : rows;
        const int64_t units = units_for(rows, per_gate, d), chunk = chunk_for(rows, per_gate, d);
        if (rows > 0) {
            if (!there(dy, dtype) || !there(o, dtype) || !there(sum, dtype) || !there(rstd_o, SSGD_F32) || !there(rstd, SSGD_F32) || !there(grad_o, dtype) || !there(grad_s, dtype) || dy_pitch < d ||
                o_pitch < d || sum_pitch < d || grad_o_pitch < d || grad_s_pitch < d)
                return op_fail(SSGD_EINVAL, "block norm backward: dy, o, sum, both rstd and the gradients of o and s, pitch >= d");
            if (dsum != nullptr && (!there(dsum, dtype) || dsum_pitch < d)) return op_fail(SSGD_EINVAL, "block norm backward: dsum, pitch >= d");
            if (units > kMostBlocks / 2) return op_fail(SSGD_EINVAL, "block norm backward: too many gates");
        }
        if ((rows > 0 || dpost != nullptr) && (!there(post_weight, post_dtype) || !there(weight, weight_dtype))) return op_fail(SSGD_EINVAL, "block norm backward: both weights");
        const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        if (rows > 0) {
            Backward a{};
            a.dy = dy; a.o = o; a.sum = sum; a.post = post_weight; a.w = weight; a.gate = gate; a.dsum = dsum; a.rstd_o = rstd_o; a.rstd = rstd; a.grad_o = grad_o; a.grad_s = grad_s;
            a.dw_parts = dpost ? work : nullptr; a.s_parts = dpost ? work + units * d : nullptr;
            a.rows = rows; a.per_gate = per_gate; a.chunk = chunk; a.chunks = (per_gate + chunk - 1) / chunk;
            a.dy_pitch = dy_pitch; a.o_pitch = o_pitch; a.sum_pitch = sum_pitch; a.gate_pitch = gate_pitch; a.dsum_pitch = dsum_pitch; a.grad_o_pitch = grad_o_pitch; a.grad_s_pitch = grad_s_pitch;
            a.d = (int32_t)d; a.post_bf16 = post_dtype == SSGD_BF16; a.w_bf16 = weight_dtype == SSGD_BF16; a.gate_bf16 = gate_dtype == SSGD_BF16; a.scale = (float)scale; a.per_column = 1.0 / (double)d;
            if (dtype == SSGD_F32) launch_backward<float>(a, units, stream); else launch_backward<bf16_t>(a, units, stream);
        }
        ssgd_status st = op_hip(hipGetLastError(), "block norm backward");
        if (st == SSGD_OK && dpost != nullptr) {
            Sums a{};
            a.dw_parts = work; a.s_parts = work + units * d; a.post = post_weight; a.gate = gate; a.dw = dweight; a.dw_post = dpost; a.dgate = dgate;
            a.gates = gate != nullptr ? gates : 1; a.chunks = units / a.gates; a.gate_pitch = gate_pitch; a.dgate_pitch = d;
            a.d = (int32_t)d; a.post_bf16 = post_dtype == SSGD_BF16; a.gate_bf16 = gate_dtype == SSGD_BF16;
            a.slots = 1;
            while (a.slots < 64 && a.slots < a.gates) a.slots *= 2;
            hipLaunchKernelGGL(sums_kernel, dim3((unsigned)((d + 15) / 16), 2), dim3(1024), 0, stream, a);
            st = op_hip(hipGetLastError(), "block norm backward");
        }
        return st;
    });
}

}  // extern "C"
#pragma GCC visibility pop
