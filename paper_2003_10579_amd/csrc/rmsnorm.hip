// Root-mean-square norm of rows with the residual's addition, output as it is or microscaled in 8 bits, and its gradients.
//
//   s = x + residual (rounded to the rows' type: what the stream keeps is what is normalised, forward and backward)
//   rstd = (mean s^2 + eps)^(-1/2),  y = (s rstd) w
//   dx = rstd (g - xhat mean(g xhat)) + dsum,  g = dy w,  xhat = s rstd;    dw = sum over rows of dy xhat
//
// About 8 operations per element forward, 12 backward: bound by memory (16384 x 4096 in bf16: forward with 8-bit output 83 us, 5.7 TB/s; backward
// 107 us and its sums over workgroups 6, 4.8 TB/s in all; rows of 999, 8192 of them, 12.8 and 15.7 us, the latter without dsum).  A row stays in the registers of 64, 256 or 1024 threads, eight
// or sixteen columns each, between the sum of squares and the output, so it is read once; the threads go on to further rows with
// their part of w, and backward with their part of dw, kept.  Rows of more than 16384 columns are read a second time instead.
#include <cmath>

#include "column_sums.hpp"
#include "rows.hpp"

using namespace ssgd;

namespace {

constexpr int kMostKept = 16384;      // columns that fit the registers of 1024 threads
constexpr int64_t kMostColumns = int64_t(1) << 25;     // 16 to a workgroup of 1024 in the sums of dw: a launch ends at 2^32 threads

struct Forward {
    const void *x, *residual, *w;
    void *sum, *y;
    uint8_t *values, *scales;
    float* rstd;
    int64_t rows, x_pitch, residual_pitch, sum_pitch, y_pitch, row_bytes, scale_bytes;
    int32_t d, w_bf16;
    double eps;
};

struct Backward {
    const void *dy, *s, *w, *dsum;
    const float* rstd;
    void* dx;
    float* partial;          // [groups][d], nullptr: dw is not wanted
    int64_t rows, dy_pitch, s_pitch, dsum_pitch, dx_pitch, groups;
    int32_t d, w_bf16;
};

// Sum over the threads of a row: across lanes in fp64, so that all that is left of the order is a thread's own few terms.
template <int LANES>
__device__ __forceinline__ double team_sum(double x, double* part) {
    x = wave_sum(x);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0.0;
#pragma unroll
        for (int q = 0; q < LANES / 64; ++q) x += part[q];
        __syncthreads();
    }
    return x;
}

// Eight columns of the stream: the sum, rounded as it is stored, and stored.
template <typename T>
__device__ __forceinline__ void take_sum(const Forward& a, int64_t row, int col, float (&s)[8]) {
    load_vec<8>(static_cast<const T*>(a.x) + row * a.x_pitch + col, a.d - col, s);
    if (a.residual != nullptr) {
        float r[8];
        load_vec<8>(static_cast<const T*>(a.residual) + row * a.residual_pitch + col, a.d - col, r);
#pragma unroll
        for (int q = 0; q < 8; ++q) s[q] = as_stored(static_cast<const T*>(nullptr), s[q] + r[q]);
        store_vec<8>(static_cast<T*>(a.sum) + row * a.sum_pitch + col, a.d - col, s);
    }
}

template <typename T, bool FP8>
__device__ __forceinline__ void store_normed(const Forward& a, int64_t row, int col, int end, const float (&s)[8], float rstd, const float (&w)[8]) {
    float y[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) y[q] = (s[q] * rstd) * w[q];
    if constexpr (FP8) {
        uint32_t most = 0;
#pragma unroll
        for (int q = 0; q < 8; ++q) most = umax(most, magnitude(y[q]));
        const uint32_t byte = mx_scale_byte<SSGD_MX_FP8>(max_of_4(most));
        *reinterpret_cast<words2*>(a.values + row * a.row_bytes + col) = mx_pack_fp8(y, byte);
        if ((threadIdx.x & 3) == 0) a.scales[row * a.scale_bytes + col / kMxBlock] = (uint8_t)byte;
    } else {
        store_vec<8>(static_cast<T*>(a.y) + row * a.y_pitch + col, end - col, y);
    }
}

// 2^LOW <= x < 2^HIGH, from the upper word of x (constants of 64 bits would take scalar registers, and from 80 of them on a SIMD holds seven waves
// instead of eight: 4000 x 6001 in bf16 with 8-bit output 43 us instead of 32).
template <int LOW, int HIGH>
__device__ __forceinline__ bool between(double x) {
    return (uint32_t)(__builtin_bit_cast(uint64_t, x) >> 32) - ((1023u + LOW) << 20) < (uint32_t)(HIGH - LOW) << 20;
}
// Whether squares in fp32 have lost nothing that their sum shows: one past the range makes it infinite, and what those below the normal numbers
// lose (2^-149 each) is far below 2^-100.  Otherwise they are taken again in fp64 (rows of zeros too, which have nothing to lose).
__device__ __forceinline__ bool held(double squares) { return between<-100, 127>(squares); }
__device__ __forceinline__ float inverse_root(double squares, const Forward& a) {
    const double mean = squares / a.d, all = mean + a.eps;
    if (between<-120, 127>(all)) return 1.0f / sqrtf((float)mean + (float)a.eps);
    return (float)(1.0 / sqrt(all));
}

// (four waves to a SIMD: sixteen fp32 columns a thread with 8-bit output are two registers above what that leaves)
template <typename T, bool FP8, int LANES, int NV>
__global__ __launch_bounds__(LANES == 64 ? 256 : LANES, 4) void forward_kernel(Forward a) {
    constexpr int kRows = LANES == 64 ? 4 : 1;         // teams of a workgroup
    constexpr bool kShort = LANES == 64 && NV == 1;
    __shared__ double part[LANES / 64];
    const int lane = threadIdx.x & (LANES - 1);
    const int64_t team = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES, teams = (int64_t)gridDim.x * kRows;
    const int end = FP8 ? (int)mx_padded(a.d) : a.d;
    // Threads whose columns are not the row's last ones know that there are eight (kernels with NV > 1 have rows that long).
    auto col_of = [&](int v) { return (v * LANES + lane) * 8; };
    auto end_of = [&](int v) { return v < NV - 1 ? col_of(v) + 8 : a.d; };
    Eight<T> next_x[NV], next_r[NV];
    auto load = [&](int64_t row) {
        if (row >= a.rows) return;
#pragma unroll
        for (int v = 0; v < NV; ++v) read<kShort>(next_x[v], a.x, row, a.x_pitch, col_of(v), end_of(v), a.d);
        if (a.residual != nullptr) {
#pragma unroll
            for (int v = 0; v < NV; ++v) read<kShort>(next_r[v], a.residual, row, a.residual_pitch, col_of(v), end_of(v), a.d);
        }
    };
    // (the next row's, while a row's sum is taken: fp32 16384 x 4096 197 us instead of 200; threads of 1024 have no registers for it)
    constexpr bool kAhead = LANES < 1024;
    if constexpr (kAhead) load(team);
    float w[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v) load_weight(a.w, a.w_bf16, col_of(v), end_of(v) - col_of(v), w[v]);
    for (int64_t row = team; row < a.rows; row += teams) {
        if constexpr (!kAhead) load(row);
        float s[NV][8];
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) numbers<kShort>(next_x[v], col_of(v), end_of(v), a.d, s[v]);
        if (a.residual != nullptr) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float r[8];
                numbers<kShort>(next_r[v], col_of(v), end_of(v), a.d, r);
#pragma unroll
                for (int q = 0; q < 8; ++q) s[v][q] = as_stored(static_cast<const T*>(nullptr), s[v][q] + r[q]);
            }
        }
        if constexpr (kAhead) load(row + teams);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int q = 0; q < 8; ++q) sum += s[v][q] * s[v][q];
        double squares = team_sum<LANES>((double)sum, part);
        if (!held(squares)) {          // (the whole team alike)
            double wide = 0.0;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int q = 0; q < 8; ++q) wide += (double)s[v][q] * (double)s[v][q];
            squares = team_sum<LANES>(wide, part);
        }
        const float rstd = inverse_root(squares, a);
        if (lane == 0) a.rstd[row] = rstd;
        // (s may go where x or the residual were: the threads have read theirs, each the row's last columns too, before they met for the sum)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = col_of(v);
            if (a.residual != nullptr) store_vec<8>(static_cast<T*>(a.sum) + row * a.sum_pitch + col, end_of(v) - col, s[v]);
            if (v < NV - 1 || col < end) store_normed<T, FP8>(a, row, col, end_of(v), s[v], rstd, w[v]);
        }
    }
}

// Rows that registers do not hold: a second read, of the sum (its own threads have written it) or of x (2048 x 20000 in bf16: 79 us, 3.6 TB/s).
template <typename T, bool FP8>
__global__ __launch_bounds__(1024) void forward_long_kernel(Forward a) {
    __shared__ double part[16];
    const int64_t end = FP8 ? mx_padded(a.d) : (int64_t)a.d;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        double sum = 0.0;
        for (int64_t col = threadIdx.x * 8; col < a.d; col += 8192) {
            float s[8];
            take_sum<T>(a, row, (int)col, s);
            float few = 0.0f;
#pragma unroll
            for (int q = 0; q < 8; ++q) few += s[q] * s[q];
            sum += few;
        }
        auto again = [&](int64_t col, float (&s)[8]) {
            if (a.residual != nullptr) load_vec<8>(static_cast<const T*>(a.sum) + row * a.sum_pitch + col, a.d - col, s);
            else load_vec<8>(static_cast<const T*>(a.x) + row * a.x_pitch + col, a.d - col, s);
        };
        double squares = team_sum<1024>(sum, part);
        if (!held(squares)) {
            sum = 0.0;
            for (int64_t col = threadIdx.x * 8; col < a.d; col += 8192) {
                float s[8];
                again(col, s);
#pragma unroll
                for (int q = 0; q < 8; ++q) sum += (double)s[q] * (double)s[q];
            }
            squares = team_sum<1024>(sum, part);
        }
        const float rstd = inverse_root(squares, a);
        if (threadIdx.x == 0) a.rstd[row] = rstd;
        for (int64_t col = threadIdx.x * 8; col < end; col += 8192) {
            float s[8], w[8];
            again(col, s);
            load_weight(a.w, a.w_bf16, (int)col, a.d - (int)col, w);
            store_normed<T, FP8>(a, row, (int)col, a.d, s, rstd, w);
        }
    }
}

template <typename T, bool AT_ONCE>
__device__ __forceinline__ void store_dx(const Backward& a, int64_t row, int64_t col, int64_t end, const float (&dy)[8], const float (&xhat)[8], const float (&w)[8], float rstd,
                                         float c) {
    float dx[8], more[8];
    if (a.dsum != nullptr) {
        Eight<T> x;        // (dx may go where dsum was: a thread reads no more than it writes)
        const T* from = static_cast<const T*>(a.dsum) + row * a.dsum_pitch;
        x.template load_own<AT_ONCE>(from, col, end);
        x.numbers(more);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        dx[q] = rstd * (dy[q] * w[q] - xhat[q] * c);
        if (a.dsum != nullptr) dx[q] += more[q];
    }
    store_vec<8>(static_cast<T*>(a.dx) + row * a.dx_pitch + col, end - col, dx);
}

// MANY: teams that take more than kChain rows.  After so many, a thread's fp32 sums of dw move to fp64 ones, in LDS (a kernel of its own, since those
// are up to 128 KB of a CU's and few calls have the rows: more than 64 for each of 256 to 4096 teams).
constexpr int kChain = 64;
template <typename T, int LANES, int NV, bool MANY>
__global__ __launch_bounds__(LANES == 64 ? 256 : LANES) void backward_kernel(Backward a) {
    constexpr int kRows = LANES == 64 ? 4 : 1;
    __shared__ double part[LANES / 64];
    __shared__ double wide[MANY ? NV * 8 : 1][MANY ? LANES * kRows : 1];
    __shared__ float dw_of[kRows > 1 ? kRows - 1 : 1][kRows > 1 ? LANES * NV * 8 : 1];
    const int lane = threadIdx.x & (LANES - 1), team = threadIdx.x / LANES;
    constexpr bool kShort = LANES == 64 && NV == 1;
    // Sixteen columns to each of 1024 threads fill their registers: they read as load_own does, one place after the other (4000 x 16000 in bf16: 116 us;
    // as the others do, 171).
    constexpr bool kWide = LANES < 1024 || NV == 1;
    // Threads whose columns are not the row's last ones know that there are eight (kernels with NV > 1 have rows that long).
    auto col_of = [&](int v) { return (v * LANES + lane) * 8; };
    auto end_of = [&](int v) { return v < NV - 1 && kWide ? col_of(v) + 8 : a.d; };
    float w[NV][8], dw[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        load_weight(a.w, a.w_bf16, col_of(v), end_of(v) - col_of(v), w[v]);
#pragma unroll
        for (int q = 0; q < 8; ++q) dw[v][q] = 0.0f;
    }
    // The next row's dy and s are on their way while a row's sum is taken (16384 x 1500: 60 us instead of 74; threads of 1024 have no registers
    // for it, 4000 x 16000: 126 us instead of 119).  (dx may go where dy was, as s in the forward pass.)
    constexpr bool kAhead = LANES < 1024;
    Eight<T> next_dy[NV], next_s[NV];
    float next_rstd = 0.0f;
    auto load = [&](int64_t row) {
        if (row >= a.rows) return;
        next_rstd = a.rstd[row];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (kWide) {
                read<kShort>(next_dy[v], a.dy, row, a.dy_pitch, col_of(v), end_of(v), a.d);
                read<kShort>(next_s[v], a.s, row, a.s_pitch, col_of(v), end_of(v), a.d);
            } else {
                next_dy[v].template load_own<false>(static_cast<const T*>(a.dy) + row * a.dy_pitch, col_of(v), a.d);
                next_s[v].template load_own<false>(static_cast<const T*>(a.s) + row * a.s_pitch, col_of(v), a.d);
            }
        }
    };
    const int64_t first = (int64_t)blockIdx.x * kRows + team, step = a.groups * kRows;
    // (a thread's own places: no other thread reads or writes them)
    auto each_sum = [&](auto f) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int q = 0; q < 8; ++q) f(wide[v * 8 + q][threadIdx.x], dw[v][q]);
    };
    if constexpr (MANY) each_sum([](double& sum, float&) { sum = 0.0; });
    int taken = 0;
    if constexpr (kAhead) load(first);
    for (int64_t row = first; row < a.rows; row += step) {
        if constexpr (MANY) {
            if (taken++ == kChain) {
                each_sum([](double& sum, float& x) { sum += x; x = 0.0f; });
                taken = 1;
            }
        }
        if constexpr (!kAhead) load(row);
        float dy[NV][8], xhat[NV][8];
        const float rstd = next_rstd;
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (kWide) {
                numbers<kShort>(next_dy[v], col_of(v), end_of(v), a.d, dy[v]);
                numbers<kShort>(next_s[v], col_of(v), end_of(v), a.d, xhat[v]);
            } else {
                next_dy[v].numbers(dy[v]);
                next_s[v].numbers(xhat[v]);
            }
        }
        if constexpr (kAhead) load(row + step);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                xhat[v][q] *= rstd;
                sum += dy[v][q] * w[v][q] * xhat[v][q];
                dw[v][q] += dy[v][q] * xhat[v][q];
            }
        }
        const float c = (float)(team_sum<LANES>((double)sum, part) / a.d);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if ((v < NV - 1 && kWide) || col_of(v) < a.d) store_dx<T, kWide>(a, row, col_of(v), end_of(v), dy[v], xhat[v], w[v], rstd, c);
        }
    }
    if (a.partial == nullptr) return;
    if constexpr (MANY) each_sum([](double& sum, float& x) { x = (float)(sum + x); });
    if constexpr (kRows > 1) {
        // the rows of a workgroup's waves first, in their order
        if (team > 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v) store_vec<8>(&dw_of[team - 1][(v * LANES + lane) * 8], 8, dw[v]);
        }
        __syncthreads();
        if (team > 0) return;
#pragma unroll
        for (int t = 0; t < kRows - 1; ++t)
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float x[8];
                load_vec<8>(&dw_of[t][(v * LANES + lane) * 8], 8, x);
#pragma unroll
                for (int q = 0; q < 8; ++q) dw[v][q] += x[q];
            }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        store_vec<8>(a.partial + (int64_t)blockIdx.x * a.d + col_of(v), end_of(v) - col_of(v), dw[v]);
    }
}

// The same backward: dy and s twice, and the workgroup's partial sum of dw read and written for every row (2048 x 20000 in bf16: 153 us, 2.1 TB/s of
// what has to be moved).  Behind the partial sums lie fp64 ones, where there are more than kChain rows to a workgroup: every kChain rows they take
// what the fp32 one holds, and the last row leaves their sum, rounded, in its place.
template <typename T>
__global__ __launch_bounds__(1024) void backward_long_kernel(Backward a) {
    __shared__ double part[16];
    const bool many = a.rows > a.groups * kChain;
    double* wide = reinterpret_cast<double*>(a.partial + a.groups * a.d) + (int64_t)blockIdx.x * a.d;
    int taken = 0;
    bool begun = false;        // the fp64 sums hold something
    for (int64_t row = blockIdx.x; row < a.rows; row += a.groups) {
        const float rstd = a.rstd[row];
        const bool last = row + a.groups >= a.rows, first = taken == 0, over = many && (last || taken == kChain - 1);
        double sum = 0.0;
        for (int64_t col = threadIdx.x * 8; col < a.d; col += 8192) {
            float dy[8], s[8], w[8];
            load_vec<8>(static_cast<const T*>(a.dy) + row * a.dy_pitch + col, a.d - col, dy);
            load_vec<8>(static_cast<const T*>(a.s) + row * a.s_pitch + col, a.d - col, s);
            load_weight(a.w, a.w_bf16, (int)col, a.d - (int)col, w);
            float few = 0.0f;
#pragma unroll
            for (int q = 0; q < 8; ++q) few += dy[q] * w[q] * (s[q] * rstd);
            sum += few;
        }
        const float c = (float)(team_sum<1024>(sum, part) / a.d);
        for (int64_t col = threadIdx.x * 8; col < a.d; col += 8192) {
            float dy[8], s[8], w[8];
            load_vec<8>(static_cast<const T*>(a.dy) + row * a.dy_pitch + col, a.d - col, dy);
            load_vec<8>(static_cast<const T*>(a.s) + row * a.s_pitch + col, a.d - col, s);
            load_weight(a.w, a.w_bf16, (int)col, a.d - (int)col, w);
#pragma unroll
            for (int q = 0; q < 8; ++q) s[q] *= rstd;
            store_dx<T, false>(a, row, col, a.d, dy, s, w, rstd, c);
            if (a.partial == nullptr) continue;
            float* to = a.partial + (int64_t)blockIdx.x * a.d + col;
            float dw[8];
            if (first) {
#pragma unroll
                for (int q = 0; q < 8; ++q) dw[q] = 0.0f;
            } else load_vec<8>(to, a.d - col, dw);
#pragma unroll
            for (int q = 0; q < 8; ++q) dw[q] += dy[q] * s[q];
            if (over) {
                for (int q = 0; q < 8 && col + q < a.d; ++q) {
                    const double all = (begun ? wide[col + q] : 0.0) + dw[q];
                    if (last) dw[q] = (float)all; else wide[col + q] = all;
                }
            }
            if (last || !over) store_vec<8>(to, a.d - col, dw);
        }
        if (over) { taken = 0; begun = true; } else ++taken;
    }
}

int lanes_for(int64_t d) { return d <= 1024 ? 64 : (d <= 4096 ? 256 : 1024); }

template <typename T, bool FP8>
void launch_forward(const Forward& a, hipStream_t s) {
    const int lanes = lanes_for(a.d), rows = lanes == 64 ? 4 : 1;
    int64_t blocks = (a.rows + rows - 1) / rows;
    const int64_t most = lanes == 1024 ? 512 : 2048;     // as many as are resident: the next rows find w in registers
    if (blocks > most) blocks = most;
    const dim3 grid((unsigned)blocks), group(lanes == 64 ? 256 : lanes);
    if (a.d > kMostKept) hipLaunchKernelGGL((forward_long_kernel<T, FP8>), grid, dim3(1024), 0, s, a);
    else if (a.d <= 512) hipLaunchKernelGGL((forward_kernel<T, FP8, 64, 1>), grid, group, 0, s, a);
    else if (a.d <= 1024) hipLaunchKernelGGL((forward_kernel<T, FP8, 64, 2>), grid, group, 0, s, a);
    else if (a.d <= 2048) hipLaunchKernelGGL((forward_kernel<T, FP8, 256, 1>), grid, group, 0, s, a);
    else if (a.d <= 4096) hipLaunchKernelGGL((forward_kernel<T, FP8, 256, 2>), grid, group, 0, s, a);
    else if (a.d <= 8192) hipLaunchKernelGGL((forward_kernel<T, FP8, 1024, 1>), grid, group, 0, s, a);
    else hipLaunchKernelGGL((forward_kernel<T, FP8, 1024, 2>), grid, group, 0, s, a);
}

// Workgroups, each with a partial sum of dw that is written and read once more: as many as are resident.  (16384 x 4096: 107 us with 768, 113 with
// 512, 128 with 1024; 16384 x 1500: 60 with 1024, 69 with 768; 4000 x 16000: 119 with 256, 125 with 512.)
int64_t groups_for(int64_t rows, int64_t d) {
    const int lanes = lanes_for(d);
    const bool two = (d > 512 && d <= 1024) || (d > 2048 && d <= 4096);      // sixteen columns a thread
    const int64_t rows_each = lanes == 64 ? 4 : 1, most = lanes == 1024 ? 256 : (two ? 768 : 1024), groups = (rows + rows_each - 1) / rows_each;
    return groups < most ? groups : most;
}

// Whether a team takes more rows than it adds in fp32.
bool many_rows(int64_t rows, int64_t d) { return rows > groups_for(rows, d) * (lanes_for(d) == 64 ? 4 : 1) * kChain; }

template <typename T, bool MANY>
void launch_backward(const Backward& a, hipStream_t s) {
    const int lanes = lanes_for(a.d);
    const dim3 grid((unsigned)a.groups), group(lanes == 64 ? 256 : lanes);
    if (a.d > kMostKept) hipLaunchKernelGGL((backward_long_kernel<T>), grid, dim3(1024), 0, s, a);
    else if (a.d <= 512) hipLaunchKernelGGL((backward_kernel<T, 64, 1, MANY>), grid, group, 0, s, a);
    else if (a.d <= 1024) hipLaunchKernelGGL((backward_kernel<T, 64, 2, MANY>), grid, group, 0, s, a);
    else if (a.d <= 2048) hipLaunchKernelGGL((backward_kernel<T, 256, 1, MANY>), grid, group, 0, s, a);
    else if (a.d <= 4096) hipLaunchKernelGGL((backward_kernel<T, 256, 2, MANY>), grid, group, 0, s, a);
    else if (a.d <= 8192) hipLaunchKernelGGL((backward_kernel<T, 1024, 1, MANY>), grid, group, 0, s, a);
    else hipLaunchKernelGGL((backward_kernel<T, 1024, 2, MANY>), grid, group, 0, s, a);
}

bool shape_ok(int32_t dtype, int32_t w_dtype, int64_t rows, int64_t d) {
    return dtype_ok(dtype) && dtype_ok(w_dtype) && rows >= 0 && rows < (int64_t(1) << 40) && d >= 1 && d < kMostColumns;
}
bool there(const void* p, int32_t dtype) { return p != nullptr && aligned(p, (uintptr_t)dtype_bytes(dtype)); }

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

ssgd_status ssgd_rmsnorm(const void* x, int64_t x_pitch, const void* residual, int64_t residual_pitch, const void* weight, int32_t dtype, int32_t weight_dtype,
                         int64_t rows, int64_t d, double eps, void* sum, int64_t sum_pitch, void* y, int64_t y_pitch, void* values, void* scales, float* rstd,
                         void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        if (!shape_ok(dtype, weight_dtype, rows, d)) return op_fail(SSGD_EINVAL, "rmsnorm: types of the enumeration, rows of zero or more, 1 <= d < 2^25");
        if (!(eps >= 0) || !std::isfinite(eps)) return op_fail(SSGD_EINVAL, "rmsnorm: eps of zero or more");
        if (rows == 0) return SSGD_OK;
        if (!there(x, dtype) || !there(weight, weight_dtype) || !there(rstd, SSGD_F32) || x_pitch < d) return op_fail(SSGD_EINVAL, "rmsnorm: x, weight and rstd, pitch >= d");
        if ((residual != nullptr) != (sum != nullptr)) return op_fail(SSGD_EINVAL, "rmsnorm: a residual and its sum go together");
        if (residual != nullptr && (!there(residual, dtype) || !there(sum, dtype) || residual_pitch < d || sum_pitch < d)) return op_fail(SSGD_EINVAL, "rmsnorm: residual and sum, pitch >= d");
        if ((y != nullptr) == (values != nullptr) || (values != nullptr) != (scales != nullptr)) return op_fail(SSGD_EINVAL, "rmsnorm: either y, or values and scales");
        if (y != nullptr && (!there(y, dtype) || y_pitch < d)) return op_fail(SSGD_EINVAL, "rmsnorm: y, pitch >= d");
        if (values != nullptr && (!aligned(values, 16) || !aligned(scales, 16))) return op_fail(SSGD_EINVAL, "rmsnorm: values and scales are 16-byte aligned");
        Forward a{};
        a.x = x; a.residual = residual; a.w = weight; a.sum = sum; a.y = y;
        a.values = static_cast<uint8_t*>(values); a.scales = static_cast<uint8_t*>(scales); a.rstd = rstd;
        a.rows = rows; a.x_pitch = x_pitch; a.residual_pitch = residual_pitch; a.sum_pitch = sum_pitch; a.y_pitch = y_pitch;
        a.row_bytes = mx_row_bytes(SSGD_MX_FP8, d); a.scale_bytes = mx_padded(d) / kMxBlock;
        a.d = (int32_t)d; a.w_bf16 = weight_dtype == SSGD_BF16; a.eps = eps;
        const hipStream_t s = static_cast<hipStream_t>(hip_stream);
        if (dtype == SSGD_F32) { if (values) launch_forward<float, true>(a, s); else launch_forward<float, false>(a, s); }
        else { if (values) launch_forward<bf16_t, true>(a, s); else launch_forward<bf16_t, false>(a, s); }
        return op_hip(hipGetLastError(), "rmsnorm");
    });
}

int64_t ssgd_rmsnorm_work_floats(int64_t rows, int64_t d) {
    if (!shape_ok(SSGD_F32, SSGD_F32, rows, d)) return -1;
    // (a sum to a workgroup, and where rows are read twice and many, one in fp64 too)
    return groups_for(rows, d) * d * (d > kMostKept && many_rows(rows, d) ? 3 : 1);
}

ssgd_status ssgd_rmsnorm_backward(const void* dy, int64_t dy_pitch, const void* s, int64_t s_pitch, const void* weight, int32_t dtype, int32_t weight_dtype,
                                  const float* rstd, const void* dsum, int64_t dsum_pitch, int64_t rows, int64_t d, void* dx, int64_t dx_pitch, float* dweight,
                                  float* work, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        if (!shape_ok(dtype, weight_dtype, rows, d)) return op_fail(SSGD_EINVAL, "rmsnorm backward: types of the enumeration, rows of zero or more, 1 <= d < 2^25");
        if (dweight != nullptr && (!aligned(dweight, 4) || (rows > 0 && (!work || !aligned(work, 16))))) return op_fail(SSGD_EINVAL, "rmsnorm backward: dweight needs a 16-byte aligned work area");
        if (rows > 0) {
            if (!there(dy, dtype) || !there(s, dtype) || !there(weight, weight_dtype) || !there(rstd, SSGD_F32) || !there(dx, dtype) || dy_pitch < d || s_pitch < d || dx_pitch < d)
                return op_fail(SSGD_EINVAL, "rmsnorm backward: dy, s, weight, rstd and dx, pitch >= d");
            if (dsum != nullptr && (!there(dsum, dtype) || dsum_pitch < d)) return op_fail(SSGD_EINVAL, "rmsnorm backward: dsum, pitch >= d");
        }
        Backward a{};
        a.dy = dy; a.s = s; a.w = weight; a.dsum = dsum; a.rstd = rstd; a.dx = dx; a.partial = dweight ? work : nullptr;
        a.rows = rows; a.dy_pitch = dy_pitch; a.s_pitch = s_pitch; a.dsum_pitch = dsum_pitch; a.dx_pitch = dx_pitch; a.groups = groups_for(rows, d);
        a.d = (int32_t)d; a.w_bf16 = weight_dtype == SSGD_BF16;
        const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        if (rows > 0) {
            // (without dw nothing is added up over rows)
            const bool many = dweight != nullptr && many_rows(rows, d);
            if (dtype == SSGD_F32) { if (many) launch_backward<float, true>(a, stream); else launch_backward<float, false>(a, stream); }
            else { if (many) launch_backward<bf16_t, true>(a, stream); else launch_backward<bf16_t, false>(a, stream); }
        }
        ssgd_status st = op_hip(hipGetLastError(), "rmsnorm backward");
        if (st == SSGD_OK && dweight != nullptr) {
            launch_column_sums(work, a.groups, d, dweight, stream);
            st = op_hip(hipGetLastError(), "rmsnorm backward");
        }
        return st;
    });
}

}  // extern "C"
#pragma GCC visibility pop
