// Product of microscaled matrices on the matrix unit: C[m][n] = sum_k A[m][k] B[n][k], A in 4 or 8 bits, B in 4, fp32 accumulation.
//
// One instruction contracts 16 x 16 x 128, each lane with a row (lane % 16), the scale of its block of 32 columns (lane / 16) and, in
// 4 bits, that block's 16 bytes; in 8 bits bytes 16 g .. 16 g + 15 and the same 64 further on.  B's rows are the instruction's first
// operand and A's its second, so that a lane's four results are consecutive columns of a row of C.
//
// 8192^3 in 4 bits: 275 to 305 us (3.6 to 4.0 PFLOP/s; 228 on zeros, whose bits draw less power), of which the matrix instructions alone take 189, with the
// reads of their operands from LDS 214 and with the stores 235; in 8 by 4 bits 376 us (2.9 PFLOP/s; instructions 292).
//
// The kernels take what becomes of the results as a type, `Out`: To<T> stores them as they are (mx_matmul.hip), an epilogue goes on with them
// (mx_dense.hip).
#pragma once
#include <type_traits>

#include "ops.hpp"

namespace ssgd {
namespace {

typedef int ints8 __attribute__((ext_vector_type(8)));

struct Matrix { const uint8_t *values, *scales; int64_t rows, row_bytes, scale_bytes; };
struct Product {
    Matrix a, b;
    void* out;
    int64_t pitch;
    int32_t steps;          // of 128 columns
    int32_t tiles_m, tiles_n;
    int32_t part_steps;     // tiles: steps of a part of the contraction (blockIdx.y), `steps` where it is not split
    int64_t part_stride;    // elements between the results of two parts
};

// The scales are byte BYTE of their words.
template <int FA, int BYTE>
__device__ __forceinline__ f32x4 mfma(const ints8& b, const ints8& a, const f32x4& c, uint32_t scale_b, uint32_t scale_a) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 4, FA == SSGD_MX_FP4 ? 4 : 0, BYTE, (int)scale_b, BYTE, (int)scale_a);
}
// Byte g of four words, in order: a lane's scales of four steps of 128 columns from 16 bytes of a row of scales.
__device__ __forceinline__ uint32_t scales_of_four(const words4& w, int g) {
    const uint32_t pick = (uint32_t)g | (uint32_t)(4 + g) << 8;
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w.w, w.z, pick), __builtin_amdgcn_perm(w.y, w.x, pick), 0x05040100u);
}

__device__ __forceinline__ ints8 operand(const words4& lo) { return ints8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, 0, 0, 0, 0}; }
__device__ __forceinline__ ints8 operand(const words4& lo, const words4& hi) {
    return ints8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
}

template <typename T> struct To { using type = T; static constexpr bool kStores = true; };

template <typename T>
__device__ __forceinline__ void store_four(const Product& p, int64_t m, int64_t n, const f32x4& c) {
    if (m >= p.a.rows || n >= p.b.rows) return;
    const float x[4] = {c.x, c.y, c.z, c.w};
    store_vec<4>(static_cast<T*>(p.out) + m * p.pitch + n, p.b.rows - n, x);
}

template <typename T>
__device__ __forceinline__ void store_eight(const Product& p, int64_t m, int64_t n, const f32x4& c, const f32x4& d) {
    if (m >= p.a.rows || n >= p.b.rows) return;
    const float x[8] = {c.x, c.y, c.z, c.w, d.x, d.y, d.z, d.w};
    store_vec<8>(static_cast<T*>(p.out) + m * p.pitch + n, p.b.rows - n, x);
}

// ---- tiles ---------------------------------------------------------------------------------------------------------
typedef __attribute__((address_space(3))) uint32_t lds_word;
typedef const __attribute__((address_space(1))) uint32_t global_word;
// Global memory to LDS without registers: lane l's bytes go to `to` + 16 l.
__device__ __forceinline__ void copy16(const uint8_t* from, uint8_t* to) { __builtin_amdgcn_global_load_lds((global_word*)from, (lds_word*)to, 16, 0, 0); }

template <int VM> __device__ __forceinline__ void wait_and_meet() {
    static_assert(VM < 64, "the counter has six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((VM & 15) | ((VM >> 4) << 14) | (7 << 4));     // vmcnt(VM), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
// WM x WN waves, a tile of BM x BN.  A step is 128 columns: rows of A (64 or 128 bytes) and rows of B (64) in a stage of LDS, in which the
// 16-byte parts of a row change places by its number, so that the lanes that read one part of 16 rows meet in no bank.  Scales come for a
// group of steps at a time (four, with three stages three), 16 bytes of a row: four bytes of every row per step would be as many cache lines
// again as the values take.  They wait in registers from the first step of the group on, one word per row, so their place in LDS is free for
// the next ones behind the next meeting.
template <int FA, int BM, int BN, int WM, int WN, int STAGES, typename Out>
__global__ __launch_bounds__(64 * WM * WN) void tile_kernel(Product p, Out out) {
    constexpr int kWaves = WM * WN, kRowA = FA == SSGD_MX_FP4 ? 64 : 128, kRowB = 64;
    constexpr int kA = BM * kRowA, kB = BN * kRowB, kStage = kA + kB;
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int kLoadsA = kA / 1024 / kWaves, kLoadsB = kB / 1024 / kWaves, kLoads = kLoadsA + kLoadsB;
    static_assert(kLoadsA * 1024 * kWaves == kA && kLoadsB * 1024 * kWaves == kB && BM + BN <= 64 * kWaves, "every wave loads the same share");
    constexpr int kGroupSteps = STAGES == 3 ? 3 : 4;
    static_assert(STAGES == 3 || STAGES == 4, "a group ends at the stage it began with");
    // (arrays of their own: the compiler then sees that loads into one do not concern reads of another)
    __shared__ __attribute__((aligned(1024))) uint8_t stage0[kStage];
    __shared__ __attribute__((aligned(1024))) uint8_t stage1[kStage];
    __shared__ __attribute__((aligned(1024))) uint8_t stage2[kStage];
    __shared__ __attribute__((aligned(1024))) uint8_t stage3[STAGES > 3 ? kStage : 16];
    __shared__ __attribute__((aligned(1024))) uint8_t scales[64 * kWaves * 16];      // (a row of A or B to a thread, the last ones again where there are more threads)

    // Workgroups go to the XCDs in turn; each XCD takes tiles that lie together, in groups of 4 rows of tiles, so that its L2 holds what
    // they share.
    const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n, per_xcd = (tiles + kXcds - 1) / kXcds;
    const int64_t id = (int64_t)(blockIdx.x % kXcds) * per_xcd + blockIdx.x / kXcds;
    if (blockIdx.x / kXcds >= per_xcd || id >= tiles) return;
    constexpr int kGroup = 4;
    const int64_t group = id / (kGroup * (int64_t)p.tiles_n), in_group = id - group * kGroup * p.tiles_n;
    const int64_t height = p.tiles_m - group * kGroup < kGroup ? p.tiles_m - group * kGroup : kGroup;
    const int64_t m0 = (group * kGroup + in_group % height) * BM, n0 = in_group / height * BN;

    const int begin = (int)blockIdx.y * p.part_steps, steps = p.steps - begin < p.part_steps ? p.steps - begin : p.part_steps;
    if constexpr (Out::kStores) p.out = static_cast<typename Out::type*>(p.out) + blockIdx.y * p.part_stride;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (offsets from the tile's first row: 256 rows of less than 2^24 bytes)
    // (a tile past the last row of B, which some epilogues have for the padding of their outputs, multiplies that row)
    const int64_t b0 = Out::kStores || n0 < p.b.rows ? n0 : p.b.rows - 1;
    const uint8_t *a_values = p.a.values + m0 * p.a.row_bytes + (int64_t)begin * kRowA, *b_values = p.b.values + b0 * p.b.row_bytes + (int64_t)begin * kRowB;
    const uint32_t rows_a = (uint32_t)(p.a.rows - m0 < BM ? p.a.rows - m0 : BM), rows_b = (uint32_t)(p.b.rows - b0 < BN ? p.b.rows - b0 : BN);
    uint32_t from[kLoads];
#pragma unroll
    for (int q = 0; q < kLoadsA; ++q) {
        const uint32_t unit = (q * kWaves + wave) * 64 + lane, per = kRowA / 16, row = unit / per;
        const uint32_t part = (unit % per) ^ (FA == SSGD_MX_FP4 ? (row >> 1) & 3 : row & 7);
        from[q] = (row < rows_a ? row : rows_a - 1) * (uint32_t)p.a.row_bytes + part * 16;
    }
#pragma unroll
    for (int q = 0; q < kLoadsB; ++q) {
        const uint32_t unit = (q * kWaves + wave) * 64 + lane, row = unit / 4, part = (unit % 4) ^ ((row >> 3) & 3);
        from[kLoadsA + q] = (row < rows_b ? row : rows_b - 1) * (uint32_t)p.b.row_bytes + part * 16;
    }
    const uint8_t* scales_from;
    {
        const uint32_t row = threadIdx.x, in_a = row < rows_a ? row : rows_a - 1, in_b = row - BM < rows_b ? row - BM : rows_b - 1;
        scales_from = row < BM ? p.a.scales + (m0 + in_a) * p.a.scale_bytes + (int64_t)begin * 4 : p.b.scales + (b0 + in_b) * p.b.scale_bytes + (int64_t)begin * 4;
    }
    // Every call issues as many loads, so that they can be counted: past the last step the last one is loaded again, and not used.
    auto issue = [&](uint8_t* stage, int step) {
        const int k = step < steps ? step : steps - 1;
        const uint8_t *a = a_values + (int64_t)k * kRowA, *b = b_values + (int64_t)k * kRowB;
#pragma unroll
        for (int q = 0; q < kLoadsA; ++q) copy16(a + from[q], stage + (q * kWaves + wave) * 1024);
#pragma unroll
        for (int q = 0; q < kLoadsB; ++q) copy16(b + from[kLoadsA + q], stage + kA + (q * kWaves + wave) * 1024);
    };
    const int whole = steps / kGroupSteps;       // groups
    // Where 16 bytes from a group's first scale on would pass the end of the row, its last 16 bytes come instead; `first` is the place of the
    // group's first scale in them.  Rows of less than 16 bytes are put together at the start.
    auto first_of = [&](int f) { return f * kGroupSteps + 4 <= steps ? 0 : f * kGroupSteps + 4 - steps; };
    auto issue_scales = [&](int f) {
        const int at = f * kGroupSteps + 4 <= steps ? f * kGroupSteps * 4 : steps * 4 - 16;
        copy16(scales_from + (at > 0 ? at : 0), scales + wave * 1024);
    };

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int r16 = lane & 15, g = lane >> 4;
    // Rows of B: of two tiles of 16 that lie together, the first takes four of every eight and the second the others, so that a lane's results in both
    // are eight columns side by side.
    const int row_a = (wave / WN) * TM * 16 + r16, col = (wave % WN) * TN * 16, row_b = col + (r16 >> 2) * 8 + (r16 & 3);
    constexpr auto row_of = [](int j) { return j / 2 * 32 + j % 2 * 4; };
    // (rows of A 16 further on, and rows of B 4 or 32, have the same exchange of parts)
    const int at_a = FA == SSGD_MX_FP4 ? row_a * 64 + (g ^ ((row_a >> 1) & 3)) * 16 : row_a * 128 + (g ^ (row_a & 7)) * 16;
    const int at_b = kA + row_b * 64 + (g ^ ((row_b >> 3) & 3)) * 16;

    uint32_t sa[TM], sb[TN];
    auto read_scales = [&](int skipped) {
#pragma unroll
        for (int j = 0; j < TN; ++j) sb[j] = scales_of_four(*reinterpret_cast<const words4*>(scales + (BM + row_b + row_of(j)) * 16), g) >> (8 * skipped);
#pragma unroll
        for (int i = 0; i < TM; ++i) sa[i] = scales_of_four(*reinterpret_cast<const words4*>(scales + (row_a + i * 16) * 16), g) >> (8 * skipped);
    };
    auto contract = [&](const uint8_t* stage, auto byte) {
        ints8 a[TM], b[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) b[j] = operand(*reinterpret_cast<const words4*>(stage + at_b + row_of(j) * 64));
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            if constexpr (FA == SSGD_MX_FP4) a[i] = operand(*reinterpret_cast<const words4*>(stage + at_a + i * 16 * 64));
            else a[i] = operand(*reinterpret_cast<const words4*>(stage + at_a + i * 16 * 128), *reinterpret_cast<const words4*>(stage + (at_a ^ 64) + i * 16 * 128));
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = mfma<FA, decltype(byte)::value>(b[j], a[i], acc[i][j], sb[j], sa[i]);
    };
    constexpr std::integral_constant<int, 0> k0{};
    constexpr std::integral_constant<int, 1> k1{};
    constexpr std::integral_constant<int, 2> k2{};
    constexpr std::integral_constant<int, 3> k3{};

    if (steps >= 4) issue_scales(0);
    else {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = q >= 4 - steps ? *reinterpret_cast<const uint32_t*>(scales_from + (q - 4 + steps) * 4) : 0u;
        *reinterpret_cast<words4*>(scales + threadIdx.x * 16) = words4{w[0], w[1], w[2], w[3]};
    }
    issue(stage0, 0);
    issue(stage1, 1);
    if constexpr (STAGES > 3) issue(stage2, 2);
    // A stage is read when its own loads have arrived in every wave, and loaded again only behind the next meeting, when all have read it.
    // The counts are those of the loads issued after it: STAGES - 2 steps, and from the second step of a group on its successor's scales
    // until the steps issued with them are read.
    constexpr int kFlying = kLoads * (STAGES - 2);
    if (steps >= 4) {
        for (int f = 0; f < whole; ++f) {
            const int k = f * kGroupSteps;
            wait_and_meet<kFlying>();
            read_scales(first_of(f));
            issue(STAGES == 3 ? stage2 : stage3, k + STAGES - 1);
            contract(stage0, k0);
            wait_and_meet<kFlying>();
            issue(stage0, k + STAGES);
            issue_scales(f + 1);
            contract(stage1, k1);
            wait_and_meet<kFlying + 1>();
            issue(stage1, k + STAGES + 1);
            contract(stage2, k2);
            if constexpr (STAGES == 4) {
                wait_and_meet<kFlying + 1>();
                issue(stage2, k + STAGES + 2);
                contract(stage3, k3);
            }
        }
    }
    const int done = steps >= 4 ? whole * kGroupSteps : 0, left = steps - done;
    wait_and_meet<0>();
    if (left > 0) {
        read_scales(steps >= 4 ? first_of(whole) : 4 - steps);
        if constexpr (STAGES == 4) {
            contract(stage0, k0);
            if (left > 1) contract(stage1, k1);
            if (left > 2) contract(stage2, k2);
        } else {
            issue(stage2, done + 2);
            contract(stage0, k0);
            if (left > 1) contract(stage1, k1);
            wait_and_meet<0>();
            if (left > 2) contract(stage2, k2);
        }
    }
    // (the last meeting has seen every load arrive: nothing is on its way into LDS when the workgroup ends)
    if constexpr (Out::kStores) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; j += 2) store_eight<typename Out::type>(p, m0 + row_a + i * 16, n0 + col + j * 16 + g * 8, acc[i][j], acc[i][j + 1]);
    } else {
        // The sums of sixteen rows of a wave at a time through the stages' room, so that an epilogue has rows: eight columns to a lane, lanes side by side.  One piece
        // of code for all: unrolled over 128 sums with every kind of output it is more than the instruction cache holds (bias, gelu and residual at 8192^3: 464 instead of 426 us, with stores through the caches).
        constexpr int kPitch = TN * 16 + 4, kStrip = 16 * kPitch * 4, kStrips = kStage / kStrip, kPerRow = TN * 2, kPass = 64 / kPerRow, kPasses = 16 / kPass;
        static_assert(kWaves <= 2 * kStrips, "a strip to every wave in two stages");
        wait_and_meet<0>();
        float* strip = reinterpret_cast<float*>(wave < kStrips ? stage0 + wave * kStrip : stage1 + (wave - kStrips) * kStrip);
        const int lane_row = lane / kPerRow, lane_col = lane % kPerRow * 8;
        const int64_t n = n0 + col + lane_col;
        const int64_t m_first = m0 + (wave / WN) * TM * 16 + lane_row;
        float b[8];
        typename Out::Raw r[kPasses];
        out.bias_of(n, b);
#pragma unroll
        for (int q = 0; q < kPasses; ++q) out.ahead(m_first + q * kPass, n, r[q]);
#pragma unroll 1
        for (int i = 0; i < TM; ++i) {
            const int64_t m = m_first + i * 16;
#pragma unroll
            for (int k = 0; k < TM; ++k) {
                if (k != i) continue;
#pragma unroll
                for (int j = 0; j < TN; ++j) *reinterpret_cast<f32x4*>(strip + r16 * kPitch + j / 2 * 32 + g * 8 + j % 2 * 4) = acc[k][j];
            }
            asm volatile("" ::: "memory");
            auto sums = [&](int q, float (&s)[8]) {
                const float* from = strip + (lane_row + q * kPass) * kPitch + lane_col;
                const f32x4 x = *reinterpret_cast<const f32x4*>(from), y = *reinterpret_cast<const f32x4*>(from + 4);
                s[0] = x.x; s[1] = x.y; s[2] = x.z; s[3] = x.w; s[4] = y.x; s[5] = y.y; s[6] = y.z; s[7] = y.w;
                out.add_bias(n, b, s);
            };
            if constexpr (Out::kAhead) {
                // What the next rows need is asked for before these are stored: a load is back when the stores before it are, too.
                float s[kPasses][8];
#pragma unroll
                for (int q = 0; q < kPasses; ++q) { sums(q, s[q]); out.results_of(m + q * kPass, n, r[q], s[q]); }
                if (i + 1 < TM) {
#pragma unroll
                    for (int q = 0; q < kPasses; ++q) out.ahead(m + 16 + q * kPass, n, r[q]);
                }
#pragma unroll
                for (int q = 0; q < kPasses; ++q) out.store_results(m + q * kPass, n, s[q]);
                if (out.keeps()) {
#pragma unroll
                    for (int q = 0; q < kPasses; ++q) { sums(q, s[q]); out.keep(m + q * kPass, n, s[q]); }
                }
            } else {
#pragma unroll
                for (int q = 0; q < kPasses; ++q) {
                    float s[8];
                    sums(q, s);
                    out.keep(m + q * kPass, n, s);
                    out.results_of(m + q * kPass, n, r[q], s);
                    out.store_results(m + q * kPass, n, s);
                }
            }
            asm volatile("" ::: "memory");
        }
    }
}

// ---- few rows of A ---------------------------------------------------------------------------------------------------
// A workgroup takes 16 or 32 rows of B and all of A, its waves take four steps of 128 columns in turn, with B and A straight from global memory to
// registers, and their sums are added through LDS in the waves' order.  Bound by reading B while A is a row or a few (16384 x 4096, one row:
// 8.1 us, 4.4 TB/s), by A's way from L2 to every workgroup from 16 rows on.
constexpr int kAhead = 4;
struct __attribute__((packed, aligned(4))) Scales { uint32_t w[kAhead]; };

template <int FA>
__device__ __forceinline__ ints8 operand_at(const uint8_t* a, int64_t step) {
    if constexpr (FA == SSGD_MX_FP4) return operand(*reinterpret_cast<const words4*>(a + step * 64));
    else return operand(*reinterpret_cast<const words4*>(a + step * 128), *reinterpret_cast<const words4*>(a + step * 128 + 64));
}

// The sums of the waves, and the results: every wave adds the waves' sums of its share of the tiles, in the waves' order.
template <int TM, int TN, int WAVES, typename Out>
__device__ __forceinline__ void join_and_store(const Product& p, const Out& out, f32x4 (&acc)[TM][TN], f32x4 (*part)[TM * TN][64], int wave, int64_t m0, int64_t n0) {
    const int lane = threadIdx.x & 63;
    auto store = [&](int i, const f32x4& sum) {
        const int64_t m = m0 + i / TN * 16 + (lane & 15), n = n0 + i % TN * 16 + (lane >> 4) * 4;
        if constexpr (Out::kStores) store_four<typename Out::type>(p, m, n, sum);
        else out.four(m, n, sum);
    };
    if constexpr (WAVES == 1) {
#pragma unroll
        for (int i = 0; i < TM * TN; ++i) store(i, acc[i / TN][i % TN]);
    } else {
#pragma unroll
        for (int i = 0; i < TM * TN; ++i) part[wave][i][lane] = acc[i / TN][i % TN];
        __syncthreads();
        for (int i = wave; i < TM * TN; i += WAVES) {
            f32x4 sum = part[0][i][lane];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) sum += part[w][i][lane];
            store(i, sum);
        }
    }
}

template <int FA, int TM, int TN, int WAVES, typename Out>
__global__ __launch_bounds__(64 * WAVES) void few_rows_kernel(Product p, Out out) {
    __shared__ f32x4 part[WAVES][TM * TN][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * (TN * 16), m0 = (int64_t)blockIdx.y * (TM * 16);
    const uint8_t *a[TM], *sa[TM], *b[TN], *sb[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int64_t rb = n0 + j * 16 + r16 < p.b.rows ? n0 + j * 16 + r16 : p.b.rows - 1;
        b[j] = p.b.values + rb * p.b.row_bytes + g * 16;
        sb[j] = p.b.scales + rb * p.b.scale_bytes;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t ra = m0 + i * 16 + r16 < p.a.rows ? m0 + i * 16 + r16 : p.a.rows - 1;
        a[i] = p.a.values + ra * p.a.row_bytes + g * 16;
        sa[i] = p.a.scales + ra * p.a.scale_bytes;
    }
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM * TN; ++i) acc[i / TN][i % TN] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = wave * kAhead; k < p.steps; k += WAVES * kAhead) {
        if (k + kAhead <= p.steps) {
            words4 bv[TN][kAhead];
            ints8 av[TM][kAhead];
            Scales as[TM], bs[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                bs[j] = *reinterpret_cast<const Scales*>(sb[j] + (int64_t)k * 4);
#pragma unroll
                for (int q = 0; q < kAhead; ++q) bv[j][q] = *reinterpret_cast<const words4*>(b[j] + (int64_t)(k + q) * 64);
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                as[i] = *reinterpret_cast<const Scales*>(sa[i] + (int64_t)k * 4);
#pragma unroll
                for (int q = 0; q < kAhead; ++q) av[i][q] = operand_at<FA>(a[i], k + q);
            }
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
#pragma unroll
                for (int i = 0; i < TM * TN; ++i)
                    acc[i / TN][i % TN] = mfma<FA, 0>(operand(bv[i % TN][q]), av[i / TN][q], acc[i / TN][i % TN], bs[i % TN].w[q] >> (8 * g), as[i / TN].w[q] >> (8 * g));
        } else {
            for (int q = k; q < p.steps; ++q) {
                ints8 bv[TN];
                uint32_t bs[TN];
#pragma unroll
                for (int j = 0; j < TN; ++j) { bv[j] = operand(*reinterpret_cast<const words4*>(b[j] + (int64_t)q * 64)); bs[j] = sb[j][(int64_t)q * 4 + g]; }
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const ints8 av = operand_at<FA>(a[i], q);
                    const uint32_t as = sa[i][(int64_t)q * 4 + g];
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = mfma<FA, 0>(bv[j], av, acc[i][j], bs[j], as);
                }
            }
        }
    }
    join_and_store<TM, TN, WAVES>(p, out, acc, part, wave, m0, n0);
}

// The same for at most two rows that are quantised on the way, by every workgroup for itself, into LDS: as many bytes as its part of B at most,
// and one launch instead of two.  The first loads of B are on their way meanwhile.
constexpr int kRoomForRows = 32768;       // bytes of quantised rows and their scales
struct Rows { const void* x; int64_t pitch, cols; };

template <int FA, int WAVES, typename X, typename Out>
__global__ __launch_bounds__(64 * WAVES) void one_row_kernel(Product p, Rows x, Out out) {
    __shared__ f32x4 part[WAVES][1][64];
    __shared__ __attribute__((aligned(16))) uint8_t rows[kRoomForRows];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int64_t rb = n0 + r16 < p.b.rows ? n0 + r16 : p.b.rows - 1;
    const uint8_t *b = p.b.values + rb * p.b.row_bytes + g * 16, *sb = p.b.scales + rb * p.b.scale_bytes;
    const int many = (int)p.a.rows, row_bytes = (int)p.a.row_bytes, scale_bytes = (int)p.a.scale_bytes;
    uint8_t* scales = rows + many * row_bytes;
    words4 bv[kAhead];
    uint32_t bs[kAhead];
    auto load = [&](int k) {
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int64_t s = k + q < p.steps ? k + q : p.steps - 1;
            bv[q] = *reinterpret_cast<const words4*>(b + s * 64);
            bs[q] = *reinterpret_cast<const uint32_t*>(sb + s * 4);
        }
    };
    load(wave * kAhead);
    const int per_row = p.steps * 16;                  // groups of eight columns
    for (int u = threadIdx.x; u < many * per_row; u += 64 * WAVES) {
        const int row = u / per_row, col = (u - row * per_row) * 8;
        Eight<X> v;
        v.load(static_cast<const X*>(x.x) + row * x.pitch, col, x.cols);     // (more than 512 columns)
        v.settle(col, x.cols);
        const uint32_t byte = mx_scale_byte<FA>(max_of_4(v.largest()));
        if constexpr (FA == SSGD_MX_FP4) *reinterpret_cast<uint32_t*>(rows + row * row_bytes + col / 2) = mx_pack_fp4(v.values(), byte);
        else *reinterpret_cast<words2*>(rows + row * row_bytes + col) = mx_pack_fp8(v.values(), byte);
        if ((threadIdx.x & 3) == 0) scales[row * scale_bytes + col / kMxBlock] = (uint8_t)byte;
    }
    __syncthreads();
    const int ra = r16 < many ? r16 : many - 1;
    const uint8_t *a = rows + ra * row_bytes + g * 16, *sa = scales + ra * scale_bytes + g;
    f32x4 acc[1][1] = {{f32x4{0.0f, 0.0f, 0.0f, 0.0f}}};
    for (int k = wave * kAhead; k < p.steps; k += WAVES * kAhead) {
        if (k > wave * kAhead) load(k);
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
            if (k + q < p.steps) acc[0][0] = mfma<FA, 0>(operand(bv[q]), operand_at<FA>(a, k + q), acc[0][0], bs[q] >> (8 * g), sa[(k + q) * 4]);
    }
    join_and_store<1, 1, WAVES>(p, out, acc, part, wave, 0, n0);
}

// ---- host --------------------------------------------------------------------------------------------------------------
constexpr int64_t kFewRows = 64;

template <int FA, int TM, int TN, int WAVES, typename Out>
void few_rows(const Product& p, const Out& out, hipStream_t s) {
    const dim3 grid((unsigned)((p.b.rows + TN * 16 - 1) / (TN * 16)), (unsigned)((p.a.rows + TM * 16 - 1) / (TM * 16)));
    if (p.steps <= kAhead) hipLaunchKernelGGL((few_rows_kernel<FA, TM, TN, 1, Out>), grid, dim3(64), 0, s, p, out);
    else hipLaunchKernelGGL((few_rows_kernel<FA, TM, TN, WAVES, Out>), grid, dim3(64 * WAVES), 0, s, p, out);
}

// Waves of a workgroup for one group of 16 rows of A, with and without their quantisation (the sums of the same columns then add up alike).
constexpr int kRowWaves = 8;
template <int FA, typename X, typename Out>
void one_row(const Product& p, const Rows& x, const Out& out, hipStream_t s) {
    hipLaunchKernelGGL((one_row_kernel<FA, kRowWaves, X, Out>), dim3((unsigned)((p.b.rows + 15) / 16)), dim3(64 * kRowWaves), 0, s, p, x, out);
}

template <int FA, int BM, int BN, int WM, int WN, int STAGES, typename Out>
void tiles(Product p, const Out& out, hipStream_t s) {
    p.tiles_m = (int32_t)((p.a.rows + BM - 1) / BM);
    if constexpr (Out::kStores) p.tiles_n = (int32_t)((p.b.rows + BN - 1) / BN);
    else p.tiles_n = (int32_t)((out.wide() + BN - 1) / BN);
    const int64_t all = (int64_t)p.tiles_m * p.tiles_n;
    const unsigned parts = (unsigned)((p.steps + p.part_steps - 1) / p.part_steps);
    hipLaunchKernelGGL((tile_kernel<FA, BM, BN, WM, WN, STAGES, Out>), dim3((unsigned)((all + kXcds - 1) / kXcds * kXcds), parts), dim3(64 * WM * WN), 0, s, p, out);
}

// Rows of A to a tile, 256 with 256 rows of B or 128, 96 (in 8 bits) and 64 with 128, and the parts that the contraction is split into: those with the least
// time by a model, a step of the tiles that one CU has, and for parts the join's launch and their results written and read.
// (8192^3 in 4 bits: 275 us with 256 rows, 398 without them.  In 8 bits: 4100 x 4100 x 4096 94 us with 256, 78 with 128; 4001 x 2100 x 1500 22.1 us with 96
// rows, 24.9 with 128, 24.6 with 64; 2100 x 1500 x 4001 25.9, 23.0 and 22.7; 300 x 6144 x 5000 22.6, 25.6 and 17.8; 128 x 8192 x 8192 18.8 with 64 rows in two
// parts, 21.9 with 128 in four, 23.0 with 64 whole.)
constexpr int64_t kMostParts = 1024;      // tiles of parts, 64 MB of results
struct Tiling { int rows, parts; double time; };
inline Tiling tiling_of(int32_t a_fmt, int64_t M, int64_t N, int64_t steps) {
    Tiling best{128, 1, 1e30};
    for (int rows : {256, 128, 96, 64}) {
        if (rows == 96 && a_fmt == SSGD_MX_FP4) continue;       // (not a whole number of loads to a wave)
        const double step = a_fmt == SSGD_MX_FP4 ? (rows == 256 ? 1.06 : (rows == 128 ? 0.36 : 0.25))       // us, with a tile for every CU
                                                 : (rows == 256 ? 1.42 : (rows == 128 ? 0.53 : (rows == 96 ? 0.41 : 0.30)));
        const int64_t across = rows == 256 ? (N + 255) / 256 : (N + 127) / 128;
        for (int n = 1; n <= 8; ++n) {
            const int64_t tiles = (M + rows - 1) / rows * across * n, rounds = (tiles + 255) / 256;
            if (n > 1 && (rows == 256 || n * 4 > steps || tiles > kMostParts)) break;
            double t = step * (double)((steps + n - 1) / n) * (tiles < 256 ? 0.7 + 0.3 / 256 * (double)tiles : (double)rounds);
            if (n > 1) t += 3.0 + (double)M * (double)N * 8.0 / 6.0e6 * n;
            if (t < best.time) best = {rows, n, t};
        }
    }
    return best;
}

// 16 rows of B to a workgroup of the kernel for few rows, or 32 where they still give as many workgroups as keep the CUs busy: A is then read half as
// often (61 x 6144 x 5000 in 4 bits: 10.2 us against 15.6; 64 x 2048 x 4096: 9.5 against 8.3).
inline bool pairs_of(int64_t N) { return N >= 5120; }
// Up to 16 rows go through that kernel whatever the contraction: the tiles, which would take them as they take 17, win with more than 8 rows of a very long one
// only (4096 x 30000, eight and 16 rows: 12.7 and 14.1 us, the tiles 14.9, in 4 bits, 15.9 and 20.2, the tiles 16.5, in 8; 1000 x 30000: 11.2 and 12.9 to 12.0,
// 14.7 and 19.6 to 14.5).
// 17 to 64 rows of A through that kernel, by the same kind of model: its steps against those of the tiles, which cost 1.5 us more to begin with.
// (64 x 8192 x 8192 in 8 bits: 14.7 us through tiles, 23.8 through this; 64 x 6144 x 1500: 7.3 and 6.9.)
inline bool takes_few_rows(int32_t a_fmt, int64_t M, int64_t N, int64_t steps) {
    if (M <= 16 || M > kFewRows) return M <= 16;
    const bool pairs = pairs_of(N);
    const double step = a_fmt == SSGD_MX_FP4 ? (M > 32 ? (pairs ? 0.20 : 0.15) : (pairs ? 0.10 : 0.066)) : (M > 32 ? (pairs ? 0.29 : 0.28) : (pairs ? 0.127 : 0.11));
    const double full = (double)((N + (pairs ? 31 : 15)) / (pairs ? 32 : 16)) / 256.0;
    return step * (double)steps * (full < 1.0 ? 0.7 + 0.3 * full : full) <= tiling_of(a_fmt, M, N, steps).time + 1.5;
}

template <int FA, typename Out>
void tiles_of(int rows, const Product& p, const Out& out, hipStream_t s) {
    // (stages: with 128 rows of B as many as LDS holds for two workgroups of a CU, four at most; 128 rows in 8 bits, 2100 x 1500 x 4001: 30 us with two, 23
    // with three.  With 256, four or three are 136 and 152 KB, a workgroup to a CU.)
    if (rows == 256) {
        if constexpr (FA == SSGD_MX_FP4) tiles<FA, 256, 256, 2, 4, 4>(p, out, s);
        else tiles<FA, 256, 256, 4, 2, 3>(p, out, s);
        return;
    }
    if (rows == 64) { tiles<FA, 64, 128, 2, 2, 4>(p, out, s); return; }
    if constexpr (FA == SSGD_MX_FP8) { if (rows == 96) { tiles<FA, 96, 128, 2, 2, 3>(p, out, s); return; } }
    tiles<FA, 128, 128, 2, 2, FA == SSGD_MX_FP4 ? 4 : 3>(p, out, s);
}

template <int FA, typename Out>
void few_rows_of(const Product& p, const Out& out, hipStream_t s) {
    const bool pairs = pairs_of(p.b.rows);
    if (p.a.rows <= 16) { if (pairs) few_rows<FA, 1, 2, kRowWaves>(p, out, s); else few_rows<FA, 1, 1, kRowWaves>(p, out, s); }
    else if (p.a.rows <= 32) { if (pairs) few_rows<FA, 2, 2, 8>(p, out, s); else few_rows<FA, 2, 1, 8>(p, out, s); }
    else { if (pairs) few_rows<FA, 4, 2, 8>(p, out, s); else few_rows<FA, 4, 1, 4>(p, out, s); }
}

constexpr int64_t kMostRows = int64_t(1) << 31, kMostCols = (int64_t(1) << 24) - kMxPad;
inline bool format_ok(int32_t f) { return f == SSGD_MX_FP4 || f == SSGD_MX_FP8; }

inline Product product_of(const void* a_values, const void* a_scales, int32_t a_fmt, int64_t M, const void* b_values, const void* b_scales, int64_t N, int64_t K, void* out,
                   int64_t out_pitch) {
    Product p{};
    const int64_t scale_bytes = mx_padded(K) / kMxBlock;
    p.a = {static_cast<const uint8_t*>(a_values), static_cast<const uint8_t*>(a_scales), M, mx_row_bytes(a_fmt, K), scale_bytes};
    p.b = {static_cast<const uint8_t*>(b_values), static_cast<const uint8_t*>(b_scales), N, mx_row_bytes(SSGD_MX_FP4, K), scale_bytes};
    p.out = out; p.pitch = out_pitch; p.steps = p.part_steps = (int32_t)(mx_padded(K) / kMxPad);
    return p;
}

// Rows that each workgroup of the product quantises for itself (16384 x 4096: one row 10.1 us, 11 as two launches, and 3 us less for the host; four
// rows 12.8 and 12).  Contractions of 512 columns and less leave one wave.
inline bool quantises_itself(int32_t a_fmt, int64_t M, int64_t K) { return M <= 2 && mx_padded(K) > kAhead * kMxPad && M * (mx_row_bytes(a_fmt, K) + mx_padded(K) / kMxBlock) <= kRoomForRows; }

inline bool sizes_ok(int32_t a_fmt, int64_t M, int64_t N, int64_t K) {
    return format_ok(a_fmt) && M >= 0 && N >= 0 && K >= 0 && M < kMostRows && N < kMostRows && K <= kMostCols;
}

// Threads of the product's launch.
inline int64_t threads_of(int32_t a_fmt, int64_t M, int64_t N, int64_t K, bool itself) {
    const int64_t steps = mx_padded(K) / kMxPad;
    if (itself) return (N + 15) / 16 * (64 * kRowWaves);
    if (takes_few_rows(a_fmt, M, N, steps)) {
        const int64_t columns = pairs_of(N) ? 32 : 16;
        return (N + columns - 1) / columns * (steps <= kAhead ? 64 : 64 * kRowWaves);
    }
    const int rows = tiling_of(a_fmt, M, N, steps).rows, across = rows == 256 ? 256 : 128;
    return ((M + rows - 1) / rows * ((N + across - 1) / across) + kXcds - 1) / kXcds * kXcds * (rows == 256 ? 512 : 256);
}

}  // namespace
}  // namespace ssgd
