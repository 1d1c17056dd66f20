// Product of microscaled matrices on the matrix unit: C[m][n] = sum_k A[m][k] B[n][k], A in 4 or 8 bits, B in 4, fp32 accumulation.
//
// One instruction contracts 16 x 16 x 128, each lane with a row (lane % 16), the scale of its block of 32 columns (lane / 16) and, in
// 4 bits, that block's 16 bytes; in 8 bits bytes 16 g .. 16 g + 15 and the same 64 further on.  B's rows are the instruction's first
// operand and A's its second, so that a lane's four results are consecutive columns of a row of C.
#include <type_traits>

#include "ops.hpp"

using namespace ssgd;

namespace {

typedef int ints8 __attribute__((ext_vector_type(8)));

struct Matrix { const uint8_t *values, *scales; int64_t rows, row_bytes, scale_bytes; };
struct Product {
    Matrix a, b;
    void* out;
    int64_t pitch;
    int32_t steps;          // of 128 columns
    int32_t tiles_m, tiles_n;
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

template <typename T>
__device__ __forceinline__ void store_four(const Product& p, int64_t m, int64_t n, const f32x4& c) {
    if (m >= p.a.rows || n >= p.b.rows) return;
    const float x[4] = {c.x, c.y, c.z, c.w};
    store_vec<4>(static_cast<T*>(p.out) + m * p.pitch + n, p.b.rows - n, x);
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
template <int FA, int BM, int BN, int WM, int WN, int STAGES, typename T>
__global__ __launch_bounds__(64 * WM * WN) void tile_kernel(Product p) {
    constexpr int kWaves = WM * WN, kRowA = FA == SSGD_MX_FP4 ? 64 : 128, kRowB = 64;
    constexpr int kA = BM * kRowA, kB = BN * kRowB, kStage = kA + kB;
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int kLoadsA = kA / 1024 / kWaves, kLoadsB = kB / 1024 / kWaves, kLoads = kLoadsA + kLoadsB;
    static_assert(kLoadsA * 1024 * kWaves == kA && kLoadsB * 1024 * kWaves == kB && BM + BN == 64 * kWaves, "every wave loads the same share");
    constexpr int kGroupSteps = STAGES == 3 ? 3 : 4;
    static_assert(STAGES >= 2 && STAGES <= 4, "a group ends at the stage it began with");
    // (arrays of their own: the compiler then sees that loads into one do not concern reads of another)
    __shared__ __attribute__((aligned(1024))) uint8_t stage0[kStage];
    __shared__ __attribute__((aligned(1024))) uint8_t stage1[kStage];
    __shared__ __attribute__((aligned(1024))) uint8_t stage2[STAGES > 2 ? kStage : 16];
    __shared__ __attribute__((aligned(1024))) uint8_t stage3[STAGES > 3 ? kStage : 16];
    __shared__ __attribute__((aligned(1024))) uint8_t scales[(BM + BN) * 16];

    // Workgroups go to the XCDs in turn; each XCD takes tiles that lie together, in groups of 8 rows of tiles, so that its L2 holds what
    // they share.
    const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n, per_xcd = (tiles + kXcds - 1) / kXcds;
    const int64_t id = (int64_t)(blockIdx.x % kXcds) * per_xcd + blockIdx.x / kXcds;
    if (blockIdx.x / kXcds >= per_xcd || id >= tiles) return;
    constexpr int kGroup = 8;
    const int64_t group = id / (kGroup * (int64_t)p.tiles_n), in_group = id - group * kGroup * p.tiles_n;
    const int64_t height = p.tiles_m - group * kGroup < kGroup ? p.tiles_m - group * kGroup : kGroup;
    const int64_t m0 = (group * kGroup + in_group % height) * BM, n0 = in_group / height * BN;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (offsets from the tile's first row: 256 rows of less than 2^24 bytes)
    const uint8_t *a_values = p.a.values + m0 * p.a.row_bytes, *b_values = p.b.values + n0 * p.b.row_bytes;
    const uint32_t rows_a = (uint32_t)(p.a.rows - m0 < BM ? p.a.rows - m0 : BM), rows_b = (uint32_t)(p.b.rows - n0 < BN ? p.b.rows - n0 : BN);
    uint32_t from[kLoads];
#pragma unroll
    for (int q = 0; q < kLoadsA; ++q) {
        const uint32_t unit = (q * kWaves + wave) * 64 + lane, per = kRowA / 16, row = unit / per;
        const uint32_t part = (unit % per) ^ (FA == SSGD_MX_FP4 ? (row >> 1) & 3 : row & 7);
        from[q] = (row < rows_a ? row : rows_a - 1) * (uint32_t)p.a.row_bytes + part * 16;
    }
#pragma unroll
    for (int q = 0; q < kLoadsB; ++q) {
        const uint32_t unit = (q * kWaves + wave) * 64 + lane, row = unit / 4, part = (unit % 4) ^ ((row >> 1) & 3);
        from[kLoadsA + q] = (row < rows_b ? row : rows_b - 1) * (uint32_t)p.b.row_bytes + part * 16;
    }
    const uint8_t* scales_from;
    {
        const uint32_t row = threadIdx.x, in_a = row < rows_a ? row : rows_a - 1, in_b = row - BM < rows_b ? row - BM : rows_b - 1;
        scales_from = row < BM ? p.a.scales + (m0 + in_a) * p.a.scale_bytes : p.b.scales + (n0 + in_b) * p.b.scale_bytes;
    }
    // Every call issues as many loads, so that they can be counted: past the last step the last one is loaded again, and not used.
    auto issue = [&](uint8_t* stage, int step) {
        const int k = step < p.steps ? step : p.steps - 1;
        const uint8_t *a = a_values + (int64_t)k * kRowA, *b = b_values + (int64_t)k * kRowB;
#pragma unroll
        for (int q = 0; q < kLoadsA; ++q) copy16(a + from[q], stage + (q * kWaves + wave) * 1024);
#pragma unroll
        for (int q = 0; q < kLoadsB; ++q) copy16(b + from[kLoadsA + q], stage + kA + (q * kWaves + wave) * 1024);
    };
    const int whole = p.steps / kGroupSteps;       // groups
    // Where 16 bytes from a group's first scale on would pass the end of the row, its last 16 bytes come instead; `first` is the place of the
    // group's first scale in them.  Rows of less than 16 bytes are put together at the start.
    auto first_of = [&](int f) { return f * kGroupSteps + 4 <= p.steps ? 0 : f * kGroupSteps + 4 - p.steps; };
    auto issue_scales = [&](int f) {
        const int at = f * kGroupSteps + 4 <= p.steps ? f * kGroupSteps * 4 : p.steps * 4 - 16;
        copy16(scales_from + (at > 0 ? at : 0), scales + wave * 1024);
    };

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int r16 = lane & 15, g = lane >> 4;
    const int row_a = (wave / WN) * TM * 16 + r16, row_b = (wave % WN) * TN * 16 + r16;
    // (rows 16 further on have the same exchange of parts)
    const int at_a = FA == SSGD_MX_FP4 ? row_a * 64 + (g ^ ((row_a >> 1) & 3)) * 16 : row_a * 128 + (g ^ (row_a & 7)) * 16;
    const int at_b = kA + row_b * 64 + (g ^ ((row_b >> 1) & 3)) * 16;

    uint32_t sa[TM], sb[TN];
    auto read_scales = [&](int skipped) {
#pragma unroll
        for (int j = 0; j < TN; ++j) sb[j] = scales_of_four(*reinterpret_cast<const words4*>(scales + (BM + row_b + j * 16) * 16), g) >> (8 * skipped);
#pragma unroll
        for (int i = 0; i < TM; ++i) sa[i] = scales_of_four(*reinterpret_cast<const words4*>(scales + (row_a + i * 16) * 16), g) >> (8 * skipped);
    };
    auto contract = [&](const uint8_t* stage, auto byte) {
        ints8 a[TM], b[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) b[j] = operand(*reinterpret_cast<const words4*>(stage + at_b + j * 16 * 64));
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

    if (p.steps >= 4) issue_scales(0);
    else {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = q >= 4 - p.steps ? *reinterpret_cast<const uint32_t*>(scales_from + (q - 4 + p.steps) * 4) : 0u;
        *reinterpret_cast<words4*>(scales + threadIdx.x * 16) = words4{w[0], w[1], w[2], w[3]};
    }
    issue(stage0, 0);
    if constexpr (STAGES > 2) issue(stage1, 1);
    if constexpr (STAGES > 3) issue(stage2, 2);
    // A stage is read when its own loads have arrived in every wave, and loaded again only behind the next meeting, when all have read it.
    // The counts are those of the loads issued after it: STAGES - 2 steps, and from the second step of a group on its successor's scales
    // until the steps issued with them are read.
    constexpr int kFlying = kLoads * (STAGES - 2);
    if (p.steps >= 4) {
        for (int f = 0; f < whole; ++f) {
            const int k = f * kGroupSteps;
            wait_and_meet<kFlying>();
            read_scales(first_of(f));
            issue(STAGES == 2 ? stage1 : (STAGES == 3 ? stage2 : stage3), k + STAGES - 1);
            contract(stage0, k0);
            wait_and_meet<kFlying>();
            issue(stage0, k + STAGES);
            issue_scales(f + 1);
            contract(stage1, k1);
            wait_and_meet<kFlying + 1>();
            issue(stage1, k + STAGES + 1);
            contract(STAGES > 2 ? stage2 : stage0, k2);
            if constexpr (STAGES != 3) {
                wait_and_meet<kFlying + (STAGES > 3 ? 1 : 0)>();
                issue(STAGES > 3 ? stage2 : stage0, k + STAGES + 2);
                contract(STAGES > 3 ? stage3 : stage1, k3);
            }
        }
    }
    const int done = p.steps >= 4 ? whole * kGroupSteps : 0, left = p.steps - done;
    wait_and_meet<0>();
    if (left > 0) {
        read_scales(p.steps >= 4 ? first_of(whole) : 4 - p.steps);
        if constexpr (STAGES > 3) {
            contract(stage0, k0);
            if (left > 1) contract(stage1, k1);
            if (left > 2) contract(stage2, k2);
        } else if constexpr (STAGES > 2) {
            issue(stage2, done + 2);
            contract(stage0, k0);
            if (left > 1) contract(stage1, k1);
            wait_and_meet<0>();
            if (left > 2) contract(stage2, k2);
        } else {
            issue(stage1, done + 1);
            contract(stage0, k0);
            wait_and_meet<0>();
            issue(stage0, done + 2);
            if (left > 1) contract(stage1, k1);
            wait_and_meet<0>();
            if (left > 2) contract(stage0, k2);
        }
    }
    // (the last meeting has seen every load arrive: nothing is on its way into LDS when the workgroup ends)
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
            store_four<T>(p, m0 + row_a + i * 16, n0 + row_b - r16 + j * 16 + g * 4, acc[i][j]);
}

// ---- few rows of A ---------------------------------------------------------------------------------------------------
// Bound by reading B: a workgroup takes 16 rows of B and all of A, its waves take 512 columns in turn, with B and A straight from global
// memory to registers, and their sums are added through LDS.
struct __attribute__((packed, aligned(4))) Scales4 { uint32_t w[4]; };

template <int FA, int TM, int WAVES, typename T>
__global__ __launch_bounds__(64 * WAVES) void few_rows_kernel(Product p) {
    __shared__ f32x4 part[WAVES > 1 ? WAVES - 1 : 1][TM][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (TM * 16);
    const int64_t rb = n0 + r16 < p.b.rows ? n0 + r16 : p.b.rows - 1;
    const uint8_t *b = p.b.values + rb * p.b.row_bytes + g * 16, *sb = p.b.scales + rb * p.b.scale_bytes;
    const uint8_t *a[TM], *sa[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t ra = m0 + i * 16 + r16 < p.a.rows ? m0 + i * 16 + r16 : p.a.rows - 1;
        a[i] = p.a.values + ra * p.a.row_bytes + g * 16;
        sa[i] = p.a.scales + ra * p.a.scale_bytes;
    }
    f32x4 acc[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = wave * 4; k < p.steps; k += WAVES * 4) {
        if (k + 4 <= p.steps) {
            words4 bv[4], av[TM][4], ah[TM][4];
            const Scales4 bs = *reinterpret_cast<const Scales4*>(sb + (int64_t)k * 4);
            Scales4 as[TM];
#pragma unroll
            for (int q = 0; q < 4; ++q) bv[q] = *reinterpret_cast<const words4*>(b + (int64_t)(k + q) * 64);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                as[i] = *reinterpret_cast<const Scales4*>(sa[i] + (int64_t)k * 4);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if constexpr (FA == SSGD_MX_FP4) av[i][q] = *reinterpret_cast<const words4*>(a[i] + (int64_t)(k + q) * 64);
                    else {
                        av[i][q] = *reinterpret_cast<const words4*>(a[i] + (int64_t)(k + q) * 128);
                        ah[i][q] = *reinterpret_cast<const words4*>(a[i] + (int64_t)(k + q) * 128 + 64);
                    }
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    ints8 op;
                    if constexpr (FA == SSGD_MX_FP4) op = operand(av[i][q]); else op = operand(av[i][q], ah[i][q]);
                    acc[i] = mfma<FA, 0>(operand(bv[q]), op, acc[i], bs.w[q] >> (8 * g), as[i].w[q] >> (8 * g));
                }
        } else {
            for (int q = k; q < p.steps; ++q) {
                const words4 bv = *reinterpret_cast<const words4*>(b + (int64_t)q * 64);
                const uint32_t bs = sb[(int64_t)q * 4 + g];
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    ints8 op;
                    if constexpr (FA == SSGD_MX_FP4) op = operand(*reinterpret_cast<const words4*>(a[i] + (int64_t)q * 64));
                    else op = operand(*reinterpret_cast<const words4*>(a[i] + (int64_t)q * 128), *reinterpret_cast<const words4*>(a[i] + (int64_t)q * 128 + 64));
                    acc[i] = mfma<FA, 0>(operand(bv), op, acc[i], bs, sa[i][(int64_t)q * 4 + g]);
                }
            }
        }
    }
    if constexpr (WAVES > 1) {
        if (wave > 0) {
#pragma unroll
            for (int i = 0; i < TM; ++i) part[wave - 1][i][lane] = acc[i];
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < WAVES - 1; ++w)
#pragma unroll
            for (int i = 0; i < TM; ++i) acc[i] += part[w][i][lane];
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) store_four<T>(p, m0 + i * 16 + r16, n0 + g * 4, acc[i]);
}

template <typename T>
__global__ __launch_bounds__(256) void zero_kernel(T* out, int64_t rows, int64_t cols, int64_t pitch) {
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < rows * cols; q += (int64_t)gridDim.x * 256) out[q / cols * pitch + q % cols] = (T)0;
}

// ---- host --------------------------------------------------------------------------------------------------------------
template <int FA, int TM, typename T>
void few_rows(const Product& p, hipStream_t s) {
    const dim3 grid((unsigned)((p.b.rows + 15) / 16), (unsigned)((p.a.rows + TM * 16 - 1) / (TM * 16)));
    // about 4096 waves, none without columns
    const int64_t want = 4096 / ((int64_t)grid.x * grid.y) + 1, most = (p.steps + 3) / 4;
    if (want >= 16 && most >= 16) hipLaunchKernelGGL((few_rows_kernel<FA, TM, 16, T>), grid, dim3(1024), 0, s, p);
    else if (want >= 8 && most >= 8) hipLaunchKernelGGL((few_rows_kernel<FA, TM, 8, T>), grid, dim3(512), 0, s, p);
    else if (most >= 4) hipLaunchKernelGGL((few_rows_kernel<FA, TM, 4, T>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((few_rows_kernel<FA, TM, 1, T>), grid, dim3(64), 0, s, p);
}

template <int FA, int BM, int BN, int WM, int WN, int STAGES, typename T>
void tiles(Product p, hipStream_t s) {
    p.tiles_m = (int32_t)((p.a.rows + BM - 1) / BM);
    p.tiles_n = (int32_t)((p.b.rows + BN - 1) / BN);
    const int64_t all = (int64_t)p.tiles_m * p.tiles_n;
    hipLaunchKernelGGL((tile_kernel<FA, BM, BN, WM, WN, STAGES, T>), dim3((unsigned)((all + kXcds - 1) / kXcds * kXcds)), dim3(64 * WM * WN), 0, s, p);
}

template <int FA, typename T>
void launch(const Product& p, hipStream_t s) {
    if (p.a.rows <= 16) few_rows<FA, 1, T>(p, s);
    else if (p.a.rows <= 32) few_rows<FA, 2, T>(p, s);
    else if (p.a.rows <= 64) few_rows<FA, 4, T>(p, s);
    // Tiles of 256 where there are enough of them to fill most CUs (8192^3: 281 us in 4 bits against 410 with tiles of 128; 1000 x 8192 x 8192, 128
    // tiles: 59 against 55).  Stages: as many as LDS holds, for tiles of 128 of two workgroups per CU (2100 x 1500 x 4001 in 8 bits: 30 us with
    // two, 22 with three; 4001 x 2100 x 1500 27 and 23, with four and one workgroup per CU 28).
    else if ((p.a.rows + 255) / 256 * ((p.b.rows + 255) / 256) < 200) tiles<FA, 128, 128, 2, 2, FA == SSGD_MX_FP4 ? 4 : 3, T>(p, s);
    else if constexpr (FA == SSGD_MX_FP4) tiles<FA, 256, 256, 2, 4, 4, T>(p, s);
    else tiles<FA, 256, 256, 4, 2, 3, T>(p, s);
}

constexpr int64_t kMostRows = int64_t(1) << 31, kMostCols = (int64_t(1) << 24) - kMxPad;
bool format_ok(int32_t f) { return f == SSGD_MX_FP4 || f == SSGD_MX_FP8; }

ssgd_status product(const void* a_values, const void* a_scales, int32_t a_fmt, int64_t M, const void* b_values, const void* b_scales, int64_t N, int64_t K,
                    void* out, int32_t out_dtype, int64_t out_pitch, hipStream_t stream) {
    if (K == 0) {
        const dim3 grid(1024);
        if (out_dtype == SSGD_F32) hipLaunchKernelGGL((zero_kernel<float>), grid, dim3(256), 0, stream, static_cast<float*>(out), M, N, out_pitch);
        else hipLaunchKernelGGL((zero_kernel<bf16_t>), grid, dim3(256), 0, stream, static_cast<bf16_t*>(out), M, N, out_pitch);
        return op_hip(hipGetLastError(), "mx product");
    }
    Product p{};
    const int64_t scale_bytes = mx_padded(K) / kMxBlock;
    p.a = {static_cast<const uint8_t*>(a_values), static_cast<const uint8_t*>(a_scales), M, mx_row_bytes(a_fmt, K), scale_bytes};
    p.b = {static_cast<const uint8_t*>(b_values), static_cast<const uint8_t*>(b_scales), N, mx_row_bytes(SSGD_MX_FP4, K), scale_bytes};
    p.out = out; p.pitch = out_pitch; p.steps = (int32_t)(mx_padded(K) / kMxPad);
    if (a_fmt == SSGD_MX_FP4) { if (out_dtype == SSGD_F32) launch<SSGD_MX_FP4, float>(p, stream); else launch<SSGD_MX_FP4, bf16_t>(p, stream); }
    else { if (out_dtype == SSGD_F32) launch<SSGD_MX_FP8, float>(p, stream); else launch<SSGD_MX_FP8, bf16_t>(p, stream); }
    return op_hip(hipGetLastError(), "mx product");
}

const char* refused(int32_t a_fmt, int64_t M, const void* b_values, const void* b_scales, int64_t N, int64_t K, const void* out, int32_t out_dtype, int64_t out_pitch) {
    if (!format_ok(a_fmt) || !dtype_ok(out_dtype)) return "mx product: a format and an output type of the enumerations";
    if (M < 0 || N < 0 || K < 0 || M >= kMostRows || N >= kMostRows || K > kMostCols || out_pitch < N) return "mx product: M and N from zero to 2^31, K to 2^24 - 128, pitch >= N";
    if (M == 0 || N == 0) return nullptr;
    if ((M + 127) / 128 * ((N + 127) / 128) > kMostBlocks) return "mx product: too many results";
    if (K > 0 && (!b_values || !b_scales || !aligned(b_values, 16) || !aligned(b_scales, 16))) return "mx product: values and scales are 16-byte aligned arrays";
    if (!out || !aligned(out, (uintptr_t)dtype_bytes(out_dtype))) return "mx product: the output is null or misaligned";
    return nullptr;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

ssgd_status ssgd_mx_matmul(const void* a_values, const void* a_scales, int32_t a_fmt, int64_t M, const void* b_values, const void* b_scales, int64_t N, int64_t K,
                           void* out, int32_t out_dtype, int64_t out_pitch, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        if (const char* why = refused(a_fmt, M, b_values, b_scales, N, K, out, out_dtype, out_pitch)) return op_fail(SSGD_EINVAL, why);
        if (M == 0 || N == 0) return SSGD_OK;
        if (K > 0 && (!a_values || !a_scales || !aligned(a_values, 16) || !aligned(a_scales, 16))) return op_fail(SSGD_EINVAL, "mx product: values and scales are 16-byte aligned arrays");
        return product(a_values, a_scales, a_fmt, M, b_values, b_scales, N, K, out, out_dtype, out_pitch, static_cast<hipStream_t>(hip_stream));
    });
}

int64_t ssgd_mx_linear_work_bytes(int32_t a_fmt, int64_t M, int64_t K) {
    if (!format_ok(a_fmt) || M < 0 || K < 0 || M >= kMostRows || K > kMostCols) return -1;
    return M * (mx_row_bytes(a_fmt, K) + mx_padded(K) / kMxBlock);
}

ssgd_status ssgd_mx_linear(const void* x, int32_t dtype, int64_t pitch, int64_t M, int32_t a_fmt, const void* b_values, const void* b_scales, int64_t N, int64_t K,
                           void* out, int32_t out_dtype, int64_t out_pitch, void* work, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        if (const char* why = refused(a_fmt, M, b_values, b_scales, N, K, out, out_dtype, out_pitch)) return op_fail(SSGD_EINVAL, why);
        if (M == 0 || N == 0) return SSGD_OK;
        uint8_t *values = static_cast<uint8_t*>(work), *scales = values + M * mx_row_bytes(a_fmt, K);
        if (K > 0) {
            if (!work || !aligned(work, 16)) return op_fail(SSGD_EINVAL, "mx linear: a 16-byte aligned work area");
            const ssgd_status st = ssgd_mx_quantize(x, dtype, M, K, pitch, a_fmt, values, scales, 0, nullptr, nullptr, hip_stream);
            if (st != SSGD_OK) return st;
        }
        return product(values, scales, a_fmt, M, b_values, b_scales, N, K, out, out_dtype, out_pitch, static_cast<hipStream_t>(hip_stream));
    });
}

}  // extern "C"
#pragma GCC visibility pop
