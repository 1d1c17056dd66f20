// Product of microscaled matrices on the matrix unit: C[m][n] = sum_k A[m][k] B[n][k], A in 4 or 8 bits, B in 4, fp32 accumulation.
//
// One instruction contracts 16 x 16 x 128, each lane with a row (lane % 16), the scale of its block of 32 columns (lane / 16) and, in
// 4 bits, that block's 16 bytes; in 8 bits bytes 16 g .. 16 g + 15 and the same 64 further on.  B's rows are the instruction's first
// operand and A's its second, so that a lane's four results are consecutive columns of a row of C.
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

template <int FA>
__device__ __forceinline__ f32x4 mfma(const ints8& b, const ints8& a, const f32x4& c, uint32_t scale_b, uint32_t scale_a) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 4, FA == SSGD_MX_FP4 ? 4 : 0, 0, (int)scale_b, 0, (int)scale_a);
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
// Global memory to LDS without registers: lane l's bytes go to `to` + 16 l (4 l).
__device__ __forceinline__ void copy16(const uint8_t* from, uint8_t* to) { __builtin_amdgcn_global_load_lds((global_word*)from, (lds_word*)to, 16, 0, 0); }
__device__ __forceinline__ void copy4(const uint8_t* from, uint8_t* to) { __builtin_amdgcn_global_load_lds((global_word*)from, (lds_word*)to, 4, 0, 0); }

template <int VM> __device__ __forceinline__ void wait_and_meet() {
    static_assert(VM < 64, "the counter has six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((VM & 15) | ((VM >> 4) << 14) | (7 << 4));     // vmcnt(VM), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// WM x WN waves, a tile of BM x BN.  A stage is 128 columns: rows of A (64 or 128 bytes), rows of B (64), a word of scales per row.  In
// LDS the 16-byte parts of a row change places by its number, so that the lanes that read one part of 16 rows meet in no bank.
template <int FA, int BM, int BN, int WM, int WN, int STAGES, typename T>
__global__ __launch_bounds__(64 * WM * WN) void tile_kernel(Product p) {
    constexpr int kWaves = WM * WN, kRowA = FA == SSGD_MX_FP4 ? 64 : 128, kRowB = 64;
    constexpr int kA = BM * kRowA, kB = BN * kRowB, kStage = kA + kB + (BM + BN) * 4;
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int kLoadsA = kA / 1024 / kWaves, kLoadsB = kB / 1024 / kWaves, kLoadsS = (BM + BN) / 64 / kWaves;
    constexpr int kLoads = kLoadsA + kLoadsB + kLoadsS;
    static_assert(kLoadsA * 1024 * kWaves == kA && kLoadsB * 1024 * kWaves == kB && kLoadsS * 64 * kWaves == BM + BN, "every wave loads the same share");
    // (arrays of their own: the compiler then sees that loads into one stage do not concern reads of another)
    __shared__ __attribute__((aligned(1024))) uint8_t stage0[kStage];
    __shared__ __attribute__((aligned(1024))) uint8_t stage1[kStage];
    __shared__ __attribute__((aligned(1024))) uint8_t stage2[STAGES > 2 ? kStage : 16];
    __shared__ __attribute__((aligned(1024))) uint8_t stage3[STAGES > 3 ? kStage : 16];

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
    const uint8_t* from[kLoads];
#pragma unroll
    for (int q = 0; q < kLoadsA; ++q) {
        const int unit = (q * kWaves + wave) * 64 + lane, per = kRowA / 16, row = unit / per;
        const int part = (unit % per) ^ (FA == SSGD_MX_FP4 ? (row >> 1) & 3 : row & 7);
        const int64_t r = m0 + row < p.a.rows ? m0 + row : p.a.rows - 1;
        from[q] = p.a.values + r * p.a.row_bytes + part * 16;
    }
#pragma unroll
    for (int q = 0; q < kLoadsB; ++q) {
        const int unit = (q * kWaves + wave) * 64 + lane, row = unit / 4, part = (unit % 4) ^ ((row >> 1) & 3);
        const int64_t r = n0 + row < p.b.rows ? n0 + row : p.b.rows - 1;
        from[kLoadsA + q] = p.b.values + r * p.b.row_bytes + part * 16;
    }
#pragma unroll
    for (int q = 0; q < kLoadsS; ++q) {
        const int row = (q * kWaves + wave) * 64 + lane;
        if (row < BM) {
            const int64_t r = m0 + row < p.a.rows ? m0 + row : p.a.rows - 1;
            from[kLoadsA + kLoadsB + q] = p.a.scales + r * p.a.scale_bytes;
        } else {
            const int64_t r = n0 + row - BM < p.b.rows ? n0 + row - BM : p.b.rows - 1;
            from[kLoadsA + kLoadsB + q] = p.b.scales + r * p.b.scale_bytes;
        }
    }
    // Every call issues as many loads, so that they can be counted: past the last step the last one is loaded again, and not used.
    auto issue = [&](uint8_t* stage, int step) {
        const int k = step < p.steps ? step : p.steps - 1;
#pragma unroll
        for (int q = 0; q < kLoadsA; ++q) copy16(from[q] + (int64_t)k * kRowA, stage + (q * kWaves + wave) * 1024);
#pragma unroll
        for (int q = 0; q < kLoadsB; ++q) copy16(from[kLoadsA + q] + (int64_t)k * kRowB, stage + kA + (q * kWaves + wave) * 1024);
#pragma unroll
        for (int q = 0; q < kLoadsS; ++q) copy4(from[kLoadsA + kLoadsB + q] + (int64_t)k * 4, stage + kA + kB + (q * kWaves + wave) * 256);
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
    const int at_sa = kA + kB + row_a * 4 + g, at_sb = kA + kB + (BM + row_b) * 4 + g;

    auto contract = [&](const uint8_t* stage) {
        ints8 a[TM], b[TN];
        uint32_t sa[TM], sb[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            b[j] = operand(*reinterpret_cast<const words4*>(stage + at_b + j * 16 * 64));
            sb[j] = stage[at_sb + j * 64];
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            if constexpr (FA == SSGD_MX_FP4) a[i] = operand(*reinterpret_cast<const words4*>(stage + at_a + i * 16 * 64));
            else a[i] = operand(*reinterpret_cast<const words4*>(stage + at_a + i * 16 * 128), *reinterpret_cast<const words4*>(stage + (at_a ^ 64) + i * 16 * 128));
            sa[i] = stage[at_sa + i * 64];
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = mfma<FA>(b[j], a[i], acc[i][j], sb[j], sa[i]);
    };

    issue(stage0, 0);
    if constexpr (STAGES > 2) issue(stage1, 1);
    if constexpr (STAGES > 3) issue(stage2, 2);
    // A stage is read when its own loads have arrived in every wave, and loaded again only behind the next meeting, when all have read it.
    constexpr int kFlying = kLoads * (STAGES - 2);
    int k = 0;
    for (; k + STAGES <= p.steps; k += STAGES) {
        wait_and_meet<kFlying>();
        issue(STAGES == 2 ? stage1 : (STAGES == 3 ? stage2 : stage3), k + STAGES - 1);
        contract(stage0);
        wait_and_meet<kFlying>();
        issue(stage0, k + STAGES);
        contract(stage1);
        if constexpr (STAGES > 2) {
            wait_and_meet<kFlying>();
            issue(stage1, k + STAGES + 1);
            contract(stage2);
        }
        if constexpr (STAGES > 3) {
            wait_and_meet<kFlying>();
            issue(stage2, k + STAGES + 2);
            contract(stage3);
        }
    }
    // the last STAGES - 1 steps at most: their loads are on the way
    wait_and_meet<0>();
    if (k < p.steps) contract(stage0);
    if constexpr (STAGES > 2) if (k + 1 < p.steps) contract(stage1);
    if constexpr (STAGES > 3) if (k + 2 < p.steps) contract(stage2);
    __builtin_amdgcn_s_waitcnt(0);      // nothing may still be on its way into LDS when the workgroup ends
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
                    acc[i] = mfma<FA>(operand(bv[q]), op, acc[i], bs.w[q] >> (8 * g), as[i].w[q] >> (8 * g));
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
                    acc[i] = mfma<FA>(operand(bv), op, acc[i], bs, sa[i][(int64_t)q * 4 + g]);
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
    else if ((p.a.rows + 255) / 256 * ((p.b.rows + 255) / 256) < 200) tiles<FA, 128, 128, 2, 2, 4, T>(p, s);
    else tiles<FA, 256, 256, 2, 4, FA == SSGD_MX_FP4 ? 4 : 3, T>(p, s);
}

constexpr int64_t kMostRows = int64_t(1) << 31, kMostCols = int64_t(1) << 31;
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
    if (M < 0 || N < 0 || K < 0 || M >= kMostRows || N >= kMostRows || K >= kMostCols || out_pitch < N) return "mx product: M, N, K from zero to 2^31, pitch >= N";
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
    if (!format_ok(a_fmt) || M < 0 || K < 0 || M >= kMostRows || K >= kMostCols) return -1;
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
