// Entry points of the product of microscaled matrices (kernels: mx_product.hpp): results as they are.
#include "mx_product.hpp"

using namespace ssgd;

namespace {

template <typename T>
__global__ __launch_bounds__(256) void zero_kernel(T* out, int64_t rows, int64_t cols, int64_t pitch) {
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < rows * cols; q += (int64_t)gridDim.x * 256) out[q / cols * pitch + q % cols] = (T)0;
}

// The parts of a split contraction, added in order: four results a thread.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(const float* parts, int32_t n, int64_t stride, T* out, int64_t rows, int64_t cols, int64_t pitch, int64_t per_row) {
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x, row = u / per_row, col = (u - row * per_row) * 4;
    if (row >= rows) return;
    float sum[4], x[8][4];
    const float* at = parts + row * cols + col;
#pragma unroll
    for (int q = 0; q < 8; ++q)
        if (q < n) load_vec<4>(at + q * stride, cols - col, x[q]);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        sum[c] = x[0][c];
#pragma unroll
        for (int q = 1; q < 8; ++q) if (q < n) sum[c] += x[q][c];
    }
    store_vec<4>(out + row * pitch + col, cols - col, sum);
}

int64_t parts_bytes(int32_t a_fmt, int64_t M, int64_t N, int64_t K) {
    const int64_t steps = mx_padded(K) / kMxPad;
    const int n = takes_few_rows(a_fmt, M, N, steps) ? 1 : tiling_of(a_fmt, M, N, steps).parts;
    return n > 1 ? n * M * N * 4 : 0;
}

template <int FA, typename T>
void launch(Product p, void* work, hipStream_t s) {
    if (takes_few_rows(FA, p.a.rows, p.b.rows, p.steps)) { few_rows_of<FA>(p, To<T>{}, s); return; }
    const Tiling how = tiling_of(FA, p.a.rows, p.b.rows, p.steps);
    if (how.parts == 1) { tiles_of<FA>(how.rows, p, To<T>{}, s); return; }
    Product q = p;
    q.out = work; q.pitch = p.b.rows; q.part_stride = p.a.rows * p.b.rows;
    q.part_steps = (p.steps + how.parts - 1) / how.parts;
    tiles_of<FA>(how.rows, q, To<float>{}, s);
    const int64_t per_row = (p.b.rows + 3) / 4, groups = p.a.rows * per_row;
    hipLaunchKernelGGL((join_kernel<T>), dim3((unsigned)((groups + 255) / 256)), dim3(256), 0, s, static_cast<const float*>(work), (p.steps + q.part_steps - 1) / q.part_steps,
                       q.part_stride, static_cast<T*>(p.out), p.a.rows, p.b.rows, p.pitch, per_row);
}

ssgd_status zeros(int64_t M, int64_t N, void* out, int32_t out_dtype, int64_t out_pitch, hipStream_t stream) {
    const dim3 grid(1024);
    if (out_dtype == SSGD_F32) hipLaunchKernelGGL((zero_kernel<float>), grid, dim3(256), 0, stream, static_cast<float*>(out), M, N, out_pitch);
    else hipLaunchKernelGGL((zero_kernel<bf16_t>), grid, dim3(256), 0, stream, static_cast<bf16_t*>(out), M, N, out_pitch);
    return op_hip(hipGetLastError(), "mx product");
}

ssgd_status product(const Product& p, int32_t a_fmt, int32_t out_dtype, void* work, hipStream_t stream) {
    if (a_fmt == SSGD_MX_FP4) { if (out_dtype == SSGD_F32) launch<SSGD_MX_FP4, float>(p, work, stream); else launch<SSGD_MX_FP4, bf16_t>(p, work, stream); }
    else { if (out_dtype == SSGD_F32) launch<SSGD_MX_FP8, float>(p, work, stream); else launch<SSGD_MX_FP8, bf16_t>(p, work, stream); }
    return op_hip(hipGetLastError(), "mx product");
}

template <typename X>
void one_row_of(const Product& p, const Rows& x, int32_t a_fmt, int32_t out_dtype, hipStream_t stream) {
    if (a_fmt == SSGD_MX_FP4) { if (out_dtype == SSGD_F32) one_row<SSGD_MX_FP4, X>(p, x, To<float>{}, stream); else one_row<SSGD_MX_FP4, X>(p, x, To<bf16_t>{}, stream); }
    else { if (out_dtype == SSGD_F32) one_row<SSGD_MX_FP8, X>(p, x, To<float>{}, stream); else one_row<SSGD_MX_FP8, X>(p, x, To<bf16_t>{}, stream); }
}

// `itself`: the product quantises its rows.
const char* refused(int32_t a_fmt, int64_t M, const void* b_values, const void* b_scales, int64_t N, int64_t K, const void* out, int32_t out_dtype, int64_t out_pitch, bool itself) {
    if (!format_ok(a_fmt) || !dtype_ok(out_dtype)) return "mx product: a format and an output type of the enumerations";
    if (!sizes_ok(a_fmt, M, N, K) || out_pitch < N) return "mx product: M and N from zero to 2^31, K to 2^24 - 128, pitch >= N";
    if (M == 0 || N == 0) return nullptr;
    // (a launch ends at 2^32 threads; what it has follows from the kernel, and is in question only where there are many results)
    const int64_t tiles = (M + 127) / 128 * ((N + 127) / 128);
    if (tiles > kMostBlocks || (K > 0 && tiles > kMostBlocks / 16 && threads_of(a_fmt, M, N, K, itself) >> 32 != 0)) return "mx product: too many results";
    if (K > 0 && (!b_values || !b_scales || !aligned(b_values, 16) || !aligned(b_scales, 16))) return "mx product: values and scales are 16-byte aligned arrays";
    if (!out || !aligned(out, (uintptr_t)dtype_bytes(out_dtype))) return "mx product: the output is null or misaligned";
    return nullptr;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int64_t ssgd_mx_matmul_work_bytes(int32_t a_fmt, int64_t M, int64_t N, int64_t K) { return sizes_ok(a_fmt, M, N, K) ? parts_bytes(a_fmt, M, N, K) : -1; }

ssgd_status ssgd_mx_matmul(const void* a_values, const void* a_scales, int32_t a_fmt, int64_t M, const void* b_values, const void* b_scales, int64_t N, int64_t K,
                           void* out, int32_t out_dtype, int64_t out_pitch, void* work, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        if (const char* why = refused(a_fmt, M, b_values, b_scales, N, K, out, out_dtype, out_pitch, false)) return op_fail(SSGD_EINVAL, why);
        if (M == 0 || N == 0) return SSGD_OK;
        if (K > 0 && (!a_values || !a_scales || !aligned(a_values, 16) || !aligned(a_scales, 16))) return op_fail(SSGD_EINVAL, "mx product: values and scales are 16-byte aligned arrays");
        if ((!work || !aligned(work, 16)) && parts_bytes(a_fmt, M, N, K) > 0) return op_fail(SSGD_EINVAL, "mx product: a 16-byte aligned work area");
        const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        if (K == 0) return zeros(M, N, out, out_dtype, out_pitch, stream);
        return product(product_of(a_values, a_scales, a_fmt, M, b_values, b_scales, N, K, out, out_pitch), a_fmt, out_dtype, work, stream);
    });
}

int64_t ssgd_mx_linear_work_bytes(int32_t a_fmt, int64_t M, int64_t N, int64_t K) {
    if (!sizes_ok(a_fmt, M, N, K)) return -1;
    return quantises_itself(a_fmt, M, K) ? 0 : parts_bytes(a_fmt, M, N, K) + (M * (mx_row_bytes(a_fmt, K) + mx_padded(K) / kMxBlock) + 15) / 16 * 16;
}

ssgd_status ssgd_mx_linear(const void* x, int32_t dtype, int64_t pitch, int64_t M, int32_t a_fmt, const void* b_values, const void* b_scales, int64_t N, int64_t K,
                           void* out, int32_t out_dtype, int64_t out_pitch, void* work, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        const bool itself = sizes_ok(a_fmt, M, N, K) && quantises_itself(a_fmt, M, K);
        if (const char* why = refused(a_fmt, M, b_values, b_scales, N, K, out, out_dtype, out_pitch, itself)) return op_fail(SSGD_EINVAL, why);
        if (M == 0 || N == 0) return SSGD_OK;
        const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        if (K == 0) return zeros(M, N, out, out_dtype, out_pitch, stream);
        if (itself) {
            if (!dtype_ok(dtype) || pitch < K) return op_fail(SSGD_EINVAL, "mx linear: a type of the enumeration, pitch >= K");
            if (!x || !aligned(x, (uintptr_t)dtype_bytes(dtype))) return op_fail(SSGD_EINVAL, "mx linear: the rows are null or misaligned");
            const Product p = product_of(nullptr, nullptr, a_fmt, M, b_values, b_scales, N, K, out, out_pitch);
            const Rows rows{x, pitch, K};
            if (dtype == SSGD_F32) one_row_of<float>(p, rows, a_fmt, out_dtype, stream); else one_row_of<bf16_t>(p, rows, a_fmt, out_dtype, stream);
            return op_hip(hipGetLastError(), "mx linear");
        }
        if (!work || !aligned(work, 16)) return op_fail(SSGD_EINVAL, "mx linear: a 16-byte aligned work area");
        // values and scales in front (whole multiples of 16 bytes in all), then the parts
        const int64_t value_bytes = M * mx_row_bytes(a_fmt, K), all = (value_bytes + M * (mx_padded(K) / kMxBlock) + 15) / 16 * 16;
        uint8_t *values = static_cast<uint8_t*>(work), *scales = values + value_bytes;
        const ssgd_status st = ssgd_mx_quantize(x, dtype, M, K, pitch, a_fmt, values, scales, 0, nullptr, nullptr, hip_stream);
        if (st != SSGD_OK) return st;
        return product(product_of(values, scales, a_fmt, M, b_values, b_scales, N, K, out, out_pitch), a_fmt, out_dtype, values + all, stream);
    });
}

}  // extern "C"
#pragma GCC visibility pop
