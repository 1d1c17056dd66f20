// Product of microscaled matrices with a dense layer's epilogue, or with that of a gated feed-forward block:
//
//   p = A B^T + bias          out[m][n] = residual + act(p[m][n])          or          out[m][c] = act(p[m][2 c]) p[m][2 c + 1]
//
// The kernels of the product (mx_product.hpp) hand their sums over, eight columns of a row to a lane, so a gate and what it multiplies are
// neighbours; p is kept for the backward pass where that is wanted, and each of the two outputs goes out as a matrix or quantised to 8 bits
// without a rounding in between.  Where a workgroup does not have the whole sum (contractions in parts) or a block of 32 columns (few rows), fp32
// sums go to a work area and a second launch finishes them.
//
// Bound by the product: 8192^3 in 8 by 4 bits, normal numbers, takes 379 us without an epilogue, 388 with a bias, 387 with relu, 396 with silu, 409 with gelu, 398 with a residual and 416
// with bias, gelu and residual; gated 382 without an activation, 389 with silu, 401 with 8-bit output and p kept in 8 bits (8192 x 16384 x 4096, with twice the results: 406 and 452); another run's clock
// or inputs make all of them up to 5 % more (421 to 441 for the first with bias, gelu and residual).
// What an epilogue adds is memory that waits (all CUs come to it at the same time) and gelu's 26 instructions a value, two of them at a quarter of the rate.
#include "activations.hpp"
#include "mx_product.hpp"

using namespace ssgd;

namespace {

struct Held { void* to; uint8_t *values, *scales; int64_t pitch, value_bytes, scale_bytes; int32_t bf16; };      // a matrix, or microscaled, or nothing

struct Common {
    const void *bias, *residual;
    Held out, kept;
    int64_t residual_pitch, rows, cols, results;      // cols: of the product, results: of the output
    int32_t activation, gated, bias_bf16, residual_bf16;

    template <int V>
    static __device__ __forceinline__ void load(const void* from, int bf16, int64_t at, int64_t left, float (&x)[V]) {
        if (bf16) load_vec<V>(static_cast<const bf16_t*>(from) + at, left, x);
        else load_vec<V>(static_cast<const float*>(from) + at, left, x);
    }
    template <int V>
    static __device__ __forceinline__ void store(const Held& h, int64_t m, int64_t n, int64_t left, const float (&x)[V]) {
        if (left <= 0) return;
        if (h.bf16) store_vec<V>(static_cast<bf16_t*>(h.to) + m * h.pitch + n, left, x);
        else store_vec<V>(static_cast<float*>(h.to) + m * h.pitch + n, left, x);
    }
    // The bias of eight columns, and their sums with it: nothing where there are no columns.
    __device__ __forceinline__ void bias_of(int64_t n, float (&b)[8]) const {
        if (bias != nullptr) load<8>(bias, bias_bf16, n, cols - n, b);
    }
    __device__ __forceinline__ void add_bias(int64_t n, const float (&b)[8], float (&p)[8]) const {
        if (bias != nullptr) {
#pragma unroll
            for (int q = 0; q < 8; ++q) p[q] += b[q];
        }
        if (n + 8 > cols) {
#pragma unroll
            for (int q = 0; q < 8; ++q) p[q] = n + q < cols ? p[q] : 0.0f;
        }
    }
    // Eight columns from n on, of `width` that there are; four lanes side by side have a block.  STREAM: past the caches' replacement (with bias, gelu
    // and residual 8192^3 takes 416 us instead of 428, 8192 x 16384 x 4096 takes 495 instead of 514; gated products take the same time either way).
    template <bool STREAM>
    static __device__ __forceinline__ void store8(const Held& h, int64_t m, int64_t n, int64_t width, bool live, const float (&x)[8]) {
        if (h.values != nullptr) {
            const uint32_t byte = mx_scale_byte<SSGD_MX_FP8>(max_of_4(largest_of(x)));
            if (live && n < h.value_bytes) {
                words2* to = reinterpret_cast<words2*>(h.values + m * h.value_bytes + n);
                if constexpr (STREAM) __builtin_nontemporal_store(mx_pack_fp8(x, byte), to);
                else *to = mx_pack_fp8(x, byte);
                if ((threadIdx.x & 3) == 0) h.scales[m * h.scale_bytes + n / kMxBlock] = (uint8_t)byte;
            }
        } else if (h.to != nullptr && live && n < width) {
            if constexpr (!STREAM) store<8>(h, m, n, width - n, x);
            else if (h.bf16) stream_vec(static_cast<bf16_t*>(h.to) + m * h.pitch + n, width - n, x);
            else stream_vec(static_cast<float*>(h.to) + m * h.pitch + n, width - n, x);
        }
    }
    // Four results of eight columns.
    __device__ __forceinline__ void gate(const float (&p)[8], float (&h)[4]) const {
#pragma unroll
        for (int q = 0; q < 4; ++q) h[q] = p[2 * q];
        activate(activation, h);
#pragma unroll
        for (int q = 0; q < 4; ++q) h[q] *= p[2 * q + 1];
    }
    // Few rows: four columns, outputs as matrices.
    __device__ __forceinline__ void four(int64_t m, int64_t n, const f32x4& sum) const {
        if (m >= rows || n >= cols) return;
        float p[4] = {sum.x, sum.y, sum.z, sum.w};
        if (bias != nullptr) {
            float b[4];
            load<4>(bias, bias_bf16, n, cols - n, b);
#pragma unroll
            for (int q = 0; q < 4; ++q) p[q] += b[q];
        }
        if (kept.to != nullptr) store<4>(kept, m, n, cols - n, p);
        if (gated) {
            float h[2] = {p[0], p[2]};
            activate(activation, h);
            h[0] *= p[1]; h[1] *= p[3];
            const int64_t at = m * out.pitch + n / 2;
            const bool both = n + 2 < cols;
            if (out.bf16) {
                bf16_t* to = static_cast<bf16_t*>(out.to) + at;
                const uint32_t w = pack_bf16(h[0], h[1]);
                to[0] = (bf16_t)w;
                if (both) to[1] = (bf16_t)(w >> 16);
            } else {
                float* to = static_cast<float*>(out.to) + at;
                to[0] = h[0];
                if (both) to[1] = h[1];
            }
            return;
        }
        activate(activation, p);
        if (residual != nullptr) {
            float r[4];
            load<4>(residual, residual_bf16, m * residual_pitch + n, cols - n, r);
#pragma unroll
            for (int q = 0; q < 4; ++q) p[q] += r[q];
        }
        store<4>(out, m, n, cols - n, p);
    }
};

template <bool GATED>
struct Epilogue : Common {
    static constexpr bool kStores = false;
    // Columns that the tiles cover: the padding of outputs in 8 bits too.
    int64_t wide() const {
        int64_t n = cols;
        if (kept.values != nullptr && mx_padded(cols) > n) n = mx_padded(cols);
        if (out.values != nullptr && mx_padded(results) * (GATED ? 2 : 1) > n) n = mx_padded(results) * (GATED ? 2 : 1);
        return n;
    }
    // What eight columns of a row need before their sums are there: the residual in bf16 as it comes (in fp32 it would take twice the registers, and is read when it is used).
    static constexpr bool kAhead = !GATED;
    struct Nothing {};
    using Raw = std::conditional_t<GATED, Nothing, words4>;
    __device__ __forceinline__ void ahead(int64_t m, int64_t n, Raw& r) const {
        if constexpr (!GATED) {
            r = words4{0u, 0u, 0u, 0u};
            if (residual == nullptr || !residual_bf16 || m >= rows || n >= cols) return;
            Eight<bf16_t> x;
            x.load_own<false>(static_cast<const bf16_t*>(residual) + m * residual_pitch, n, cols);
            r = x.w;
        }
    }
    __device__ __forceinline__ void add_residual(int64_t m, int64_t n, const Raw& r, float (&p)[8]) const {
        float x[8];
        if (residual_bf16) {
            Eight<bf16_t> e;
            e.w = r;
            e.numbers(x);
        } else load_vec<8>(static_cast<const float*>(residual) + m * residual_pitch + n, m < rows ? cols - n : 0, x);
#pragma unroll
        for (int q = 0; q < 8; ++q) p[q] += x[q];
    }
    // Eight columns of p, with what `ahead` has brought, to eight results, or four, and these to their output; p itself to where it is kept.  Lanes side by side have
    // columns side by side, whole blocks of them.
    __device__ __forceinline__ void results_of(int64_t m, int64_t n, const Raw& r, float (&p)[8]) const {
        if constexpr (!GATED) {
            activate(activation, p);
            if (residual != nullptr) add_residual(m, n, r, p);
        } else {
            float h[4];
            gate(p, h);
#pragma unroll
            for (int q = 0; q < 4; ++q) p[q] = h[q];
        }
    }
    __device__ __forceinline__ void store_results(int64_t m, int64_t n, const float (&p)[8]) const {
        const bool live = m < rows;
        if constexpr (!GATED) store8<true>(out, m, n, cols, live, p);
        else {
            const float h[4] = {p[0], p[1], p[2], p[3]};
            const int64_t c = n / 2;
            if (out.values != nullptr) {
                uint32_t most = 0;
#pragma unroll
                for (int q = 0; q < 4; ++q) most = umax(most, magnitude(h[q]));
                const uint32_t byte = mx_scale_byte<SSGD_MX_FP8>(max_of_8(most));
                if (live && c < out.value_bytes) {
                    *reinterpret_cast<uint32_t*>(out.values + m * out.value_bytes + c) = mx_pack_fp8(h[0], h[1], h[2], h[3], byte);
                    if ((threadIdx.x & 7) == 0) out.scales[m * out.scale_bytes + c / kMxBlock] = (uint8_t)byte;
                }
            } else if (live) store<4>(out, m, c, results - c, h);
        }
    }
    __device__ __forceinline__ bool keeps() const { return kept.to != nullptr || kept.values != nullptr; }
    __device__ __forceinline__ void keep(int64_t m, int64_t n, const float (&p)[8]) const { store8<!GATED>(kept, m, n, cols, m < rows, p); }
};

// The parts of a contraction (none: a contraction of no columns), added in order, and the epilogue: eight columns a thread.
template <bool GATED>
__global__ __launch_bounds__(256) void finish_kernel(const float* parts, int32_t n, int64_t stride, Epilogue<GATED> e, int64_t groups, int64_t per_row) {
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= groups) return;                 // (rows have a multiple of 16 groups, gated 32: whole blocks)
    const int64_t row = u / per_row, col = (u - row * per_row) * 8;
    float p[8], b[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) p[q] = 0.0f;
    typename Epilogue<GATED>::Raw r;
    e.ahead(row, col, r);
    e.bias_of(col, b);
    const float* at = parts + row * e.cols + col;
    float x[8][8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) load_vec<8>(at + k * stride, e.cols - col, x[k]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (k >= n) break;
#pragma unroll
        for (int q = 0; q < 8; ++q) p[q] += x[k][q];
    }
    e.add_bias(col, b, p);
    e.keep(row, col, p);
    e.results_of(row, col, r, p);
    e.store_results(row, col, p);
}

// ---- host --------------------------------------------------------------------------------------------------------------
// How a product with an epilogue goes: the rows quantised in the product or before it, the sums finished where they are or through `parts` sets of
// fp32 sums in the work area.
struct Way { bool itself, few; int parts; int64_t row_bytes, part_bytes; };
Way way_of(int32_t a_fmt, bool from_rows, bool eight_bits, int64_t M, int64_t N, int64_t K) {
    Way w{};
    const int64_t steps = mx_padded(K) / kMxPad;
    w.itself = from_rows && quantises_itself(a_fmt, M, K);
    w.few = takes_few_rows(a_fmt, M, N, steps);
    if (K == 0) w.parts = 0;
    else if (w.few || w.itself) w.parts = eight_bits ? 1 : 0;
    else { const int n = tiling_of(a_fmt, M, N, steps).parts; w.parts = n > 1 ? n : 0; }
    if (from_rows && !w.itself && K > 0) w.row_bytes = (M * (mx_row_bytes(a_fmt, K) + mx_padded(K) / kMxBlock) + 15) / 16 * 16;
    w.part_bytes = w.parts * M * N * 4;
    return w;
}

// What finishes sums covers: the padding of outputs in 8 bits too.
int64_t finish_columns(int64_t results, bool gated) { return (gated ? 2 : 1) * mx_padded(results); }
template <bool GATED>
void finish(const Common& e, const float* parts, int n, hipStream_t s) {
    const int64_t per_row = finish_columns(e.results, GATED) / 8, groups = e.rows * per_row;
    hipLaunchKernelGGL((finish_kernel<GATED>), dim3((unsigned)((groups + 255) / 256)), dim3(256), 0, s, parts, n, e.rows * e.cols, Epilogue<GATED>{e}, groups, per_row);
}

// The product, its results to Out.
template <int FA, typename Out>
void few_with(const Way& w, const Product& p, const Rows& x, int32_t dtype, const Out& out, hipStream_t s) {
    if (!w.itself) few_rows_of<FA>(p, out, s);
    else if (dtype == SSGD_F32) one_row<FA, float>(p, x, out, s);
    else one_row<FA, bf16_t>(p, x, out, s);
}

template <int FA>
void launch(const Way& w, Product p, const Rows& x, int32_t dtype, const Common& e, float* sums, hipStream_t s) {
    if (p.steps == 0) { if (e.gated) finish<true>(e, nullptr, 0, s); else finish<false>(e, nullptr, 0, s); return; }
    int n = w.parts;
    if (n > 0) { p.out = sums; p.pitch = p.b.rows; p.part_stride = p.a.rows * p.b.rows; }
    if (w.few || w.itself) {
        if (n > 0) few_with<FA>(w, p, x, dtype, To<float>{}, s);
        else few_with<FA>(w, p, x, dtype, Epilogue<false>{e}, s);
    } else {
        const Tiling how = tiling_of(FA, p.a.rows, p.b.rows, p.steps);
        if (n > 0) {
            p.part_steps = (p.steps + n - 1) / n;
            n = (p.steps + p.part_steps - 1) / p.part_steps;
            tiles_of<FA>(how.rows, p, To<float>{}, s);
        } else if (e.gated) tiles_of<FA>(how.rows, p, Epilogue<true>{e}, s);
        else tiles_of<FA>(how.rows, p, Epilogue<false>{e}, s);
    }
    if (n > 0) { if (e.gated) finish<true>(e, sums, n, s); else finish<false>(e, sums, n, s); }
}

bool place_ok(const void* p, int32_t dtype) { return aligned(p, (uintptr_t)dtype_bytes(dtype)); }
// An output: nothing (where that is allowed), a matrix, or values and scales.
const char* held_ok(const void* to, int32_t dtype, int64_t pitch, const void* values, const void* scales, int64_t cols, bool optional) {
    if ((values != nullptr) != (scales != nullptr) || (to != nullptr && values != nullptr)) return "mx dense: an output is a matrix, or values and scales";
    if (!optional && to == nullptr && values == nullptr) return "mx dense: no output";
    if (to != nullptr && (!dtype_ok(dtype) || !place_ok(to, dtype) || pitch < cols)) return "mx dense: outputs have a type of the enumeration, its alignment and pitch >= columns";
    if (values != nullptr && (!aligned(values, 16) || !aligned(scales, 16))) return "mx dense: values and scales are 16-byte aligned";
    return nullptr;
}
Held held_of(void* to, int32_t dtype, int64_t pitch, void* values, void* scales, int64_t cols) {
    return {to, static_cast<uint8_t*>(values), static_cast<uint8_t*>(scales), pitch, mx_row_bytes(SSGD_MX_FP8, cols), mx_padded(cols) / kMxBlock, dtype == SSGD_BF16};
}

const char* refused(const void* x, int32_t dtype, int64_t pitch, const void* a_values, const void* a_scales, int32_t a_fmt, int64_t M, const void* b_values, const void* b_scales, int64_t N,
                    int64_t K, const ssgd_mx_epilogue& e) {
    if (!format_ok(a_fmt) || !sizes_ok(a_fmt, M, N, K)) return "mx dense: a format of the enumeration, M and N from zero to 2^31, K to 2^24 - 128";
    if ((e.gated != 0 && e.gated != 1) || e.activation < SSGD_ACT_NONE || e.activation > SSGD_ACT_SILU) return "mx dense: an activation of the enumeration, gated or not";
    if (e.gated && (N % 2 != 0 || e.bias != nullptr || e.residual != nullptr)) return "mx dense: a gated product has an even number of columns, no bias and no residual";
    if (M == 0 || N == 0) return nullptr;
    const int64_t results = e.gated ? N / 2 : N;
    if (const char* why = held_ok(e.out, e.out_dtype, e.out_pitch, e.values, e.scales, results, false)) return why;
    if (const char* why = held_ok(e.kept, e.kept_dtype, e.kept_pitch, e.kept_values, e.kept_scales, N, true)) return why;
    if (e.bias != nullptr && (!dtype_ok(e.bias_dtype) || !place_ok(e.bias, e.bias_dtype))) return "mx dense: a bias has a type of the enumeration and its alignment";
    if (e.residual != nullptr && (!dtype_ok(e.residual_dtype) || !place_ok(e.residual, e.residual_dtype) || e.residual_pitch < N))
        return "mx dense: a residual has a type of the enumeration, its alignment and pitch >= columns";
    // (a launch ends at 2^32 threads: tiles of the product with the padding of its outputs, and what finishes eight columns a thread)
    const Way w = way_of(a_fmt, x != nullptr, e.values != nullptr || e.kept_values != nullptr, M, N, K);
    const int64_t wide = finish_columns(results, e.gated != 0);
    if (K > 0 && (w.few || w.itself)) { if (threads_of(a_fmt, M, N, K, w.itself) >> 32 != 0) return "mx dense: too many results"; }
    else if (K > 0) {
        const int rows = tiling_of(a_fmt, M, N, mx_padded(K) / kMxPad).rows, across = rows == 256 ? 256 : 128;
        if ((M + rows - 1) / rows * ((wide + across - 1) / across) > kMostBlocks) return "mx dense: too many results";
    }
    if ((K == 0 || w.parts > 0) && M > kMostBlocks * 256 / (wide / 8)) return "mx dense: too many results";
    if (K == 0) return nullptr;
    if (!b_values || !b_scales || !aligned(b_values, 16) || !aligned(b_scales, 16)) return "mx dense: values and scales are 16-byte aligned arrays";
    if (x != nullptr) {
        if (a_values != nullptr || a_scales != nullptr) return "mx dense: either rows, or their values and scales";
        if (!dtype_ok(dtype) || !place_ok(x, dtype) || pitch < K) return "mx dense: rows have a type of the enumeration, its alignment and pitch >= K";
    } else if (!a_values || !a_scales || !aligned(a_values, 16) || !aligned(a_scales, 16)) return "mx dense: values and scales are 16-byte aligned arrays";
    return nullptr;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int64_t ssgd_mx_dense_work_bytes(int32_t a_fmt, int32_t from_rows, int32_t eight_bits, int64_t M, int64_t N, int64_t K) {
    if (!sizes_ok(a_fmt, M, N, K)) return -1;
    const Way w = way_of(a_fmt, from_rows != 0, eight_bits != 0, M, N, K);
    return w.row_bytes + w.part_bytes;
}

ssgd_status ssgd_mx_dense(const void* x, int32_t dtype, int64_t pitch, const void* a_values, const void* a_scales, int32_t a_fmt, int64_t M, const void* b_values, const void* b_scales,
                          int64_t N, int64_t K, const ssgd_mx_epilogue* epilogue, void* work, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        if (epilogue == nullptr) return op_fail(SSGD_EINVAL, "mx dense: no epilogue");
        const ssgd_mx_epilogue& o = *epilogue;
        if (const char* why = refused(x, dtype, pitch, a_values, a_scales, a_fmt, M, b_values, b_scales, N, K, o)) return op_fail(SSGD_EINVAL, why);
        if (M == 0 || N == 0) return SSGD_OK;
        const Way w = way_of(a_fmt, x != nullptr, o.values != nullptr || o.kept_values != nullptr, M, N, K);
        if (w.row_bytes + w.part_bytes > 0 && (!work || !aligned(work, 16))) return op_fail(SSGD_EINVAL, "mx dense: a 16-byte aligned work area");
        const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        Common e{};
        e.bias = o.bias; e.residual = o.residual; e.residual_pitch = o.residual_pitch;
        e.rows = M; e.cols = N; e.results = o.gated ? N / 2 : N;
        e.out = held_of(o.out, o.out_dtype, o.out_pitch, o.values, o.scales, e.results);
        e.kept = held_of(o.kept, o.kept_dtype, o.kept_pitch, o.kept_values, o.kept_scales, N);
        e.activation = o.activation; e.gated = o.gated; e.bias_bf16 = o.bias_dtype == SSGD_BF16; e.residual_bf16 = o.residual_dtype == SSGD_BF16;
        // values and scales of rows in front, then the sums
        if (w.row_bytes > 0) {
            uint8_t* room = static_cast<uint8_t*>(work);
            a_values = room; a_scales = room + M * mx_row_bytes(a_fmt, K);
            const ssgd_status st = ssgd_mx_quantize(x, dtype, M, K, pitch, a_fmt, room, room + M * mx_row_bytes(a_fmt, K), 0, nullptr, nullptr, hip_stream);
            if (st != SSGD_OK) return st;
        }
        const Product p = product_of(a_values, a_scales, a_fmt, M, b_values, b_scales, N, K, nullptr, 0);
        float* sums = reinterpret_cast<float*>(static_cast<uint8_t*>(work) + w.row_bytes);
        if (a_fmt == SSGD_MX_FP4) launch<SSGD_MX_FP4>(w, p, Rows{x, pitch, K}, dtype, e, sums, stream);
        else launch<SSGD_MX_FP8>(w, p, Rows{x, pitch, K}, dtype, e, sums, stream);
        return op_hip(hipGetLastError(), "mx dense");
    });
}

}  // extern "C"
#pragma GCC visibility pop
