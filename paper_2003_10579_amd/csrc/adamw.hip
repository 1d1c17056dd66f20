// AdamW over many tensors in one launch (two with clipping), moments in 32 or 8 bits.
//
// Per element: 28 bytes with fp32 moments and gradients (p, m, v read and written, g read), 16.1 with 8-bit moments and fp32
// gradients, 14.1 with bf16 ones; clipping reads the gradients a second time.  About 20 operations an element: bound by memory.  Tensors are cut
// into pieces of 8192 elements, a workgroup each, from a table made with the handle; what changes from call to call, the
// gradients' addresses, travels in the kernel's arguments, so a step copies nothing and has no host work per piece.
#include <cmath>
#include <vector>

#include "ops.hpp"

using namespace ssgd;

namespace {

constexpr int kThreads = 256;
// Elements of a workgroup: 8192, or 2048 where that leaves fewer than four workgroups per CU (1.58 M parameters: 7.1 us instead of 11.2).
constexpr int kPiece = 8192, kSmallPiece = 2048;
constexpr int64_t kFewElements = int64_t(4) * 256 * kPiece;
constexpr int kStateBlock = 128;         // elements per scale of an 8-bit moment
constexpr int kTensorsPerLaunch = 384;   // gradient addresses in the kernel's arguments
constexpr int kPartials = 1024;          // sums of squares, over all launches of a step (more only where there are more launches)

struct Piece {
    float* p;
    bf16_t* copy;
    int64_t state;      // place of its first element in the moments
    int64_t first;      // of its tensor
    int32_t n;
    int32_t tensor;     // of its launch
    float decay;
    int32_t pad;
};

template <typename G>
struct Grads { const G* of[kTensorsPerLaunch]; };

struct Rule {
    float beta1, rest1, beta2, rest2, eps, lr, step, root_scale, max_norm;
    uint32_t key;
    void *m, *v;
    float *m_scale, *v_scale;
    const double* partials;
    int32_t n_partials;
    float* norm_out;
};

// Two rounds of a shifted exclusive or and an odd factor (2^32 over the golden ratio; the fraction of the root of 3).
__host__ __device__ inline uint32_t mix(uint32_t x) {
    x ^= x >> 16; x *= 0x9E3779B1u;
    x ^= x >> 15; x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

// A magnitude of at most 448 on the grid of E4M3, up with the probability of what is cut off; `dither` has 16 bits.  From 2^-6 on
// the grid is the top 12 bits of the number; below, where it is even, 2^-6 is added first, which puts the same 20 bits under it.
__device__ __forceinline__ float dithered(float a, uint32_t dither) {
    const float lift = a < 0x1p-6f ? 0x1p-6f : 0.0f;
    const uint32_t u = __builtin_bit_cast(uint32_t, a + lift) + (dither << 4);
    return fminf(__builtin_bit_cast(float, u & 0xFFF00000u) - lift, 448.0f);
}

// Eight values of a block that sixteen lanes share -> bytes and scale.
template <bool FLOOR>
__device__ __forceinline__ words2 round_block(const float (&x)[8], const uint32_t (&dither)[8], float* scale) {
    uint32_t most = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) most = umax(most, magnitude(x[q]));
    const float amax = __builtin_bit_cast(float, max_of_16(most));
    const bool some = !(amax < 0x1p-100f);
    const float inv = some ? (1.0f / amax) * 448.0f : 0.0f;
    *scale = some ? amax * (1.0f / 448.0f) : 0.0f;
    float y[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const float a = fabsf(x[q]) * inv;
        float r = dithered(a, dither[q]);
        if (FLOOR) r = a > 0.0f ? fmaxf(r, 0x1p-9f) : r;
        r = a != a ? a : r;
        y[q] = copysignf(r, x[q]);
    }
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], lo, false); lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], hi, false); hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
    return words2{(uint32_t)lo, (uint32_t)hi};
}

__device__ __forceinline__ void unpack_fp8(words2 w, float scale, float (&x)[8]) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, true);
    const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, true);
    x[0] = a.x * scale; x[1] = a.y * scale; x[2] = b.x * scale; x[3] = b.y * scale;
    x[4] = c.x * scale; x[5] = c.y * scale; x[6] = d.x * scale; x[7] = d.y * scale;
}

// Sum of squares of the pieces of a launch, in fp64 (fp32 squares overflow from 1.8e19 on), one number per workgroup.  Bound by memory: 268 M bf16
// gradients 138 us, 3.9 TB/s, behind an update that left the caches full of lines to be written back.
template <typename G>
__global__ __launch_bounds__(kThreads) void square_kernel(const Piece* pieces, int32_t n_pieces, Grads<G> grads, double* partials) {
    __shared__ double part[kThreads / 64];
    double sum = 0.0;
    for (int c = blockIdx.x; c < n_pieces; c += gridDim.x) {
        const Piece w = pieces[c];
        const G* g = grads.of[w.tensor] + w.first;
        for (int i = threadIdx.x * 8; i < w.n; i += kThreads * 32) {
            Eight<G> four[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) four[u].template load_own<false>(g, i + u * kThreads * 8, w.n);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float x[8];
                four[u].numbers(x);
#pragma unroll
                for (int q = 0; q < 8; ++q) sum += (double)x[q] * (double)x[q];
            }
        }
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) partials[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// The factor of the gradients, the same in every workgroup: all add the same partial sums in the same order.
__device__ __forceinline__ float clip_factor(const Rule& rule, double* part) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < rule.n_partials; i += kThreads) sum += rule.partials[i];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    // (an fp64 root in every workgroup only where fp32 does not reach)
    const double all = (part[0] + part[1]) + (part[2] + part[3]);
    const float norm = all > 0x1p-100 && all < 0x1p127 ? sqrtf((float)all) : (float)sqrt(all);
    if (blockIdx.x == 0 && threadIdx.x == 0 && rule.norm_out != nullptr) *rule.norm_out = norm;
    const float c = rule.max_norm / (norm + 1e-6f);
    return c > 1.0f ? 1.0f : c;           // (a NaN stays)
}

// The update.  268 M parameters with bf16 gradients and copy: 1416 us with 32-bit moments (5.3 TB/s), 950 us with 8-bit ones (4.6 TB/s; 820 where no
// clipping has read the gradients before).  Four elements a thread at a time with 32-bit moments, so that a wave's accesses are whole lines; eight
// with 8-bit ones, so that sixteen lanes hold a block.
template <int BITS, typename G>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const Piece* pieces, int32_t n_pieces, Grads<G> grads, Rule rule) {
    constexpr int V = BITS == 8 ? 8 : 4;
    __shared__ double part[kThreads / 64];
    float clip = 1.0f;
    if (rule.max_norm > 0.0f) clip = clip_factor(rule, part);
    if ((int)blockIdx.x >= n_pieces) return;          // no elements at all: the norm alone
    const Piece w = pieces[blockIdx.x];
    const G* g = grads.of[w.tensor] + w.first;
    const float keep = 1.0f - rule.lr * w.decay;
    // (whole blocks of the moments: lanes past the end hold zeros)
    const int end = (w.n + kStateBlock - 1) / kStateBlock * kStateBlock;
    for (int i = threadIdx.x * V; i < end; i += kThreads * V) {
        const int left = w.n - i;
        const int64_t at = w.state + i;
        float p[V], gr[V], m[V], v[V];
        // (the gradients last: in bf16 they are waited for at once, and the others then arrive meanwhile)
        if constexpr (BITS == 32) {
            load_vec<V>(static_cast<const float*>(rule.m) + at, V, m);
            load_vec<V>(static_cast<const float*>(rule.v) + at, V, v);
            load_vec<V>(w.p + i, left, p);
            load_vec<V>(g + i, left, gr);
        } else {
            const words2 some_m = *reinterpret_cast<const words2*>(static_cast<const uint8_t*>(rule.m) + at), some_v = *reinterpret_cast<const words2*>(static_cast<const uint8_t*>(rule.v) + at);
            const float m_scale = rule.m_scale[at / kStateBlock], v_scale = rule.v_scale[at / kStateBlock];
            load_vec<V>(w.p + i, left, p);
            load_vec<V>(g + i, left, gr);
            unpack_fp8(some_m, m_scale, m);
            unpack_fp8(some_v, v_scale, v);
#pragma unroll
            for (int q = 0; q < V; ++q) v[q] = v[q] * v[q];
        }
        float root[V];
#pragma unroll
        for (int q = 0; q < V; ++q) {
            const float x = gr[q] * clip;
            m[q] = rule.beta1 * m[q] + rule.rest1 * x;
            v[q] = rule.beta2 * v[q] + rule.rest2 * (x * x);
            root[q] = sqrtf(v[q]);
            p[q] = p[q] * keep - rule.step * m[q] / (root[q] * rule.root_scale + rule.eps);
        }
        store_vec<V>(w.p + i, left, p);
        if (w.copy != nullptr) store_vec<V>(w.copy + i, left, p);
        if constexpr (BITS == 32) {
            if (left < V) {
#pragma unroll
                for (int q = 0; q < V; ++q) if (q >= left) { m[q] = 0.0f; v[q] = 0.0f; }
            }
            store_vec<V>(static_cast<float*>(rule.m) + at, V, m);
            store_vec<V>(static_cast<float*>(rule.v) + at, V, v);
        } else {
            uint32_t dm[8], dr[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                if (q >= left) { m[q] = 0.0f; root[q] = 0.0f; }
                const uint64_t place = (uint64_t)(at + q);
                const uint32_t h = mix(((uint32_t)place + (uint32_t)(place >> 32) * 0x9E3779B1u) ^ rule.key);
                dm[q] = h & 0xFFFFu; dr[q] = h >> 16;
            }
            float sm, sr;
            *reinterpret_cast<words2*>(static_cast<uint8_t*>(rule.m) + at) = round_block<false>(m, dm, &sm);
            *reinterpret_cast<words2*>(static_cast<uint8_t*>(rule.v) + at) = round_block<true>(root, dr, &sr);
            if ((threadIdx.x & 15) == 0) { rule.m_scale[at / kStateBlock] = sm; rule.v_scale[at / kStateBlock] = sr; }
        }
    }
}

struct Launch { int32_t first_tensor, tensors; int64_t first_piece; int32_t pieces, partials, first_partial; };

}  // namespace

struct ssgd_adamw {
    int device = 0;
    ssgd_adamw_options opt{};
    void *m = nullptr, *v = nullptr;
    float *m_scale = nullptr, *v_scale = nullptr;
    std::vector<Launch> launches;
    std::vector<int64_t> sizes;
    Piece* pieces = nullptr;      // device
    double* partials = nullptr;   // device
    int32_t n_partials = 0;
};

namespace {

template <typename G>
hipError_t step(const ssgd_adamw& h, const void* const* grads, Rule rule, hipStream_t s) {
    Grads<G> g{};
    const bool clip = rule.max_norm > 0.0f;
    for (int pass = clip ? 0 : 1; pass < 2; ++pass)
        for (const Launch& l : h.launches) {
            if (l.pieces == 0 && l.partials == 0) continue;
            for (int k = 0; k < l.tensors; ++k) g.of[k] = static_cast<const G*>(grads[l.first_tensor + k]);
            const Piece* pieces = h.pieces + l.first_piece;
            const dim3 grid(l.pieces > 0 ? l.pieces : 1);
            if (pass == 0) hipLaunchKernelGGL((square_kernel<G>), dim3(l.partials), dim3(kThreads), 0, s, pieces, l.pieces, g, h.partials + l.first_partial);
            else if (h.opt.state_bits == 8) hipLaunchKernelGGL((adamw_kernel<8, G>), grid, dim3(kThreads), 0, s, pieces, l.pieces, g, rule);
            else hipLaunchKernelGGL((adamw_kernel<32, G>), grid, dim3(kThreads), 0, s, pieces, l.pieces, g, rule);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

bool unit(double x) { return x >= 0.0 && x < 1.0; }

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int64_t ssgd_adamw_state_elements(int32_t tensors, const int64_t* sizes) {
    if (tensors < 1 || !sizes) return -1;
    int64_t total = 0;
    for (int32_t k = 0; k < tensors; ++k) {
        if (sizes[k] < 0 || sizes[k] > (int64_t(1) << 48)) return -1;
        total += (sizes[k] + kStateBlock - 1) / kStateBlock * kStateBlock;
        if (total > (int64_t(1) << 48)) return -1;
    }
    return total;
}

ssgd_status ssgd_adamw_create(int32_t tensors, const int64_t* sizes, float* const* params, void* const* copies, const double* weight_decay,
                              const ssgd_adamw_options* options, void* m, void* v, float* m_scale, float* v_scale, ssgd_adamw** out) {
    return op_entry([&]() -> ssgd_status {
        if (!params || !weight_decay || !options || !out) return op_fail(SSGD_EINVAL, "adamw: params, weight_decay, options and out must not be null");
        const int64_t total = ssgd_adamw_state_elements(tensors, sizes);
        if (total < 0) return op_fail(SSGD_EINVAL, "adamw: at least one tensor, sizes of zero or more");
        const ssgd_adamw_options o = *options;
        // (as the update has them, in fp32)
        const float eps = (float)o.eps, max_norm = (float)o.max_norm;
        if (!unit(o.beta1) || !unit(o.beta2) || !(eps > 0) || !std::isfinite(eps) || !(o.max_norm >= 0) || (max_norm == 0 && o.max_norm > 0) ||
            (o.state_bits != 8 && o.state_bits != 32))
            return op_fail(SSGD_EINVAL, "adamw: betas in [0, 1), eps > 0 and max_norm >= 0 as fp32 numbers, state_bits 8 or 32");
        if (total > 0 && (!m || !v || !aligned(m, 16) || !aligned(v, 16))) return op_fail(SSGD_EINVAL, "adamw: m and v must be 16-byte aligned device arrays");
        if (total > 0 && o.state_bits == 8 && (!m_scale || !v_scale)) return op_fail(SSGD_EINVAL, "adamw: 8-bit moments need m_scale and v_scale");
        const int64_t piece = total < kFewElements ? kSmallPiece : kPiece;
        if (total / piece + tensors > kMostBlocks) return op_fail(SSGD_EINVAL, "adamw: too many elements");
        for (int32_t k = 0; k < tensors; ++k) {
            if (sizes[k] > 0 && (!params[k] || !aligned(params[k], 4) || (copies && !aligned(copies[k], 2)))) return op_fail(SSGD_EINVAL, "adamw: a parameter pointer is null or misaligned");
            if (!std::isfinite(weight_decay[k])) return op_fail(SSGD_EINVAL, "adamw: a weight decay is no number");
        }
        struct Owner { ssgd_adamw* h; ~Owner() { if (h) ssgd_adamw_destroy(h); } } owner{new ssgd_adamw};
        ssgd_adamw* h = owner.h;
        h->opt = o; h->m = m; h->v = v; h->m_scale = m_scale; h->v_scale = v_scale;
        h->sizes.assign(sizes, sizes + tensors);
        std::vector<Piece> pieces;
        int64_t state = 0;
        for (int32_t k = 0; k < tensors; ++k) {
            if (k % kTensorsPerLaunch == 0) h->launches.push_back({k, 0, (int64_t)pieces.size(), 0, 0, 0});
            Launch& l = h->launches.back();
            for (int64_t first = 0; first < sizes[k]; first += piece) {
                bf16_t* copy = copies && copies[k] ? static_cast<bf16_t*>(copies[k]) + first : nullptr;
                const int64_t rest = sizes[k] - first;
                pieces.push_back({params[k] + first, copy, state + first, first, (int32_t)(rest < piece ? rest : piece), l.tensors, (float)weight_decay[k], 0});
                ++l.pieces;
            }
            ++l.tensors;
            state += (sizes[k] + kStateBlock - 1) / kStateBlock * kStateBlock;
        }
        const int share = kPartials / (int)h->launches.size() > 16 ? kPartials / (int)h->launches.size() : 16;
        for (Launch& l : h->launches) {
            l.partials = l.pieces < share ? l.pieces : share;
            l.first_partial = h->n_partials;
            h->n_partials += l.partials;
        }
        if (h->n_partials == 0) { h->launches[0].partials = 1; h->n_partials = 1; }      // nothing but empty tensors: their norm is zero
        ssgd_status st = op_hip(hipGetDevice(&h->device), "adamw: device");
        if (st == SSGD_OK) st = op_hip(hipMalloc(reinterpret_cast<void**>(&h->partials), sizeof(double) * h->n_partials), "adamw: work area");
        if (st == SSGD_OK) st = op_hip(hipMalloc(reinterpret_cast<void**>(&h->pieces), sizeof(Piece) * (pieces.empty() ? 1 : pieces.size())), "adamw: work area");
        if (st == SSGD_OK && !pieces.empty()) st = op_hip(hipMemcpy(h->pieces, pieces.data(), sizeof(Piece) * pieces.size(), hipMemcpyHostToDevice), "adamw: work area");
        if (st != SSGD_OK) return st;
        owner.h = nullptr;
        *out = h;
        return SSGD_OK;
    });
}

ssgd_status ssgd_adamw_step(ssgd_adamw* h, const void* const* grads, int32_t grad_dtype, double lr, int64_t t, float* norm_out, void* hip_stream) {
    return op_entry([&]() -> ssgd_status {
        if (!h || !grads) return op_fail(SSGD_EINVAL, "adamw step: handle and gradients must not be null");
        if (!dtype_ok(grad_dtype) || t < 1 || !std::isfinite(lr)) return op_fail(SSGD_EINVAL, "adamw step: a gradient type of the enumeration, t >= 1, a finite rate");
        for (size_t k = 0; k < h->sizes.size(); ++k)
            if (h->sizes[k] > 0 && (!grads[k] || !aligned(grads[k], (uintptr_t)dtype_bytes(grad_dtype)))) return op_fail(SSGD_EINVAL, "adamw step: a gradient pointer is null or misaligned");
        int dev = -1;
        const ssgd_status st = op_hip(hipGetDevice(&dev), "adamw step");
        if (st != SSGD_OK) return st;
        if (dev != h->device) return op_fail(SSGD_EINVAL, "adamw step: the handle belongs to another device");
        const ssgd_adamw_options& o = h->opt;
        Rule r{};
        r.beta1 = (float)o.beta1; r.rest1 = (float)(1.0 - o.beta1); r.beta2 = (float)o.beta2; r.rest2 = (float)(1.0 - o.beta2);
        r.eps = (float)o.eps; r.lr = (float)lr; r.max_norm = (float)o.max_norm;
        r.step = (float)(lr / (1.0 - std::pow(o.beta1, (double)t)));
        r.root_scale = (float)(1.0 / std::sqrt(1.0 - std::pow(o.beta2, (double)t)));
        r.key = mix((uint32_t)(o.seed >> 32) ^ mix((uint32_t)o.seed ^ mix((uint32_t)t)));
        r.m = h->m; r.v = h->v; r.m_scale = h->m_scale; r.v_scale = h->v_scale;
        r.partials = h->partials; r.n_partials = h->n_partials; r.norm_out = norm_out;
        const hipStream_t s = static_cast<hipStream_t>(hip_stream);
        return op_hip(grad_dtype == SSGD_F32 ? step<float>(*h, grads, r, s) : step<bf16_t>(*h, grads, r, s), "adamw step");
    });
}

void ssgd_adamw_destroy(ssgd_adamw* h) {
    if (!h) return;
    if (h->pieces) (void)hipFree(h->pieces);
    if (h->partials) (void)hipFree(h->partials);
    delete h;
}

}  // extern "C"
#pragma GCC visibility pop
