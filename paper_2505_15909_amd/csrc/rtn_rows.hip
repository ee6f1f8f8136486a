// Rows of activations in 8 bits: the residual's addition with the root-mean-square norm, the feed-forward's gated activation, and plain
// rows, quantised with a scale for each token (or, the first two, left in 16 bits).
//
// Every one of them is v_k times a factor of the row: v = h w with the factor rsqrt(mean(h^2) + eps) for the norm, v = act(a) b and v = x
// with 1.  The largest |v| and the sum of squares are found in one sweep and the codes are rne(v / (max|v| / 127)), which the factor does not
// enter; so a row is read once, kept in registers, and meets once over the workgroup, not once for the norm and again for the scale.
// Plain rows and their largest magnitude are exact, and h w is (two significands of at most 11 bits) unless it is below fp32's range; the step, its reciprocal and the value
// times that are one rounding in fp32 each, in the order that the header of the entry points gives: the codes of plain and normed rows and the scales of plain ones are what
// the same steps give anywhere else.  The norm's factor (sums in an order of their own, a reciprocal root to about one unit) and the gate (an exponential to about one unit)
// are not, nor what they enter: the norm's scales and 16-bit results, and all that a gate gives.
//
// Bound by memory: the norm with a residual moves 7 bytes an element quantised, the gated activation 5, plain rows 3 (8192 x 8192 in 82 us,
// 5.7 TB/s; 4096 x 28672 in 107 us, 5.5; 3001 x 16384 in 27.7, 5.3, where a copy of 1 GiB reaches 4.8 to 5.5).
#include "rtn_paged.h"

namespace rtn {

enum { ROW_PLAIN, ROW_NORM, ROW_SILU, ROW_GELU };

struct RowParams {
    const void *x, *residual, *weight;
    void *sum, *out;
    float* scales;
    int64_t x_stride, residual_stride, sum_stride;
    int rows, dim;
    float eps, inv_dim;
};

constexpr float kLeastRow = 0x1p-100f;                       // rows whose largest magnitude is below have scale 0 and codes 0

// Of values that are not negative, in every lane; NaN stays.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ float wave_total(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wave_scan(x)), 63));
}

__device__ __forceinline__ float wave_largest(float x) {
    x = larger(x, from_lane<0x111, 0xF>(x));
    x = larger(x, from_lane<0x112, 0xF>(x));
    x = larger(x, from_lane<0x114, 0xF>(x));
    x = larger(x, from_lane<0x118, 0xF>(x));
    x = larger(x, from_lane<0x142, 0xA>(x));
    x = larger(x, from_lane<0x143, 0xC>(x));
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

#pragma clang fp contract(off)

// exp(x) = 2^n 2^f with x log2(e) = n + f, reduced with the constant in two parts as Cody and Waite do it: what the product rounds off and log2(e)'s second part go into
// f, whose power the hardware has to about one unit.  No special cases within +-88.
__device__ __forceinline__ float exp_within_88(float x) {
    const float t = x * 1.44269504f, n = __builtin_rintf(t);
    const float rest = fmaf(x, 1.92596299e-8f, fmaf(x, 1.44269504f, -t));
    return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(t - n + rest), (int)n);
}

// a / d, rounded as a division is, for 1 <= d < 2^126: Newton's step on a reciprocal and one correction of the quotient (5 instructions, 10 with the scaling
// that a division of any two numbers needs).
__device__ __forceinline__ float quotient(float a, float d) {
    const float r0 = __builtin_amdgcn_rcpf(d), r = fmaf(fmaf(-d, r0, 1.0f), r0, r0), q = a * r;
    return fmaf(fmaf(-d, q, a), r, q);
}

// act(a) b.  Both activations are a / (1 + exp(-z)): z = a, or a (1 + 0.044715 a^2) sqrt(8 / pi), for which it is a / 2 (1 + tanh(z / 2)).  Below
// z = -87.33 the divisor is beyond 2^126, its reciprocal counts as 0 and so does the result, whose magnitude is at most 87.4 / 2^126 |b|.
template <bool GELU>
__device__ __forceinline__ float gated(float a, float b) {
    const float z = GELU ? a * (1.0f + 0.044715f * a * a) * 1.59576912f : a;
    return quotient(a, 1.0f + exp_within_88(__builtin_amdgcn_fmed3f(-z, -88.0f, 88.0f))) * b;
}

// Four codes of v * inv within +-127: adding 1.5 2^23 rounds to nearest even and leaves the code in the lowest byte.
__device__ __forceinline__ uint32_t four_codes(const float* v, float inv) {
    uint32_t t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = __builtin_bit_cast(uint32_t, v[i] * inv + 12582912.0f);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(t[3], t[2], 0x0C0C0400u), __builtin_amdgcn_perm(t[1], t[0], 0x0C0C0400u), 0x05040100u);
}

// 16-bit results, sums and the values of codes are stored as streaming: 8192 x 8192 normed and then dequantised 126 -> 112 us, 4096 x 28672 gated
// and dequantised 193 -> 172, 1897 x 5120 normed 7.7 -> 7.0.  Codes are not: they are few, and what reads them next finds them in the caches (3001 x 16384 quantised and
// dequantised 51, as streaming 55).  Streaming loads gained nothing in such pairs.
template <typename V>
__device__ __forceinline__ void store_out(void* at, V v) { __builtin_nontemporal_store(v, static_cast<V*>(at)); }

// T threads a row, C pieces of eight elements a thread; workgroups of at least 256 threads.
template <int TYPE, int OP, bool QUANT, int T, int C>
__global__ __launch_bounds__(T < 256 ? 256 : T) void rows_kernel(const RowParams p) {
    typedef typename Elem<TYPE>::one E;
    typedef typename Elem<TYPE>::x8 E8;
    constexpr int ROWS = T < 256 ? 256 / T : 1, WAVES = T / 64;
    constexpr bool GATED = OP == ROW_SILU || OP == ROW_GELU;
    __shared__ float part[2][WAVES];
    const int t = threadIdx.x % T, row = (int)blockIdx.x * ROWS + (int)threadIdx.x / T;
    if (row >= p.rows) return;                               // (a whole wavefront; with more wavefronts a row there is one row)
    const E* const x = static_cast<const E*>(p.x) + row * p.x_stride;
    // Everything is requested before the first store (which may be to the same memory).  What is kept for the second sweep: the elements, the
    // norm's with its weight; of the gated activation the values, whose exponentials are not formed twice.
    E8 in[C], with[C], weight[OP == ROW_NORM ? C : 1];
    float kept[GATED ? C : 1][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int k = (c * T + t) * 8;
        if (k >= p.dim) continue;
        in[c] = *reinterpret_cast<const E8*>(x + k);
        if constexpr (GATED) with[c] = *reinterpret_cast<const E8*>(x + p.dim + k);
        if constexpr (OP == ROW_NORM) {
            if (p.residual) with[c] = *reinterpret_cast<const E8*>(static_cast<const E*>(p.residual) + row * p.residual_stride + k);
            weight[c] = *reinterpret_cast<const E8*>(static_cast<const E*>(p.weight) + k);
        }
    }
    auto value = [&](int c, int i) -> float {
        if constexpr (GATED) return kept[c][i];
        else if constexpr (OP == ROW_NORM) return (float)in[c][i] * (float)weight[c][i];
        else return (float)in[c][i];
    };
    float square = 0.f, most = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int k = (c * T + t) * 8;
        if (k >= p.dim) continue;
        if constexpr (OP == ROW_NORM)
            if (p.residual) {
                // the sum is held in the type, as the next layer finds it, and what is held is normed
#pragma unroll
                for (int i = 0; i < 8; ++i) in[c][i] = (E)((float)in[c][i] + (float)with[c][i]);
                store_out(static_cast<E*>(p.sum) + row * p.sum_stride + k, in[c]);
            }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = (float)in[c][i];
            if constexpr (OP == ROW_NORM) square = fmaf(a, a, square);
            if constexpr (GATED) kept[c][i] = gated<OP == ROW_GELU>(a, (float)with[c][i]);
            if constexpr (QUANT) most = larger(most, fabsf(value(c, i)));
        }
    }
    if constexpr (OP == ROW_NORM) square = wave_total(square);
    if constexpr (QUANT) most = wave_largest(most);
    if constexpr (WAVES > 1 && (QUANT || OP == ROW_NORM)) {
        if (t % 64 == 0) {
            part[0][t / 64] = square;
            part[1][t / 64] = most;
        }
        __syncthreads();
        square = part[0][0];
        most = part[1][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) {
            square += part[0][w];
            most = larger(most, part[1][w]);
        }
    }
    float factor = 1.f;
    if constexpr (OP == ROW_NORM) {
        const float mean = fmaf(square, p.inv_dim, p.eps);
        factor = mean == 0.f ? 0.f : rsqrtf(mean);           // (a row of zeros without eps)
    }
    float inv = 0.f;
    if constexpr (QUANT) {
        const bool none = most < kLeastRow;
        const float step = most * (1.0f / 127.0f);
        inv = none ? 0.f : 1.0f / step;
        if (t == 0) p.scales[row] = none ? 0.f : step * factor;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int k = (c * T + t) * 8;
        if (k >= p.dim) continue;
        if constexpr (QUANT) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = value(c, i);
            const u32x2_t codes = {four_codes(v, inv), four_codes(v + 4, inv)};
            *reinterpret_cast<u32x2_t*>(static_cast<uint8_t*>(p.out) + (int64_t)row * p.dim + k) = codes;
        } else {
            E8 y;
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = (E)(value(c, i) * factor);
            store_out(static_cast<E*>(p.out) + (int64_t)row * p.dim + k, y);
        }
    }
}

// A thread has up to four pieces of eight codes of a row; segments of 8192 elements.
template <int TYPE>
__global__ __launch_bounds__(256) void dequantize_rows_kernel(const uint8_t* q, const float* scales, void* out, int dim, int segments) {
    typedef typename Elem<TYPE>::one E;
    typedef typename Elem<TYPE>::x8 E8;
    const int row = blockIdx.x / segments, segment = blockIdx.x - row * segments;
    const float s = scales[row];
    const int64_t at = (int64_t)row * dim;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int k = segment * 8192 + (c * 256 + (int)threadIdx.x) * 8;
        if (k >= dim) return;
        const u32x2_t codes = *reinterpret_cast<const u32x2_t*>(q + at + k);
        E8 y;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (E)((float)(int8_t)(codes[i / 4] >> (i % 4 * 8)) * s);
        store_out(static_cast<E*>(out) + at + k, y);
    }
}

template <int TYPE, int OP, bool QUANT, int T, int C>
static void launch_rows_as(const RowParams& p, hipStream_t st) {
    constexpr int ROWS = T < 256 ? 256 / T : 1;
    hipLaunchKernelGGL((rows_kernel<TYPE, OP, QUANT, T, C>), dim3((unsigned)((p.rows + ROWS - 1) / ROWS)), dim3(T < 256 ? 256 : T), 0, st, p);
}

template <int TYPE, int OP, bool QUANT>
static hipError_t launch_rows(const RowParams& p, hipStream_t st) {
    // About as many threads as a row has pieces, so that a few rows do not wait (256 rows of 8192 normed: 1024 threads 4.6 us, 512 4.7, 256 5.4; 64 of 16384 5.0,
    // 5.3, 7.1), and two to four pieces each once there are many (8192 rows of 8192: 83.2, 81.7, 83.5).
    const int pieces = p.dim / 8;
    if (pieces <= 64) launch_rows_as<TYPE, OP, QUANT, 64, 1>(p, st);
    else if (pieces <= 256) launch_rows_as<TYPE, OP, QUANT, 256, 1>(p, st);
    else if (pieces <= 512) launch_rows_as<TYPE, OP, QUANT, 256, 2>(p, st);
    else if (pieces <= 768) launch_rows_as<TYPE, OP, QUANT, 256, 3>(p, st);
    else if (pieces <= 1024) launch_rows_as<TYPE, OP, QUANT, 512, 2>(p, st);
    else if (pieces <= 2048) launch_rows_as<TYPE, OP, QUANT, 1024, 2>(p, st);
    else if (pieces <= 4096) launch_rows_as<TYPE, OP, QUANT, 1024, 4>(p, st);
    else launch_rows_as<TYPE, OP, QUANT, 1024, 8>(p, st);
    return hipGetLastError();
}

template <int OP, bool QUANT>
static rtn_status launch_typed(const RowParams& p, int dtype, void* stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    return (dtype == RTN_TYPE_F16 ? launch_rows<RTN_TYPE_F16, OP, QUANT>(p, st) : launch_rows<RTN_TYPE_BF16, OP, QUANT>(p, st)) == hipSuccess ? RTN_OK : RTN_ERR_HIP;
}

static bool row_sizes_fit(int64_t rows, int64_t dim) { return rows >= 0 && rows <= 1 << 20 && dim >= 8 && dim <= 65536 && dim % 8 == 0; }

// Rows of `width` elements, `stride` apart: the status that they alone give.
static rtn_status check_rows(const void* p, int64_t stride, int64_t width) {
    if (stride < width || stride > (int64_t)1 << 36) return RTN_ERR_SHAPE;
    return stride % 8 || !aligned_to(p, 16) ? RTN_ERR_ALIGN : RTN_OK;
}

// What every entry checks of its output: one of 16 bits, or codes and scales.
static rtn_status check_outputs(int64_t rows, int64_t dim, int dtype, const void* out16, const void* codes, const void* scales) {
    if (rows != 0 && (!out16 == !codes || (codes && !scales))) return RTN_ERR_NULL;
    if (dtype != RTN_TYPE_F16 && dtype != RTN_TYPE_BF16) return RTN_ERR_CONFIG;
    if (!row_sizes_fit(rows, dim)) return RTN_ERR_SHAPE;
    return aligned_to(out16, 16) && aligned_to(codes, 8) && aligned_to(scales, 4) ? RTN_OK : RTN_ERR_ALIGN;
}

}  // namespace rtn

extern "C" rtn_status rtn_norm_rows(const void* dev_x, int64_t rows, int64_t x_stride, int64_t dim, int dtype, const void* dev_residual, int64_t residual_stride,
                                    void* dev_residual_out, int64_t residual_out_stride, const void* dev_weight, float eps, void* dev_out, void* dev_q,
                                    float* dev_q_scales, void* stream) {
    if (rows != 0 && (!dev_x || !dev_weight || !dev_residual != !dev_residual_out)) return RTN_ERR_NULL;
    rtn_status st = rtn::check_outputs(rows, dim, dtype, dev_out, dev_q, dev_q_scales);
    if (st == RTN_OK) st = rtn::check_rows(dev_x, x_stride, dim);
    if (st == RTN_OK && dev_residual) st = rtn::check_rows(dev_residual, residual_stride, dim);
    if (st == RTN_OK && dev_residual) st = rtn::check_rows(dev_residual_out, residual_out_stride, dim);
    if (st != RTN_OK) return st;
    if (!rtn::aligned_to(dev_weight, 16)) return RTN_ERR_ALIGN;
    if (!(eps >= 0.f)) return RTN_ERR_CONFIG;
    if (rows == 0) return RTN_OK;
    const rtn::RowParams p = {dev_x, dev_residual, dev_weight, dev_residual_out, dev_q ? dev_q : dev_out, dev_q_scales, x_stride, residual_stride,
                              residual_out_stride, (int)rows, (int)dim, eps, 1.0f / (float)dim};
    return dev_q ? rtn::launch_typed<rtn::ROW_NORM, true>(p, dtype, stream) : rtn::launch_typed<rtn::ROW_NORM, false>(p, dtype, stream);
}

extern "C" rtn_status rtn_gated_rows(const void* dev_x, int64_t rows, int64_t x_stride, int64_t dim, int dtype, int activation, void* dev_out, void* dev_q,
                                     float* dev_q_scales, void* stream) {
    if (rows != 0 && !dev_x) return RTN_ERR_NULL;
    rtn_status st = rtn::check_outputs(rows, dim, dtype, dev_out, dev_q, dev_q_scales);
    if (st == RTN_OK) st = rtn::check_rows(dev_x, x_stride, 2 * dim);
    if (st != RTN_OK) return st;
    if (activation != RTN_ACT_SILU && activation != RTN_ACT_GELU_TANH) return RTN_ERR_CONFIG;
    if (rows == 0) return RTN_OK;
    const rtn::RowParams p = {dev_x, nullptr, nullptr, nullptr, dev_q ? dev_q : dev_out, dev_q_scales, x_stride, 0, 0, (int)rows, (int)dim, 0.f, 0.f};
    if (activation == RTN_ACT_SILU) return dev_q ? rtn::launch_typed<rtn::ROW_SILU, true>(p, dtype, stream) : rtn::launch_typed<rtn::ROW_SILU, false>(p, dtype, stream);
    return dev_q ? rtn::launch_typed<rtn::ROW_GELU, true>(p, dtype, stream) : rtn::launch_typed<rtn::ROW_GELU, false>(p, dtype, stream);
}

extern "C" rtn_status rtn_quantize_rows(const void* dev_x, int64_t rows, int64_t x_stride, int64_t dim, int dtype, void* dev_q, float* dev_q_scales, void* stream) {
    if (rows != 0 && !dev_x) return RTN_ERR_NULL;
    rtn_status st = rtn::check_outputs(rows, dim, dtype, nullptr, dev_q, dev_q_scales);
    if (st == RTN_OK) st = rtn::check_rows(dev_x, x_stride, dim);
    if (st != RTN_OK || rows == 0) return st;
    const rtn::RowParams p = {dev_x, nullptr, nullptr, nullptr, dev_q, dev_q_scales, x_stride, 0, 0, (int)rows, (int)dim, 0.f, 0.f};
    return rtn::launch_typed<rtn::ROW_PLAIN, true>(p, dtype, stream);
}

extern "C" rtn_status rtn_dequantize_rows(const void* dev_q, const float* dev_q_scales, int64_t rows, int64_t dim, int dtype, void* dev_out, void* stream) {
    if (rows != 0 && (!dev_q || !dev_q_scales || !dev_out)) return RTN_ERR_NULL;
    if (dtype != RTN_TYPE_F16 && dtype != RTN_TYPE_BF16) return RTN_ERR_CONFIG;
    if (!rtn::row_sizes_fit(rows, dim)) return RTN_ERR_SHAPE;
    if (!rtn::aligned_to(dev_q, 8) || !rtn::aligned_to(dev_out, 16) || !rtn::aligned_to(dev_q_scales, 4)) return RTN_ERR_ALIGN;
    if (rows == 0) return RTN_OK;
    const int segments = (int)((dim + 8191) / 8192);
    const dim3 grid((unsigned)(rows * segments));
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uint8_t* q = static_cast<const uint8_t*>(dev_q);
    if (dtype == RTN_TYPE_F16) hipLaunchKernelGGL((rtn::dequantize_rows_kernel<RTN_TYPE_F16>), grid, dim3(256), 0, st, q, dev_q_scales, dev_out, (int)dim, segments);
    else hipLaunchKernelGGL((rtn::dequantize_rows_kernel<RTN_TYPE_BF16>), grid, dim3(256), 0, st, q, dev_q_scales, dev_out, (int)dim, segments);
    return hipGetLastError() == hipSuccess ? RTN_OK : RTN_ERR_HIP;
}
