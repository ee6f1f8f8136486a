// Products of 8-bit rows with packed 8-bit weights: C = T(sum_k q_a q_w * (S_a S_w)), sums in 32-bit integers.
//
// v_mfma_i32_16x16x64_i8 takes 16 bytes a lane of each side: row (lane & 15), and the same 16 columns of 64 on both sides, in any order.  A packed
// tile is 16 rows x 64 columns and lane (row, quarter kq) owns the columns 8 kq .. and 32 + 8 kq .., codes + 128.  Two v_permlane16_swap
// bring the eights of neighbouring quarters together, so that quarters 0 .. 3 hold the sixteens 0, 2, 1, 3, which are 16 bytes in a row of
// row-major activations; four v_xor take the 128 off.
#include <algorithm>

#include "rtn_paged.h"

namespace rtn {

typedef int int4_t __attribute__((ext_vector_type(4)));

// A packed chunk as operand: sixteen 2 (kq & 1) + (kq >> 1) of the tile's columns.
__device__ __forceinline__ int4_t weight_operand(u32x4_t c) {
    const auto a = __builtin_amdgcn_permlane16_swap(c[0], c[2], false, false), b = __builtin_amdgcn_permlane16_swap(c[1], c[3], false, false);
    const u32x4_t w = {a[0], b[0], a[1], b[1]};
    return __builtin_bit_cast(int4_t, w ^ 0x80808080u);
}

template <int TYPE>
__device__ __forceinline__ u32x2_t four_results(int4_t sum, float row_scale, const half_t* scales) {
    typedef typename Elem<TYPE>::x4 E4;
    typedef typename Elem<TYPE>::one E;
    const half4_t s = *reinterpret_cast<const half4_t*>(scales);
    E4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (E)((float)sum[e] * (row_scale * (float)s[e]));
    return __builtin_bit_cast(u32x2_t, y);
}

struct W8A8Params {
    const int8_t* A;
    const float* a_scales;
    const uint8_t* B;
    const half_t* scales;
    void* C;
    int* ws;
    int M, N, KT;           // KT: tiles of 64 columns
    int XB, YB, split;      // workgroups along N, along M, along K
};

// ---- Few rows: bound by the stream of weights.  A wavefront multiplies NT tile rows of weights by MB blocks of 16 rows, both straight
// from memory into registers, D tiles ahead; the WK wavefronts of a workgroup take the tiles of its K range in turn (what they read
// together is in one piece), and add up in LDS. ----
template <int TYPE, int MB, int NT, int WK, int D>
__global__ __launch_bounds__(WK * 64) void w8a8_stream_kernel(const W8A8Params p) {
    __shared__ __align__(16) int4_t sums[WK * MB * NT * 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nl = lane & 15, kq = lane >> 4;
    int b = blockIdx.x;
    const int z = b / (p.XB * p.YB);
    b -= z * (p.XB * p.YB);
    const int x = b / p.YB, y = b - x * p.YB;
    const int t0 = (int)((int64_t)p.KT * z / p.split), t1 = (int)((int64_t)p.KT * (z + 1) / p.split);
    const int n = max(0, (t1 - t0 - wave + WK - 1) / WK);    // this wavefront's tiles: t0 + wave + WK i

    const int m0 = y * (16 * MB), rows16 = p.N / 16, K = p.KT * 64;
    const int8_t* a_at[MB];
    const uint8_t* b_at[NT];
#pragma unroll
    for (int i = 0; i < MB; ++i)                             // rows beyond M: the last one, not stored
        a_at[i] = p.A + (int64_t)min(m0 + 16 * i + nl, p.M - 1) * K + ((kq & 1) * 2 + (kq >> 1)) * 16;
#pragma unroll
    for (int j = 0; j < NT; ++j) b_at[j] = p.B + ((int64_t)min(x * NT + j, rows16 - 1) * p.KT) * 1024 + lane * 16;

    int4_t acc[MB][NT];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = (int4_t){0, 0, 0, 0};
    int4_t a[D][MB];
    u32x4_t w[D][NT];
    auto load = [&](int s, int i) {
        const int64_t t = t0 + wave + WK * min(i, n - 1);
#pragma unroll
        for (int j = 0; j < NT; ++j) w[s][j] = load_stream16(b_at[j] + t * 1024);
#pragma unroll
        for (int k = 0; k < MB; ++k) a[s][k] = *reinterpret_cast<const int4_t*>(a_at[k] + t * 64);
    };
    auto multiply = [&](int s) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int4_t wj = weight_operand(w[s][j]);
#pragma unroll
            for (int k = 0; k < MB; ++k) acc[k][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wj, a[s][k], acc[k][j], 0, 0, 0);
        }
    };
    if (n > 0) {
#pragma unroll
        for (int s = 0; s < D; ++s) load(s, s);
        int i = 0;
        for (; i + 2 * D <= n; i += D) {
#pragma unroll
            for (int s = 0; s < D; ++s) {
                multiply(s);
                load(s, i + D + s);
            }
        }
        // D to 2 D - 1 tiles are left (or fewer than D in all)
        const int more = n - i - D;
#pragma unroll
        for (int s = 0; s < D; ++s) {
            if (i + s < n) multiply(s);
            if (s < more) load(s, i + D + s);
        }
#pragma unroll
        for (int s = 0; s < D - 1; ++s)
            if (s < more) multiply(s);
    }

#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[((wave * MB + i) * NT + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    // the weights are the first operand: a lane has row nl and columns 4 kq .. 4 kq + 3
    for (int v = tid; v < MB * NT * 64; v += WK * 64) {
        int4_t s = sums[v];
#pragma unroll
        for (int k = 1; k < WK; ++k) s += sums[k * (MB * NT * 64) + v];
        const int l = v & 63, j = (v >> 6) % NT, i = (v >> 6) / NT;
        const int m = m0 + i * 16 + (l & 15), c = (x * NT + j) * 16 + (l >> 4) * 4;
        if (m >= p.M || c >= p.N) continue;
        const int64_t at = (int64_t)m * p.N + c;
        if (p.split > 1) *reinterpret_cast<int4_t*>(p.ws + (int64_t)z * p.M * p.N + at) = s;
        else *reinterpret_cast<u32x2_t*>(static_cast<half_t*>(p.C) + at) = four_results<TYPE>(s, p.a_scales[m], p.scales + c);
    }
}

// Sums of the K splits' parts, four columns a thread.
template <int TYPE>
__global__ __launch_bounds__(256) void w8a8_join_kernel(const W8A8Params p) {
    const int64_t all = (int64_t)p.M * p.N, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= all) return;
    int4_t s = *reinterpret_cast<const int4_t*>(p.ws + at);
    for (int z = 1; z < p.split; ++z) s += *reinterpret_cast<const int4_t*>(p.ws + z * all + at);
    const int m = (int)(at / p.N), c = (int)(at - (int64_t)m * p.N);
    *reinterpret_cast<u32x2_t*>(static_cast<half_t*>(p.C) + at) = four_results<TYPE>(s, p.a_scales[m], p.scales + c);
}

constexpr int kCompute = 256;                                // compute units
constexpr size_t kW8A8Workspace = (size_t)64 << 20;

struct W8A8Plan {
    int mb, nt, wk, split;
    int64_t XB, YB;
};

static W8A8Plan w8a8_plan(int64_t M, int64_t N, int64_t K, size_t workspace) {
    W8A8Plan p;
    p.mb = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    p.nt = p.mb == 1 ? 1 : 2;
    p.wk = 8;
    p.XB = (N / 16 + p.nt - 1) / p.nt;
    p.YB = (M + 16 * p.mb - 1) / (16 * p.mb);
    const int64_t most = std::min<int64_t>({16, K / 64 / p.wk, (int64_t)(std::min(workspace, kW8A8Workspace) / ((size_t)M * N * 4))});
    p.split = (int)std::max<int64_t>(1, std::min<int64_t>(most, kCompute / (p.XB * p.YB)));
    return p;
}

static rtn_status check_w8a8(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || M > 1 << 20 || N < 16 || N > 1 << 30 || N % 16 || K < 256 || K % 256 || K >= 1 << 17 || N * K >= 0x7FFF0000ll) return RTN_ERR_SHAPE;
    return RTN_OK;
}

template <int TYPE>
static hipError_t launch_w8a8(W8A8Params p, const W8A8Plan& plan, hipStream_t st) {
    const dim3 grid((unsigned)(plan.XB * plan.YB * plan.split)), block(plan.wk * 64);
    if (plan.mb == 1) hipLaunchKernelGGL((w8a8_stream_kernel<TYPE, 1, 1, 8, 4>), grid, block, 0, st, p);
    else if (plan.mb == 2) hipLaunchKernelGGL((w8a8_stream_kernel<TYPE, 2, 2, 8, 4>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((w8a8_stream_kernel<TYPE, 4, 2, 8, 4>), grid, block, 0, st, p);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.split > 1) {
        hipLaunchKernelGGL((w8a8_join_kernel<TYPE>), dim3((unsigned)(((int64_t)p.M * p.N / 4 + 255) / 256)), dim3(256), 0, st, p);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace rtn

extern "C" size_t rtn_linear_w8a8_workspace_nbytes(int64_t M, int64_t N, int64_t K) {
    if (rtn::check_w8a8(M, N, K) != RTN_OK || M == 0) return 0;
    const rtn::W8A8Plan plan = rtn::w8a8_plan(M, N, K, rtn::kW8A8Workspace);
    return plan.split > 1 ? (size_t)plan.split * M * N * 4 : 0;
}

extern "C" rtn_status rtn_linear_w8a8(const void* dev_q, const float* dev_q_scales, int64_t M, const void* dev_qweight, const void* dev_scales, int64_t N, int64_t K,
                                      int dtype, void* dev_C, void* dev_workspace, size_t workspace_nbytes, void* stream) {
    if (M != 0 && (!dev_q || !dev_q_scales || !dev_qweight || !dev_scales || !dev_C)) return RTN_ERR_NULL;
    if (dtype != RTN_TYPE_F16 && dtype != RTN_TYPE_BF16) return RTN_ERR_CONFIG;
    const rtn_status st = rtn::check_w8a8(M, N, K);
    if (st != RTN_OK) return st;
    for (const void* q : {dev_q, dev_qweight, dev_scales, (const void*)dev_C, (const void*)dev_workspace})
        if (!rtn::aligned_to(q, 16)) return RTN_ERR_ALIGN;
    if (!rtn::aligned_to(dev_q_scales, 4)) return RTN_ERR_ALIGN;
    if (M == 0) return RTN_OK;
    const rtn::W8A8Plan plan = rtn::w8a8_plan(M, N, K, dev_workspace ? workspace_nbytes : 0);
    if (!rtn::launchable(plan.XB * plan.YB * plan.split, plan.wk * 64) || 
        (plan.split > 1 && !rtn::launchable((M * N / 4 + 255) / 256, 256)))
        return RTN_ERR_SHAPE;
    const rtn::W8A8Params p = {static_cast<const int8_t*>(dev_q), dev_q_scales, static_cast<const uint8_t*>(dev_qweight), static_cast<const rtn::half_t*>(dev_scales),
                               dev_C, static_cast<int*>(dev_workspace), (int)M, (int)N, (int)(K / 64), (int)plan.XB, (int)plan.YB, plan.split};
    hipStream_t s = static_cast<hipStream_t>(stream);
    return (dtype == RTN_TYPE_F16 ? rtn::launch_w8a8<RTN_TYPE_F16>(p, plan, s) : rtn::launch_w8a8<RTN_TYPE_BF16>(p, plan, s)) == hipSuccess ? RTN_OK : RTN_ERR_HIP;
}
