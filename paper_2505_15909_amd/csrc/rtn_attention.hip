// Attention of a batch of requests' new tokens over their pages.
//
// A request's queries of one KV head are rows: row r is token r / G and head r % G of the G query heads that share the KV head, so that what is
// read of K and V serves all of them, in a decode step of one token as in a piece of a prompt.  A workgroup takes a tile of rows of
// one request and KV head.  Which request that is it finds from query_start itself: the host knows no lengths.
//
// Scores are formed transposed, S^T = K Q^T, one query a lane: the matrix instruction then leaves each lane several keys of one
// query, whose maximum and sum are the lane's own but for the last steps, and what it leaves is, as it stands, the operand P^T of
// O^T = V^T P^T, if V's keys are taken in the same order.  V^T's operands come out of LDS by transposing reads.
#include "rtn_paged.h"

#include <math.h>

namespace rtn {

struct AttnParams {
    const void *q, *k, *v;
    void* out;
    const int32_t *table, *seq, *start;
    int64_t q_stride, page_stride, head_stride, token_stride, table_stride;
    int pages, shift, max_blocks, B, T, Hq, Hk, G, window;
    float scale2, cap, cap_in, cap_out;                      // scale log2 e; softcap: cap_out tanh(cap_in q.k), cap_out = softcap log2 e
};

// exp2 of scores: the softmax is taken to base 2, with log2 e in the scale
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// cap_out tanh(x) = cap_out (1 - 2 / (e^2x + 1)); right at both ends, where e^2x is 0 or infinite
__device__ __forceinline__ float capped(float x, float cap_out) {
    const float e = exp2_of(x * 2.8853900817779268f);
    return cap_out * (1.0f - 2.0f * __builtin_amdgcn_rcpf(e + 1.0f));
}

// A workgroup's piece of work: rows row0 .. of request b.
struct Item {
    int b, row0, tok0, n, seq;                               // first query row of the batch, new tokens, cached and new tokens
};

// The item-th tile of `bm` rows, over the requests in order; false where there are no more.  All threads of the workgroup call it.
__device__ __forceinline__ bool find_item(const AttnParams& p, int item, int bm, Item* out, int* lds) {
    const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 63, wave = tid >> 6;
    const int per = (p.B + threads - 1) / threads, b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
    auto tiles = [&](int b) {
        const int s = min(max(p.start[b], 0), p.T), e = min(max(p.start[b + 1], s), p.T);
        return ((e - s) * p.G + bm - 1) / bm;
    };
    int sum = 0;
    for (int b = b0; b < b1; ++b) sum += tiles(b);
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 63) lds[wave] = incl;
    if (tid == 0) lds[16] = -1;
    __syncthreads();
    int before = incl - sum;
    for (int w = 0; w < wave; ++w) before += lds[w];
    if (item >= before && item < before + sum) {
        for (int b = b0; b < b1; ++b) {
            const int n = tiles(b);
            if (item < before + n) {
                lds[16] = b;
                lds[17] = item - before;
                break;
            }
            before += n;
        }
    }
    __syncthreads();
    const int b = __builtin_amdgcn_readfirstlane(lds[16]);
    if (b < 0) return false;
    out->b = b;
    out->row0 = __builtin_amdgcn_readfirstlane(lds[17]) * bm;
    out->tok0 = min(max(p.start[b], 0), p.T);
    out->n = min(max(p.start[b + 1], out->tok0), p.T) - out->tok0;
    out->seq = min(max(p.seq[b], 0), p.max_blocks << p.shift);
    return true;
}

template <int TYPE, int D>
__global__ __launch_bounds__(256) void attend_rows_kernel(const AttnParams p) {
    typedef typename Elem<TYPE>::one T;
    typedef typename Elem<TYPE>::x8 T8;
    typedef typename Elem<TYPE>::x4 T4;
    constexpr int KS = D / 32, DT = D / 16, KEYS = 32;       // k-steps of K Q^T, 16-row tiles of O^T, keys of a step of a wavefront
    constexpr int SW_SHIFT = D == 64 ? 1 : 0, SW_MASK = D == 64 ? 3 : 7;
    __shared__ __align__(16) uint8_t vbuf[4][KEYS * D * 2];
    __shared__ __align__(16) float merge_o[4][16][D + 4];
    __shared__ float merge_ml[4][2][16];
    __shared__ int found[18];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, grp = lane >> 4;
    const int head = blockIdx.x % p.Hk, item_no = blockIdx.x / p.Hk;

    // rows of a padded batch
    const int tail = min(max(p.start[p.B], 0), p.T);
    for (int64_t i = ((int64_t)tail * p.Hq * D) / 8 + (int64_t)blockIdx.x * 256 + tid; i < (int64_t)p.T * p.Hq * D / 8; i += (int64_t)gridDim.x * 256)
        reinterpret_cast<u32x4_t*>(p.out)[i] = (u32x4_t){0u, 0u, 0u, 0u};

    Item it;
    if (!find_item(p, item_no, 16, &it, found)) return;
    const int rows = min(16, it.n * p.G - it.row0), ctx = it.seq - it.n;
    const int row = it.row0 + min(col, rows - 1), tok = row / p.G, qh = head * p.G + row - tok * p.G;
    const int pos = ctx + tok;                               // (negative where the length is below the number of new tokens)
    const int pos_first = ctx + it.row0 / p.G, pos_last = ctx + (it.row0 + rows - 1) / p.G;
    const int kv0 = p.window ? max(0, pos_first - p.window + 1) : 0, kv1 = pos_last + 1;

    T8 q[KS];
    const T* const qp = static_cast<const T*>(p.q) + (int64_t)(it.tok0 + tok) * p.q_stride + (int64_t)qh * D + grp * 8;
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const T8*>(qp + s * 32);

    float4_t o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = (float4_t){0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    uint8_t* const vb = vbuf[wave];
    const int32_t* const table = p.table + (int64_t)it.b * p.table_stride;
    const int ps = 1 << p.shift;
    constexpr int VI = KEYS * D * 2 / 1024, CH = D / 8;      // loads of V, 16-byte pieces of a row

    for (int k0 = (kv0 & ~(KEYS - 1)) + wave * KEYS; k0 < kv1; k0 += 4 * KEYS) {
        // pages: those of tiles outside what is seen are not looked up
        const T *kt[2], *vt[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int key = min(max(k0 + 16 * h, kv0), kv1 - 1);
            const uint32_t page = min((uint32_t)table[key >> p.shift], (uint32_t)(p.pages - 1));
            const int64_t off = page * p.page_stride + head * p.head_stride + (int64_t)((k0 + 16 * h) & (ps - 1)) * p.token_stride;
            kt[h] = static_cast<const T*>(p.k) + off;
            vt[h] = static_cast<const T*>(p.v) + off;
        }
        u32x4_t v[VI];
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            const int key = (i * 64 + lane) / CH, piece = lane % CH;
            v[i] = *reinterpret_cast<const u32x4_t*>(vt[key >> 4] + (key & 15) * p.token_stride + piece * 8);
            if (k0 + key < kv0 || k0 + key >= kv1) v[i] = (u32x4_t){0u, 0u, 0u, 0u};
        }
        float4_t s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s[h] = (float4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < KS; ++t)
                s[h] = Elem<TYPE>::mfma16(*reinterpret_cast<const T8*>(kt[h] + col * p.token_stride + t * 32 + grp * 8), q[t], s[h]);
        }
        float e[8], top = -INFINITY;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = k0 + 16 * h + 4 * grp + i;
                float x = p.cap > 0.f ? capped(s[h][i] * p.cap_in, p.cap_out) : s[h][i] * p.scale2;
                if (key > pos || (p.window && pos - key >= p.window)) x = -INFINITY;
                e[4 * h + i] = x;
                top = fmaxf(top, x);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m, top), base = m_new == -INFINITY ? 0.f : m_new, back = exp2_of(m - base);
        T8 pt;
        l *= back;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float w = exp2_of(e[i] - base);
            l += w;
            pt[i] = (T)w;
        }
        m = m_new;
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            const int key = (i * 64 + lane) / CH, piece = lane % CH, sw = (key >> SW_SHIFT) & SW_MASK;
            *reinterpret_cast<u32x4_t*>(vb + key * (D * 2) + ((piece >> 1) ^ sw) * 32 + (piece & 1) * 16) = v[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            union { T8 v; short4_t s[2]; } a;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int key = 16 * h + 4 * grp + (col >> 2), sw = (key >> SW_SHIFT) & SW_MASK;
                a.s[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) short4_t*)(vb + key * (D * 2) + (t ^ sw) * 32 + (col & 3) * 8));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) o[t][i] *= back;
            o[t] = Elem<TYPE>::mfma16(a.v, pt, o[t]);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    // the four wavefronts' keys
#pragma unroll
    for (int t = 0; t < DT; ++t) *reinterpret_cast<float4_t*>(&merge_o[wave][col][t * 16 + grp * 4]) = o[t];
    if (grp == 0) {
        merge_ml[wave][0][col] = m;
        merge_ml[wave][1][col] = l;
    }
    __syncthreads();
    for (int i = tid; i < rows * (D / 4); i += 256) {
        const int r = i / (D / 4), d = i % (D / 4) * 4;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, merge_ml[w][0][r]);
        const float base = top == -INFINITY ? 0.f : top;
        float4_t acc = {0.f, 0.f, 0.f, 0.f};
        float den = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = exp2_of(merge_ml[w][0][r] - base);
            den += f * merge_ml[w][1][r];
            const float4_t x = *reinterpret_cast<const float4_t*>(&merge_o[w][r][d]);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] += f * x[j];
        }
        const float inv = den > 0.f ? 1.0f / den : 0.f;
        const int rr = it.row0 + r, tk = rr / p.G;
        T4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = (T)(acc[j] * inv);
        *reinterpret_cast<T4*>(static_cast<T*>(p.out) + ((int64_t)(it.tok0 + tk) * p.Hq + head * p.G + rr - tk * p.G) * D + d) = y;
    }
}

template <int TYPE>
static void launch_rows(const AttnParams& p, int D, hipStream_t st) {
    const int64_t items = (int64_t)p.T * p.G / 16 + p.B;
    const dim3 grid((unsigned)(items * p.Hk));
    if (D == 64) hipLaunchKernelGGL((attend_rows_kernel<TYPE, 64>), grid, dim3(256), 0, st, p);
    else if (D == 128) hipLaunchKernelGGL((attend_rows_kernel<TYPE, 128>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((attend_rows_kernel<TYPE, 256>), grid, dim3(256), 0, st, p);
}

}  // namespace rtn

extern "C" size_t rtn_paged_attention_workspace_nbytes(int64_t tokens, int n_requests, int q_heads, const rtn_kv_cache* cache, int max_new) {
    (void)tokens; (void)n_requests; (void)q_heads; (void)cache; (void)max_new;
    return 0;
}

extern "C" rtn_status rtn_paged_attention(const void* dev_q, int64_t tokens, int64_t q_stride, int q_heads, const rtn_kv_cache* cache,
                                          const int32_t* dev_block_table, int64_t table_stride, int max_blocks, const int32_t* dev_seq_lens,
                                          const int32_t* dev_query_start, int n_requests, int max_new, float scale, float softcap, int window,
                                          void* dev_out, void* dev_workspace, size_t workspace_nbytes, void* stream) {
    const rtn_status st = rtn::check_cache(cache);
    if (st != RTN_OK) return st;
    if (!dev_block_table || !dev_seq_lens || !dev_query_start || (tokens != 0 && (!dev_q || !dev_out))) return RTN_ERR_NULL;
    const int D = cache->head_dim;
    if (tokens < 0 || tokens > 1 << 24 || n_requests < 1 || n_requests > 65536 || q_heads < 1 || q_heads % cache->kv_heads != 0 ||
        q_heads / cache->kv_heads > 64 || q_stride < (int64_t)q_heads * D || q_stride > (int64_t)1 << 36 || max_blocks < 1 ||
        max_blocks > (1 << 30) / cache->page_size || table_stride < max_blocks || max_new < 1)
        return RTN_ERR_SHAPE;
    if (!(scale > 0.f) || !(scale < INFINITY) || !(softcap >= 0.f) || !(softcap < INFINITY) || window < 0) return RTN_ERR_CONFIG;
    if (q_stride % 8 || !rtn::aligned_to(dev_q, 16) || !rtn::aligned_to(dev_out, 16) || !rtn::aligned_to(dev_workspace, 16) ||
        !rtn::aligned_to(dev_block_table, 4) || !rtn::aligned_to(dev_seq_lens, 4) || !rtn::aligned_to(dev_query_start, 4))
        return RTN_ERR_ALIGN;
    if ((tokens * (q_heads / cache->kv_heads) / 16 + n_requests) * cache->kv_heads >= 0x7FFFFFFF) return RTN_ERR_SHAPE;
    if (tokens == 0) return RTN_OK;
    const float log2e = 1.4426950408889634f;
    const rtn::AttnParams p = {dev_q, cache->dev_k, cache->dev_v, dev_out, dev_block_table, dev_seq_lens, dev_query_start, q_stride, cache->page_stride,
                               cache->head_stride, cache->token_stride, table_stride, (int)cache->pages, rtn::log2_of(cache->page_size), max_blocks,
                               n_requests, (int)tokens, q_heads, cache->kv_heads, q_heads / cache->kv_heads, window, scale * log2e, softcap,
                               softcap > 0.f ? scale / softcap : 0.f, softcap * log2e};
    if (cache->dtype == RTN_TYPE_F16) rtn::launch_rows<RTN_TYPE_F16>(p, D, static_cast<hipStream_t>(stream));
    else rtn::launch_rows<RTN_TYPE_BF16>(p, D, static_cast<hipStream_t>(stream));
    return hipGetLastError() == hipSuccess ? RTN_OK : RTN_ERR_HIP;
}
