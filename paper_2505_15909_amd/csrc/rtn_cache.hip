// The paged KV cache: block tables and slots from the requests' lengths, and the rotation with the cache write.
#include "rtn_paged.h"

namespace rtn {

// ---- Block tables, slots and positions ----------------------------------------------------------------------------------------
//
// Three running sums over the requests (new tokens, pages to pop, pages pushed back) say where everything goes: token i belongs to the
// request whose sum first exceeds i, pop number p is entry count + pushed - 1 - p of the stack, and an entry from count on
// is a page of an ended request.  So nothing written is read again: a page that is pushed and popped in the same step goes from one table to
// the other, and every workgroup forms the sums for itself (a few KiB from the L2) and takes its share of the tokens.

struct PlanParams {
    const int32_t *step, *cached, *count;
    int32_t *table, *free_pages, *seq, *start, *positions, *slots, *count_out, *status;
    int64_t table_stride, pool;
    int B, shift, max_blocks, max_tokens;
};

// First of n rising sums that exceeds i.
__device__ __forceinline__ int owner_of(const int* sums, int n, int i) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] > i) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

struct Request {
    int cached, old, tokens, need, freed, flags;
};

__device__ __forceinline__ Request read_request(const PlanParams& p, int b) {
    Request r = {};
    const int step = p.step[b], mask = (1 << p.shift) - 1;
    r.cached = p.cached[b];
    if (r.cached < 0 || (r.cached + (int64_t)mask) >> p.shift > p.max_blocks) {
        r.flags = 8;
        return r;
    }
    r.old = (int)((r.cached + (int64_t)mask) >> p.shift);
    if (step < 0) {
        r.freed = r.old;
        return r;
    }
    const int64_t blocks = (r.cached + (int64_t)step + mask) >> p.shift;
    if (blocks > p.max_blocks) r.flags = 2;
    if (step > p.max_tokens) r.flags |= 4;
    if (r.flags) return r;
    r.tokens = step;
    r.need = (int)blocks - r.old;
    return r;
}

__global__ __launch_bounds__(1024) void cache_plan_kernel(const PlanParams p) {
    extern __shared__ int lds[];
    __shared__ int part[16][4];
    __shared__ int high[16][3];
    int *const ends = lds, *const pops = ends + p.B, *const frees = pops + p.B, *const cached = frees + p.B;
    const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 63, wave = tid >> 6, waves = threads >> 6;
    const int count = *p.count;

    // Each thread's requests, then the sums before it: within the wavefront, then over the wavefronts.  32 bits hold every sum that is used; what the whole batch
    // comes to is known exactly, from the sum of the numbers' upper parts beside it.
    const int per = (p.B + threads - 1) / threads, b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
    constexpr int KEEP = 4;                                  // read at once and kept: up to 1024 requests of 256 threads
    Request own[KEEP];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) own[i] = b0 + i < b1 ? read_request(p, b0 + i) : Request{};
    auto each = [&](auto&& f) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (b0 + i < b1) f(b0 + i, own[i]);
        for (int b = b0 + KEEP; b < b1; ++b) f(b, read_request(p, b));
    };
    uint32_t sum[3] = {0, 0, 0};
    int upper[3] = {0, 0, 0};                                // of 16 bits and above: below 2^26 in all, and what is left of the sum below 2^28
    int flags = 0;
    each([&](int, const Request& r) {
        sum[0] += r.tokens;
        sum[1] += r.need;
        sum[2] += r.freed;
        upper[0] += r.tokens >> 16;
        upper[1] += r.need >> 16;
        upper[2] += r.freed >> 16;
        flags |= r.flags;
    });
    uint32_t before[3], total[3] = {0, 0, 0};
    int above[3] = {0, 0, 0};
    flags = (__any(flags & 1) ? 1 : 0) | (__any(flags & 2) ? 2 : 0) | (__any(flags & 4) ? 4 : 0) | (__any(flags & 8) ? 8 : 0);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const uint32_t s = wave_scan(sum[k]);
        const int u = wave_scan(upper[k]);
        before[k] = s - sum[k];
        if (lane == 63) {
            part[wave][k] = s;
            high[wave][k] = u;
        }
    }
    if (lane == 63) part[wave][3] = flags;
    __syncthreads();
    flags = 0;
    for (int w = 0; w < waves; ++w) {
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            if (w < wave) before[k] += part[w][k];
            total[k] += part[w][k];
            above[k] += high[w][k];
        }
        flags |= part[w][3];
    }
    auto whole = [&](int k) { return ((int64_t)above[k] << 16) + (uint32_t)(total[k] - ((uint32_t)above[k] << 16)); };
    const int64_t back = whole(2), left = count + back - whole(1);
    if (count < 0 || count > p.pool || back > p.pool || left > p.pool) flags |= 8;
    if (left < 0) flags |= 1;
    if (whole(0) > p.max_tokens) flags |= 4;

    // (where flags are set, the sums are not used)
    each([&](int b, const Request& r) {
        before[0] += r.tokens;
        before[1] += r.need;
        before[2] += r.freed;
        ends[b] = (int)before[0];
        pops[b] = (int)before[1];
        frees[b] = (int)before[2];
        cached[b] = r.cached;
    });
    __syncthreads();

    const int ps = 1 << p.shift, new_tokens = flags ? 0 : (int)total[0];
    auto start_of = [](const int* sums, int b) { return b ? sums[b - 1] : 0; };
    auto entry = [&](int at) -> int {                        // of the stack
        if (at < count) return p.free_pages[at];
        const int f = at - count, b = owner_of(frees, p.B, f);
        return p.table[b * p.table_stride + (f - start_of(frees, b))];
    };
    auto popped = [&](int n) { return entry(count + (int)total[2] - 1 - n); };

    // The four outputs' first elements go to different wavefronts: in a step of few tokens none waits for another's loads.
    const int step = gridDim.x * threads;
    auto first = [&](int k) { return (int)blockIdx.x * threads + ((tid + 64 * k) & 255) + (tid & ~255); };
    for (int i = first(0); i < p.max_tokens; i += step) {
        int pos = -1, slot = -1;
        if (i < new_tokens) {
            const int b = owner_of(ends, p.B, i), c = cached[b], old = (c + ps - 1) >> p.shift;
            pos = c + i - start_of(ends, b);
            const int j = pos >> p.shift;
            const int page = j < old ? p.table[b * p.table_stride + j] : popped(start_of(pops, b) + j - old);
            // (a page that no cache can have is no slot, rather than, in 32 bits, one of another page)
            slot = (uint32_t)page > (uint32_t)INT32_MAX >> p.shift ? -1 : (page << p.shift) + (pos & (ps - 1));
        }
        p.positions[i] = pos;
        p.slots[i] = slot;
    }
    if (!flags) {
        for (int i = first(1); i < (int)total[1]; i += step) {
            const int b = owner_of(pops, p.B, i), old = (cached[b] + ps - 1) >> p.shift;
            p.table[b * p.table_stride + old + i - start_of(pops, b)] = popped(i);
        }
        for (int i = count + first(2); i < (int)left; i += step) p.free_pages[i] = entry(i);
    }
    for (int b = first(3); b < p.B; b += step) {
        const int n = ends[b] - start_of(ends, b);
        const bool ended = frees[b] > start_of(frees, b);
        p.seq[b] = flags ? cached[b] : ended ? 0 : cached[b] + n;
        p.start[b + 1] = flags ? 0 : ends[b];
    }
    if (blockIdx.x == 0 && tid == 0) {
        p.start[0] = 0;
        *p.count_out = flags ? count : (int)left;
        *p.status = flags;
    }
}

// ---- Norms, rotation, cache write ---------------------------------------------------------------------------------------------
//
// A head is eight elements a lane: 8, 16 or 32 lanes.  For pairs half a rotation apart a lane takes four elements of each half, so that both
// members of a pair and the four cosines and sines that go with them are its own.

struct RopeParams {
    const void *qkv, *q_norm, *k_norm;
    const float* rope;
    const int32_t *positions, *slots;
    void *q_out, *k, *v;
    int64_t qkv_stride, page_stride, head_stride, token_stride, max_positions, slot_count;
    int tokens, Hq, Hk, rotary, shift;
    float eps;
};

template <int TYPE, int D, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_cache_kernel(const RopeParams p) {
    typedef typename Elem<TYPE>::one T;
    typedef typename Elem<TYPE>::x4 T4;
    constexpr int L = D / 8;                                 // lanes of a head
    const int H = p.Hq + 2 * p.Hk;
    const uint32_t row = blockIdx.x * (256 / L) + threadIdx.x / L;       // (below 2^29: a launch has fewer than 2^32 threads)
    const int c = threadIdx.x % L;
    if (row >= (uint32_t)(p.tokens * H)) return;             // (whole heads: the lanes of one stay together)
    const int t = (int)(row / (uint32_t)H), h = (int)(row - (uint32_t)t * H);
    const T* const src = static_cast<const T*>(p.qkv) + t * p.qkv_stride + (int64_t)h * D;
    const bool rotated = h < p.Hq + p.Hk && c * 8 < p.rotary;
    const int e0 = INTERLEAVED || !rotated ? c * 8 : c * 4, e1 = INTERLEAVED || !rotated ? c * 8 + 4 : p.rotary / 2 + c * 4;
    const T4 x0 = *reinterpret_cast<const T4*>(src + e0), x1 = *reinterpret_cast<const T4*>(src + e1);
    T4 y0 = x0, y1 = x1;
    const int32_t slot = p.slots[t];
    if (h < p.Hq + p.Hk) {
        float a[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) { a[i] = (float)x0[i]; a[4 + i] = (float)x1[i]; }
        const void* const norm = h < p.Hq ? p.q_norm : p.k_norm;
        if (norm) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(a[i], a[i], s);
#pragma unroll
            for (int d = 1; d < L; d <<= 1) s += __shfl_xor(s, d);
            const float r = rsqrtf(s * (1.0f / D) + p.eps);
            const T4 w0 = *reinterpret_cast<const T4*>(static_cast<const T*>(norm) + e0), w1 = *reinterpret_cast<const T4*>(static_cast<const T*>(norm) + e1);
#pragma unroll
            for (int i = 0; i < 4; ++i) { a[i] *= r * (float)w0[i]; a[4 + i] *= r * (float)w1[i]; }
        }
        if (rotated) {
            const int64_t pos = min((int64_t)max(p.positions[t], 0), p.max_positions - 1);
            const float* const cs = p.rope + pos * p.rotary + c * 4;
            const float4_t cos = *reinterpret_cast<const float4_t*>(cs), sin = *reinterpret_cast<const float4_t*>(cs + p.rotary / 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int ia = INTERLEAVED ? 2 * i : i, ib = INTERLEAVED ? 2 * i + 1 : 4 + i;
                const float u = a[ia], v = a[ib];
                a[ia] = u * cos[i] - v * sin[i];
                a[ib] = v * cos[i] + u * sin[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) { y0[i] = (T)a[i]; y1[i] = (T)a[4 + i]; }
    }
    T* dst;
    if (h < p.Hq) {
        dst = static_cast<T*>(p.q_out) + ((int64_t)t * p.Hq + h) * D;
    } else {
        if (slot < 0 || slot >= p.slot_count) return;
        const int kh = h - p.Hq, hk = kh < p.Hk ? kh : kh - p.Hk;
        dst = static_cast<T*>(kh < p.Hk ? p.k : p.v) + (slot >> p.shift) * p.page_stride + hk * p.head_stride + (slot & ((1 << p.shift) - 1)) * p.token_stride;
    }
    // (as streaming: what a prompt writes does not fit the caches, and a decode step's is written through at the end of the kernel either way.  7704
    // tokens of 80 heads 63.2 -> 56.4 us, 5.6 TB/s; 1896 tokens of 48 half-heads with norms 6.7 -> 6.0; 16 tokens 2.9 both ways.  Streaming loads
    // gained nothing.)
    __builtin_nontemporal_store(y0, reinterpret_cast<T4*>(dst + e0));
    __builtin_nontemporal_store(y1, reinterpret_cast<T4*>(dst + e1));
}

static int64_t rope_blocks(int64_t tokens, int heads, int D) { return (tokens * heads * (D / 8) + 255) / 256; }

template <int TYPE, int D>
static void launch_rope(const RopeParams& p, bool interleaved, hipStream_t st) {
    const dim3 grid((unsigned)rope_blocks(p.tokens, p.Hq + 2 * p.Hk, D));
    if (interleaved) hipLaunchKernelGGL((rope_cache_kernel<TYPE, D, true>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((rope_cache_kernel<TYPE, D, false>), grid, dim3(256), 0, st, p);
}

}  // namespace rtn

extern "C" rtn_status rtn_cache_plan(const int32_t* dev_step, const int32_t* dev_cached_lens, int n_requests, int page_size,
                                     int32_t* dev_block_table, int64_t table_stride, int max_blocks,
                                     int32_t* dev_free_pages, int64_t pool, const int32_t* dev_free_count,
                                     int32_t* dev_seq_lens, int32_t* dev_query_start, int32_t* dev_positions, int32_t* dev_slots, int64_t max_tokens,
                                     int32_t* dev_free_count_out, int32_t* dev_status, void* stream) {
    if (!dev_step || !dev_cached_lens || !dev_block_table || !dev_free_pages || !dev_free_count || !dev_seq_lens || !dev_query_start ||
        (max_tokens > 0 && (!dev_positions || !dev_slots)) || !dev_free_count_out || !dev_status)
        return RTN_ERR_NULL;
    if (n_requests < 1 || n_requests > 4096 || !rtn::page_size_valid(page_size) || max_blocks < 1 || max_blocks > (1 << 30) / page_size ||
        table_stride < max_blocks || pool < 1 || pool > 1 << 27 || max_tokens < 0 || max_tokens >= (int64_t)1 << 30)
        return RTN_ERR_SHAPE;
    for (const void* q : {(const void*)dev_step, (const void*)dev_cached_lens, (const void*)dev_block_table, (const void*)dev_free_pages,
                          (const void*)dev_free_count, (const void*)dev_seq_lens, (const void*)dev_query_start, (const void*)dev_positions,
                          (const void*)dev_slots, (const void*)dev_free_count_out, (const void*)dev_status})
        if (!rtn::aligned_to(q, 4)) return RTN_ERR_ALIGN;
    const rtn::PlanParams p = {dev_step, dev_cached_lens, dev_free_count, dev_block_table, dev_free_pages, dev_seq_lens, dev_query_start, dev_positions,
                               dev_slots, dev_free_count_out, dev_status, table_stride, pool, n_requests, rtn::log2_of(page_size), max_blocks, (int)max_tokens};
    // In place, one workgroup reads everything before it writes; otherwise a thread has a token or a few.  (In the kernel, in place and not: a token each of 64 requests 4.8 and
    // 4.0 us, of 1024 6.4 and 5.4; 3608 tokens of 64 requests 7.3 and 4.5, 15670 of 1024 19.9 and 5.9.)
    const bool in_place = dev_seq_lens == dev_cached_lens || dev_free_count_out == dev_free_count;
    const int threads = in_place ? 1024 : 256;
    const int64_t work = max_tokens > n_requests ? max_tokens : n_requests;
    const unsigned blocks = in_place ? 1 : (unsigned)(work < threads * 64 ? (work + threads - 1) / threads : 64);
    const size_t lds = (size_t)n_requests * 16;
    if (lds > 61440 && hipFuncSetAttribute(reinterpret_cast<const void*>(&rtn::cache_plan_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
        return RTN_ERR_HIP;
    hipLaunchKernelGGL(rtn::cache_plan_kernel, dim3(blocks), dim3(threads), lds, static_cast<hipStream_t>(stream), p);
    return hipGetLastError() == hipSuccess ? RTN_OK : RTN_ERR_HIP;
}

extern "C" rtn_status rtn_rope_cache(const void* dev_qkv, int64_t tokens, int64_t qkv_stride, int q_heads, const float* dev_rope, int rotary_dim,
                                     int64_t max_positions, int interleaved, const int32_t* dev_positions, const int32_t* dev_slots,
                                     const void* dev_q_norm, const void* dev_k_norm, float eps, const rtn_kv_cache* cache, void* dev_q_out, void* stream) {
    const rtn_status st = rtn::check_cache(cache);
    if (st != RTN_OK) return st;
    if (tokens != 0 && (!dev_qkv || !dev_rope || !dev_positions || !dev_slots || !dev_q_out)) return RTN_ERR_NULL;
    const int D = cache->head_dim;
    if (tokens < 0 || tokens > 1 << 24 || q_heads < 1 || q_heads > 65536 || rotary_dim < 8 || rotary_dim > D || rotary_dim % 8 || max_positions < 1 ||
        qkv_stride < (int64_t)(q_heads + 2 * cache->kv_heads) * D || qkv_stride > (int64_t)1 << 36)
        return RTN_ERR_SHAPE;
    if (qkv_stride % 8 || !rtn::aligned_to(dev_qkv, 16) || !rtn::aligned_to(dev_rope, 16) || !rtn::aligned_to(dev_q_norm, 16) ||
        !rtn::aligned_to(dev_k_norm, 16) || !rtn::aligned_to(dev_q_out, 16) || !rtn::aligned_to(dev_positions, 4) || !rtn::aligned_to(dev_slots, 4))
        return RTN_ERR_ALIGN;
    if (!(eps >= 0.f) || (interleaved != 0 && interleaved != 1)) return RTN_ERR_CONFIG;
    if (!rtn::launchable(rtn::rope_blocks(tokens, q_heads + 2 * cache->kv_heads, D), 256)) return RTN_ERR_SHAPE;
    if (tokens == 0) return RTN_OK;
    const rtn::RopeParams p = {dev_qkv, dev_q_norm, dev_k_norm, dev_rope, dev_positions, dev_slots, dev_q_out, cache->dev_k, cache->dev_v, qkv_stride,
                               cache->page_stride, cache->head_stride, cache->token_stride, max_positions, cache->pages * cache->page_size, (int)tokens,
                               q_heads, cache->kv_heads, rotary_dim, rtn::log2_of(cache->page_size), eps};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool il = interleaved != 0;
    if (cache->dtype == RTN_TYPE_F16) {
        if (D == 64) rtn::launch_rope<RTN_TYPE_F16, 64>(p, il, s);
        else if (D == 128) rtn::launch_rope<RTN_TYPE_F16, 128>(p, il, s);
        else rtn::launch_rope<RTN_TYPE_F16, 256>(p, il, s);
    } else {
        if (D == 64) rtn::launch_rope<RTN_TYPE_BF16, 64>(p, il, s);
        else if (D == 128) rtn::launch_rope<RTN_TYPE_BF16, 128>(p, il, s);
        else rtn::launch_rope<RTN_TYPE_BF16, 256>(p, il, s);
    }
    return hipGetLastError() == hipSuccess ? RTN_OK : RTN_ERR_HIP;
}
