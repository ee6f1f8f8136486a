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

// Pieces that a batch is cut into where its tiles alone are fewer (see find_piece).
constexpr int kPieces = 1024, kTilePieces = 512;

struct AttnParams {
    const void *q, *k, *v;
    void* out;
    const int32_t *table, *seq, *start;
    int64_t q_stride, page_stride, head_stride, token_stride, table_stride;
    int pages, shift, max_blocks, B, T, Hq, Hk, G, window;
    float scale2, cap, cap_in, cap_out;                      // scale log2 e; softcap: cap_out tanh(cap_in q.k), cap_out = softcap log2 e
    // Split requests: `pieces` a KV head are aimed at (0: none is split), and a head has room for twice as many partial results,
    // [Hk][2 pieces][rows][D] sums and, behind them, [Hk][2 pieces][rows][2] maxima and sums of weights.
    float* partial;
    int pieces;
};

// exp2 of scores: the softmax is taken to base 2, with log2 e in the scale
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// cap_out tanh(x) = cap_out (1 - 2 / (e^2x + 1)); right at both ends, where e^2x is 0 or infinite
__device__ __forceinline__ float capped(float x, float cap_out) {
    const float e = exp2_of(x * 2.8853900817779268f);
    return cap_out * (1.0f - 2.0f * __builtin_amdgcn_rcpf(e + 1.0f));
}

// What a workgroup does: ROWS rows from row0 of request b, a part of their keys.
struct Piece {
    int b, row0, rows, tok0, n, ctx;                         // rows of the tile, first token in the batch, new tokens, cached tokens
    int kv0, kv1;                                            // keys that some row sees
    int part, parts, slot;                                   // of the tile's keys; where the first part's partial result goes
    int k0, k1;                                              // this part's, in blocks of KEYS from kv0's
};

// Each workgroup finds its own piece from the requests' lengths, which the host does not know: with n_b blocks of keys and t_b
// tiles of rows, pieces of c = ceil(sum t_b n_b / `pieces`) blocks put a like share of the whole batch's keys on every workgroup, whatever the
// requests' lengths; tile t of request b has the t_b ceil(n_b / c) pieces after those of the requests before it.  Two scans over the requests, a
// microsecond or two.  PART: number `no` of the pieces; otherwise of the tiles (what joins the parts).  All 256 threads call it.
template <int ROWS, int KEYS, bool PART>
__device__ __forceinline__ bool find_piece(const AttnParams& p, int no, Piece* out) {
    __shared__ int64_t totals[4];
    __shared__ int sums[4][2], found[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (p.B + 255) / 256, b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
    struct Request { int tok0, n, seq, tiles, blocks; };
    auto request = [&](int b) {
        Request r;
        r.tok0 = min(max(p.start[b], 0), p.T);
        r.n = min(max(p.start[b + 1], r.tok0), p.T) - r.tok0;
        r.seq = min(max(p.seq[b], 0), p.max_blocks << p.shift);
        r.tiles = (r.n * p.G + ROWS - 1) / ROWS;
        // (with a window, a bound on what a tile sees: the windows of its tokens, unaligned)
        r.blocks = (r.seq + KEYS - 1) / KEYS;
        if (p.window) r.blocks = (int)min((int64_t)r.blocks, ((int64_t)p.window + ROWS / p.G + 1 + KEYS - 1) / KEYS + 1);
        return r;
    };
    int c = 0x7FFFFFFF;
    if (p.pieces) {
        int64_t total = 0;
        for (int b = b0; b < b1; ++b) {
            const Request r = request(b);
            total += (int64_t)r.tiles * r.blocks;
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) total += __shfl_xor((long long)total, d);
        if (lane == 0) totals[wave] = total;
        __syncthreads();
        total = totals[0] + totals[1] + totals[2] + totals[3];
        c = (int)min((int64_t)0x7FFFFFFF, max((int64_t)1, (total + p.pieces - 1) / p.pieces));
    }
    auto parts_of = [&](int blocks) { return max(1, (int)(((int64_t)blocks + c - 1) / c)); };
    int mine[2] = {0, 0};                                    // numbers (of pieces or tiles), slots
    for (int b = b0; b < b1; ++b) {
        const Request r = request(b);
        const int parts = parts_of(r.blocks);
        mine[0] += PART ? r.tiles * parts : r.tiles;
        mine[1] += parts > 1 ? r.tiles * parts : 0;
    }
    int incl[2] = {mine[0], mine[1]};
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int o = __shfl_up(incl[k], d);
            if (lane >= d) incl[k] += o;
        }
    }
    if (lane == 63) {
        sums[wave][0] = incl[0];
        sums[wave][1] = incl[1];
    }
    if (tid == 0) found[0] = -1;
    __syncthreads();
    int before = incl[0] - mine[0], slot = incl[1] - mine[1];
    for (int w = 0; w < wave; ++w) {
        before += sums[w][0];
        slot += sums[w][1];
    }
    if (no >= before && no < before + mine[0]) {
        for (int b = b0; b < b1; ++b) {
            const Request r = request(b);
            const int parts = parts_of(r.blocks), have = PART ? r.tiles * parts : r.tiles;
            if (no < before + have) {
                found[0] = b;
                found[1] = no - before;
                found[2] = slot;
                found[3] = parts;
                break;
            }
            before += have;
            slot += parts > 1 ? r.tiles * parts : 0;
        }
    }
    __syncthreads();
    const int b = __builtin_amdgcn_readfirstlane(found[0]);
    if (b < 0) return false;
    const int local = __builtin_amdgcn_readfirstlane(found[1]), most = __builtin_amdgcn_readfirstlane(found[3]);
    const Request r = request(b);
    const int tile = PART ? local / most : local;
    out->b = b;
    out->tok0 = r.tok0;
    out->n = r.n;
    out->ctx = r.seq - r.n;
    out->row0 = tile * ROWS;
    out->rows = min(ROWS, r.n * p.G - out->row0);
    const int first = out->ctx + out->row0 / p.G, last = out->ctx + (out->row0 + out->rows - 1) / p.G;
    out->kv0 = p.window ? max(0, first - p.window + 1) : 0;
    out->kv1 = last + 1;                                     // (not above the length; 0 and less where nothing is seen)
    // the tile's own blocks, which may be fewer than its request's: as many parts as they fill, of like size
    const int blocks = max(0, (out->kv1 + KEYS - 1) / KEYS - out->kv0 / KEYS);
    out->parts = min(most, parts_of(blocks));
    out->part = PART ? local - tile * most : 0;
    out->slot = __builtin_amdgcn_readfirstlane(found[2]) + tile * most;
    const int each = (blocks + out->parts - 1) / out->parts;
    out->k0 = out->kv0 / KEYS + out->part * each;
    out->k1 = min(out->k0 + each, out->kv0 / KEYS + blocks);
    return out->part < out->parts;
}

__device__ __forceinline__ float* partial_sums(const AttnParams& p, int head, int slot, int rows, int D) {
    return p.partial + ((int64_t)head * 2 * p.pieces + slot) * rows * D;
}
__device__ __forceinline__ float* partial_stats(const AttnParams& p, int head, int slot, int rows, int D) {
    return p.partial + (int64_t)p.Hk * 2 * p.pieces * rows * D + ((int64_t)head * 2 * p.pieces + slot) * rows * 2;
}

// Rows of a padded batch get zeros: every workgroup a share, whatever it does else.
template <int THREADS>
__device__ __forceinline__ void clear_padding(const AttnParams& p, int D) {
    const int64_t per_token = (int64_t)p.Hq * D / 8, first = min(max(p.start[p.B], 0), p.T) * per_token;
    for (int64_t i = first + (int64_t)blockIdx.x * THREADS + threadIdx.x; i < p.T * per_token; i += (int64_t)gridDim.x * THREADS)
        reinterpret_cast<u32x4_t*>(p.out)[i] = (u32x4_t){0u, 0u, 0u, 0u};
}

// The parts of a tile's keys, brought to their common maximum and added up in their order.
template <int TYPE, int D, int ROWS, int KEYS>
__global__ __launch_bounds__(256) void join_parts_kernel(const AttnParams p) {
    typedef typename Elem<TYPE>::one T;
    typedef typename Elem<TYPE>::x4 T4;
    const int head = blockIdx.x % p.Hk;
    Piece w;
    if (!find_piece<ROWS, KEYS, false>(p, blockIdx.x / p.Hk, &w) || w.parts == 1) return;
    const float *const po = partial_sums(p, head, w.slot, ROWS, D), *const pm = partial_stats(p, head, w.slot, ROWS, D);
    for (int i = threadIdx.x; i < w.rows * (D / 4); i += 256) {
        const int r = i / (D / 4), d = i % (D / 4) * 4;
        float top = -INFINITY;
        for (int s = 0; s < w.parts; ++s) top = fmaxf(top, pm[((int64_t)s * ROWS + r) * 2]);
        const float base = top == -INFINITY ? 0.f : top;
        float4_t acc = {0.f, 0.f, 0.f, 0.f};
        float den = 0.f;
#pragma unroll 4
        for (int s = 0; s < w.parts; ++s) {
            const float f = exp2_of(pm[((int64_t)s * ROWS + r) * 2] - base);
            den += f * pm[((int64_t)s * ROWS + r) * 2 + 1];
            const float4_t x = *reinterpret_cast<const float4_t*>(po + ((int64_t)s * ROWS + r) * D + d);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] += f * x[j];
        }
        const float inv = den > 0.f ? 1.0f / den : 0.f;
        const int row = w.row0 + r, tok = row / p.G;
        T4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = (T)(acc[j] * inv);
        *reinterpret_cast<T4*>(static_cast<T*>(p.out) + ((int64_t)(w.tok0 + tok) * p.Hq + head * p.G + row - tok * p.G) * D + d) = y;
    }
}

// Within a wavefront: its own writes to LDS are there for its reads.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Few rows: 16 NQ of them a workgroup, whose four wavefronts take blocks of 32 keys in turn, each with a softmax of its own until they join
// at the end.  Bound by the reading of K and V: K goes from memory into the matrix cores' registers, V by way of 8 KiB of LDS
// that only its wavefront touches, so that the loop has no barrier.
template <int TYPE, int D, int NQ>
__global__ __launch_bounds__(256, D == 64 ? 4 : D == 128 && NQ == 1 ? 3 : 2) void attend_rows_kernel(const AttnParams p) {
    typedef typename Elem<TYPE>::one T;
    typedef typename Elem<TYPE>::x8 T8;
    typedef typename Elem<TYPE>::x4 T4;
    constexpr int KS = D / 32, DT = D / 16, STEP = 32, ROWS = 16 * NQ, KEYS = 4 * STEP;     // k-steps of K Q^T, 16-row tiles of O^T, keys of a step
    constexpr int SW_SHIFT = D == 64 ? 1 : 0, SW_MASK = D == 64 ? 3 : 7;
    constexpr int VI = STEP * D * 2 / 1024, CH = D / 8;      // loads of V, 16-byte pieces of a row
    constexpr int MERGE = 16 * (D + 4) * 4;                  // bytes of a wavefront's sums of 16 rows, in place of its V
    __shared__ __align__(16) uint8_t buf[4][MERGE > STEP * D * 2 ? MERGE : STEP * D * 2];
    __shared__ float stats[4][2][ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, grp = lane >> 4;
    const int head = blockIdx.x % p.Hk;
    clear_padding<256>(p, D);
    Piece w;
    if (!find_piece<ROWS, KEYS, true>(p, blockIdx.x / p.Hk, &w)) return;

    T8 q[NQ][KS];
    int pos[NQ];                                             // (negative where the length is below the number of new tokens)
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int row = w.row0 + min(16 * n + col, w.rows - 1), tok = row / p.G, qh = head * p.G + row - tok * p.G;
        pos[n] = w.ctx + tok;
        const T* const qp = static_cast<const T*>(p.q) + (int64_t)(w.tok0 + tok) * p.q_stride + (int64_t)qh * D + grp * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[n][s] = *reinterpret_cast<const T8*>(qp + s * 32);
    }
    float4_t o[NQ][DT];
    float m[NQ], l[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        m[n] = -INFINITY;
        l[n] = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[n][t] = (float4_t){0.f, 0.f, 0.f, 0.f};
    }
    uint8_t* const vb = buf[wave];
    const int32_t* const table = p.table + (int64_t)w.b * p.table_stride;
    const int ps = 1 << p.shift;
    // keys that every row sees need no masks
    const int window = p.window ? p.window : 0x7FFFFFFF;     // (a position less this does not wrap: lengths are up to 2^30)
    const int all0 = p.window ? w.ctx + (w.row0 + w.rows - 1) / p.G - p.window + 1 : 0, all1 = w.ctx + w.row0 / p.G + 1;
    const int end = min(w.kv1, w.k1 * KEYS);
    int ids = 0;                                             // lane i: the page of the 16 keys that are number i of 64 this wavefront comes to

    for (int k0 = w.k0 * KEYS + wave * STEP, i = 0; k0 < end; k0 += KEYS, ++i) {
        if ((i & 31) == 0) {
            const int key = min(max(k0 + (lane >> 1) * KEYS + (lane & 1) * 16, w.kv0), w.kv1 - 1);     // (none outside what is seen)
            ids = min((uint32_t)table[key >> p.shift], (uint32_t)(p.pages - 1));
        }
        const T *kt[2], *vt[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t page = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + h);
            const int64_t off = page * p.page_stride + head * p.head_stride + (int64_t)((k0 + 16 * h) & (ps - 1)) * p.token_stride;
            kt[h] = static_cast<const T*>(p.k) + off;
            vt[h] = static_cast<const T*>(p.v) + off;
        }
        T8 k[2][KS];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < KS; ++t) k[h][t] = *reinterpret_cast<const T8*>(kt[h] + col * (int)p.token_stride + t * 32 + grp * 8);
        u32x4_t v[VI];
#pragma unroll
        for (int j = 0; j < VI; ++j) {
            const int key = (j * 64 + lane) / CH, piece = lane % CH;
            v[j] = *reinterpret_cast<const u32x4_t*>(vt[j * 64 / CH >> 4] + (key & 15) * (int)p.token_stride + piece * 8);
        }
        if (k0 < w.kv0 || k0 + STEP > w.kv1) {               // slots without a token of the request may hold anything
#pragma unroll
            for (int j = 0; j < VI; ++j) {
                const int key = k0 + (j * 64 + lane) / CH;
                if (key < w.kv0 || key >= w.kv1) v[j] = (u32x4_t){0u, 0u, 0u, 0u};
            }
        }
        const bool masked = k0 < all0 || k0 + STEP > all1;
        T8 pt[NQ];
        float back[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float4_t s[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[h] = (float4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < KS; ++t) s[h] = Elem<TYPE>::mfma16(k[h][t], q[n][t], s[h]);
            }
            float e[8], top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = p.cap > 0.f ? capped(s[j >> 2][j & 3] * p.cap_in, p.cap_out) : s[j >> 2][j & 3] * p.scale2;
            if (masked) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int key = k0 + 16 * (j >> 2) + 4 * grp + (j & 3);
                    e[j] = key > pos[n] || key <= pos[n] - window ? -INFINITY : e[j];
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, e[j]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m_new = fmaxf(m[n], top), base = m_new == -INFINITY ? 0.f : m_new;
            back[n] = exp2_of(m[n] - base);
            m[n] = m_new;
            l[n] *= back[n];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = exp2_of(e[j] - base);
                l[n] += x;
                pt[n][j] = (T)x;                             // (the weight of V in the element type: half an ulp of it, as much as the result's own rounding)
            }
        }
#pragma unroll
        for (int j = 0; j < VI; ++j) {
            const int key = (j * 64 + lane) / CH, piece = lane % CH, sw = (key >> SW_SHIFT) & SW_MASK;
            *reinterpret_cast<u32x4_t*>(vb + key * (D * 2) + ((piece >> 1) ^ sw) * 32 + (piece & 1) * 16) = v[j];
        }
        wave_sync();
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
            for (int n = 0; n < NQ; ++n) {
#pragma unroll
                for (int j = 0; j < 4; ++j) o[n][t][j] *= back[n];
                o[n][t] = Elem<TYPE>::mfma16(a.v, pt[n], o[n][t]);
            }
        }
        wave_sync();
    }
    // the four wavefronts' keys, 16 rows at a time
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        l[n] += __shfl_xor(l[n], 16);
        l[n] += __shfl_xor(l[n], 32);
        if (grp == 0) {
            stats[wave][0][16 * n + col] = m[n];
            stats[wave][1][16 * n + col] = l[n];
        }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        if (n) __syncthreads();
        float* const mine = reinterpret_cast<float*>(vb) + col * (D + 4);
#pragma unroll
        for (int t = 0; t < DT; ++t) *reinterpret_cast<float4_t*>(mine + t * 16 + grp * 4) = o[n][t];
        __syncthreads();
        for (int i = tid; i < min(16, w.rows - 16 * n) * (D / 4); i += 256) {
            const int r = i / (D / 4), d = i % (D / 4) * 4;
            float top = -INFINITY;
#pragma unroll
            for (int x = 0; x < 4; ++x) top = fmaxf(top, stats[x][0][16 * n + r]);
            const float base = top == -INFINITY ? 0.f : top;
            float4_t acc = {0.f, 0.f, 0.f, 0.f};
            float den = 0.f;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float f = exp2_of(stats[x][0][16 * n + r] - base);
                den += f * stats[x][1][16 * n + r];
                const float4_t y = *reinterpret_cast<const float4_t*>(reinterpret_cast<const float*>(buf[x]) + r * (D + 4) + d);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] += f * y[j];
            }
            if (w.parts > 1) {
                *reinterpret_cast<float4_t*>(partial_sums(p, head, w.slot + w.part, ROWS, D) + (16 * n + r) * D + d) = acc;
                if (d == 0) {
                    float* const st = partial_stats(p, head, w.slot + w.part, ROWS, D) + (16 * n + r) * 2;
                    st[0] = top;
                    st[1] = den;
                }
            } else {
                const float inv = den > 0.f ? 1.0f / den : 0.f;
                const int row = w.row0 + 16 * n + r, tok = row / p.G;
                T4 y;
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = (T)(acc[j] * inv);
                *reinterpret_cast<T4*>(static_cast<T*>(p.out) + ((int64_t)(w.tok0 + tok) * p.Hq + head * p.G + row - tok * p.G) * D + d) = y;
            }
        }
    }
}

// Workgroup barrier behind a wavefront's loads into LDS and its reads.  (The builtin wait: the compiler counts on from it, where after one in
// assembly it would have a stage's reads wait for the next stage's loads.)
__device__ __forceinline__ void landed() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);                      // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Many rows: 128 of them a workgroup, 32 a wavefront, over blocks of KEYS keys that are staged in LDS, the next block on its way while one is
// worked on.  Bound by the matrix cores and, about as much, by the exponentials: two workgroups share a compute unit, so that one's
// products run beside the other's softmax.  Rows of a staged block are permuted by 16-byte pieces (K: by the key's last three
// bits; V: four pieces at a time by its last two, or, two rows of 64 lying side by side, the second of them), which spreads what the matrix operands read over all banks; the loads into LDS, whose
// destinations are in lane order, take their sources permuted instead.
constexpr int kTileRows = 128;

__device__ __align__(16) uint32_t attention_zeros[4];        // what a key outside the request has for V

template <int TYPE, int D, int KEYS>
__global__ __launch_bounds__(256, 2) void attend_tiles_kernel(const AttnParams p) {
    typedef typename Elem<TYPE>::one T;
    typedef typename Elem<TYPE>::x8 T8;
    typedef typename Elem<TYPE>::x4 T4;
    constexpr int KS = D / 16, DT = D / 32, KT = KEYS / 32;  // k-steps of K Q^T, 32-row tiles of O^T, 32-key tiles of S^T
    constexpr int CH = D / 8, PER = 64 / CH;                 // 16-byte pieces of a row, rows a load of a wavefront brings
    constexpr int MINE = KEYS / 4, LOADS = MINE / PER;       // rows of a block that a wavefront brings, in so many loads
    static_assert(LOADS >= 1 && MINE <= 16, "a wavefront's share of a block is in one page");
    __shared__ __align__(16) uint8_t lds_k0[KEYS * D * 2], lds_k1[KEYS * D * 2], lds_v0[KEYS * D * 2], lds_v1[KEYS * D * 2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, hi = lane >> 5;
    const int head = blockIdx.x % p.Hk;
    clear_padding<256>(p, D);
    Piece w;
    if (!find_piece<kTileRows, KEYS, true>(p, blockIdx.x / p.Hk, &w)) return;

    const int wrow = wave * 32, row = w.row0 + min(wrow + col, w.rows - 1), tok = row / p.G, qh = head * p.G + row - tok * p.G;
    const int pos = w.ctx + tok;
    T8 q[KS];
    {
        const T* const qp = static_cast<const T*>(p.q) + (int64_t)(w.tok0 + tok) * p.q_stride + (int64_t)qh * D + hi * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const T8*>(qp + s * 16);
    }
    float16_t o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[t][j] = 0.f;
    float m = -INFINITY, l = 0.f;
    const int32_t* const table = p.table + (int64_t)w.b * p.table_stride;
    const int ps = 1 << p.shift;
    // keys that every row of this wavefront sees need no masks; those that none sees no work
    const int lo_row = w.row0 + min(wrow, w.rows - 1), hi_row = w.row0 + min(wrow + 31, w.rows - 1);
    const int pos_lo = w.ctx + __builtin_amdgcn_readfirstlane(lo_row / p.G), pos_hi = w.ctx + __builtin_amdgcn_readfirstlane(hi_row / p.G);
    const int window = p.window ? p.window : 0x7FFFFFFF;
    const int all0 = p.window ? pos_hi - p.window + 1 : 0, all1 = pos_lo + 1;
    const int any0 = p.window ? pos_lo - p.window + 1 : 0, any1 = wrow < w.rows ? pos_hi + 1 : 0;

    // sources of a wavefront's loads: rows MINE wave .. of a block, a lane's piece permuted back
    uint32_t koff[LOADS], voff[LOADS];                       // in elements
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        const int r = j * PER + lane / CH, rr = MINE * wave + r, piece = lane % CH;
        koff[j] = r * (uint32_t)p.token_stride + (piece ^ (rr & 7)) * 8;
        voff[j] = r * (uint32_t)p.token_stride + (piece ^ (D == 64 ? (rr & 2) * 2 : (rr & 3) * 4)) * 8;
    }
    int ids = 0;
    auto stage = [&](int block, uint8_t* kb, uint8_t* vb) {
        const int key = block * KEYS + MINE * wave, i = block - w.k0;
        if ((i & 63) == 0) {                                 // the pages of the next 64 blocks, none outside what is seen
            const int at = min(max(key + lane * KEYS, w.kv0), w.kv1 - 1);
            ids = min((uint32_t)table[at >> p.shift], (uint32_t)(p.pages - 1));
        }
        const int64_t page = __builtin_amdgcn_readlane(ids, i & 63);
        const int64_t off = page * p.page_stride + head * p.head_stride + (int64_t)(key & (ps - 1)) * p.token_stride;
        const T *const kp = static_cast<const T*>(p.k) + off, *const vp = static_cast<const T*>(p.v) + off;
        const bool edge = key < w.kv0 || key + MINE > w.kv1;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)(kp + koff[j]),
                                             (__attribute__((address_space(3))) void*)(kb + (MINE * wave + j * PER) * D * 2), 16, 0, 0);
            const T* src = vp + voff[j];
            if (edge) {                                      // slots without a token of the request may hold anything
                const int k = key + j * PER + lane / CH;
                if (k < w.kv0 || k >= w.kv1) src = reinterpret_cast<const T*>(attention_zeros);
            }
            __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)src,
                                             (__attribute__((address_space(3))) void*)(vb + (MINE * wave + j * PER) * D * 2), 16, 0, 0);
        }
    };
    auto work = [&](int block, const uint8_t* kb, const uint8_t* vb) {
        const int k0 = block * KEYS;
        if (k0 >= any1 || k0 + KEYS <= any0) return;
        float16_t s[KT];
#pragma unroll
        for (int h = 0; h < KT; ++h) {
#pragma unroll
            for (int j = 0; j < 16; ++j) s[h][j] = 0.f;
#pragma unroll
            for (int t = 0; t < KS; ++t) {
                const T8 a = *reinterpret_cast<const T8*>(kb + (32 * h + col) * D * 2 + (((2 * t + hi) ^ (col & 7)) * 16));
                s[h] = Elem<TYPE>::mfma32(a, q[t], s[h]);
            }
        }
        float scale = p.scale2;
        if (p.cap > 0.f) {
            scale = 1.f;
#pragma unroll
            for (int h = 0; h < KT; ++h)
#pragma unroll
                for (int j = 0; j < 16; ++j) s[h][j] = capped(s[h][j] * p.cap_in, p.cap_out);
        }
        if (k0 < all0 || k0 + KEYS > all1) {
#pragma unroll
            for (int h = 0; h < KT; ++h)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int key = k0 + 32 * h + 8 * (j >> 2) + 4 * hi + (j & 3);
                    s[h][j] = key > pos || key <= pos - window ? -INFINITY : s[h][j];
                }
        }
        float top = -INFINITY;
#pragma unroll
        for (int h = 0; h < KT; ++h)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, s[h][j]);
        top = fmaxf(top, __shfl_xor(top, 32)) * scale;
        // The weights are relative to a maximum that is only followed where it has grown by 2^8: they stay below 2^8, exact to the same share, and the
        // sums, most of the time, need no rescaling.
        if (__any(top > m + 8.f)) {
            const float m_new = fmaxf(m, top), back = m_new == -INFINITY ? 1.f : exp2_of(m - m_new);
            m = m_new;
            l *= back;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[t][j] *= back;
        }
        const float base = m == -INFINITY ? 0.f : m;
        T8 pt[KT * 2];
#pragma unroll
        for (int h = 0; h < KT; ++h)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float x = exp2_of(fmaf(s[h][j], scale, -base));
                l += x;
                pt[2 * h + (j >> 3)][j & 7] = (T)x;          // (the weight of V in the element type: half an ulp of it, as much as the result's own rounding)
            }
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int h = 0; h < KT * 2; ++h) {
                union { T8 v; short4_t s[2]; } a;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int i = lane & 15, g = lane >> 4, key = 16 * h + 8 * x + 4 * (g >> 1) + (i >> 2);
                    const int piece = (4 * t + 2 * (g & 1) + ((i & 3) >> 1)) ^ (D == 64 ? (key & 2) * 2 : (key & 3) * 4);
                    a.s[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) short4_t*)(vb + key * D * 2 + piece * 16 + (i & 1) * 8));
                }
                o[t] = Elem<TYPE>::mfma32(a.v, pt[h], o[t]);
            }
    };

    // (the queries are waited for here: in the loop that would be a wait for the loads into LDS as well)
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(q[s]));
    if (w.k0 < w.k1) stage(w.k0, lds_k0, lds_v0);
    for (int block = w.k0; block < w.k1; block += 2) {
        landed();
        if (block + 1 < w.k1) stage(block + 1, lds_k1, lds_v1);
        work(block, lds_k0, lds_v0);
        if (block + 1 >= w.k1) break;
        landed();
        if (block + 2 < w.k1) stage(block + 2, lds_k0, lds_v0);
        work(block + 1, lds_k1, lds_v1);
    }
    l += __shfl_xor(l, 32);
    if (wrow + col >= w.rows) return;
    if (w.parts > 1) {
        float* const po = partial_sums(p, head, w.slot + w.part, kTileRows, D) + (wrow + col) * D;
        float* const st = partial_stats(p, head, w.slot + w.part, kTileRows, D) + (wrow + col) * 2;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int j = 0; j < 16; j += 4)
                *reinterpret_cast<float4_t*>(po + t * 32 + 2 * j + 4 * hi) = (float4_t){o[t][j], o[t][j + 1], o[t][j + 2], o[t][j + 3]};
        if (hi == 0) {
            st[0] = m;
            st[1] = l;
        }
    } else {
        const float inv = l > 0.f ? 1.0f / l : 0.f;
        T* const dst = static_cast<T*>(p.out) + ((int64_t)(w.tok0 + tok) * p.Hq + qh) * D;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                T4 y;
#pragma unroll
                for (int x = 0; x < 4; ++x) y[x] = (T)(o[t][j + x] * inv);
                *reinterpret_cast<T4*>(dst + t * 32 + 2 * j + 4 * hi) = y;
            }
    }
}

// The launch for a call: tiles of 16 or 32 rows, and the pieces aimed at.  Bytes of a partial result of one KV head: rows (D + 2) floats.
struct AttnPlan {
    int rows, pieces;
    int64_t slot_bytes(int D) const { return (int64_t)rows * (D + 2) * 4; }
    size_t bytes(int Hk, int D) const { return (size_t)(2 * (int64_t)pieces * Hk * slot_bytes(D)); }
};

static AttnPlan plan_attention(int64_t T, int B, int Hq, int Hk, int D, int max_new) {
    const int G = Hq / Hk;
    AttnPlan a;
    const int64_t rows = (int64_t)max_new * G;
    a.rows = rows > 64 ? kTileRows : rows <= 16 || D == 256 ? 16 : 32;
    a.pieces = ((a.rows == kTileRows ? kTilePieces : kPieces) + Hk - 1) / Hk;
    return a;
}

template <int TYPE, int D, int NQ>
static void launch_rows(const AttnParams& p, hipStream_t st) {
    const int64_t tiles = (int64_t)p.T * p.G / (16 * NQ) + p.B;
    hipLaunchKernelGGL((attend_rows_kernel<TYPE, D, NQ>), dim3((unsigned)((tiles + p.pieces) * p.Hk)), dim3(256), 0, st, p);
    if (p.pieces) hipLaunchKernelGGL((join_parts_kernel<TYPE, D, 16 * NQ, 128>), dim3((unsigned)(tiles * p.Hk)), dim3(256), 0, st, p);
}

template <int TYPE, int D>
static void launch_attention(const AttnParams& p, const AttnPlan& a, hipStream_t st) {
    if (a.rows == kTileRows) {
        constexpr int KEYS = D == 256 ? 32 : 64;
        const int64_t tiles = (int64_t)p.T * p.G / kTileRows + p.B;
        hipLaunchKernelGGL((attend_tiles_kernel<TYPE, D, KEYS>), dim3((unsigned)((tiles + p.pieces) * p.Hk)), dim3(256), 0, st, p);
        if (p.pieces) hipLaunchKernelGGL((join_parts_kernel<TYPE, D, kTileRows, KEYS>), dim3((unsigned)(tiles * p.Hk)), dim3(256), 0, st, p);
        return;
    }
    if constexpr (D < 256) {
        if (a.rows == 32) return launch_rows<TYPE, D, 2>(p, st);
    }
    launch_rows<TYPE, D, 1>(p, st);
}

}  // namespace rtn

extern "C" size_t rtn_paged_attention_workspace_nbytes(int64_t tokens, int n_requests, int q_heads, const rtn_kv_cache* cache, int max_new) {
    if (rtn::check_cache(cache) != RTN_OK || tokens < 0 || tokens > 1 << 24 || n_requests < 1 || n_requests > 65536 || q_heads < 1 ||
        q_heads % cache->kv_heads != 0 || q_heads / cache->kv_heads > 64 || max_new < 1)
        return 0;
    return rtn::plan_attention(tokens, n_requests, q_heads, cache->kv_heads, cache->head_dim, max_new).bytes(cache->kv_heads, cache->head_dim);
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
    const rtn::AttnPlan a = rtn::plan_attention(tokens, n_requests, q_heads, cache->kv_heads, D, max_new);
    const int64_t room = dev_workspace ? (int64_t)(workspace_nbytes / (size_t)(2 * cache->kv_heads * a.slot_bytes(D))) : 0;
    const float log2e = 1.4426950408889634f;
    const rtn::AttnParams p = {dev_q, cache->dev_k, cache->dev_v, dev_out, dev_block_table, dev_seq_lens, dev_query_start, q_stride, cache->page_stride,
                               cache->head_stride, cache->token_stride, table_stride, (int)cache->pages, rtn::log2_of(cache->page_size), max_blocks,
                               n_requests, (int)tokens, q_heads, cache->kv_heads, q_heads / cache->kv_heads, window, scale * log2e, softcap,
                               softcap > 0.f ? scale / softcap : 0.f, softcap * log2e, static_cast<float*>(dev_workspace),
                               (int)(room < a.pieces ? room : a.pieces)};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (cache->dtype == RTN_TYPE_F16) {
        if (D == 64) rtn::launch_attention<RTN_TYPE_F16, 64>(p, a, s);
        else if (D == 128) rtn::launch_attention<RTN_TYPE_F16, 128>(p, a, s);
        else rtn::launch_attention<RTN_TYPE_F16, 256>(p, a, s);
    } else {
        if (D == 64) rtn::launch_attention<RTN_TYPE_BF16, 64>(p, a, s);
        else if (D == 128) rtn::launch_attention<RTN_TYPE_BF16, 128>(p, a, s);
        else rtn::launch_attention<RTN_TYPE_BF16, 256>(p, a, s);
    }
    return hipGetLastError() == hipSuccess ? RTN_OK : RTN_ERR_HIP;
}
