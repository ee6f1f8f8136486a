// Attention of a batch of requests' new tokens over their pages.
//
// A request's queries of one KV head are rows: row r is token r / G and head r % G of the G query heads that share the KV head, so that what a
// tile of rows reads of K and V serves all of them, in a decode step of one token as in a piece of a prompt.  A workgroup takes a tile of rows of
// one request and KV head.  Which request that is it finds from query_start itself: the host knows no lengths.
//
// Scores are formed transposed, S^T = K Q^T, one query a lane: the matrix instruction then leaves each lane several keys of one
// query, whose maximum and sum are the lane's own but for the last steps, and what it leaves is, as it stands, the operand P^T of
// O^T = V^T P^T, if V's keys are taken in the same order.  V^T's operands come out of LDS by transposing reads.
#include "rtn_paged.h"

#include <algorithm>
#include <float.h>
#include <math.h>

namespace rtn {

// Requests of up to kFew rows go to the workgroups for few rows, longer ones to those for many (kTileRows).
constexpr int kFew = 64, kTileRows = 256;

// One of the two kinds of workgroups in a launch.  `pieces` a KV head are aimed at (0: no request is split), and a head has room for twice as many
// partial results, [Hk][2 pieces][rows][D] sums and, behind them, [Hk][2 pieces][rows][2] maxima and sums of weights.
struct AttnKind {
    float* partial;
    int pieces, most, slots;                                 // bounds on the pieces of a KV head and on those of split requests
};

struct AttnParams {
    const void *q, *k, *v;
    void* out;
    const int32_t *table, *seq, *start;
    int64_t q_stride, page_stride, head_stride, token_stride, table_stride;
    int pages, shift, max_blocks, B, T, Hq, Hk, G, window;
    float scale2, cap, cap_in, cap_out;                      // scale log2 e; softcap: 2 scale log2 e / softcap, softcap log2 e
    uint32_t g_inv, g_one;                                   // row -> token is umulhi(row, g_inv) + (row & g_one): exact below 2^26 rows and G <= 64
    int few_rows;                                            // kFew, or no bound where the call's requests are all taken to have few
    AttnKind few, many;
};

__device__ __forceinline__ int token_of(const AttnParams& p, int row) { return (int)(__umulhi((uint32_t)row, p.g_inv) + ((uint32_t)row & p.g_one)); }

// exp2 of scores: the softmax is taken to base 2, with log2 e in the scale
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// softcap tanh(x) log2 e, x = s scale / softcap, for s = q.k, with z = 2 x log2 e = cap_in s.  From |x| = 1/5 on cap_out (1 - 2 / (2^z + 1)), right at both ends, where
// 2^z is 0 or infinite, with an error of a few ulps of the result.  Below, where that difference would leave an error of cap_out 2^-23 whatever the score, the
// series of tanh(x) / x (its next term is below 2^-24) times the score without a cap: the error is relative to the score at any cap, one that makes z underflow
// included.  (Both are formed first, so that the choice is no branch.  Ten more instructions a score: three prompt pieces on 16 heads of 256 157 us, 146 without the
// series; a branch for wavefronts without large scores keeps both forms' registers, 166.)
__device__ __forceinline__ float capped(const AttnParams& p, float s) {
    constexpr double k = 0.12011325347955035;                // x^2 = k z^2
    constexpr float c1 = (float)(-k / 3), c2 = (float)(2 * k * k / 15), c3 = (float)(-17 * k * k * k / 315), limit = 0.57707802f;
    const float z = s * p.cap_in, y = z * z;
    const float series = fmaf(y, fmaf(y, (y + c2 / c3) * c3, c1), 1.0f);         // (a sum and a product take their constants as they are, a register less)
    const float small = s * p.scale2 * series, large = p.cap_out * (1.0f - 2.0f * __builtin_amdgcn_rcpf(exp2_of(z) + 1.0f));
    return fabsf(z) < limit ? small : large;
}

// Weights of V go to the matrix cores in the element type.  fp16 has normal numbers from 2^-14 to 2^16 only, and a long cache whose largest score is far above the others
// has its sum in weights below that: they are multiplied by a power of two that takes the largest possible one to 2^15.  The sums carry it too, so it divides out.
// (bf16 has fp32's range.)
template <int TYPE> constexpr float weight_lift(float most) { return TYPE == RTN_TYPE_F16 ? 15.0f - most : 0.0f; }      // log2; `most`: that of the largest weight

// What a workgroup does: ROWS rows from row0 of request b, a part of their keys.
struct Piece {
    int b, row0, rows, tok0, n, ctx;                         // rows of the tile, first token in the batch, new tokens, cached tokens
    int kv0, kv1;                                            // keys that some row sees
    int part, parts, slot;                                   // of the tile's keys; where the first part's partial result goes
    int k0, k1;                                              // this part's, in blocks of KEYS
};

// Each workgroup finds its own piece from the requests' lengths, which the host does not know: with n_b blocks of keys and t_b
// tiles of rows, pieces of c = ceil(sum t_b n_b / `pieces`) blocks put a like share of the whole batch's keys on every workgroup, whatever the
// requests' lengths; tile t of request b has the t_b ceil(n_b / c) pieces after those of the requests before it.  Two scans over the requests, each
// thread's own (one, up to as many requests as threads) read once.  `no` counts the pieces, or, JOIN, those of split requests alone.  All threads call it.
template <int ROWS, int KEYS, bool JOIN, int WAVES>
__device__ __forceinline__ bool find_piece(const AttnParams& p, int pieces, int no, Piece* out) {
#pragma clang fp contract(off)                               // (the workgroups of a piece and those that join its parts come to the same shares)
    __shared__ float totals[WAVES];
    __shared__ int counts[WAVES][2], sums[WAVES][2], found[8];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (p.B + 64 * WAVES - 1) / (64 * WAVES), b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
    struct Request { int tok0, n, seq, tiles, blocks; };
    auto read = [&](int b) {
        Request r;
        const int s = p.start[b], e = p.start[b + 1], len = p.seq[b];
        r.tok0 = min(max(s, 0), p.T);
        r.n = min(max(e, r.tok0), p.T) - r.tok0;
        r.seq = min(max(len, 0), p.max_blocks << p.shift);
        const int rows = r.n * p.G;
        r.tiles = (rows > p.few_rows) == (ROWS > kFew) ? (rows + ROWS - 1) / ROWS : 0;
        // (with a window, a bound on what a tile sees: the windows of its tokens, unaligned)
        r.blocks = (r.seq + KEYS - 1) / KEYS;
        if (p.window) r.blocks = (int)min((int64_t)r.blocks, ((int64_t)p.window + ROWS / p.G + 1 + KEYS - 1) / KEYS + 1);
        return r;
    };
    // Blocks of a piece.  Few rows: where the tiles alone fill the compute units and the longest has little more than its share, none is split (64 requests of
    // 1020 tokens 49 us split in two, 43 whole; of 300 to 8000 tokens 199 split, 210 with parts twice as long).
    auto shares = [&](float total, int tiles, int longest) {
        if (pieces == 0 || (ROWS <= kFew && 2 * tiles >= pieces && (float)longest * (float)tiles <= 1.25f * total)) return 1 << 30;
        // (not below the exact share, for the room that there is for partial results: the sums' rounding is less than 2^-10)
        return (int)fminf(0x1p30f, fmaxf(1.f, ceilf(total * (1.0f + 0x1p-10f) / (float)pieces)));
    };
    int c, local, most, slot, n, seq;
    auto parts_of = [&](int blocks) { return max(1, (int)(((uint32_t)blocks + c - 1) / c)); };      // (up to 2^26 blocks)
    if (p.B <= 64) {                                         // a lane a request: each wavefront by itself, without LDS
        Request r = {};
        if (lane < p.B) r = read(lane);
        c = shares(__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wave_scan((float)r.tiles * (float)r.blocks)), 63)),
                   __builtin_amdgcn_readlane(wave_scan(r.tiles), 63), __builtin_amdgcn_readlane(wave_max(r.tiles ? r.blocks : 0), 63));
        const int parts = parts_of(r.blocks), have = r.tiles * parts, slots = parts > 1 ? have : 0;
        const int slots_before = wave_scan(slots) - slots, before = JOIN ? slots_before : wave_scan(have) - have;
        const uint64_t hit = __ballot(no >= before && no < before + (JOIN ? slots : have));
        if (hit == 0) return false;
        const int b = __builtin_ctzll(hit);
        out->b = b;
        local = no - __builtin_amdgcn_readlane(before, b);
        slot = __builtin_amdgcn_readlane(slots_before, b);
        most = __builtin_amdgcn_readlane(parts, b);
        out->tok0 = __builtin_amdgcn_readlane(r.tok0, b);
        n = __builtin_amdgcn_readlane(r.n, b);
        seq = __builtin_amdgcn_readlane(r.seq, b);
    } else {
        Request own = {};
        if (b0 < b1) own = read(b0);
        auto request = [&](int b) { return b == b0 ? own : read(b); };
        float total = 0.f;
        int all = 0, longest = 0;
        for (int b = b0; b < b1; ++b) {
            const Request r = request(b);
            total += (float)r.tiles * (float)r.blocks;
            all += r.tiles;
            longest = max(longest, r.tiles ? r.blocks : 0);
        }
        total = wave_scan(total);
        all = wave_scan(all);
        longest = wave_max(longest);
        if (lane == 63) {
            totals[wave] = total;
            counts[wave][0] = all;
            counts[wave][1] = longest;
        }
        __syncthreads();
        total = 0.f;
        all = longest = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            total += totals[w];
            all += counts[w][0];
            longest = max(longest, counts[w][1]);
        }
        c = shares(total, all, longest);
        int mine[2] = {0, 0};                                // pieces, and those of split requests
        for (int b = b0; b < b1; ++b) {
            const Request r = request(b);
            const int parts = parts_of(r.blocks);
            mine[0] += r.tiles * parts;
            mine[1] += parts > 1 ? r.tiles * parts : 0;
        }
        const int incl[2] = {wave_scan(mine[0]), wave_scan(mine[1])};
        if (lane == 63) {
            sums[wave][0] = incl[0];
            sums[wave][1] = incl[1];
        }
        if (tid == 0) found[0] = -1;
        __syncthreads();
        int before = incl[0] - mine[0], slots_before = incl[1] - mine[1];
        for (int w = 0; w < wave; ++w) {
            before += sums[w][0];
            slots_before += sums[w][1];
        }
        if (JOIN) before = slots_before;
        if (no >= before && no < before + mine[JOIN ? 1 : 0]) {
            for (int b = b0; b < b1; ++b) {
                const Request r = request(b);
                const int parts = parts_of(r.blocks), slots = parts > 1 ? r.tiles * parts : 0, have = JOIN ? slots : r.tiles * parts;
                if (no < before + have) {
                    found[0] = b;
                    found[1] = no - before;
                    found[2] = slots_before;
                    found[3] = parts;
                    found[4] = r.tok0;
                    found[5] = r.n;
                    found[6] = r.seq;
                    break;
                }
                before += have;
                slots_before += slots;
            }
        }
        __syncthreads();
        out->b = __builtin_amdgcn_readfirstlane(found[0]);
        if (out->b < 0) return false;
        local = __builtin_amdgcn_readfirstlane(found[1]);
        slot = __builtin_amdgcn_readfirstlane(found[2]);
        most = __builtin_amdgcn_readfirstlane(found[3]);
        out->tok0 = __builtin_amdgcn_readfirstlane(found[4]);
        n = __builtin_amdgcn_readfirstlane(found[5]);
        seq = __builtin_amdgcn_readfirstlane(found[6]);
    }
    const int tiles = (n * p.G + ROWS - 1) / ROWS, nth = local / most;
    const int tile = tiles - 1 - nth;                        // the last rows see most keys: they come first
    out->n = n;
    out->ctx = seq - n;
    out->row0 = tile * ROWS;
    out->rows = min(ROWS, out->n * p.G - out->row0);
    const int first = out->ctx + token_of(p, out->row0), last = out->ctx + token_of(p, out->row0 + out->rows - 1);
    out->kv0 = p.window ? max(0, first - p.window + 1) : 0;
    out->kv1 = last + 1;                                     // (not above the length; 0 and less where nothing is seen)
    // the tile's own blocks, which may be fewer than its request's: as many parts as they fill, of like size
    const int blocks = max(0, (out->kv1 + KEYS - 1) / KEYS - out->kv0 / KEYS);
    out->parts = min(most, parts_of(blocks));
    out->part = local - nth * most;
    out->slot = slot + nth * most;
    const int each = (blocks + out->parts - 1) / out->parts;
    out->k0 = out->kv0 / KEYS + out->part * each;
    out->k1 = min(out->k0 + each, out->kv0 / KEYS + blocks);
    return out->part < out->parts;
}

__device__ __forceinline__ float* partial_sums(const AttnParams& p, const AttnKind& kind, int head, int slot, int rows, int D) {
    return kind.partial + ((int64_t)head * 2 * kind.pieces + slot) * rows * D;
}
__device__ __forceinline__ float* partial_stats(const AttnParams& p, const AttnKind& kind, int head, int slot, int rows, int D) {
    return kind.partial + (int64_t)p.Hk * 2 * kind.pieces * rows * D + ((int64_t)head * 2 * kind.pieces + slot) * rows * 2;
}

// Rows of a padded batch, from `end` on, get zeros: every workgroup a share, whatever it does else.  (The end is read before the piece is found,
// used after it: as a wait of its own it would be most of a microsecond.)
template <int THREADS>
__device__ __forceinline__ void clear_padding(const AttnParams& p, int end, int D) {
    const int64_t per_token = (int64_t)p.Hq * D / 8, first = min(max(end, 0), p.T) * per_token;
    for (int64_t i = first + (int64_t)blockIdx.x * THREADS + threadIdx.x; i < p.T * per_token; i += (int64_t)gridDim.x * THREADS)
        reinterpret_cast<u32x4_t*>(p.out)[i] = (u32x4_t){0u, 0u, 0u, 0u};
}

// The parts of a tile's keys, brought to their common maximum and added up.  The workgroups of a tile, as many as it has parts, share its rows.
// D / 4 threads take a row's sums of a part: as many rows at a time as there are threads for or, of fewer rows, several parts of them.
template <int TYPE, int D, int ROWS, int KEYS, int WAVES>
__device__ __forceinline__ void join_parts(const AttnParams& p, const AttnKind& kind, int block) {
    typedef typename Elem<TYPE>::one T;
    typedef typename Elem<TYPE>::x4 T4;
    constexpr int LANES = D / 4, GROUPS = 64 * WAVES / LANES;
    __shared__ __align__(16) float sums[GROUPS][D];
    __shared__ float stats[GROUPS][2];
    const int head = block % p.Hk, lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    Piece w;
    if (!find_piece<ROWS, KEYS, true, WAVES>(p, kind.pieces, block / p.Hk, &w) || w.parts == 1) return;
    const float *const po = partial_sums(p, kind, head, w.slot, ROWS, D) + lane * 4, *const pm = partial_stats(p, kind, head, w.slot, ROWS, D);
    const int r0 = w.rows * w.part / w.parts, r1 = w.rows * (w.part + 1) / w.parts;
    int at_once = 1;                                         // rows; the other groups share a row's parts
    while (at_once < GROUPS && at_once < r1 - r0) at_once *= 2;
    const int by_parts = GROUPS / at_once, first = group & (by_parts - 1);
    const int turns = (r1 - r0 + at_once - 1) / at_once;     // as many for all groups: there are barriers in them
    for (int turn = 0; turn < turns; ++turn) {
        const int r = r0 + turn * at_once + group / by_parts;
        float4_t acc = {0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        auto add = [&](float m2, float l2, const float4_t& x) {
            const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.f : top, f = exp2_of(m - base), g = exp2_of(m2 - base);
            l = l * f + l2 * g;
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = acc[j] * f + x[j] * g;
            m = top;
        };
        if (r < r1) {
#pragma unroll 4
            for (int s = first; s < w.parts; s += by_parts) {
                const float2 st = *reinterpret_cast<const float2*>(pm + ((int64_t)s * ROWS + r) * 2);
                add(st.x, st.y, *reinterpret_cast<const float4_t*>(po + ((int64_t)s * ROWS + r) * D));
            }
        }
        if (by_parts > 1) {
            *reinterpret_cast<float4_t*>(&sums[group][lane * 4]) = acc;
            if (lane == 0) {
                stats[group][0] = m;
                stats[group][1] = l;
            }
            __syncthreads();
            if (first == 0)
                for (int g = 1; g < by_parts; ++g) add(stats[group + g][0], stats[group + g][1], *reinterpret_cast<const float4_t*>(&sums[group + g][lane * 4]));
            __syncthreads();
        }
        if (first == 0 && r < r1) {
            const float inv = l > 0.f ? 1.0f / l : 0.f;
            const int row = w.row0 + r, tok = token_of(p, row);
            T4 y;
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = (T)(acc[j] * inv);
            *reinterpret_cast<T4*>(static_cast<T*>(p.out) + ((int64_t)(w.tok0 + tok) * p.Hq + head * p.G + row - tok * p.G) * D + lane * 4) = y;
        }
    }
}

// Within a wavefront: its own writes to LDS are there for its reads.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Where a 16-byte piece of a staged key row is: 16 rows, as many as the lanes that read at once, in different banks.
template <int D>
__device__ __forceinline__ int k_swizzle(int row) { return D == 64 ? (row >> 1) & 7 : row & 15; }

// Few rows: 16 NQ of them a workgroup, whose wavefronts take blocks of 32 keys in turn, each with a softmax of its own until they join
// at the end.  Bound by the reading of K and V, which go through LDS one after the other, 8 KiB that only its wavefront touches (D = 128), so that
// the loop has no barrier.
constexpr int few_keys(int waves) { return 32 * waves; }              // of a step of the wavefronts
constexpr int few_lds_bytes(int D) { return 16 * (D + 4) * 4; }        // of a wavefront: 32 rows of V, and, later, sums of 16 rows

template <int TYPE, int D, int NQ, int WAVES>
__device__ __forceinline__ void attend_few(const AttnParams& p, int block, uint8_t* const (&buf)[WAVES], uint8_t* const vb) {
    typedef typename Elem<TYPE>::one T;
    typedef typename Elem<TYPE>::x8 T8;
    typedef typename Elem<TYPE>::x4 T4;
    constexpr int KS = D / 32, DT = D / 16, STEP = 32, ROWS = 16 * NQ, KEYS = few_keys(WAVES);     // k-steps of K Q^T, 16-row tiles of O^T, keys of a step
    constexpr int SW_SHIFT = D == 64 ? 1 : 0, SW_MASK = D == 64 ? 3 : 7;
    constexpr int VI = STEP * D * 2 / 1024, CH = D / 8;      // loads of V, 16-byte pieces of a row
    __shared__ float stats[WAVES][2][ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, grp = lane >> 4;
    const int head = block % p.Hk;
    const int end_of_tokens = p.start[p.B];
    Piece w;
    const bool found = find_piece<ROWS, KEYS, false, WAVES>(p, p.few.pieces, block / p.Hk, &w);
    clear_padding<64 * WAVES>(p, end_of_tokens, D);
    if (!found) return;

    T8 q[NQ][KS];
    int pos[NQ];                                             // (negative where the length is below the number of new tokens)
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int row = w.row0 + min(16 * n + col, w.rows - 1), tok = token_of(p, row), qh = head * p.G + row - tok * p.G;
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
    const int32_t* const table = p.table + (int64_t)w.b * p.table_stride;
    const int ps = 1 << p.shift;
    // keys that every row sees need no masks
    const int window = p.window ? p.window : 1 << 30;        // (no length is above 2^30)
    const int all0 = p.window ? w.ctx + token_of(p, w.row0 + w.rows - 1) - p.window + 1 : 0, all1 = w.ctx + token_of(p, w.row0) + 1;
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
        // Whole rows by neighbouring lanes, as streaming: half rows, as the matrix cores take K, read 5 to 10 % slower.
        auto load = [&](u32x4_t (&x)[VI], const T* const (&from)[2]) {
#pragma unroll
            for (int j = 0; j < VI; ++j) {
                const int key = (j * 64 + lane) / CH, piece = lane % CH;
                x[j] = load_stream16(from[j * 64 / CH >> 4] + (key & 15) * (int)p.token_stride + piece * 8);
            }
        };
        u32x4_t k[VI], v[VI];
        load(k, kt);
        if constexpr (D < 256) load(v, vt);
#pragma unroll
        for (int j = 0; j < VI; ++j) {
            const int key = (j * 64 + lane) / CH, piece = lane % CH;
            *reinterpret_cast<u32x4_t*>(vb + key * (D * 2) + (piece ^ k_swizzle<D>(key)) * 16) = k[j];
        }
        wave_sync();
        float4_t s[NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[n][0] = s[n][1] = (float4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < KS; ++t) {
                const T8 a = *reinterpret_cast<const T8*>(vb + (16 * h + col) * (D * 2) + ((4 * t + grp) ^ k_swizzle<D>(col)) * 16);
#pragma unroll
                for (int n = 0; n < NQ; ++n) s[n][h] = Elem<TYPE>::mfma16(a, q[n][t], s[n][h]);
            }
        wave_sync();
        const bool masked = k0 < all0 || k0 + STEP > all1;
        // The weights of V are rounded to the element type and, up to 128 elements a head, so is what that leaves of them: a second product with it, in a
        // kernel that waits for memory, costs nothing (64 ragged requests 199 us both ways) and takes the result's error, against 64 bits, from 1.3 to
        // 1.0 times that of its own rounding.  Heads of 256 have no registers for it (65 us, 72 with it).
        constexpr bool REST = D < 256;
        T8 pt[NQ], rest[REST ? NQ : 1];
        float back[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float e[8], top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = p.cap > 0.f ? capped(p, s[n][j >> 2][j & 3]) : s[n][j >> 2][j & 3] * p.scale2;
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
            const float m_new = fmaxf(m[n], top), base = m_new == -INFINITY ? 0.f : m_new, from = base - weight_lift<TYPE>(0.f);
            back[n] = exp2_of(m[n] - base);
            m[n] = m_new;
            l[n] *= back[n];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = exp2_of(e[j] - from);
                l[n] += x;
                pt[n][j] = (T)x;
                if constexpr (REST) rest[n][j] = (T)(x - (float)pt[n][j]);
            }
        }
        if constexpr (D == 256) load(v, vt);                 // (not beside K: 128 registers)
        if (k0 < w.kv0 || k0 + STEP > w.kv1) {               // slots without a token of the request may hold anything
#pragma unroll
            for (int j = 0; j < VI; ++j) {
                const int key = k0 + (j * 64 + lane) / CH;
                if (key < w.kv0 || key >= w.kv1) v[j] = (u32x4_t){0u, 0u, 0u, 0u};
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
                if constexpr (REST) o[n][t] = Elem<TYPE>::mfma16(a.v, rest[n], o[n][t]);
            }
        }
        wave_sync();
    }
    // the wavefronts' keys, 16 rows at a time
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
        for (int i = tid; i < min(16, w.rows - 16 * n) * (D / 4); i += 64 * WAVES) {
            const int r = i / (D / 4), d = i % (D / 4) * 4;
            float top = -INFINITY;
#pragma unroll
            for (int x = 0; x < WAVES; ++x) top = fmaxf(top, stats[x][0][16 * n + r]);
            const float base = top == -INFINITY ? 0.f : top;
            float4_t acc = {0.f, 0.f, 0.f, 0.f};
            float den = 0.f;
#pragma unroll
            for (int x = 0; x < WAVES; ++x) {
                const float f = exp2_of(stats[x][0][16 * n + r] - base);
                den += f * stats[x][1][16 * n + r];
                const float4_t y = *reinterpret_cast<const float4_t*>(reinterpret_cast<const float*>(buf[x]) + r * (D + 4) + d);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] += f * y[j];
            }
            if (w.parts > 1) {
                *reinterpret_cast<float4_t*>(partial_sums(p, p.few, head, w.slot + w.part, ROWS, D) + (16 * n + r) * D + d) = acc;
                if (d == 0) {
                    float* const st = partial_stats(p, p.few, head, w.slot + w.part, ROWS, D) + (16 * n + r) * 2;
                    st[0] = top;
                    st[1] = den;
                }
            } else {
                const float inv = den > 0.f ? 1.0f / den : 0.f;
                const int row = w.row0 + 16 * n + r, tok = token_of(p, row);
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

// Many rows: 256 of them a workgroup, 32 a wavefront, over blocks of KEYS keys that are staged in LDS, the next block on its way while one is
// worked on.  Bound by the matrix cores and, about as much, by the exponentials, at a clock that the power lets go down to 1.6 GHz: what counts is
// what is moved for a product.  Of a compute unit's eight wavefronts, two to a SIMD, one's products run beside the other's softmax.  (Two workgroups of 128 rows,
// which bring each block twice: 2000 tokens over 30001 2002 us, 1881 this way; 4096 tokens of a prompt 162 and 151.  A wavefront a SIMD with 64 rows, which
// would read LDS half as often, keeps its sums where the softmax cannot use them and takes 2.9 ms; halves of the keys half a step apart, two barriers a
// block, 2.1.)  Rows of a staged block are permuted by 16-byte pieces (K: by the key's last four
// bits; V: four pieces at a time by its last two, or, two rows of 64 lying side by side, the second of them), which spreads what the matrix operands read over all banks; the loads into LDS, whose
// destinations are in lane order, take their sources permuted instead.
__device__ __align__(16) uint32_t attention_zeros[4];        // what a key outside the request has for V

constexpr int tile_keys(int D) { return D == 256 ? 32 : 64; }

template <int TYPE, int D, bool CAP>
__device__ __forceinline__ void attend_many(const AttnParams& p, int block_no, uint8_t* lds_k0, uint8_t* lds_k1, uint8_t* lds_v0, uint8_t* lds_v1) {
    typedef typename Elem<TYPE>::one T;
    typedef typename Elem<TYPE>::x8 T8;
    typedef typename Elem<TYPE>::x4 T4;
    constexpr int KEYS = tile_keys(D), KS = D / 16, DT = D / 32, KT = KEYS / 32;  // k-steps of K Q^T, 32-row tiles of O^T, 32-key tiles of S^T
    constexpr int CH = D / 8, PER = 64 / CH;                 // 16-byte pieces of a row, rows a load of a wavefront brings
    constexpr int MINE = KEYS / 8, LOADS = MINE / PER;       // rows of a block that a wavefront brings, in so many loads
    static_assert(LOADS >= 1 && MINE <= 16, "a wavefront's share of a block is in one page");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, hi = lane >> 5;
    const int head = block_no % p.Hk;
    const int end_of_tokens = p.start[p.B];
    Piece w;
    const bool found = find_piece<kTileRows, KEYS, false, 8>(p, p.many.pieces, block_no / p.Hk, &w);
    clear_padding<512>(p, end_of_tokens, D);
    if (!found) return;

    const int wrow = wave * 32, row = w.row0 + min(wrow + col, w.rows - 1), tok = token_of(p, row), qh = head * p.G + row - tok * p.G;
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
    const int pos_lo = w.ctx + __builtin_amdgcn_readfirstlane(token_of(p, lo_row)), pos_hi = w.ctx + __builtin_amdgcn_readfirstlane(token_of(p, hi_row));
    const int window = p.window ? p.window : 1 << 30;
    const int all0 = p.window ? pos_hi - p.window + 1 : 0, all1 = pos_lo + 1;
    const int any0 = p.window ? pos_lo - p.window + 1 : 0, any1 = wrow < w.rows ? pos_hi + 1 : 0;

    // sources of a wavefront's loads: rows MINE wave .. of a block, a lane's piece permuted back
    uint32_t koff[LOADS], voff[LOADS];                       // in bytes
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        const int r = j * PER + lane / CH, rr = MINE * wave + r, piece = lane % CH;
        koff[j] = (r * (uint32_t)p.token_stride + (piece ^ k_swizzle<D>(rr)) * 8) * sizeof(T);
        voff[j] = (r * (uint32_t)p.token_stride + (piece ^ (D == 64 ? (rr & 2) * 2 : (rr & 3) * 4)) * 8) * sizeof(T);
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
        const char *const kp = reinterpret_cast<const char*>(static_cast<const T*>(p.k) + off), *const vp = reinterpret_cast<const char*>(static_cast<const T*>(p.v) + off);
        auto to_lds = [&](const char* from, uint8_t* to, int j) {
            __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)from,
                                             (__attribute__((address_space(3))) void*)(to + (MINE * wave + j * PER) * D * 2), 16, 0, 0);
        };
#pragma unroll
        for (int j = 0; j < LOADS; ++j) to_lds(kp + koff[j], kb, j);
        if (key >= w.kv0 && key + MINE <= w.kv1) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) to_lds(vp + voff[j], vb, j);
        } else {                                             // slots without a token of the request may hold anything
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int at = key + j * PER + lane / CH;
                to_lds(at < w.kv0 || at >= w.kv1 ? reinterpret_cast<const char*>(attention_zeros) : vp + voff[j], vb, j);
            }
        }
    };
    auto work = [&](int block, const uint8_t* kb, const uint8_t* vb) {
        const int k0 = block * KEYS;
        if (k0 >= any1 || k0 + KEYS <= any0) return;
        float16_t s[KT];
#pragma unroll
        for (int h = 0; h < KT; ++h)
#pragma unroll
            for (int j = 0; j < 16; ++j) s[h][j] = 0.f;
        // The operands are read four products ahead (2000 tokens over 30001 1858 us, 1890 without, 1930 without the order of the second product below either; 4096
        // tokens of a prompt 151, 154, 156), and of a SIMD's two wavefronts the one in its products goes before the one in its softmax (1858 us, 1860 without;
        // on heads of 256 390 and 392).
        constexpr int kAhead = 4;
        __builtin_amdgcn_s_setprio(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < KS; ++t)
#pragma unroll
            for (int h = 0; h < KT; ++h) {
                const T8 a = *reinterpret_cast<const T8*>(kb + (32 * h + col) * D * 2 + (((2 * t + hi) ^ k_swizzle<D>(col)) * 16));
                s[h] = Elem<TYPE>::mfma32(a, q[t], s[h]);
            }
        __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
        for (int i = 0; i < KS * KT; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i < KS * KT - kAhead) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        const float scale = CAP ? 1.f : p.scale2;
        if constexpr (CAP) {
#pragma unroll
            for (int h = 0; h < KT; ++h)
#pragma unroll
                for (int j = 0; j < 16; ++j) s[h][j] = capped(p, s[h][j]);
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
        // The weights are relative to a maximum that is only followed where it has grown by 2^kLag: they stay below that, exact to the same share, and the
        // sums, most of the time, need no rescaling.  (fp16 keeps more of its range for small weights: 2000 tokens over 30001 1913 us, and
        // 1911 where it lets 2^8 pass too.)
        constexpr float kLag = TYPE == RTN_TYPE_F16 ? 4.f : 8.f;
        if (__any(top > m + kLag)) {
            const float m_new = fmaxf(m, top), back = m_new == -INFINITY ? 1.f : exp2_of(m - m_new);
            m = m_new;
            l *= back;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[t][j] *= back;
        }
        const float base = (m == -INFINITY ? 0.f : m) - weight_lift<TYPE>(kLag);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int h = 0; h < KT * 2; ++h) {
            T8 pt;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = exp2_of(fmaf(s[h >> 1][8 * (h & 1) + j], scale, -base));
                l += x;
                pt[j] = (T)x;                                // (the weight of V in the element type: half an ulp of it, as much as the result's own rounding)
            }
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                union { T8 v; short4_t s[2]; } a;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int i = lane & 15, g = lane >> 4, key = 16 * h + 8 * x + 4 * (g >> 1) + (i >> 2);
                    const int piece = (4 * t + 2 * (g & 1) + ((i & 3) >> 1)) ^ (D == 64 ? (key & 2) * 2 : (key & 3) * 4);
                    a.s[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) short4_t*)(vb + key * D * 2 + piece * 16 + (i & 1) * 8));
                }
                o[t] = Elem<TYPE>::mfma32(a.v, pt, o[t]);
            }
        }
        // the first weights behind the first operands; then a product, two operand reads and a share of the other weights at a time
        constexpr int N = 2 * KT * DT, REST = (56 * KT - 28 + N - DT - 1) / (N - DT);
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * DT, 1);
        __builtin_amdgcn_sched_group_barrier(0x002, 28, 1);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
            if (i < N - DT) {
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
                __builtin_amdgcn_sched_group_barrier(0x002, REST, 1);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
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
        float* const po = partial_sums(p, p.many, head, w.slot + w.part, kTileRows, D) + (wrow + col) * D;
        float* const st = partial_stats(p, p.many, head, w.slot + w.part, kTileRows, D) + (wrow + col) * 2;
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

template <int TYPE, int D, int NQ>
__global__ __launch_bounds__(256, D == 64 && NQ == 1 ? 4 : D == 64 || (D == 128 && NQ == 1) ? 3 : 2) void attend_few_kernel(const AttnParams p) {
    __shared__ __align__(16) uint8_t lds[4][few_lds_bytes(D)];
    uint8_t* const buf[4] = {lds[0], lds[1], lds[2], lds[3]};
    attend_few<TYPE, D, NQ, 4>(p, blockIdx.x, buf, lds[__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)]);
}

// Requests of few rows and of many in one launch, so that a step of both has no more launches than one of either and its last workgroups are of both kinds.  A compute unit
// holds one workgroup at a time, of 128 elements by its registers, of 256 by LDS (134.5 KB) as well, so products run beside reading over the chip at most: three
// pieces of 300 to 900 tokens and 61 decode steps on 32 heads of 128 337 us, 189 and 186 apart; three and 21 on heads of 256 214, 156 and 65.  Heads of 256 take all 256
// registers and spill 13.  Kernels apart for tiles with a cap and without (one for both
// keeps the cap's registers where none is: 1024 tokens over 8000 on heads of 256 403 us, 392 so).
template <int TYPE, int D, bool CAP>
__global__ __launch_bounds__(512, 2) void attend_mixed_kernel(const AttnParams p) {
    constexpr int STAGE = tile_keys(D) * D * 2, FEW = few_lds_bytes(D), BYTES = STAGE > 2 * FEW ? STAGE : 2 * FEW;
    __shared__ __align__(16) uint8_t lds_k0[BYTES], lds_k1[BYTES], lds_v0[BYTES], lds_v1[BYTES];
    const int tiles = p.many.most * p.Hk;
    if ((int)blockIdx.x < tiles) {
        attend_many<TYPE, D, CAP>(p, blockIdx.x, lds_k0, lds_k1, lds_v0, lds_v1);
    } else {
        uint8_t* const buf[8] = {lds_k0, lds_k0 + FEW, lds_k1, lds_k1 + FEW, lds_v0, lds_v0 + FEW, lds_v1, lds_v1 + FEW};
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        uint8_t* const mine = (wave < 4 ? wave < 2 ? lds_k0 : lds_k1 : wave < 6 ? lds_v0 : lds_v1) + (wave & 1) * FEW;
        attend_few<TYPE, D, 1, 8>(p, blockIdx.x - tiles, buf, mine);
    }
}

template <int TYPE, int D, int ROWS>
__global__ __launch_bounds__(256) void join_few_kernel(const AttnParams p) {
    join_parts<TYPE, D, ROWS, few_keys(4), 4>(p, p.few, blockIdx.x);
}

template <int TYPE, int D>
__global__ __launch_bounds__(512) void join_mixed_kernel(const AttnParams p) {
    const int tiles = p.many.slots * p.Hk;
    if ((int)blockIdx.x < tiles) join_parts<TYPE, D, kTileRows, tile_keys(D), 8>(p, p.many, blockIdx.x);
    else join_parts<TYPE, D, 16, few_keys(8), 8>(p, p.few, blockIdx.x - tiles);
}

// The launch for a call: whether requests may have more than kFew rows, the rows of a tile of few (16 or 32), and the pieces aimed at over all KV heads.
// Few rows, 768 workgroups at a time, bound by reading: 64 ragged requests of 64 heads with 768, 1024 and 2048 pieces 236, 228, 235 us, 8 of 32k on 128
// heads 217, 204, 213, one of 4101 tokens 19.5, 19.8, 23.6 (the kernel of the time).  Beside tiles, in workgroups twice as large, half as many.  Many rows,
// 256 at a time, bound by the matrix cores, where a last round of few workgroups costs as much as a full one and parts more than whole
// tiles: three quarters of a round, since parts are rounded up (three pieces of prompts on 16 heads of 256 with 160, 192, 224 and 256 pieces
// 180, 145, 143, 190 us, beside 21 decode steps 210, 198, 201, 202; 1024 tokens over 8000 on 32 heads of 256 392 with each).
constexpr int kPieces = 1024, kMixedPieces = 512, kTilePieces = 192;

struct AttnPlan {
    bool mixed;
    int rows, few, many;                                     // pieces a KV head
    static size_t slots_bytes(int pieces, int rows, int Hk, int D) { return (size_t)2 * pieces * Hk * rows * (D + 2) * 4; }
    size_t bytes(int Hk, int D) const { return slots_bytes(few, rows, Hk, D) + slots_bytes(many, kTileRows, Hk, D); }
};

static AttnPlan plan_attention(int64_t T, int B, int Hq, int Hk, int D, int max_new) {
    const int64_t rows = std::min<int64_t>(max_new, T) * (Hq / Hk);
    AttnPlan a;
    a.mixed = rows > kFew;
    a.rows = a.mixed || rows <= 16 || D == 256 ? 16 : 32;
    a.few = a.mixed && B == 1 ? 0 : ((a.mixed ? kMixedPieces : kPieces) + Hk - 1) / Hk;
    a.many = a.mixed ? (kTilePieces + Hk - 1) / Hk : 0;
    return a;
}

template <int TYPE, int D>
static void launch_attention(const AttnParams& p, const AttnPlan& a, hipStream_t st) {
    if (a.mixed) {
        const dim3 grid((unsigned)((p.many.most + p.few.most) * p.Hk));
        if (p.cap > 0.f) hipLaunchKernelGGL((attend_mixed_kernel<TYPE, D, true>), grid, dim3(512), 0, st, p);
        else hipLaunchKernelGGL((attend_mixed_kernel<TYPE, D, false>), grid, dim3(512), 0, st, p);
        const unsigned slots = (p.many.slots + p.few.slots) * p.Hk;
        if (slots) hipLaunchKernelGGL((join_mixed_kernel<TYPE, D>), dim3(slots), dim3(512), 0, st, p);
        return;
    }
    const dim3 grid((unsigned)(p.few.most * p.Hk)), join((unsigned)(p.few.slots * p.Hk));
    if constexpr (D < 256) {
        if (a.rows == 32) {
            hipLaunchKernelGGL((attend_few_kernel<TYPE, D, 2>), grid, dim3(256), 0, st, p);
            if (p.few.slots) hipLaunchKernelGGL((join_few_kernel<TYPE, D, 32>), join, dim3(256), 0, st, p);
            return;
        }
    }
    hipLaunchKernelGGL((attend_few_kernel<TYPE, D, 1>), grid, dim3(256), 0, st, p);
    if (p.few.slots) hipLaunchKernelGGL((join_few_kernel<TYPE, D, 16>), join, dim3(256), 0, st, p);
}

}  // namespace rtn

extern "C" size_t rtn_paged_attention_workspace_nbytes(int64_t tokens, int n_requests, int q_heads, const rtn_kv_cache* cache, int max_new) {
    if (rtn::check_cache(cache) != RTN_OK || tokens < 0 || tokens > 1 << 20 || n_requests < 1 || n_requests > 65536 || q_heads < 1 ||
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
    if (tokens < 0 || tokens > 1 << 20 || n_requests < 1 || n_requests > 65536 || q_heads < 1 || q_heads % cache->kv_heads != 0 ||
        q_heads / cache->kv_heads > 64 || q_stride < (int64_t)q_heads * D || q_stride > (int64_t)1 << 36 || max_blocks < 1 ||
        max_blocks > (1 << 30) / cache->page_size || table_stride < max_blocks || max_new < 1)
        return RTN_ERR_SHAPE;
    if (!(scale > 0.f) || !(scale < INFINITY) || !(softcap >= 0.f) || !(softcap < INFINITY) || window < 0) return RTN_ERR_CONFIG;
    if (q_stride % 8 || !rtn::aligned_to(dev_q, 16) || !rtn::aligned_to(dev_out, 16) || !rtn::aligned_to(dev_workspace, 16) ||
        !rtn::aligned_to(dev_block_table, 4) || !rtn::aligned_to(dev_seq_lens, 4) || !rtn::aligned_to(dev_query_start, 4))
        return RTN_ERR_ALIGN;
    if (tokens == 0) return RTN_OK;
    if (window >= 1 << 30) window = 0;                       // (as wide as any length)
    const int Hk = cache->kv_heads, G = q_heads / Hk;
    rtn::AttnPlan a = rtn::plan_attention(tokens, n_requests, q_heads, Hk, D, max_new);
    // a smaller workspace than asked for: fewer pieces of either kind
    auto room = [&](size_t bytes, int rows) { return (int)std::min<size_t>(bytes / rtn::AttnPlan::slots_bytes(1, rows, Hk, D), 1 << 20); };
    size_t left = dev_workspace ? workspace_nbytes : 0;
    a.many = std::min(a.many, room(left, rtn::kTileRows));
    const size_t tiles_bytes = rtn::AttnPlan::slots_bytes(a.many, rtn::kTileRows, Hk, D);
    a.few = std::min(a.few, room(left - tiles_bytes, a.rows));
    // bounds on the pieces of a KV head: a request's last tile may be ragged, and each of its tiles have one part more than its share
    const int64_t rows = tokens * G;
    const int64_t few_tiles = std::min(rows / a.rows + n_requests, a.mixed ? (int64_t)n_requests * (rtn::kFew / a.rows) : rows);
    const int64_t many_tiles = a.mixed ? rows / rtn::kTileRows + std::min<int64_t>(n_requests, rows / rtn::kFew) : 0;
    auto bounds = [&](int64_t tiles, int pieces, int keys, int* most, int* slots) {
        const int64_t parts = ((int64_t)max_blocks * cache->page_size + keys - 1) / keys;     // of the longest request that the table holds
        *most = (int)std::min(tiles + pieces, tiles * parts);
        *slots = (int)std::min((int64_t)2 * pieces, tiles * parts);
    };
    // Requests of few rows of up to four steps of a workgroup are not split, and nothing is joined, where the table can hold no longer ones (one request of 250 tokens
    // 8.9 us split, 6.5 whole, of 500 8.7 and 9.1; sixteen of 500 11.6 and 11.0).
    if ((int64_t)max_blocks * cache->page_size <= 4 * 128) a.few = 0;
    int few_most, few_slots, many_most, many_slots;
    bounds(few_tiles, a.few, rtn::few_keys(a.mixed ? 8 : 4), &few_most, &few_slots);
    bounds(many_tiles, a.many, rtn::tile_keys(D), &many_most, &many_slots);
    if (!rtn::launchable(((int64_t)few_most + many_most) * Hk, a.mixed ? 512 : 256)) return RTN_ERR_SHAPE;      // (the join's launch is far smaller)
    float* const ws = static_cast<float*>(dev_workspace);
    // Factors that would pass fp32's range become its largest number: a score of zero stays zero.  (With a cap so small that its factor does, all others are at the cap either way.)
    auto finite = [](double x) { return (float)std::min(x, (double)FLT_MAX); };
    const double log2e = 1.4426950408889634;
    const float cap_in = softcap > 0.f ? finite(2.0 * scale / softcap * log2e) : 0.f;
    const rtn::AttnParams p = {dev_q, cache->dev_k, cache->dev_v, dev_out, dev_block_table, dev_seq_lens, dev_query_start, q_stride, cache->page_stride,
                               cache->head_stride, cache->token_stride, table_stride, (int)cache->pages, rtn::log2_of(cache->page_size), max_blocks,
                               n_requests, (int)tokens, q_heads, Hk, G, window, finite(scale * log2e), softcap, cap_in,
                               finite(softcap * log2e), G == 1 ? 0u : (uint32_t)(((uint64_t)1 << 32) / G) + 1, G == 1 ? 0xFFFFFFFFu : 0u, a.mixed ? rtn::kFew : 0x7FFFFFFF, {ws + tiles_bytes / 4, a.few, few_most, few_slots}, {ws, a.many, many_most, many_slots}};
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
