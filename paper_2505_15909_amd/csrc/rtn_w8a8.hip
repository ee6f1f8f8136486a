// Products of 8-bit rows with packed 8-bit weights: C = T(sum_k q_a q_w * S_a * S_w), sums in 32-bit integers.
//
// v_mfma_i32_16x16x64_i8 takes 16 bytes a lane of each side: row (lane & 15), and the same 16 columns of 64 on both sides, in any order.  A packed
// tile is 16 rows x 64 columns and lane (row, quarter kq) owns the columns 8 kq .. and 32 + 8 kq .., codes + 128.  Two v_permlane16_swap
// bring the eights of neighbouring quarters together, so that quarters 0 .. 3 hold the sixteens 0, 2, 1, 3, which are 16 bytes in a row of
// row-major activations; four v_xor take the 128 off.
#include "rtn_paged.h"
#include "rtn_w8a8_plan.h"

namespace rtn {

typedef int int4_t __attribute__((ext_vector_type(4)));

// A packed chunk as operand: sixteen 2 (kq & 1) + (kq >> 1) of the tile's columns.
__device__ __forceinline__ int4_t weight_operand(u32x4_t c) {
    const auto a = __builtin_amdgcn_permlane16_swap(c[0], c[2], false, false), b = __builtin_amdgcn_permlane16_swap(c[1], c[3], false, false);
    const u32x4_t w = {a[0], b[0], a[1], b[1]};
    return __builtin_bit_cast(int4_t, w ^ 0x80808080u);
}

template <int TYPE>
__device__ __forceinline__ u32x2_t four_results(int4_t sum, float row_scale, half4_t s) {
    typedef typename Elem<TYPE>::x4 E4;
    typedef typename Elem<TYPE>::one E;
    E4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (E)((float)sum[e] * row_scale * (float)s[e]);
    return __builtin_bit_cast(u32x2_t, y);
}

// Workgroups on other columns read the same activations, and with K a power of two their weights start on the same memory channels.  Each begins at another place of
// its n steps along K and goes round (sums of whole numbers have no order).  16 rows of 28672 x 4096 26.0 -> 20.9 us, 64 rows 26.2 -> 22.0; 16 rows of 28672 x
// 8192 41.3 -> 37.7; where K is no power of two the same to 3 % (K = 4352: 21.5 and 22.6).  Tiles only where a round holds them all: in more,
// neighbours take turns on an L2's contents (8192 rows 2 % slower).
__device__ __forceinline__ int first_step(int column_tile, int n) { return (int)__umulhi((uint32_t)column_tile * 2654435769u, (uint32_t)n); }
__device__ __forceinline__ int around(int i, int n) { return i < n ? i : i - n; }

// The 16-byte piece of a row's 128 columns that stands at place v of eight: place kq (+ 4) is the piece that weight_operand's lane kq multiplies.  A row's places are
// stored at v ^ (row & 7), and in this order the lanes that LDS serves together are on different banks.
__device__ __forceinline__ int piece_at(int v) { return (v & 4) | (v & 1) << 1 | (v >> 1 & 1); }

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

constexpr int kBufferFlags = 0x00020000;
constexpr uint32_t kNoRow = 0x80000000u;                     // beyond every resource: reads zeros
constexpr int kStreaming = 2;                                // read once

// ---- Few rows: bound by the stream of weights.  A wavefront multiplies NT tile rows of weights by MB blocks of 16 rows, both straight
// from memory into registers, D tiles ahead; the WK wavefronts of a workgroup take the tiles of its K range in turn (what they read
// together is in one piece), and add up in LDS.  No wavefront waits for another before the end.  More tile rows to a wavefront (NT) fetch the activations less often,
// fewer make more workgroups: 8 rows of 106496 x 16384 (NT 1, 2, 4) 302, 253, 263 us, 16 rows of 28672 x 4096 27, 22, 21, one row of 4096 x 4096 5.0, 7.2, 8.
// 6.8 to 7 TB/s on the large ones; 20 us for one row of 28672 x 4096 (5.8 TB/s). ----
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
    const int begin = first_step(x, n);

    // Through resources that start at this workgroup's rows: rows past M or N read zeros, at no cost.
    const int m0 = y * (16 * MB), K = p.KT * 64, a_rows = min(16 * MB, p.M - m0), b_tiles = min(NT, p.N / 16 - x * NT);
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(p.A) + (int64_t)m0 * K, 0, (uint32_t)a_rows * (uint32_t)K, kBufferFlags);
    const __amdgpu_buffer_rsrc_t rb =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p.B) + (int64_t)x * NT * p.KT * 1024, 0, (uint32_t)b_tiles * (uint32_t)p.KT * 1024u, kBufferFlags);
    uint32_t a_at[MB], b_at[NT];
#pragma unroll
    for (int i = 0; i < MB; ++i)
        a_at[i] = 16 * i + nl < a_rows ? (uint32_t)(16 * i + nl) * (uint32_t)K + piece_at(kq) * 16 : kNoRow;
#pragma unroll
    for (int j = 0; j < NT; ++j) b_at[j] = j < b_tiles ? (uint32_t)j * (uint32_t)p.KT * 1024u + lane * 16 : kNoRow;

    int4_t acc[MB][NT];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = (int4_t){0, 0, 0, 0};
    int4_t a[D][MB];
    u32x4_t w[D][NT];
    auto load = [&](int s, int i) {
        const int t = t0 + wave + WK * around(begin + min(i, n - 1), n);
#pragma unroll
        for (int j = 0; j < NT; ++j) w[s][j] = __builtin_amdgcn_raw_buffer_load_b128(rb, b_at[j], t * 1024, kStreaming);
#pragma unroll
        for (int k = 0; k < MB; ++k) a[s][k] = __builtin_bit_cast(int4_t, __builtin_amdgcn_raw_buffer_load_b128(ra, a_at[k], t * 64, 0));
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
        else *reinterpret_cast<u32x2_t*>(static_cast<half_t*>(p.C) + at) = four_results<TYPE>(s, p.a_scales[m], *reinterpret_cast<const half4_t*>(p.scales + c));
    }
}

// ---- Many rows: bound by the matrix cores, at the clock that the power allows.  A workgroup of 8 wavefronts (2 along M x 4 along N) computes
// 32 MBW rows x 256 columns of C, a wavefront 16 MBW x 64 of them.  K advances by 128 columns a step: 128 bytes of a row are eight 16-byte pieces in
// LDS (piece_at); packed tiles lie as they are, a lane reads its own chunk.  Both come
// straight into LDS, SA and SB steps ahead.  A step runs in phases of two row blocks and both halves of its columns; a phase reads the next one's operands, and
// the one barrier of a step stands before its last phase, whose operands are in registers by then: the stage is free behind it, and the
// requests for it go out over the phases that follow.  8192 rows of 28672 x 4096 700 to 785 us on different cards (2.45 to 2.75 PFLOP/s), 8192 x 8192 x 8192 373
// to 399 (2.95), where the vendor library's int8 product takes 988 and 445; matrix cores 69 % busy at 1.65 GHz.  Turning weights into operands
// costs 6 % of that.  A round of tiles begins and ends for 5 us (K = 4096: 10 %): workgroups that stay and request the next tile's first steps under the last
// one's end have registers for two stages of weights only, and lose more on every step than they gain (749 -> 791; K = 512 170 -> 161). ----
constexpr int kTileThreads = 512, kZGroup = 4;

// 16 bytes per lane from global memory into 1 KiB of LDS at a wave-uniform address
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, uint8_t* lds, uint32_t lane_off, int off) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 16, lane_off, off, 0, 0);
}

// Workgroup barrier behind the loads older than the N newest ones and every LDS access.
template <int N>
__device__ __forceinline__ void wait_and_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

template <int TYPE, int MBW>
__global__ __launch_bounds__(kTileThreads, 2) void w8a8_tile_kernel(const W8A8Params p) {
    constexpr int TM = 32 * MBW, A_BYTES = TM * 128, B_BYTES = kTileN * 128;
    constexpr int PH = MBW / 2;                              // phases of a step
    constexpr int SA = MBW == 4 ? 3 : 2, SB = 3;             // stages: 144 or 160 KiB
    constexpr int AP = 2, BP = PH == 4 ? 2 : 0;              // the activations' requests go out in AP phases from the barrier on, the weights' from phase BP on
    constexpr int NA = TM / 64, NB = kTileN / 64;            // requests of a wavefront and step, 1 KiB each
    constexpr int U = 6;                                     // steps a turn of the loop: every stage index is a literal
    __shared__ __align__(16) uint8_t lds_a0[A_BYTES], lds_a1[A_BYTES], lds_a2[SA > 2 ? A_BYTES : 16];
    __shared__ __align__(16) uint8_t lds_b0[B_BYTES], lds_b1[B_BYTES], lds_b2[B_BYTES];
    auto stage_a = [&](int i) { return i == 0 ? lds_a0 : i == 1 ? lds_a1 : lds_a2; };
    auto stage_b = [&](int i) { return i == 0 ? lds_b0 : i == 1 ? lds_b1 : lds_b2; };

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 2, wn = wave & 3, nl = lane & 15, kq = lane >> 4;
    const int blocks = (p.XB * p.YB + kXcds - 1) / kXcds * kXcds, z = blockIdx.x / blocks;
    int xb, yb;
    if (!xcd_tile((int)blockIdx.x - z * blocks, p.XB, p.YB, kZGroup, &xb, &yb)) return;
    const int m0 = yb * TM, n0 = xb * kTileN, K = p.KT * 64;
    const int pairs = p.KT / 4;                              // (two steps each: a workgroup has an even number of them)
    const int s0 = 2 * (int)((int64_t)pairs * z / p.split), T = 2 * (int)((int64_t)pairs * (z + 1) / p.split) - s0;
    const int begin = p.XB * p.YB * p.split <= 256 ? first_step(xb, T) : 0;

    // Both operands through resources that start at this workgroup's first row; rows past M or N read zeros, steps past the last one the last.
    const int a_rows = min(TM, p.M - m0), b_tiles = min(kTileN, p.N - n0) / 16;
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(p.A) + (int64_t)m0 * K, 0, (uint32_t)a_rows * (uint32_t)K, kBufferFlags);
    const __amdgpu_buffer_rsrc_t rb =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p.B) + (int64_t)(n0 / 16) * p.KT * 1024, 0, (uint32_t)b_tiles * (uint32_t)p.KT * 1024u, kBufferFlags);
    uint32_t a_lane[NA], b_lane[NB / 2];
    const int st_row = lane >> 3, st_piece = piece_at((lane & 7) ^ (lane >> 3));
#pragma unroll
    for (int i = 0; i < NA; ++i) {
        const int row = (wave * NA + i) * 8 + st_row;
        a_lane[i] = row < a_rows ? (uint32_t)row * (uint32_t)K + st_piece * 16 : kNoRow;
    }
#pragma unroll
    for (int i = 0; i < NB / 2; ++i) {
        const int row = wave * (NB / 2) + i;
        b_lane[i] = row < b_tiles ? (uint32_t)row * (uint32_t)p.KT * 1024u + lane * 16 : kNoRow;
    }
    auto a_dma = [&](int stage, int t, int i) { load_to_lds(ra, stage_a(stage) + (wave * NA + i) * 1024, a_lane[i], (s0 + around(begin + min(t, T - 1), T)) * 128); };
    auto b_dma = [&](int stage, int t, int i) {
        load_to_lds(rb, stage_b(stage) + (wave * NB + i) * 1024, b_lane[i >> 1], (s0 + around(begin + min(t, T - 1), T)) * 2048 + (i & 1) * 1024);
    };

    int4_t acc[MBW][4];
#pragma unroll
    for (int b = 0; b < MBW; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[b][r] = (int4_t){0, 0, 0, 0};
    const uint32_t a_rd = (uint32_t)((wm * (TM / 2) + nl) * 128), b_rd = (uint32_t)(wn * 8192 + lane * 16);
    const uint32_t po0 = (uint32_t)((kq ^ (nl & 7)) * 16), po1 = (uint32_t)(((4 + kq) ^ (nl & 7)) * 16);
    int4_t aop[2][2][2];                                     // of two phases, row block, half
    int4_t bop[2][4];                                        // half, tile row
    u32x4_t raw[2][4];
    auto read_a = [&](int u, int ph, int b) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            aop[ph & 1][b][i] = *reinterpret_cast<const int4_t*>(stage_a(u % SA) + a_rd + (ph * 2 + b) * 2048 + (i ? po1 : po0));
    };
    auto read_b = [&](int u, int r) {
#pragma unroll
        for (int i = 0; i < 2; ++i) raw[i][r] = *reinterpret_cast<const u32x4_t*>(stage_b(u % SB) + b_rd + r * 2048 + i * 1024);
    };

    auto step = [&](int u, int t) {
#pragma unroll
        for (int ph = 0; ph < PH; ++ph) {
            if (ph == PH - 1) {
                wait_and_barrier<(SA - 2) * NA + (SB - 2) * NB>();           // the next step's tiles have landed
                __builtin_amdgcn_sched_barrier(0);
            }
            auto mfma = [&](int b, int r) {
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[ph * 2 + b][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bop[i][r], aop[ph & 1][b][i], acc[ph * 2 + b][r], 0, 0, 0);
            };
            for (int b = 0; b < 2; ++b) read_a(ph == PH - 1 ? u + 1 : u, ph == PH - 1 ? 0 : ph + 1, b);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (ph == 0) {
                    bop[0][r] = weight_operand(raw[0][r]);
                    bop[1][r] = weight_operand(raw[1][r]);
                }
                mfma(r & 1, r);
                mfma(~r & 1, r);
                if (ph == PH - 1) read_b(u + 1, r);
            }
            const int pa = (ph + 1) % PH;                     // phases since the barrier
            int vm = 0;
            const int fu = pa == 0 ? u : u + U - 1, ft = pa == 0 ? t : t - 1;    // the step whose stage that barrier freed
            if (pa < AP) {
#pragma unroll
                for (int k = pa * NA / AP; k < (pa + 1) * NA / AP; ++k) a_dma(fu % SA, ft + SA, k);
                vm += NA / AP;
                __builtin_amdgcn_sched_barrier(0x78F);       // everything but memory loads may cross: the counted waits rely on their order
            }
            if (BP == 0 ? pa == 0 : pa >= BP) {
                constexpr int EACH = BP == 0 ? NB : NB / (PH - BP);
#pragma unroll
                for (int k = (pa - BP) * EACH; k < (pa - BP + 1) * EACH; ++k) b_dma(fu % SB, ft + SB, k);
                vm += EACH;
            }
            if (ph == 0) __builtin_amdgcn_sched_group_barrier(0x002, 12, 0);
#pragma unroll
            for (int g = 0; g < 8; ++g) {
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                if (ph == PH - 1) {
                    if (g < 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                    if (g & 1) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                } else if (g < 4) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                if (ph == 0 && g < 6) __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);
                if (g < vm) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // the requests of the steps before the first one, in the order of the loop (its waits are counts)
#pragma unroll
    for (int k = 0; k < (SB > SA ? NB : 0); ++k) b_dma(0, 0, k);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int v = 0; v < SA; ++v) {
#pragma unroll
        for (int k = 0; k < (v == SA - 1 ? NA / AP : NA); ++k) a_dma(v, v, k);       // (the rest, in the first step)
        __builtin_amdgcn_sched_barrier(0);
        if (v < SA - 1 || BP == 0)
#pragma unroll
            for (int k = 0; k < NB; ++k) b_dma(v + SB - SA, v + SB - SA, k);
        __builtin_amdgcn_sched_barrier(0);
    }
    wait_and_barrier<(SA - 2) * NA + NA / AP + (SB - (BP == 0 ? 1 : 2)) * NB>();
    for (int b = 0; b < 2; ++b) read_a(0, 0, b);
#pragma unroll
    for (int r = 0; r < 4; ++r) read_b(0, r);
    __builtin_amdgcn_sched_barrier(0);

    for (int t = 0;; t += U) {            // T is even; leaving between two steps keeps every wait inside an exact count
        bool done = false;
#pragma unroll
        for (int u = 0; u < U; u += 2) {
            step(u, t + u);
            step(u + 1, t + u + 1);
            if (t + u + 2 >= T) {
                done = true;
                break;
            }
        }
        if (done) break;
    }
    wait_and_barrier<0>();                // no load into LDS outlives the workgroup

    // a lane holds row 16 b + nl and the four columns 16 r + 4 kq + e
    if (p.split > 1) {
#pragma unroll
        for (int b = 0; b < MBW; ++b) {
            const int m = m0 + wm * (TM / 2) + b * 16 + nl;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int n = n0 + wn * 64 + r * 16 + kq * 4;
                if (m < p.M && n < p.N) *reinterpret_cast<int4_t*>(p.ws + ((int64_t)z * p.M + m) * p.N + n) = acc[b][r];
            }
        }
        return;
    }
    // results change lanes through the wavefront's own part of LDS, 16 rows x 128 bytes at a time, so that a store writes whole 128-byte runs
    half4_t scale[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) scale[r] = *reinterpret_cast<const half4_t*>(p.scales + min(n0 + wn * 64 + r * 16, p.N - 16) + kq * 4);
    uint8_t* const mine = lds_b0 + wave * 2048;
#pragma unroll
    for (int b = 0; b < MBW; ++b) {
        const float row_scale = p.a_scales[min(m0 + wm * (TM / 2) + b * 16 + nl, p.M - 1)];
#pragma unroll
        for (int r = 0; r < 4; ++r)
            *reinterpret_cast<u32x2_t*>(mine + nl * 128 + (((r * 2 + (kq >> 1)) ^ (nl & 7)) * 16) + (kq & 1) * 8) = four_results<TYPE>(acc[b][r], row_scale, scale[r]);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = h * 8 + (lane >> 3), piece = lane & 7;
            const u32x4_t v = *reinterpret_cast<const u32x4_t*>(mine + row * 128 + ((piece ^ (row & 7)) * 16));
            const int m = m0 + wm * (TM / 2) + b * 16 + row, n = n0 + wn * 64 + piece * 8;
            if (m < p.M && n < p.N) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(static_cast<half_t*>(p.C) + (int64_t)m * p.N + n));
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- Rows between: bound by the stream of weights where enough of them is on its way.  The eight wavefronts of a workgroup stand 8 / WK along N and WK along K.
// A wavefront has NT tile rows of weights, straight into registers; the activations, 16 MB rows, come into LDS once for the wavefronts along N.
// A step is 128 columns for each wavefront along K; both are requested two steps ahead, and one barrier a step says that its activations have landed
// and the last one's are used up.  The waits before it count loads, so what they leave on its way is always one whole request, which a barrier to the
// scheduler closes; the last steps request nothing, since of what nobody multiplies the compiler keeps the loads into LDS alone.  The wavefronts along K add up in LDS at the end, so that a small matrix fills the chip without a join: 217 rows of 4096 x 4096 10.6 us
// (two along K, 256 workgroups; one 16.1, tiles 20.7), 128 rows 8.3 (four; out of the last-level cache, from memory 10.4).  64 rows of 28672 x 4096 22.5 us (5.4 TB/s), 128 rows 30.  ONCE: the weights are marked as read once -- one row tile, or more weights
// than the L2s hold: 64 rows of 8192 x 28672 43.9 us, 46.8 unmarked; marked where two row tiles share them, 128 rows of 4096 x 4096 take 9.6 for 8.3,
// 160 of 5120 x 5120 14.0 for 12.0. ----
template <int TYPE, int MB, int NT, int WK, bool ONCE>
__global__ __launch_bounds__(512, MB * NT <= 8 && MB * WK <= 8 ? 4 : 2) void w8a8_block_kernel(const W8A8Params p) {
    constexpr int WN = 8 / WK, NA = MB * WK / 4, EACH = NA + 2 * NT;         // requests of a wavefront and step: of activations, in all
    constexpr int A_BYTES = MB * WK * 2048;
    static_assert(MB * NT * 8192 * (WK - 1) / WK <= 2 * A_BYTES, "sums of the wavefronts along K");
    __shared__ __align__(16) uint8_t lds0[A_BYTES], lds1[A_BYTES], lds2[A_BYTES];
    auto stage = [&](int i) { return i == 0 ? lds0 : i == 1 ? lds1 : lds2; };
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), nl = lane & 15, kq = lane >> 4;
    const int wn = wave % WN, wk = wave / WN;
    const int blocks = (p.XB * p.YB + kXcds - 1) / kXcds * kXcds, z = blockIdx.x / blocks;
    int xb, yb;
    if (!xcd_tile((int)blockIdx.x - z * blocks, p.XB, p.YB, kZGroup, &xb, &yb)) return;
    const int m0 = yb * (16 * MB), K = p.KT * 64, tile0 = (xb * WN + wn) * NT;
    const int s0 = (int)((int64_t)(p.KT / 2) * z / p.split), units = (int)((int64_t)(p.KT / 2) * (z + 1) / p.split) - s0;      // of 128 columns
    const int T = (units + WK - 1) / WK, begin = first_step(xb, units);

    const int a_rows = min(16 * MB, p.M - m0), b_tiles = __builtin_amdgcn_readfirstlane(max(0, min(NT, p.N / 16 - tile0)));      // (none: a wavefront beyond N)
    const int first = __builtin_amdgcn_readfirstlane(min(tile0, p.N / 16 - 1));
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(p.A) + (int64_t)m0 * K, 0, (uint32_t)a_rows * (uint32_t)K, kBufferFlags);
    const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p.B) + (int64_t)first * p.KT * 1024, 0,
                                                                        (uint32_t)b_tiles * (uint32_t)p.KT * 1024u, kBufferFlags);
    uint32_t a_lane[NA], b_lane[NT];
    int a_unit[NA];                                          // request i of the wavefront: eight rows of the activations of wavefronts a_unit along K
#pragma unroll
    for (int i = 0; i < NA; ++i) {
        const int r = wave * NA + i, row = r % (2 * MB) * 8 + (lane >> 3);
        a_unit[i] = r / (2 * MB);
        a_lane[i] = row < a_rows ? (uint32_t)row * (uint32_t)K + piece_at((lane & 7) ^ (lane >> 3)) * 16 : kNoRow;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) b_lane[j] = j < b_tiles ? (uint32_t)j * (uint32_t)p.KT * 1024u + lane * 16 : kNoRow;

    u32x4_t w[3][NT][2];
    auto request = [&](int u, int t) {                       // step t, into stage and registers u; units past the last one: the last, not multiplied
#pragma unroll
        for (int i = 0; i < NA; ++i) load_to_lds(ra, stage(u) + (wave * NA + i) * 1024, a_lane[i], (s0 + around(begin + min(t * WK + a_unit[i], units - 1), units)) * 128);
        const int at = s0 + around(begin + min(t * WK + wk, units - 1), units);
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) w[u][j][h] = __builtin_amdgcn_raw_buffer_load_b128(rb, b_lane[j], at * 2048 + h * 1024, ONCE ? kStreaming : 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    int4_t acc[MB][NT];
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[b][j] = (int4_t){0, 0, 0, 0};
    const uint32_t a_rd = (uint32_t)(wk * MB * 2048 + nl * 128), po[2] = {(uint32_t)((kq ^ (nl & 7)) * 16), (uint32_t)(((4 + kq) ^ (nl & 7)) * 16)};
    auto multiply = [&](int u, int t) {
        if (WK > 1 && t * WK + wk >= units) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int4_t wj[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) wj[j] = weight_operand(w[u][j][h]);
#pragma unroll
            for (int b = 0; b < MB; ++b) {
                const int4_t a = *reinterpret_cast<const int4_t*>(stage(u) + a_rd + b * 2048 + po[h]);
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[b][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wj[j], a, acc[b][j], 0, 0, 0);
            }
        }
    };
    auto landed_but_one = [&]() {                            // all requests have, but for the newest
        __builtin_amdgcn_sched_barrier(0);
        wait_and_barrier<EACH>();
        __builtin_amdgcn_sched_barrier(0);
    };
    request(0, 0);
    request(1, 1);
    // whole turns, then what is left: an exit within a turn would be, to the compiler's counts of loads, one more way into the next
    int t = 0;
    for (; t + 3 <= T; t += 3) {
#pragma unroll
        for (int u = 0; u < 3; ++u) {
            landed_but_one();
            request((u + 2) % 3, t + u + 2);
            multiply(u, t + u);
        }
    }
    if (t < T) {                          // two requests are on their way, used or not
        landed_but_one();
        multiply(0, t);
    }
    if (T - t == 2) {
        wait_and_barrier<0>();
        multiply(1, t + 1);
    }
    wait_and_barrier<0>();                // no load into LDS outlives the workgroup

    if constexpr (WK > 1) {
        // half of the row blocks in one stage, half in the other; the first wavefront along K adds the others' sums to its own
        auto place = [&](int k, int b, int j) {
            uint8_t* const half = b < MB / 2 ? lds0 : lds1;
            return reinterpret_cast<int4_t*>(half + ((((k - 1) * WN + wn) * (MB / 2) + b % (MB / 2)) * NT + j) * 1024 + lane * 16);
        };
        if (wk > 0) {
#pragma unroll
            for (int b = 0; b < MB; ++b)
#pragma unroll
                for (int j = 0; j < NT; ++j) *place(wk, b, j) = acc[b][j];
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int k = 1; k < WK; ++k)
#pragma unroll
            for (int b = 0; b < MB; ++b)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[b][j] += *place(k, b, j);
    }
    // a lane holds row 16 b + nl and the four columns 16 j + 4 kq + e
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n = (tile0 + j) * 16 + kq * 4;
        if (n >= p.N) continue;
        const half4_t scale = *reinterpret_cast<const half4_t*>(p.scales + n);
#pragma unroll
        for (int b = 0; b < MB; ++b) {
            const int m = m0 + b * 16 + nl;
            if (m >= p.M) continue;
            if (p.split > 1) *reinterpret_cast<int4_t*>(p.ws + ((int64_t)z * p.M + m) * p.N + n) = acc[b][j];
            else *reinterpret_cast<u32x2_t*>(static_cast<half_t*>(p.C) + (int64_t)m * p.N + n) = four_results<TYPE>(acc[b][j], p.a_scales[m], scale);
        }
    }
}

// Sums of the K splits' parts, four columns a thread.
template <int TYPE>
__global__ __launch_bounds__(256) void w8a8_join_kernel(const W8A8Params p) {
    const int64_t all = (int64_t)p.M * p.N, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= all) return;
    int4_t part[kMostSplits];                                // all requested before the first is added
#pragma unroll
    for (int z = 0; z < kMostSplits; ++z) part[z] = z < p.split ? *reinterpret_cast<const int4_t*>(p.ws + z * all + at) : (int4_t){0, 0, 0, 0};
    const int m = (int)(at / p.N), c = (int)(at - (int64_t)m * p.N);
    const float row_scale = p.a_scales[m];
    const half4_t scale = *reinterpret_cast<const half4_t*>(p.scales + c);
    int4_t s = part[0];
#pragma unroll
    for (int z = 1; z < kMostSplits; ++z) s += part[z];
    *reinterpret_cast<u32x2_t*>(static_cast<half_t*>(p.C) + at) = four_results<TYPE>(s, row_scale, scale);
}

static rtn_status check_w8a8(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || M > 1 << 20 || N < 16 || N > 1 << 30 || N % 16 || K < 256 || K % 256 || K >= 1 << 17 || N * K >= 0x7FFF0000ll) return RTN_ERR_SHAPE;
    return RTN_OK;
}

template <int TYPE, int I>
static void launch_shape(const W8A8Params& p, dim3 grid, hipStream_t st) {
    constexpr W8A8Shape k = kShapes[I];
    if constexpr (k.kind == W8A8_STREAM) hipLaunchKernelGGL((w8a8_stream_kernel<TYPE, k.mb, k.nt, k.wk, k.depth>), grid, dim3(k.wk * 64), 0, st, p);
    else if constexpr (k.kind == W8A8_BLOCK) {
        // (128 rows x 256 columns are not chosen where row tiles share near weights)
        constexpr bool near_too = k.mb * k.nt / k.wk < 16;
        if (!near_too || p.YB == 1 || !weights_near(p.N, (int64_t)p.KT * 64)) hipLaunchKernelGGL((w8a8_block_kernel<TYPE, k.mb, k.nt, k.wk, true>), grid, dim3(512), 0, st, p);
        else if constexpr (near_too) hipLaunchKernelGGL((w8a8_block_kernel<TYPE, k.mb, k.nt, k.wk, false>), grid, dim3(512), 0, st, p);
    }
    else hipLaunchKernelGGL((w8a8_tile_kernel<TYPE, k.mb>), grid, dim3(kTileThreads), 0, st, p);
}

template <int TYPE, int... I>
static void launch_one_of(std::integer_sequence<int, I...>, int shape, const W8A8Params& p, dim3 grid, hipStream_t st) {
    (void)((shape == I && (launch_shape<TYPE, I>(p, grid, st), true)) || ...);
}

template <int TYPE>
static hipError_t launch_w8a8(const W8A8Params& p, const W8A8Plan& plan, hipStream_t st) {
    launch_one_of<TYPE>(std::make_integer_sequence<int, kShapeCount>(), plan.shape, p, dim3((unsigned)plan.workgroups()), st);
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
    if (!rtn::launchable(plan.workgroups(), plan.threads()) || (plan.split > 1 && !rtn::launchable((M * N / 4 + 255) / 256, 256)))
        return RTN_ERR_SHAPE;
    const rtn::W8A8Params p = {static_cast<const int8_t*>(dev_q), dev_q_scales, static_cast<const uint8_t*>(dev_qweight), static_cast<const rtn::half_t*>(dev_scales),
                               dev_C, static_cast<int*>(dev_workspace), (int)M, (int)N, (int)(K / 64), (int)plan.XB, (int)plan.YB, plan.split};
    hipStream_t s = static_cast<hipStream_t>(stream);
    return (dtype == RTN_TYPE_F16 ? rtn::launch_w8a8<RTN_TYPE_F16>(p, plan, s) : rtn::launch_w8a8<RTN_TYPE_BF16>(p, plan, s)) == hipSuccess ? RTN_OK : RTN_ERR_HIP;
}
