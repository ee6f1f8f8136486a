// Which kernel a product of 8-bit rows takes, and with how many workgroups along K.  Host code only: the kernels are in rtn_w8a8.hip.
#pragma once
#include <algorithm>
#include <array>
#include <cmath>
#include <stdint.h>
#include <utility>

#include "rtn_device.h"

namespace rtn {

constexpr int kTileN = 256, kMostSplits = 8;                 // columns of a tile kernel's workgroup; parts that the join adds

constexpr size_t kW8A8Workspace = (size_t)64 << 20;

// The kernels' shapes and what their time is made of, in us.  Stream and block kernels: start + units x (workgroups on the fullest compute unit) x
// (each + more x the share of a workgroup's rows that M has), a unit being the 64 (128) columns of a step of each wavefront along K: a compute unit
// has some 32 KiB on their way at once, 50 to 65 GB/s where they come from beyond its L2, whatever the workgroups on it; and a block kernel's next round.  Tile kernels: rounds of one
// workgroup a compute unit, whose step takes `each` where half the chip is busy and `each + more` where all of it is (power).  That against the weights' stream,
// and a K split's join.  `depth`: a stream kernel's tiles on their way, the workgroups of a block kernel that a compute unit holds.
// The constants are chosen for their picks, by tuning/w8a8_fit.py: the modelled times are 12 to 22 % off (rms).  2910 problems (1 to 8192 rows, 128 to 106496 columns, K 512 to 53248; tuning/w8a8_sweep.hip,
// every shape with every split up to 8): the pick is 1.4 % behind the fastest launch on the mean, 5 to 12 % in one problem of twenty (most at 41 to 128 rows), 26 % at most (384 rows of 6144 x 4096); on
// another card, problems that no constant was fitted to: 684 of the same ranges 1.8 % and 25 % (115 rows of 144 x 512), 100 of 512 to 8192 rows on matrices of layers within the L2s 0.8 % and 16 %.
enum { W8A8_STREAM, W8A8_BLOCK, W8A8_TILE };
struct W8A8Shape {
    int kind, mb, nt, wk, depth;
    float start, each, more;
};
constexpr W8A8Shape kShapes[] = {
    {W8A8_STREAM, 1, 1, 16, 4, 3.424f, 0.326f, 0.358f}, {W8A8_STREAM, 1, 1, 8, 4, 2.141f, 0.18f, 0.198f},   {W8A8_STREAM, 1, 1, 8, 2, 1.727f, 0.375f, 0.004f},
    {W8A8_STREAM, 1, 2, 8, 2, 1.813f, 0.367f, 0.181f},  {W8A8_STREAM, 1, 4, 8, 2, 2.39f, 0.694f, 0.138f},   {W8A8_STREAM, 2, 2, 8, 2, 2.788f, 0.355f, 0.24f},
    {W8A8_BLOCK, 2, 1, 4, 3, 2.703f, 0.426f, 0.012f},   {W8A8_BLOCK, 2, 2, 4, 2, 3.154f, 0.727f, 0.001f},   {W8A8_BLOCK, 2, 2, 2, 2, 3.662f, 0.71f, 0.001f},
    {W8A8_BLOCK, 4, 1, 4, 1, 2.563f, 0.423f, 0.433f},   {W8A8_BLOCK, 4, 1, 2, 3, 2.87f, 0.431f, 0.097f},    {W8A8_BLOCK, 4, 1, 1, 4, 2.937f, 0.434f, 0.008f},
    {W8A8_BLOCK, 4, 2, 2, 2, 5.822f, 0.686f, 0.063f},   {W8A8_BLOCK, 4, 2, 1, 2, 6.576f, 0.585f, 0.001f},   {W8A8_BLOCK, 8, 2, 2, 1, 8.65f, 0.582f, 0.501f},
    {W8A8_BLOCK, 8, 2, 1, 1, 11.428f, 0.476f, 0.326f},  {W8A8_TILE, 4, 0, 0, 0, 5.71f, 0.715f, 0.036f},     {W8A8_TILE, 8, 0, 0, 0, 7.557f, 0.942f, 0.109f}};
// What a round of tiles and a further round of a block kernel's workgroups take beyond their steps, a join's launch and wait (us), and bytes a us.
constexpr float kTileRound = 10.591f, kBlockRound = 3.301f;
constexpr float kJoin = 2.585f, kJoinTile = 6.106f;
constexpr float kStreamRate = 10.901e6f, kOutRate = 16.215e6f, kJoinRate = 5.442e6f;
// Where row tiles share weights, times: in the stream kernels, whose wavefronts share nothing; in the block kernels, out of the L2s (32 MiB) and beyond.
// A tile kernel's one row tile, which has the weights to itself, the last.
constexpr float kSharedStream = 1.322f, kSharedNear = 0.998f, kSharedFar = 1.102f, kTileAlone = 1.256f;
// Block kernels for more than 128 rows only where tiles of 128 x 256 would leave half of the 256 compute units idle.  The faster of all block launches against the faster of all
// tile launches: up to 64 such tiles block kernels win 92 problems of 100, 1.6 times as fast on the mean of all; 65 to 128 tiles 68, 1.08 times; more 8, and take 1.21 times as long
// (6144 x 4096, 3000 rows: 92 us, the fastest block launch 92, the one that the model of block kernels alone preferred 119; 8192 rows 163 and 226).
constexpr int kMostTiles = 128;
constexpr int kShapeCount = sizeof(kShapes) / sizeof(kShapes[0]);

struct W8A8Plan {
    int shape, split;
    int64_t XB, YB;
    int threads() const { return kShapes[shape].kind == W8A8_STREAM ? kShapes[shape].wk * 64 : 512; }
    int64_t workgroups() const { return (kShapes[shape].kind == W8A8_STREAM ? XB * YB : (XB * YB + kXcds - 1) / kXcds * kXcds) * split; }
};

constexpr int log2_const(int n) { return n > 1 ? 1 + log2_const(n / 2) : 0; }

// What a shape covers, as powers of two: a workgroup's rows and columns, a unit's columns of K, wavefronts along K.
struct W8A8Cover { int rows, columns, unit, along; };
constexpr W8A8Cover cover_of(const W8A8Shape& k) {
    return k.kind == W8A8_TILE ? W8A8Cover{log2_const(32 * k.mb), log2_const(kTileN), 8, 0}
                               : W8A8Cover{log2_const(16 * k.mb), log2_const(k.kind == W8A8_BLOCK ? 128 * k.nt / k.wk : 16 * k.nt), k.kind == W8A8_BLOCK ? 7 : 6, log2_const(k.wk)};
}
template <int... I>
constexpr std::array<W8A8Cover, sizeof...(I)> covers(std::integer_sequence<int, I...>) { return {cover_of(kShapes[I])...}; }
constexpr auto kCovers = covers(std::make_integer_sequence<int, kShapeCount>());

// Weights that the L2s hold together: row tiles that share them find them there.
inline bool weights_near(int64_t N, int64_t K) { return N * K <= (int64_t)32 << 20; }

inline W8A8Plan w8a8_plan(int64_t M, int64_t N, int64_t K, size_t workspace) {
    W8A8Plan plan = {};
    float best = 1e30f;
    const float MN = (float)M * (float)N, outputs = 2.f * MN, stream = ((float)N + (float)M) * (float)K * (1.f / kStreamRate);
    const float s4 = stream * stream * stream * stream;
    const int splits = (int)std::min<uint64_t>(kMostSplits, std::min(workspace, kW8A8Workspace) / 4 / (uint64_t)(M * N));
    const int pieces = (int)((M + 15) / 16);
    const bool near = weights_near(N, K);
    auto up = [](int64_t n, int log2) { return (n + ((int64_t)1 << log2) - 1) >> log2; };
    for (int i = 0; i < kShapeCount; ++i) {
        const W8A8Shape& k = kShapes[i];
        const W8A8Cover& c = kCovers[i];
        if ((1 << c.rows) >= 32 * pieces && c.rows > 5) continue;            // mostly rows beyond M
        const int64_t XB = up(N, c.columns), YB = up(M, c.rows), tiles = XB * YB, all_units = K >> c.unit;
        if (k.kind == W8A8_STREAM && YB > 8) continue;
        if (k.kind == W8A8_BLOCK && M > 128 && up(M, 7) * up(N, 8) > kMostTiles) continue;
        const float shared = YB == 1 ? 1.f : k.kind == W8A8_STREAM ? kSharedStream : near ? kSharedNear : kSharedFar;
        const float unit_us = (k.each + k.more * (float)M / (float)(YB << c.rows)) * shared;
        const float once = k.start + (k.kind == W8A8_TILE ? 0.f : outputs * (1.f / kOutRate));
        for (int split = 1; split <= std::max(1, splits); ++split) {
            if (split > 1 && ((split << c.along) > all_units || tiles * split > 800)) break;
            const float steps = (float)up((uint32_t)(all_units + split - 1) / (uint32_t)split, c.along);
            float work;
            if (k.kind == W8A8_TILE) {
                const int64_t on_xcd = up(tiles, 3) * split;
                const float part = (float)(on_xcd & 31) * (1.f / 32.f);
                work = (float)(on_xcd >> 5) * (2.f * steps * (k.each + k.more) + kTileRound) - kTileRound;
                if (part > 0.f) work += 2.f * steps * (k.each + k.more * std::max(0.f, 2.f * part - 1.f)) + kTileRound;
                if (YB == 1) work *= kTileAlone;
            } else {
                const int64_t on_unit = k.kind == W8A8_STREAM ? up(tiles * split, 8) : up(up(tiles, 3) * split, 5);
                work = steps * unit_us * (float)on_unit;
                if (k.kind == W8A8_BLOCK) work += kBlockRound * (float)((uint32_t)(on_unit - 1) / (uint32_t)k.depth);
            }
            const float rest = once + (split > 1 ? (k.kind == W8A8_TILE ? kJoinTile : kJoin) + (outputs + 4.f * outputs * (float)split) * (1.f / kJoinRate) : 0.f);
            if (rest + std::max(work, stream) >= best) {
                if (rest + stream >= best || work < 0.6f * stream) break;    // (more splits only add to the rest)
                continue;
            }
            const float t = rest + std::sqrt(std::sqrt(work * work * work * work + s4));
            if (t < best) {
                best = t;
                plan = {i, split, XB, YB};
            }
            if (work < 0.6f * stream) break;
        }
    }
    return plan;
}

}  // namespace rtn
