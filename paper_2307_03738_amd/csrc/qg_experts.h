// Products whose matrix is chosen by token: what the kernels of qg_experts_product share.
#pragma once

#include "qg_mma.h"
#include "qg_types.h"

struct QgExpertsArgs {
    const char *packed;        // blobs
    const char *x;             // rows
    const int32_t *offsets, *rows;
    void *y;
    int64_t expert_stride, x_rows, x_stride, slots;
    int64_t scales_off, zeros_off;             // of a blob's sections
    int64_t tile_codes, tile_scales, tile_zeros;      // bytes of one tile's codes, scales, zero words
    int N, K, columns;         // outputs of a matrix, inputs, columns of y (N, or N / 2)
    int group, experts, x_type, y_type, gated;
    int row_tiles;             // tiles of slots the grid has places for
};

namespace {

// Tiles of `most` slots that so many slots of so many experts can need.
static inline int64_t qg_most_tiles(int64_t slots, int experts, int most)
{
    const int64_t used = experts < slots ? experts : slots;
    return (slots + used * (most - 1)) / most;
}

// Slots of an expert, from where to where: offsets are taken into 0 ... slots whatever they are.
__device__ inline void expert_slots(const QgExpertsArgs &a, int e, int64_t &begin, int64_t &count)
{
    begin = a.offsets[e];
    int64_t end = a.offsets[e + 1];
    begin = begin < 0 ? 0 : begin > a.slots ? a.slots : begin;
    end = end < 0 ? 0 : end > a.slots ? a.slots : end;
    count = end > begin ? end - begin : 0;
}

// Sums of v over the lanes up to each, on the vector ALU: inside a row of 16 lanes, then rows' last sums to the rows behind them.
__device__ inline int sum_upto(int v)
{
    v += (int)dpp<0x111, 0xf>((uint32_t)v);
    v += (int)dpp<0x112, 0xf>((uint32_t)v);
    v += (int)dpp<0x114, 0xf>((uint32_t)v);
    v += (int)dpp<0x118, 0xf>((uint32_t)v);
    v += (int)dpp<0x142, 0xa>((uint32_t)v);
    v += (int)dpp<0x143, 0xc>((uint32_t)v);
    return v;
}

struct ExpertTile {
    int expert, rows;          // rows 0: there is no such tile
    int64_t begin;             // its first slot
};

// 64 experts' tiles of `most` slots, an expert a lane.
struct ExpertTiles {
    int e0, begin, count, mine, upto;
    __device__ inline ExpertTiles(const QgExpertsArgs &a, int first, int most) : e0(first)
    {
        const int e = first + (int)(threadIdx.x & 63);
        int64_t from = 0, slots = 0;
        if (e < a.experts) expert_slots(a, e, from, slots);
        begin = (int)from;
        count = (int)slots;
        mine = (int)((slots + most - 1) / most);
        upto = sum_upto(mine);
    }
    __device__ inline int total() const { return __builtin_amdgcn_readlane(upto, 63); }
    // tile `tile` of these, if there is one
    __device__ inline bool take(int64_t tile, int most, ExpertTile &t) const
    {
        const uint64_t past = __ballot(upto > tile);
        if (!past) return false;
        const int at = __builtin_ctzll(past);
        const int64_t skip = (tile - __builtin_amdgcn_readlane(upto - mine, at)) * most, n = __builtin_amdgcn_readlane(count, at), left = n - skip;
        t.expert = e0 + at;
        t.begin = __builtin_amdgcn_readlane(begin, at) + skip;
        t.rows = (int)(left < most ? left : most);
        if (left <= 0 || left > n) t.rows = 0;          // (offsets that decrease, whose tiles do not add up in 32 bits)
        return true;
    }
};

// Tile number `tile` of the experts' tiles, expert by expert: a wavefront adds up 64 experts' tiles at a time.
__device__ inline ExpertTile expert_tile(const QgExpertsArgs &a, int64_t tile, int most)
{
    ExpertTile t = {0, 0, 0};
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
        const ExpertTiles tiles(a, e0, most);
        if (tiles.take(tile, most, t)) break;
        tile -= tiles.total();
    }
    return t;
}

// As many as there are, row_tiles at most.
__device__ inline int expert_tiles(const QgExpertsArgs &a, int most)
{
    int64_t sum = 0;
    for (int e0 = 0; e0 < a.experts; e0 += 64) sum += ExpertTiles(a, e0, most).total();
    return sum < 0 || sum > a.row_tiles ? a.row_tiles : (int)sum;
}

// Where the weights of a lane's output lie: addresses for the whole wavefront (of the first output's tile) and the lane's distance from them.
struct OutputWeights {
    const char *codes, *scales, *zeros;
    uint32_t codes_lane, scales_lane, zeros_lane;
};
__device__ inline OutputWeights output_weights(const QgExpertsArgs &a, int expert, int64_t n)
{
    const uint32_t tile = (uint32_t)(n >> 6), first = __builtin_amdgcn_readfirstlane(tile), in_tile = (uint32_t)n & 63;
    const char *blob = a.packed + expert * a.expert_stride;
    OutputWeights w;
    w.codes = blob + first * a.tile_codes;
    w.scales = blob + a.scales_off + first * a.tile_scales;
    w.zeros = blob + a.zeros_off + first * a.tile_zeros;
    w.codes_lane = (tile - first) * (uint32_t)a.tile_codes + in_tile * 16;
    w.scales_lane = (tile - first) * (uint32_t)a.tile_scales + in_tile * 4;
    w.zeros_lane = (tile - first) * (uint32_t)a.tile_zeros + in_tile * 4;
    return w;
}

// v / (1 + e^-v) to 8 x 2^-24 of itself: with t = e^-|v| = 2^n e, e = 2^f, it is v / (1 + t) above zero and 2^n (v e / (1 + t)) below, the power of two last, so that nothing
// overflows and a result is rounded to the steps below the normal numbers once, by itself (t is such a number from v = -87 on, where v t is one from -92 on only).  n ends at
// |v| = 200, where e takes over and becomes 0.  Half as many instructions as the library's exponential and a division
// (many rows of short K: 37 to 34 us together with scans on the vector ALU).
__device__ inline float silu(float v)
{
    const float n = __builtin_rintf(__builtin_fminf(__builtin_fabsf(v), 200.0f) * -0x1.715476p0f);
    float f = __builtin_fmaf(__builtin_fabsf(v), -0x1.715476p0f, -n);              // log2 e in two parts
    f = __builtin_fmaf(__builtin_fabsf(v), -0x1.4ae0cp-26f, f);
    const float e = __builtin_amdgcn_exp2f(f), above = v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_ldexpf(e, (int)n));
    const float below = __builtin_amdgcn_ldexpf(above * e, (int)n);
    return v < 0.0f ? below : above;
}

__device__ inline void store_typed(int type, void *p, int64_t i, float v)
{
    if (type == QG_F32) store_float<QG_F32>(p, i, v);
    else if (type == QG_BF16) store_float<QG_BF16>(p, i, v);
    else store_float<QG_F16>(p, i, v);
}

}  // namespace
