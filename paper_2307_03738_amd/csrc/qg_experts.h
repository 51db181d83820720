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

// Tiles of `most` slots that the experts have, row_tiles at most.
__device__ inline int expert_tiles(const QgExpertsArgs &a, int most)
{
    int64_t tiles = 0;
    for (int e = threadIdx.x & 63; e < a.experts; e += 64) {
        int64_t begin, count;
        expert_slots(a, e, begin, count);
        tiles += (count + most - 1) / most;
    }
    int sum = (int)(tiles < a.row_tiles ? tiles : a.row_tiles);
#pragma unroll
    for (int off = 1; off < 64; off *= 2) sum = min(sum + __shfl_xor(sum, off), a.row_tiles);
    return __builtin_amdgcn_readfirstlane(sum);
}

struct ExpertTile {
    int expert, rows;          // rows 0: there is no such tile
    int64_t begin;             // its first slot
};

// Tile number `tile` of the experts' tiles of `most` slots, expert by expert: a wavefront adds up 64 experts' tiles at a time.
__device__ inline ExpertTile expert_tile(const QgExpertsArgs &a, int64_t tile, int most)
{
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
        const int e = e0 + lane;
        int64_t begin = 0, count = 0;
        if (e < a.experts) expert_slots(a, e, begin, count);
        const int mine = (int)((count + most - 1) / most);
        int upto = mine;
#pragma unroll
        for (int off = 1; off < 64; off *= 2) {
            const int o = __shfl_up(upto, off);
            if (lane >= off) upto += o;
        }
        const uint64_t past = __ballot(before + upto > tile);
        if (past) {
            const int at = __builtin_ctzll(past);
            const int64_t first = before + __shfl(upto - mine, at);
            ExpertTile t;
            t.expert = e0 + at;
            const int b = __shfl((int)begin, at), n = __shfl((int)count, at);
            t.begin = b + (tile - first) * most;
            const int64_t left = n - (tile - first) * most;
            if (left <= 0 || left > n) return {0, 0, 0};         // (offsets that decrease, whose tiles do not add up in 32 bits)
            t.rows = (int)(left < most ? left : most);
            return t;
        }
        before += __shfl(upto, 63);
    }
    return {0, 0, 0};
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

__device__ inline float silu(float v) { return v / (1.0f + expf(-v)); }

__device__ inline void store_typed(int type, void *p, int64_t i, float v)
{
    if (type == QG_F32) store_float<QG_F32>(p, i, v);
    else if (type == QG_BF16) store_float<QG_BF16>(p, i, v);
    else store_float<QG_F16>(p, i, v);
}

}  // namespace
