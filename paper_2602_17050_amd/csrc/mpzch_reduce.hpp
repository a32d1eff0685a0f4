// What the host and the kernel of the sums over sorted entries share.
#pragma once
#include "../../include/mpzch.h"
#include "mpzch_embed_kernels.hpp"

namespace mpzch {

constexpr int kReduceBlock = 512;
constexpr int kReduceTile = 2048;                // entries of a workgroup at most
struct ReduceArgs {
    const uint64_t *entries;
    int64_t n;
    uint32_t num_rows;
    int32_t tiles, tile;         // entries of a workgroup, a multiple of its groups
    int32_t lanes;               // of a group
    int32_t col_blocks;          // workgroups that share out the columns of a tile
    const char *grad;
    uint32_t grad_stride;        // bytes, as row_stride
    bool read_past_caches;       // grad is loaded non-temporally
    int32_t dim;
    float factor;
    Mask mask;
    // shares of the tiles, tiles x dim each: of a run that began before, and of one that begins in the tile
    float *head, *tail;
    uint32_t *tail_index;        // of the run that begins in the tile, among all
    uint32_t *arrived;           // shares of the run that begins in the tile, for each block of columns; zero between the calls
    const uint32_t *heads;       // runs that begin in a tile, or (heads_are == kBeforeTile) in all tiles before
    int32_t heads_are;
    // gradient
    int64_t *out_slots, *out_count;
    char *out_rows;
    int64_t cap;
    bool past_caches;            // out_rows are stored non-temporally
    // step
    char *rows;
    uint32_t row_stride;
    float per_element;           // 1 / dim
    float *state;
    const float *lr;
    float eps;
    int32_t type;                // of out_rows or rows
};
constexpr int32_t kOfTile = 0, kBeforeTile = 1, kCountHere = 2;

__device__ __forceinline__ uint32_t row_at(const uint64_t *entries, int64_t i) { return (uint32_t)(entries[i] >> 32); }

// The kernel of the sums, compiled once for each size of a table's elements (0: the gradient).
#define MPZCH_LAUNCH_REDUCE(bytes)                                                                                         \
    mpzch_status_t launch_reduce_##bytes(const ReduceArgs &a, int32_t grad_type, int width, int pieces, int grid, hipStream_t s)
MPZCH_LAUNCH_REDUCE(0);
MPZCH_LAUNCH_REDUCE(2);
MPZCH_LAUNCH_REDUCE(4);

}  // namespace mpzch
