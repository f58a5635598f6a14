// Parameters that the attention kernels share.
#pragma once
#include "tensor_ops.cuh"

namespace hbf {

struct AttnDev {
    const uint16_t *k, *v;
    int64_t page_stride, slot_stride, head_stride;
    uint32_t n_pages, Hk, G, Hq, B;
    Div32 div_page, div_g;
    uint32_t page_tokens;
    const uint16_t *q; int64_t q_row, q_head;
    uint16_t *out; int64_t out_row, out_head;
    float *lse;
    float scale_log2;                                        // scores are kept in units of log 2
    uint32_t prefix_len, max_own, own_stride;
    const int32_t *prefix_pages, *own_pages, *own_len;
    // the pieces: `row_tiles` * Hk * prefix_pieces of the prefix, then B * Hk * group_tiles * own_pieces of the requests' own keys
    uint32_t row_tiles, prefix_pieces, prefix_chunk, group_tiles, own_pieces, own_chunk, n_prefix_items;
    uint32_t rows, prefix_rows;                              // rows of a tile; of the prefix's: the same, or 256 (two tiles) with k_prefix_tiles
    // what a piece leaves: sums not yet divided, [piece][row][d], and (largest score, sum of weights), [piece][row]
    float *part_o; float2 *part_ml;
    uint32_t pieces;                                         // own_pieces + prefix_pieces of every row; 1: written straight to `out`
    uint32_t behind;                                         // k_attend was launched to overlap k_prefix_tiles
    uint32_t polls;                                          // of a wait in k_prefix_tiles
};

// The place of key `i` of a table's sequence; false: its page is none of the cache's.
__device__ __forceinline__ bool key_place(const AttnDev &p, int32_t page, uint32_t slot, int64_t &at) {
    at = (int64_t)page * p.page_stride + (int64_t)slot * p.slot_stride;
    return (uint32_t)page < p.n_pages;
}

cudaError_t launch_prefix_tiles(const AttnDev &p, uint32_t dim, bool bf16, cudaStream_t st);

}  // namespace hbf
