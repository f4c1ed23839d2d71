// Launcher of the attention of new tokens over the paged cache.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fast_div.h"

namespace vitq {

struct PagedParams {
    const uint8_t *q; int64_t q_ld; int64_t tokens;          // strides of q, out in elements
    int q_heads, kv_heads, group;                             // group = q_heads / kv_heads
    const int32_t *q_offsets, *kv_lens; int seqs;
    const int32_t *page_table; int64_t table_stride; int table_cols;
    const uint8_t *k, *v; uint32_t pages, page_size;
    uint32_t page_units, head_units, token_units;             // strides of the cache in units of 16 bytes
    int whole_rows;                                           // sixteen aligned keys lie in one page, within 2^31 bytes
    FastDiv page_div, group_div;
    float scale_log2, v_scale;                                // |scale| * k_scale * log2(e), not 0; scale of the values
    int negative;                                             // the scale is negative
    int causal, window;
    uint8_t *out; int64_t out_ld; float *lse;
    int splits; float *part, *part_lse;                       // [split][token][head][head_dim], [split][token][head]
    // set by the launcher: keys of a split, row tiles over all sequences, rows up to which a sequence is the streaming form's
    int split_keys, row_tiles; int64_t few_rows;
};

// Splits of the keys that the launcher chooses for these sizes (1: no workspace).
int paged_splits(int64_t tokens, int seqs, int q_heads, int kv_heads, int head_dim, int64_t max_kv);
// longest: keys that a row tile may see, as far as the host knows
hipError_t paged_launch(PagedParams p, int dtype, int cache_dtype, int head_dim, int64_t longest, hipStream_t stream);

}  // namespace vitq
