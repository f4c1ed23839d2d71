// Launcher of the per-head norm + rotation that appends to the paged cache.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fast_div.h"

namespace vitq {

struct RotateParams {
    const void *qkv; int64_t ld; int64_t tokens;
    int q_heads, kv_heads, head_dim;
    int head_begin, head_end;                          // heads of a row (queries, keys, values) whose outputs are wanted
    int norm, rot_dim, interleaved;
    const float *q_gamma, *q_beta, *k_gamma, *k_beta; int64_t gamma_stride;
    const float *cos_table, *sin_table; int64_t table_rows;
    float eps, inv_dim;
    const int32_t *positions;
    void *q_out; int q_dtype; int64_t q_ld;
    uint8_t *k, *v; int cache_dtype;                   // strides in elements
    int64_t page_stride, head_stride, token_stride;
    int64_t slots_end;                                 // pages * page_size
    uint32_t page_size; FastDiv page_div;
    float k_inv, v_inv;
    const int64_t *slots;
};
hipError_t rotate_launch(const RotateParams &p, int dtype, hipStream_t stream);

}  // namespace vitq
