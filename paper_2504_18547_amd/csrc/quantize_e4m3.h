// Launcher of the 8-bit float quantizer with a scale per block of 128.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vitq {

struct QuantE4M3Params {
    const void *x; int64_t rows, cols, ld;
    int aligned;                                  // rows of x are 16-byte aligned
    uint8_t *codes; int64_t code_stride;
    float *scales; int64_t scale_stride;
};
hipError_t quantize_e4m3_launch(const QuantE4M3Params &p, int x_dtype, int block_rows, hipStream_t stream);

}  // namespace vitq
