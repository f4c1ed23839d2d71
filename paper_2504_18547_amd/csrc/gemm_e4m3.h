// Launcher of the block-scaled E4M3 linear.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vitq {

struct GemmE4M3Params {
    const uint8_t *x; int64_t x_stride; const float *xs; int64_t xs_stride; int M;      // tokens  [M x K]
    const uint8_t *w; int64_t w_stride; const float *ws; int64_t ws_stride; int Nout;   // weights [Nout x K]
    int K;
    int kbytes16;                 // bytes of a row up to its padding
    const float *bias; int act;
    void *y; int y_dtype; int64_t ld;
    int vec_ok;                   // rows of y are 16-byte aligned
};
hipError_t gemm_e4m3_launch(const GemmE4M3Params &p, hipStream_t stream);

}  // namespace vitq
