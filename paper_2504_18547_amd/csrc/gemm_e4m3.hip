// Linear on E4M3 operands with a scale per block of 128 along the contraction:
//   y[m][n] = act(sum_j xs[j][m] * ws[j][n/128] * (sum_{k in block j} x[m][k] * w[n][k]) + bias[n])
//
// One v_mfma_f32_16x16x128_f8f6f4 is exactly one block of the contraction for 16 channels x 16 tokens: it starts from zero,
// and its four results per lane go into the fp32 total by an FMA with the product of the two scales.  A operand = weights
// (rows = channels), B operand = tokens (columns): a lane then holds ONE token, so its scale product is one value per token
// tile, and four consecutive channels, which leave as one store.
#include "gemm_e4m3.h"
#include "serve_dev.h"

namespace vitq {

namespace {

// One block of the contraction from zero.  The 8-bit matrix cores (twice the 16-bit rate) align the products of every sixteen
// consecutive bytes of an operand to the largest and drop what lies more than 2^13 below it (measured with single products:
// 2^-13 of the largest arrives, 2^-14 does not): 1.5e-5 of a result of normal data, a tenth of a half-precision output's own
// rounding, but far from fp32.  So a result that leaves in fp32 takes the same values widened to bf16, which holds E4M3
// exactly, and the cores whose sums are fp32 (WIDE).
template <bool WIDE>
__device__ __forceinline__ v4f mfma_block(const v8i &w, const v8i &x) {
    v4f c = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (!WIDE) {
        // formats 0 / 0: E4M3 on both sides; the constant scale 127 is the exponent of 1
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 0, 0, 0, 0x7F7F7F7F, 0, 0x7F7F7F7F);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = mfma16<kBF16>(widen8<kBF16>((u32)w[2 * i], (u32)w[2 * i + 1]), widen8<kBF16>((u32)x[2 * i], (u32)x[2 * i + 1]), c);
        return c;
    }
}

// Four consecutive outputs n.. of token m.
__device__ __forceinline__ void store4(const GemmE4M3Params &p, int m, int n, v4f y) {
    if (m >= p.M || n >= p.Nout) return;
    const int valid = p.Nout - n;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (p.bias && r < valid) y[r] += p.bias[n + r];
        if (p.act) y[r] = gelu_fast(y[r]);
    }
    const int64_t at = (int64_t)m * p.ld + n;
    if (p.y_dtype == kF32) {
        float *d = reinterpret_cast<float *>(p.y) + at;
        if (p.vec_ok && valid >= 4) *reinterpret_cast<v4f *>(d) = y;
        else
            for (int r = 0; r < 4; ++r)
                if (r < valid) d[r] = y[r];
    } else {
        uint2 w;
        if (p.y_dtype == kBF16) { w.x = pack_bf16(y[0], y[1]); w.y = pack_bf16(y[2], y[3]); }
        else { w.x = pack_f16(y[0], y[1]); w.y = pack_f16(y[2], y[3]); }
        uint16_t *d = reinterpret_cast<uint16_t *>(p.y) + at;
        if (p.vec_ok && valid >= 4) *reinterpret_cast<uint2 *>(d) = w;
        else {
            if (valid > 0) d[0] = (uint16_t)w.x;
            if (valid > 1) d[1] = (uint16_t)(w.x >> 16);
            if (valid > 2) d[2] = (uint16_t)w.y;
            if (valid > 3) d[3] = (uint16_t)(w.y >> 16);
        }
    }
}

__device__ __forceinline__ v8i operand(const uint4 &a, const uint4 &b) {
    v8i r;
    r[0] = (int)a.x; r[1] = (int)a.y; r[2] = (int)a.z; r[3] = (int)a.w;
    r[4] = (int)b.x; r[5] = (int)b.y; r[6] = (int)b.z; r[7] = (int)b.w;
    return r;
}

// ---- few rows or few tiles: the waves of a workgroup share K ------------------------------------------------------------
// A workgroup owns AT*16 channels x TT*16 tokens; wave w takes the blocks w, w + NW, ... of the contraction, operands straight
// from memory into registers (a weight row is read by one workgroup per token tile, nothing to share through LDS), and the
// fp32 totals are added in LDS in the order of the waves.
template <bool WIDE, int AT, int TT, int U>
__global__ __launch_bounds__(1024) void gemm_e4m3_split_kernel(const GemmE4M3Params p) {
    extern __shared__ __attribute__((aligned(16))) float part[];       // [wave][tile][lane][4]
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    const int l16 = lane & 15, q = lane >> 4;
    const int c0 = blockIdx.x * (16 * AT), t0 = blockIdx.y * (16 * TT);
    const int nk = (p.K + 127) >> 7;
    const uint8_t *wrow[AT], *xrow[TT];
    const float *xsc[TT];
#pragma unroll
    for (int a = 0; a < AT; ++a) wrow[a] = p.w + (int64_t)min(c0 + 16 * a + l16, p.Nout - 1) * p.w_stride + 16 * q;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        const int m = min(t0 + 16 * t + l16, p.M - 1);
        xrow[t] = p.x + (int64_t)m * p.x_stride + 16 * q;
        xsc[t] = p.xs + m;
    }
    const float *wsc = p.ws + (c0 >> 7);
    v4f acc[AT][TT];
#pragma unroll
    for (int a = 0; a < AT; ++a)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[a][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    for (int kb0 = wave; kb0 < nk; kb0 += nw * U) {
        uint4 wv[U][AT][2], xv[U][TT][2];
        float s[U][TT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int kb = kb0 + u * nw;
            if (kb < nk) {
                // a chunk of 16 bytes lies wholly inside the padded row or wholly beyond it
                const bool in0 = kb * 128 + 16 * q < p.kbytes16, in1 = kb * 128 + 64 + 16 * q < p.kbytes16;
                const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int a = 0; a < AT; ++a) {
                    wv[u][a][0] = in0 ? *reinterpret_cast<const uint4 *>(wrow[a] + kb * 128) : zero;
                    wv[u][a][1] = in1 ? *reinterpret_cast<const uint4 *>(wrow[a] + kb * 128 + 64) : zero;
                }
                const float sw = wsc[(int64_t)kb * p.ws_stride];
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    xv[u][t][0] = in0 ? *reinterpret_cast<const uint4 *>(xrow[t] + kb * 128) : zero;
                    xv[u][t][1] = in1 ? *reinterpret_cast<const uint4 *>(xrow[t] + kb * 128 + 64) : zero;
                    s[u][t] = sw * xsc[t][(int64_t)kb * p.xs_stride];
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (kb0 + u * nw < nk) {
#pragma unroll
                for (int a = 0; a < AT; ++a)
#pragma unroll
                    for (int t = 0; t < TT; ++t) {
                        const v4f d = mfma_block<WIDE>(operand(wv[u][a][0], wv[u][a][1]), operand(xv[u][t][0], xv[u][t][1]));
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[a][t][r] = fmaf(d[r], s[u][t], acc[a][t][r]);
                    }
            }
        }
    }
    constexpr int kTiles = AT * TT;
    if (nw > 1) {
#pragma unroll
        for (int a = 0; a < AT; ++a)
#pragma unroll
            for (int t = 0; t < TT; ++t)
                *reinterpret_cast<v4f *>(part + ((wave * kTiles + a * TT + t) * 64 + lane) * 4) = acc[a][t];
        __syncthreads();
        for (int tile = wave; tile < kTiles; tile += nw) {
            v4f y = *reinterpret_cast<const v4f *>(part + (tile * 64 + lane) * 4);
            for (int i = 1; i < nw; ++i) y += *reinterpret_cast<const v4f *>(part + ((i * kTiles + tile) * 64 + lane) * 4);
            const int a = tile / TT, t = tile % TT;
            store4(p, t0 + 16 * t + l16, c0 + 16 * a + 4 * q, y);
        }
    } else {
#pragma unroll
        for (int a = 0; a < AT; ++a)
#pragma unroll
            for (int t = 0; t < TT; ++t) store4(p, t0 + 16 * t + l16, c0 + 16 * a + 4 * q, acc[a][t]);
    }
}

template <bool WIDE, int AT, int TT, int U>
hipError_t launch_split(const GemmE4M3Params &p, hipStream_t stream) {
    const int nk = (p.K + 127) / 128;
    int nw = (nk + U - 1) / U;
    if (nw > 16) nw = 16;
    const dim3 grid((p.Nout + 16 * AT - 1) / (16 * AT), (p.M + 16 * TT - 1) / (16 * TT));
    hipLaunchKernelGGL((gemm_e4m3_split_kernel<WIDE, AT, TT, U>), grid, dim3(64 * nw), nw > 1 ? nw * AT * TT * 1024 : 0, stream, p);
    return hipGetLastError();
}

template <bool WIDE>
hipError_t launch(const GemmE4M3Params &p, hipStream_t stream) {
    if (p.M <= 16) return launch_split<WIDE, 1, 1, 4>(p, stream);
    return launch_split<WIDE, 2, 2, 1>(p, stream);
}

}  // namespace

hipError_t gemm_e4m3_launch(const GemmE4M3Params &p, hipStream_t stream) {
    return p.y_dtype == kF32 ? launch<true>(p, stream) : launch<false>(p, stream);
}

}  // namespace vitq
