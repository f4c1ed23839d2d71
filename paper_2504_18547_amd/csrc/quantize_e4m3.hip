// E4M3 codes with one scale per 1 x 128 or 128 x 128 block: a = max(max |x|, 2^-100), scale = a / 448,
// code = x * (448 / a) rounded to nearest even.  Bound by HBM (bytes of x, one byte per code, scales).
//
// The maximum is taken on the bit patterns of |x|: there unsigned order is float order, and a NaN lies above
// every number, so it reaches the scale (and by the multiplication every code) as the definition wants.  |x| <= a
// makes |x * (448 / a)| <= 448 * (1 + 2^-23), which rounds to 448: nothing has to be limited.
#include "quantize_e4m3.h"
#include "serve_dev.h"

namespace vitq {

namespace {

constexpr float kMaxE4M3 = 448.0f;
constexpr float kTiny = 0x1p-100f;

__device__ __forceinline__ u32 max_bits(const float (&v)[8]) {
    u32 m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
}

// The eight columns c.. of a row as floats, zeros beyond the matrix.
template <int DT>
__device__ __forceinline__ void gather8(const QuantE4M3Params &p, int64_t r, int64_t c, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (r < p.rows && c + i < p.cols) ? load1<DT>(p.x, r * p.ld + c + i) : 0.0f;
}

// The bytes of the eight columns c.. that are the matrix's own: a row's padding is written as zero, beside a NaN too (where zero
// times the factor is not).
__device__ __forceinline__ uint2 own_bytes(const QuantE4M3Params &p, int64_t c) {
    const int valid = (int)min(p.cols - c, (int64_t)8);
    const uint64_t keep = valid > 0 ? ~uint64_t(0) >> (64 - 8 * valid) : 0;
    return make_uint2((u32)keep, (u32)(keep >> 32));
}
__device__ __forceinline__ void store8(const QuantE4M3Params &p, int64_t r, int64_t c, const float (&v)[8], float f, uint2 keep) {
    uint2 w;
    w.x = pack_e4m3(v[0] * f, v[1] * f, v[2] * f, v[3] * f) & keep.x;
    w.y = pack_e4m3(v[4] * f, v[5] * f, v[6] * f, v[7] * f) & keep.y;
    *reinterpret_cast<uint2 *>(p.codes + r * p.code_stride + c) = w;
}

// One row per 16 lanes, sixteen rows and U column blocks per workgroup: a lane owns eight columns of each block, so loads
// and stores are whole 256- (128-) byte pieces of a row, and the sixteen scales of a column block leave as one line.
// 16,384 x 4,096 bf16: 45 us, 4.5 TB/s of the 5.2 that a large copy reaches on this card (read and written).
template <int DT, int U>
__global__ __launch_bounds__(256) void quantize_e4m3_rows_kernel(const QuantE4M3Params p) {
    const int lane16 = threadIdx.x & 15;
    const int64_t r = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int64_t c0 = (int64_t)blockIdx.y * (128 * U) + 8 * lane16;
    const int64_t padded = (p.cols + 15) / 16 * 16;
    float v[U][8];
    Raw8<DT> raw[U];
    const bool vec = p.aligned && r < p.rows;
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (vec && c0 + 128 * u + 8 <= p.cols) raw[u] = load8<DT>(p.x, r * p.ld + c0 + 128 * u);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (vec && c0 + 128 * u + 8 <= p.cols) values8<DT>(raw[u], v[u]);
        else gather8<DT>(p, r, c0 + 128 * u, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t c = c0 + 128 * u;
        const u32 m = reduce_lanes(max_bits(v[u]), 16, [](u32 a, u32 b) { return max(a, b); });
        const float a = __uint_as_float(max(m, __float_as_uint(kTiny)));
        if (r < p.rows && c < padded) {
            store8(p, r, c, v[u], kMaxE4M3 / a, own_bytes(p, c));
            if (lane16 == 0) p.scales[(c >> 7) * p.scale_stride + r] = a / kMaxE4M3;
        }
    }
}

// A 128 x 128 block per workgroup, held in registers between the maximum and the codes.  14,336 x 4,096 bf16: 41.6 us, 4.2 TB/s;
// 8,192 x 8,192 fp32: 80.6 us, the same rate.
template <int DT>
__global__ __launch_bounds__(256) void quantize_e4m3_blocks_kernel(const QuantE4M3Params p) {
    __shared__ u32 top[4];
    const int lane16 = threadIdx.x & 15, row0 = threadIdx.x >> 4;
    const int64_t r0 = (int64_t)blockIdx.x * 128, c = (int64_t)blockIdx.y * 128 + 8 * lane16;
    const int64_t padded = (p.cols + 15) / 16 * 16;
    Raw8<DT> raw[8];
    const bool vec = p.aligned && c + 8 <= p.cols;
    u32 m = 0;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + row0 + 16 * i;
        if (vec && r < p.rows) raw[i] = load8<DT>(p.x, r * p.ld + c);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + row0 + 16 * i;
        if (vec && r < p.rows) values8<DT>(raw[i], v);
        else gather8<DT>(p, r, c, v);
        m = max(m, max_bits(v));
    }
    m = reduce_lanes(m, 16, [](u32 a, u32 b) { return max(a, b); });
    {
        auto s = __builtin_amdgcn_permlane16_swap(m, m, false, false);
        m = max((u32)s[0], (u32)s[1]);
        s = __builtin_amdgcn_permlane32_swap(m, m, false, false);
        m = max((u32)s[0], (u32)s[1]);
    }
    if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max(max(top[0], top[1]), max(top[2], top[3]));
    const float a = __uint_as_float(max(m, __float_as_uint(kTiny)));
    const float f = kMaxE4M3 / a;
    if (threadIdx.x == 0) p.scales[(int64_t)blockIdx.y * p.scale_stride + blockIdx.x] = a / kMaxE4M3;
    if (c >= padded) return;
    const uint2 keep = own_bytes(p, c);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + row0 + 16 * i;
        if (r >= p.rows) continue;
        if (vec) values8<DT>(raw[i], v);
        else gather8<DT>(p, r, c, v);
        store8(p, r, c, v, f, keep);
    }
}

template <int DT>
hipError_t launch(const QuantE4M3Params &p, int block_rows, hipStream_t stream) {
    const int64_t nb = (p.cols + 127) / 128;
    if (block_rows == 1) {
        const int64_t rg = (p.rows + 15) / 16;
        // four column blocks per workgroup keep enough loads in flight once there are workgroups to spare; below that
        // every block is its own workgroup (197 x 768: 78 workgroups, the device done in 2.5 us, the call in 6.7)
        if (rg * nb >= 8192) {
            hipLaunchKernelGGL((quantize_e4m3_rows_kernel<DT, 4>), dim3((u32)rg, (u32)((nb + 3) / 4)), dim3(256), 0, stream, p);
        } else {
            hipLaunchKernelGGL((quantize_e4m3_rows_kernel<DT, 1>), dim3((u32)rg, (u32)nb), dim3(256), 0, stream, p);
        }
    } else {
        hipLaunchKernelGGL((quantize_e4m3_blocks_kernel<DT>), dim3((u32)((p.rows + 127) / 128), (u32)nb), dim3(256), 0, stream, p);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t quantize_e4m3_launch(const QuantE4M3Params &p, int x_dtype, int block_rows, hipStream_t stream) {
    switch (x_dtype) {
        case kF32: return launch<kF32>(p, block_rows, stream);
        case kBF16: return launch<kBF16>(p, block_rows, stream);
        default: return launch<kF16>(p, block_rows, stream);
    }
}

}  // namespace vitq
