// Device-side helpers of the 16-bit and 8-bit floating-point kernels (gfx950 only).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vitq_dev.h"

namespace vitq {

enum DType { kF32 = 0, kBF16 = 1, kF16 = 2, kE4M3 = 3 };

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf_lo(u32 w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(u32 w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ u32 pack_bf16(float a, float b) {
    v2bf v; v[0] = (__bf16)a; v[1] = (__bf16)b;
    return __builtin_bit_cast(u32, v);
}
__device__ __forceinline__ u32 pack_f16(float a, float b) {
    v2h v; v[0] = (_Float16)a; v[1] = (_Float16)b;
    return __builtin_bit_cast(u32, v);
}
template <int DT>
__device__ __forceinline__ u32 pack16bit(float a, float b) {
    return DT == kBF16 ? pack_bf16(a, b) : pack_f16(a, b);
}
template <int DT>
__device__ __forceinline__ void unpack16bit(u32 w, float &a, float &b) {
    if constexpr (DT == kBF16) { a = bf_lo(w); b = bf_hi(w); }
    else { const v2h v = __builtin_bit_cast(v2h, w); a = (float)v[0]; b = (float)v[1]; }
}

// four floats -> four E4M3 bytes, nearest even; the conversion has no infinities, so magnitudes must not exceed 448 (463.9
// still rounds to it); NaN stays NaN
__device__ __forceinline__ u32 pack_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (u32)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef u32 v4u __attribute__((ext_vector_type(4)));

template <int DT>
__device__ __forceinline__ v4f mfma16(const v4u &a, const v4u &b, const v4f &c) {
    if constexpr (DT == kBF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// two E4M3 bytes (the low or the high half of w) -> two 16-bit floats, exact
template <int DT, bool HI>
__device__ __forceinline__ u32 widen(u32 w) {
    if constexpr (DT == kBF16) return __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
    else return __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HI));
}

// eight E4M3 bytes -> eight 16-bit floats
template <int DT>
__device__ __forceinline__ v4u widen8(u32 lo, u32 hi) {
    v4u r;
    r[0] = widen<DT, false>(lo); r[1] = widen<DT, true>(lo); r[2] = widen<DT, false>(hi); r[3] = widen<DT, true>(hi);
    return r;
}

// 0.5 y (1 + tanh(sqrt(2 / pi) (y + 0.044715 y^3))) for any y, as y / (1 + 2^(w y)) with w = -2 log2(e) sqrt(2 / pi) (1 + 0.044715 y^2):
// within 2^-21 of |y|; infinity at +infinity, where gelu_fast, which is for finite y, takes infinity times zero from it; NaN at
// -infinity like the definition (times zero).
__device__ __forceinline__ float gelu_any(float y) {
    const float w = fmaf(y * y, -0x1.a5a7d0p-4f, -0x1.26aec2p+1f);
    return y * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(w * y));
}

// One element of any of the three input types.
template <int DT>
__device__ __forceinline__ float load1(const void *p, int64_t i) {
    if constexpr (DT == kF32) return reinterpret_cast<const float *>(p)[i];
    else if constexpr (DT == kBF16) return __uint_as_float((u32)reinterpret_cast<const uint16_t *>(p)[i] << 16);
    else return (float)reinterpret_cast<const _Float16 *>(p)[i];
}
// Eight consecutive elements as they are in memory (16-byte aligned), and their values.
template <int DT> struct Raw8 { uint4 a; };
template <> struct Raw8<kF32> { uint4 a, b; };
template <int DT>
__device__ __forceinline__ Raw8<DT> load8(const void *p, int64_t i) {
    Raw8<DT> r;
    if constexpr (DT == kF32) {
        const uint4 *q = reinterpret_cast<const uint4 *>(reinterpret_cast<const float *>(p) + i);
        r.a = q[0]; r.b = q[1];
    } else {
        r.a = *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(p) + i);
    }
    return r;
}
template <int DT>
__device__ __forceinline__ void values8(const Raw8<DT> &r, float (&v)[8]) {
    if constexpr (DT == kF32) {
        v[0] = __uint_as_float(r.a.x); v[1] = __uint_as_float(r.a.y); v[2] = __uint_as_float(r.a.z); v[3] = __uint_as_float(r.a.w);
        v[4] = __uint_as_float(r.b.x); v[5] = __uint_as_float(r.b.y); v[6] = __uint_as_float(r.b.z); v[7] = __uint_as_float(r.b.w);
    } else {
        unpack16bit<DT>(r.a.x, v[0], v[1]); unpack16bit<DT>(r.a.y, v[2], v[3]);
        unpack16bit<DT>(r.a.z, v[4], v[5]); unpack16bit<DT>(r.a.w, v[6], v[7]);
    }
}

// All-reduce over aligned groups of 2..16 lanes: quads by permutation, then mirrored halves.
template <int CTRL>
__device__ __forceinline__ u32 dpp(u32 v) {
    return (u32)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
template <class F>
__device__ __forceinline__ u32 reduce_lanes(u32 v, int lanes, F &&f) {
    if (lanes > 1) v = f(v, dpp<0xB1>(v));        // quad_perm 1,0,3,2
    if (lanes > 2) v = f(v, dpp<0x4E>(v));        // quad_perm 2,3,0,1
    if (lanes > 4) v = f(v, dpp<0x141>(v));       // mirror of eight
    if (lanes > 8) v = f(v, dpp<0x140>(v));       // mirror of sixteen
    return v;
}
__device__ __forceinline__ float sum_lanes(float v, int lanes) {
    u32 r = reduce_lanes(__float_as_uint(v), lanes, [](u32 a, u32 b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); });
    if (lanes > 16) { const auto s = __builtin_amdgcn_permlane16_swap(r, r, false, false); r = __float_as_uint(__uint_as_float(s[0]) + __uint_as_float(s[1])); }
    return __uint_as_float(r);
}

}  // namespace vitq
