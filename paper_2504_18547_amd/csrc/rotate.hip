// Per-head norm of queries and keys, rotation by position, and the keys' and values' way into the paged cache: one pass over
// the fused projection's rows.  Bound by HBM: every input read once, every output written once (16,384 tokens of 32 + 2 x 8 heads of
// 128 in bf16: 80 us, 5.1 TB/s, what a large copy reaches on this card; 5,193 tokens of 3 x 16 heads of 64, fp32 to an E4M3 cache
// 18 us, 4.7 TB/s).
//
// A group of L lanes (the power of two with 8 L >= head_dim) owns one head of one token, eight channels per lane: loads and
// stores of 16 bytes per lane are whole rows of a head, the statistics are sums over the group, and the rotation's partner
// channels (rot_dim/2 further) are eight channels of one other lane.  A workgroup takes 256 / L x ITER heads of one token, so the
// token's angles are read once for ITER heads.  The heads are those whose outputs are wanted: of the others neither values nor
// gammas are read (there may be none).
#include "rotate.h"
#include "serve_dev.h"

namespace vitq {

namespace {

// Writes eight channels in the type of the destination (elements, 16-byte aligned; E4M3: 8-byte).
__device__ __forceinline__ void store_channels(uint8_t *base, int64_t at, int dtype, const float (&v)[8], float inv) {
    if (dtype == kE4M3) {
        float s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float t = v[i] * inv;
            s[i] = t != t ? t : __builtin_amdgcn_fmed3f(t, -448.0f, 448.0f);
        }
        *reinterpret_cast<uint2 *>(base + at) = make_uint2(pack_e4m3(s[0], s[1], s[2], s[3]), pack_e4m3(s[4], s[5], s[6], s[7]));
    } else {
        uint4 w;
        if (dtype == kBF16) {
            w = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
        } else {
            w = make_uint4(pack_f16(v[0], v[1]), pack_f16(v[2], v[3]), pack_f16(v[4], v[5]), pack_f16(v[6], v[7]));
        }
        *reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(base) + at) = w;
    }
}

__device__ __forceinline__ void load_floats8(const float *p, float (&v)[8]) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

template <int DT, int L, int ITER>
__global__ __launch_bounds__(256) void rotate_kernel(const RotateParams p) {
    constexpr int kGroups = 256 / L;
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const int c0 = 8 * lane;
    const bool live = c0 < p.head_dim;
    const int heads = p.head_end;
    const int h0 = p.head_begin + blockIdx.y * (kGroups * ITER) + group;

    float c[8], s[8];
    const int half = p.rot_dim >> 1;
    const bool turns = live && c0 < p.rot_dim;
    const bool upper = !p.interleaved && c0 >= half;
    Raw8<DT> raw[ITER];
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int h = h0 + i * kGroups;
        if (live && h < heads) raw[i] = load8<DT>(p.qkv, t * p.ld + (int64_t)h * p.head_dim + c0);
    }
    if (p.rot_dim > 0) {
        const int64_t pos = p.positions[t];
        if (pos < 0 || pos >= p.table_rows) return;             // padding (the same for the whole workgroup)
        if (turns) {
            if (p.interleaved) {                                // pairs (c0/2 .. c0/2 + 3), each for two channels
                const float4 cc = *reinterpret_cast<const float4 *>(p.cos_table + pos * half + (c0 >> 1));
                const float4 ss = *reinterpret_cast<const float4 *>(p.sin_table + pos * half + (c0 >> 1));
                c[0] = cc.x; c[2] = cc.y; c[4] = cc.z; c[6] = cc.w;
                s[0] = ss.x; s[2] = ss.y; s[4] = ss.z; s[6] = ss.w;
            } else {
                const int64_t at = pos * half + (upper ? c0 - half : c0);
                load_floats8(p.cos_table + at, c);
                load_floats8(p.sin_table + at, s);
            }
        }
    }
    // the token's place in the cache
    int64_t row = -1;
    if (p.slots) {
        const int64_t slot = p.slots[t];
        if (slot >= 0 && slot < p.slots_end) {
            const u32 page = divide((u32)slot, p.page_div);
            row = page * p.page_stride + ((u32)slot - page * p.page_size) * p.token_stride;
        }
    }
    const int partner = (int)(threadIdx.x & 63) + (upper ? -(half >> 3) : (half >> 3));

#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int h = h0 + i * kGroups;
        if (h0 - group + i * kGroups >= heads) break;            // uniform: no group of the workgroup has a head left
        const bool mine = live && h < heads;
        float v[8];
        if (mine) values8<DT>(raw[i], v);
        else
            for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        const bool is_q = h < p.q_heads;
        const int hk = h - p.q_heads;
        const bool is_v = hk >= p.kv_heads;
        // (lanes of a wave may hold heads of different kinds; the group's reductions stay inside the group)
        if (p.norm != 0) {
            float mean = 0.0f;
            if (p.norm == 2) {
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += v[j];
                mean = sum_lanes(sum, L) * p.inv_dim;
            }
            float sq = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = v[j] - mean;
                sq = fmaf(d, d, sq);
            }
            if (!live) sq = 0.0f;
            const float var = sum_lanes(sq, L) * p.inv_dim;
            if (mine && !is_v) {
                const float r = 1.0f / sqrtf(var + p.eps);
                const float *gamma = (is_q ? p.q_gamma : p.k_gamma) + (is_q ? h : hk) * p.gamma_stride + c0;
                const float *beta = is_q ? p.q_beta : p.k_beta;
                float g[8];
                load_floats8(gamma, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = ((v[j] - mean) * r) * g[j];
                if (p.norm == 2 && beta) {
                    float b[8];
                    load_floats8(beta + (is_q ? h : hk) * p.gamma_stride + c0, b);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] += b[j];
                }
            }
        }
        if (p.rot_dim > 0) {
            if (p.interleaved) {
                if (turns && !is_v) {
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const float a = v[j], b = v[j + 1];
                        v[j] = fmaf(a, c[j], -(b * s[j]));
                        v[j + 1] = fmaf(b, c[j], a * s[j]);
                    }
                }
            } else {
                float o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = __shfl(v[j], partner);
                if (turns && !is_v) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = upper ? fmaf(v[j], c[j], o[j] * s[j]) : fmaf(v[j], c[j], -(o[j] * s[j]));
                }
            }
        }
        if (mine) {
            if (is_q) {
                store_channels((uint8_t *)p.q_out, t * p.q_ld + (int64_t)h * p.head_dim + c0, p.q_dtype, v, 1.0f);
            } else if (row >= 0) {
                const int hh = is_v ? hk - p.kv_heads : hk;
                store_channels(is_v ? p.v : p.k, row + hh * p.head_stride + c0, p.cache_dtype, v, is_v ? p.v_inv : p.k_inv);
            }
        }
    }
}

template <int DT, int L>
hipError_t launch(const RotateParams &p, hipStream_t stream) {
    constexpr int kGroups = 256 / L;
    const int heads = p.head_end - p.head_begin;
    const int rounds = (heads + kGroups - 1) / kGroups;
    // few tokens: every round of heads is a workgroup of its own (one token: 7.4 us a call, nearly all of it the host's); else three
    // rounds a workgroup.  us with one, two, three, six: 16,384 tokens of 32 + 2 x 8 heads of 128 bf16 94.5 / 88.3 / 82.2 / 88.3,
    // 8,192 of 28 + 2 x 4 33.4 / 33.2 / 29.8 / 31.7, 5,193 of 3 x 16 heads of 64 fp32 16.3 / 16.9 / 17.4 / 18.7
    if (p.tokens * rounds <= 2048 || rounds == 1) {
        hipLaunchKernelGGL((rotate_kernel<DT, L, 1>), dim3((u32)p.tokens, rounds), dim3(256), 0, stream, p);
    } else {
        hipLaunchKernelGGL((rotate_kernel<DT, L, 3>), dim3((u32)p.tokens, (rounds + 2) / 3), dim3(256), 0, stream, p);
    }
    return hipGetLastError();
}

template <int DT>
hipError_t launch_dim(const RotateParams &p, hipStream_t stream) {
    if (p.head_dim <= 64) return launch<DT, 8>(p, stream);
    if (p.head_dim <= 128) return launch<DT, 16>(p, stream);
    return launch<DT, 32>(p, stream);
}

}  // namespace

hipError_t rotate_launch(const RotateParams &p, int dtype, hipStream_t stream) {
    switch (dtype) {
        case kF32: return launch_dim<kF32>(p, stream);
        case kBF16: return launch_dim<kBF16>(p, stream);
        default: return launch_dim<kF16>(p, stream);
    }
}

}  // namespace vitq
