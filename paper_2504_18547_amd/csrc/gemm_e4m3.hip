// Linear on E4M3 operands with a scale per block of 128 along the contraction:
//   y[m][n] = act(sum_j xs[j][m] * ws[j][n/128] * (sum_{k in block j} x[m][k] * w[n][k]) + bias[n])
//
// One v_mfma_f32_16x16x128_f8f6f4 is exactly one block of the contraction for 16 channels x 16 tokens: it starts from zero,
// and its four results per lane go into the fp32 total by an FMA with the product of the two scales.  A operand = weights
// (rows = channels), B operand = tokens (columns): a lane then holds ONE token, so its scale product is one value per token
// tile, and four consecutive channels, which leave as one store.
#include "gemm_e4m3.h"

#include "launch_util.h"
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
        // formats 0 / 0: E4M3 on both sides; constant zero scales select the instruction without them
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 0, 0, 0, 0, 0, 0);
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
        if (p.act) y[r] = gelu_any(y[r]);
    }
    const int64_t at = (int64_t)m * p.ld + n;
    if (p.y_dtype == kF32) {
        float *d = reinterpret_cast<float *>(p.y) + at;
        if (p.vec_ok && valid >= 4) *reinterpret_cast<v4f *>(d) = y;
        else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < valid) d[r] = y[r];
        }
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

// Eight consecutive outputs n.. of token m; full: all of them exist and are aligned for whole stores.
__device__ __forceinline__ void store8_f32(const GemmE4M3Params &p, int m, int n, const float (&y)[8], bool full) {
    float *d = reinterpret_cast<float *>(p.y) + (int64_t)m * p.ld + n;
    if (full) {
        reinterpret_cast<v4f *>(d)[0] = v4f{y[0], y[1], y[2], y[3]};
        reinterpret_cast<v4f *>(d)[1] = v4f{y[4], y[5], y[6], y[7]};
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (n + j < p.Nout) d[j] = y[j];
    }
}
__device__ __forceinline__ void store8_16bit(const GemmE4M3Params &p, int m, int n, const float (&y)[8], bool full) {
    u32 w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = p.y_dtype == kBF16 ? pack_bf16(y[2 * j], y[2 * j + 1]) : pack_f16(y[2 * j], y[2 * j + 1]);
    uint16_t *d = reinterpret_cast<uint16_t *>(p.y) + (int64_t)m * p.ld + n;
    if (full) *reinterpret_cast<uint4 *>(d) = make_uint4(w[0], w[1], w[2], w[3]);
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (n + j < p.Nout) d[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
}

__device__ __forceinline__ v8i operand(const v4i &a, const v4i &b) {
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
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
    // rows beyond the matrix and chunks beyond the padded row read as zeros
    const auto wbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w + (int64_t)c0 * p.w_stride), 0,
                                                        (u32)(min(16 * AT, p.Nout - c0) - 1) * (u32)p.w_stride + (u32)p.kbytes16, 0x00020000);
    const auto xbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.x + (int64_t)t0 * p.x_stride), 0,
                                                        (u32)(min(16 * TT, p.M - t0) - 1) * (u32)p.x_stride + (u32)p.kbytes16, 0x00020000);
    u32 wrow[AT], xrow[TT];
    const float *xsc[TT];
#pragma unroll
    for (int a = 0; a < AT; ++a) wrow[a] = (u32)(16 * a + l16) * (u32)p.w_stride;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        xrow[t] = (u32)(16 * t + l16) * (u32)p.x_stride;
        xsc[t] = p.xs + min(t0 + 16 * t + l16, p.M - 1);
    }
    const float *wsc = p.ws + (c0 >> 7);
    v4f acc[AT][TT];
#pragma unroll
    for (int a = 0; a < AT; ++a)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[a][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    for (int kb0 = wave; kb0 < nk; kb0 += nw * U) {
        v4i wv[U][AT][2], xv[U][TT][2];
        float sx[U][TT], sw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int kb = kb0 + u * nw;
            const u32 at0 = (u32)(kb * 128 + 16 * q), at1 = at0 + 64;
            // (a chunk of 16 bytes lies wholly inside the padded row or wholly beyond it)
            const bool in0 = at0 < (u32)p.kbytes16, in1 = at1 < (u32)p.kbytes16;
#pragma unroll
            for (int a = 0; a < AT; ++a) {
                wv[u][a][0] = __builtin_amdgcn_raw_buffer_load_b128(wbuf, in0 ? wrow[a] + at0 : ~15u, 0, 0);
                wv[u][a][1] = __builtin_amdgcn_raw_buffer_load_b128(wbuf, in1 ? wrow[a] + at1 : ~15u, 0, 0);
            }
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                xv[u][t][0] = __builtin_amdgcn_raw_buffer_load_b128(xbuf, in0 ? xrow[t] + at0 : ~15u, 0, 0);
                xv[u][t][1] = __builtin_amdgcn_raw_buffer_load_b128(xbuf, in1 ? xrow[t] + at1 : ~15u, 0, 0);
            }
            const int64_t row = min(kb, nk - 1);               // (behind the last block the operands are zeros: any scale will do)
            sw[u] = wsc[row * p.ws_stride];
#pragma unroll
            for (int t = 0; t < TT; ++t) sx[u][t] = xsc[t][row * p.xs_stride];
        }
        __builtin_amdgcn_sched_barrier(0);                      // all loads are on their way before the first product
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (kb0 + u * nw >= nk) break;                     // (a scale may be infinite or NaN: nothing is added behind the last)
#pragma unroll
            for (int a = 0; a < AT; ++a)
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    const v4f d = mfma_block<WIDE>(operand(wv[u][a][0], wv[u][a][1]), operand(xv[u][t][0], xv[u][t][1]));
                    const float s = sw[u] * sx[u][t];
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[a][t][r] = fmaf(d[r], s, acc[a][t][r]);
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

// ---- many tiles: operands through LDS ------------------------------------------------------------------------------------
// A workgroup of WC x WT waves owns WC*AT*16 channels x WT*TT*16 tokens; a stage is one block of the contraction (128 bytes of
// every row and the tokens' scales), S stages in LDS, filled by loads that go straight there.  LDS rows are unpadded, their
// 16-byte chunks permuted by the row so that the sixteen rows of an operand spread over the banks; weight rows sit in an order
// that gives a lane eight consecutive channels over two channel tiles.
// 8192 x 4096 -> 8192: 258 us, with GELU 267 (three sets of buffers in turn), 2.1 PFLOP/s; with one scale a tensor a library product reaches 3.2 on this card.  The matrix cores
// are busy 51 % of the time.  Without the FMAs that scale each block's products into the totals it took 27 us less, without the loads
// to LDS 43, without the stores 34: they add up, for a SIMD's two waves issue little more than an instruction every four cycles.
// Left out: products of the next stage's loads all at once (254 as well), 16 waves (registers spill).
__device__ __forceinline__ u32 lds_address_of(const void *p) {
    return (u32)(uintptr_t)(const __attribute__((address_space(3))) uint8_t *)p;
}
// Loads straight to LDS through a buffer descriptor: lane i's 16 (4) bytes at byte `off` go to dst + 16 i (4 i), zeros where
// `off` lies beyond the descriptor's size.  The compiler does not see them; they are waited for with vmcnt by hand.  (Nothing
// else here uses M0.)
__device__ __forceinline__ u32 uniform(u32 v) { return (u32)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ v4i descriptor(uint64_t base, u32 bytes) {
    v4i d;
    d[0] = (int)uniform((u32)base); d[1] = (int)uniform((u32)(base >> 32)); d[2] = (int)uniform(bytes); d[3] = 0x00020000;
    return d;
}
// `rows` rows (none if not positive) of `stride` bytes, the last one `tail` bytes long
__device__ __forceinline__ v4i rows_descriptor(uint64_t base, int rows, u32 stride, u32 tail) {
    return descriptor(base, rows > 0 ? (u32)(rows - 1) * stride + tail : 0u);
}
__device__ __forceinline__ void to_lds16(u32 off, const v4i &buf, u32 dst) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" :: "v"(off), "s"(buf), "s"(dst) : "memory");
}
__device__ __forceinline__ void to_lds4(u32 off, const v4i &buf, u32 dst) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" :: "v"(off), "s"(buf), "s"(dst) : "memory");
}

template <bool WIDE, int WC, int WT, int AT, int TT, int S>
__global__ __launch_bounds__(WC *WT * 64, 2) void gemm_e4m3_tile_kernel(const GemmE4M3Params p) {
    constexpr int kThreads = WC * WT * 64;
    constexpr int TC = WC * AT * 16, TK = WT * TT * 16;              // channels, tokens of the tile
    constexpr int kStage = (TC + TK) * 128 + TK * 4;
    static_assert((TC * 8) % kThreads == 0 && (TK * 8) % kThreads == 0, "a load instruction takes rows of one operand");
    static_assert(TK <= kThreads && TK % 64 == 0, "one scale load per wave");
    static_assert(S >= 2, "stages");
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wc = wave % WC, wt = wave / WC;
    const int l16 = lane & 15, q = lane >> 4;

    // The tiles in strips of four token tiles; workgroups go round-robin to the eight XCDs, each XCD has a run of consecutive
    // tiles, so that the workgroups of one L2 share operand rows, and a workgroup every `stride`-th of its XCD's.
    const int n_ct = (p.Nout + TC - 1) / TC, n_tt = (p.M + TK - 1) / TK, tiles = n_ct * n_tt;
    const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
    const int per = tiles >> 3, rem = tiles & 7;
    const int run0 = xcd < rem ? xcd * (per + 1) : rem * (per + 1) + (xcd - rem) * per, run1 = run0 + per + (xcd < rem ? 1 : 0);
    const int stride = ((int)gridDim.x + 7 - xcd) >> 3;               // workgroups of this XCD
    const int nk = (p.K + 127) >> 7;
    auto place = [&](int id, int &c0, int &t0) {
        const int strip = id / (4 * n_ct), in_strip = id - strip * 4 * n_ct;
        const int height = min(4, n_tt - 4 * strip);
        // (the divisions run on the vector unit: back to scalars, and with them every address that follows)
        const int col = (int)uniform((u32)(in_strip / height));
        c0 = col * TC;
        t0 = ((int)uniform((u32)(4 * strip + in_strip)) - col * (int)uniform((u32)height)) * TK;
    };
    int id = run0 + slot;
    if (id >= run1) return;

    // What each lane fetches per stage: chunk `chunk` of the rows r0 + kStep*i of the weights, then of the tokens.  LDS row r
    // of the weights is channel 32*(r/32) + 8*((r/4)%4) + 4*((r/16)%2) + r%4 of the tile: a lane's results of two channel tiles
    // are then eight consecutive channels.  Rows beyond the matrix and chunks beyond a ragged K arrive as zeros.
    constexpr int kStep = kThreads / 8, kLoadsW = TC / kStep, kLoadsX = TK / kStep;
    static_assert(TC % kStep == 0 && TK % kStep == 0 && kStep % 32 == 0, "whole channel groups per load instruction");
    const int r0 = (int)threadIdx.x >> 3;
    const u32 chunk = (u32)((threadIdx.x & 7) ^ (r0 & 7)) * 16u;
    const u32 w_stride = (u32)p.w_stride, x_stride = (u32)p.x_stride;
    const u32 lds0 = __builtin_amdgcn_readfirstlane(lds_address_of(smem)) + (u32)wave * 1024u;
    const u32 woff = (u32)(32 * (r0 >> 5) + 8 * ((r0 >> 2) & 3) + 4 * ((r0 >> 4) & 1) + (r0 & 3)) * w_stride + chunk;
    const u32 xoff = (u32)r0 * x_stride + chunk;

    // The stages of all tiles of the workgroup are one sequence; the load cursor runs up to S stages ahead of the sums.
    v4i wbuf[kLoadsW], xbuf[kLoadsX];
    uint64_t sbase = 0;
    u32 sbytes = 0;
    int next_id = id, load_kt = 0;
    u32 w_at = 0, x_at = 0;                                          // this lane's offsets; past the end beyond a ragged K
    auto aim = [&]() {
        const bool in = load_kt * 128 + (int)chunk < p.kbytes16;
        w_at = in ? woff + (u32)load_kt * 128u : ~15u;
        x_at = in ? xoff + (u32)load_kt * 128u : ~15u;
    };
    auto point = [&](bool some) {                                    // descriptors of tile next_id (empty ones behind the last)
        int c0 = 0, t0 = 0;
        if (some) place(next_id, c0, t0);
        const int rows_w = some ? min(TC, p.Nout - c0) : 0, rows_x = some ? min(TK, p.M - t0) : 0;
        const uint64_t wbase = (uint64_t)(uintptr_t)p.w + (uint64_t)c0 * p.w_stride, xbase = (uint64_t)(uintptr_t)p.x + (uint64_t)t0 * p.x_stride;
#pragma unroll
        for (int i = 0; i < kLoadsW; ++i) wbuf[i] = rows_descriptor(wbase + (u32)(kStep * i) * w_stride, rows_w - kStep * i, w_stride, p.kbytes16);
#pragma unroll
        for (int i = 0; i < kLoadsX; ++i) xbuf[i] = rows_descriptor(xbase + (u32)(kStep * i) * x_stride, rows_x - kStep * i, x_stride, p.kbytes16);
        sbase = (uint64_t)(uintptr_t)(p.xs + t0);
        sbytes = (u32)rows_x * 4u;
        aim();
    };
    // part i of the loads of the cursor's stage into buffer `buf`; the last part: the tokens' scales
    constexpr int kParts = kLoadsW + kLoadsX + 1;
    auto issue = [&](int buf, auto I) {
        constexpr int i = decltype(I)::value;
        const u32 dst = lds0 + (u32)buf * kStage + i * (kThreads * 16);
        if constexpr (i < kLoadsW) to_lds16(w_at, wbuf[i], dst);
        else if constexpr (i < kLoadsW + kLoadsX) to_lds16(x_at, xbuf[i - kLoadsW], dst);
        else {
            // (every wave, so that all have the same number of loads in flight; beyond the tokens the same ones again)
            const u32 part = (u32)wave % (TK / 64);
            to_lds4((part * 64u + (u32)lane) * 4u, descriptor(sbase, sbytes), lds0 - (u32)wave * 1024u + part * 256u + (u32)buf * kStage + (TC + TK) * 128);
            sbase += (uint64_t)p.xs_stride * 4u;
            if (++load_kt == nk) {
                load_kt = 0;
                next_id += stride;
                point(next_id < run1);
            } else {
                aim();
            }
        }
    };
    // The first parts go out when the buffer is free, the others one per channel tile: a burst of all of them queues in the
    // CU's one address path and holds the waves up.
    constexpr int kFirst = kParts - (AT - 2) > 2 ? kParts - (AT - 2) : 2;
    // Loads retire in order: with the S - 2 younger stages still on their way the oldest one is there.
    auto landed = []() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"((S - 2) * kParts) : "memory"); };
    point(true);
#pragma unroll
    for (int st = 0; st < S - 1; ++st) static_for<kParts>([&](auto I) { issue(st, I); });
    landed();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    static_for<kFirst>([&](auto I) { issue(S - 1, I); });

    // byte offsets of this lane's two chunks inside a row, and of its rows inside a stage
    const u32 p0 = (u32)((q ^ (l16 & 7)) * 16), p1 = (u32)(((q + 4) ^ (l16 & 7)) * 16);
    const u32 wrow = (u32)((wc * (16 * AT) + l16) * 128), xrow = (u32)((TC + wt * (16 * TT) + l16) * 128);
    auto frag = [&](const uint8_t *stage, u32 row) {
        return operand(*reinterpret_cast<const v4i *>(stage + row + p0), *reinterpret_cast<const v4i *>(stage + row + p1));
    };
    v8i xf[TT], wf[3];
    float sc[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) xf[t] = frag(smem, xrow + t * 2048);
    wf[0] = frag(smem, wrow);
    wf[1] = frag(smem, wrow + 2048);
    // Products run kLag ahead of the FMAs that add them to the totals, so that neither waits for the other.
    constexpr int kLag = 3;
    v4f d[kLag + 1], acc[AT][TT];
    auto add = [&](int i) {
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[i / TT][i % TT][r] = fmaf(d[i % (kLag + 1)][r], sc[i % TT], acc[i / TT][i % TT][r]);
        asm volatile("" : "+v"(acc[i / TT][i % TT]));           // here, not later: the products' registers are needed again
    };
    int buf = 0;
    for (; id < run1; id += stride) {
    int c0, t0;
    place(id, c0, t0);
    // (read-only for the whole kernel: scalar loads)
    const __attribute__((address_space(4))) float *wsc =
        (const __attribute__((address_space(4))) float *)(uintptr_t)(p.ws + (min(c0 + wc * (16 * AT), p.Nout - 1) >> 7));
    float sw = wsc[0];
#pragma unroll
    for (int a = 0; a < AT; ++a)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[a][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int kt = 0; kt < nk; ++kt) {
        const int buf1 = buf + 1 == S ? 0 : buf + 1, behind = buf == 0 ? S - 1 : buf - 1;
        const uint8_t *stage = smem + buf * kStage;
        const uint8_t *next = smem + buf1 * kStage;
        const float *xs = reinterpret_cast<const float *>(stage + (TC + TK) * 128) + wt * (16 * TT) + l16;
#pragma unroll
        for (int t = 0; t < TT; ++t) sc[t] = xs[16 * t] * sw;
        sw = wsc[(int64_t)min(kt + 1, nk - 1) * p.ws_stride];
        v8i next0, next1;
        static_for<AT * TT>([&](auto I) {
            constexpr int i = decltype(I)::value, a = i / TT, t = i % TT;
            // channel tiles are read two ahead; tile j of the next stage is tile AT + j of this one
            if constexpr (t == 0) {
                if constexpr (a + 2 < AT) {
                    wf[(a + 2) % 3] = frag(stage, wrow + (a + 2) * 2048);
                    if constexpr (kFirst + a < kParts) issue(behind, std::integral_constant<int, kFirst + a>{});
                } else if constexpr (a + 1 == AT) {
                    // every operand of this stage is in registers: its buffer is free once all waves say so, the next is full
                    landed();
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    next0 = frag(next, wrow);
                    next1 = frag(next, wrow + 2048);
                    static_for<kFirst>([&](auto J) { issue(buf, J); });
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            d[i % (kLag + 1)] = mfma_block<WIDE>(wf[a % 3], xf[t]);
            if constexpr (a + 1 == AT) xf[t] = frag(next, xrow + t * 2048);      // (behind the last stage: read, never used)
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (i >= kLag) add(i - kLag);
            __builtin_amdgcn_sched_barrier(0);
        });
        wf[0] = next0;
        wf[1] = next1;
        static_for<kLag>([&](auto I) { add(AT * TT - kLag + decltype(I)::value); });
        buf = buf1;
    }

    // a lane's eight consecutive channels of one token per two channel tiles
#pragma unroll
    for (int g = 0; g < AT / 2; ++g) {
        const int n = c0 + wc * (16 * AT) + 32 * g + 8 * q;
        float b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = p.bias && n + j < p.Nout ? p.bias[n + j] : 0.0f;
        const bool full = p.vec_ok && n + 8 <= p.Nout;
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const int m = t0 + wt * (16 * TT) + 16 * t + l16;
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = acc[2 * g + (j >> 2)][t][j & 3] + b[j];
            if (p.act) {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = gelu_any(y[j]);
            }
            if (m < p.M) {
                if constexpr (WIDE) store8_f32(p, m, n, y, full);
                else store8_16bit(p, m, n, y, full);
            }
        }
    }
    }
    // the loads behind the last stage (zeros, into a buffer that nobody reads) land before the LDS is given back
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <bool WIDE, int WC, int WT, int AT, int TT, int S>
hipError_t launch_tile(const GemmE4M3Params &p, hipStream_t stream) {
    constexpr int TC = WC * AT * 16, TK = WT * TT * 16;
    constexpr int lds = S * ((TC + TK) * 128 + TK * 4);
    static std::atomic<uint64_t> done{0};
    auto kern = gemm_e4m3_tile_kernel<WIDE, WC, WT, AT, TT, S>;
    hipError_t e = allow_dynamic_lds(reinterpret_cast<const void *>(kern), lds, done);
    if (e != hipSuccess) return e;
    const int64_t tiles = (int64_t)((p.Nout + TC - 1) / TC) * ((p.M + TK - 1) / TK);
    // as many workgroups as the 256 CUs hold at once, each with its share of the tiles
    const int64_t most = 256 * (163840 / lds);
    hipLaunchKernelGGL(kern, dim3((u32)(tiles < most ? tiles : most)), dim3(WC * WT * 64), lds, stream, p);
    return hipGetLastError();
}

// Which form (us, MI355X, K = 4096 unless given).
//   Up to 16 tokens: 16 channels a workgroup, so that 256 CUs share 4096 of them (16 x 4096 -> 4096 8.0, 16.8 MB of weights); up to 32:
//   both token tiles there (9.4, with 32 x 32 blocks 10.8).
//   Up to 512 blocks of 32 x 32: the waves share K (64 x 4096 -> 4096 11.0, 64 x 128 tiles 21; 256 x 1024 -> 1024 5.7 / 7.9); past
//   that the operands' second and third reading costs more than LDS (300 x 4096 -> 2000, 630 blocks, 26.4 / 18.8), the sooner where
//   rows are a multiple of 128 bytes and start in the same memory channels.  fp32 results, which are bound by the widening, stay up to
//   768, three workgroups a CU (760 x 4096 -> 1000 26.3 / 28.9; 777 x 4096 -> 1000, 800 blocks, 32.0 / 28.6).  Up to 1000 blocks of a short K: fp32
//   (777 x 1000 -> 1000 7.6 / 10.9, K 1024 10.8 / 10.8, K 1536 15.5 / 13.8); 16 bits where K is ragged (7.2 / 8.0, K 896 9.7 / 7.6,
//   K 1536 13.7 / 9.5) or the channels are, whose results leave as single stores (777 x 1000 -> 1001 7.5 / 10.2, 540 x 896 -> 1001
//   8.2 / 9.5).  The rule looks at sizes alone, not at where the results go, so that equal products have equal bits.
//   192 tiles of 256 x 256 and more fill the chip (8192 x 4096 -> 8192 258, with 128 x 128 tiles 345).  fp32 results, whose operands
//   are widened in registers, do not gain from them (594 against 510, in one run).
//   Up to 256 tiles of 64 x 128: a workgroup per CU, so four stages in its LDS and eight waves, two a SIMD, for one wave a SIMD issues
//   an instruction every eight to ten cycles (512 x 4096 -> 4096 22.8, 128 x 128 on eight waves 28.0, 64 x 128 on four 26.3).
//   Else 128 x 128 on eight waves (1024 x 4096 -> 4096 29.8, on four 35.3), fp32 results past a round on four (8192 x 4096 -> 8192 527 / 562).
template <bool WIDE>
hipError_t launch(const GemmE4M3Params &p, hipStream_t stream) {
    auto tiles = [&](int tokens, int channels) { return (int64_t)((p.M + tokens - 1) / tokens) * ((p.Nout + channels - 1) / channels); };
    if (p.M <= 16) return launch_split<WIDE, 1, 1, 4>(p, stream);
    if (p.M <= 32) return launch_split<WIDE, 1, 2, 2>(p, stream);
    const int64_t blocks = tiles(32, 32);
    const bool short_k = WIDE ? p.K <= 1024 : p.K <= 1000 && (p.K % 128 != 0 || p.Nout % 8 != 0);
    if (blocks <= (WIDE ? 768 : 512) || (blocks <= 1000 && short_k)) return launch_split<WIDE, 2, 2, 1>(p, stream);
    if constexpr (!WIDE) {
        if (tiles(256, 256) >= 192) return launch_tile<false, 2, 4, 8, 4, 2>(p, stream);
    }
    if (tiles(64, 128) <= 256) return launch_tile<WIDE, 4, 2, 2, 2, 4>(p, stream);
    if constexpr (WIDE) {
        if (tiles(128, 128) > 512) return launch_tile<true, 2, 2, 4, 4, 2>(p, stream);
    }
    return launch_tile<WIDE, 2, 4, 4, 2, 2>(p, stream);
}

}  // namespace

hipError_t gemm_e4m3_launch(const GemmE4M3Params &p, hipStream_t stream) {
    return p.y_dtype == kF32 ? launch<true>(p, stream) : launch<false>(p, stream);
}

}  // namespace vitq
