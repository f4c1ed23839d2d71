// Attention of new tokens over a paged cache: softmax(scale q.k) v per query head, one pass over the keys with the running
// maximum and sum of the softmax, on 16-bit MFMAs.
//
// The rows of a sequence and a key-value head are its new tokens times the query heads that share the head: row r is token
// r / group, head r % group of the group, so a cache row is read once for all of them.  Scores are computed transposed
// (S^T = K Q^T): a lane of the result holds keys of ONE row, the softmax statistics are per lane, and the probabilities are
// already the B operand of O^T = V^T P^T, whose order of keys is that of the score registers.
#include "attention_paged.h"
#include "serve_dev.h"

namespace vitq {

namespace {

// max / sum over the four lanes l, l+16, l+32, l+48
__device__ __forceinline__ float max_quarters(float v) {
    auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
    s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float sum_quarters(float v) {
    auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// ---- which rows a workgroup has ------------------------------------------------------------------------------------------
// Row tiles of all sequences in one line: sequence s starts at tile floor(q_offsets[s] * group / ROWS) + s, which leaves it
// at least the tiles that its rows need, wherever they begin; the number of tiles follows from the totals alone.
struct RowTile {
    int first, count;        // first token of the sequence, its tokens
    int kv_len;
    int seq;
    int row0, rows;          // first row of the tile and the rows it has
};

__device__ __forceinline__ int64_t clamp_offset(const PagedParams &p, int s) {
    const int64_t o = p.q_offsets[s];
    return o < 0 ? 0 : (o > p.tokens ? p.tokens : o);
}

template <int ROWS>
__device__ __forceinline__ bool find_tile(const PagedParams &p, int tile, RowTile &t) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = p.seqs;
    while (n > 1) {                                            // 64-way search over a non-decreasing function
        const int step = (n + 63) / 64;
        const int s = lo + lane * step;
        const bool before = lane * step < n && clamp_offset(p, s) * p.group / ROWS + s <= tile;
        const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(before));
        const int skip = c > 0 ? (c - 1) * step : 0;
        lo += skip;
        n = min(step, n - skip);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const int64_t first = clamp_offset(p, lo), end = clamp_offset(p, lo + 1);
    const int64_t tile0 = first * p.group / ROWS + lo;
    t.seq = lo; t.first = (int)first; t.count = (int)(end - first);
    if (tile < tile0 || t.count <= 0) return false;
    const int64_t row0 = (tile - tile0) * ROWS, rows = (int64_t)t.count * p.group;
    if (row0 >= rows) return false;
    t.row0 = (int)row0;
    t.rows = (int)min((int64_t)ROWS, rows - row0);
    const int64_t most = (int64_t)p.table_cols * p.page_size;
    const int64_t kv = p.kv_lens[lo];
    t.kv_len = (int)(kv < 0 ? 0 : (kv > most ? most : kv));
    return true;
}

// keys [lo, hi) that the row of token i of a sequence sees
__device__ __forceinline__ void row_range(const PagedParams &p, const RowTile &t, int i, int &lo, int &hi) {
    const int place = t.kv_len - t.count + i;
    hi = p.causal ? min(t.kv_len, place + 1) : t.kv_len;
    lo = p.window > 0 ? max(0, place - p.window + 1) : 0;
    hi = max(hi, 0);
    lo = min(lo, hi);
}

// ---- up to sixteen rows: waves share the keys, operands straight into registers --------------------------------------------
// A wave takes steps of 32 keys.  K: the A operand of a 16-key tile is 16 bytes per lane of the cache rows as they lie (the
// channels' order inside the contraction is free, Q has the same).  V: a lane loads channels 8m.. (head dimension 128; 4m..
// for 64) of the eight keys whose probabilities it holds, and interleaving key pairs by v_perm turns them into the A operands
// of O^T: operand t has channel 8m + t in row m.  Nothing passes through LDS until the waves' results are joined.
constexpr int kRows = 16, kStep = 32, kWaves = 4;

template <int DT, bool C8, int DH>
__global__ __launch_bounds__(kWaves * 64) void paged_rows_kernel(const PagedParams p) {
    constexpr int NQ = DH / 32;                               // contraction steps of 32 channels
    constexpr int NT = DH / 16;                               // 16-channel tiles of the output
    constexpr int ND = DH / 32;                               // words of two channels that a lane holds of a V row
    constexpr int KL = C8 ? DH / 64 : DH / 32;                // 16-byte loads of a lane per K tile
    __shared__ __attribute__((aligned(16))) float part[kWaves][kRows][DH + 4];
    __shared__ float part_m[kWaves][kRows], part_l[kWaves][kRows];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, q4 = lane >> 4;
    const int split = blockIdx.x % p.splits;
    const int rest = blockIdx.x / p.splits;
    const int head = rest % p.kv_heads;
    RowTile t;
    if (!find_tile<kRows>(p, rest / p.kv_heads, t)) return;

    // this lane's row
    const int r = min(l16, t.rows - 1) + t.row0;
    const int tok = (int)divide(r, p.group_div), g = r - tok * p.group;
    int my_lo, my_hi, lo, hi, first_hi, last_lo;
    row_range(p, t, tok, my_lo, my_hi);
    {
        const int ta = (int)divide(t.row0, p.group_div), tb = (int)divide(t.row0 + t.rows - 1, p.group_div);
        row_range(p, t, ta, lo, first_hi);
        row_range(p, t, tb, last_lo, hi);
    }
    const int lowest = lo;
    lo &= ~(kStep - 1);
    const int all_steps = hi > lo ? (hi - lo + kStep - 1) / kStep : 0;
    const int per = (all_steps + p.splits - 1) / p.splits;
    const int step0 = split * per, step1 = min(all_steps, step0 + per);

    v4u qf[NQ];
    {
        const uint8_t *qr = p.q + ((int64_t)(t.first + tok) * p.q_ld + (int64_t)(head * p.group + g) * DH) * 2;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const int c = C8 ? ((i >> 1) * 4 + q4) * 16 + (i & 1) * 8 : (i * 4 + q4) * 8;
            qf[i] = *reinterpret_cast<const v4u *>(qr + c * 2);
        }
    }
    const int32_t *table = p.page_table + (int64_t)t.seq * p.table_stride;
    const u32 head_unit = (u32)head * p.head_units;

    v4f o[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) o[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, l = 0.0f;

    for (int st = step0 + wave; st < step1; st += kWaves) {
        const int key0 = lo + st * kStep;
        // each lane finds one key's row (the upper half repeats the lower)
        const int key = key0 + (lane & 31);
        u32 unit = head_unit;
        bool there = key >= lowest && key < hi;
        if (there) {
            const u32 pg = divide((u32)key, p.page_div);
            const u32 page = (u32)table[pg];
            there = page < p.pages;
            if (there) unit += page * p.page_units + ((u32)key - pg * p.page_size) * p.token_units;
        }
        const u32 seen = (u32)__builtin_amdgcn_ballot_w64(there);        // bit i: some row sees key0 + i, and it is in the cache
        v4u kf[2][KL];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            const u32 u = (u32)__shfl((int)unit, tt * 16 + l16);
            const uint8_t *row = p.k + (uint64_t)u * 16 + 16 * q4;
#pragma unroll
            for (int i = 0; i < KL; ++i) kf[tt][i] = *reinterpret_cast<const v4u *>(row + 64 * i);
        }
        u32 vw[8][ND];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const u32 u = (u32)__shfl((int)unit, (j >> 2) * 16 + 4 * q4 + (j & 3));
            if constexpr (C8) {
                const uint8_t *at = p.v + (uint64_t)u * 16 + l16 * (2 * ND);
                if constexpr (DH == 128) {
                    const uint2 w = *reinterpret_cast<const uint2 *>(at);
                    vw[j][0] = widen<DT, false>(w.x); vw[j][1] = widen<DT, true>(w.x);
                    vw[j][2] = widen<DT, false>(w.y); vw[j][3] = widen<DT, true>(w.y);
                } else {
                    const u32 w = *reinterpret_cast<const u32 *>(at);
                    vw[j][0] = widen<DT, false>(w); vw[j][1] = widen<DT, true>(w);
                }
            } else {
                const uint8_t *at = p.v + (uint64_t)u * 16 + l16 * (4 * ND);
                if constexpr (DH == 128) {
                    const v4u w = *reinterpret_cast<const v4u *>(at);
#pragma unroll
                    for (int i = 0; i < 4; ++i) vw[j][i] = w[i];
                } else {
                    const uint2 w = *reinterpret_cast<const uint2 *>(at);
                    vw[j][0] = w.x; vw[j][1] = w.y;
                }
            }
        }
        // scores: register i of tile tt is key 16 tt + 4 q4 + i of this lane's row
        float s[8];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            v4f a = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                v4u f;
                if constexpr (C8) {
                    const u32 w0 = kf[tt][i >> 1][(i & 1) * 2], w1 = kf[tt][i >> 1][(i & 1) * 2 + 1];
                    f[0] = widen<DT, false>(w0); f[1] = widen<DT, true>(w0);
                    f[2] = widen<DT, false>(w1); f[3] = widen<DT, true>(w1);
                } else {
                    f = kf[tt][i];
                }
                a = mfma16<DT>(f, qf[i], a);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s[4 * tt + i] = a[i] * p.scale_log2;
        }
        if (seen != 0xFFFFFFFFu || key0 < last_lo || key0 + kStep > first_hi) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = (i >> 2) * 16 + 4 * q4 + (i & 3);
                const bool on = ((seen >> at) & 1u) && key0 + at >= my_lo && key0 + at < my_hi;
                s[i] = on ? s[i] : -INFINITY;
            }
            // what is not in the cache must not reach the sums, not even times zero
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (!((seen >> ((j >> 2) * 16 + 4 * q4 + (j & 3))) & 1u)) {
#pragma unroll
                    for (int i = 0; i < ND; ++i) vw[j][i] = 0;
                }
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i]);
        top = fmaxf(m, max_quarters(top));
        const float base = top == -INFINITY ? 0.0f : top;
        const float alpha = __builtin_amdgcn_exp2f(m - base);
        m = top;
        float pr[8], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            pr[i] = __builtin_amdgcn_exp2f(s[i] - base);
            sum += pr[i];
        }
        l = fmaf(l, alpha, sum);
        v4u pf;
#pragma unroll
        for (int i = 0; i < 4; ++i) pf[i] = pack16bit<DT>(pr[2 * i], pr[2 * i + 1]);
#pragma unroll
        for (int i = 0; i < NT; ++i) o[i] *= alpha;
#pragma unroll
        for (int w = 0; w < ND; ++w) {
            v4u a, b;
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) {
                a[jj] = __builtin_amdgcn_perm(vw[2 * jj + 1][w], vw[2 * jj][w], 0x05040100u);
                b[jj] = __builtin_amdgcn_perm(vw[2 * jj + 1][w], vw[2 * jj][w], 0x07060302u);
            }
            o[2 * w] = mfma16<DT>(a, pf, o[2 * w]);
            o[2 * w + 1] = mfma16<DT>(b, pf, o[2 * w + 1]);
        }
    }
    l = sum_quarters(l);

    // join the waves: tile i, register r is channel NT * (4 q4 + r) + i of this lane's row
#pragma unroll
    for (int rr = 0; rr < 4; ++rr)
#pragma unroll
        for (int i = 0; i < NT; i += 4)
            *reinterpret_cast<v4f *>(&part[wave][l16][NT * (4 * q4 + rr) + i]) = v4f{o[i][rr], o[i + 1][rr], o[i + 2][rr], o[i + 3][rr]};
    if (q4 == 0) { part_m[wave][l16] = m; part_l[wave][l16] = l; }
    __syncthreads();
    constexpr int CH = DH / 16;                               // channels per thread: sixteen threads per row
    const int row = threadIdx.x >> 4, c = (threadIdx.x & 15) * CH;
    if (row >= t.rows) return;
    float best = part_m[0][row];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) best = fmaxf(best, part_m[w][row]);
    const float base = best == -INFINITY ? 0.0f : best;
    float total = 0.0f, y[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) y[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(part_m[w][row] - base);
        total = fmaf(part_l[w][row], f, total);
#pragma unroll
        for (int i = 0; i < CH; ++i) y[i] = fmaf(part[w][row][c + i], f, y[i]);
    }
    const float inv = total == 0.0f ? 0.0f : p.v_scale / total;
#pragma unroll
    for (int i = 0; i < CH; ++i) y[i] = total == 0.0f ? 0.0f : y[i] * inv;
    const int rr = t.row0 + row;
    const int token = t.first + (int)divide(rr, p.group_div);
    const int qh = head * p.group + rr - (int)divide(rr, p.group_div) * p.group;
    const int64_t at = (int64_t)token * p.q_heads + qh;
    const float lse2 = total == 0.0f ? -INFINITY : base + __builtin_amdgcn_logf(total);   // base 2
    if (p.splits > 1) {
        const int64_t slot = (int64_t)split * p.tokens * p.q_heads + at;
        if (c == 0) p.part_lse[slot] = lse2;
        if (total != 0.0f) {
#pragma unroll
            for (int i = 0; i < CH; i += 4) *reinterpret_cast<v4f *>(p.part + slot * DH + c + i) = v4f{y[i], y[i + 1], y[i + 2], y[i + 3]};
        }
    } else {
        if (c == 0 && p.lse) p.lse[at] = lse2 * 0x1.62e430p-1f;
        u32 w[CH / 2];
#pragma unroll
        for (int i = 0; i < CH / 2; ++i) w[i] = pack16bit<DT>(y[2 * i], y[2 * i + 1]);
        u32 *d = reinterpret_cast<u32 *>(p.out + ((int64_t)token * p.out_ld + (int64_t)qh * DH + c) * 2);
#pragma unroll
        for (int i = 0; i < CH / 2; i += 2) *reinterpret_cast<uint2 *>(d + i) = make_uint2(w[i], w[i + 1]);
    }
}

// ---- joins the splits of a row: a weighted mean with weights exp2(lse_split - the largest) --------------------------------
template <int DT, int DH>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedParams p) {
    constexpr int CH = DH / 16;
    const int64_t rows = p.tokens * p.q_heads;
    const int64_t at = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (at >= rows) return;
    const int64_t token = at / p.q_heads;
    if (token < clamp_offset(p, 0) || token >= clamp_offset(p, p.seqs)) return;      // a row outside every sequence
    const int c = (threadIdx.x & 15) * CH;
    float best = -INFINITY;
    for (int s = 0; s < p.splits; ++s) best = fmaxf(best, p.part_lse[s * rows + at]);
    const float base = best == -INFINITY ? 0.0f : best;
    float total = 0.0f, y[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) y[i] = 0.0f;
    for (int s = 0; s < p.splits; ++s) {
        const float lse = p.part_lse[s * rows + at];
        if (lse == -INFINITY) continue;                          // nothing was written for it
        const float f = __builtin_amdgcn_exp2f(lse - base);
        total += f;
        const float *src = p.part + (s * rows + at) * DH + c;
#pragma unroll
        for (int i = 0; i < CH; i += 4) {
            const v4f v = *reinterpret_cast<const v4f *>(src + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) y[i + j] = fmaf(v[j], f, y[i + j]);
        }
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    if (c == 0 && p.lse) p.lse[at] = total == 0.0f ? -INFINITY : (base + __builtin_amdgcn_logf(total)) * 0x1.62e430p-1f;
    u32 w[CH / 2];
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) w[i] = pack16bit<DT>(y[2 * i] * inv, y[2 * i + 1] * inv);
    u32 *d = reinterpret_cast<u32 *>(p.out + (token * p.out_ld + (at - token * p.q_heads) * DH + c) * 2);
#pragma unroll
    for (int i = 0; i < CH / 2; i += 2) *reinterpret_cast<uint2 *>(d + i) = make_uint2(w[i], w[i + 1]);
}

template <int DT, bool C8, int DH>
hipError_t launch(PagedParams &p, int64_t max_kv, hipStream_t stream) {
    const int64_t tiles = p.tokens * p.group / kRows + p.seqs;
    hipLaunchKernelGGL((paged_rows_kernel<DT, C8, DH>), dim3((u32)(tiles * p.kv_heads * p.splits)), dim3(kWaves * 64), 0, stream, p);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.splits > 1) {
        hipLaunchKernelGGL((paged_join_kernel<DT, DH>), dim3((u32)((p.tokens * p.q_heads + 15) / 16)), dim3(256), 0, stream, p);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

int paged_splits(int64_t tokens, int seqs, int q_heads, int kv_heads, int head_dim, int64_t max_kv) {
    const int64_t tiles = tokens * (q_heads / kv_heads) / kRows + seqs;
    // enough workgroups for the chip, each with at least two steps per wave
    const int64_t want = (1024 + tiles * kv_heads - 1) / (tiles * kv_heads);
    const int64_t most = max_kv / (kWaves * kStep * 2);
    int64_t s = want < most ? want : most;
    return s < 1 ? 1 : (s > 64 ? 64 : (int)s);
}

hipError_t paged_launch(PagedParams p, int dtype, int cache_dtype, int head_dim, int64_t max_kv, hipStream_t stream) {
    const bool c8 = cache_dtype == kE4M3;
#define VITQ_PAGED(DT) \
    if (head_dim == 64) return c8 ? launch<DT, true, 64>(p, max_kv, stream) : launch<DT, false, 64>(p, max_kv, stream); \
    return c8 ? launch<DT, true, 128>(p, max_kv, stream) : launch<DT, false, 128>(p, max_kv, stream);
    if (dtype == kBF16) { VITQ_PAGED(kBF16) }
    VITQ_PAGED(kF16)
#undef VITQ_PAGED
}

}  // namespace vitq
