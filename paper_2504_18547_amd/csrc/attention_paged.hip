// Attention of new tokens over a paged cache: softmax(scale q.k) v per query head, one pass over the keys with the running
// maximum and sum of the softmax, on 16-bit MFMAs.
//
// The rows of a sequence and a key-value head are its new tokens times the query heads that share the head: row r is token
// r / group, head r % group of the group, so a cache row is read once for all of them.  Scores are computed transposed
// (S^T = K Q^T): a lane of the result holds keys of ONE row, the softmax statistics are per lane, and the probabilities are
// already the B operand of O^T = V^T P^T, whose order of keys is that of the score registers.
#include "attention_paged.h"

#include <algorithm>

#include "launch_util.h"
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

// Probabilities are exp2(score - base), and in half precision base lies this far below the largest score (in powers of two): what is
// far below the largest keeps 2^-39 of it (rows kernel; 2^-31 at least in the tiles kernel, whose base lags) instead of 2^-24, which
// counts where many such keys stand beside a strong one.  The sums carry the same factor, so it falls out by itself.
template <int DT>
constexpr float kLiftRows = DT == kF16 ? 15.0f : 0.0f;        // 2^15: half precision ends at 65504
constexpr float kLag = 8.0f;                                  // by how much a row's largest score may pass base + lift in the tiles kernel
template <int DT>
constexpr float kLiftTiles = DT == kF16 ? 15.0f - kLag : 0.0f;

// Zeroes the halves of w that are not finite; not 0 if there was one.  (Adding one to an exponent of all ones sets the sign bit
// alone, and twice a sign bit minus itself shifted to the bottom is a half of ones.)
template <int DT>
__device__ __forceinline__ u32 strip(u32 &w) {
    constexpr u32 kExp = DT == kBF16 ? 0x7F807F80u : 0x7C007C00u, kOne = DT == kBF16 ? 0x00800080u : 0x04000400u;
    const u32 odd = ((w & kExp) + kOne) & 0x80008000u;
    w &= ~((odd << 1) - (odd >> 15));
    return odd;
}
// The same for four E4M3 codes, whose one NaN is 0x7F with either sign.
__device__ __forceinline__ u32 strip_codes(u32 &w) {
    const u32 odd = ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
    w &= ~((odd << 1) - (odd >> 7));
    return odd;
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

// false: no such tile, or its sequence belongs to the other form (FEW: up to p.few_rows rows)
template <int ROWS, bool FEW>
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
    if (row0 >= rows || (rows <= p.few_rows) != FEW) return false;
    t.row0 = (int)row0;
    t.rows = (int)min((int64_t)ROWS, rows - row0);
    const int64_t most = (int64_t)p.table_cols * p.page_size;
    const int64_t kv = p.kv_lens[lo];
    t.kv_len = (int)(kv < 0 ? 0 : (kv > most ? most : kv));
    return true;
}

// Infinities and NaN among the values of keys that some rows of a tile see and others do not: zero times them is not zero, so the
// products of such steps go without them (strip), and where there was one the rows that see its key get it afterwards, here.
// add(row): the lane's channels of the cache row whose key its row sees.
template <class F>
__device__ __forceinline__ void give_back(const PagedParams &p, const int32_t *table, u32 head_unit, int key0, int count, int my_lo, u32 my_span, F &&add) {
#pragma unroll 1
    for (int key = key0; key < key0 + count; ++key) {
        if ((u32)(key - my_lo) >= my_span) continue;
        const u32 pg = divide((u32)key, p.page_div), page = (u32)table[pg];
        if (page < p.pages) add(p.v + (uint64_t)(head_unit + page * p.page_units + ((u32)key - pg * p.page_size) * p.token_units) * 16);
    }
}
template <int DT, bool C8>
__device__ __forceinline__ float odd_value(const uint8_t *row, int c) {       // the channel if it is not finite, or 0
    if constexpr (C8) return (row[c] & 0x7F) == 0x7F ? __builtin_nanf("") : 0.0f;
    else {
        const float v = load1<DT>(row, c);
        return fabsf(v) < INFINITY ? 0.0f : v;
    }
}

// Which tile, head and split a workgroup has.  Workgroups go round-robin to the eight XCDs, each with an L2 of its own.
// RUNS: one XCD has a run of consecutive tiles of one head and split, which share keys; the last tiles, which see most under a
// causal mask, start first.  Else splits, then heads, then tiles: evenly spread whatever the lengths (and tiles of one sequence are
// a multiple of eight apart where heads or splits are).
template <bool RUNS>
__device__ __forceinline__ int tile_of_block(const PagedParams &p, int &head, int &split) {
    // (the divisions run on the vector unit: back to scalars)
    const int block = blockIdx.x;
    if constexpr (!RUNS) {
        const int rest = __builtin_amdgcn_readfirstlane(block / p.splits), tile = __builtin_amdgcn_readfirstlane(rest / p.kv_heads);
        split = block - rest * p.splits;
        head = rest - tile * p.kv_heads;
        return tile;
    } else {
        const int total = gridDim.x, xcd = block & 7, slot = block >> 3, per = total >> 3, rem = total & 7;
        const int id = (xcd < rem ? xcd * (per + 1) : rem * (per + 1) + (xcd - rem) * per) + slot;
        const int unit = __builtin_amdgcn_readfirstlane(id / p.row_tiles);
        split = __builtin_amdgcn_readfirstlane(unit / p.kv_heads);
        head = unit - split * p.kv_heads;
        return p.row_tiles - 1 - (id - unit * p.row_tiles);
    }
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
// Bound by HBM: 64 x 8,192 keys of 8 heads of 128 in bf16 362-367 us, 5.9 TB/s; in E4M3 with lengths of 1 to 8,192 122 us, 4.6 TB/s
// (the widening and the unequal lengths); a step's operands requested while the step before is worked on took 10 % off both.
// Waves a SIMD: as many as the registers give without spills.  64 channels of 16 bits forced to four spill 20-92 bytes: single tokens,
// 64 x 4,096 keys of 4 heads, 66-77 us against 61; a chunk of 511 rows among single tokens 48-67 against 50.
constexpr int kRows = 16, kStep = 32, kWaves = 4;

template <int DT, bool C8, int DH>
__global__ __launch_bounds__(kWaves * 64, (DH == 64 ? 3 : 2) + (C8 ? 1 : 0)) void paged_rows_kernel(const PagedParams p) {
    constexpr int NQ = DH / 32;                               // contraction steps of 32 channels
    constexpr int NT = DH / 16;                               // 16-channel tiles of the output
    constexpr int ND = DH / 32;                               // words of two channels that a lane holds of a V row
    constexpr int KL = C8 ? DH / 64 : DH / 32;                // 16-byte loads of a lane per K tile
    __shared__ __attribute__((aligned(16))) float part[kWaves][kRows][DH + 4];
    __shared__ float part_m[kWaves][kRows], part_l[kWaves][kRows];
    __shared__ int part_odd[kWaves];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, q4 = lane >> 4;
    int head, split;
    const int tile = tile_of_block<false>(p, head, split);
    RowTile t;
    if (!find_tile<kRows, true>(p, tile, t)) return;

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
    const u32 my_span = (u32)(my_hi - my_lo);
    lo &= ~(kStep - 1);
    const int all_steps = hi > lo ? (hi - lo + kStep - 1) / kStep : 0;
    const int step0 = split * (p.split_keys / kStep), step1 = split + 1 == p.splits ? all_steps : min(all_steps, step0 + p.split_keys / kStep);

    v4u qf[NQ];
    {
        const uint8_t *qr = p.q + ((int64_t)(t.first + tok) * p.q_ld + (int64_t)(head * p.group + g) * DH) * 2;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const int c = C8 ? ((i >> 1) * 4 + q4) * 16 + (i & 1) * 8 : (i * 4 + q4) * 8;
            qf[i] = *reinterpret_cast<const v4u *>(qr + c * 2);
            if (p.negative) qf[i] ^= 0x80008000u;
        }
    }
    const int32_t *table = p.page_table + (int64_t)t.seq * p.table_stride;
    const u32 head_unit = (u32)head * p.head_units;

    v4f o[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) o[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, l = 0.0f;
    const bool uneven = last_lo > lowest || first_hi < hi;        // the rows do not all see the same keys
    auto partly = [&](int st) { const int key0 = lo + st * kStep; return key0 < last_lo || key0 + kStep > first_hi; };
    u32 odd = 0;

    // A step's operands as they lie in the cache.  They are requested a step before they are used, and their page numbers a step
    // before that: a wave has one step's keys and values in flight while it works on another's.
    typedef u32 VRow __attribute__((ext_vector_type(C8 ? ND / 2 : ND)));
    struct Operands { v4u k[2][KL]; VRow v[8]; u32 seen; };    // bit i of seen: some row sees key i of the step, and it is in the cache
    u32 asked_page = ~0u, asked_place = ~0u;
    // (each lane looks after one key; the upper half repeats the lower)
    auto ask = [&](int st) {
        const int key = lo + st * kStep + (lane & 31);
        const bool want = st < step1 && key >= lowest && key < hi;
        const u32 pg = divide((u32)(want ? key : lowest), p.page_div);
        asked_page = (u32)table[pg];                          // (some page of this sequence where the lane has no key)
        asked_place = want ? (u32)key - pg * p.page_size : ~0u;
    };
    auto fetch = [&](Operands &x) {
        const bool there = asked_place != ~0u && asked_page < p.pages;
        const u32 unit = head_unit + (there ? asked_page * p.page_units + asked_place * p.token_units : 0u);
        x.seen = (u32)__builtin_amdgcn_ballot_w64(there);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            const u32 u = (u32)__shfl((int)unit, tt * 16 + l16);
            const uint8_t *row = p.k + (uint64_t)u * 16 + 16 * q4;
#pragma unroll
            for (int i = 0; i < KL; ++i) x.k[tt][i] = *reinterpret_cast<const v4u *>(row + 64 * i);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const u32 u = (u32)__shfl((int)unit, (j >> 2) * 16 + 4 * q4 + (j & 3));
            x.v[j] = *reinterpret_cast<const VRow *>(p.v + (uint64_t)u * 16 + l16 * sizeof(VRow));
        }
    };
    auto work = [&](Operands &x, int st) {
        const int key0 = lo + st * kStep;
        // scores: register i of tile tt is key 16 tt + 4 q4 + i of this lane's row
        float s[8];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            v4f a = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                v4u f;
                if constexpr (C8) f = widen8<DT>(x.k[tt][i >> 1][(i & 1) * 2], x.k[tt][i >> 1][(i & 1) * 2 + 1]);
                else f = x.k[tt][i];
                a = mfma16<DT>(f, qf[i], a);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s[4 * tt + i] = a[i] * p.scale_log2;
        }
        if (x.seen != 0xFFFFFFFFu || partly(st)) {
            const u32 mine = x.seen >> (4 * q4);
            const int first = key0 + 4 * q4 - my_lo;              // this lane's key 0 against what its row sees
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = (i >> 2) * 16 + (i & 3);
                const bool there = (mine & (1u << at)) != 0;
                s[i] = there && (u32)(first + at) < my_span ? s[i] : -INFINITY;
                // what is not in the cache must not reach the sums, not even times zero
                if (!there) x.v[i] = 0;
            }
            if (uneven && partly(st)) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int w = 0; w < (C8 ? ND / 2 : ND); ++w) {
                        u32 v = x.v[i][w];
                        odd |= C8 ? strip_codes(v) : strip<DT>(v);
                        x.v[i][w] = v;
                    }
            }
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i]);
        top = fmaxf(m, max_quarters(top) - kLiftRows<DT>);
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
            u32 row[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (C8) row[j] = (w & 1) ? widen<DT, true>(x.v[j][w >> 1]) : widen<DT, false>(x.v[j][w >> 1]);
                else row[j] = x.v[j][w];
            }
            v4u a, b;
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) {
                a[jj] = __builtin_amdgcn_perm(row[2 * jj + 1], row[2 * jj], 0x05040100u);
                b[jj] = __builtin_amdgcn_perm(row[2 * jj + 1], row[2 * jj], 0x07060302u);
            }
            o[2 * w] = mfma16<DT>(a, pf, o[2 * w]);
            o[2 * w + 1] = mfma16<DT>(b, pf, o[2 * w + 1]);
        }
    };
    {
        int st = step0 + wave;
        if (st < step1) {
            Operands x, y;
            ask(st);
            fetch(x);
            ask(st + kWaves);
            for (; st < step1; st += 2 * kWaves) {
                if (st + kWaves < step1) fetch(y);
                ask(st + 2 * kWaves);
                work(x, st);
                if (st + kWaves >= step1) break;
                if (st + 2 * kWaves < step1) fetch(x);
                ask(st + 3 * kWaves);
                work(y, st + kWaves);
            }
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
    const bool any_odd = __builtin_amdgcn_ballot_w64(odd != 0) != 0;
    if (lane == 0) part_odd[wave] = any_odd;
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
    if (part_odd[0] | part_odd[1] | part_odd[2] | part_odd[3]) {
        int row_lo, row_hi;
        row_range(p, t, (int)divide(rr, p.group_div), row_lo, row_hi);
        for (int st = step0; st < step1; ++st) {
            if (!partly(st)) continue;
            give_back(p, table, head_unit, lo + st * kStep, kStep, row_lo, (u32)(row_hi - row_lo), [&](const uint8_t *v) {
#pragma unroll
                for (int i = 0; i < CH; ++i) y[i] += odd_value<DT, C8>(v, c + i);
            });
        }
    }
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

// ---- many rows: 32 rows per wave, keys through LDS -------------------------------------------------------------------------
// A workgroup's eight waves have 32 rows each and share steps of 64 keys, K and V each in two LDS buffers.  16-bit caches go there
// straight from memory, E4M3 ones are widened on the way.  Scores: A = K rows from LDS, B = Q in registers.  O^T: A = V^T by the
// transposing LDS read, four keys of one channel per lane, in the order in which the score registers hold the keys; B = P^T.
// LDS rows are unpadded with their 16-byte chunks permuted by the row: K's so that 16 rows' equal chunks cover all banks, V's so
// that four rows' 64-byte pieces do.
// 2 x 2,048 tokens over 8,192 keys, 32 / 8 heads of 128: 442-450 us, 1.07-1.09 PFLOP/s of the 1.43 that a large bf16 library product
// reaches on this card (3 % of the time keeps infinities and NaN from rows that do not see their keys); the matrix cores are busy 57 % of the time, the rest goes to the issue of what stands between their
// instructions (no loads: 391, no exponentials: 410).  Left out: steps of 32 keys (535), with them three waves a SIMD (535), the
// exponentials of one step among the score products of the next in one wave (504, registers spill).

template <int DT>
__device__ __forceinline__ v16f mfma32(const v4u &a, const v4u &b, const v16f &c) {
    if constexpr (DT == kBF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}
__device__ __forceinline__ float max_halves(float v) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ u32 lds_address_of(const void *p) {
    return (u32)(uintptr_t)(const __attribute__((address_space(3))) uint8_t *)p;
}
// 16 bytes per lane straight to LDS (dst + 16 * lane); waited for with vmcnt by hand.  (Nothing else here uses M0.)
__device__ __forceinline__ void to_lds16(u32 off, const uint8_t *base, u32 dst) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(off), "s"(base), "s"(dst) : "memory");
}
__device__ __forceinline__ void to_lds16_ptr(const uint8_t *src, u32 dst) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" :: "v"(src), "s"(dst) : "memory");
}
__device__ __attribute__((aligned(16))) const u32 g_no_key[4] = {0u, 0u, 0u, 0u};

template <int DT, bool C8, int DH, int W>
__global__ __launch_bounds__(W * 64, 2) void paged_tiles_kernel(const PagedParams p) {
    constexpr int kTileKeys = 64;
    constexpr int RB = DH * 2;                                // bytes of an LDS row
    constexpr int kBuf = kTileKeys * RB;                      // K or V of a step
    constexpr int NQ = DH / 16, ND = DH / 32;
    constexpr int kBytes = C8 && DH == 64 ? 8 : 16;           // that a lane loads at a time
    constexpr int kRowsPerLoad = 64 * kBytes / (C8 ? DH : RB);      // rows that a wave's load instruction covers
    constexpr int kLoads = kTileKeys / W / kRowsPerLoad;      // per wave, for K and again for V
    constexpr int kTileRows = 32 * W;
    static_assert(kLoads > 0 && kRowsPerLoad <= 16, "every wave loads whole rows");
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];       // K0 K1 V0 V1, a flag
    int *odd = reinterpret_cast<int *>(smem + 4 * kBuf);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, h = lane >> 5;

    int head, split;
    const int tile = tile_of_block<true>(p, head, split);
    RowTile t;
    if (!find_tile<kTileRows, false>(p, tile, t)) return;

    // this lane's row, and what the wave's rows see
    const int wave_rows = min(32, t.rows - 32 * wave);        // may be <= 0: the wave only helps to load
    const int r = t.row0 + min(32 * wave + l32, t.rows - 1);
    const int tok = (int)divide(r, p.group_div), g = r - tok * p.group;
    int my_lo, my_hi, lo, hi, first_hi, last_lo, w_lo, w_hi, w_first_hi, w_last_lo;
    row_range(p, t, tok, my_lo, my_hi);
    row_range(p, t, (int)divide(t.row0, p.group_div), lo, first_hi);
    row_range(p, t, (int)divide(t.row0 + t.rows - 1, p.group_div), last_lo, hi);
    {
        const int ra = t.row0 + min(32 * wave, t.rows - 1), rb = t.row0 + min(32 * wave + 31, t.rows - 1);
        row_range(p, t, (int)divide(ra, p.group_div), w_lo, w_first_hi);
        row_range(p, t, (int)divide(rb, p.group_div), w_last_lo, w_hi);
    }
    const u32 my_span = (u32)(my_hi - my_lo);
    const int lowest = lo;
    lo &= ~(kTileKeys - 1);
    const int all_steps = hi > lo ? (hi - lo + kTileKeys - 1) / kTileKeys : 0;
    const int step0 = split * (p.split_keys / kTileKeys), step1 = split + 1 == p.splits ? all_steps : min(all_steps, step0 + p.split_keys / kTileKeys);

    // Q: channels 16 i + 8 h .. of this lane's row; a negative scale is a sign of the queries (maxima are taken before scaling)
    v4u qf[NQ];
    {
        const uint8_t *qr = p.q + ((int64_t)(t.first + tok) * p.q_ld + (int64_t)(head * p.group + g) * DH) * 2;
        const u32 flip = p.negative ? 0x80008000u : 0u;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            qf[i] = *reinterpret_cast<const v4u *>(qr + (16 * i + 8 * h) * 2);
#pragma unroll
            for (int j = 0; j < 4; ++j) qf[i][j] ^= flip;
        }
    }
    const int32_t *table = p.page_table + (int64_t)t.seq * p.table_stride;
    const u32 head_unit = (u32)head * p.head_units;
    const u32 lds0 = (u32)__builtin_amdgcn_readfirstlane((int)lds_address_of(smem));

    // The cache row of key (first key of the step) + lane, in units of 16 bytes, ~0 where there is none.  Its page number is
    // requested a step before it is looked at: between the two all loads are waited for anyway.
    u32 asked_page = ~0u, asked_place = 0;
    auto ask = [&](int st) {
        const int key = lo + st * kTileKeys + lane;
        const bool want = st < step1 && key >= lowest && key < hi;
        const u32 pg = divide((u32)(want ? key : lowest), p.page_div);
        asked_page = (u32)table[pg];                          // (some page of this sequence where the lane has no key)
        asked_place = want ? (u32)key - pg * p.page_size : ~0u;
    };
    auto answer = [&]() -> u32 {
        return asked_place != ~0u && asked_page < p.pages ? head_unit + asked_page * p.page_units + asked_place * p.token_units : ~0u;
    };
    // Which row and chunk of the step this lane loads: row0 + kNext n for load n.  kNext is a multiple of what the permutations of
    // the chunks look at, so they are the same for every n.
    constexpr int kLanes = 64 / kRowsPerLoad, kNext = W * kRowsPerLoad;
    const int row0 = wave * kRowsPerLoad + lane / kLanes, lc = lane % kLanes;
    typedef u32 Stage __attribute__((ext_vector_type(kBytes / 4)));
    Stage stage_k[C8 ? kLoads : 1], stage_v[C8 ? kLoads : 1];
    auto k_swizzle = [](int row) { return DH == 128 ? row & 15 : (row >> 1) & 7; };
    auto v_swizzle = [](int row) { return DH == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; };
    // The rows of a load instruction lie in one page wherever pages are multiples of sixteen tokens: then their place is a scalar
    // and a constant per lane.  A step with keys that do not exist, or other page sizes: one address per lane, zeros for no key.
    const u32 k_lane = (u32)(lane / kLanes) * p.token_units * 16u + (u32)(C8 ? lc : lc ^ k_swizzle(row0)) * kBytes;
    const u32 v_lane = (u32)(lane / kLanes) * p.token_units * 16u + (u32)(C8 ? lc : lc ^ v_swizzle(row0)) * kBytes;
    // (rows of a step, `all`: none is missing, into buffer `buf`; E4M3 into registers first)
    auto load = [&](u32 unit, bool all, int buf, auto IsV) {
        constexpr bool is_v = decltype(IsV)::value;
        const u32 dst0 = lds0 + (u32)((is_v ? 2 * kBuf : 0) + buf * kBuf + wave * kRowsPerLoad * RB);
        const uint8_t *cache = is_v ? p.v : p.k;
        const u32 in_lane = is_v ? v_lane : k_lane;
        if (all && p.whole_rows) {
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                const uint8_t *row = cache + (uint64_t)(u32)__builtin_amdgcn_readlane((int)unit, wave * kRowsPerLoad + kNext * n) * 16;
                if constexpr (C8) (is_v ? stage_v : stage_k)[n] = *reinterpret_cast<const Stage *>(row + in_lane);
                else to_lds16(in_lane, row, dst0 + n * (kNext * RB));
            }
        } else {
            const u32 in_row = in_lane - (u32)(lane / kLanes) * p.token_units * 16u;
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                const u32 u = (u32)__builtin_amdgcn_ds_bpermute(4 * row0 + 4 * kNext * n, (int)unit);
                const uint8_t *src = u != ~0u ? cache + (uint64_t)u * 16 + in_row : reinterpret_cast<const uint8_t *>(g_no_key);
                if constexpr (C8) (is_v ? stage_v : stage_k)[n] = *reinterpret_cast<const Stage *>(src);
                else to_lds16_ptr(src, dst0 + n * (kNext * RB));
            }
        }
    };
    auto widen_to_lds = [&](int buf, auto IsV) {              // E4M3: eight channels are a chunk
        constexpr bool is_v = decltype(IsV)::value;
        constexpr int chunks = kBytes / 8;
        uint8_t *row = smem + (is_v ? 2 * kBuf : 0) + buf * kBuf + row0 * RB;
        const int chunk = ((chunks * lc) ^ (is_v ? v_swizzle(row0) : k_swizzle(row0))) * 16;
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const Stage &w = (is_v ? stage_v : stage_k)[n];
#pragma unroll
            for (int e = 0; e < chunks; ++e) *reinterpret_cast<v4u *>(row + kNext * n * RB + (chunk ^ (16 * e))) = widen8<DT>(w[2 * e], w[2 * e + 1]);
        }
    };
    const std::integral_constant<bool, false> K;
    const std::integral_constant<bool, true> V;

    // LDS offsets of this lane's pieces: K row l32 (+32), chunk 2 i + h; V rows 4 h + (lane % 16) / 4 (+8, +16 ...), channels
    // 32 d + 16 ((lane / 16) % 2) + 4 (lane % 4) ..
    const int vrow = 4 * h + ((lane >> 2) & 3);
    const int vchunk = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
    auto v_offset = [&](int d) { return (u32)(vrow * RB + (((4 * d + vchunk) ^ v_swizzle(vrow)) * 16) + (lane & 1) * 8); };

    v16f o[ND], s[2];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    float m = -INFINITY, l = 0.0f;
    const float c = p.scale_log2;
    v4u pf[4];                                                // probabilities: group e is keys 16 e .. of the step

    // Products with the operands read kAhead ahead.  Product n of the output: keys 16 (n / ND) .., channels 32 (n % ND) ..; product
    // n of the scores: key tile n % 2, channels 16 (n / 2) ..
    constexpr int kAhead = 4, kOut = 4 * ND, kScore = 2 * NQ;
    auto v_read = [&](const uint8_t *vb, int n) {
        typedef short v4s __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) v4s *lds_v4s;
        const uint8_t *at = vb + 16 * (n / ND) * RB + v_offset(n % ND);
        // (rows 8 further: the chunk permutation depends on the row modulo 4 only)
        const v4s a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(uintptr_t)lds_address_of(at));
        const v4s a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(uintptr_t)lds_address_of(at + 8 * RB));
        const uint2 u0 = __builtin_bit_cast(uint2, a0), u1 = __builtin_bit_cast(uint2, a1);
        return v4u{u0.x, u0.y, u1.x, u1.y};
    };
    auto k_read = [&](const uint8_t *kb, int n) {
        const int row = 32 * (n & 1) + l32;
        return *reinterpret_cast<const v4u *>(kb + row * RB + (((2 * (n >> 1) + h) ^ k_swizzle(row)) * 16));
    };
    // the products of a step: the output of the step before (OUT), then the scores of this one (SCORE)
    auto products = [&](auto Out, auto Score, const uint8_t *vb, const uint8_t *kb) {
        constexpr int outs = decltype(Out)::value ? kOut : 0, all = outs + (decltype(Score)::value ? kScore : 0);
        v4u f[kAhead];
        auto read = [&](auto N) {
            constexpr int n = decltype(N)::value;
            if constexpr (n < outs) f[n % kAhead] = v_read(vb, n);
            else f[n % kAhead] = k_read(kb, n - outs);
        };
        static_for<kAhead>(read);
        __builtin_amdgcn_s_setprio(1);                        // ahead of the other group's softmax
        if constexpr (decltype(Score)::value) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[0][i] = s[1][i] = 0.0f;
        }
        __builtin_amdgcn_sched_barrier(0);
        static_for<all>([&](auto N) {
            constexpr int n = decltype(N)::value;
            if constexpr (n < outs) o[n % ND] = mfma32<DT>(f[n % kAhead], pf[n / ND], o[n % ND]);
            else s[(n - outs) & 1] = mfma32<DT>(f[n % kAhead], qf[(n - outs) >> 1], s[(n - outs) & 1]);
            if constexpr (n + kAhead < all) read(std::integral_constant<int, n + kAhead>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        __builtin_amdgcn_s_setprio(0);
    };
    // from the scores of step `st` to its probabilities.  Register i of tile kt is key 32 kt + 8 (i / 4) + 4 h + i % 4.
    auto softmax = [&](int st, uint64_t seen) {
        const int key0 = lo + st * kTileKeys;
        if (~seen != 0 || key0 < w_last_lo || key0 + kTileKeys > w_first_hi) {
            const int first = key0 + 4 * h - my_lo;               // this lane's key 0 against what its row sees
            const uint64_t mine = seen >> (4 * h);
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const u32 there = (u32)(mine >> (32 * kt));
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int at = 8 * (i >> 2) + (i & 3);
                    const bool on = (there & (1u << at)) != 0 && (u32)(first + 32 * kt + at) < my_span;
                    s[kt][i] = on ? s[kt][i] : -INFINITY;
                }
            }
        }
        asm volatile("" : "+v"(s[0]), "+v"(s[1]));            // both ways end in the same registers
        float top = s[0][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[0][i]);
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[1][i]);
        top = max_halves(top) * c - kLiftTiles<DT>;
        // The base of the exponents follows the largest score only when that has passed it by kLag: rescaling the sums in every step
        // costs as much as a quarter of the exponentials.  The largest probability is then rounded to 16 bits like the others (with a
        // base that follows at once it is a power of two): over 8,192 random keys a bf16 result is off by 0.00234 of its norm instead of
        // 0.00228, its own rounding among it.
        if (__builtin_amdgcn_ballot_w64(top > m + kLag) != 0) {
            const float now = fmaxf(m, top);
            const float alpha = __builtin_amdgcn_exp2f(m - (now == -INFINITY ? 0.0f : now));
            m = now;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
        }
        const float base = m == -INFINITY ? 0.0f : m;
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float a = __builtin_amdgcn_exp2f(fmaf(s[kt][i], c, -base)), b = __builtin_amdgcn_exp2f(fmaf(s[kt][i + 1], c, -base));
                sum[0] += a;
                sum[1] += b;
                pf[2 * kt + (i >> 3)][(i >> 1) & 3] = pack16bit<DT>(a, b);
            }
        l += sum[0] + sum[1];
    };

    // Two groups of waves, four each, one wave of either on every SIMD, half a step apart: while one group multiplies, the other
    // has its softmax, so that the matrix cores and the vector unit work side by side.  A barrier ends each half.  With the first
    // group's products of step j begin the loads of the keys of step j + 1 and the values of step j (everybody is past the
    // buffers that they go to); they are waited for before the half in which the first group needs them.
    const int steps = step1 - step0;
    const bool second = wave >= W / 2, works = wave_rows > 0;      // (a wave without rows only helps to load)
    u32 unit = ~0u;                                           // rows of the step whose values are loaded next
    uint64_t seen = 0, seen_before = 0;
    auto issue = [&](int j) {                                  // keys of step j + 1, values of step j
        const u32 next = answer();
        ask(step0 + j + 2);
        seen_before = seen;
        seen = __builtin_amdgcn_ballot_w64(next != ~0u);
        if (j + 1 < steps) load(next, ~seen == 0, (j + 1) & 1, K);
        load(unit, ~seen_before == 0, j & 1, V);
        unit = next;
    };
    const bool uneven = last_lo > lowest || first_hi < hi;               // the rows of the tile do not all see the same keys
    auto partly = [&](int j) { const int key0 = lo + (step0 + j) * kTileKeys; return key0 < last_lo || key0 + kTileKeys > first_hi; };
    auto arrive = [&](int j) {                                 // ends the half before the products of step j + 1
        if constexpr (C8) {
            if (j + 1 < steps) widen_to_lds((j + 1) & 1, K);
            widen_to_lds(j & 1, V);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        if (uneven && partly(j)) {                            // the wave's own rows of the values
#pragma unroll
            for (int n = 0; n < kLoads; ++n)
#pragma unroll
                for (int i = 0; i < kRowsPerLoad * RB / 1024; ++i) {
                    v4u *at = reinterpret_cast<v4u *>(smem + (2 + (j & 1)) * kBuf + (kNext * n + wave * kRowsPerLoad) * RB + i * 1024 + lane * 16);
                    v4u w = *at;
                    u32 found = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) { u32 x = w[e]; found |= strip<DT>(x); w[e] = x; }
                    if (found != 0) { *at = w; *odd = 1; }
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    };
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
    };
    const std::integral_constant<bool, true> yes;
    const std::integral_constant<bool, false> no;
    if (threadIdx.x == 0) *odd = 0;                           // (waited for before the first barrier, which is ahead of its first use)
    if (steps > 0) {
        ask(step0);
        unit = answer();
        ask(step0 + 1);
        seen = __builtin_amdgcn_ballot_w64(unit != ~0u);
        load(unit, ~seen == 0, 0, K);
        if constexpr (C8) {
            widen_to_lds(0, K);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");      // the keys, and the flag's zero
        }
        barrier();
        if (second) {
            issue(0);
            barrier();
            if (works) products(no, yes, nullptr, smem);
            arrive(0);
            barrier();
            for (int j = 1; j < steps; ++j) {
                const uint64_t now = seen_before;
                issue(j);
                if (works) softmax(step0 + j - 1, now);
                barrier();
                if (works) products(yes, yes, smem + (2 + ((j - 1) & 1)) * kBuf, smem + (j & 1) * kBuf);
                arrive(j);
                barrier();
            }
            if (works) {
                softmax(step0 + steps - 1, seen_before);
                products(yes, no, smem + (2 + ((steps - 1) & 1)) * kBuf, nullptr);
            }
        } else {
            issue(0);
            if (works) products(no, yes, nullptr, smem);
            barrier();
            for (int j = 1; j < steps; ++j) {
                if (works) softmax(step0 + j - 1, seen_before);
                arrive(j - 1);
                barrier();
                issue(j);
                if (works) products(yes, yes, smem + (2 + ((j - 1) & 1)) * kBuf, smem + (j & 1) * kBuf);
                barrier();
            }
            if (works) softmax(step0 + steps - 1, seen_before);
            arrive(steps - 1);
            barrier();
            if (works) products(yes, no, smem + (2 + ((steps - 1) & 1)) * kBuf, nullptr);
        }
        if (uneven && works && *odd) {
            for (int j = 0; j < steps; ++j) {
                if (!partly(j)) continue;
                give_back(p, table, head_unit, lo + (step0 + j) * kTileKeys, kTileKeys, my_lo, my_span, [&](const uint8_t *row) {
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            o[d][i] += odd_value<DT, C8>(row, 32 * d + 8 * (i >> 2) + 4 * h + (i & 3));
                            __builtin_amdgcn_sched_barrier(0);  // (rare: registers count, not time)
                        }
                });
            }
        }
    }
    {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        l = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }
    if (32 * wave + l32 >= t.rows) return;
    const float inv = l == 0.0f ? 0.0f : p.v_scale / l;
    const float lse2 = l == 0.0f ? -INFINITY : m + __builtin_amdgcn_logf(l);                 // base 2
    const int token = t.first + tok, qh = head * p.group + g;
    const int64_t at = (int64_t)token * p.q_heads + qh;
    if (p.splits > 1) {
        const int64_t slot = (int64_t)split * p.tokens * p.q_heads + at;
        if (h == 0) p.part_lse[slot] = lse2;
        if (l != 0.0f) {
            float *dst = p.part + slot * DH + 4 * h;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<v4f *>(dst + 32 * d + 2 * i) = v4f{o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv};
        }
    } else {
        if (h == 0 && p.lse) p.lse[at] = lse2 * 0x1.62e430p-1f;
        uint8_t *dst = p.out + ((int64_t)token * p.out_ld + (int64_t)qh * DH) * 2;
        const bool none = l == 0.0f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                // channels 32 d + 2 i + 4 h .. and eight further: trading with the other half gives eight in a row
                u32 w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = none ? 0u : pack16bit<DT>(o[d][i + 2 * j] * inv, o[d][i + 2 * j + 1] * inv);
                const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
                *reinterpret_cast<uint4 *>(dst + (32 * d + 2 * i + 8 * h) * 2) = make_uint4(a[0], b[0], a[1], b[1]);
            }
    }
}

// ---- joins the splits of a row: a weighted mean with weights exp2(lse_split - the largest) --------------------------------
// Sixteen lanes have the channels of a row; `1 << lanes_log2` such groups share its splits and are joined in LDS.
template <int DT, int DH>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedParams p, int groups_log2) {
    constexpr int CH = DH / 16;
    __shared__ __attribute__((aligned(16))) float part[16][DH + 4];
    __shared__ float part_m[16], part_l[16];
    const int64_t rows = p.tokens * p.q_heads;
    const int group = threadIdx.x >> 4, groups = 1 << groups_log2, mine = group & (groups - 1);
    const int64_t at = ((int64_t)blockIdx.x << (4 - groups_log2)) + (group >> groups_log2);
    const int64_t token = at / p.q_heads;
    const bool live = at < rows && token >= clamp_offset(p, 0) && token < clamp_offset(p, p.seqs);      // (a row of a sequence)
    const int c = (threadIdx.x & 15) * CH;
    float m = -INFINITY, l = 0.0f, y[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) y[i] = 0.0f;
    if (live) {
        constexpr int U = 4;                                     // splits whose loads are in flight together
        for (int s0 = mine; s0 < p.splits; s0 += groups * U) {
            float lse[U];
            v4f v[U][CH / 4];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int s = s0 + u * groups;
                lse[u] = s < p.splits ? p.part_lse[s * rows + at] : -INFINITY;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int s = s0 + u * groups;
                // (where nothing is seen nothing was written either)
#pragma unroll
                for (int i = 0; i < CH / 4; ++i)
                    v[u][i] = lse[u] != -INFINITY ? *reinterpret_cast<const v4f *>(p.part + (s * rows + at) * DH + c + 4 * i) : v4f{0.0f, 0.0f, 0.0f, 0.0f};
            }
            float top = m;
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, lse[u]);
            const float base = top == -INFINITY ? 0.0f : top;
            const float keep = __builtin_amdgcn_exp2f(m - base);
            m = top;
            l *= keep;
#pragma unroll
            for (int i = 0; i < CH; ++i) y[i] *= keep;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float f = __builtin_amdgcn_exp2f(lse[u] - base);
                l += f;
#pragma unroll
                for (int i = 0; i < CH; ++i) y[i] = fmaf(v[u][i >> 2][i & 3], f, y[i]);
            }
        }
    }
    if (groups > 1) {
#pragma unroll
        for (int i = 0; i < CH; i += 4) *reinterpret_cast<v4f *>(&part[group][c + i]) = v4f{y[i], y[i + 1], y[i + 2], y[i + 3]};
        if (c == 0) { part_m[group] = m; part_l[group] = l; }
        __syncthreads();
        if (!live || mine != 0) return;
        float top = m;
        for (int o = 1; o < groups; ++o) top = fmaxf(top, part_m[group + o]);
        const float base = top == -INFINITY ? 0.0f : top;
        const float keep = __builtin_amdgcn_exp2f(m - base);
        l *= keep;
#pragma unroll
        for (int i = 0; i < CH; ++i) y[i] *= keep;
        for (int o = 1; o < groups; ++o) {
            const float f = __builtin_amdgcn_exp2f(part_m[group + o] - base);
            l = fmaf(part_l[group + o], f, l);
#pragma unroll
            for (int i = 0; i < CH; ++i) y[i] = fmaf(part[group + o][c + i], f, y[i]);
        }
        m = top;
    }
    if (!live) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    if (c == 0 && p.lse) p.lse[at] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0x1.62e430p-1f;
    u32 w[CH / 2];
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) w[i] = pack16bit<DT>(y[2 * i] * inv, y[2 * i + 1] * inv);
    u32 *d = reinterpret_cast<u32 *>(p.out + (token * p.out_ld + (at - token * p.q_heads) * DH + c) * 2);
#pragma unroll
    for (int i = 0; i < CH / 2; i += 2) *reinterpret_cast<uint2 *>(d + i) = make_uint2(w[i], w[i + 1]);
}

constexpr int kFewRows = 64, kWgRows = 256;

// Which forms a batch needs; the host knows the totals alone.  A mean above kFewRows rows a sequence: tiles.  Below it the
// streaming form, and both where one sequence can have a chunk of four tiles and more beside single tokens (each form then
// passes over the other's sequences).  us, streaming / tiles, 16 sequences over 4,096 keys: 16 / 4 heads of 128 with 48 rows each
// 51.7 / 37.0, 64 51.5 / 37.6, 96 96.3 / 51.7, 128 116 / 53.5; 8 heads of 64 with 48 rows 46.0 / 64.5, 64 62.5 / 64.6, 96 86.2 / 67.0.
// One chunk beside 63 single tokens over up to 8,000 keys, streaming alone / both: 16 heads of 64, 256 rows 211 / 324, 511 285 / 257,
// 1,024 281 / 274, 2,048 331 / 306; 32 / 8 heads of 128, 280 rows 220 / 259, 512 293 / 264, 1,024 278 / 276, 2,044 491 / 291.  With a
// window of 1,024 the second launch never pays: 511 rows of 64 53 / 93, 1,024 rows of 128 63 / 86, 2,044 85 / 88.
struct Forms { bool few, many; };
Forms forms_of(int64_t tokens, int seqs, int group) {
    if (tokens * group > (int64_t)kFewRows * seqs) return Forms{false, true};
    return Forms{true, (tokens - seqs + 1) * group >= 4 * kWgRows};
}

template <int DT, bool C8, int DH>
hipError_t launch(PagedParams &p, hipStream_t stream) {
    const Forms f = forms_of(p.tokens, p.seqs, p.group);
    p.few_rows = !f.many ? INT64_MAX : (f.few ? kFewRows : -1);
    hipError_t e = hipSuccess;
    if (f.many) {
        p.row_tiles = (int)(p.tokens * p.group / kWgRows) + p.seqs;
        auto kern = paged_tiles_kernel<DT, C8, DH, kWgRows / 32>;
        constexpr int lds = 4 * 64 * DH * 2 + 16;
        static std::atomic<uint64_t> done{0};
        e = allow_dynamic_lds(reinterpret_cast<const void *>(kern), lds, done);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kern, dim3((u32)((int64_t)p.row_tiles * p.kv_heads * p.splits)), dim3(2 * kWgRows), lds, stream, p);
        e = hipGetLastError();
    }
    if (e == hipSuccess && f.few) {
        p.row_tiles = (int)(p.tokens * p.group / kRows) + p.seqs;
        hipLaunchKernelGGL((paged_rows_kernel<DT, C8, DH>), dim3((u32)((int64_t)p.row_tiles * p.kv_heads * p.splits)), dim3(kWaves * 64), 0, stream, p);
        e = hipGetLastError();
    }
    if (e == hipSuccess && p.splits > 1) {
        const int groups_log2 = p.splits <= 4 ? 0 : (p.splits <= 16 ? 2 : 4);
        const int64_t rows = p.tokens * p.q_heads, per = 16 >> groups_log2;
        hipLaunchKernelGGL((paged_join_kernel<DT, DH>), dim3((u32)((rows + per - 1) / per)), dim3(256), 0, stream, p, groups_log2);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

int paged_splits(int64_t tokens, int seqs, int q_heads, int kv_heads, int head_dim, int64_t max_kv) {
    const int group = q_heads / kv_heads;
    const Forms f = forms_of(tokens, seqs, group);
    int64_t s = 1;
    auto at_least = [&](int64_t n) { s = n > s ? n : s; };
    if (f.few) {
        // A round of workgroups with as little as 256 keys each; more rounds, which even out unequal lengths, only of longer
        // pieces (a piece costs its prologue and its way through the workspace).  us, 256 / 512 / 1024 keys a piece: one token,
        // 16,384 keys 19.8 / 19.0 / 21.9; eight, 8,192 keys 59.9 / 55.9 / 54.1; 16 x 8 over 4,096 78.0 / 78.3 / 68.2.
        const int64_t blocks = (tokens * group / kRows + seqs) * kv_heads;
        at_least(std::min(512 / blocks, max_kv / 256));
        at_least(std::min(1024 / blocks, max_kv / 512));
        at_least(std::min(4096 / blocks, max_kv / 1024));
    }
    if (f.many) {
        // a workgroup per CU: 64 rows x 4 over 16,384 keys 42.7 us, with twice as many 57.5, four times 78.5
        const int64_t blocks = (tokens * group / kWgRows + (f.few ? 1 : seqs)) * kv_heads;
        at_least(std::min(256 / blocks, max_kv / 256));
    }
    return (int)std::min<int64_t>(s, 64);
}

hipError_t paged_launch(PagedParams p, int dtype, int cache_dtype, int head_dim, int64_t longest, hipStream_t stream) {
    // equal pieces of the longest range, whole steps of either form; the last one takes what a longer sequence has left
    p.split_keys = (int)(((longest + p.splits - 1) / p.splits + 63) / 64 * 64);
    if (p.split_keys < 64) p.split_keys = 64;
    const bool c8 = cache_dtype == kE4M3;
#define VITQ_PAGED(DT) \
    if (head_dim == 64) return c8 ? launch<DT, true, 64>(p, stream) : launch<DT, false, 64>(p, stream); \
    return c8 ? launch<DT, true, 128>(p, stream) : launch<DT, false, 128>(p, stream);
    if (dtype == kBF16) { VITQ_PAGED(kBF16) }
    VITQ_PAGED(kF16)
#undef VITQ_PAGED
}

}  // namespace vitq
