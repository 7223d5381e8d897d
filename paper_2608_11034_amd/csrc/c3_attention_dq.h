// A unit of the first pass of attention's gradient: dq of a tile of rows, and lse in
// powers of two and delta of every row for the second.
//
// A wave holds 32 rows' queries and output gradients and walks the keys, as the
// forward does: S^T = K Q^T, dP^T = V dO^T, dS = P (dP - delta), dQ^T += K^T dS.
// 2 x 4,096 causal tokens of 32 heads of 128: 408 us, 1,010 TFLOP/s; 16,384 tokens of 16
// heads on 2 key heads 1,508 us, 1,094.
#pragma once

#include "c3_attention.h"

namespace c3 {

constexpr int kDqKeys = 64;         // keys of a tile
constexpr int kShortWalk = 2;       // tiles
constexpr int kFewKeys = 16;

// Returns whether a tile that the mask cuts held an infinity or NaN, which only
// CAREFUL keeps from rows that do not see it.  REPEATED: lse2 and delta are there, and
// workgroups beside this one read them.
template <typename T, int DP, bool CAREFUL, bool REPEATED = false>
__device__ __forceinline__ bool dq_unit(const AttnArgs& a, const AttnTable& tab, uint32_t block) {
    constexpr int KS = DP / 16, NDB = DP / 32, kSub = 32 * DP * 2;
    constexpr int kRows = 32 * kAttnWaves;
    using L = TileLoads<DP, kDqKeys>;
    __shared__ __attribute__((aligned(1024))) char k0[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char v0[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char k1[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char v1[L::kBytes];
    __shared__ T words[CAREFUL ? kAttnWaves : 1][32 * 32];        // for the masked product

    const AttnUnit w = attn_unit(a, tab, 0, block);
    const AttnSide& side = a.side[0];
    const int G = (int)a.group.d;
    const int n_rows = w.q_pad * G, off = w.k_len - w.q_len;
    const int tiles = (n_rows + kRows - 1) / kRows;
    const int nth = (int)side.splits.quot(w.unit), part = (int)w.unit - nth * (int)side.splits.d;
    const int tile = a.causal ? tiles - 1 - nth : nth;
    const int row0 = tile * kRows;
    const int lane = threadIdx.x & 63, h = lane >> 5, c = lane & 31;
    const int wave = threadIdx.x >> 6;

    const int first = (int)a.group.quot(row0);
    const int last = min((int)a.group.quot(min(row0 + kRows, n_rows) - 1), w.q_len - 1);
    int lo = 0, hi = w.k_len;
    if (a.causal) hi = min(hi, last + off + 1);
    if (a.window) lo = max(lo, first + off - a.window + 1);
    if (first >= w.q_len) hi = 0;
    int t0 = lo / kDqKeys, t1 = hi > lo ? (hi + kDqKeys - 1) / kDqKeys : t0;
    const int all0 = t0, all1 = t1;
    if (side.splits.d > 1) {       // this workgroup's part of the walk
        const int64_t n = t1 - t0;
        t1 = t0 + (int)side.splits.quot((uint32_t)(n * (part + 1)));
        t0 = t0 + (int)side.splits.quot((uint32_t)(n * part));
    }

    const int row = row0 + wave * 32 + c;
    const int pos = (int)a.group.quot(row), head = w.hk * G + row - pos * G;
    const bool there = row < n_rows, valid = there && pos < w.q_len;
    const int see_hi = !valid ? INT32_MAX : a.causal ? min(w.k_len, pos + off + 1) : w.k_len;
    const int see_lo = valid && a.window ? pos + off - a.window + 1 : 0;
    u32x4 qf[KS], gf[KS];
    load_row<DP>(qf, seq_base(a.q, a.packed, w.b, w.q_start, head) + (int64_t)pos * a.q.st, valid, a.dim);
    load_row<DP>(gf, seq_base(a.d_o, a.packed, w.b, w.q_start, head) + (int64_t)pos * a.d_o.st, valid, a.dim);
    float delta = 0.0f, lse2 = __builtin_inff();
    {
        u32x4 of[KS];
        load_row<DP>(of, seq_base(a.o, a.packed, w.b, w.q_start, head) + (int64_t)pos * a.o.st, valid, a.dim);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            T x[8], y[8];
            __builtin_memcpy(x, &of[ks], 16);
            __builtin_memcpy(y, &gf[ks], 16);
#pragma unroll
            for (int i = 0; i < 8; ++i) delta = fmaf(to_f32(x[i]), to_f32(y[i]), delta);
        }
        delta += __shfl_xor(delta, 32);
        const int64_t at = seq_row(a, w) + (int64_t)pos * a.heads + head;
        if (valid) {
            const float lse = a.lse[at];
            if (lse != -__builtin_inff()) lse2 = lse * kLog2e;
        }
        if (!REPEATED && there && h == 0 && part == 0) a.lse2[at] = lse2;
    }

    TileReads<DP> rd;
    const TokenOffsets<DP, kDqKeys> k_off(a.k.st, a.dim), v_off(a.v.st, a.dim);
    const char* kb = seq_base(a.k, a.packed, w.b, w.k_start, w.hk);
    const char* vb = seq_base(a.v, a.packed, w.b, w.k_start, w.hk);
    const float cs = a.scale * kLog2e;

    f32x16 acc[NDB] = {};
    uint32_t bad = 0;
    float factor = kDsScaled<T> ? kDsFactor : 1.0f;     // of dS: it comes with the probabilities
    float shift = kDsScaled<T> ? 64.0f - lse2 : -lse2;

    auto load = [&](int t, char* kt, char* vt) {
        const int key = t * kDqKeys;
        load_tile<DP, kDqKeys>(kb + (int64_t)key * a.k.st, a.k.st, a.dim, w.k_len - key, k_off, kt);
        load_tile<DP, kDqKeys>(vb + (int64_t)key * a.v.st, a.v.st, a.dim, w.k_len - key, v_off, vt);
    };
    // Rows that see few keys have an output near the values' size, and its rounding to 16
    // bits would enter delta as much as that of dS enters the product (bf16, two keys: dq
    // off by 0.0036 in the norm, not 0.0023): for them delta is the sum of P dP, which
    // needs no output.  From 16 keys on it shows no more; the walk over a tile with a row
    // of so few is of 16 and a tile's rows at most.  Two tiles of keys cost little, so
    // they go this way too.
    int fewest = INT32_MAX;
    if (a.causal) fewest = first + off + 1;
    if (a.window) fewest = min(fewest, a.causal ? a.window : w.q_len - 1 - last + a.window);
    if (all1 - all0 <= kShortWalk || fewest <= kFewKeys) {
        float sum = 0.0f;
        for (int t = all0; t < all1; ++t) {
            load(t, k0, v0);
            tiles_ready();
#pragma unroll 1
            for (int n = 0; n < 2; ++n) {
                const int key0 = t * kDqKeys + n * 32;
                f32x16 s = {}, dp = {};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    s = mfma<T>(rd.along(k0 + n * kSub, ks), qf[ks], s);
                    dp = mfma<T>(rd.along(v0 + n * kSub, ks), gf[ks], dp);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = key0 + (i >> 2) * 8 + h * 4 + (i & 3);
                    const bool see = valid && key < see_hi && key >= see_lo;
                    sum += see ? __builtin_amdgcn_exp2f(fmaf(s[i], cs, -lse2)) * dp[i] : 0.0f;
                }
            }
            __syncthreads();        // before the tile is loaded anew
        }
        delta = sum + __shfl_xor(sum, 32);
    }
    if (!REPEATED && there && h == 0 && part == 0) a.delta[seq_row(a, w) + (int64_t)pos * a.heads + head] = delta;

    auto step = [&](int t, const char* kt, const char* vt) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int key0 = t * kDqKeys + n * 32;
            if (!__any(valid && key0 < see_hi && key0 + 32 > see_lo)) continue;
            const bool masked = __any(key0 + 32 > see_hi || key0 < see_lo);
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s = mfma<T>(rd.along(kt + n * kSub, ks), qf[ks], s);
                dp = mfma<T>(rd.along(vt + n * kSub, ks), gf[ks], dp);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], cs, shift)) * (dp[i] - delta);
            uint32_t seen = 0;
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = key0 + (i >> 2) * 8 + h * 4 + (i & 3);
                    const bool see = key < see_hi && key >= see_lo;
                    seen |= see ? 1u << i : 0u;
                    s[i] = see ? s[i] : 0.0f;
                }
            }
            if constexpr (kDsScaled<T>) shift -= fit_ds<NDB>(s, acc, factor);
            if (masked) {
                const char* sub = kt + n * kSub;
                const uint32_t here = tile_not_finite<T>(KS, [&](int ks) { return rd.along(sub, ks); });
                bad |= here;
                if constexpr (CAREFUL) {
                    if (__any(here != 0)) {
                        masked_product<T, NDB>(acc, s, seen, words[wave],
                                               [&](int k, int d) { return rd.four(sub, k, d); },
                                               [&](int j, int db) { return rd.across(sub + j * 16 * DP * 2, db); });
                        continue;
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const u32x4 ds = operand<T>(s, j);
#pragma unroll
                for (int db = 0; db < NDB; ++db)
                    acc[db] = mfma<T>(rd.across(kt + n * kSub + j * 16 * DP * 2, db), ds, acc[db]);
            }
        }
    };

    if (t0 < t1) load(t0, k0, v0);
    for (int t = t0; t < t1; t += 2) {
        tiles_ready();
        if (t + 1 < t1) load(t + 1, k1, v1);
        step(t, k0, v0);
        if (t + 1 >= t1) break;
        tiles_ready();
        if (t + 2 < t1) load(t + 2, k0, v0);
        step(t + 1, k1, v1);
    }

    if (!there) return bad != 0;
    if constexpr (kDsScaled<T>) {
        const float back = 1.0f / factor;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[db][i] *= back;
    }
    if (side.splits.d > 1) {
        // this part's sum, in fp32 and not yet scaled
        float* to = side.part + (part * side.part_rows + seq_row(a, w) + (int64_t)pos * a.heads + head) * a.dim;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int d = db * 32 + q * 8 + h * 4;
                if (d >= a.dim) continue;
                f32x4 x;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = valid ? acc[db][4 * q + i] : 0.0f;
                *reinterpret_cast<f32x4*>(to + d) = x;
            }
        return bad != 0;
    }
    char* out = seq_base(a.dq, a.packed, w.b, w.q_start, head) + (int64_t)pos * a.dq.st;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int d = db * 32 + q * 8 + h * 4;
            if (d >= a.dim) continue;
            T e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = valid ? (T)(acc[db][4 * q + i] * a.scale) : (T)0.0f;
            u32x2 x;
            __builtin_memcpy(&x, e, 8);
            *reinterpret_cast<u32x2*>(out + d * 2) = x;
        }
    return bad != 0;
}

}  // namespace c3
