// A unit of the second pass of attention's gradient: dk and dv of a block of keys.
//
// A wave holds 32 keys and values and walks the rows of the query heads that share
// them: S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS.  2 x 4,096 causal tokens of
// 32 heads of 128: 606 us, 907 TFLOP/s; 16,384 tokens of 16 heads on 2 key heads 2,279 us,
// 965.  With 64 keys a wave half of the LDS reads go, but one wave a SIMD has nothing to
// run beside its exponentials: 890 us.
#pragma once

#include "c3_attention.h"

namespace c3 {

constexpr int kDkvKeys = 32 * kAttnWaves;       // of a unit

// Returns whether a tile that the mask cuts held an infinity or NaN, which only
// CAREFUL keeps from keys that its row does not see.
template <typename T, int DP, bool CAREFUL>
__device__ __forceinline__ bool dkv_unit(const AttnArgs& a, const AttnTable& tab, uint32_t block) {
    constexpr int KS = DP / 16, NDB = DP / 32, kSub = 32 * DP * 2;
    // Heads over 64: the values lie in LDS and tiles have 32 rows, so that two
    // workgroups fit a compute unit's registers (256 a lane) and LDS (160 KiB).
    constexpr bool kValuesLds = DP > 64;
    constexpr int kTileRows = kValuesLds ? 32 : 64;
    constexpr int kTileBytes = kTileRows * DP * 2, kSteps = 2;
    static_assert(kTileRows / 32 * KS == kSteps * kAttnWaves, "two steps of a tile to each wave");
    __shared__ __attribute__((aligned(1024))) char q0[kTileBytes];
    __shared__ __attribute__((aligned(1024))) char g0[kTileBytes];
    __shared__ __attribute__((aligned(1024))) float s0[2 * 64];      // lse2, delta: 64 lanes' words each
    __shared__ __attribute__((aligned(1024))) char q1[kTileBytes];
    __shared__ __attribute__((aligned(1024))) char g1[kTileBytes];
    __shared__ __attribute__((aligned(1024))) float s1[2 * 64];
    __shared__ __attribute__((aligned(1024))) char v_tile[kValuesLds ? kDkvKeys * DP * 2 : 16];
    __shared__ T words[CAREFUL ? kAttnWaves : 1][32 * 32];        // for the masked product

    const AttnUnit w = attn_unit(a, tab, 1, block);
    const AttnSide& side = a.side[1];
    const int G = (int)a.group.d;
    const int n_rows = w.q_len * G, off = w.k_len - w.q_len;
    const int k_pad = a.packed ? w.k_len : a.k_tokens;
    const int tile = (int)side.splits.quot(w.unit), part = (int)w.unit - tile * (int)side.splits.d;
    const int key_block = tile * kDkvKeys;
    const int lane = threadIdx.x & 63, h = lane >> 5, c = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wkey = key_block + wave * 32, key = wkey + c;

    // queries that see any of the block's keys
    int p_lo = 0, p_hi = w.q_len;
    if (a.causal) p_lo = max(0, key_block - off);
    if (a.window) p_hi = min(p_hi, key_block + kDkvKeys - 1 - off + a.window);
    if (key_block >= w.k_len) p_hi = 0;
    int t0 = p_lo * G / kTileRows;
    int t1 = p_hi > p_lo ? (p_hi * G + kTileRows - 1) / kTileRows : t0;
    if (side.splits.d > 1) {       // this workgroup's part of the walk
        const int64_t n = t1 - t0;
        t1 = t0 + (int)side.splits.quot((uint32_t)(n * (part + 1)));
        t0 = t0 + (int)side.splits.quot((uint32_t)(n * part));
    }

    const StepReads<DP> rd;
    const char* qb = seq_base(a.q, a.packed, w.b, w.q_start, w.hk * G);
    const char* gb = seq_base(a.d_o, a.packed, w.b, w.q_start, w.hk * G);
    const int64_t stat_row = seq_row(a, w) + w.hk * G;
    const float cs = a.scale * kLog2e;

    f32x16 dk[NDB] = {}, dv[NDB] = {};
    uint32_t bad = 0;
    float factor = kDsScaled<T> ? kDsFactor : 1.0f;     // of dS

    auto load = [&](int t, char* qt, char* gt, float* st) {
        const int row0 = t * kTileRows, rows = min(kTileRows, n_rows - row0);
        const int p0 = __builtin_amdgcn_readfirstlane((int)a.group.quot(row0));
        const int p1 = __builtin_amdgcn_readfirstlane((int)a.group.quot(row0 + rows - 1)) - p0;
        const char* qr = qb + (int64_t)p0 * a.q.st;
        const char* gr = gb + (int64_t)p0 * a.d_o.st;
        const uint32_t q_bytes = (uint32_t)(p1 * a.q.st + (G - 1) * a.q.sh) + a.dim * 2;
        const uint32_t g_bytes = (uint32_t)(p1 * a.d_o.st + (G - 1) * a.d_o.sh) + a.dim * 2;
        // the wave's steps, all odd or all even, lie in one of the tile's 32 rows; a lane
        // takes half a row's 32 bytes of each
        const int first = wave / 2 * 4 + (wave & 1), i = first / KS * 32 + rd.load_row(lane, first);
        const int r = row0 + i, p = (int)a.group.quot(r), g = r - p * G;
        const uint32_t qo = (uint32_t)((p - p0) * (int)a.q.st + g * (int)a.q.sh);
        const uint32_t go = (uint32_t)((p - p0) * (int)a.d_o.st + g * (int)a.d_o.sh);
#pragma unroll
        for (int n = 0; n < kSteps; ++n) {
            const int at = first + 2 * n, piece = 2 * (at % KS) + rd.load_half(lane);
            const bool ok = i < rows && piece * 8 < a.dim;
            load_piece_lds(qr, q_bytes, ok ? qo + piece * 16 : 0xFFFFFF00u, qt + at * 1024);
            load_piece_lds(gr, g_bytes, ok ? go + piece * 16 : 0xFFFFFF00u, gt + at * 1024);
        }
        if (wave < 2) {         // a lane for each row: lse2 by the first wave, delta by the second
            const float* from = (wave == 0 ? a.lse2 : a.delta) + stat_row + (int64_t)p0 * a.heads;
            const int r = row0 + lane, p = (int)a.group.quot(r), g = r - p * G;
            const uint32_t bytes = (uint32_t)(p1 * a.heads + G) * 4;
            const uint32_t at = lane < rows ? (uint32_t)((p - p0) * a.heads + g) * 4 : 0xFFFFFF00u;
            const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(from), 0, (int)bytes, 0x00027000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(st + wave * 64), 4, (int)at, 0, 0, 0);
        }
    };
    u32x4 kf[KS], vf[KS];
    {
        const char* kb = seq_base(a.k, a.packed, w.b, w.k_start, w.hk);
        const char* vb = seq_base(a.v, a.packed, w.b, w.k_start, w.hk);
        load_row<DP>(kf, kb + (int64_t)key * a.k.st, key < w.k_len, a.dim);
        if constexpr (!kValuesLds) load_row<DP>(vf, vb + (int64_t)key * a.v.st, key < w.k_len, a.dim);
        if constexpr (kValuesLds) {
            // each wave its own keys'
            const int rows = min(w.k_len - wkey, 32);
            const uint32_t bytes = rows > 0 ? (uint32_t)((rows - 1) * a.v.st) + a.dim * 2 : 0;
#pragma unroll
            for (int n = 0; n < KS; ++n) {
                const int i = rd.load_row(lane, n), piece = 2 * n + rd.load_half(lane);
                const bool ok = i < rows && piece * 8 < a.dim;
                load_piece_lds(vb + (int64_t)wkey * a.v.st, bytes,
                               ok ? (uint32_t)(i * (int)a.v.st + piece * 16) : 0xFFFFFF00u,
                               v_tile + (wave * KS + n) * 1024);
            }
        }
    }

    // The four parts of 32 rows' work: scores and dP; P and dS; what they add to
    // dv and dk.
    auto scores = [&](int n, const char* qt, const char* gt, f32x16& s, f32x16& dp) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            s = mfma<T>(rd.along(qt + n * kSub, ks), kf[ks], s);
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const u32x4 x = rd.along(gt + n * kSub, ks);
            if constexpr (kValuesLds)
                dp = mfma<T>(x, rd.along(v_tile + wave * kSub, ks), dp);
            else
                dp = mfma<T>(x, vf[ks], dp);
        }
    };
    auto probabilities = [&](int n, const float* st, f32x16& s, f32x16& dp) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 l2 = *reinterpret_cast<const f32x4*>(st + n * 32 + q * 8 + h * 4);
            const f32x4 de = *reinterpret_cast<const f32x4*>(st + 64 + n * 32 + q * 8 + h * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[4 * q + i] = __builtin_amdgcn_exp2f(fmaf(s[4 * q + i], cs, -l2[i]));
                dp[4 * q + i] = s[4 * q + i] * (dp[4 * q + i] - de[i]);
                if constexpr (kDsScaled<T>) dp[4 * q + i] *= factor;
            }
        }
    };
    auto gradients = [&](int n, const char* qt, const char* gt, const f32x16& s, const f32x16& dp) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const u32x4 p = operand<T>(s, j), ds = operand<T>(dp, j);
#pragma unroll
            for (int db = 0; db < NDB; ++db) dv[db] = mfma<T>(rd.across(gt + n * kSub, j, db), p, dv[db]);
#pragma unroll
            for (int db = 0; db < NDB; ++db) dk[db] = mfma<T>(rd.across(qt + n * kSub, j, db), ds, dk[db]);
        }
    };
    auto step = [&](int t, const char* qt, const char* gt, const float* st) {
#pragma unroll
        for (int n = 0; n < kTileRows / 32; ++n) {
            const int row0 = t * kTileRows + n * 32;
            if (row0 >= n_rows) continue;
            const int pa = (int)a.group.quot(row0) + off;
            const int pb = (int)a.group.quot(min(row0 + 31, n_rows - 1)) + off;
            if (a.causal && wkey > pb) continue;
            if (a.window && wkey + 31 <= pa - a.window) continue;
            // rows behind the last hold zeros, which times an infinite key is NaN: hidden too
            const bool masked = (a.causal && wkey + 31 > pa) || (a.window && wkey <= pb - a.window) ||
                                row0 + 32 > n_rows;
            f32x16 s = {}, dp = {};
            uint32_t seen = 0;
            scores(n, qt, gt, s, dp);
            probabilities(n, st, s, dp);
            if (masked) {
                // formed here, not held in registers through the walk
                int k_ = key, h_ = h * 4;
                asm volatile("" : "+v"(k_), "+v"(h_));
                // rows from r_lo to below r_hi of these 32 see the lane's key
                const int64_t at = (int64_t)(k_ - off) * G - row0, all = (int64_t)a.window * G;
                const int r_lo = a.causal ? (int)min(max(at, (int64_t)0), (int64_t)32) : 0;
                const int r_hi = min(a.window ? (int)min(max(at + all, (int64_t)0), (int64_t)32) : 32,
                                     n_rows - row0);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int r = (i >> 2) * 8 + h_ + (i & 3);
                    const bool see = r >= r_lo && r < r_hi;
                    seen |= see ? 1u << i : 0u;
                    s[i] = see ? s[i] : 0.0f;
                    dp[i] = see ? dp[i] : 0.0f;
                }
            }
            if constexpr (kDsScaled<T>) fit_ds<NDB>(dp, dk, factor);
            if (masked) {
                const char *q_sub = qt + n * kSub, *g_sub = gt + n * kSub;
                const uint32_t here = tile_not_finite<T>(KS, [&](int ks) { return rd.along(q_sub, ks); }) |
                                      tile_not_finite<T>(KS, [&](int ks) { return rd.along(g_sub, ks); });
                bad |= here;
                if constexpr (CAREFUL) {
                    if (__any(here != 0)) {
                        masked_product<T, NDB>(dv, s, seen, words[wave],
                                               [&](int k, int d) { return rd.four(g_sub, k, d); },
                                               [&](int j, int db) { return rd.across(g_sub, j, db); });
                        masked_product<T, NDB>(dk, dp, seen, words[wave],
                                               [&](int k, int d) { return rd.four(q_sub, k, d); },
                                               [&](int j, int db) { return rd.across(q_sub, j, db); });
                        continue;
                    }
                }
            }
            gradients(n, qt, gt, s, dp);
        }
    };

    if (t0 < t1) load(t0, q0, g0, s0);
    for (int t = t0; t < t1; t += 2) {
        tiles_ready();
        if (t + 1 < t1) load(t + 1, q1, g1, s1);
        step(t, q0, g0, s0);
        if (t + 1 >= t1) break;
        tiles_ready();
        if (t + 2 < t1) load(t + 2, q0, g0, s0);
        step(t + 1, q1, g1, s1);
    }

    if (key >= k_pad) return bad != 0;
    const bool valid = key < w.k_len;
    if constexpr (kDsScaled<T>) {
        const float back = 1.0f / factor;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) dk[db][i] *= back;
    }
    if (side.splits.d > 1) {
        // dk and dv of this part, in fp32 and not yet scaled
        const int64_t keys = (int64_t)(a.packed ? 0 : w.b) * a.k_tokens + w.k_start + key;
        float* to = side.part + (part * 2 * side.part_rows + keys * a.kv_heads + w.hk) * a.dim;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int d = db * 32 + q * 8 + h * 4;
                if (d >= a.dim) continue;
                f32x4 x, y;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = valid ? dk[db][4 * q + i] : 0.0f;
                    y[i] = valid ? dv[db][4 * q + i] : 0.0f;
                }
                *reinterpret_cast<f32x4*>(to + d) = x;
                *reinterpret_cast<f32x4*>(to + side.part_rows * a.dim + d) = y;
            }
        return bad != 0;
    }
    char* ok = seq_base(a.dk, a.packed, w.b, w.k_start, w.hk) + (int64_t)key * a.dk.st;
    char* ov = seq_base(a.dv, a.packed, w.b, w.k_start, w.hk) + (int64_t)key * a.dv.st;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int d = db * 32 + q * 8 + h * 4;
            if (d >= a.dim) continue;
            T e[4], f[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e[i] = valid ? (T)(dk[db][4 * q + i] * a.scale) : (T)0.0f;
                f[i] = valid ? (T)dv[db][4 * q + i] : (T)0.0f;
            }
            u32x2 x, y;
            __builtin_memcpy(&x, e, 8);
            __builtin_memcpy(&y, f, 8);
            *reinterpret_cast<u32x2*>(ok + d * 2) = x;
            *reinterpret_cast<u32x2*>(ov + d * 2) = y;
        }
    return bad != 0;
}

}  // namespace c3
