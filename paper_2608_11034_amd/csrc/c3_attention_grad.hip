// Attention's gradient (include/c3_replay.h), in two passes that recompute the
// probabilities from lse:
//
//   dq pass   a wave holds 32 rows' queries and output gradients and walks the
//             keys, as the forward does: S^T = K Q^T, dP^T = V dO^T, dS = P (dP -
//             delta), dQ^T += K^T dS.  It also forms delta, the sum of dO O of a
//             row, and leaves it and lse in powers of two for the other pass.
//   dkv pass  a wave holds 32 keys and values and walks the rows: S = Q K^T, dP =
//             dO V^T, dV^T += dO^T P, dK^T += Q^T dS.
//
// Seven products where one pass would do with five: there the dq of a row would
// be added up by workgroups in the order in which they come, and the bits would
// change from run to run.  Matrix products bound both.
#include <algorithm>

#include "c3_attention.h"

namespace c3 {
namespace {

constexpr int kKeys = 64;           // keys of a tile of the dq pass
constexpr int kTileRows = 64;       // rows of a tile of the dkv pass

template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, 2) void attn_dq_kernel(AttnArgs a, AttnTable tab) {
    constexpr int KS = DP / 16, NDB = DP / 32, kSub = 32 * DP * 2;
    constexpr int kRows = 32 * kAttnWaves;
    using L = TileLoads<DP, kKeys>;
    __shared__ __attribute__((aligned(1024))) char k0[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char v0[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char k1[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char v1[L::kBytes];

    const AttnUnit w = attn_unit(a, tab, die_order(blockIdx.x, gridDim.x));
    const int G = (int)a.group.d;
    const int n_rows = w.q_pad * G, off = w.k_len - w.q_len;
    const int tiles = (n_rows + kRows - 1) / kRows;
    const int tile = a.causal ? tiles - 1 - (int)w.unit : (int)w.unit;
    const int row0 = tile * kRows;
    const int lane = threadIdx.x & 63, h = lane >> 5, c = lane & 31;
    const int wave = threadIdx.x >> 6;

    const int first = (int)a.group.quot(row0);
    const int last = min((int)a.group.quot(min(row0 + kRows, n_rows) - 1), w.q_len - 1);
    int lo = 0, hi = w.k_len;
    if (a.causal) hi = min(hi, last + off + 1);
    if (a.window) lo = max(lo, first + off - a.window + 1);
    if (first >= w.q_len) hi = 0;
    const int t0 = lo / kKeys, t1 = hi > lo ? (hi + kKeys - 1) / kKeys : t0;

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
        if (there && h == 0) {
            a.lse2[at] = lse2;
            a.delta[at] = delta;
        }
    }

    const TileReads<DP> rd;
    const TokenOffsets<DP, kKeys> k_off(a.k.st, a.dim), v_off(a.v.st, a.dim);
    const char* kb = seq_base(a.k, a.packed, w.b, w.k_start, w.hk);
    const char* vb = seq_base(a.v, a.packed, w.b, w.k_start, w.hk);
    const float cs = a.scale * kLog2e;

    f32x16 acc[NDB] = {};
    uint32_t special[NDB] = {};

    auto load = [&](int t, char* kt, char* vt) {
        const int key = t * kKeys;
        load_tile<DP, kKeys>(kb + (int64_t)key * a.k.st, a.k.st, a.dim, w.k_len - key, k_off, kt);
        load_tile<DP, kKeys>(vb + (int64_t)key * a.v.st, a.v.st, a.dim, w.k_len - key, v_off, vt);
    };
    auto step = [&](int t, const char* kt, const char* vt) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int key0 = t * kKeys + n * 32;
            if (!__any(valid && key0 < see_hi && key0 + 32 > see_lo)) continue;
            const bool masked = __any(key0 + 32 > see_hi || key0 < see_lo);
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s = mfma<T>(read_along(kt, rd.along[ks] + n * kSub), qf[ks], s);
                dp = mfma<T>(read_along(vt, rd.along[ks] + n * kSub), gf[ks], dp);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], cs, -lse2)) * (dp[i] - delta);
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
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const u32x4 ds = operand<T>(s, j);
                u32x4 A[NDB];
#pragma unroll
                for (int db = 0; db < NDB; ++db)
                    A[db] = read_across(kt + n * kSub, rd.across[db], j * 16 * DP * 2);
                if (masked) finite_operands<T, NDB>(A, ds, seen >> (8 * j), special);
#pragma unroll
                for (int db = 0; db < NDB; ++db) acc[db] = mfma<T>(A[db], ds, acc[db]);
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

    add_special<NDB>(acc, special);
    if (!there) return;
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
}

// Rows `row0 ..` of queries or output gradients to LDS; `at` and `ok` are the
// lane's rows of the tile (query minus the tile's first, head of the group).
template <int DP>
struct RowPieces {
    using L = TileLoads<DP, kTileRows>;
    int row[L::kSteps], piece[L::kSteps];
    bool inside[L::kSteps];
    __device__ __forceinline__ explicit RowPieces(int dim) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int n = 0; n < L::kSteps; ++n) {
            row[n] = (wave * L::kSteps + n) * L::kStepRows + lane / L::kPieces;
            const int p = (lane % L::kPieces) ^ swizzle<DP>(row[n]);
            piece[n] = p * 16;
            inside[n] = p * 8 < dim;
        }
    }
};

template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, 2) void attn_dkv_kernel(AttnArgs a, AttnTable tab) {
    constexpr int KS = DP / 16, NDB = DP / 32, kSub = 32 * DP * 2;
    constexpr int kBlockKeys = 32 * kAttnWaves;
    using L = TileLoads<DP, kTileRows>;
    __shared__ __attribute__((aligned(1024))) char q0[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char g0[L::kBytes];
    __shared__ __attribute__((aligned(1024))) float s0[2 * kTileRows];      // lse2, delta
    __shared__ __attribute__((aligned(1024))) char q1[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char g1[L::kBytes];
    __shared__ __attribute__((aligned(1024))) float s1[2 * kTileRows];

    const AttnUnit w = attn_unit(a, tab, die_order(blockIdx.x, gridDim.x));
    const int G = (int)a.group.d;
    const int n_rows = w.q_len * G, off = w.k_len - w.q_len;
    const int k_pad = a.packed ? w.k_len : a.k_tokens;
    const int key_block = (int)w.unit * kBlockKeys;
    const int lane = threadIdx.x & 63, h = lane >> 5, c = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wkey = key_block + wave * 32, key = wkey + c;
    const bool valid = key < w.k_len;

    // queries that see any of the block's keys
    int p_lo = 0, p_hi = w.q_len;
    if (a.causal) p_lo = max(0, key_block - off);
    if (a.window) p_hi = min(p_hi, key_block + kBlockKeys - 1 - off + a.window);
    if (key_block >= w.k_len) p_hi = 0;
    const int t0 = p_lo * G / kTileRows;
    const int t1 = p_hi > p_lo ? (p_hi * G + kTileRows - 1) / kTileRows : t0;

    u32x4 kf[KS], vf[KS];
    load_row<DP>(kf, seq_base(a.k, a.packed, w.b, w.k_start, w.hk) + (int64_t)key * a.k.st, valid, a.dim);
    load_row<DP>(vf, seq_base(a.v, a.packed, w.b, w.k_start, w.hk) + (int64_t)key * a.v.st, valid, a.dim);

    const TileReads<DP> rd;
    const RowPieces<DP> rp(a.dim);
    const char* qb = seq_base(a.q, a.packed, w.b, w.q_start, w.hk * G);
    const char* gb = seq_base(a.d_o, a.packed, w.b, w.q_start, w.hk * G);
    const int64_t stat_row = seq_row(a, w) + w.hk * G;
    const float cs = a.scale * kLog2e;

    f32x16 dk[NDB] = {}, dv[NDB] = {};
    uint32_t dk_special[NDB] = {}, dv_special[NDB] = {};

    auto load = [&](int t, char* qt, char* gt, float* st) {
        const int row0 = t * kTileRows, rows = min(kTileRows, n_rows - row0);
        const int p0 = __builtin_amdgcn_readfirstlane((int)a.group.quot(row0));
        const int p1 = __builtin_amdgcn_readfirstlane((int)a.group.quot(row0 + rows - 1)) - p0;
        const char* qr = qb + (int64_t)p0 * a.q.st;
        const char* gr = gb + (int64_t)p0 * a.d_o.st;
        const uint32_t q_bytes = (uint32_t)(p1 * a.q.st + (G - 1) * a.q.sh) + a.dim * 2;
        const uint32_t g_bytes = (uint32_t)(p1 * a.d_o.st + (G - 1) * a.d_o.sh) + a.dim * 2;
#pragma unroll
        for (int n = 0; n < L::kSteps; ++n) {
            const int r = row0 + rp.row[n], p = (int)a.group.quot(r), g = r - p * G;
            const bool ok = rp.inside[n] && rp.row[n] < rows;
            const uint32_t qo = (uint32_t)((p - p0) * (int)a.q.st + g * (int)a.q.sh + rp.piece[n]);
            const uint32_t go = (uint32_t)((p - p0) * (int)a.d_o.st + g * (int)a.d_o.sh + rp.piece[n]);
            load_piece_lds(qr, q_bytes, ok ? qo : 0xFFFFFF00u, qt + (wave * L::kSteps + n) * 1024);
            load_piece_lds(gr, g_bytes, ok ? go : 0xFFFFFF00u, gt + (wave * L::kSteps + n) * 1024);
        }
        if (wave < 2) {         // a lane for each row: lse2 by the first wave, delta by the second
            const float* from = (wave == 0 ? a.lse2 : a.delta) + stat_row + (int64_t)p0 * a.heads;
            const int r = row0 + lane, p = (int)a.group.quot(r), g = r - p * G;
            const uint32_t bytes = (uint32_t)(p1 * a.heads + G) * 4;
            const uint32_t at = lane < rows ? (uint32_t)((p - p0) * a.heads + g) * 4 : 0xFFFFFF00u;
            const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(from), 0, (int)bytes, 0x00027000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(st + wave * kTileRows), 4, (int)at, 0, 0, 0);
        }
    };
    auto step = [&](int t, const char* qt, const char* gt, const float* st) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int row0 = t * kTileRows + n * 32;
            if (row0 >= n_rows) continue;
            const int pa = (int)a.group.quot(row0) + off;
            const int pb = (int)a.group.quot(min(row0 + 31, n_rows - 1)) + off;
            if (a.causal && wkey > pb) continue;
            if (a.window && wkey + 31 <= pa - a.window) continue;
            const bool masked = (a.causal && wkey + 31 > pa) || (a.window && wkey <= pb - a.window);
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s = mfma<T>(read_along(qt, rd.along[ks] + n * kSub), kf[ks], s);
                dp = mfma<T>(read_along(gt, rd.along[ks] + n * kSub), vf[ks], dp);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 l2 = *reinterpret_cast<const f32x4*>(st + n * 32 + q * 8 + h * 4);
                const f32x4 de = *reinterpret_cast<const f32x4*>(st + kTileRows + n * 32 + q * 8 + h * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[4 * q + i] = __builtin_amdgcn_exp2f(fmaf(s[4 * q + i], cs, -l2[i]));
                    dp[4 * q + i] = s[4 * q + i] * (dp[4 * q + i] - de[i]);
                }
            }
            uint32_t seen = 0;
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int at = (int)a.group.quot(row0 + (i >> 2) * 8 + h * 4 + (i & 3)) + off;
                    const bool see = (!a.causal || key <= at) && (!a.window || key > at - a.window);
                    seen |= see ? 1u << i : 0u;
                    s[i] = see ? s[i] : 0.0f;
                    dp[i] = see ? dp[i] : 0.0f;
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const u32x4 p = operand<T>(s, j), ds = operand<T>(dp, j);
                u32x4 A[NDB];
#pragma unroll
                for (int db = 0; db < NDB; ++db)
                    A[db] = read_across(gt + n * kSub, rd.across[db], j * 16 * DP * 2);
                if (masked) finite_operands<T, NDB>(A, p, seen >> (8 * j), dv_special);
#pragma unroll
                for (int db = 0; db < NDB; ++db) dv[db] = mfma<T>(A[db], p, dv[db]);
#pragma unroll
                for (int db = 0; db < NDB; ++db)
                    A[db] = read_across(qt + n * kSub, rd.across[db], j * 16 * DP * 2);
                if (masked) finite_operands<T, NDB>(A, ds, seen >> (8 * j), dk_special);
#pragma unroll
                for (int db = 0; db < NDB; ++db) dk[db] = mfma<T>(A[db], ds, dk[db]);
            }
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

    add_special<NDB>(dk, dk_special);
    add_special<NDB>(dv, dv_special);
    if (key >= k_pad) return;
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
}

inline uint64_t align256(uint64_t x) { return (x + 255) / 256 * 256; }

// Workspace: lse2 and delta of every row, then the tables of both passes.
struct GradSpace {
    uint64_t lse2, delta, table_q, table_k, total;
    GradSpace(const c3_attention_t* a, const AttnPlan& p) {
        uint64_t at = 0;
        auto take = [&at](uint64_t bytes) { const uint64_t r = at; at = align256(at + bytes); return r; };
        lse2 = take(4 * (uint64_t)p.rows);
        delta = take(4 * (uint64_t)p.rows);
        table_q = take(attn_table_bytes(a));
        table_k = take(attn_table_bytes(a));
        total = std::max<uint64_t>(at, 256);
    }
};

// Numbers the sequences' units for one pass and stages the list if it is long.
int number_units(const c3_attention_t* a, AttnPlan& p, char* table, bool keys, hipStream_t s) {
    const int64_t group = p.args.group.d;
    const int64_t units = attn_number(p, a->batch, [&](int64_t nq, int64_t, int64_t nk) {
        return keys ? (nk + 32 * kAttnWaves - 1) / (32 * kAttnWaves)
                    : (nq * group + 32 * kAttnWaves - 1) / (32 * kAttnWaves);
    });
    if (units < 0 || units * p.args.kv_heads >= (1ll << 31)) return C3_E_UNSUPPORTED;
    p.args.units = FastDiv((uint32_t)(units < 1 ? 1 : units));
    if (units > 0 && p.seqs != nullptr) {
        if (stage_bytes(table, p.seqs, sizeof(AttnSeq) * (size_t)a->batch, s) != hipSuccess) return C3_E_HIP;
        p.table.staged = reinterpret_cast<const AttnSeq*>(table);
    }
    return C3_OK;
}

template <typename T, int DP>
hipError_t launch_dq(const AttnPlan& p, hipStream_t s) {
    attn_dq_kernel<T, DP><<<dim3(p.args.units.d * p.args.kv_heads), dim3(kAttnThreads), 0, s>>>(p.args, p.table);
    return hipGetLastError();
}
template <typename T, int DP>
hipError_t launch_dkv(const AttnPlan& p, hipStream_t s) {
    attn_dkv_kernel<T, DP><<<dim3(p.args.units.d * p.args.kv_heads), dim3(kAttnThreads), 0, s>>>(p.args, p.table);
    return hipGetLastError();
}

}  // namespace
}  // namespace c3

extern "C" {

size_t c3_attention_grad_workspace_size(const c3_attention_t* a) {
    try {
        c3::AttnPlan p;
        if (c3::attn_plan(a, p) != C3_OK) return 0;
        return c3::GradSpace(a, p).total;
    } catch (...) {
        return 0;
    }
}

int c3_attention_grad(const c3_attention_t* a, const c3_attn_tensor_t* dout,
                      const c3_attn_tensor_t* q, const c3_attn_tensor_t* k,
                      const c3_attn_tensor_t* v, const c3_attn_tensor_t* out, const float* lse,
                      const c3_attn_tensor_t* dq, const c3_attn_tensor_t* dk,
                      const c3_attn_tensor_t* dv, void* ws, size_t ws_bytes, c3_stream_t stream) {
    using namespace c3;
    try {
        AttnPlan p;
        int rc = attn_plan(a, p);
        if (rc != C3_OK) return rc;
        AttnArgs& g = p.args;
        if ((rc = attn_tensor(dout, p, false, g.d_o)) != C3_OK) return rc;
        if ((rc = attn_tensor(q, p, false, g.q)) != C3_OK) return rc;
        if ((rc = attn_tensor(k, p, true, g.k)) != C3_OK) return rc;
        if ((rc = attn_tensor(v, p, true, g.v)) != C3_OK) return rc;
        if ((rc = attn_tensor(out, p, false, g.o)) != C3_OK) return rc;
        if ((rc = attn_tensor(dq, p, false, g.dq)) != C3_OK) return rc;
        if ((rc = attn_tensor(dk, p, true, g.dk)) != C3_OK) return rc;
        if ((rc = attn_tensor(dv, p, true, g.dv)) != C3_OK) return rc;
        if (p.rows > 0 && lse == nullptr) return C3_E_INVAL;
        if ((uintptr_t)lse % 4 != 0) return C3_E_ALIGN;
        const GradSpace sp(a, p);
        if (ws == nullptr || (uintptr_t)ws % 256 != 0 || ws_bytes < sp.total) return C3_E_WORKSPACE;
        char* base = static_cast<char*>(ws);
        g.lse = const_cast<float*>(lse);
        g.lse2 = reinterpret_cast<float*>(base + sp.lse2);
        g.delta = reinterpret_cast<float*>(base + sp.delta);
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        const bool bf16 = a->dtype == C3_BF16, wide = a->dim > 64;
        hipError_t e = hipSuccess;
        if (p.rows > 0) {
            if ((rc = number_units(a, p, base + sp.table_q, false, s)) != C3_OK) return rc;
            e = bf16 ? (wide ? launch_dq<__bf16, 128>(p, s) : launch_dq<__bf16, 64>(p, s))
                     : (wide ? launch_dq<_Float16, 128>(p, s) : launch_dq<_Float16, 64>(p, s));
            if (e != hipSuccess) return C3_E_HIP;
        }
        if (p.key_rows > 0) {
            if ((rc = number_units(a, p, base + sp.table_k, true, s)) != C3_OK) return rc;
            e = bf16 ? (wide ? launch_dkv<__bf16, 128>(p, s) : launch_dkv<__bf16, 64>(p, s))
                     : (wide ? launch_dkv<_Float16, 128>(p, s) : launch_dkv<_Float16, 64>(p, s));
        }
        return e == hipSuccess ? C3_OK : C3_E_HIP;
    } catch (...) {
        return C3_E_INVAL;
    }
}

}  // extern "C"
