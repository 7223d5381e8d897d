// Attention's forward (include/c3_replay.h): softmax(scale q k^T) v and the rows'
// log-sum-exp in one pass over keys and values.
//
// A wave holds 32 rows' queries as B operands and walks the keys; scores come out
// with a query per lane and half of the keys in its registers, so the running
// maximum and sum of a row are lane values (one exchange with the other half), and
// the probabilities are the next product's operand where they are.  Scores are
// kept in units of the raw product; exp is exp2 of (s - m) scale log2 e, one fma
// and one v_exp_f32 an element.  2 x 4,096 causal tokens of 32 heads of 128: 310 us,
// 888 TFLOP/s (a large library product 1,290).  Matrix units are busy 45% of the time,
// vector units 44%, at a clock of 1.9 GHz; reading operands further ahead of their products
// (scheduling barriers) or raising the waves' priority there changed nothing once the
// clock has settled.  Heads of 64 have half the products for the same exponentials:
// packed documents of 8,192 tokens, 32 heads, window 1,024: 82 us, 565 TFLOP/s.
#include <algorithm>
#include <new>

#include "c3_attention.h"

namespace c3 {
namespace {

constexpr int kKeys = 64;           // keys of a tile
// Parts of a walk: at most, and those that one wave joins for a row.
constexpr int kMostParts = 256, kFewParts = 16;
// Workgroups of the kernel for few rows that run at a time: two a compute unit.
constexpr int64_t kTokenSlots = 512;

// Parts that a walk over k_len keys is divided into.
__device__ __forceinline__ int key_parts(const AttnArgs& a, int k_len) {
    return a.split_keys ? max(1, (k_len + a.split_keys - 1) / a.split_keys) : 1;
}

// Maximum (scaled, in powers of two) and sum of a row's part; the first part also
// marks those that the row's sequence does not have.
__device__ __forceinline__ void write_part_stats(const AttnArgs& a, int64_t row, int part, int parts, float mc,
                                                 float l) {
    float2* to = reinterpret_cast<float2*>(a.part_ml) + row;
    to[part * a.side[0].part_rows] = make_float2(mc, l);
    if (part == 0)
        for (int p = parts; p < (int)a.side[0].splits.d; ++p) to[p * a.side[0].part_rows] = make_float2(0.0f, 0.0f);
}
// Columns 32 db .. of a row's part.
__device__ __forceinline__ void write_part(const AttnArgs& a, int64_t row, int part, int db, int h,
                                           const f32x16& x) {
    float* to = a.side[0].part + (part * a.side[0].part_rows + row) * a.dim;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int d = db * 32 + q * 8 + h * 4;
        if (d < a.dim) *reinterpret_cast<f32x4*>(to + d) = f32x4{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
    }
}
// Columns 32 db .. of a row of the output; zeros where it saw nothing.
template <typename T>
__device__ __forceinline__ void write_out(char* out, int db, int h, int dim, const f32x16& x, float f, bool some) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int d = db * 32 + q * 8 + h * 4;
        if (d >= dim) continue;
        T e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = some ? (T)(x[4 * q + i] * f) : (T)0.0f;
        u32x2 w;
        __builtin_memcpy(&w, e, 8);
        *reinterpret_cast<u32x2*>(out + d * 2) = w;
    }
}

// A unit: the output of a tile of rows.  Returns whether a tile of keys that the mask
// cuts held an infinity or NaN among its values, which only CAREFUL keeps from rows
// that do not see it.
template <typename T, int DP, bool CAREFUL>
__device__ __forceinline__ bool forward_unit(const AttnArgs& a, const AttnTable& tab, uint32_t block) {
    constexpr int KS = DP / 16, NDB = DP / 32, kSub = 32 * DP * 2;
    constexpr int kRows = 32 * kAttnWaves;
    using L = TileLoads<DP, kKeys>;
    __shared__ __attribute__((aligned(1024))) char k0[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char v0[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char k1[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char v1[L::kBytes];
    __shared__ T words[CAREFUL ? kAttnWaves : 1][32 * 32];        // for the masked product

    const AttnUnit w = attn_unit(a, tab, 0, block);
    const int G = (int)a.group.d;
    const int n_rows = w.q_pad * G, off = w.k_len - w.q_len;
    const int tiles = (n_rows + kRows - 1) / kRows;
    // the last queries see the most keys: they go first
    const int parts = key_parts(a, w.k_len), nth = parts > 1 ? (int)w.unit / parts : (int)w.unit;
    const int part = (int)w.unit - nth * parts, tile = a.causal ? tiles - 1 - nth : nth;
    const int row0 = tile * kRows;
    const int lane = threadIdx.x & 63, h = lane >> 5, c = lane & 31;
    const int wave = threadIdx.x >> 6;

    // the keys that any row of the tile sees
    const int first = (int)a.group.quot(row0);
    const int last = min((int)a.group.quot(min(row0 + kRows, n_rows) - 1), w.q_len - 1);
    int lo = 0, hi = w.k_len;
    if (a.causal) hi = min(hi, last + off + 1);
    if (a.window) lo = max(lo, first + off - a.window + 1);
    if (first >= w.q_len) hi = 0;
    if (a.split_keys) {
        lo = max(lo, part * a.split_keys);
        hi = min(hi, part * a.split_keys + a.split_keys);
    }
    const int t0 = lo / kKeys, t1 = hi > lo ? (hi + kKeys - 1) / kKeys : t0;

    // the lane's row and the keys that it sees; a row that does not exist hides
    // nothing, so that it makes no tile a masked one
    const int row = row0 + wave * 32 + c;
    const int pos = (int)a.group.quot(row), head = w.hk * G + row - pos * G;
    const bool there = row < n_rows, valid = there && pos < w.q_len;
    const int see_hi = !valid ? INT32_MAX : a.causal ? min(w.k_len, pos + off + 1) : w.k_len;
    const int see_lo = valid && a.window ? pos + off - a.window + 1 : 0;
    u32x4 qf[KS];
    load_row<DP>(qf, seq_base(a.q, a.packed, w.b, w.q_start, head) + (int64_t)pos * a.q.st, valid, a.dim);

    TileReads<DP> rd;
    const TokenOffsets<DP, kKeys> k_off(a.k.st, a.dim), v_off(a.v.st, a.dim);
    const char* kb = seq_base(a.k, a.packed, w.b, w.k_start, w.hk);
    const char* vb = seq_base(a.v, a.packed, w.b, w.k_start, w.hk);
    const float cs = a.scale * kLog2e;

    f32x16 acc[NDB] = {};
    uint32_t bad = 0;
    float m = -__builtin_inff(), l = 0.0f;

    auto load = [&](int t, char* kt, char* vt) {
        const int key = t * kKeys;
        load_tile<DP, kKeys>(kb + (int64_t)key * a.k.st, a.k.st, a.dim, w.k_len - key, k_off, kt);
        load_tile<DP, kKeys>(vb + (int64_t)key * a.v.st, a.v.st, a.dim, w.k_len - key, v_off, vt);
    };
    auto step = [&](int t, const char* kt, const char* vt) {
        const int key0 = t * kKeys;
        if (!__any(valid && key0 < see_hi && key0 + kKeys > see_lo)) return;
        const bool masked = __any(key0 + kKeys > see_hi || key0 < see_lo);
        f32x16 s[2] = {};
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                s[n] = mfma<T>(rd.along(kt + n * kSub, ks), qf[ks], s[n]);
        uint32_t seen[2] = {0, 0};
        if (masked) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = key0 + n * 32 + (i >> 2) * 8 + h * 4 + (i & 3);
                    const bool see = key < see_hi && key >= see_lo;
                    seen[n] |= see ? 1u << i : 0u;
                    s[n][i] = see ? s[n][i] : -__builtin_inff();
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
        top = fmaxf(top, __shfl_xor(top, 32));
        // The reference m follows the maximum only where a score would exceed
        // 2^8 of it: sums and products keep their relative precision, and the
        // accumulators are rescaled in few steps.
        if (__any((top - m) * cs > 8.0f)) {
            const float next = (top - m) * cs > 8.0f ? top : m;     // each row by itself
            const float f = next == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((m - next) * cs);
            m = next;
            l *= f;
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[db][i] *= f;
        }
        const float mc = m == -__builtin_inff() ? 0.0f : m * cs;
        float sum = 0.0f;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], cs, -mc));
                sum += s[n][i];
            }
        l += sum;
        if (masked) {
            const uint32_t here =
                tile_not_finite<T>(2 * KS, [&](int i) { return rd.along(vt + i / KS * kSub, i % KS); });
            bad |= here;
            if constexpr (CAREFUL) {
                if (__any(here != 0)) {
#pragma unroll
                    for (int n = 0; n < 2; ++n)
                        masked_product<T, NDB>(acc, s[n], seen[n], words[wave],
                                               [&](int k, int d) { return rd.four(vt + n * kSub, k, d); },
                                               [&](int j, int db) {
                                                   return rd.across(vt + n * kSub + j * 16 * DP * 2, db);
                                               });
                    return;
                }
            }
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const u32x4 p = operand<T>(s[n], j);
#pragma unroll
                for (int db = 0; db < NDB; ++db)
                    acc[db] = mfma<T>(rd.across(vt + n * kSub + j * 16 * DP * 2, db), p, acc[db]);
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

    l += __shfl_xor(l, 32);
    if (!there) return bad != 0;
    const float mc = m == -__builtin_inff() ? 0.0f : m * cs;
    const int64_t at = seq_row(a, w) + (int64_t)pos * a.heads + head;
    // a row that saw nothing (l = 0) and one of the padding: zeros and -inf
    const bool some = valid && l != 0.0f;
    if (a.split_keys) {
        if (h == 0) write_part_stats(a, at, part, parts, mc, some ? l : 0.0f);
        if (some)
#pragma unroll
            for (int db = 0; db < NDB; ++db) write_part(a, at, part, db, h, acc[db]);
        return bad != 0;
    }
    const float f = some ? 1.0f / l : 0.0f;
    char* out = seq_base(a.o, a.packed, w.b, w.q_start, head) + (int64_t)pos * a.o.st;
#pragma unroll
    for (int db = 0; db < NDB; ++db) write_out<T>(out, db, h, a.dim, acc[db], f, some);
    if (h == 0) a.lse[at] = some ? (mc + __log2f(l)) * kLn2 : -__builtin_inff();
    return bad != 0;
}

template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, 2) void attn_forward_kernel(AttnArgs a, AttnTable tab) {
    const bool bad = forward_unit<T, DP, false>(a, tab, blockIdx.x);
    if (a.causal || a.window) {
        const int any = __syncthreads_or(bad);
        if (threadIdx.x == 0) a.side[0].marks[blockIdx.x] = any;
    }
}
template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, 1) void attn_forward_careful_kernel(AttnArgs a, AttnTable tab,
                                                                               uint32_t blocks) {
    repeat_marked(a.side[0].marks, blocks, blockIdx.x, gridDim.x,
                  [&](uint32_t unit) { forward_unit<T, DP, true>(a, tab, unit); });
}

template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, 1) void attn_forward_direct_kernel(AttnArgs a, AttnTable tab) {
    forward_unit<T, DP, true>(a, tab, blockIdx.x);
}

// Few rows against many keys, as new tokens against a cache: the keys are read
// once and bound it.  The 32 rows of a workgroup stand in every one of its four
// waves, which share out the keys 32 at a time, each through buffers of its own, so
// that no wave waits for another before the end; there their maxima and sums are
// joined in LDS.  Long caches are divided among workgroups as well.  One buffer each
// for keys and values, refilled as soon as its product has read it, lets two
// workgroups share a compute unit: one starts or ends while the other streams
// (16 caches of 1 to 32,768 tokens, 8 key heads of 128: 115 us with the joining, 4.9
// TB/s; two buffers each and one workgroup 124).
template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, 2) void attn_tokens_kernel(AttnArgs a, AttnTable tab) {
    constexpr int KS = DP / 16, NDB = DP / 32, kSub = 32 * DP * 2;
    __shared__ __attribute__((aligned(1024))) char k0[kAttnWaves * kSub];
    __shared__ __attribute__((aligned(1024))) char v0[kAttnWaves * kSub];
    __shared__ T words[kAttnWaves][32 * 32];      // for the masked product
    __shared__ float stats[2][kAttnWaves][64];

    const AttnUnit w = attn_unit(a, tab, 0, blockIdx.x);
    const int G = (int)a.group.d;
    const int n_rows = w.q_pad * G, off = w.k_len - w.q_len;
    const int parts = key_parts(a, w.k_len), tile = parts > 1 ? (int)w.unit / parts : (int)w.unit;
    const int part = (int)w.unit - tile * parts, row0 = tile * 32;
    const int lane = threadIdx.x & 63, h = lane >> 5, c = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    const int first = (int)a.group.quot(row0);
    const int last = min((int)a.group.quot(min(row0 + 32, n_rows) - 1), w.q_len - 1);
    int lo = 0, hi = w.k_len;
    if (a.causal) hi = min(hi, last + off + 1);
    if (a.window) lo = max(lo, first + off - a.window + 1);
    if (first >= w.q_len) hi = 0;
    if (a.split_keys) {
        lo = max(lo, part * a.split_keys);
        hi = min(hi, part * a.split_keys + a.split_keys);
    }
    // blocks of 32 keys, this wave's every fourth
    const int t0 = lo / 32 + wave, t1 = hi > lo ? (hi + 31) / 32 : 0;

    const int row = row0 + c;
    const int pos = (int)a.group.quot(row), head = w.hk * G + row - pos * G;
    const bool there = row < n_rows, valid = there && pos < w.q_len;
    const int see_hi = !valid ? INT32_MAX : a.causal ? min(w.k_len, pos + off + 1) : w.k_len;
    const int see_lo = valid && a.window ? pos + off - a.window + 1 : 0;
    u32x4 qf[KS];
    load_row<DP>(qf, seq_base(a.q, a.packed, w.b, w.q_start, head) + (int64_t)pos * a.q.st, valid, a.dim);

    const TileReads<DP> rd;
    // byte offsets of the lane's pieces of 32 keys, as TokenOffsets for one wave
    constexpr int kPieces = DP / 8, kStepRows = 64 / kPieces, kLoads = 32 / kStepRows;
    uint32_t k_off[kLoads], v_off[kLoads];
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
        const int r = n * kStepRows + lane / kPieces, p = (lane % kPieces) ^ swizzle<DP>(r);
        k_off[n] = p * 8 < a.dim ? (uint32_t)(r * (int)a.k.st + p * 16) : 0xFFFFFF00u;
        v_off[n] = p * 8 < a.dim ? (uint32_t)(r * (int)a.v.st + p * 16) : 0xFFFFFF00u;
    }
    const char* kb = seq_base(a.k, a.packed, w.b, w.k_start, w.hk);
    const char* vb = seq_base(a.v, a.packed, w.b, w.k_start, w.hk);
    const float cs = a.scale * kLog2e;

    f32x16 acc[NDB] = {};
    float m = -__builtin_inff(), l = 0.0f;

    // 32 rows of keys or values to the wave's buffer
    auto load = [&](int t, const char* from, int64_t st, const uint32_t (&off)[kLoads], char* to) {
        const int rows = min(w.k_len - t * 32, 32);
        const uint32_t bytes = (uint32_t)((rows - 1) * (int)st) + a.dim * 2;
        const char* first_row = from + (int64_t)t * 32 * st;
#pragma unroll
        for (int n = 0; n < kLoads; ++n) load_piece_lds(first_row, bytes, off[n], to + wave * kSub + n * 1024);
    };
    // The wave's own loads, in order: all but the latest kLoads have landed.
    auto landed = [&](bool more) {
        if (more)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    // reads of the buffer that is filled next have ended: their values are used
    auto read = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
    const char *kt = k0 + wave * kSub, *vt = v0 + wave * kSub;
    // One block of keys; the next block's keys are on their way during the softmax and
    // the second product, its values during the first.
    auto step = [&](int t, bool more) {
        const int key0 = t * 32;
        landed(true);
        const bool masked = __any(key0 + 32 > see_hi || key0 < see_lo);
        f32x16 s = {};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = mfma<T>(rd.along(kt, ks), qf[ks], s);
        read();
        if (more) load(t + kAttnWaves, kb, a.k.st, k_off, k0);
        uint32_t seen = 0;
        if (masked) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = key0 + (i >> 2) * 8 + h * 4 + (i & 3);
                const bool see = key < see_hi && key >= see_lo;
                seen |= see ? 1u << i : 0u;
                s[i] = see ? s[i] : -__builtin_inff();
            }
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any((top - m) * cs > 8.0f)) {         // as in the kernel above
            const float next = (top - m) * cs > 8.0f ? top : m;     // each row by itself
            const float f = next == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((m - next) * cs);
            m = next;
            l *= f;
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[db][i] *= f;
        }
        const float mc = m == -__builtin_inff() ? 0.0f : m * cs;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], cs, -mc));
            l += s[i];
        }
        landed(more);
        if (masked && __any(tile_not_finite<T>(KS, [&](int ks) { return rd.along(vt, ks); }) != 0)) {
            masked_product<T, NDB>(acc, s, seen, words[wave], [&](int k, int d) { return rd.four(vt, k, d); },
                                   [&](int j, int db) { return rd.across(vt + j * 16 * DP * 2, db); });
            return;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const u32x4 p = operand<T>(s, j);
#pragma unroll
            for (int db = 0; db < NDB; ++db) acc[db] = mfma<T>(rd.across(vt + j * 16 * DP * 2, db), p, acc[db]);
        }
    };
    if (t0 < t1) {
        load(t0, kb, a.k.st, k_off, k0);
        load(t0, vb, a.v.st, v_off, v0);
    }
    for (int t = t0; t < t1; t += kAttnWaves) {
        const bool more = t + kAttnWaves < t1;
        step(t, more);
        read();
        if (more) load(t + kAttnWaves, vb, a.v.st, v_off, v0);
    }
    l += __shfl_xor(l, 32);

    // join the four waves: maxima and sums first, then the rescaled accumulators,
    // block db of them by wave db, in the order of the waves
    const float mine = m == -__builtin_inff() ? m : m * cs;
    stats[0][wave][lane] = mine;
    stats[1][wave][lane] = l;
    __syncthreads();
    float top = stats[0][0][lane];
#pragma unroll
    for (int v = 1; v < kAttnWaves; ++v) top = fmaxf(top, stats[0][v][lane]);
    const float mc = top == -__builtin_inff() ? 0.0f : top;
    float total = 0.0f;
#pragma unroll
    for (int v = 0; v < kAttnWaves; ++v)
        total = fmaf(stats[1][v][lane], __builtin_amdgcn_exp2f(stats[0][v][lane] - mc), total);
    const float f = __builtin_amdgcn_exp2f(mine - mc);
    // [wave][db][register / 4][lane] of four floats, over the buffers (a power of two
    // apart in all: 32 KiB for 64 columns, 64 KiB for 128)
    constexpr int kHalf = kAttnWaves * kSub / 16;       // four-float words of one buffer
    auto cell = [&](int v, int db, int q) -> f32x4* {
        const int i = ((v * NDB + db) * 4 + q) * 64 + lane;
        return reinterpret_cast<f32x4*>(i < kHalf ? k0 : v0) + (i < kHalf ? i : i - kHalf);
    };
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            f32x4 x;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = acc[db][4 * q + i] * f;
            *cell(wave, db, q) = x;
        }
    __syncthreads();
    const int64_t at = seq_row(a, w) + (int64_t)pos * a.heads + head;
    const bool some = valid && total != 0.0f;
    if (there && wave == 0 && h == 0) {
        if (a.split_keys)
            write_part_stats(a, at, part, parts, mc, some ? total : 0.0f);
        else
            a.lse[at] = some ? (mc + __log2f(total)) * kLn2 : -__builtin_inff();
    }
    if (wave >= NDB || !there) return;
    f32x16 sum = {};
#pragma unroll
    for (int v = 0; v < kAttnWaves; ++v)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 x = *cell(v, wave, q);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[4 * q + i] += x[i];
        }
    if (a.split_keys) {
        if (some) write_part(a, at, part, wave, h, sum);
        return;
    }
    char* out = seq_base(a.o, a.packed, w.b, w.q_start, head) + (int64_t)pos * a.o.st;
    write_out<T>(out, wave, h, a.dim, sum, some ? 1.0f / total : 0.0f, some);
}

// Joins the parts of divided walks.  A wave takes a row: lane p the maximum and sum
// of part p (kFewParts at most), then each lane two elements of the row.
template <typename T>
__global__ __launch_bounds__(256) void attn_join_parts_kernel(AttnArgs a, int64_t rows, int parts, FastDiv tokens) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    float m = -__builtin_inff(), l = 0.0f;
    if (lane < parts) {
        const float2 x = reinterpret_cast<const float2*>(a.part_ml)[lane * rows + row];
        m = x.x;
        l = x.y;
    }
    if (l == 0.0f) m = -__builtin_inff();
    float top = m;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const bool none = top == -__builtin_inff() && !__any(l != 0.0f);
    const float f = none || l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(m - top);
    float total = f * l;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) total += __shfl_xor(total, d);
    const int64_t token = row / a.heads, b = token / tokens.d;
    const int head = (int)(row - token * a.heads);
    if (lane == 0) a.lse[row] = none ? -__builtin_inff() : (top + __log2f(total)) * kLn2;
    // Every lane stays to the end, whatever the head's size: lane p has part p's factor.
    // Those behind the head take its last elements again.
    float x = 0.0f, y = 0.0f;
    const uint64_t full = __ballot(l != 0.0f);
    const float* from = a.side[0].part + row * a.dim + min(2 * lane, a.dim - 2);
    for (int p0 = 0; p0 < parts; p0 += 8) {         // eight parts' loads together
        float2 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = *reinterpret_cast<const float2*>(from + min(p0 + j, parts - 1) * rows * a.dim);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (p0 + j >= parts || !((full >> (p0 + j)) & 1)) continue;      // not written
            const float g = __shfl(f, p0 + j);
            x = fmaf(v[j].x, g, x);
            y = fmaf(v[j].y, g, y);
        }
    }
    if (2 * lane >= a.dim) return;
    const float inv = none ? 0.0f : 1.0f / total;
    T e[2] = {(T)(none ? 0.0f : x * inv), (T)(none ? 0.0f : y * inv)};
    uint32_t two;
    __builtin_memcpy(&two, e, 4);
    *reinterpret_cast<uint32_t*>(a.o.ptr + b * a.o.sb + (token - b * tokens.d) * a.o.st + head * a.o.sh + lane * 4) = two;
}

// The same with a workgroup a row, for many parts (256 at most): thread p the maximum
// and sum of part p, then each wave a quarter of the parts, joined in the waves' order.
template <typename T>
__global__ __launch_bounds__(256) void attn_join_many_kernel(AttnArgs a, int64_t rows, int parts, FastDiv tokens) {
    __shared__ float factor[256], tops[4], sums[4];
    __shared__ float2 partial[4][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x;
    float m = -__builtin_inff(), l = 0.0f;
    if (tid < parts) {
        const float2 x = reinterpret_cast<const float2*>(a.part_ml)[tid * rows + row];
        m = x.x;
        l = x.y;
    }
    if (l == 0.0f) m = -__builtin_inff();
    float top = m;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (lane == 0) tops[wave] = top;
    const bool none = !__syncthreads_or(l != 0.0f);
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float f = l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(m - top);
    factor[tid] = l == 0.0f ? -1.0f : f;            // -1: not written
    float total = f * l;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) total += __shfl_xor(total, d);
    if (lane == 0) sums[wave] = total;
    __syncthreads();
    total = sums[0] + sums[1] + sums[2] + sums[3];
    float x = 0.0f, y = 0.0f;
    const int each = (parts + 3) / 4, end = min(wave * each + each, parts);
    if (2 * lane < a.dim) {
        const float* from = a.side[0].part + row * a.dim + 2 * lane;
        for (int p0 = wave * each; p0 < end; p0 += 8) {
            float2 v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] = *reinterpret_cast<const float2*>(from + min(p0 + j, end - 1) * rows * a.dim);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float g = p0 + j < end ? factor[p0 + j] : -1.0f;
                if (g < 0.0f) continue;
                x = fmaf(v[j].x, g, x);
                y = fmaf(v[j].y, g, y);
            }
        }
    }
    partial[wave][lane] = make_float2(x, y);
    __syncthreads();
    if (wave != 0) return;
    const int64_t token = row / a.heads, b = token / tokens.d;
    const int head = (int)(row - token * a.heads);
    if (lane == 0) a.lse[row] = none ? -__builtin_inff() : (top + __log2f(total)) * kLn2;
    if (2 * lane >= a.dim) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) {
        x += partial[w][lane].x;
        y += partial[w][lane].y;
    }
    const float inv = none ? 0.0f : 1.0f / total;
    T e[2] = {(T)(none ? 0.0f : x * inv), (T)(none ? 0.0f : y * inv)};
    uint32_t two;
    __builtin_memcpy(&two, e, 4);
    *reinterpret_cast<uint32_t*>(a.o.ptr + b * a.o.sb + (token - b * tokens.d) * a.o.st + head * a.o.sh + lane * 4) = two;
}

template <typename T, int DP>
hipError_t launch_forward(const AttnPlan& p, bool tokens, hipStream_t s) {
    const dim3 grid(attn_blocks(p, 0)), block(kAttnThreads);
    if (tokens) {
        attn_tokens_kernel<T, DP><<<grid, block, 0, s>>>(p.args, p.table);
    } else if (attn_direct(p, 0)) {
        attn_forward_direct_kernel<T, DP><<<grid, block, 0, s>>>(p.args, p.table);
    } else {
        attn_forward_kernel<T, DP><<<grid, block, 0, s>>>(p.args, p.table);
        if ((p.args.causal || p.args.window) && p.key_rows > 0)
            attn_forward_careful_kernel<T, DP><<<dim3(32), block, 0, s>>>(p.args, p.table, grid.x);
    }
    if (p.args.split_keys) {
        const int parts = (int)p.args.side[0].splits.d;
        const FastDiv q_tokens((uint32_t)p.args.q_tokens);
        if (parts > kFewParts)
            attn_join_many_kernel<T><<<dim3((unsigned)p.rows), dim3(256), 0, s>>>(p.args, p.rows, parts, q_tokens);
        else
            attn_join_parts_kernel<T><<<dim3((unsigned)((p.rows + 3) / 4)), dim3(256), 0, s>>>(p.args, p.rows, parts,
                                                                                            q_tokens);
    }
    return hipGetLastError();
}

inline uint64_t align256(uint64_t x) { return (x + 255) / 256 * 256; }

// How a call's rows and keys are divided: 32 rows a workgroup where no sequence and
// key head has more, 128 otherwise; and where that gives too few workgroups for the
// compute units, keys in parts of split_keys, whose results a further kernel joins.
struct ForwardShape {
    bool tokens;
    int64_t rows, split_keys, parts;
    uint64_t table, marks, part, part_ml, total;
    bool fits;
    ForwardShape(const c3_attention_t* a, AttnPlan& p) {
        const int64_t group = p.args.group.d, kv = p.args.kv_heads;
        tokens = p.max_q * group <= 32;
        rows = tokens ? 32 : 32 * kAttnWaves;
        auto units = [&](int64_t split) {
            return kv * attn_number(p, a->batch, 0, [&](int64_t nq, int64_t nk, int64_t) {
                const int64_t t = (nq * group + rows - 1) / rows;
                return split ? t * std::max<int64_t>(1, (nk + split - 1) / split) : t;
            }, split != 1);
        };
        split_keys = 0;
        parts = 1;
        const int64_t n = units(0), all = std::max<int64_t>(units(1), 1);       // all: keys times tiles of rows
        const int64_t least = tokens ? 256 : 512;
        auto whole = [&](int64_t keys) {        // in whole tiles, and no more parts than can be joined
            keys = std::max({keys, least, (p.max_k + kMostParts - 1) / kMostParts});
            return (keys + 127) / 128 * 128;
        };
        if (n > 0 && p.max_k > least && tokens && n < 4 * kTokenSlots) {
            // The cheapest of a few divisions, in keys' time.  A workgroup costs kFixed
            // beside its keys and joining costs kJoin; one round of workgroups lasts as long
            // as its longest, more of them as long as the mean and half of the longest.
            // With one workgroup a compute unit, us at 256, 512 and 768 of them: 8 caches of
            // 8,192 tokens and 8 heads of 128 52, 56, 62; one of 32,768 tokens 31, 35, 41;
            // 16 of 1 to 32,768 tokens 152, 134, 118.  By this rule: 53, 31 and 115.
            constexpr int64_t kFixed = 100, kJoin = 250;
            auto cost = [&](int64_t split) {
                const int64_t u = units(split), longest = split ? std::min(split, p.max_k) : p.max_k;
                if (u < 0) return INT64_MAX;
                const int64_t join = split ? kJoin : 0;
                return u <= kTokenSlots ? longest + kFixed + join
                                        : (all + kFixed * u) / kTokenSlots + longest / 2 + join;
            };
            int64_t best = cost(0);
            for (const int64_t twelfths : {3, 4, 6, 8, 12, 18, 24}) {
                const int64_t split = whole(all * twelfths / 12 / kTokenSlots), c = cost(split);
                if (split < p.max_k && c < best) best = c, split_keys = split;
            }
        } else if (n > 0 && n < 512 && p.max_k > least && !tokens) {
            split_keys = whole(all / 512);              // as many keys to each of 512 workgroups
        }
        if (split_keys) parts = (p.max_k + split_keys - 1) / split_keys;
        if (parts < 2) split_keys = 0, parts = 1;
        const int64_t blocks = units(split_keys);
        fits = blocks >= 0;
        uint64_t at = 0;
        auto take = [&at](uint64_t bytes) { const uint64_t r = at; at = align256(at + bytes); return r; };
        table = take(attn_table_bytes(a));
        marks = take(fits && !tokens ? 4 * (uint64_t)blocks : 0);
        part = take(split_keys ? 4 * (uint64_t)(parts * p.rows * p.args.dim) : 0);
        part_ml = take(split_keys ? 8 * (uint64_t)(parts * p.rows) : 0);
        total = std::max<uint64_t>(at, 256);
    }
};

}  // namespace

size_t attn_table_bytes(const c3_attention_t* a) {
    return a->q_lens != nullptr && a->batch > kAttnArgSeqs ? align256(sizeof(AttnSeq) * (size_t)a->batch) : 0;
}

int attn_stage(const c3_attention_t* a, AttnPlan& p, char* to, hipStream_t s) {
    if (p.seqs == nullptr) return C3_OK;
    // A captured fetch would read its pinned slot again at every replay, when the slot
    // holds what a later call staged there.
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(s, &status) != hipSuccess) return C3_E_HIP;
    if (status != hipStreamCaptureStatusNone) return C3_E_UNSUPPORTED;
    if (stage_bytes(to, p.seqs, sizeof(AttnSeq) * (size_t)a->batch, s) != hipSuccess) return C3_E_HIP;
    p.table.staged = reinterpret_cast<const AttnSeq*>(to);
    return C3_OK;
}

int attn_plan(const c3_attention_t* a, AttnPlan& p) {
    if (a == nullptr || a->batch < 0 || a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads != 0 ||
        a->heads > 65536 || a->dim < 1 || a->q_tokens < 0 || a->k_tokens < 0 || a->window < 0 ||
        !(a->scale > 0.0f) || !(a->scale - a->scale == 0.0f))
        return C3_E_INVAL;
    if ((a->dtype != C3_BF16 && a->dtype != C3_F16) || a->dim % 8 != 0 || a->dim > 128)
        return C3_E_UNSUPPORTED;
    if ((a->q_lens == nullptr) != (a->k_lens == nullptr) || (a->packed && a->q_lens == nullptr && a->batch > 0))
        return C3_E_INVAL;
    if (a->packed && a->batch == 0 && (a->q_tokens != 0 || a->k_tokens != 0)) return C3_E_INVAL;
    // positions, rows of a group and their sums with a window stay in 32 bits
    const int64_t most = 1ll << 29;
    if (a->q_tokens >= most / (a->heads / a->kv_heads) || a->k_tokens >= most) return C3_E_UNSUPPORTED;
    AttnArgs& g = p.args;
    g.heads = a->heads;
    g.kv_heads = a->kv_heads;
    g.dim = a->dim;
    g.causal = a->causal != 0;
    g.window = std::min(a->window, 1 << 29);      // every key there can be
    g.packed = a->packed != 0;
    g.q_tokens = (int32_t)a->q_tokens;
    g.k_tokens = (int32_t)a->k_tokens;
    g.scale = a->scale;
    g.group = FastDiv((uint32_t)(a->heads / a->kv_heads));
    g.kv = FastDiv((uint32_t)a->kv_heads);
    g.batch = FastDiv((uint32_t)std::max(a->batch, 1));
    p.table.n = 0;
    p.table.staged = nullptr;
    p.max_q = a->q_tokens;
    p.max_k = a->k_tokens;
    const int64_t seqs = a->packed ? 1 : a->batch;
    if (seqs > 0 && (a->q_tokens * a->heads >= (1ll << 40) / seqs || a->k_tokens * a->kv_heads >= (1ll << 40) / seqs))
        return C3_E_UNSUPPORTED;
    p.rows = seqs * a->q_tokens * a->heads;
    p.key_rows = seqs * a->k_tokens * a->kv_heads;
    if (a->q_lens == nullptr || a->batch == 0) return C3_OK;
    if (a->batch > kAttnArgSeqs) {
        p.seqs = new (std::nothrow) AttnSeq[a->batch];
        if (p.seqs == nullptr) return C3_E_INVAL;
    }
    AttnSeq* s = p.list();
    int64_t nq = 0, nk = 0;
    p.max_q = p.max_k = 0;
    for (int i = 0; i < a->batch; ++i) {
        const int64_t q = a->q_lens[i], k = a->k_lens[i];
        if (q < 0 || k < 0 || (!a->packed && (q > a->q_tokens || k > a->k_tokens))) return C3_E_INVAL;
        if (a->packed && (nq + q > a->q_tokens || nk + k > a->k_tokens)) return C3_E_INVAL;
        s[i] = AttnSeq{i, a->packed ? (int32_t)nq : 0, (int32_t)q, a->packed ? (int32_t)nk : 0, (int32_t)k, {0, 0}};
        nq += q;
        nk += k;
        p.max_q = std::max(p.max_q, q);
        p.max_k = std::max(p.max_k, k);
    }
    if (a->packed && (nq != a->q_tokens || nk != a->k_tokens)) return C3_E_INVAL;
    // the longest walks first, so that short ones fill the end
    std::stable_sort(s, s + a->batch, [](const AttnSeq& x, const AttnSeq& y) {
        return (int64_t)x.q_len * x.k_len > (int64_t)y.q_len * y.k_len;
    });
    p.table.n = a->batch;
    return C3_OK;
}

int attn_tensor(const c3_attn_tensor_t* t, const AttnPlan& p, bool keys, Tiles tiles, AttnTensor& to) {
    if (t == nullptr) return C3_E_INVAL;
    const AttnArgs& g = p.args;
    const bool none = (keys ? p.key_rows : p.rows) == 0;
    if (none) {
        to = AttnTensor{nullptr, 0, 0, 0};
        return C3_OK;
    }
    if (t->ptr == nullptr) return C3_E_INVAL;
    if ((uintptr_t)t->ptr % 16 != 0) return C3_E_ALIGN;
    // The stride of a dimension with one entry says nothing.  A row's length stands for
    // the tokens', so that rows behind a tile's only one lie behind its end.
    const int64_t entries[3] = {g.packed ? 1 : (int64_t)g.batch.d, keys ? g.k_tokens : g.q_tokens,
                                keys ? g.kv_heads : g.heads};
    int64_t stride[3] = {0, g.dim, 0};
    for (int i = 0; i < 3; ++i) {
        if (entries[i] == 1) continue;
        if (t->stride[i] < 0 || t->stride[i] >= (1ll << 40)) return C3_E_INVAL;
        if (t->stride[i] % 8 != 0) return C3_E_ALIGN;
        stride[i] = t->stride[i];
    }
    to.ptr = static_cast<char*>(t->ptr);
    to.sb = stride[0] * 2;
    to.st = stride[1] * 2;
    to.sh = stride[2] * 2;
    const int64_t span = tiles == Tiles::kNone ? 0 : to.st * 64 + (tiles == Tiles::kGroup ? to.sh * (g.group.d - 1) : 0);
    if (span >= (1ll << 31) - 4096) return C3_E_UNSUPPORTED;
    return C3_OK;
}

bool attn_overlap(std::initializer_list<const AttnTensor*> results, std::initializer_list<const AttnTensor*> inputs) {
    for (const AttnTensor* r : results) {
        if (r->ptr == nullptr) continue;
        for (const AttnTensor* t : results)
            if (t != r && t->ptr == r->ptr) return true;
        for (const AttnTensor* t : inputs)
            if (t->ptr == r->ptr) return true;
    }
    return false;
}

}  // namespace c3

extern "C" {

size_t c3_attention_workspace_size(const c3_attention_t* a) {
    try {
        c3::AttnPlan p;
        if (c3::attn_plan(a, p) != C3_OK) return 0;
        const c3::ForwardShape f(a, p);
        return f.fits ? f.total : 0;
    } catch (...) {
        return 0;
    }
}

int c3_attention(const c3_attention_t* a, const c3_attn_tensor_t* q, const c3_attn_tensor_t* k,
                 const c3_attn_tensor_t* v, const c3_attn_tensor_t* out, float* lse, void* ws,
                 size_t ws_bytes, c3_stream_t stream) {
    using namespace c3;
    try {
        AttnPlan p;
        int rc = attn_plan(a, p);
        if (rc != C3_OK) return rc;
        if ((rc = attn_tensor(q, p, false, Tiles::kNone, p.args.q)) != C3_OK) return rc;
        if ((rc = attn_tensor(k, p, true, Tiles::kHead, p.args.k)) != C3_OK) return rc;
        if ((rc = attn_tensor(v, p, true, Tiles::kHead, p.args.v)) != C3_OK) return rc;
        if ((rc = attn_tensor(out, p, false, Tiles::kNone, p.args.o)) != C3_OK) return rc;
        if (p.rows > 0 && lse == nullptr) return C3_E_INVAL;
        if ((uintptr_t)lse % 4 != 0) return C3_E_ALIGN;
        const ForwardShape f(a, p);
        if (!f.fits) return C3_E_UNSUPPORTED;
        if (ws == nullptr || (uintptr_t)ws % 256 != 0 || ws_bytes < (size_t)f.total) return C3_E_WORKSPACE;
        if (p.rows == 0) return C3_OK;
        if (attn_overlap({&p.args.o}, {&p.args.q, &p.args.k, &p.args.v})) return C3_E_INVAL;
        p.args.lse = lse;
        char* base = static_cast<char*>(ws);
        AttnSide& side = p.args.side[0];
        side.splits = FastDiv((uint32_t)f.parts);
        side.marks = reinterpret_cast<uint32_t*>(base + f.marks);
        side.part = reinterpret_cast<float*>(base + f.part);
        side.part_rows = p.rows;
        p.args.split_keys = (int32_t)f.split_keys;
        p.args.part_ml = reinterpret_cast<float*>(base + f.part_ml);
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        if ((rc = attn_stage(a, p, base + f.table, s)) != C3_OK) return rc;
        hipError_t e;
        if (a->dtype == C3_BF16)
            e = a->dim > 64 ? launch_forward<__bf16, 128>(p, f.tokens, s) : launch_forward<__bf16, 64>(p, f.tokens, s);
        else
            e = a->dim > 64 ? launch_forward<_Float16, 128>(p, f.tokens, s)
                            : launch_forward<_Float16, 64>(p, f.tokens, s);
        return e == hipSuccess ? C3_OK : C3_E_HIP;
    } catch (...) {
        return C3_E_INVAL;
    }
}

}  // extern "C"
