// Attention's forward (include/c3_replay.h): softmax(scale q k^T) v and the rows'
// log-sum-exp in one pass over keys and values.
//
// A wave holds 32 rows' queries as B operands and walks the keys; scores come out
// with a query per lane and half of the keys in its registers, so the running
// maximum and sum of a row are lane values (one exchange with the other half), and
// the probabilities are the next product's operand where they are.  Scores are
// kept in units of the raw product; exp is exp2 of (s - m) scale log2 e, one fma
// and one v_exp_f32 an element.
#include <algorithm>
#include <new>

#include "c3_attention.h"

namespace c3 {
namespace {

constexpr int kKeys = 64;           // keys of a tile

template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, 2) void attn_forward_kernel(AttnArgs a, AttnTable tab) {
    constexpr int KS = DP / 16, NDB = DP / 32, kSub = 32 * DP * 2;
    constexpr int kRows = 32 * kAttnWaves;
    using L = TileLoads<DP, kKeys>;
    __shared__ __attribute__((aligned(1024))) char k0[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char v0[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char k1[L::kBytes];
    __shared__ __attribute__((aligned(1024))) char v1[L::kBytes];
    __shared__ uint32_t special_words[NDB * kAttnThreads];

    const AttnUnit w = attn_unit(a, tab, die_order(blockIdx.x, gridDim.x));
    const int G = (int)a.group.d;
    const int n_rows = w.q_pad * G, off = w.k_len - w.q_len;
    const int tiles = (n_rows + kRows - 1) / kRows;
    // the last queries see the most keys: they go first
    const int tile = a.causal ? tiles - 1 - (int)w.unit : (int)w.unit;
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
    const Special<NDB> special(special_words);
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
            const float next = fmaxf(m, top);
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
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const u32x4 p = operand<T>(s[n], j);
                u32x4 A[NDB];
#pragma unroll
                for (int db = 0; db < NDB; ++db)
                    A[db] = rd.across(vt + n * kSub + j * 16 * DP * 2, db);
                if (masked) finite_operands<T, NDB>(A, p, seen[n] >> (8 * j), special);
#pragma unroll
                for (int db = 0; db < NDB; ++db) acc[db] = mfma<T>(A[db], p, acc[db]);
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
    l += __shfl_xor(l, 32);
    if (!there) return;
    // a row that saw nothing (l = 0) and one of the padding: zeros and -inf
    const bool some = valid && l != 0.0f;
    const float f = some ? 1.0f / l : 0.0f;
    char* out = seq_base(a.o, a.packed, w.b, w.q_start, head) + (int64_t)pos * a.o.st;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int d = db * 32 + q * 8 + h * 4;
            if (d >= a.dim) continue;
            T e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = some ? (T)(acc[db][4 * q + i] * f) : (T)0.0f;
            u32x2 x;
            __builtin_memcpy(&x, e, 8);
            *reinterpret_cast<u32x2*>(out + d * 2) = x;
        }
    if (h == 0) {
        const float mc = m == -__builtin_inff() ? 0.0f : m * cs;
        a.lse[seq_row(a, w) + (int64_t)pos * a.heads + head] =
            some ? (mc + __log2f(l)) * kLn2 : -__builtin_inff();
    }
}

template <typename T, int DP>
hipError_t launch_forward(AttnPlan& p, hipStream_t s) {
    const int64_t units = (int64_t)p.args.units.d * p.args.kv_heads;
    attn_forward_kernel<T, DP><<<dim3((unsigned)units), dim3(kAttnThreads), 0, s>>>(p.args, p.table);
    return hipGetLastError();
}

inline uint64_t align256(uint64_t x) { return (x + 255) / 256 * 256; }

}  // namespace

size_t attn_table_bytes(const c3_attention_t* a) {
    return a->q_lens != nullptr && a->batch > kAttnArgSeqs ? align256(sizeof(AttnSeq) * (size_t)a->batch) : 0;
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
    p.table.n = 0;
    p.table.staged = nullptr;
    p.max_q = a->q_tokens;
    p.max_k = a->k_tokens;
    p.work = a->batch * a->q_tokens * a->k_tokens;
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
    p.max_q = p.max_k = p.work = 0;
    for (int i = 0; i < a->batch; ++i) {
        const int64_t q = a->q_lens[i], k = a->k_lens[i];
        if (q < 0 || k < 0 || (!a->packed && (q > a->q_tokens || k > a->k_tokens))) return C3_E_INVAL;
        if (a->packed && (nq + q > a->q_tokens || nk + k > a->k_tokens)) return C3_E_INVAL;
        s[i] = AttnSeq{i, a->packed ? (int32_t)nq : 0, (int32_t)q, a->packed ? (int32_t)nk : 0, (int32_t)k, 0};
        nq += q;
        nk += k;
        p.max_q = std::max(p.max_q, q);
        p.max_k = std::max(p.max_k, k);
        p.work += q * k;
    }
    if (a->packed && (nq != a->q_tokens || nk != a->k_tokens)) return C3_E_INVAL;
    // the longest walks first, so that short ones fill the end
    std::stable_sort(s, s + a->batch, [](const AttnSeq& x, const AttnSeq& y) {
        return (int64_t)x.q_len * x.k_len > (int64_t)y.q_len * y.k_len;
    });
    p.table.n = a->batch;
    return C3_OK;
}

int attn_tensor(const c3_attn_tensor_t* t, const AttnPlan& p, bool keys, AttnTensor& to) {
    if (t == nullptr) return C3_E_INVAL;
    const AttnArgs& g = p.args;
    const bool none = (keys ? p.key_rows : p.rows) == 0;
    if (none) {
        to = AttnTensor{nullptr, 0, 0, 0};
        return C3_OK;
    }
    if (t->ptr == nullptr) return C3_E_INVAL;
    if ((uintptr_t)t->ptr % 16 != 0) return C3_E_ALIGN;
    for (int i = g.packed ? 1 : 0; i < 3; ++i) {
        if (t->stride[i] < 0 || t->stride[i] >= (1ll << 40)) return C3_E_INVAL;
        if (t->stride[i] % 8 != 0) return C3_E_ALIGN;
    }
    to.ptr = static_cast<char*>(t->ptr);
    to.sb = g.packed ? 0 : t->stride[0] * 2;
    to.st = t->stride[1] * 2;
    to.sh = t->stride[2] * 2;
    // a tile is addressed with 31 bits from its first row
    if (to.st * 64 + to.sh * (int64_t)g.group.d >= (1ll << 31) - 4096) return C3_E_UNSUPPORTED;
    return C3_OK;
}

}  // namespace c3

extern "C" {

size_t c3_attention_workspace_size(const c3_attention_t* a) {
    try {
        c3::AttnPlan p;
        if (c3::attn_plan(a, p) != C3_OK) return 0;
        return 256 + c3::attn_table_bytes(a);
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
        if ((rc = attn_tensor(q, p, false, p.args.q)) != C3_OK) return rc;
        if ((rc = attn_tensor(k, p, true, p.args.k)) != C3_OK) return rc;
        if ((rc = attn_tensor(v, p, true, p.args.v)) != C3_OK) return rc;
        if ((rc = attn_tensor(out, p, false, p.args.o)) != C3_OK) return rc;
        if (p.rows > 0 && lse == nullptr) return C3_E_INVAL;
        if ((uintptr_t)lse % 4 != 0) return C3_E_ALIGN;
        if (ws == nullptr || (uintptr_t)ws % 256 != 0 || ws_bytes < 256 + attn_table_bytes(a))
            return C3_E_WORKSPACE;
        if (p.rows == 0) return C3_OK;
        p.args.lse = lse;
        const int64_t group = p.args.group.d, rows = 32 * kAttnWaves;
        const int64_t units = attn_number(p, a->batch, [&](int64_t nq, int64_t, int64_t) {
            return (nq * group + rows - 1) / rows;
        });
        if (units < 0 || units * p.args.kv_heads >= (1ll << 31)) return C3_E_UNSUPPORTED;
        p.args.units = FastDiv((uint32_t)units);
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        if (p.seqs != nullptr) {
            if (stage_bytes(ws, p.seqs, sizeof(AttnSeq) * (size_t)a->batch, s) != hipSuccess) return C3_E_HIP;
            p.table.staged = static_cast<const AttnSeq*>(ws);
        }
        hipError_t e;
        if (a->dtype == C3_BF16)
            e = a->dim > 64 ? launch_forward<__bf16, 128>(p, s) : launch_forward<__bf16, 64>(p, s);
        else
            e = a->dim > 64 ? launch_forward<_Float16, 128>(p, s) : launch_forward<_Float16, 64>(p, s);
        return e == hipSuccess ? C3_OK : C3_E_HIP;
    } catch (...) {
        return C3_E_INVAL;
    }
}

}  // extern "C"
