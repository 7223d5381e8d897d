// Attention's gradient (include/c3_replay.h): the host side of its two passes
// (c3_attention_dq.hip, c3_attention_dkv.hip), which recompute the probabilities
// from lse.
//
// Seven products where one pass would do with five: there the dq of a row would
// be added up by workgroups in the order in which they come, and the bits would
// change from run to run.  Matrix products bound both.
#include <algorithm>

#include "c3_attention.h"

namespace c3 {
namespace {

inline uint64_t align256(uint64_t x) { return (x + 255) / 256 * 256; }

// Workspace: lse2 and delta of every row, then the tables of both passes.
struct GradSpace {
    uint64_t lse2, delta, careful, table_q, table_k, total;
    GradSpace(const c3_attention_t* a, const AttnPlan& p) {
        uint64_t at = 0;
        auto take = [&at](uint64_t bytes) { const uint64_t r = at; at = align256(at + bytes); return r; };
        lse2 = take(4 * (uint64_t)p.rows);
        delta = take(4 * (uint64_t)p.rows);
        // a mark for every workgroup: key blocks of all sequences, one in part for each
        careful = take(4 * (uint64_t)(p.key_rows / attn_dkv_keys(a->dim) + (int64_t)a->kv_heads * a->batch));
        table_q = take(attn_table_bytes(a));
        table_k = take(attn_table_bytes(a));
        total = std::max<uint64_t>(at, 256);
    }
};

// Numbers the sequences' units for one pass and stages the list if it is long.
int number_units(const c3_attention_t* a, AttnPlan& p, char* table, bool keys, hipStream_t s) {
    const int64_t group = p.args.group.d, block_keys = attn_dkv_keys(p.args.dim);
    const int64_t units = attn_number(p, a->batch, [&](int64_t nq, int64_t, int64_t nk) {
        return keys ? (nk + block_keys - 1) / block_keys
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
        g.careful = reinterpret_cast<uint32_t*>(base + sp.careful);
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        const bool bf16 = a->dtype == C3_BF16;
        if (p.rows > 0) {
            if ((rc = number_units(a, p, base + sp.table_q, false, s)) != C3_OK) return rc;
            if (launch_attn_dq(p, bf16, s) != hipSuccess) return C3_E_HIP;
        }
        if (p.key_rows > 0) {
            if ((rc = number_units(a, p, base + sp.table_k, true, s)) != C3_OK) return rc;
            if (launch_attn_dkv(p, bf16, s) != hipSuccess) return C3_E_HIP;
        }
        return C3_OK;
    } catch (...) {
        return C3_E_INVAL;
    }
}

}  // extern "C"
