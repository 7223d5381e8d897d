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

// out = factor * the sum of the parts, in their order.  A thread takes four elements
// of a row; `rows` rows [tokens][heads] of `dim`.
template <typename T>
__global__ __launch_bounds__(256) void attn_sum_parts_kernel(const float* part, int64_t stride, int parts,
                                                             int64_t rows, FastDiv quads, FastDiv heads,
                                                             FastDiv tokens, AttnTensor out, float factor) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * quads.d) return;
    const int64_t row = i / quads.d;
    const int d = (int)(i - row * quads.d) * 4;
    const float* from = part + row * quads.d * 4 + d;
    f32x4 sum = *reinterpret_cast<const f32x4*>(from);
#pragma unroll 4
    for (int p = 1; p < parts; ++p) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(from + p * stride);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] += x[j];
    }
    const int64_t token = row / heads.d, b = token / tokens.d;
    const int head = (int)(row - token * heads.d);
    T e[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = (T)(sum[j] * factor);
    u32x2 x;
    __builtin_memcpy(&x, e, 8);
    *reinterpret_cast<u32x2*>(out.ptr + b * out.sb + (token - b * tokens.d) * out.st + head * out.sh + d * 2) = x;
}

hipError_t sum_parts(const AttnPlan& p, bool bf16, const float* part, int64_t stride, int64_t rows, int heads,
                     int64_t tokens, const AttnTensor& out, float factor, hipStream_t s) {
    const FastDiv quads((uint32_t)p.args.dim / 4), h((uint32_t)heads), t((uint32_t)tokens);
    const int64_t blocks = (rows * quads.d + 255) / 256;
    if (bf16)
        attn_sum_parts_kernel<__bf16><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(
            part, stride, (int)p.args.splits.d, rows, quads, h, t, out, factor);
    else
        attn_sum_parts_kernel<_Float16><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(
            part, stride, (int)p.args.splits.d, rows, quads, h, t, out, factor);
    return hipGetLastError();
}

// Parts of a walk.  A pass whose tiles give fewer than `want` workgroups divides
// each tile's walk, of `steps` tiles on the other side at most, into parts of at
// least kPartSteps, whose fp32 sums a further kernel adds up in order.
constexpr int64_t kPartSteps = 4, kMostParts = 16;
int64_t walk_parts(int64_t units, int64_t want, int64_t steps) {
    if (units < 1 || units >= want) return 1;
    return std::max<int64_t>(1, std::min({(want + units - 1) / units, steps / kPartSteps, kMostParts}));
}

inline uint64_t align256(uint64_t x) { return (x + 255) / 256 * 256; }

constexpr int64_t kDqRows = 32 * kAttnWaves;        // rows of a unit of the first pass

// Units of one key head, all sequences, of either pass before its walks are
// divided.
int64_t tiles_of(const c3_attention_t* a, AttnPlan& p, bool keys) {
    const int64_t group = p.args.group.d, block_keys = attn_dkv_keys(a->dim);
    return attn_number(p, a->batch, [&](int64_t nq, int64_t, int64_t nk) {
        return keys ? (nk + block_keys - 1) / block_keys : (nq * group + kDqRows - 1) / kDqRows;
    });
}

// Workspace: lse2 and delta of every row, the marks of the second pass, the tables
// of both, parts of sums; and how the walks are divided.
struct GradSpace {
    uint64_t lse2, delta, careful, table_q, table_k, part, total;
    int64_t parts_q, parts_k;
    GradSpace(const c3_attention_t* a, AttnPlan& p) {
        const int64_t group = p.args.group.d, kv = p.args.kv_heads;
        const int64_t units_k = tiles_of(a, p, true) * kv;
        parts_q = walk_parts(tiles_of(a, p, false) * kv, 512, p.max_k / 64);
        // walks under a causal mask differ in length: more of them even that out
        parts_k = walk_parts(units_k, a->causal ? 1024 : 512, p.max_q * group / 64);
        uint64_t at = 0;
        auto take = [&at](uint64_t bytes) { const uint64_t r = at; at = align256(at + bytes); return r; };
        lse2 = take(4 * (uint64_t)p.rows);
        delta = take(4 * (uint64_t)p.rows);
        careful = take(4 * (uint64_t)std::max<int64_t>(units_k * parts_k, 0));
        table_q = take(attn_table_bytes(a));
        table_k = take(attn_table_bytes(a));
        uint64_t bytes = 0;     // the passes follow each other
        if (parts_q > 1) bytes = 4 * (uint64_t)(parts_q * p.rows * p.args.dim);
        if (parts_k > 1) bytes = std::max(bytes, 8 * (uint64_t)(parts_k * p.key_rows * p.args.dim));
        part = take(bytes);
        total = std::max<uint64_t>(at, 256);
    }
};

// Numbers the sequences' units for one pass and stages the list if it is long.
int number_units(const c3_attention_t* a, AttnPlan& p, char* table, bool keys, int64_t parts, hipStream_t s) {
    const int64_t group = p.args.group.d, block_keys = attn_dkv_keys(a->dim);
    const int64_t units = attn_number(p, a->batch, [&](int64_t nq, int64_t, int64_t nk) {
        return parts * (keys ? (nk + block_keys - 1) / block_keys : (nq * group + kDqRows - 1) / kDqRows);
    });
    if (units < 0 || units * p.args.kv_heads >= (1ll << 31)) return C3_E_UNSUPPORTED;
    p.args.units = FastDiv((uint32_t)(units < 1 ? 1 : units));
    p.args.splits = FastDiv((uint32_t)parts);
    p.args.part_rows = keys ? p.key_rows : p.rows;
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
        g.part = reinterpret_cast<float*>(base + sp.part);
        g.careful = reinterpret_cast<uint32_t*>(base + sp.careful);
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        const bool bf16 = a->dtype == C3_BF16;
        if (p.rows > 0) {
            if ((rc = number_units(a, p, base + sp.table_q, false, sp.parts_q, s)) != C3_OK) return rc;
            if (launch_attn_dq(p, bf16, s) != hipSuccess) return C3_E_HIP;
            if (sp.parts_q > 1 &&
                sum_parts(p, bf16, g.part, p.rows * g.dim, p.rows, g.heads, g.q_tokens, g.dq, g.scale, s) != hipSuccess)
                return C3_E_HIP;
        }
        if (p.key_rows > 0) {
            if ((rc = number_units(a, p, base + sp.table_k, true, sp.parts_k, s)) != C3_OK) return rc;
            if (launch_attn_dkv(p, bf16, s) != hipSuccess) return C3_E_HIP;
            if (sp.parts_k > 1) {
                const int64_t n = p.key_rows * g.dim;
                if (sum_parts(p, bf16, g.part, 2 * n, p.key_rows, g.kv_heads, g.k_tokens, g.dk, g.scale, s) != hipSuccess ||
                    sum_parts(p, bf16, g.part + n, 2 * n, p.key_rows, g.kv_heads, g.k_tokens, g.dv, 1.0f, s) != hipSuccess)
                    return C3_E_HIP;
            }
        }
        return C3_OK;
    } catch (...) {
        return C3_E_INVAL;
    }
}

}  // extern "C"
