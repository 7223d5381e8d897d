// Attention's gradient (include/c3_replay.h): the host side of its two passes
// (c3_attention_dq.hip, c3_attention_dkv.hip), which recompute the probabilities
// from lse.
//
// Seven products where one pass would do with five: there the dq of a row would
// be added up by workgroups in the order in which they come, and the bits would
// change from run to run.  Matrix products bound both.
#include <algorithm>

#include "c3_attention_dkv.h"
#include "c3_attention_dq.h"

namespace c3 {
namespace {

// One gradient's parts: out = factor * their sum, in their order.
struct PartSum {
    const float* part;      // `rows` rows [tokens][heads] of `dim` each
    int64_t stride;         // elements from one part to the next
    int64_t rows;
    FastDiv heads, tokens;
    AttnTensor out;
    int32_t parts;
    float factor;
};
struct PartSums {
    PartSum of[3];
};

// All the divided gradients in one launch (blockIdx.y); a thread takes four elements
// of a row.
template <typename T>
__global__ __launch_bounds__(256) void attn_sum_parts_kernel(PartSums sums, FastDiv quads) {
    const PartSum& j = sums.of[blockIdx.y];
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= j.rows * quads.d) return;
    const int64_t row = i / quads.d;
    const int d = (int)(i - row * quads.d) * 4;
    const float* from = j.part + row * quads.d * 4 + d;
    f32x4 sum = *reinterpret_cast<const f32x4*>(from);
#pragma unroll 4
    for (int p = 1; p < j.parts; ++p) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(from + p * j.stride);
#pragma unroll
        for (int n = 0; n < 4; ++n) sum[n] += x[n];
    }
    const int64_t token = row / j.heads.d, b = token / j.tokens.d;
    const int head = (int)(row - token * j.heads.d);
    T e[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) e[n] = (T)(sum[n] * j.factor);
    u32x2 x;
    __builtin_memcpy(&x, e, 8);
    *reinterpret_cast<u32x2*>(j.out.ptr + b * j.out.sb + (token - b * j.tokens.d) * j.out.st + head * j.out.sh +
                              d * 2) = x;
}

hipError_t sum_parts(const AttnPlan& p, bool bf16, hipStream_t s) {
    const AttnArgs& g = p.args;
    PartSums sums{};
    int n = 0;
    int64_t most = 0;
    auto add = [&](const AttnSide& side, int which, int of, int heads, int64_t tokens, const AttnTensor& out,
                   float factor) {
        if (side.splits.d < 2 || side.part_rows == 0) return;
        const int64_t size = side.part_rows * g.dim;
        sums.of[n++] = PartSum{side.part + which * size, of * size, side.part_rows, FastDiv((uint32_t)heads),
                               FastDiv((uint32_t)tokens), out, (int32_t)side.splits.d, factor};
        most = std::max(most, side.part_rows);
    };
    add(g.side[0], 0, 1, g.heads, g.q_tokens, g.dq, g.scale);
    add(g.side[1], 0, 2, g.kv_heads, g.k_tokens, g.dk, g.scale);
    add(g.side[1], 1, 2, g.kv_heads, g.k_tokens, g.dv, 1.0f);
    if (n == 0) return hipSuccess;
    const FastDiv quads((uint32_t)g.dim / 4);
    const dim3 grid((unsigned)((most * quads.d + 255) / 256), (unsigned)n), block(256);
    if (bf16)
        attn_sum_parts_kernel<__bf16><<<grid, block, 0, s>>>(sums, quads);
    else
        attn_sum_parts_kernel<_Float16><<<grid, block, 0, s>>>(sums, quads);
    return hipGetLastError();
}

// Repeats with care the units that either pass marked: the first half of the
// workgroups those of the first.
template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, 1) void attn_grad_careful_kernel(AttnArgs a, AttnTable tab,
                                                                            uint32_t q_blocks, uint32_t k_blocks) {
    const uint32_t half = gridDim.x / 2;
    if (blockIdx.x < half)
        repeat_marked(a.side[0].marks, q_blocks, blockIdx.x, half,
                      [&](uint32_t unit) { dq_unit<T, DP, true, true>(a, tab, unit); });
    else
        repeat_marked(a.side[1].marks, k_blocks, blockIdx.x - half, half,
                      [&](uint32_t unit) { dkv_unit<T, DP, true>(a, tab, unit); });
}

template <typename T, int DP>
hipError_t launch_careful(const AttnPlan& p, hipStream_t s) {
    const uint32_t q = attn_direct(p, 0) ? 0 : attn_blocks(p, 0);
    const uint32_t k = attn_direct(p, 1) ? 0 : attn_blocks(p, 1);
    if (q + k == 0) return hipSuccess;
    attn_grad_careful_kernel<T, DP><<<dim3(64), dim3(kAttnThreads), 0, s>>>(p.args, p.table, q, k);
    return hipGetLastError();
}

// Parts of a walk.  A pass whose tiles give fewer than `want` workgroups divides
// each tile's walk, of `steps` tiles on the other side at most, into parts of at
// least kPartSteps, whose fp32 sums a further kernel adds up in order.
constexpr int64_t kPartSteps = 2, kMostParts = 16;
int64_t walk_parts(int64_t units, int64_t want, int64_t steps) {
    if (units < 1 || units >= want) return 1;
    return std::max<int64_t>(1, std::min({(want + units - 1) / units, steps / kPartSteps, kMostParts}));
}

inline uint64_t align256(uint64_t x) { return (x + 255) / 256 * 256; }

constexpr int64_t kDqRows = 32 * kAttnWaves;        // rows of a unit of the first pass

// Divides the work of both passes and lays out the workspace: lse2 and delta of every
// row, marks, the table of sequences, parts of sums.
struct GradSpace {
    uint64_t lse2, delta, marks[2], table, part[2], total;
    int64_t parts[2];
    bool fits;
    GradSpace(const c3_attention_t* a, AttnPlan& p) {
        const int64_t group = p.args.group.d, kv = p.args.kv_heads, block_keys = kDkvKeys;
        auto number = [&](int side, int64_t times) {
            return kv * attn_number(p, a->batch, side, [&](int64_t nq, int64_t, int64_t nk) {
                return times * (side ? (nk + block_keys - 1) / block_keys : (nq * group + kDqRows - 1) / kDqRows);
            });
        };
        parts[0] = walk_parts(number(0, 1), 512, p.max_k / kDqKeys);
        // walks under a causal mask differ in length: more of them even that out
        parts[1] = walk_parts(number(1, 1), a->causal ? 1024 : 512, p.max_q * group / 64);
        const int64_t units[2] = {number(0, parts[0]), number(1, parts[1])};
        fits = units[0] >= 0 && units[1] >= 0;
        uint64_t at = 0;
        auto take = [&at](int64_t bytes) { const uint64_t r = at; at = align256(at + (uint64_t)bytes); return r; };
        lse2 = take(4 * p.rows);
        delta = take(4 * p.rows);
        table = take((int64_t)attn_table_bytes(a));
        for (int i = 0; i < 2; ++i) {
            const int64_t rows = i ? p.key_rows : p.rows;
            p.args.side[i].splits = FastDiv((uint32_t)parts[i]);
            p.args.side[i].part_rows = rows;
            marks[i] = take(fits ? 4 * units[i] : 0);
            part[i] = take(parts[i] > 1 ? 4 * (i + 1) * parts[i] * rows * p.args.dim : 0);
        }
        total = std::max<uint64_t>(at, 256);
    }
};

}  // namespace
}  // namespace c3

extern "C" {

size_t c3_attention_grad_workspace_size(const c3_attention_t* a) {
    try {
        c3::AttnPlan p;
        if (c3::attn_plan(a, p) != C3_OK) return 0;
        const c3::GradSpace sp(a, p);
        return sp.fits ? sp.total : 0;
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
        if ((rc = attn_tensor(dout, p, false, Tiles::kGroup, g.d_o)) != C3_OK) return rc;
        if ((rc = attn_tensor(q, p, false, Tiles::kGroup, g.q)) != C3_OK) return rc;
        if ((rc = attn_tensor(k, p, true, Tiles::kHead, g.k)) != C3_OK) return rc;
        if ((rc = attn_tensor(v, p, true, Tiles::kHead, g.v)) != C3_OK) return rc;
        if ((rc = attn_tensor(out, p, false, Tiles::kNone, g.o)) != C3_OK) return rc;
        if ((rc = attn_tensor(dq, p, false, Tiles::kNone, g.dq)) != C3_OK) return rc;
        if ((rc = attn_tensor(dk, p, true, Tiles::kNone, g.dk)) != C3_OK) return rc;
        if ((rc = attn_tensor(dv, p, true, Tiles::kNone, g.dv)) != C3_OK) return rc;
        if (p.rows > 0 && lse == nullptr) return C3_E_INVAL;
        if ((uintptr_t)lse % 4 != 0) return C3_E_ALIGN;
        const GradSpace sp(a, p);
        if (!sp.fits) return C3_E_UNSUPPORTED;
        if (ws == nullptr || (uintptr_t)ws % 256 != 0 || ws_bytes < sp.total) return C3_E_WORKSPACE;
        if (attn_overlap({&g.dq, &g.dk, &g.dv}, {&g.d_o, &g.q, &g.k, &g.v, &g.o})) return C3_E_INVAL;
        char* base = static_cast<char*>(ws);
        g.lse = const_cast<float*>(lse);
        g.lse2 = reinterpret_cast<float*>(base + sp.lse2);
        g.delta = reinterpret_cast<float*>(base + sp.delta);
        for (int i = 0; i < 2; ++i) {
            g.side[i].marks = reinterpret_cast<uint32_t*>(base + sp.marks[i]);
            g.side[i].part = reinterpret_cast<float*>(base + sp.part[i]);
        }
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        const bool bf16 = a->dtype == C3_BF16, wide = a->dim > 64;
        if (p.rows + p.key_rows > 0 && (rc = attn_stage(a, p, base + sp.table, s)) != C3_OK) return rc;
        if (p.rows > 0 && launch_attn_dq(p, bf16, s) != hipSuccess) return C3_E_HIP;
        if (p.key_rows > 0 && launch_attn_dkv(p, bf16, s) != hipSuccess) return C3_E_HIP;
        if ((g.causal || g.window) && p.rows > 0 && p.key_rows > 0) {
            const hipError_t e =
                bf16 ? (wide ? launch_careful<__bf16, 128>(p, s) : launch_careful<__bf16, 64>(p, s))
                     : (wide ? launch_careful<_Float16, 128>(p, s) : launch_careful<_Float16, 64>(p, s));
            if (e != hipSuccess) return C3_E_HIP;
        }
        if (sum_parts(p, bf16, s) != hipSuccess) return C3_E_HIP;
        return C3_OK;
    } catch (...) {
        return C3_E_INVAL;
    }
}

}  // extern "C"
