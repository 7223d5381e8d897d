// Tokens to their experts and back (include/c3_replay.h).
//
// The sort is a stable counting sort of `choices` small integers.  A workgroup
// owns a run of choices; the place of a choice is its expert's first place plus
// the expert's choices in earlier runs, in earlier waves of the run and in
// earlier lanes of the wave.  Integer counts do not depend on the order of their
// additions, so the places are those of a serial sort.  Up to kOneRun choices
// take one launch (latency bounds it), more take a counting launch before it.
//
// The calls that move rows are bound by HBM: each row on the token side is read
// or written once, each sorted row once.  One wave moves 64 pieces of 16 bytes
// (four times as many where there are enough rows) of one token's row to or
// from the rows of all its choices, so a token's row stays in registers for all
// of them, and sums run in fp32 in the order of the choices.
#include <type_traits>

#include "c3_internal.h"
#include "c3_replay_types.h"

namespace c3 {
namespace {

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kOneRun = 8192;
constexpr int kMostRuns = 64;

// Choices of a run: whole multiples of a workgroup's threads, at most kMostRuns
// runs, so that every run can add up the counts of those before it.
int64_t run_length(int64_t n) {
    if (n <= kOneRun) return n < 1 ? kSortThreads : (n + kSortThreads - 1) / kSortThreads * kSortThreads;
    const int64_t r = (n + kMostRuns - 1) / kMostRuns;
    return (r + 2 * kSortThreads - 1) / (2 * kSortThreads) * (2 * kSortThreads);
}

__global__ __launch_bounds__(kSortThreads) void expert_count_kernel(const int32_t* ids, int64_t n,
                                                                    int experts, int64_t run,
                                                                    int32_t* counts) {
    extern __shared__ int32_t hist[];
    for (int e = threadIdx.x; e < experts; e += kSortThreads) hist[e] = 0;
    __syncthreads();
    const int64_t begin = (int64_t)blockIdx.x * run, end = min(begin + run, n);
    for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads) {
        const int32_t e = ids[i];
        if ((uint32_t)e < (uint32_t)experts) atomicAdd(&hist[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += kSortThreads)
        counts[(int64_t)blockIdx.x * experts + e] = hist[e];
}

// counts: [runs][experts], not read where there is one run.
__global__ __launch_bounds__(kSortThreads) void expert_place_kernel(
    const int32_t* ids, int64_t n, int experts, int bits, int64_t run, const int32_t* counts,
    int32_t* offsets, int32_t* source, int32_t* slot) {
    extern __shared__ int32_t lds[];            // [kSortWaves][experts], then [kSortWaves]
    int32_t* wave_sum = lds + kSortWaves * experts;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t begin = (int64_t)blockIdx.x * run, end = min(begin + run, n);
    // a wave's part of the run: whole steps of 64 choices in a row
    const int64_t part = run / kSortWaves;
    const int64_t wb = begin + wave * part, we = min(wb + part, end);
    for (int i = tid; i < kSortWaves * experts; i += kSortThreads) lds[i] = 0;
    __syncthreads();
    int32_t* mine = lds + wave * experts;
    for (int64_t i = wb + lane; i < we; i += 64) {
        const int32_t e = ids[i];
        if ((uint32_t)e < (uint32_t)experts) atomicAdd(&mine[e], 1);
    }
    __syncthreads();
    // thread e: all choices of expert e, and those of earlier runs (experts <=
    // kSortThreads)
    int32_t total = 0, before = 0;
    if (tid < experts) {
        if (gridDim.x > 1) {
            // sixteen counts in flight: one after the other their latencies add up
            const int runs = gridDim.x;
            for (int b = 0; b < runs; b += 16) {
                int32_t c[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) c[j] = counts[(int64_t)min(b + j, runs - 1) * experts + tid];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    before += b + j < (int)blockIdx.x ? c[j] : 0;
                    total += b + j < runs ? c[j] : 0;
                }
            }
        } else {
            for (int w = 0; w < kSortWaves; ++w) total += lds[w * experts + tid];
        }
    }
    // exclusive sum of the totals over the experts
    int32_t sum = total;
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t up = __shfl_up(sum, d);
        if (lane >= d) sum += up;
    }
    if (lane == 63) wave_sum[wave] = sum;
    __syncthreads();
    int32_t earlier = 0, all = 0;
    for (int w = 0; w < kSortWaves; ++w) {
        const int32_t s = wave_sum[w];
        if (w < wave) earlier += s;
        all += s;
    }
    const int32_t first = earlier + sum - total;
    if (tid < experts) {
        if (blockIdx.x == 0) offsets[tid] = first;
        int32_t at = first + before;
        for (int w = 0; w < kSortWaves; ++w) {
            const int32_t c = lds[w * experts + tid];
            lds[w * experts + tid] = at;
            at += c;
        }
    }
    if (tid == 0 && blockIdx.x == 0) offsets[experts] = all;
    __syncthreads();
    // places: the wave's next place of the expert plus the lanes below that
    // have the same one
    for (int64_t i0 = wb; i0 < we; i0 += 64) {
        const int64_t i = i0 + lane;
        const bool there = i < we;
        const int32_t e = there ? ids[i] : -1;
        const bool kept = (uint32_t)e < (uint32_t)experts;
        uint64_t same = __ballot(kept);
        for (int b = 0; b < bits; ++b) {
            const bool bit = (e >> b) & 1;
            const uint64_t m = __ballot(bit);
            same &= bit ? m : ~m;
        }
        int32_t place = -1;
        if (kept) place = mine[e] + __popcll(same & ((1ull << lane) - 1));
        __builtin_amdgcn_wave_barrier();
        if (kept && (same >> lane) == 1) mine[e] = place + 1;     // the last lane of its expert
        __builtin_amdgcn_wave_barrier();
        if (there) slot[i] = place;
        if (kept) source[place] = (int32_t)i;
    }
    for (int64_t i = begin + tid; i < end; i += kSortThreads)
        if (i >= all) source[i] = -1;
}

// ---------------------------------------------------------------------------
// rows
// ---------------------------------------------------------------------------
struct RowArgs {
    int64_t tokens, pieces;         // pieces of V elements of a row
    int64_t token_stride, sorted_stride;
    const int32_t* slot;
    const int32_t* kept;
    const float* weights;
    float* dweights;
    int32_t top;
    uint32_t parts;                 // waves that share a row
};

template <typename T, int V>
using Piece = AlignedPack<T, V>;

// Zeros in the sorted rows that hold no token: wave w of `waves` takes every
// waves-th of them.
template <typename T, int V>
__device__ void zero_tail(const RowArgs& a, T* sorted, int64_t kept, int64_t w, int64_t waves) {
    const int lane = threadIdx.x & 63;
    const int64_t rows = a.tokens * a.top;
    Piece<T, V> zero;
#pragma unroll
    for (int j = 0; j < V; ++j) zero.v[j] = (T)0.0f;
    for (int64_t r = kept + w; r < rows; r += waves)
        for (int64_t c = lane; c < a.pieces; c += 64)
            *reinterpret_cast<Piece<T, V>*>(sorted + r * a.sorted_stride + c * V) = zero;
}

template <typename T, int V, int U>
__global__ __launch_bounds__(256) void expert_dispatch_kernel(RowArgs a, const T* x, T* sorted) {
    // a piece that is only moved: kept as one word, or the compiler holds it in LDS
    using Word = std::conditional_t<sizeof(Piece<T, V>) == 16, u32x4, T>;
    const int lane = threadIdx.x & 63;
    const int64_t w = wide_block() * 4 + (threadIdx.x >> 6);
    const int64_t waves = wide_blocks() * 4;
    const int64_t token = w / a.parts, c0 = (w - token * a.parts) * 64 * U + lane;
    const int64_t kept = max(*a.kept, 0);
    if (token < a.tokens) {
        const uint32_t rows = (uint32_t)(a.tokens * a.top);     // a slot outside is a dropped choice
        const int32_t my_slot = lane < a.top ? a.slot[token * a.top + lane] : -1;
        const T* row = x + token * a.token_stride;
        Word p[U];
#pragma unroll
        for (int u = 0; u < U; ++u)             // behind the row's end the last piece again
            p[u] = *reinterpret_cast<const Word*>(row + min(c0 + u * 64, a.pieces - 1) * V);
        for (int k = 0; k < a.top; ++k) {
            const int32_t s = __builtin_amdgcn_readlane(my_slot, k);
            if ((uint32_t)s >= rows) continue;
            T* to = sorted + (int64_t)s * a.sorted_stride;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c0 + u * 64 < a.pieces)
                    *reinterpret_cast<Word*>(to + (c0 + u * 64) * V) = p[u];
        }
    }
    zero_tail<T, V>(a, sorted, kept, w, waves);
}

template <typename T, int V, int U>
__global__ __launch_bounds__(256) void expert_combine_kernel(RowArgs a, const T* sorted, T* out) {
    const int lane = threadIdx.x & 63;
    const int64_t w = wide_block() * 4 + (threadIdx.x >> 6);
    const int64_t token = w / a.parts, c0 = (w - token * a.parts) * 64 * U + lane;
    if (token >= a.tokens) return;
    const uint32_t rows = (uint32_t)(a.tokens * a.top);     // a slot outside is a dropped choice
    const int32_t my_slot = lane < a.top ? a.slot[token * a.top + lane] : -1;
    float my_weight = 1.0f;
    if (a.weights != nullptr && lane < a.top) my_weight = a.weights[token * a.top + lane];
    float acc[U][V] = {};
    // Pieces behind the row's end are the last one again, and a choice without a row
    // takes row 0: the loads stand without a branch between them, four rows at a time.
    int64_t at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) at[u] = min(c0 + u * 64, a.pieces - 1) * V;
    for (int k0 = 0; k0 < a.top; k0 += 4) {
        Piece<T, V> p[4][U];
        bool there[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int32_t s = k0 + q < a.top ? __builtin_amdgcn_readlane(my_slot, (k0 + q) & 63) : -1;
            there[q] = (uint32_t)s < rows;
            const T* row = sorted + (there[q] ? (int64_t)s : 0) * a.sorted_stride;
#pragma unroll
            for (int u = 0; u < U; ++u) p[q][u] = *reinterpret_cast<const Piece<T, V>*>(row + at[u]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (!there[q]) continue;
            const float weight = __shfl(my_weight, (k0 + q) & 63);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < V; ++j) acc[u][j] = fmaf(weight, to_f32(p[q][u].v[j]), acc[u][j]);
        }
    }
    T* row = out + token * a.token_stride;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (c0 + u * 64 >= a.pieces) continue;
        Piece<T, V> y;
#pragma unroll
        for (int j = 0; j < V; ++j) y.v[j] = (T)acc[u][j];
        *reinterpret_cast<Piece<T, V>*>(row + (c0 + u * 64) * V) = y;
    }
}

// One workgroup a token: a product <dout, sorted row> runs over the whole row.
// Lane sums in the order of the pieces, a butterfly over the wave, then the four
// waves in order; lane k of a wave keeps the sum of choice k.
template <typename T, int V, int U>
__global__ __launch_bounds__(256) void expert_combine_grad_kernel(RowArgs a, const T* dout,
                                                                  const T* sorted, T* dsorted) {
    __shared__ float part[4][C3_MAX_EXPERT_TOP];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t token = wide_block(), kept = max(*a.kept, 0);
    if (token >= a.tokens) return;          // zero_tail's waves are those of tokens
    const uint32_t rows = (uint32_t)(a.tokens * a.top);     // a slot outside is a dropped choice
    const int32_t my_slot = lane < a.top ? a.slot[token * a.top + lane] : -1;
    float my_weight = 1.0f;
    if (a.weights != nullptr && lane < a.top) my_weight = a.weights[token * a.top + lane];
    const T* grow = dout + token * a.token_stride;
    float my_dot = 0.0f;
    for (int64_t c = threadIdx.x; c - threadIdx.x < a.pieces; c += 256 * U) {
        Piece<T, V> g[U] = {};
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c + u * 256 < a.pieces)
                g[u] = *reinterpret_cast<const Piece<T, V>*>(grow + (c + u * 256) * V);
        for (int k = 0; k < a.top; ++k) {
            const int32_t s = __builtin_amdgcn_readlane(my_slot, k);
            if ((uint32_t)s >= rows) continue;
            const float weight = __shfl(my_weight, k);
            float dot = 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (c + u * 256 >= a.pieces) continue;
                const int64_t at = (int64_t)s * a.sorted_stride + (c + u * 256) * V;
                if (a.dweights != nullptr) {
                    const Piece<T, V> y = *reinterpret_cast<const Piece<T, V>*>(sorted + at);
#pragma unroll
                    for (int j = 0; j < V; ++j) dot = fmaf(to_f32(g[u].v[j]), to_f32(y.v[j]), dot);
                }
                Piece<T, V> d;
#pragma unroll
                for (int j = 0; j < V; ++j) d.v[j] = (T)(weight * to_f32(g[u].v[j]));
                *reinterpret_cast<Piece<T, V>*>(dsorted + at) = d;
            }
            if (a.dweights != nullptr) {
#pragma unroll
                for (int m = 32; m >= 1; m >>= 1) dot += __shfl_xor(dot, m);
                if (lane == k) my_dot += dot;
            }
        }
    }
    if (a.dweights != nullptr) {
        part[wave][lane] = my_dot;
        __syncthreads();
        if ((int)threadIdx.x < a.top)
            a.dweights[token * a.top + threadIdx.x] =
                part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane];
    }
    zero_tail<T, V>(a, dsorted, kept, token * 4 + wave, a.tokens * 4);
}

enum class Move { kDispatch, kCombine, kGrad };

// Waves below which a row is shared by four times as many of them: 256 compute
// units hold 2,048 waves of eight each.
constexpr int64_t kFewWaves = 4096;

template <typename T, int V>
hipError_t launch_rows(Move m, RowArgs a, int64_t hidden, const void* in, const void* sorted, void* to,
                       hipStream_t s) {
    a.pieces = hidden / V;
    if (m == Move::kGrad) {
        const dim3 grid = wide_grid((uint64_t)a.tokens), block(256);
        if (a.pieces > 512)
            expert_combine_grad_kernel<T, V, 4><<<grid, block, 0, s>>>(a, (const T*)in, (const T*)sorted, (T*)to);
        else if (a.pieces > 256)
            expert_combine_grad_kernel<T, V, 2><<<grid, block, 0, s>>>(a, (const T*)in, (const T*)sorted, (T*)to);
        else
            expert_combine_grad_kernel<T, V, 1><<<grid, block, 0, s>>>(a, (const T*)in, (const T*)sorted, (T*)to);
        return hipGetLastError();
    }
    const int64_t parts4 = (a.pieces + 255) / 256;
    const bool few = a.tokens * parts4 < kFewWaves;
    a.parts = (uint32_t)(few ? (a.pieces + 63) / 64 : parts4);
    const dim3 grid = wide_grid((uint64_t)(a.tokens * a.parts + 3) / 4), block(256);
    if (m == Move::kDispatch) {
        if (few)
            expert_dispatch_kernel<T, V, 1><<<grid, block, 0, s>>>(a, (const T*)in, (T*)to);
        else
            expert_dispatch_kernel<T, V, 4><<<grid, block, 0, s>>>(a, (const T*)in, (T*)to);
    } else {
        if (few)
            expert_combine_kernel<T, V, 1><<<grid, block, 0, s>>>(a, (const T*)sorted, (T*)to);
        else
            expert_combine_kernel<T, V, 4><<<grid, block, 0, s>>>(a, (const T*)sorted, (T*)to);
    }
    return hipGetLastError();
}

// in: the token-side input or null, sorted: the sorted input or null, to: output
int move_rows(Move m, const c3_expert_rows_t* r, const void* in, const void* sorted,
              const float* weights, void* to, float* dweights, c3_stream_t stream) {
    if (r == nullptr || r->top < 1 || r->top > C3_MAX_EXPERT_TOP || r->tokens < 0 || r->hidden < 0 ||
        r->tokens >= (1ll << 31) || r->tokens * r->top >= (1ll << 31) || r->hidden >= (1ll << 31) ||
        r->token_stride < 0 || r->sorted_stride < 0)
        return C3_E_INVAL;
    const int es = replay_elem_size(r->dtype);
    if (es == 0) return C3_E_UNSUPPORTED;
    if (r->tokens == 0 || (r->hidden == 0 && dweights == nullptr)) return C3_OK;
    if (r->slot == nullptr || r->kept == nullptr) return C3_E_INVAL;
    if (r->hidden > 0) {
        if (to == nullptr || (m != Move::kCombine && in == nullptr)) return C3_E_INVAL;
        if ((m == Move::kCombine || dweights != nullptr) && sorted == nullptr) return C3_E_INVAL;
    }
    if (r->token_stride < r->hidden || r->sorted_stride < r->hidden) return C3_E_INVAL;
    for (const void* p : {(const void*)in, (const void*)sorted, (const void*)to})
        if ((uintptr_t)p % es != 0) return C3_E_ALIGN;
    for (const void* p : {(const void*)r->slot, (const void*)r->kept, (const void*)weights,
                          (const void*)dweights})
        if ((uintptr_t)p % 4 != 0) return C3_E_ALIGN;
    const int v = 16 / es;
    const bool wide = r->hidden % v == 0 && r->token_stride % v == 0 && r->sorted_stride % v == 0 &&
                      (uintptr_t)in % 16 == 0 && (uintptr_t)sorted % 16 == 0 && (uintptr_t)to % 16 == 0;
    RowArgs a{};
    a.tokens = r->tokens;
    a.token_stride = r->token_stride;
    a.sorted_stride = r->sorted_stride;
    a.slot = r->slot;
    a.kept = r->kept;
    a.weights = weights;
    a.dweights = dweights;
    a.top = r->top;
    // waves are counted in 32 bits
    if (r->tokens * ((r->hidden / (wide ? v : 1) + 255) / 256) >= (1ll << 31)) return C3_E_UNSUPPORTED;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    hipError_t e;
    if (r->dtype == C3_F32)
        e = wide ? launch_rows<float, 4>(m, a, r->hidden, in, sorted, to, s)
                 : launch_rows<float, 1>(m, a, r->hidden, in, sorted, to, s);
    else if (r->dtype == C3_BF16)
        e = wide ? launch_rows<__bf16, 8>(m, a, r->hidden, in, sorted, to, s)
                 : launch_rows<__bf16, 1>(m, a, r->hidden, in, sorted, to, s);
    else
        e = wide ? launch_rows<_Float16, 8>(m, a, r->hidden, in, sorted, to, s)
                 : launch_rows<_Float16, 1>(m, a, r->hidden, in, sorted, to, s);
    return e == hipSuccess ? C3_OK : C3_E_HIP;
}

}  // namespace
}  // namespace c3

extern "C" {

size_t c3_expert_sort_workspace_size(int64_t choices, int experts) {
    if (choices < 0 || choices >= (1ll << 31) || experts < 1 || experts > C3_MAX_EXPERTS) return 0;
    const size_t n = choices <= c3::kOneRun ? 0 : sizeof(int32_t) * c3::kMostRuns * (size_t)experts;
    return n < 256 ? 256 : (n + 255) / 256 * 256;
}

int c3_expert_sort(const int32_t* ids, int64_t choices, int experts, int32_t* offsets,
                   int32_t* source, int32_t* slot, void* ws, size_t ws_bytes,
                   c3_stream_t stream) {
    using namespace c3;
    const size_t need = c3_expert_sort_workspace_size(choices, experts);
    if (need == 0 || offsets == nullptr) return C3_E_INVAL;
    if (choices > 0 && (ids == nullptr || source == nullptr || slot == nullptr)) return C3_E_INVAL;
    for (const void* p : {(const void*)ids, (const void*)offsets, (const void*)source, (const void*)slot})
        if ((uintptr_t)p % 4 != 0) return C3_E_ALIGN;
    if (ws == nullptr || (uintptr_t)ws % 256 != 0 || ws_bytes < need) return C3_E_WORKSPACE;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    int bits = 0;
    while ((1 << bits) < experts) ++bits;
    const int64_t run = run_length(choices);
    const int64_t runs = choices == 0 ? 1 : (choices + run - 1) / run;
    int32_t* counts = static_cast<int32_t*>(ws);
    if (runs > 1)
        expert_count_kernel<<<dim3((unsigned)runs), dim3(kSortThreads), sizeof(int32_t) * experts, s>>>(
            ids, choices, experts, run, counts);
    const size_t lds = sizeof(int32_t) * (size_t)(kSortWaves * experts + kSortWaves);
    expert_place_kernel<<<dim3((unsigned)runs), dim3(kSortThreads), lds, s>>>(
        ids, choices, experts, bits, run, counts, offsets, source, slot);
    return hipGetLastError() == hipSuccess ? C3_OK : C3_E_HIP;
}

int c3_expert_dispatch(const c3_expert_rows_t* r, const void* x, void* sorted, c3_stream_t stream) {
    return c3::move_rows(c3::Move::kDispatch, r, x, nullptr, nullptr, sorted, nullptr, stream);
}

int c3_expert_combine(const c3_expert_rows_t* r, const void* sorted, const float* weights,
                      void* out, c3_stream_t stream) {
    return c3::move_rows(c3::Move::kCombine, r, nullptr, sorted, weights, out, nullptr, stream);
}

int c3_expert_combine_grad(const c3_expert_rows_t* r, const void* dout, const void* sorted,
                           const float* weights, void* dsorted, float* dweights,
                           c3_stream_t stream) {
    return c3::move_rows(c3::Move::kGrad, r, dout, sorted, weights, dsorted, dweights, stream);
}

}  // extern "C"
