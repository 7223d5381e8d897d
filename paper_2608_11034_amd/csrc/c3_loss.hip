// Softmax cross entropy over a vocabulary and its gradient (include/c3_replay.h).
//
// Three products bound both: logits x W^T in the forward pass, and again in the gradient
// together with d W and d^T x, where d = (softmax - onehot) * dloss.  The logits are never
// kept: the forward pass reduces each tile to a maximum and a sum a token, and the
// gradient makes d for a piece of the vocabulary at a time, rounded to the inputs' 16
// bits as the matrix units take it, and adds its part of dx in fp32.
//
// Tokens whose target is no row of the vocabulary take no part: the others are copied
// together first, so that neither their time nor what they hold enters anything.
//
// 8,192 tokens over 131,072 rows of 4,096 in bf16: 6.7 ms forward; back 1.79 ms for the
// logits, 1.63 for dx and 1.67 for dweight of each quarter of the vocabulary, so that all
// four products run at 1,300 TFLOP/s, as a large library product does (c3_product.h has
// what bounds them).  8 tokens over 32,000 rows: bound by the weights, 262 MB in 43 us
// forward; back 46 us for the logits, 52 for dx, which reads the weights again, and 63 for
// 262 MB of dweight.
#include <algorithm>
#include <type_traits>

#include "c3_internal.h"
#include "c3_product.h"
#include "c3_sort.h"

namespace c3 {
namespace {

// What the first launch finds out, at the workspace's start.
struct Found {
    int32_t count;          // tokens that take part
    float raise, lower;     // d is kept times `raise`; sums of it go out times `lower`
    int32_t low;            // rows of d that hold what rounding left of as many others
};

// d is rounded to 16 bits, and where one entry outweighs a token's others, as its target's
// does, so does that one's rounding: as large as rounding the result, but the same way in
// all of a row.  So what rounding left of it is kept as well.
//   Up to kLowTokens tokens have a second row of d each, with what rounding left of all of
// the first, and their rows of x twice: dweight's sums run over both, and dx takes both up
// to kLowDx tokens, which no tile is fuller for.
//   Of more tokens only what was left of the target's entry counts.  dx takes it times its
// row of the weights, in fp32.  For dweight tokens stand in the order of their targets, so
// that those of one tile of the vocabulary are neighbours, and what was left of their
// entries, kLowCols columns of zeros and one number for each token, is a second operand,
// behind the first: few inner indices for most tiles, and never more than once as many.
constexpr int kLowTokens = 128, kLowDx = 64, kLowCols = 256, kBlockRows = 128;
constexpr int kPieceRows = 256;             // a piece of the vocabulary is a multiple of

struct LossArgs {
    const char* x;
    const char* weight;
    const void* targets;
    const float* dloss;         // null in the forward pass
    const float* lse_in;
    float* loss;
    float* lse;
    int64_t x_stride, weight_stride, dloss_stride;      // bytes, bytes, elements
    int64_t tokens, rows;
    int32_t hidden, wide_targets, half;
    float scale;
    // workspace
    Found* found;
    int32_t* token;             // [tokens] of each place
    int32_t* place;             // [tokens] of each token, -1
    int32_t* target;            // [tokens] by place
    float* grad;                // [tokens] by place: dloss * scale * raise
    float* lse_at;              // [tokens] by place
    float* low_target;          // [tokens] by place: what rounding left of the target's d
    char* xc;                   // [tokens and low][pitch] the rows that take part
    float2* parts;              // [row tiles][tokens] maximum and sum
    float* picked;              // [tokens] the target's logit
    char* d;                    // [tokens and low][d_pitch]
    float* dx_parts;            // [splits][dx_rows][pitch] fp32
    int32_t pitch;              // elements: hidden
    int32_t d_pitch;
    int64_t dx_rows;            // most rows of d that dx takes: the tokens', up to kLowDx twice
    // this piece of the vocabulary
    int64_t row0;
    int32_t piece, first;
    int32_t splits, split_len;  // of the inner index
    char* out;                  // dweight
    int64_t out_stride;
    float* w_parts;             // [splits][piece][pitch] fp32
    // beyond kLowTokens
    char* low_d;                // [tokens][kLowCols] the same as columns of d; null: not kept
    int32_t* block_first;       // with low_d: the first place of each kBlockRows rows, and behind the last
    Found* run_found;           // of each run of the sort, for more tokens than kGather: count, and in raise the largest dloss
};

__device__ __forceinline__ int32_t target_of(const LossArgs& a, int64_t t) {
    const int64_t v = a.wide_targets ? static_cast<const int64_t*>(a.targets)[t]
                                     : (int64_t)static_cast<const int32_t*>(a.targets)[t];
    return (uint64_t)v < (uint64_t)a.rows ? (int32_t)v : -1;
}

// What rounding leaves of an entry of d; nothing of one that is not finite.
template <typename T>
__device__ __forceinline__ float left_of(float d) {
    const float rounded = to_f32(from_f32<T>(d));
    return fabsf(rounded) < __builtin_inff() ? d - rounded : 0.0f;
}

// ---------------------------------------------------------------------------
// which tokens take part
// ---------------------------------------------------------------------------
// The size of a token's dloss if it is finite: one that is not makes infinities of its own
// row, and is no measure of the others.
__device__ __forceinline__ float size_of(const LossArgs& a, int64_t t) {
    const float size = fabsf(a.dloss[t * a.dloss_stride] * a.scale);
    return size < __builtin_inff() ? size : 0.0f;
}

__device__ __forceinline__ Found found_of(const LossArgs& a, int count, float most) {
    // d is kept relative to the largest dloss: with one dloss for all tokens, a mean's, the
    // target's entry of an unlikely token then is -1 in 16 bits, and not wherever that dloss
    // falls between two numbers, for all tokens on the same side.  In fp16 times 2^13, as
    // that holds 6e-8 to 65,504 and most entries are about one over the vocabulary's size.
    // The bounds keep `up` and `lower` normal numbers.
    const float unit = a.half ? 8192.0f : 1.0f;
    const float largest = most > 0.0f ? fminf(fmaxf(most, 0x1p-100f), 0x1p126f) : 1.0f;
    const float up = unit / largest;
    return Found{count, up, largest / unit, a.dloss != nullptr && count <= kLowTokens ? count : 0};
}

__device__ __forceinline__ void put_grad(const LossArgs& a, const Found& found, int64_t t, int32_t p) {
    a.grad[p] = a.dloss[t * a.dloss_stride] * a.scale * found.raise;
    a.lse_at[p] = a.lse_in[t];
    a.place[t] = p;
}

// Token t, which takes part at place p or, target < 0, does not.
__device__ __forceinline__ void put_token(const LossArgs& a, const Found& found, int64_t t, int32_t target, int32_t p) {
    if (target >= 0) {
        a.token[p] = (int32_t)t;
        a.target[p] = target;
        if (a.dloss != nullptr) put_grad(a, found, t, p);
    } else if (a.dloss != nullptr) {
        a.place[t] = -1;
    } else {
        a.loss[t] = 0.0f;
        a.lse[t] = 0.0f;
    }
}

__device__ __forceinline__ void copy_row(const LossArgs& a, int64_t t, int64_t p) {
    const u32x4* from = reinterpret_cast<const u32x4*>(a.x + t * a.x_stride);
    u32x4* to = reinterpret_cast<u32x4*>(a.xc + p * a.pitch * 2);
    for (int c = threadIdx.x & 63; c < a.hidden / 8; c += 64) to[c] = from[c];
}

// For low_d, by the wave of the token with `target` at place p, behind one with `before`
// (-1: none): zeros, and the blocks that begin there.
__device__ __forceinline__ void start_low(const LossArgs& a, int32_t before, int32_t target, int32_t p, int32_t count) {
    const int lane = threadIdx.x & 63;
    static_assert(kLowCols * 2 == 64 * 8, "eight bytes a lane");
    reinterpret_cast<u32x2*>(a.low_d + (int64_t)p * kLowCols * 2)[lane] = u32x2{};
    const int32_t mine = target / kBlockRows, end = (int32_t)((a.rows + kBlockRows - 1) / kBlockRows);
    for (int32_t b = (before < 0 ? 0 : before / kBlockRows + 1) + lane; b <= mine; b += 64) a.block_first[b] = p;
    if (p == count - 1)
        for (int32_t b = mine + 1 + lane; b <= end; b += 64) a.block_first[b] = count;
}

// Up to kGather tokens: a workgroup has four of them, a wave each, and looks at all the
// others' targets itself, which is quicker than a launch before it.  SORTED: places in the
// order of the targets, for low_d; else in that of the tokens.
constexpr int kGather = 4096;
template <bool SORTED>
__global__ __launch_bounds__(256) void loss_gather_kernel(LossArgs a) {
    constexpr int N = SORTED ? 4 : 1;
    __shared__ int32_t wave_count[4], wave_before[4][N], wave_lower[4][N];
    __shared__ float wave_most[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int tokens = (int)a.tokens, mine = blockIdx.x * 4;
    int32_t count = 0, before[N] = {}, lower[N], own[N];        // lower: the target of the place before
#pragma unroll
    for (int n = 0; n < N; ++n) {
        lower[n] = -1;
        own[n] = SORTED ? target_of(a, min(mine + n, tokens - 1)) : 0;
    }
    float most = 0.0f;
    for (int t0 = 0; t0 < tokens; t0 += 1024) {
        int32_t target[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) target[i] = target_of(a, min(t0 + i * 256 + tid, tokens - 1));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + i * 256 + tid;
            if (t >= tokens || target[i] < 0) continue;
            ++count;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const bool ahead = SORTED ? target[i] < own[n] || (target[i] == own[n] && t < mine + n) : t < mine;
                before[n] += ahead;
                if (SORTED && ahead) lower[n] = max(lower[n], target[i]);
            }
            if (a.dloss != nullptr) most = fmaxf(most, size_of(a, t));
        }
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        count += __shfl_xor(count, m);
        most = fmaxf(most, __shfl_xor(most, m));
#pragma unroll
        for (int n = 0; n < N; ++n) {
            before[n] += __shfl_xor(before[n], m);
            if constexpr (SORTED) lower[n] = max(lower[n], __shfl_xor(lower[n], m));
        }
    }
    if (lane == 0) {
        wave_count[wave] = count;
        wave_most[wave] = most;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            wave_before[wave][n] = before[n];
            wave_lower[wave][n] = lower[n];
        }
    }
    __syncthreads();
    const int n = SORTED ? wave : 0;
    int32_t place = 0, below = -1;
    count = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        count += wave_count[w];
        most = fmaxf(most, wave_most[w]);
        place += wave_before[w][n];
        below = max(below, wave_lower[w][n]);
    }
    const Found found = found_of(a, count, most);
    if (blockIdx.x == 0 && tid == 0) *a.found = found;
    const int t = mine + wave;
    if (t >= tokens) return;
    if constexpr (!SORTED)
        for (int i = 0; i < wave; ++i) place += target_of(a, mine + i) >= 0;
    const int32_t target = target_of(a, t);
    if (lane == 0) put_token(a, found, t, target, place);
    if (target < 0) return;
    copy_row(a, t, place);
    if (found.low > 0) copy_row(a, t, found.count + place);
    if constexpr (SORTED) start_low(a, below, target, place, count);
}

// The forward pass of more tokens (and the gradient of none): one workgroup for which they
// are, then their rows.
__global__ __launch_bounds__(1024) void loss_tokens_kernel(LossArgs a) {
    __shared__ int32_t wave_count[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // a wave's tokens: whole steps of 64 in a row
    const int64_t each = (a.tokens + 1023) / 1024 * 64;
    const int64_t begin = wave * each, end = min(a.tokens, begin + each);
    int32_t count = 0;
    for (int64_t t = begin + lane; t < end; t += 64) count += target_of(a, t) >= 0;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) count += __shfl_xor(count, m);
    if (lane == 0) wave_count[wave] = count;
    __syncthreads();
    int32_t at = 0, all = 0;
    for (int w = 0; w < 16; ++w) {
        if (w < wave) at += wave_count[w];
        all += wave_count[w];
    }
    const Found found = found_of(a, all, 0.0f);
    for (int64_t t0 = begin; t0 < end; t0 += 64) {
        const int64_t t = t0 + lane;
        const int32_t target = t < end ? target_of(a, t) : -1;
        const uint64_t some = __ballot(target >= 0);
        const int32_t p = at + __popcll(some & ((1ull << lane) - 1));
        at += __popcll(some);
        if (t >= end) continue;
        put_token(a, found, t, target, p);
    }
    if (tid == 0) *a.found = found;
}

// Their rows, one a wave.
__global__ __launch_bounds__(256) void loss_rows_kernel(LossArgs a) {
    const int64_t p = wide_block() * 4 + (threadIdx.x >> 6);
    if (p < a.found->count) copy_row(a, a.token[p], p);
}

// The gradient of more tokens: a sort by their targets, whose first launch also finds how
// many take part and the largest dloss, and whose lists are a.target and a.token; then, a
// wave a place, what belongs there.
__global__ __launch_bounds__(kSortThreads) void loss_count_kernel(LossArgs a, SortPass q) {
    __shared__ int32_t wave_count[kSortWaves];
    __shared__ float wave_most[kSortWaves];
    sort_count(q);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t begin = (int64_t)blockIdx.x << q.run_shift, end = min(begin + (1ll << q.run_shift), q.n);
    int32_t count = 0;
    float most = 0.0f;
    for (int64_t t = begin + tid; t < end; t += kSortThreads) {
        if (target_of(a, t) < 0) continue;
        ++count;
        most = fmaxf(most, size_of(a, t));
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        count += __shfl_xor(count, m);
        most = fmaxf(most, __shfl_xor(most, m));
    }
    if (lane == 0) {
        wave_count[wave] = count;
        wave_most[wave] = most;
    }
    __syncthreads();
    if (tid != 0) return;
    for (int w = 1; w < kSortWaves; ++w) {
        count += wave_count[w];
        most = fmaxf(most, wave_most[w]);
    }
    a.run_found[blockIdx.x] = Found{count, most, 0.0f, 0};
}

__global__ __launch_bounds__(kSortThreads) void loss_place_kernel(SortPass q) { sort_place(q); }

__global__ __launch_bounds__(256) void loss_sorted_rows_kernel(LossArgs a, int runs) {
    const int64_t p = wide_block() * 4 + (threadIdx.x >> 6);
    if (p >= a.tokens) return;
    static_assert(kMostRuns <= 64, "a run a lane");
    const int lane = threadIdx.x & 63;
    int32_t count = lane < runs ? a.run_found[lane].count : 0;
    float most = lane < runs ? a.run_found[lane].raise : 0.0f;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        count += __shfl_xor(count, m);
        most = fmaxf(most, __shfl_xor(most, m));
    }
    const Found found = found_of(a, count, most);
    if (p == 0 && lane == 0) *a.found = found;
    const int32_t token = a.token[p];
    if (p >= count) {                       // behind all rows' tokens
        if (lane == 0) a.place[token] = -1;
        return;
    }
    if (lane == 0) put_grad(a, found, token, (int32_t)p);
    copy_row(a, token, p);
    if (found.low > 0) copy_row(a, token, count + p);
    start_low(a, p > 0 ? a.target[p - 1] : -1, a.target[p], (int32_t)p, count);
}

// ---------------------------------------------------------------------------
// logits
// ---------------------------------------------------------------------------
// Tokens from n0 on by the rows of tile tm.
template <typename T, bool GRAD, int WM, int WN, int MB, int NB>
__device__ __forceinline__ void logits_tile(const LossArgs& a, int count, uint32_t tm, int n0) {
    using P = Product<T, WM, WN, MB, NB, true, true>;
    const int m0 = tm * P::TM;
    const int64_t row0 = a.row0 + m0;
    const int rows = (int)min((int64_t)P::TM, a.rows - row0);       // of the vocabulary, left in the tile
    f32x16 acc[MB][NB] = {};
    const Operand wa{a.weight + row0 * a.weight_stride, a.weight_stride, rows, a.hidden};
    const Operand xb{a.xc + (int64_t)n0 * a.pitch * 2, (int64_t)a.pitch * 2, count - n0, a.hidden};
    P::run(acc, wa, xb);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if constexpr (!GRAD) {
        // maximum and sum a token: in the lane, with the other half's rows, then over the waves
        float2(*stat)[P::TN] = reinterpret_cast<float2(*)[P::TN]>(P::lds_of_wave(0));
        static_assert(WM * P::TN * sizeof(float2) <= P::kWaveBytes, "room for the statistics");
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int n = P::n_of(j);
            float most = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < MB; ++i) acc[i][j] *= a.scale;
            if (rows < P::TM)
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (P::m_of(i, r) >= rows) acc[i][j][r] = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, acc[i][j][r]);
            most = fmaxf(most, __shfl_xor(most, 32));
            const float from = most == -__builtin_inff() ? 0.0f : most;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum += __expf(acc[i][j][r] - from);
            sum += __shfl_xor(sum, 32);
            const int32_t target = n0 + n < count ? a.target[n0 + n] - (int32_t)row0 : -1;
            if (__ballot(target >= 0 && target < P::TM) != 0) {
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (P::m_of(i, r) == target) a.picked[n0 + n] = acc[i][j][r];
            }
            if (lane < 32) stat[wave % WM][n] = make_float2(most, sum);
        }
        __syncthreads();
        for (int n = threadIdx.x; n < P::TN; n += P::kThreads) {
            if (n0 + n >= count) continue;
            float most = stat[0][n].x;
#pragma unroll
            for (int w = 1; w < WM; ++w) most = fmaxf(most, stat[w][n].x);
            const float from = most == -__builtin_inff() ? 0.0f : most;
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < WM; ++w) sum += stat[w][n].y * __expf(stat[w][n].x - from);
            a.parts[(int64_t)tm * a.tokens + n0 + n] = make_float2(most, sum);
        }
    } else {
        // the sums become d, in place
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int n = n0 + P::n_of(j), at = min(n, count - 1);
            const float lse = a.lse_at[at], g = a.grad[at];
            const int32_t target = a.target[at] - (int32_t)row0;
            const bool here = __ballot(n < count && target >= 0 && target < P::TM) != 0;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int m = P::m_of(i, r);
                    float p = __expf(fmaf(acc[i][j][r], a.scale, -lse));
                    if (m == target) p -= 1.0f;
                    acc[i][j][r] = m < rows ? p * g : 0.0f;
                }
            if (!here) continue;
            // the target's entry, if the lane has it
            bool mine = false;
            float entry = 0.0f;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const bool this_one = P::m_of(i, r) == target;
                    mine = mine || this_one;
                    entry = this_one ? acc[i][j][r] : entry;
                }
            if (!mine || n >= count) continue;
            const float low = left_of<T>(entry);
            a.low_target[n] = low;
            if (a.low_d != nullptr)
                reinterpret_cast<T*>(a.low_d)[(int64_t)n * kLowCols + a.target[n] % kLowCols] = from_f32<T>(low);
        }
        const auto row_of = [&](int n, int first) {
            return n0 + n < count ? reinterpret_cast<T*>(a.d) + (int64_t)(first + n0 + n) * a.d_pitch + m0 : nullptr;
        };
        // zeros up to the pitch
        store_rows<P, T, MB, NB>(a.d_pitch - m0, [&](int j, int i, int r) { return from_f32<T>(acc[i][j][r]); },
                                 [&](int n) { return row_of(n, 0); });
        if (a.found->low > 0)
            store_rows<P, T, MB, NB>(
                a.d_pitch - m0,
                [&](int j, int i, int r) { return from_f32<T>(left_of<T>(acc[i][j][r])); },
                [&](int n) { return row_of(n, count); });
    }
}

// Where the last round of 256 by 256 tiles has work for half of a die's 32 compute units
// at most, two take a tile of it, 128 tokens each, which costs three quarters of a round:
// 233 of 333 fp16 tokens over 32,000 rows of 1,000 are 125 tiles, 30.6 us, and 24.3 so;
// 2,047 over 50,001 of 2,048 six rounds and 32 tiles, 388 us, and 377 so (medians of 600
// launches: the first forty go through a dip of the clock to 500).  How many tokens take
// part is known here only.
constexpr uint32_t kUnitsOfDie = 32;
template <typename T, bool GRAD, int WM, int WN, int MB, int NB>
__global__ __launch_bounds__(WM * WN * 64) void loss_logits_kernel(LossArgs a) {
    constexpr int TM = WM * MB * 32, TN = WN * NB * 32;
    const int count = __builtin_amdgcn_readfirstlane(a.found->count);
    const uint32_t first = (a.piece + TM - 1) / TM, second = (count + TN - 1) / TN, v = blockIdx.x / 8;
    uint32_t tm, tn;
    if constexpr (TN == 256) {
        const uint32_t each = (first * second + 7) / 8, whole = each / kUnitsOfDie * kUnitsOfDie;
        if (v >= whole && each - whole <= kUnitsOfDie / 2) {
            const int n1 = (v - whole) % 2 * (TN / 2);
            if (tile_at(first, second, kTileGroup, whole + (v - whole) / 2, tm, tn) && (int)tn * TN + n1 < count)
                logits_tile<T, GRAD, 4, 2, 2, 2>(a, count, tm, tn * TN + n1);
            return;
        }
    }
    if (tile_at(first, second, kTileGroup, v, tm, tn)) logits_tile<T, GRAD, WM, WN, MB, NB>(a, count, tm, tn * TN);
}

// The forward pass of few tokens is bound by reading the weights once.  A workgroup has
// 64 rows of them, and its two waves take every other tile of the inner index: each
// loads tiles to LDS of its own, three ahead of the one that it multiplies, and waits for
// no other wave.  Hidden states go to registers, as far ahead.  The sums come together at
// the end, in the order of the waves.  Every workgroup begins at another tile: rows of the
// weights lie a power of two apart as a rule, and if all workgroups read the same part of
// their rows, they would meet at few of the memory's channels (8 tokens over 32,000 rows of
// 4,096: 53 us, and 43 this way).
constexpr int kFewWaves = 2, kFewRows = 64;

template <typename T, bool GRAD, int NB>
__global__ __launch_bounds__(kFewWaves * 64) void loss_few_kernel(LossArgs a) {
    // each wave's tiles as those of a workgroup of one wave
    using TileW = Tile<kFewRows, true, 1, true>;
    constexpr int MB = kFewRows / 32, kLoads = TileW::kLoads + NB * kInner / 16, kFar = 3;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // the forward pass takes tokens as they lie, the gradient those that take part
    const int tokens = GRAD ? __builtin_amdgcn_readfirstlane(a.found->count) : (int)a.tokens;
    const char* x = GRAD ? a.xc : a.x;
    const int64_t x_stride = GRAD ? (int64_t)a.pitch * 2 : a.x_stride;
    if (tokens == 0) return;
    const int64_t row0 = a.row0 + (int64_t)blockIdx.x * kFewRows;
    const int rows = (int)min((int64_t)kFewRows, a.rows - row0);
    const Operand ow{a.weight + row0 * a.weight_stride, a.weight_stride, rows, a.hidden};
    const TileW tw(ow, 0);
    f32x16 acc[MB][NB] = {};
    u32x4 fx[kFar + 1][NB][kInner / 16];
    const int steps = (a.hidden + kInner - 1) / kInner;     // of all waves
    const auto rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(x), 0,
                                                      (int)((tokens - 1) * x_stride + a.hidden * 2), 0x00027000);
    const int turn = blockIdx.x % steps;
    const auto load = [&](int s, char* stage, u32x4(&to)[NB][kInner / 16]) {     // zeros behind the last step
        const int at_step = s + turn < steps ? s + turn : s + turn - steps;
        const int k = s < steps ? at_step * kInner : steps * kInner;
        tw.load(ow, k, stage + wave * TileW::kBytes, 0);
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int ks = 0; ks < kInner / 16; ++ks) {
                const int n = j * 32 + (lane & 31), at = k + ks * 16 + (lane >> 5) * 8;
                const uint32_t offset = n < tokens && at < a.hidden ? (uint32_t)(n * x_stride) + at * 2 : kNowhere;
                to[j][ks] = __builtin_amdgcn_raw_buffer_load_b128(rx, (int)offset, 0, 0);
            }
    };
    const auto step = [&](int s, const char* stage, const u32x4(&hx)[NB][kInner / 16], char* ahead,
                          u32x4(&far)[NB][kInner / 16]) {
        // the reads of the tile that was in `ahead` are through
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        load(s + kFar * kFewWaves, ahead, far);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kFar * kLoads < 63 ? kFar * kLoads : 63) : "memory");
        const char* p = stage + wave * TileW::kBytes;
#pragma unroll
        for (int ks = 0; ks < kInner / 16; ++ks) {
            u32x4 fw[MB];
#pragma unroll
            for (int i = 0; i < MB; ++i) fw[i] = tw.operand(p, i, ks);
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = mfma_32x32x16<T>(fw[i], hx[j][ks], acc[i][j]);
        }
    };
    constexpr int kStage = kFewWaves * TileW::kBytes;
    char *s0 = lds_object<0, kStage>(), *s1 = lds_object<1, kStage>(), *s2 = lds_object<2, kStage>(),
         *s3 = lds_object<3, kStage>();
    load(wave, s0, fx[0]);
    load(wave + kFewWaves, s1, fx[1]);
    load(wave + 2 * kFewWaves, s2, fx[2]);
    for (int s = wave; s < steps; s += 4 * kFewWaves) {
        step(s, s0, fx[0], s3, fx[3]);
        step(s + kFewWaves, s1, fx[1], s0, fx[0]);
        step(s + 2 * kFewWaves, s2, fx[2], s1, fx[1]);
        step(s + 3 * kFewWaves, s3, fx[3], s2, fx[2]);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    // block i, j, register r of wave w: [(w - 1)][i][j][r][lane]
    float* sums = reinterpret_cast<float*>(lds_object<4, (kFewWaves - 1) * MB * NB * 4096>());
    if (wave > 0)
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    sums[((((wave - 1) * MB + i) * NB + j) * 16 + r) * 64 + lane] = acc[i][j][r];
    __syncthreads();
    if (wave > 0) return;
    // the sums of all waves
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
#pragma unroll
                for (int w = 0; w < kFewWaves - 1; ++w)
                    acc[i][j][r] += sums[(((w * MB + i) * NB + j) * 16 + r) * 64 + lane];
            }
    const auto m_of = [&](int i, int r) { return i * 32 + (r & 3) + 8 * (r >> 2) + 4 * (lane >> 5); };
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int n = j * 32 + (lane & 31);
        if constexpr (GRAD) {
            if (n >= tokens) continue;
            const float lse = a.lse_at[n], g = a.grad[n];
            const int64_t target = a.target[n] - row0;
            T* to = reinterpret_cast<T*>(a.d) + (int64_t)n * a.d_pitch + (row0 - a.row0);
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    AlignedPack<T, 4> v, low;       // the pitch holds whole workgroups' rows
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int m = m_of(i, 4 * q + r);
                        float p = __expf(fmaf(acc[i][j][4 * q + r], a.scale, -lse));
                        if (m == target) p -= 1.0f;
                        const float d = m < rows ? p * g : 0.0f;
                        v.v[r] = from_f32<T>(d);
                        low.v[r] = from_f32<T>(left_of<T>(d));
                    }
                    *reinterpret_cast<AlignedPack<T, 4>*>(to + m_of(i, 4 * q)) = v;
                    *reinterpret_cast<AlignedPack<T, 4>*>(to + (int64_t)tokens * a.d_pitch + m_of(i, 4 * q)) = low;
                }
        } else {
            const int32_t target = n < tokens ? target_of(a, n) : -1;
            const int64_t at = target >= 0 ? target - row0 : -1;
            float most = -__builtin_inff(), sum = 0.0f;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float v = m_of(i, r) < rows ? acc[i][j][r] * a.scale : -__builtin_inff();
                    if (m_of(i, r) == at) a.picked[n] = v;
                    acc[i][j][r] = v;
                    most = fmaxf(most, v);
                }
            most = fmaxf(most, __shfl_xor(most, 32));
            const float from = most == -__builtin_inff() ? 0.0f : most;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum += __expf(acc[i][j][r] - from);
            sum += __shfl_xor(sum, 32);
            if (lane < 32 && n < tokens) a.parts[(int64_t)n * gridDim.x + blockIdx.x] = make_float2(most, sum);
        }
    }
}

// lse and loss of one of few tokens a workgroup.
__global__ __launch_bounds__(1024) void loss_few_join_kernel(LossArgs a, int tiles) {
    __shared__ float2 stat[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t = blockIdx.x;
    float most = -__builtin_inff(), sum = 0.0f;
    const auto join = [&](float2 v) {
        const float next = fmaxf(most, v.x), from = next == -__builtin_inff() ? 0.0f : next;
        sum = sum * __expf(most - from) + v.y * __expf(v.x - from);
        most = next;
    };
    for (int i = threadIdx.x; i < tiles; i += 1024) join(a.parts[t * tiles + i]);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) join(make_float2(__shfl_xor(most, m), __shfl_xor(sum, m)));
    if (lane == 0) stat[wave] = make_float2(most, sum);
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < 16; ++w) join(stat[w]);
    const bool kept = target_of(a, t) >= 0;
    const float lse = logf(sum) + (most == -__builtin_inff() ? 0.0f : most);
    a.lse[t] = kept ? lse : 0.0f;
    a.loss[t] = kept ? lse - a.picked[t] : 0.0f;
}

// lse and loss of 64 places a workgroup: each of its sixteen waves a run of the tiles.
__global__ __launch_bounds__(1024) void loss_join_kernel(LossArgs a, int tiles) {
    __shared__ float2 stat[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t p = (int64_t)blockIdx.x * 64 + lane, count = a.found->count;
    if ((int64_t)blockIdx.x * 64 >= count) return;
    const int64_t at = min(p, count - 1);
    const int each = (tiles + 15) / 16, begin = wave * each, end = min(tiles, begin + each);
    float most = -__builtin_inff(), sum = 0.0f;
    for (int t0 = begin; t0 < end; t0 += 8) {
        float2 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = a.parts[(int64_t)min(t0 + i, end - 1) * a.tokens + at];
        float next = most;
#pragma unroll
        for (int i = 0; i < 8; ++i) next = fmaxf(next, v[i].x);
        const float from = next == -__builtin_inff() ? 0.0f : next;
        sum *= __expf(most - from);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += t0 + i < end ? v[i].y * __expf(v[i].x - from) : 0.0f;
        most = next;
    }
    stat[wave][lane] = make_float2(most, sum);
    __syncthreads();
    if (wave != 0 || p >= count) return;
    for (int w = 1; w < 16; ++w) most = fmaxf(most, stat[w][lane].x);
    const float from = most == -__builtin_inff() ? 0.0f : most;
    sum = 0.0f;
    for (int w = 0; w < 16; ++w) sum += stat[w][lane].y * __expf(stat[w][lane].x - from);
    const float lse = logf(sum) + from;
    const int32_t token = a.token[p];
    a.lse[token] = lse;
    a.loss[token] = lse - a.picked[p];
}

// ---------------------------------------------------------------------------
// dx and dweight
// ---------------------------------------------------------------------------
// A split's sums in fp32: rows n of `pitch`, added to what earlier pieces left.
template <typename P, int MB, int NB>
__device__ __forceinline__ void store_parts(const f32x16 (&acc)[MB][NB], float* to, int64_t pitch, int n_left, int m_left,
                                            bool add) {
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int n = P::n_of(j);
        if (n >= n_left) continue;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int m = P::m_of(i, 4 * q);
                if (m >= m_left) continue;
                f32x4* at = reinterpret_cast<f32x4*>(to + n * pitch + m);
                f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                if (add) v += *at;
                *at = v;
            }
    }
}

// dx_parts[split] += d W over the split's share of the piece.
template <typename T, int WM, int WN, int MB, int NB>
__global__ __launch_bounds__(WM * WN * 64) void loss_dx_kernel(LossArgs a) {
    using P = Product<T, WM, WN, MB, NB, false, true>;
    uint32_t tm, tn;
    const int tokens = __builtin_amdgcn_readfirstlane(a.found->count), count = tokens <= kLowDx ? 2 * tokens : tokens;
    if (!tile_of((uint32_t)((a.hidden + P::TM - 1) / P::TM), (uint32_t)((count + P::TN - 1) / P::TN), kTileGroup, tm, tn)) return;
    const int n0 = tn * P::TN, m0 = tm * P::TM, k0 = blockIdx.y * a.split_len;
    const int inner = min(a.split_len, a.piece - k0);
    f32x16 acc[MB][NB] = {};
    const Operand w{a.weight + (a.row0 + k0) * a.weight_stride + (int64_t)m0 * 2, a.weight_stride, a.hidden - m0, inner};
    const Operand d{a.d + ((int64_t)n0 * a.d_pitch + k0) * 2, (int64_t)a.d_pitch * 2, count - n0, inner};
    P::run(acc, w, d);
    float* to = a.dx_parts + ((int64_t)blockIdx.y * a.dx_rows + n0) * a.pitch + m0;
    store_parts<P>(acc, to, a.pitch, count - n0, a.hidden - m0, a.first == 0);
}

// dweight's rows of the piece, or with SPLIT a share of their sums.  Behind the tokens' d
// the tile's own low_d, of which a split has a share too.  With few inner indices
// writing them is what counts: then a row's tiles run one after the other (262 MB for 8
// tokens: 69 us in groups of four, 63 so).
constexpr uint32_t kWholeRows = 4096;
template <typename T, bool SPLIT, int WM, int WN, int MB, int NB>
__global__ __launch_bounds__(WM * WN * 64) void loss_dweight_kernel(LossArgs a) {
    using P = Product<T, WM, WN, MB, NB, false, false>;
    uint32_t tm, tn;
    if (!tile_of((uint32_t)((a.hidden + P::TM - 1) / P::TM), (uint32_t)((a.piece + P::TN - 1) / P::TN),
                 a.tokens <= 1024 ? kWholeRows : kTileGroup, tm, tn))
        return;
    const int count = __builtin_amdgcn_readfirstlane(a.found->count + a.found->low);
    const int n0 = tn * P::TN, m0 = tm * P::TM, k0 = SPLIT ? blockIdx.y * a.split_len : 0;
    int low0 = 0, low1 = 0;                 // places
    if (a.low_d != nullptr && a.found->low == 0 && count > 0) {
        static_assert(P::TN % kBlockRows == 0 && kLowCols % P::TN == 0 && kPieceRows % kLowCols == 0, "blocks of a tile");
        const int64_t block = (a.row0 + n0) / kBlockRows, end = (a.rows + kBlockRows - 1) / kBlockRows;
        low0 = __builtin_amdgcn_readfirstlane(a.block_first[block]);
        low1 = __builtin_amdgcn_readfirstlane(a.block_first[min(end, block + P::TN / kBlockRows)]);
        if constexpr (SPLIT) {
            const int share = ((low1 - low0 + (int)gridDim.y - 1) / (int)gridDim.y + kInner - 1) / kInner * kInner;
            low0 = min(low1, low0 + (int)blockIdx.y * share);
            low1 = min(low1, low0 + share);
        }
    }
    const int inner = SPLIT ? min(a.split_len, count - k0) : count;
    f32x16 acc[MB][NB] = {};
    const Operand x{a.xc + ((int64_t)k0 * a.pitch + m0) * 2, (int64_t)a.pitch * 2, a.hidden - m0, inner};
    const Operand d{a.d + ((int64_t)k0 * a.d_pitch + n0) * 2, (int64_t)a.d_pitch * 2, a.d_pitch - n0, inner};
    const Operand low_x{a.xc + ((int64_t)low0 * a.pitch + m0) * 2, (int64_t)a.pitch * 2, a.hidden - m0, low1 - low0};
    const Operand low_d{a.low_d + ((int64_t)low0 * kLowCols + n0 % kLowCols) * 2, kLowCols * 2, kLowCols - n0 % kLowCols,
                        low1 - low0};
    P::template run<true>(acc, x, d, low_x, low_d);
    const int n_left = a.piece - n0;
    if constexpr (SPLIT) {
        float* to = a.w_parts + ((int64_t)blockIdx.y * a.piece + n0) * a.pitch + m0;
        store_parts<P>(acc, to, a.pitch, n_left, a.hidden - m0, false);
    } else {
        const float lower = a.found->lower;
        store_rows<P, T, MB, NB>(
            a.hidden - m0, [&](int j, int i, int r) { return from_f32<T>(acc[i][j][r] * lower); },
            [&](int n) {
                return n < n_left ? reinterpret_cast<T*>(a.out + (a.row0 + n0 + n) * a.out_stride) + m0 : nullptr;
            });
    }
}

// Rows of results from the splits' sums, in order; a wave has 256 columns of a row.
__device__ __forceinline__ f32x4 split_sums(const float* from, int splits, int64_t stride) {
    f32x4 sum = {};
    for (int s0 = 0; s0 < splits; s0 += 8) {
        f32x4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const f32x4*>(from + min(s0 + i, splits - 1) * stride);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (s0 + i < splits) sum += v[i];
    }
    return sum;
}

template <typename T>
__device__ __forceinline__ void store_four(char* to, f32x4 x) {
    AlignedPack<T, 4> v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v.v[i] = from_f32<T>(x[i]);
    *reinterpret_cast<AlignedPack<T, 4>*>(to) = v;
}

// Rows of the piece of dweight.
template <typename T>
__global__ __launch_bounds__(256) void loss_dweight_finish_kernel(LossArgs a) {
    const int64_t w = wide_block() * 4 + (threadIdx.x >> 6);
    const uint32_t slabs = (a.hidden + 255) / 256;
    const int64_t r = w / slabs;
    const int c = (int)(w - r * slabs) * 256 + (threadIdx.x & 63) * 4;
    if (r >= a.piece || c >= a.hidden) return;
    const f32x4 sum = split_sums(a.w_parts + r * a.pitch + c, a.splits, (int64_t)a.piece * a.pitch);
    store_four<T>(a.out + (a.row0 + r) * a.out_stride + c * 2, sum * a.found->lower);
}

// Rows of dx: zeros for a token that takes no part.
template <typename T>
__global__ __launch_bounds__(256) void loss_dx_finish_kernel(LossArgs a, char* dx, int64_t dx_stride) {
    const int64_t w = wide_block() * 4 + (threadIdx.x >> 6);
    const uint32_t slabs = (a.hidden + 255) / 256;
    const int64_t t = w / slabs;
    const int c = (int)(w - t * slabs) * 256 + (threadIdx.x & 63) * 4;
    if (t >= a.tokens || c >= a.hidden) return;
    const int64_t p = a.place[t], count = a.found->count, stride = a.dx_rows * a.pitch;
    f32x4 sum = {};
    if (p >= 0) {
        sum = split_sums(a.dx_parts + p * a.pitch + c, a.splits, stride);
        if (count <= kLowDx) {
            sum += split_sums(a.dx_parts + (count + p) * a.pitch + c, a.splits, stride);
        } else {
            const AlignedPack<T, 4> row = *reinterpret_cast<const AlignedPack<T, 4>*>(
                a.weight + a.target[p] * a.weight_stride + c * 2);
            const float low = a.low_target[p];
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = fmaf(low, to_f32(row.v[i]), sum[i]);
        }
    }
    store_four<T>(dx + t * dx_stride + c * 2, sum * a.found->lower);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
constexpr int64_t kPieceBytes = 512ll << 20;        // of d, up to 131,072 tokens
constexpr int kFewTokens = 64;

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
int64_t tiles(int64_t x, int64_t size) { return (x + size - 1) / size; }

// Tiles of 256 by 256 sums a workgroup and one workgroup a compute unit, or of 128 by 128
// and two.  A round of the former takes 7/5 of one of the latter (106 and 75 us with 4,096
// inner indices) for twice the sums: what counts is how many rounds there are.
int tile_size(int64_t first, int64_t second) {
    const int64_t large = tiles(tiles(first, 256) * tiles(second, 256), 256);
    const int64_t small = tiles(tiles(first, 128) * tiles(second, 128), 512);
    return 7 * large <= 5 * small ? 256 : 128;
}

struct LossPlan {
    int64_t found, token, place, target, grad, lse_at, low_target, xc, parts, picked, d, dx_parts, w_parts, bytes;
    int64_t low_d, block_first, token2, target2, counts, run_found;
    int64_t dx_rows, pitch, piece, row_tiles, splits, split_len, w_splits, w_split_len;
    int tile, dx_tile, w_tile;
    bool few;
};

// How often an inner index of `length` is split, with 512 indices or more each: as makes
// the rounds of workgroups shortest, each of which costs as much as 640 indices beside its
// own (its launch, first loads and stores).
void split(int64_t first, int64_t second, int tile, int64_t length, int64_t* splits, int64_t* split_len) {
    const int64_t sums = std::max<int64_t>(1, tiles(first, tile) * tiles(second, tile)), slots = tile == 256 ? 256 : 512;
    int64_t best = INT64_MAX;
    for (int64_t s = 1; s <= 64 && (s == 1 || length / s >= 512); ++s) {
        const int64_t cost = tiles(sums * s, slots) * (length / s + 640);
        if (cost >= best) continue;
        best = cost;
        *splits = s;
    }
    *split_len = std::max<int64_t>(kInner, up((length + *splits - 1) / *splits, kInner));
    *splits = std::max<int64_t>(1, tiles(length, *split_len));
}

LossPlan loss_plan(const c3_vocab_loss_t* a, bool grad) {
    LossPlan p{};
    auto take = [&](int64_t bytes) {
        const int64_t at = p.bytes;
        p.bytes += up(bytes, 256);
        return at;
    };
    const int64_t T = a->tokens, H = a->hidden;
    p.pitch = H;
    p.found = take(sizeof(Found));
    p.few = T <= kFewTokens;
    if (!grad) {
        p.tile = tile_size(a->rows, T);
        p.row_tiles = tiles(a->rows, p.few ? kFewRows : p.tile);
        p.parts = take(8 * T * p.row_tiles);
        p.picked = take(4 * T);
        if (p.few) return p;
    }
    p.token = take(4 * T);
    p.target = take(4 * T);
    // second rows are there only where no more than kLowTokens take part
    const int64_t with_low = grad ? std::max<int64_t>(T, 2 * std::min<int64_t>(T, kLowTokens)) : T;
    p.xc = take(2 * with_low * H);
    if (!grad) return p;
    p.place = take(4 * T);
    p.grad = take(4 * T);
    p.lse_at = take(4 * T);
    p.low_target = take(4 * T);
    if (T > kLowTokens) {
        p.low_d = take(2 * T * kLowCols);
        p.block_first = take(4 * (tiles(a->rows, kBlockRows) + 1));
    }
    if (T > kGather) {
        p.token2 = take(4 * T);
        p.target2 = take(4 * T);
        p.counts = take(kSortCountBytes);
        p.run_found = take(kMostRuns * sizeof(Found));
    }
    // d of kPieceBytes, second rows with it, but 2,048 rows of the vocabulary at least; and no
    // more than that 256 rows of d stay within 31 bits of bytes
    p.piece = std::min({up(a->rows, kPieceRows), (int64_t)(1 << 22) - kPieceRows,
                        std::max<int64_t>(2048, kPieceBytes / 2 / std::max<int64_t>(with_low, 1) / kPieceRows * kPieceRows)});
    p.d = take(2 * with_low * p.piece);
    p.tile = tile_size(p.piece, T);
    p.dx_rows = T <= kLowDx ? 2 * T : std::max<int64_t>(T, 2 * kLowDx);
    p.dx_tile = tile_size(H, p.dx_rows);
    split(H, p.dx_rows, p.dx_tile, p.piece, &p.splits, &p.split_len);
    p.dx_parts = take(4 * p.splits * p.dx_rows * H);
    p.w_tile = tile_size(H, p.piece);
    split(H, p.piece, p.w_tile, with_low, &p.w_splits, &p.w_split_len);
    if (p.w_splits > 1) p.w_parts = take(4 * p.w_splits * p.piece * H);
    return p;
}

int check_sizes(const c3_vocab_loss_t* a) {
    if (a == nullptr || a->tokens < 0 || a->tokens >= (1ll << 31) || a->rows < 1 || a->rows >= (1ll << 31) ||
        a->hidden < 1 || (a->target_bytes != 4 && a->target_bytes != 8) || !(a->scale - a->scale == 0.0f) ||
        a->x_stride < 0 || a->weight_stride < 0)
        return C3_E_INVAL;
    if ((a->dtype != C3_BF16 && a->dtype != C3_F16) || a->hidden % 8 != 0 || a->hidden >= (1 << 20)) return C3_E_UNSUPPORTED;
    // a launch holds fewer than 2^32 threads
    const int64_t t = tiles(a->tokens, 256), v = tiles(a->rows, 256), h = tiles(a->hidden, 256), most = 1 << 22;
    if (a->tokens >= (1 << 26) || a->rows >= (1 << 28) || v * t >= most || h * t >= most || h * v >= most)
        return C3_E_UNSUPPORTED;
    return C3_OK;
}

// Rows of 16-byte pieces, `rows` of them.
int check_rows(const void* p, int64_t stride, int64_t rows, int64_t hidden) {
    if (p == nullptr || (rows > 1 && stride < hidden)) return C3_E_INVAL;
    if ((uintptr_t)p % 16 != 0 || (rows > 1 && stride % 8 != 0)) return C3_E_ALIGN;
    if (rows > 1 && stride >= (1ll << 22)) return C3_E_UNSUPPORTED;    // 256 rows in 31 bits of bytes
    return C3_OK;
}

LossArgs loss_args(const c3_vocab_loss_t* c, const LossPlan& p, const void* x, const void* weight, const void* targets,
                   char* ws) {
    LossArgs a{};
    a.x = static_cast<const char*>(x);
    a.weight = static_cast<const char*>(weight);
    a.targets = targets;
    // the stride of a single row says nothing
    a.x_stride = (c->tokens > 1 ? c->x_stride : c->hidden) * 2;
    a.weight_stride = (c->rows > 1 ? c->weight_stride : c->hidden) * 2;
    a.tokens = c->tokens;
    a.rows = c->rows;
    a.hidden = (int32_t)c->hidden;
    a.wide_targets = c->target_bytes == 8;
    a.half = c->dtype == C3_F16;
    a.scale = c->scale;
    a.found = reinterpret_cast<Found*>(ws + p.found);
    a.token = reinterpret_cast<int32_t*>(ws + p.token);
    a.target = reinterpret_cast<int32_t*>(ws + p.target);
    a.place = reinterpret_cast<int32_t*>(ws + p.place);
    a.grad = reinterpret_cast<float*>(ws + p.grad);
    a.lse_at = reinterpret_cast<float*>(ws + p.lse_at);
    a.low_target = reinterpret_cast<float*>(ws + p.low_target);
    // the loss itself, and the gradient of few tokens, have no such thing
    a.low_d = p.low_d > 0 ? ws + p.low_d : nullptr;
    a.block_first = reinterpret_cast<int32_t*>(ws + p.block_first);
    a.run_found = reinterpret_cast<Found*>(ws + p.run_found);
    a.dx_rows = p.dx_rows;
    a.xc = ws + p.xc;
    a.parts = reinterpret_cast<float2*>(ws + p.parts);
    a.picked = reinterpret_cast<float*>(ws + p.picked);
    a.d = ws + p.d;
    a.dx_parts = reinterpret_cast<float*>(ws + p.dx_parts);
    a.w_parts = reinterpret_cast<float*>(ws + p.w_parts);
    a.pitch = (int32_t)p.pitch;
    a.d_pitch = (int32_t)p.piece;
    return a;
}

// Calls f with the waves and blocks of a tile.
template <int WM_, int WN_, int MB_, int NB_>
struct Shape {
    static constexpr int WM = WM_, WN = WN_, MB = MB_, NB = NB_, kThreads = WM * WN * 64;
};
template <typename F>
void by_tile(int size, F f) {
    if (size == 256) f(Shape<2, 4, 4, 2>{});
    else f(Shape<2, 2, 2, 2>{});
}

template <typename T, bool GRAD>
void launch_few(const LossArgs& a, int64_t rows, hipStream_t s) {
    const dim3 grid((unsigned)tiles(rows, kFewRows)), block(kFewWaves * 64);
    if (a.tokens <= 32) loss_few_kernel<T, GRAD, 1><<<grid, block, 0, s>>>(a);
    else loss_few_kernel<T, GRAD, 2><<<grid, block, 0, s>>>(a);
}

template <typename T, bool GRAD>
void launch_logits(const LossArgs& a, int64_t rows, int tile, hipStream_t s) {
    by_tile(tile, [&](auto shape) {
        using S = decltype(shape);
        // whole rounds, as the last one's tiles may be halved
        const unsigned blocks = (unsigned)up(tile_blocks(tiles(rows, tile), tiles(a.tokens, tile)), 8 * kUnitsOfDie);
        loss_logits_kernel<T, GRAD, S::WM, S::WN, S::MB, S::NB><<<dim3(blocks), dim3(S::kThreads), 0, s>>>(a);
    });
}

// Which tokens take part, and their rows together.
void launch_tokens(const LossArgs& a, const LossPlan& p, char* ws, hipStream_t s) {
    const uint64_t blocks = (uint64_t)(a.tokens + 3) / 4;
    if (a.tokens > 0 && a.tokens <= kGather) {
        if (a.low_d != nullptr) loss_gather_kernel<true><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(a);
        else loss_gather_kernel<false><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(a);
        return;
    }
    if (a.tokens > 0 && a.dloss != nullptr) {
        SortPass q = sort_of(Ids{a.targets, a.wide_targets}, a.tokens, (uint32_t)a.rows,
                             reinterpret_cast<int32_t*>(ws + p.counts), nullptr);
        const SortLists lists{reinterpret_cast<uint32_t*>(a.target), a.token, reinterpret_cast<uint32_t*>(ws + p.target2),
                              reinterpret_cast<int32_t*>(ws + p.token2)};
        loss_count_kernel<<<dim3((unsigned)q.runs), dim3(kSortThreads), 0, s>>>(a, q);
        for (int pass = 0; pass < q.passes; ++pass) {
            set_pass(q, pass, lists);
            loss_place_kernel<<<dim3((unsigned)q.runs), dim3(kSortThreads), 0, s>>>(q);
        }
        loss_sorted_rows_kernel<<<wide_grid(blocks), dim3(256), 0, s>>>(a, q.runs);
        return;
    }
    loss_tokens_kernel<<<dim3(1), dim3(1024), 0, s>>>(a);
    if (a.tokens > 0) loss_rows_kernel<<<wide_grid(blocks), dim3(256), 0, s>>>(a);
}

template <typename T>
hipError_t launch_loss(LossArgs a, const LossPlan& p, char* ws, hipStream_t s) {
    if (p.few) {
        launch_few<T, false>(a, a.rows, s);
        loss_few_join_kernel<<<dim3((unsigned)a.tokens), dim3(1024), 0, s>>>(a, (int)p.row_tiles);
        return hipGetLastError();
    }
    launch_tokens(a, p, ws, s);
    a.row0 = 0;
    a.piece = (int32_t)a.rows;
    launch_logits<T, false>(a, a.rows, p.tile, s);
    loss_join_kernel<<<dim3((unsigned)((a.tokens + 63) / 64)), dim3(1024), 0, s>>>(a, (int)p.row_tiles);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_grad(LossArgs a, const LossPlan& p, char* ws, char* dx, int64_t dx_stride, hipStream_t s) {
    const uint64_t slabs = (a.hidden + 255) / 256;
    launch_tokens(a, p, ws, s);
    for (a.row0 = 0; a.row0 < a.rows; a.row0 += p.piece) {
        a.piece = (int32_t)std::min(p.piece, a.rows - a.row0);
        a.first = a.row0 == 0;
        if (a.tokens > 0) {
            if (p.few) launch_few<T, true>(a, a.piece, s);
            else launch_logits<T, true>(a, a.piece, p.tile, s);
            a.split_len = (int32_t)p.split_len;
            by_tile(p.dx_tile, [&](auto shape) {
                using S = decltype(shape);
                loss_dx_kernel<T, S::WM, S::WN, S::MB, S::NB>
                    <<<dim3(tile_blocks(tiles(a.hidden, p.dx_tile), tiles(a.dx_rows, p.dx_tile)), (unsigned)p.splits),
                       dim3(S::kThreads), 0, s>>>(a);
            });
        }
        a.split_len = (int32_t)p.w_split_len;
        by_tile(p.w_tile, [&](auto shape) {
            using S = decltype(shape);
            const dim3 grid(tile_blocks(tiles(a.hidden, p.w_tile), tiles(a.piece, p.w_tile)), (unsigned)p.w_splits);
            if (p.w_splits > 1)
                loss_dweight_kernel<T, true, S::WM, S::WN, S::MB, S::NB><<<grid, dim3(S::kThreads), 0, s>>>(a);
            else
                loss_dweight_kernel<T, false, S::WM, S::WN, S::MB, S::NB><<<grid, dim3(S::kThreads), 0, s>>>(a);
        });
        a.splits = (int32_t)p.w_splits;
        if (p.w_splits > 1)
            loss_dweight_finish_kernel<T><<<wide_grid((a.piece * slabs + 3) / 4), dim3(256), 0, s>>>(a);
    }
    a.splits = (int32_t)p.splits;
    if (a.tokens > 0)
        loss_dx_finish_kernel<T><<<wide_grid((a.tokens * slabs + 3) / 4), dim3(256), 0, s>>>(a, dx, dx_stride);
    return hipGetLastError();
}

}  // namespace
}  // namespace c3

extern "C" {

size_t c3_vocab_loss_workspace_size(const c3_vocab_loss_t* a) {
    return c3::check_sizes(a) == C3_OK ? (size_t)c3::loss_plan(a, false).bytes : 0;
}

size_t c3_vocab_loss_grad_workspace_size(const c3_vocab_loss_t* a) {
    return c3::check_sizes(a) == C3_OK ? (size_t)c3::loss_plan(a, true).bytes : 0;
}

int c3_vocab_loss(const c3_vocab_loss_t* a, const void* x, const void* weight, const void* targets, float* loss,
                  float* lse, void* ws, size_t ws_bytes, c3_stream_t stream) {
    using namespace c3;
    int rc = check_sizes(a);
    if (rc != C3_OK || a->tokens == 0) return rc;
    if (targets == nullptr || loss == nullptr || lse == nullptr || loss == lse) return C3_E_INVAL;
    if ((rc = check_rows(x, a->x_stride, a->tokens, a->hidden)) != C3_OK ||
        (rc = check_rows(weight, a->weight_stride, a->rows, a->hidden)) != C3_OK)
        return rc;
    if ((uintptr_t)targets % a->target_bytes != 0 || (uintptr_t)loss % 4 != 0 || (uintptr_t)lse % 4 != 0) return C3_E_ALIGN;
    const LossPlan p = loss_plan(a, false);
    if (ws == nullptr || (uintptr_t)ws % 256 != 0 || ws_bytes < (size_t)p.bytes) return C3_E_WORKSPACE;
    LossArgs k = loss_args(a, p, x, weight, targets, static_cast<char*>(ws));
    k.loss = loss;
    k.lse = lse;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const hipError_t e = a->dtype == C3_BF16 ? launch_loss<__bf16>(k, p, static_cast<char*>(ws), s)
                                             : launch_loss<_Float16>(k, p, static_cast<char*>(ws), s);
    return e == hipSuccess ? C3_OK : C3_E_HIP;
}

int c3_vocab_loss_grad(const c3_vocab_loss_t* a, const float* dloss, int64_t dloss_stride, const void* x,
                       const void* weight, const void* targets, const float* lse, void* dx, int64_t dx_stride,
                       void* dweight, int64_t dweight_stride, void* ws, size_t ws_bytes, c3_stream_t stream) {
    using namespace c3;
    int rc = check_sizes(a);
    if (rc != C3_OK) return rc;
    if ((rc = check_rows(dweight, dweight_stride, a->rows, a->hidden)) != C3_OK) return rc;
    if (a->tokens > 0) {
        if (targets == nullptr || dloss == nullptr || lse == nullptr || dloss_stride < 0) return C3_E_INVAL;
        if ((rc = check_rows(x, a->x_stride, a->tokens, a->hidden)) != C3_OK ||
            (rc = check_rows(weight, a->weight_stride, a->rows, a->hidden)) != C3_OK ||
            (rc = check_rows(dx, dx_stride, a->tokens, a->hidden)) != C3_OK)
            return rc;
        if (dx == x || dx == weight || dx == dweight || dweight == x || dweight == weight) return C3_E_INVAL;
        if ((uintptr_t)targets % a->target_bytes != 0 || (uintptr_t)dloss % 4 != 0 || (uintptr_t)lse % 4 != 0)
            return C3_E_ALIGN;
    }
    const LossPlan p = loss_plan(a, true);
    if (ws == nullptr || (uintptr_t)ws % 256 != 0 || ws_bytes < (size_t)p.bytes) return C3_E_WORKSPACE;
    LossArgs k = loss_args(a, p, x, weight, targets, static_cast<char*>(ws));
    k.dloss = dloss != nullptr ? dloss : reinterpret_cast<const float*>(ws);       // not read without tokens
    k.dloss_stride = dloss_stride;
    k.lse_in = lse;
    k.out = static_cast<char*>(dweight);
    k.out_stride = dweight_stride * 2;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const hipError_t e = a->dtype == C3_BF16 ? launch_grad<__bf16>(k, p, static_cast<char*>(ws), static_cast<char*>(dx), dx_stride * 2, s)
                                             : launch_grad<_Float16>(k, p, static_cast<char*>(ws), static_cast<char*>(dx), dx_stride * 2, s);
    return e == hipSuccess ? C3_OK : C3_E_HIP;
}

}  // extern "C"
