// Embedding lookup and its gradient (include/c3_replay.h).
//
// The lookup is bound by HBM, or for few tokens by its launch: one wave moves up to
// 256 pieces of 16 bytes of one row.
//
// The gradient of a row of the table is the sum over the tokens that read it.  Tokens
// are sorted by row, stably, so a row's tokens are a run of the sorted list in the
// order of their numbers.  A wave takes kChunk places of the list and a slab of the
// width: runs that lie within its places are summed and written, the parts of runs
// that cross into other chunks go to the workspace in fp32, and a last launch adds
// up each crossing run's parts in their order.  So a frequent token is the work of
// many waves, and every sum is a function of the list alone.
//
// Writing a whole table of zeros is most of the gradient's bytes.  It needs no sorted
// list, so it runs on the other compute units while one workgroup sorts.
#include <algorithm>

#include "c3_internal.h"
#include "c3_replay_types.h"

namespace c3 {
namespace {

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kOneSort = 16384;             // tokens that one workgroup sorts in LDS
constexpr int kPerThread = kOneSort / kSortThreads;
constexpr int kMostBits = 11;               // of a digit
constexpr int kOneBits = 9;                 // of a digit where one workgroup sorts
constexpr int kMostRuns = 64;
constexpr int kMostChunk = 64;

struct Ids {
    const void* p;
    int wide;                               // 8-byte numbers
    // The row that a token reads; `rows`, behind all of them, for none.
    __device__ __forceinline__ uint32_t key(int64_t t, uint32_t rows) const {
        if (wide) {
            const int64_t i = static_cast<const int64_t*>(p)[t];
            return (uint64_t)i < rows ? (uint32_t)i : rows;
        }
        const int32_t i = static_cast<const int32_t*>(p)[t];
        return (uint32_t)i < rows ? (uint32_t)i : rows;
    }
};

// ---------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------
template <typename T, int V, int U>
__global__ __launch_bounds__(256) void embedding_kernel(Ids ids, int64_t tokens, uint32_t rows, int64_t pieces,
                                                        uint32_t parts, const T* table, int64_t table_stride,
                                                        T* out, int64_t out_stride, float scale) {
    const int lane = threadIdx.x & 63;
    const int64_t w = wide_block() * 4 + (threadIdx.x >> 6);
    const int64_t token = w / parts, c0 = (w - token * parts) * 64 * U + lane;
    if (token >= tokens) return;
    const uint32_t id = ids.key(token, rows);
    const T* row = table + (int64_t)(id < rows ? id : 0) * table_stride;
    AlignedPack<T, V> p[U];
#pragma unroll
    for (int u = 0; u < U; ++u)             // behind the row's end the last piece again
        p[u] = *reinterpret_cast<const AlignedPack<T, V>*>(row + min(c0 + u * 64, pieces - 1) * V);
    T* to = out + token * out_stride;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (c0 + u * 64 >= pieces) continue;
        AlignedPack<T, V> y;
#pragma unroll
        for (int j = 0; j < V; ++j) y.v[j] = from_f32<T>(id < rows ? to_f32(p[u].v[j]) * scale : 0.0f);
        *reinterpret_cast<AlignedPack<T, V>*>(to + (c0 + u * 64) * V) = y;
    }
}

// ---------------------------------------------------------------------------
// sort
// ---------------------------------------------------------------------------
// One step of a stable sort by `bits` bits of the key: the places of 64 keys in a row,
// given the wave's next place of every digit (`mine`), which it moves on.
__device__ __forceinline__ int32_t place_of(uint32_t digit, bool there, int bits, int32_t* mine) {
    const int lane = threadIdx.x & 63;
    uint64_t same = __ballot(there);
    for (int b = 0; b < bits; ++b) {
        const bool bit = (digit >> b) & 1;
        const uint64_t m = __ballot(bit);
        same &= bit ? m : ~m;
    }
    int32_t place = -1;
    if (there) place = mine[digit] + __popcll(same & ((1ull << lane) - 1));
    __builtin_amdgcn_wave_barrier();
    if (there && (same >> lane) == 1) mine[digit] = place + 1;     // the last lane of its digit
    __builtin_amdgcn_wave_barrier();
    return place;
}

// lds[w][digit] holds wave w's number of keys with the digit: turns it into the wave's
// first place of the digit.  A thread takes 1 << kPerDigit digits in a row.
// `extra`: keys of earlier workgroups with the digit, `total`: of all workgroups.
template <typename Total, typename Before>
__device__ __forceinline__ void first_places(int32_t* lds, int32_t* wave_sum, int digits, Total total,
                                             Before before) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int kEach = (1 << kMostBits) / kSortThreads;
    int32_t t[kEach], sum = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int d = tid * kEach + j;
        t[j] = d < digits ? total(d) : 0;
        sum += t[j];
    }
    const int32_t own = sum;
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t up = __shfl_up(sum, d);
        if (lane >= d) sum += up;
    }
    if (lane == 63) wave_sum[wave] = sum;
    __syncthreads();
    int32_t first = sum - own;
    for (int w = 0; w < wave; ++w) first += wave_sum[w];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int d = tid * kEach + j;
        if (d < digits) {
            int32_t at = first + before(d);
            for (int w = 0; w < kSortWaves; ++w) {
                const int32_t c = lds[w * digits + d];
                lds[w * digits + d] = at;
                at += c;
            }
        }
        first += t[j];
    }
    __syncthreads();
}

// Up to kOneSort tokens: the keys stay in registers between the passes and change
// places through LDS.
__device__ void sort_one(const Ids& ids, int n, uint32_t rows, int key_bits, uint32_t* keys, int32_t* source,
                         int32_t* lds) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t* wave_sum = lds + (kSortWaves << kOneBits);
    uint32_t* key_at = reinterpret_cast<uint32_t*>(wave_sum + kSortWaves);
    uint16_t* token_at = reinterpret_cast<uint16_t*>(key_at + kOneSort);
    const int steps = (n + kSortThreads - 1) / kSortThreads;       // of 64 keys, for each wave
    const int base = wave * steps * 64 + lane;
    uint32_t k[kPerThread];
    int32_t t[kPerThread];
#pragma unroll
    for (int s = 0; s < kPerThread; ++s) {
        t[s] = base + s * 64;
        k[s] = s < steps && t[s] < n ? ids.key(t[s], rows) : 0;
    }
    const int passes = (key_bits + kOneBits - 1) / kOneBits;
    for (int pass = 0; pass < passes; ++pass) {
        const int lo = key_bits * pass / passes, bits = key_bits * (pass + 1) / passes - lo, digits = 1 << bits;
        for (int i = tid; i < kSortWaves * digits; i += kSortThreads) lds[i] = 0;
        __syncthreads();
        int32_t* mine = lds + wave * digits;
#pragma unroll
        for (int s = 0; s < kPerThread; ++s)
            if (s < steps && base + s * 64 < n) atomicAdd(&mine[(k[s] >> lo) & (digits - 1)], 1);
        __syncthreads();
        first_places(lds, wave_sum, digits,
                     [&](int d) {
                         int32_t c = 0;
                         for (int w = 0; w < kSortWaves; ++w) c += lds[w * digits + d];
                         return c;
                     },
                     [](int) { return 0; });
        const bool last = pass == passes - 1;
#pragma unroll
        for (int s = 0; s < kPerThread; ++s) {
            if (s >= steps) continue;
            const int32_t at = place_of((k[s] >> lo) & (digits - 1), base + s * 64 < n, bits, mine);
            if (at < 0) continue;
            if (last) {
                keys[at] = k[s];
                source[at] = t[s];
            } else {
                key_at[at] = k[s];
                token_at[at] = (uint16_t)t[s];
            }
        }
        __syncthreads();
        if (last) break;
#pragma unroll
        for (int s = 0; s < kPerThread; ++s) {
            if (s >= steps || base + s * 64 >= n) continue;
            k[s] = key_at[base + s * 64];
            t[s] = token_at[base + s * 64];
        }
        __syncthreads();
    }
}
constexpr int kOneSortWords = (kSortWaves << kOneBits) + kSortWaves + kOneSort + kOneSort / 2;

// Zeros in the whole table, workgroup b of `blocks`.
template <typename D, int V>
__device__ void zero_table(D* table, int64_t stride, int64_t rows, int64_t pieces, int64_t b, int64_t blocks) {
    AlignedPack<D, V> zero;
#pragma unroll
    for (int j = 0; j < V; ++j) zero.v[j] = (D)0.0f;
    if (stride == pieces * V) {             // one long row
        pieces *= rows;
        rows = 1;
        const int64_t part = (pieces + blocks - 1) / blocks, end = min(pieces, (b + 1) * part);
        for (int64_t c = b * part + threadIdx.x; c < end; c += kSortThreads)
            *reinterpret_cast<AlignedPack<D, V>*>(table + c * V) = zero;
        return;
    }
    for (int64_t r = b; r < rows; r += blocks)
        for (int64_t c = threadIdx.x; c < pieces; c += kSortThreads)
            *reinterpret_cast<AlignedPack<D, V>*>(table + r * stride + c * V) = zero;
}

// Workgroup 0 sorts, the others write zeros; or, not SORTS, all write zeros.
template <typename D, int V, bool SORTS>
__global__ __launch_bounds__(kSortThreads) void sort_and_zero_kernel(Ids ids, int n, uint32_t rows, int key_bits,
                                                                     uint32_t* keys, int32_t* source, D* table,
                                                                     int64_t stride, int64_t pieces) {
    if constexpr (SORTS) {
        __shared__ int32_t lds[kOneSortWords];
        if (blockIdx.x == 0) {
            sort_one(ids, n, rows, key_bits, keys, source, lds);
            return;
        }
    }
    zero_table<D, V>(table, stride, rows, pieces, (int64_t)blockIdx.x - SORTS, (int64_t)gridDim.x - SORTS);
}

// More tokens: a counting and a placing launch for every digit.
struct SortPass {
    Ids ids;                // of the first pass, whose keys and tokens are not written down
    const uint32_t* in_keys;
    const int32_t* in_source;
    uint32_t* keys;
    int32_t* source;
    int32_t* counts;        // [runs][digits]
    int64_t n, run;
    uint32_t rows;
    int lo, bits, first;
    __device__ __forceinline__ uint32_t key(int64_t i) const { return first ? ids.key(i, rows) : in_keys[i]; }
};

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortPass p) {
    __shared__ int32_t lds[1 << kMostBits];
    const int digits = 1 << p.bits;
    for (int d = threadIdx.x; d < digits; d += kSortThreads) lds[d] = 0;
    __syncthreads();
    const int64_t begin = (int64_t)blockIdx.x * p.run, end = min(begin + p.run, p.n);
    for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads)
        atomicAdd(&lds[(p.key(i) >> p.lo) & (digits - 1)], 1);
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kSortThreads) p.counts[(int64_t)blockIdx.x * digits + d] = lds[d];
}

__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(SortPass p) {
    __shared__ int32_t lds[(kSortWaves << kMostBits) + kSortWaves];
    const int digits = 1 << p.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t* wave_sum = lds + kSortWaves * digits;
    const int64_t begin = (int64_t)blockIdx.x * p.run, end = min(begin + p.run, p.n);
    const int64_t part = p.run / kSortWaves, wb = begin + wave * part, we = min(wb + part, end);
    for (int i = threadIdx.x; i < kSortWaves * digits; i += kSortThreads) lds[i] = 0;
    __syncthreads();
    int32_t* mine = lds + wave * digits;
    for (int64_t i = wb + lane; i < we; i += 64) atomicAdd(&mine[(p.key(i) >> p.lo) & (digits - 1)], 1);
    __syncthreads();
    const int runs = gridDim.x;
    auto counted = [&](int d, int before) {
        int32_t c[16], sum = 0;             // sixteen loads in flight
        for (int b = 0; b < before; b += 16) {
#pragma unroll
            for (int j = 0; j < 16; ++j) c[j] = p.counts[(int64_t)min(b + j, runs - 1) * digits + d];
#pragma unroll
            for (int j = 0; j < 16; ++j) sum += b + j < before ? c[j] : 0;
        }
        return sum;
    };
    first_places(lds, wave_sum, digits, [&](int d) { return counted(d, runs); },
                 [&](int d) { return counted(d, (int)blockIdx.x); });
    for (int64_t i0 = wb; i0 < we; i0 += 64) {
        const int64_t i = i0 + lane;
        const uint32_t k = i < we ? p.key(i) : 0;
        const int32_t at = place_of((k >> p.lo) & (digits - 1), i < we, p.bits, mine);
        if (at < 0) continue;
        p.keys[at] = k;
        p.source[at] = p.first ? (int32_t)i : p.in_source[i];
    }
}

// ---------------------------------------------------------------------------
// sums
// ---------------------------------------------------------------------------
struct SumArgs {
    const uint32_t* keys;
    const int32_t* source;
    float* parts;               // [chunks][2][width]: of the run from before, of the run that goes on
    int64_t n, chunks, pieces, dout_stride, table_stride, width;
    uint32_t rows;
    int32_t chunk;
    uint32_t slabs;
    float scale;
    int32_t accumulate;
};

template <typename D, int V>
__device__ __forceinline__ void write_row(const SumArgs& a, D* table, uint32_t row, int64_t c, const float* sum) {
    AlignedPack<D, V>* to = reinterpret_cast<AlignedPack<D, V>*>(table + (int64_t)row * a.table_stride + c * V);
    AlignedPack<D, V> y;
    if (a.accumulate) y = *to;
#pragma unroll
    for (int j = 0; j < V; ++j) y.v[j] = from_f32<D>(a.accumulate ? fmaf(sum[j], a.scale, to_f32(y.v[j])) : sum[j] * a.scale);
    *to = y;
}

// A wave: the places of one chunk, 64 pieces of the width.
template <typename S, typename D, int V>
__global__ __launch_bounds__(256) void embedding_sum_kernel(SumArgs a, const S* dout, D* table) {
    const int lane = threadIdx.x & 63;
    const int64_t w = wide_block() * 4 + (threadIdx.x >> 6);
    const int64_t chunk = w / a.slabs, c = (w - chunk * a.slabs) * 64 + lane;
    if (chunk >= a.chunks) return;
    const int64_t begin = chunk * a.chunk;
    const int count = (int)min((int64_t)a.chunk, a.n - begin);
    // lane i's key and token; the keys before and behind the chunk
    const uint32_t my_key = a.keys[begin + min(lane, count - 1)];
    const int32_t my_token = a.source[begin + min(lane, count - 1)];
    const uint32_t before = begin > 0 ? a.keys[begin - 1] : a.rows;
    const uint32_t behind = begin + count < a.n ? a.keys[begin + count] : a.rows;
    const bool in = c < a.pieces;
    const int64_t col = (in ? c : 0) * V;
    float sum[V] = {};
    bool whole = (uint32_t)__builtin_amdgcn_readlane(my_key, 0) != before;      // the run began here
    for (int i0 = 0; i0 < count; i0 += 8) {
        AlignedPack<S, V> p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)         // the rows stand without a branch between the loads
            p[i] = *reinterpret_cast<const AlignedPack<S, V>*>(
                dout + (int64_t)__builtin_amdgcn_readlane(my_token, min(i0 + i, count - 1)) * a.dout_stride + col);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = i0 + i;
            if (at >= count) break;
            const uint32_t key = __builtin_amdgcn_readlane(my_key, at);
            if (key >= a.rows) return;      // the tokens without a row stand last
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += to_f32(p[i].v[j]);
            const uint32_t next = at + 1 < count ? (uint32_t)__builtin_amdgcn_readlane(my_key, (at + 1) & 63) : behind;
            if (next == key && at + 1 < count) continue;
            if (in) {
                if (whole && next != key) {
                    write_row<D, V>(a, table, key, c, sum);
                } else {
                    float* to = a.parts + (chunk * 2 + whole) * a.width + c * V;
#pragma unroll
                    for (int j = 0; j < V; ++j) to[j] = sum[j];
                }
            }
            whole = true;
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] = 0.0f;
        }
    }
}

// A workgroup: the parts of the run that begins in one chunk and goes on, 64 pieces of
// the width.  Its four waves take a quarter of the parts each.
template <typename D, int V>
__global__ __launch_bounds__(256) void embedding_join_kernel(SumArgs a, D* table) {
    __shared__ float quarter[3][V][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t b = wide_block(), chunk = b / a.slabs, c = (b - chunk * a.slabs) * 64 + lane;
    if (chunk + 1 >= a.chunks) return;
    const int64_t begin = chunk * a.chunk, next = begin + a.chunk;
    const uint32_t key = a.keys[next - 1];
    if (key >= a.rows || a.keys[next] != key) return;
    if (a.keys[begin] == key && begin > 0 && a.keys[begin - 1] == key) return;      // began before
    // the run's last place
    int64_t lo = next, hi = a.n - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) >> 1;
        if (a.keys[mid] == key) lo = mid; else hi = mid - 1;
    }
    const int64_t last = lo / a.chunk, count = last - chunk + 1, each = (count + 3) / 4;
    const bool in = c < a.pieces;
    const int64_t col = (in ? c : 0) * V;
    float sum[V] = {};
    const int64_t end = min(count, (wave + 1) * each);
    for (int64_t i0 = wave * each; i0 < end; i0 += 8) {
        AlignedPack<float, V == 1 ? 1 : 4> p[8][V == 1 ? 1 : V / 4];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t at = min(i0 + i, end - 1);
            const float* from = a.parts + ((chunk + at) * 2 + (at == 0)) * a.width + col;
#pragma unroll
            for (int j = 0; j < (V == 1 ? 1 : V / 4); ++j)
                p[i][j] = *reinterpret_cast<const AlignedPack<float, V == 1 ? 1 : 4>*>(from + j * 4);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i0 + i < end)
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += p[i][j / 4].v[j % 4];
    }
    if (wave > 0)
#pragma unroll
        for (int j = 0; j < V; ++j) quarter[wave - 1][j][lane] = sum[j];
    __syncthreads();
    if (wave > 0 || !in) return;
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = sum[j] + quarter[0][j][lane] + quarter[1][j][lane] + quarter[2][j][lane];
    write_row<D, V>(a, table, key, c, sum);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
int key_bits_of(int64_t rows) {             // keys are 0 .. rows
    int bits = 1;
    while ((rows >> bits) != 0) ++bits;
    return bits;
}

// Places of a wave.  Sixteen, and with enough of them to fill the device 64, which
// writes and reads a quarter of the parts.  The sizes alone decide, not the alignment:
// the order of the sums goes by it.
int chunk_of(int64_t n, int64_t hidden) {
    return n * ((hidden + 511) / 512) >= ((int64_t)1 << 19) ? kMostChunk : 16;
}

// What stands where in the workspace.
struct GradPlan {
    int64_t keys, source, keys2, source2, counts, parts, bytes;
    bool one;
};
GradPlan grad_plan(int64_t n, int64_t hidden) {
    GradPlan p{};
    auto take = [&](int64_t bytes) {
        const int64_t at = p.bytes;
        p.bytes += (bytes + 255) / 256 * 256;
        return at;
    };
    p.one = n <= kOneSort;
    p.keys = take(4 * n);
    p.source = take(4 * n);
    if (!p.one) {
        p.keys2 = take(4 * n);
        p.source2 = take(4 * n);
        p.counts = take(4 * (int64_t)kMostRuns << kMostBits);
    }
    const int chunk = chunk_of(n, hidden);
    p.parts = take(4 * 2 * ((n + chunk - 1) / chunk) * hidden);
    if (p.bytes < 256) p.bytes = 256;
    return p;
}

struct GradCall {
    Ids ids;
    int64_t n, rows, hidden, dout_stride, table_stride;
    const void* dout;
    void* table;
    float scale;
    int accumulate;
    char* ws;
    hipStream_t s;
};

template <typename S, typename D, int V>
hipError_t launch_grad(const GradCall& g) {
    const GradPlan p = grad_plan(g.n, g.hidden);
    SumArgs a{};
    a.keys = reinterpret_cast<uint32_t*>(g.ws + p.keys);
    a.source = reinterpret_cast<int32_t*>(g.ws + p.source);
    a.parts = reinterpret_cast<float*>(g.ws + p.parts);
    a.n = g.n;
    a.pieces = g.hidden / V;
    a.width = g.hidden;
    a.dout_stride = g.dout_stride;
    a.table_stride = g.table_stride;
    a.rows = (uint32_t)g.rows;
    a.slabs = (uint32_t)((a.pieces + 63) / 64);
    a.chunk = chunk_of(g.n, g.hidden);
    a.chunks = (g.n + a.chunk - 1) / a.chunk;
    a.scale = g.scale;
    a.accumulate = g.accumulate;
    const int key_bits = key_bits_of(g.rows);
    uint32_t* keys = reinterpret_cast<uint32_t*>(g.ws + p.keys);
    int32_t* source = reinterpret_cast<int32_t*>(g.ws + p.source);
    // 1,024 threads write 64 KiB of zeros at least, two workgroups a compute unit
    const int64_t bytes = g.rows * g.hidden * (int64_t)sizeof(D);
    const int64_t most = std::min<int64_t>(512, (bytes + 65535) / 65536);
    const unsigned zeros = g.accumulate ? 0u : (unsigned)most;
    if (p.one && g.n > 0)
        sort_and_zero_kernel<D, V, true><<<dim3(1 + zeros), dim3(kSortThreads), 0, g.s>>>(
            g.ids, (int)g.n, a.rows, key_bits, keys, source, static_cast<D*>(g.table), g.table_stride, a.pieces);
    else if (zeros > 0)
        sort_and_zero_kernel<D, V, false><<<dim3(zeros), dim3(kSortThreads), 0, g.s>>>(
            g.ids, 0, a.rows, key_bits, keys, source, static_cast<D*>(g.table), g.table_stride, a.pieces);
    if (g.n == 0) return hipGetLastError();
    if (!p.one) {
        const int passes = (key_bits + kMostBits - 1) / kMostBits;
        int64_t run = (g.n + kMostRuns - 1) / kMostRuns;
        run = (run + kSortThreads - 1) / kSortThreads * kSortThreads;
        const unsigned runs = (unsigned)((g.n + run - 1) / run);
        for (int pass = 0; pass < passes; ++pass) {
            // the last pass writes to the first pair of lists
            const bool to_first = (passes - 1 - pass) % 2 == 0;
            uint32_t* k2 = reinterpret_cast<uint32_t*>(g.ws + p.keys2);
            int32_t* s2 = reinterpret_cast<int32_t*>(g.ws + p.source2);
            SortPass q{};
            q.ids = g.ids;
            q.in_keys = to_first ? k2 : keys;
            q.in_source = to_first ? s2 : source;
            q.keys = to_first ? keys : k2;
            q.source = to_first ? source : s2;
            q.counts = reinterpret_cast<int32_t*>(g.ws + p.counts);
            q.n = g.n;
            q.run = run;
            q.rows = a.rows;
            q.lo = key_bits * pass / passes;
            q.bits = key_bits * (pass + 1) / passes - q.lo;
            q.first = pass == 0;
            sort_count_kernel<<<dim3(runs), dim3(kSortThreads), 0, g.s>>>(q);
            sort_place_kernel<<<dim3(runs), dim3(kSortThreads), 0, g.s>>>(q);
        }
    }
    embedding_sum_kernel<S, D, V><<<wide_grid((uint64_t)(a.chunks * a.slabs + 3) / 4), dim3(256), 0, g.s>>>(
        a, static_cast<const S*>(g.dout), static_cast<D*>(g.table));
    if (a.chunks > 1)
        embedding_join_kernel<D, V><<<wide_grid((uint64_t)(a.chunks - 1) * a.slabs), dim3(256), 0, g.s>>>(
            a, static_cast<D*>(g.table));
    return hipGetLastError();
}

template <typename S, typename D>
hipError_t grad_of(const GradCall& g) {
    constexpr int V = 16 / sizeof(S);
    // a piece is 16 bytes of dout, and of the table 16 or, in fp32 for a 16-bit dout, 32
    const bool wide = g.hidden % V == 0 && g.dout_stride % V == 0 && g.table_stride % V == 0 &&
                      (uintptr_t)g.dout % 16 == 0 && (uintptr_t)g.table % (V * sizeof(D)) == 0;
    return wide ? launch_grad<S, D, V>(g) : launch_grad<S, D, 1>(g);
}

struct LookupCall {
    Ids ids;
    int64_t n, rows, hidden, table_stride, out_stride;
    const void* table;
    void* out;
    float scale;
    hipStream_t s;
};

template <typename T, int V>
hipError_t launch_lookup(const LookupCall& g) {
    const int64_t pieces = g.hidden / V;
    // four pieces a lane, or one where that leaves the device waves to spare
    const bool few = g.n * ((pieces + 255) / 256) < 4096;
    const uint32_t parts = (uint32_t)(few ? (pieces + 63) / 64 : (pieces + 255) / 256);
    const dim3 grid = wide_grid((uint64_t)(g.n * parts + 3) / 4);
    if (few)
        embedding_kernel<T, V, 1><<<grid, dim3(256), 0, g.s>>>(g.ids, g.n, (uint32_t)g.rows, pieces, parts,
                                                              static_cast<const T*>(g.table), g.table_stride,
                                                              static_cast<T*>(g.out), g.out_stride, g.scale);
    else
        embedding_kernel<T, V, 4><<<grid, dim3(256), 0, g.s>>>(g.ids, g.n, (uint32_t)g.rows, pieces, parts,
                                                              static_cast<const T*>(g.table), g.table_stride,
                                                              static_cast<T*>(g.out), g.out_stride, g.scale);
    return hipGetLastError();
}

template <typename T>
hipError_t lookup_of(const LookupCall& g) {
    constexpr int V = 16 / sizeof(T);
    const bool wide = g.hidden % V == 0 && g.table_stride % V == 0 && g.out_stride % V == 0 &&
                      (uintptr_t)g.table % 16 == 0 && (uintptr_t)g.out % 16 == 0;
    return wide ? launch_lookup<T, V>(g) : launch_lookup<T, 1>(g);
}

// What both calls ask of their sizes.
int check_sizes(const c3_embedding_t* a) {
    if (a == nullptr || a->tokens < 0 || a->tokens >= (1ll << 31) || a->rows < 1 || a->rows >= (1ll << 31) ||
        a->hidden < 0 || a->hidden >= (1ll << 31) || a->row_stride < 0 || a->table_stride < 0 ||
        (a->id_bytes != 4 && a->id_bytes != 8) || !(a->scale - a->scale == 0.0f))
        return C3_E_INVAL;
    if (replay_elem_size(a->dtype) == 0) return C3_E_UNSUPPORTED;
    return C3_OK;
}

}  // namespace
}  // namespace c3

extern "C" {

int c3_embedding(const c3_embedding_t* a, const void* ids, const void* table, void* out, c3_stream_t stream) {
    using namespace c3;
    const int rc = check_sizes(a);
    if (rc != C3_OK) return rc;
    if (a->tokens == 0 || a->hidden == 0) return C3_OK;
    if (ids == nullptr || table == nullptr || out == nullptr || table == out) return C3_E_INVAL;
    if ((a->tokens > 1 && a->row_stride < a->hidden) || (a->rows > 1 && a->table_stride < a->hidden)) return C3_E_INVAL;
    const int es = replay_elem_size(a->dtype);
    if ((uintptr_t)ids % a->id_bytes != 0 || (uintptr_t)table % es != 0 || (uintptr_t)out % es != 0) return C3_E_ALIGN;
    // waves are counted in 32 bits
    if (a->tokens * ((a->hidden + 63) / 64) >= (1ll << 36)) return C3_E_UNSUPPORTED;
    const LookupCall g{{ids, a->id_bytes == 8}, a->tokens, a->rows, a->hidden, a->table_stride, a->row_stride, table,
                       out, a->scale, reinterpret_cast<hipStream_t>(stream)};
    const hipError_t e = a->dtype == C3_F32 ? lookup_of<float>(g)
                         : a->dtype == C3_BF16 ? lookup_of<__bf16>(g) : lookup_of<_Float16>(g);
    return e == hipSuccess ? C3_OK : C3_E_HIP;
}

size_t c3_embedding_grad_workspace_size(const c3_embedding_t* a) {
    using namespace c3;
    if (check_sizes(a) != C3_OK) return 0;
    return (size_t)grad_plan(a->tokens, a->hidden).bytes;
}

int c3_embedding_grad(const c3_embedding_t* a, const void* dout, const void* ids, void* dtable, int table_dtype,
                      int accumulate, void* ws, size_t ws_bytes, c3_stream_t stream) {
    using namespace c3;
    const int rc = check_sizes(a);
    if (rc != C3_OK) return rc;
    if (table_dtype != a->dtype && table_dtype != C3_F32) return C3_E_UNSUPPORTED;
    if (a->hidden == 0 || (a->tokens == 0 && accumulate)) return C3_OK;
    if (dtable == nullptr || dtable == dout || (a->tokens > 0 && (ids == nullptr || dout == nullptr)))
        return C3_E_INVAL;
    if ((a->tokens > 1 && a->row_stride < a->hidden) || (a->rows > 1 && a->table_stride < a->hidden)) return C3_E_INVAL;
    if ((uintptr_t)ids % a->id_bytes != 0 || (uintptr_t)dout % replay_elem_size(a->dtype) != 0 ||
        (uintptr_t)dtable % replay_elem_size(table_dtype) != 0)
        return C3_E_ALIGN;
    if (ws == nullptr || (uintptr_t)ws % 256 != 0 || ws_bytes < (size_t)grad_plan(a->tokens, a->hidden).bytes)
        return C3_E_WORKSPACE;
    // workgroups are counted in 32 bits
    if (a->tokens * ((a->hidden + 63) / 64) >= (1ll << 34)) return C3_E_UNSUPPORTED;
    const GradCall g{{ids, a->id_bytes == 8}, a->tokens, a->rows, a->hidden, a->row_stride, a->table_stride, dout,
                     dtable, a->scale, accumulate != 0, static_cast<char*>(ws), reinterpret_cast<hipStream_t>(stream)};
    hipError_t e;
    if (a->dtype == C3_F32)
        e = grad_of<float, float>(g);
    else if (a->dtype == C3_BF16)
        e = table_dtype == C3_F32 ? grad_of<__bf16, float>(g) : grad_of<__bf16, __bf16>(g);
    else
        e = table_dtype == C3_F32 ? grad_of<_Float16, float>(g) : grad_of<_Float16, _Float16>(g);
    return e == hipSuccess ? C3_OK : C3_E_HIP;
}

}  // extern "C"
