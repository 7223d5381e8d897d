// Embedding lookup and its gradient (include/c3_replay.h).
//
// The lookup is bound by HBM, or for few tokens by its launch: one wave moves up to
// 256 pieces of 16 bytes of one row.  8,191 fp32 rows of 2,048: 134 MB in 17 us, where
// the caches take most of the results in; 16 bf16 rows of 4,096: 2.6 us.
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
// list, so it runs beside the sort, on compute units that have no part in that.
//
// 16,384 bf16 tokens into 32,000 rows of 4,096: 22 us for the sort's three launches, 57
// for the sums and what is left of the zeros (HBM), 9 to join.  4,095 fp16 tokens into
// 131,072 fp32 rows of 1,000: 24 us for one workgroup's sort and 151 of 520 MB of zeros
// beside it, 66 for the sums and the others at 5.8 TB/s, 5 to join.
#include <algorithm>

#include "c3_sort.h"

namespace c3 {
namespace {

constexpr int kOneSort = 4096;              // tokens that one workgroup sorts in LDS
constexpr int kPerThread = kOneSort / kSortThreads;
constexpr int kMostChunk = 64;
constexpr int kSumRows = 16;                // rows that a wave has in flight

// V elements in memory.  WIDE: on their own size; else on an element's, which the memory
// units take too (the gradient of 16,384 bf16 tokens of 4,097 into 32,000 rows: 113 us,
// and 226 element by element).  A row's last piece then begins V elements before its end,
// and what it shares with the piece before is written twice, with the same bits.
template <typename T, int V, bool WIDE>
struct alignas(WIDE ? sizeof(T) * V : sizeof(T)) Piece {
    T v[V];
};
template <int V, bool WIDE>
__device__ __forceinline__ int64_t column(int64_t piece, int64_t hidden) {
    return WIDE ? piece * V : min(piece * V, hidden - V);
}

// ---------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------
template <typename T, int V, bool WIDE, int U>
__global__ __launch_bounds__(256) void embedding_kernel(Ids ids, int64_t tokens, uint32_t rows, int64_t hidden,
                                                        int64_t pieces, uint32_t parts, const T* table, int64_t table_stride,
                                                        T* out, int64_t out_stride, float scale) {
    const int lane = threadIdx.x & 63;
    const int64_t w = wide_block() * 4 + (threadIdx.x >> 6);
    const int64_t token = w / parts, c0 = (w - token * parts) * 64 * U + lane;
    if (token >= tokens) return;
    const uint32_t id = ids.key(token, rows);
    const T* row = table + (int64_t)(id < rows ? id : 0) * table_stride;
    using Pack = Piece<T, V, WIDE>;
    Pack p[U];
#pragma unroll
    for (int u = 0; u < U; ++u)             // behind the row's end the last piece again
        p[u] = *reinterpret_cast<const Pack*>(row + column<V, WIDE>(min(c0 + u * 64, pieces - 1), hidden));
    T* to = out + token * out_stride;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (c0 + u * 64 >= pieces) continue;
        Pack y;
#pragma unroll
        for (int j = 0; j < V; ++j) y.v[j] = from_f32<T>(id < rows ? to_f32(p[u].v[j]) * scale : 0.0f);
        *reinterpret_cast<Pack*>(to + column<V, WIDE>(c0 + u * 64, hidden)) = y;
    }
}

// ---------------------------------------------------------------------------
// sort
// ---------------------------------------------------------------------------
// Up to kOneSort tokens: the keys stay in registers between the passes and change
// places through LDS.
__device__ void sort_one(const Ids& ids, int n, uint32_t rows, int key_bits, uint32_t* keys, int32_t* source,
                         uint8_t* present, int32_t* lds) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t* wave_sum = lds + (kSortWaves << kMostBits);
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
    for (uint32_t i = tid; i <= rows / 4; i += kSortThreads) reinterpret_cast<uint32_t*>(present)[i] = 0;
    // written before the first mark, barriers later; a fence for the whole device would
    // write back what the zeros' workgroups leave in the cache (30 us)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const int passes = (key_bits + kMostBits - 1) / kMostBits;
    for (int pass = 0; pass < passes; ++pass) {
        const int lo = key_bits * pass / passes, bits = key_bits * (pass + 1) / passes - lo, digits = 1 << bits;
        for (int i = tid; i < kSortWaves * digits; i += kSortThreads) lds[i] = 0;
        __syncthreads();
        int32_t* mine = lds + wave * digits;
#pragma unroll
        for (int s = 0; s < kPerThread; ++s)
            if (s < steps && base + s * 64 < n) atomicAdd(&mine[(k[s] >> lo) & (digits - 1)], 1);
        __syncthreads();
        first_places(lds, wave_sum, digits, [&](int d, int32_t& total, int32_t&) {
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) total += lds[w * digits + d];
        });
        const bool last = pass == passes - 1;
#pragma unroll
        for (int s = 0; s < kPerThread; ++s) {
            if (s >= steps) continue;
            const int32_t at = place_of((k[s] >> lo) & (digits - 1), base + s * 64 < n, bits, mine);
            if (at < 0) continue;
            if (last) {
                keys[at] = k[s];
                source[at] = t[s];
                if (k[s] < rows) present[k[s]] = 1;
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
constexpr int kOneSortWords = (kSortWaves << kMostBits) + kSortWaves + kOneSort + kOneSort / 2;

// Rows row0 .. row1 - 1 as zeros, each by one of the workgroups from `first` on, but for
// those that `present` (null: none) marks.  They go past the caches, in whole lines: what
// the sums read stays there (16,384 tokens into 32,000 rows of 4,096 in bf16: 112 us, and
// 95 so).
template <typename D, int V, bool WIDE>
struct Zeros {
    static constexpr int kUnit = V == 1 ? 1 : 16 / (int)sizeof(D);     // elements of a store
    typedef uint32_t Loose __attribute__((ext_vector_type(4), aligned(2)));
    D* table;
    int64_t stride, row0, row1;
    const uint8_t* present;
    FastDiv units;                          // of a row, the last as a last Piece
    int64_t hidden;
    uint32_t each;                          // rows of a workgroup
    int first;
    static Zeros of(void* table, int64_t stride, int64_t hidden) {      // `each` is set for a launch
        Zeros z{};
        z.table = static_cast<D*>(table);
        z.stride = stride;
        z.units = FastDiv((uint32_t)((hidden + kUnit - 1) / kUnit));
        z.hidden = hidden;
        return z;
    }
    int64_t blocks() const { return (row1 - row0 + each - 1) / each; }
    __device__ __forceinline__ void write() const {
        const int64_t at = row0 + (wide_block() - first) * each;
        const uint32_t all = (uint32_t)max((int64_t)0, min((int64_t)each, row1 - at)) * units.d;
        constexpr int kAhead = 4;           // marks on their way together, without a branch between them
        for (uint32_t i0 = threadIdx.x; i0 < all; i0 += blockDim.x * kAhead) {
            D* to[kAhead];
            uint8_t mark[kAhead];
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const uint32_t i = min(i0 + q * blockDim.x, all - 1), r = units.quot(i), c = i - r * units.d;
                to[q] = table + (at + r) * stride + column<kUnit, WIDE>(c, hidden);
                mark[q] = present != nullptr ? present[at + r] : 0;
            }
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                if (mark[q] != 0 || i0 + q * blockDim.x >= all) continue;
                if constexpr (V == 1) *to[q] = (D)0.0f;
                else if constexpr (WIDE) __builtin_nontemporal_store(u32x4{}, reinterpret_cast<u32x4*>(to[q]));
                else __builtin_nontemporal_store(Loose{}, reinterpret_cast<Loose*>(to[q]));
            }
        }
    }
};

// Workgroup 0 sorts, the others write zeros.
template <typename D, int V, bool WIDE>
__global__ __launch_bounds__(kSortThreads) void sort_one_kernel(Ids ids, int n, uint32_t rows, int key_bits,
                                                                uint32_t* keys, int32_t* source, uint8_t* present,
                                                                Zeros<D, V, WIDE> z) {
    __shared__ int32_t lds[kOneSortWords];
    if (wide_block() < z.first)
        sort_one(ids, n, rows, key_bits, keys, source, present, lds);
    else
        z.write();
}

// More tokens: a launch that counts, and one for each digit.
template <typename D, int V, bool WIDE>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortPass p, Zeros<D, V, WIDE> z) {
    if (wide_block() >= z.first) z.write();
    else sort_count(p);
}
template <typename D, int V, bool WIDE>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(SortPass p, Zeros<D, V, WIDE> z) {
    if (wide_block() >= z.first) z.write();
    else sort_place(p);
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

// skip: elements that the piece before adds to.
template <typename D, int V, bool WIDE>
__device__ __forceinline__ void write_row(const SumArgs& a, D* table, uint32_t row, int64_t col, int skip, const float* sum) {
    using Pack = Piece<D, V, WIDE>;
    Pack* to = reinterpret_cast<Pack*>(table + (int64_t)row * a.table_stride + col);
    Pack y;
    if (!WIDE && a.accumulate && skip != 0) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j >= skip) to->v[j] = from_f32<D>(fmaf(sum[j], a.scale, to_f32(to->v[j])));
        return;
    }
    if (a.accumulate) y = *to;
#pragma unroll
    for (int j = 0; j < V; ++j) y.v[j] = from_f32<D>(a.accumulate ? fmaf(sum[j], a.scale, to_f32(y.v[j])) : sum[j] * a.scale);
    *to = y;
}

// A wave: the places of one chunk, 64 pieces of the width.
template <typename S, typename D, int V, bool WIDE>
__global__ __launch_bounds__(256) void embedding_sum_kernel(SumArgs a, const S* dout, D* table, Zeros<D, V, WIDE> z) {
    if (wide_block() >= z.first) {
        z.write();
        return;
    }
    const int lane = threadIdx.x & 63;
    // the same for every lane, in scalar registers; chunks are fewer than 2^31
    const int64_t w = wide_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t chunk = __builtin_amdgcn_readfirstlane((int)(w / a.slabs)), c = (w - chunk * a.slabs) * 64 + lane;
    if (chunk >= a.chunks) return;
    const int64_t begin = chunk * a.chunk;
    const int count = (int)min((int64_t)a.chunk, a.n - begin);
    // lane i's key and token; the keys before and behind the chunk
    const uint32_t my_key = a.keys[begin + min(lane, count - 1)];
    const int32_t my_token = a.source[begin + min(lane, count - 1)];
    const uint32_t before = begin > 0 ? a.keys[begin - 1] : a.rows;
    const uint32_t behind = begin + count < a.n ? a.keys[begin + count] : a.rows;
    const bool in = c < a.pieces;
    const int64_t col = column<V, WIDE>(in ? c : 0, a.width);
    const int skip = in ? (int)(c * V - col) : 0;
    float sum[V] = {};
    bool whole = (uint32_t)__builtin_amdgcn_readlane(my_key, 0) != before;      // the run began here
    for (int i0 = 0; i0 < count; i0 += kSumRows) {
        Piece<S, V, WIDE> p[kSumRows];
#pragma unroll
        for (int i = 0; i < kSumRows; ++i)  // the rows stand without a branch between the loads
            p[i] = *reinterpret_cast<const Piece<S, V, WIDE>*>(
                dout + (int64_t)__builtin_amdgcn_readlane(my_token, min(i0 + i, count - 1)) * a.dout_stride + col);
#pragma unroll
        for (int i = 0; i < kSumRows; ++i) {
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
                    write_row<D, V, WIDE>(a, table, key, col, skip, sum);
                } else {
                    float* to = a.parts + (chunk * 2 + whole) * a.width + col;
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
template <typename D, int V, bool WIDE>
__global__ __launch_bounds__(256) void embedding_join_kernel(SumArgs a, D* table) {
    __shared__ float quarter[3][V][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t b = wide_block(), chunk = b / a.slabs, c = (b - chunk * a.slabs) * 64 + lane;
    if (chunk + 1 >= a.chunks) return;
    const int64_t begin = chunk * a.chunk, next = begin + a.chunk;
    const uint32_t key = a.keys[next - 1], behind = a.keys[next], at_begin = a.keys[begin];
    const uint32_t before = begin > 0 ? a.keys[begin - 1] : a.rows;
    if (key >= a.rows || behind != key || (at_begin == key && before == key)) return;   // no run, or it began before
    // the run's last place: 64 places are looked at in a step, not one
    int64_t lo = next, hi = a.n;            // keys[lo] == key, and from hi on it is another
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + 63) / 64, probe = lo + lane * step;
        const uint64_t same = __ballot(probe < hi && a.keys[min(probe, hi - 1)] == key);
        const int last = 63 - __clzll(same);            // lane 0 looks at lo
        hi = min(hi, lo + (last + 1) * step);
        lo += last * step;
    }
    const int64_t last = lo / a.chunk, count = last - chunk + 1, each = (count + 3) / 4;
    const bool in = c < a.pieces;
    const int64_t col = column<V, WIDE>(in ? c : 0, a.width);
    const int skip = in ? (int)(c * V - col) : 0;
    float sum[V] = {};
    const int64_t end = min(count, (wave + 1) * each);
    for (int64_t i0 = wave * each; i0 < end; i0 += 8) {
        Piece<float, V == 1 ? 1 : 4, WIDE> p[8][V == 1 ? 1 : V / 4];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t at = min(i0 + i, end - 1);
            const float* from = a.parts + ((chunk + at) * 2 + (at == 0)) * a.width + col;
#pragma unroll
            for (int j = 0; j < (V == 1 ? 1 : V / 4); ++j)
                p[i][j] = *reinterpret_cast<const Piece<float, V == 1 ? 1 : 4, WIDE>*>(from + j * 4);
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
    write_row<D, V, WIDE>(a, table, key, col, skip, sum);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
// Places of a wave: 16 to 64, as many as leave 4,096 waves.  The sizes alone decide, not
// the alignment: the order of the sums goes by it.
int chunk_of(int64_t n, int64_t hidden) {
    int chunk = 16;
    while (chunk < kMostChunk && n / (2 * chunk) * ((hidden + 511) / 512) >= 4096) chunk *= 2;
    return chunk;
}

// What stands where in the workspace.
struct GradPlan {
    int64_t keys, source, keys2, source2, counts, present, parts, bytes;
    bool one;
};
GradPlan grad_plan(int64_t n, int64_t rows, int64_t hidden) {
    GradPlan p{};
    auto take = [&](int64_t bytes) {
        const int64_t at = p.bytes;
        p.bytes += (bytes + 255) / 256 * 256;
        return at;
    };
    p.one = n <= kOneSort;
    p.keys = take(4 * n);
    p.source = take(4 * n);
    p.present = take(rows + 4);
    if (!p.one) {
        p.keys2 = take(4 * n);
        p.source2 = take(4 * n);
        p.counts = take(kSortCountBytes);
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

template <typename S, typename D, int V, bool WIDE>
hipError_t launch_grad(const GradCall& g) {
    const GradPlan p = grad_plan(g.n, g.rows, g.hidden);
    SumArgs a{};
    a.keys = reinterpret_cast<uint32_t*>(g.ws + p.keys);
    a.source = reinterpret_cast<int32_t*>(g.ws + p.source);
    a.parts = reinterpret_cast<float*>(g.ws + p.parts);
    a.n = g.n;
    a.pieces = (g.hidden + V - 1) / V;
    a.width = g.hidden;
    a.dout_stride = g.dout_stride;
    a.table_stride = g.table_stride;
    a.rows = (uint32_t)g.rows;
    a.slabs = (uint32_t)((a.pieces + 63) / 64);
    a.chunk = chunk_of(g.n, g.hidden);
    a.chunks = (g.n + a.chunk - 1) / a.chunk;
    a.scale = g.scale;
    a.accumulate = g.accumulate;
    uint32_t* keys = reinterpret_cast<uint32_t*>(g.ws + p.keys);
    int32_t* source = reinterpret_cast<int32_t*>(g.ws + p.source);
    uint8_t* present = reinterpret_cast<uint8_t*>(g.ws + p.present);
    // The sort's launches leave most of the device idle for some microseconds, in which
    // kBeside bytes of zeros are written, or kBesideOne where one workgroup sorts for 20 us;
    // the rest comes beside the sums, without the rows that have one.  A workgroup writes
    // rows of 32 KiB, or beside the sums, where it has a quarter of the threads, 16 (4,095
    // tokens into 131,072 fp32 rows of 1,000: 106 us with 32 there and 96 MiB beside the
    // sort, 100 with 16, 114 with 8; 97 with 16 and 144 MiB, 94 with four marks ahead and
    // not eight).
    constexpr int64_t kBeside = 24 << 20, kBesideOne = 144 << 20;
    Zeros<D, V, WIDE> z = Zeros<D, V, WIDE>::of(g.table, g.table_stride, g.hidden);
    z.row1 = g.accumulate ? g.rows : 0;
    // the grid of a launch with `blocks` workgroups of its own that takes `bytes` of the zeros
    const auto with_zeros = [&](int64_t blocks, int64_t bytes, int64_t of_block) {
        z.each = (uint32_t)std::max<int64_t>(1, of_block / (int64_t)sizeof(D) / g.hidden);
        z.first = (int)blocks;
        z.row0 = z.row1;
        z.row1 = std::min(g.rows, z.row0 + bytes / (g.hidden * (int64_t)sizeof(D)) / z.each * z.each);
        return wide_grid((uint64_t)(blocks + z.blocks()));
    };
    constexpr int64_t kAll = (int64_t)1 << 62, kOfSort = 32768, kOfSum = 16384;
    if (g.n == 0) {
        const dim3 grid = with_zeros(0, kAll, kOfSum);
        embedding_sum_kernel<S, D, V, WIDE><<<grid, dim3(256), 0, g.s>>>(a, static_cast<const S*>(g.dout),
                                                                  static_cast<D*>(g.table), z);
        return hipGetLastError();
    }
    if (p.one) {
        const dim3 grid = with_zeros(1, kBesideOne, kOfSort);
        sort_one_kernel<D, V, WIDE><<<grid, dim3(kSortThreads), 0, g.s>>>(g.ids, (int)g.n, a.rows, key_bits_of(g.rows), keys, source,
                                                                   present, z);
    } else {
        SortPass q = sort_of(g.ids, g.n, a.rows, reinterpret_cast<int32_t*>(g.ws + p.counts), present);
        const SortLists lists{keys, source, reinterpret_cast<uint32_t*>(g.ws + p.keys2),
                              reinterpret_cast<int32_t*>(g.ws + p.source2)};
        dim3 grid = with_zeros(q.runs, kBeside, kOfSort);
        sort_count_kernel<D, V, WIDE><<<grid, dim3(kSortThreads), 0, g.s>>>(q, z);
        for (int pass = 0; pass < q.passes; ++pass) {
            set_pass(q, pass, lists);
            grid = with_zeros(q.runs, kBeside, kOfSort);
            sort_place_kernel<D, V, WIDE><<<grid, dim3(kSortThreads), 0, g.s>>>(q, z);
        }
    }
    const dim3 grid = with_zeros((a.chunks * a.slabs + 3) / 4, kAll, kOfSum);
    z.present = present;
    embedding_sum_kernel<S, D, V, WIDE><<<grid, dim3(256), 0, g.s>>>(a, static_cast<const S*>(g.dout),
                                                              static_cast<D*>(g.table), z);
    if (a.chunks > 1)
        embedding_join_kernel<D, V, WIDE><<<wide_grid((uint64_t)(a.chunks - 1) * a.slabs), dim3(256), 0, g.s>>>(
            a, static_cast<D*>(g.table));
    return hipGetLastError();
}

template <typename S, typename D>
hipError_t grad_of(const GradCall& g) {
    constexpr int V = 16 / sizeof(S);
    // a piece is 16 bytes of dout, and of the table 16 or, in fp32 for a 16-bit dout, 32
    const bool wide = g.hidden % V == 0 && g.dout_stride % V == 0 && g.table_stride % V == 0 &&
                      (uintptr_t)g.dout % 16 == 0 && (uintptr_t)g.table % (V * sizeof(D)) == 0;
    if (wide) return launch_grad<S, D, V, true>(g);
    return g.hidden >= V ? launch_grad<S, D, V, false>(g) : launch_grad<S, D, 1, true>(g);
}

struct LookupCall {
    Ids ids;
    int64_t n, rows, hidden, table_stride, out_stride;
    const void* table;
    void* out;
    float scale;
    hipStream_t s;
};

template <typename T, int V, bool WIDE>
hipError_t launch_lookup(const LookupCall& g) {
    const int64_t pieces = (g.hidden + V - 1) / V;
    // four pieces a lane, or one where that leaves the device waves to spare
    const bool few = g.n * ((pieces + 255) / 256) < 4096;
    const uint32_t parts = (uint32_t)(few ? (pieces + 63) / 64 : (pieces + 255) / 256);
    const dim3 grid = wide_grid((uint64_t)(g.n * parts + 3) / 4);
    if (few)
        embedding_kernel<T, V, WIDE, 1><<<grid, dim3(256), 0, g.s>>>(g.ids, g.n, (uint32_t)g.rows, g.hidden, pieces, parts,
                                                              static_cast<const T*>(g.table), g.table_stride,
                                                              static_cast<T*>(g.out), g.out_stride, g.scale);
    else
        embedding_kernel<T, V, WIDE, 4><<<grid, dim3(256), 0, g.s>>>(g.ids, g.n, (uint32_t)g.rows, g.hidden, pieces, parts,
                                                              static_cast<const T*>(g.table), g.table_stride,
                                                              static_cast<T*>(g.out), g.out_stride, g.scale);
    return hipGetLastError();
}

template <typename T>
hipError_t lookup_of(const LookupCall& g) {
    constexpr int V = 16 / sizeof(T);
    const bool wide = g.hidden % V == 0 && g.table_stride % V == 0 && g.out_stride % V == 0 &&
                      (uintptr_t)g.table % 16 == 0 && (uintptr_t)g.out % 16 == 0;
    if (wide) return launch_lookup<T, V, true>(g);
    return g.hidden >= V ? launch_lookup<T, V, false>(g) : launch_lookup<T, 1, true>(g);
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
    // a grid has 2^22 by 2^16 workgroups, of four waves
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
    return (size_t)grad_plan(a->tokens, a->rows, a->hidden).bytes;
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
    if (ws == nullptr || (uintptr_t)ws % 256 != 0 || ws_bytes < (size_t)grad_plan(a->tokens, a->rows, a->hidden).bytes)
        return C3_E_WORKSPACE;
    // the sums' workgroups are counted in 31 bits; the zeros' are no more than rows
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
