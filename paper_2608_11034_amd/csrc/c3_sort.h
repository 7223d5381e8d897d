// A stable counting sort of tokens by the row that each names, in launches of up to
// kMostRuns workgroups: the embedding's gradient sums its runs, that of the loss over a
// vocabulary lays tokens out by their targets.
#pragma once

#include <algorithm>

#include "c3_internal.h"
#include "c3_replay_types.h"

namespace c3 {

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kMostBits = 10;               // of a digit
constexpr int kMostPasses = 4;              // keys have 32 bits at most
constexpr int kMostRuns = 64;
constexpr int kNextCounts = 16384;          // runs times digits at most: they are counted in LDS

struct Ids {
    const void* p;
    int wide;                               // 8-byte numbers
    // The row that a token names; `rows`, behind all of them, for none.
    __device__ __forceinline__ uint32_t key(int64_t t, uint32_t rows) const {
        if (wide) {
            const int64_t i = static_cast<const int64_t*>(p)[t];
            return (uint64_t)i < rows ? (uint32_t)i : rows;
        }
        const int32_t i = static_cast<const int32_t*>(p)[t];
        return (uint32_t)i < rows ? (uint32_t)i : rows;
    }
};

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
// first place of the digit, of which a thread has one.  total, before: keys with the
// digit in all workgroups, and in those before this one.
template <typename Counted>
__device__ __forceinline__ void first_places(int32_t* lds, int32_t* wave_sum, int digits, Counted counted) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t total = 0, before = 0;
    if (tid < digits) counted(tid, total, before);
    int32_t sum = total;
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t up = __shfl_up(sum, d);
        if (lane >= d) sum += up;
    }
    if (lane == 63) wave_sum[wave] = sum;
    __syncthreads();
    int32_t at = sum - total + before;
    for (int w = 0; w < wave; ++w) at += wave_sum[w];
    if (tid < digits) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const int32_t c = lds[w * digits + tid];
            lds[w * digits + tid] = at;
            at += c;
        }
    }
    __syncthreads();
}

// A launch counts the lowest digits of every run of tokens, and one for each
// digit places them.  A placed key counts its next digit for the run that it comes to;
// these are integers, so their order does not matter.  A workgroup counts in LDS first:
// one by one a frequent digit's counts would wait for each other in memory (10 us of 18
// with 16,384 tokens of which half have one high digit).
struct SortPass {
    Ids ids;                // of the first pass, whose keys and tokens are not written down
    const uint32_t* in_keys;
    const int32_t* in_source;
    uint32_t* keys;
    int32_t* source;
    int32_t* counts;        // [passes][runs][1 << kMostBits]
    uint8_t* present;       // or null: 1 for each row that a token names, 4 bytes behind the
                            // last; stores of one value, where bits would be atomics on few words
    int64_t n;
    uint32_t rows;
    int run_shift;          // log2 of a run's length
    int runs, pass, passes, key_bits;
    __device__ __forceinline__ uint32_t key(int64_t i) const { return pass == 0 ? ids.key(i, rows) : in_keys[i]; }
    __device__ __forceinline__ int lo(int p) const { return key_bits * p / passes; }
    __device__ __forceinline__ int bits(int p) const { return lo(p + 1) - lo(p); }
    __device__ __forceinline__ int32_t* count(int p, int64_t r) const {
        return counts + (((int64_t)p * runs + r) << kMostBits);
    }
};

// Workgroups 0 .. runs - 1 of the launch that counts.
__device__ __forceinline__ void sort_count(const SortPass& p) {
    __shared__ int32_t lds[1 << kMostBits];
    const int digits = 1 << p.bits(0);
    lds[threadIdx.x] = 0;
    for (int q = 1; q < p.passes; ++q) p.count(q, blockIdx.x)[threadIdx.x] = 0;
    if (p.present != nullptr)
        for (int64_t i = (int64_t)blockIdx.x * kSortThreads + threadIdx.x; i <= p.rows / 4; i += (int64_t)p.runs * kSortThreads)
            reinterpret_cast<uint32_t*>(p.present)[i] = 0;
    __syncthreads();
    const int64_t begin = (int64_t)blockIdx.x << p.run_shift, end = min(begin + (1ll << p.run_shift), p.n);
    for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads) atomicAdd(&lds[p.key(i) & (digits - 1)], 1);
    __syncthreads();
    p.count(0, blockIdx.x)[threadIdx.x] = lds[threadIdx.x];
}

// And of the launch for one digit.
__device__ __forceinline__ void sort_place(const SortPass& p) {
    __shared__ int32_t lds[(kSortWaves << kMostBits) + kSortWaves];
    __shared__ int32_t next[kNextCounts];
    const int lo = p.lo(p.pass), bits = p.bits(p.pass), digits = 1 << bits;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t* wave_sum = lds + kSortWaves * digits;
    const int64_t begin = (int64_t)blockIdx.x << p.run_shift, end = min(begin + (1ll << p.run_shift), p.n);
    const int64_t part = (1ll << p.run_shift) / kSortWaves, wb = begin + wave * part, we = min(wb + part, end);
    const bool last = p.pass == p.passes - 1;
    const int next_lo = p.lo(p.pass + 1), next_bits = last ? 0 : p.bits(p.pass + 1);
    for (int i = threadIdx.x; i < kSortWaves * digits; i += kSortThreads) lds[i] = 0;
    if (!last)
        for (int i = threadIdx.x; i < p.runs << next_bits; i += kSortThreads) next[i] = 0;
    __syncthreads();
    int32_t* mine = lds + wave * digits;
    for (int64_t i = wb + lane; i < we; i += 64) atomicAdd(&mine[(p.key(i) >> lo) & (digits - 1)], 1);
    __syncthreads();
    first_places(lds, wave_sum, digits, [&](int d, int32_t& total, int32_t& before) {
        for (int b = 0; b < p.runs; b += 16) {          // sixteen loads in flight
            int32_t c[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) c[j] = p.count(p.pass, min(b + j, p.runs - 1))[d];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                before += b + j < (int)blockIdx.x ? c[j] : 0;
                total += b + j < p.runs ? c[j] : 0;
            }
        }
    });
    for (int64_t i0 = wb; i0 < we; i0 += 64) {
        const int64_t i = i0 + lane;
        const uint32_t k = i < we ? p.key(i) : 0;
        // a mark for each lane would crowd a frequent row's; every lane takes part in the shuffle
        const uint32_t lower = __shfl_up(k, 1);
        const bool repeats = lane > 0 && lower == k;
        const int32_t at = place_of((k >> lo) & (digits - 1), i < we, bits, mine);
        if (at < 0) continue;
        p.keys[at] = k;
        p.source[at] = p.pass == 0 ? (int32_t)i : p.in_source[i];
        if (last && p.present != nullptr && k < p.rows && !repeats) p.present[k] = 1;
        if (!last) atomicAdd(&next[((at >> p.run_shift) << next_bits) + ((k >> next_lo) & ((1 << next_bits) - 1))], 1);
    }
    if (last) return;
    __syncthreads();
    for (int i = threadIdx.x; i < p.runs << next_bits; i += kSortThreads)
        if (next[i] != 0) atomicAdd(&p.count(p.pass + 1, i >> next_bits)[i & ((1 << next_bits) - 1)], next[i]);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
inline int key_bits_of(int64_t rows) {      // keys are 0 .. rows
    int bits = 1;
    while ((rows >> bits) != 0) ++bits;
    return bits;
}

// The last pass writes to the first pair of lists.
struct SortLists {
    uint32_t* keys;
    int32_t* source;
    uint32_t* keys2;
    int32_t* source2;
};
constexpr int64_t kSortCountBytes = 4 * (int64_t)kMostPasses * kMostRuns << kMostBits;

inline SortPass sort_of(const Ids& ids, int64_t n, uint32_t rows, int32_t* counts, uint8_t* present) {
    SortPass q{};
    q.ids = ids;
    q.counts = counts;
    q.present = present;
    q.n = n;
    q.rows = rows;
    q.key_bits = key_bits_of(rows);
    q.passes = (q.key_bits + kMostBits - 1) / kMostBits;
    q.run_shift = 10;
    const int most_runs = std::min(kMostRuns, kNextCounts >> ((q.key_bits + q.passes - 1) / q.passes));
    while (((n - 1) >> q.run_shift) >= most_runs) ++q.run_shift;
    q.runs = (int)((n - 1) >> q.run_shift) + 1;
    return q;
}
inline void set_pass(SortPass& q, int pass, const SortLists& l) {
    const bool to_first = (q.passes - 1 - pass) % 2 == 0;
    q.pass = pass;
    q.in_keys = to_first ? l.keys2 : l.keys;
    q.in_source = to_first ? l.source2 : l.source;
    q.keys = to_first ? l.keys : l.keys2;
    q.source = to_first ? l.source : l.source2;
}

}  // namespace c3
