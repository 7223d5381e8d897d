// Products of two 16-bit matrices on the matrix units, as tiles that kernels put an
// epilogue of their own behind: acc[n][m] = sum over k of a(m, k) b(n, k).
//
// A workgroup holds TM x TN sums in registers, each wave MB x NB blocks of 32 x 32.
// Tiles of kInner inner indices come into LDS straight from memory, two of each operand in
// turn: one is on its way while the other is multiplied.  An operand lies in memory along
// the inner index (rows of k) or across it (rows of m or n); the latter is turned by the
// reads from LDS, so that no operand is copied in another order first.
//
// What bounds it is the matrix units at the clock that the card's power leaves them: 8,192
// x 4,096 by 131,072 x 4,096 in bf16 with the epilogue of the forward loss take 6.8 ms,
// 1,290 TFLOP/s at 1.77 GHz with the units busy 70% of the cycles and LDS 26%, without bank
// conflicts; a large library product reaches 1,310 there.  Eight waves of 128 x 64 sums:
// four of 128 x 128 read a third less of LDS, but nothing is left to run while one of them
// waits (7.14 ms against 6.75); tiles of 32 inner indices, four in turn, read half lines
// (7.55 on those four).
#pragma once

#include "c3_replay_types.h"

namespace c3 {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kInner = 64;

template <typename T>
__device__ __forceinline__ f32x16 mfma_32x32x16(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (std::is_same_v<T, __bf16>)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b),
                                                       c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b),
                                                      c, 0, 0, 0);
}

__device__ __forceinline__ u32x2 read_turned(const char* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(p)));
}

// 16 bytes a lane from memory to LDS; zeros from `bytes` on.  ONCE: the bytes are not read
// again, and need no place in the caches.
template <bool ONCE>
__device__ __forceinline__ void load_lds(const char* base, uint32_t bytes, uint32_t offset, char* lds) {
    constexpr int kNonTemporal = 2;
    const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, (int)bytes, 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds), 16, (int)offset, 0, 0,
                                             ONCE ? kNonTemporal : 0);
}
constexpr uint32_t kNowhere = 0xFFFFFF00u;

// The same for every lane, where the compiler cannot tell: it would go through the lanes
// one by one for a load's base.
__device__ __forceinline__ const char* scalar(const char* p) {
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const char*>((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) << 32 |
                                         (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a));
}
__device__ __forceinline__ uint32_t scalar(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// One operand in memory: outer index m or n in rows (ALONG) or columns, `stride` bytes
// between rows, `outer` indices and `inner` inner ones from `p` on.  Rows hold whole
// pieces of 8 elements: where `inner` (ALONG) is no multiple of 8, what is behind it in
// its last piece is read, and the other operand's zeros there, or its own, take it out.
// 256 rows span less than 2^31 bytes.
struct Operand {
    const char* p;
    int64_t stride;
    int outer, inner;
};

// A tile of R outer by kInner inner indices in LDS.
//   ALONG: R rows of 2 kInner bytes; the 16-byte pieces of a row change places with bits
//   of the row, so that 16 rows' reads of one piece spread over all banks.
//   Across: for each 128 outer indices kInner rows of 256 bytes; the pieces of a row
//   change places with its low four bits, so that a turned read's four rows, 64 bytes of
//   each, do too.
template <int R, bool ALONG, int WAVES, bool ONCE = false>
struct Tile {
    static constexpr int kLoads = R * kInner / 512 / WAVES;     // of a wave, 1 KiB each
    static constexpr int kBytes = R * kInner * 2;
    static constexpr int kPieces = kInner / 8;                  // of a row, ALONG
    static constexpr int kTurns = kInner / 32;
    static_assert(kLoads * WAVES * 512 == R * kInner && (ALONG || R % 128 == 0), "rows of a tile");
    uint32_t at[kLoads];        // byte offset of a lane's piece
    int piece[ALONG ? kTurns : 1];      // ALONG: which piece, in every kTurns-th load
    int read, read2;            // byte offsets of a lane's reads

    static __device__ __forceinline__ int swap_along(int row) {
        return (((row >> 1) & 1) << 2) | (((row >> 2) & 1) << 1) | ((row >> 3) & 1);
    }
    static __device__ __forceinline__ int swap_across(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }

    // ALONG: the row that a lane loads a piece of.
    static __device__ __forceinline__ int row_of(int load) {
        return load * (64 / kPieces) + (threadIdx.x & 63) / kPieces;
    }
    // wave: which of the WAVES that load the tile
    __device__ __forceinline__ Tile(const Operand& x, int wave) {
        const int lane = threadIdx.x & 63;
        const int h = lane >> 5, c = lane & 31, i = lane & 15, g = (lane >> 4) & 1;
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const int load = wave * kLoads + n;
            if constexpr (ALONG) {
                const int row = row_of(load), q = (lane & (kPieces - 1)) ^ swap_along(row);
                at[n] = row < x.outer ? (uint32_t)(row * x.stride) + q * 16 : kNowhere;
            } else {
                const int row = load % (kInner / 4) * 4 + lane / 16;
                const int col = load / (kInner / 4) * 128 + ((lane & 15) ^ swap_across(row)) * 8;
                at[n] = col < x.outer ? (uint32_t)(row * x.stride) + col * 2 : kNowhere;
            }
        }
        if constexpr (ALONG) {
#pragma unroll
            for (int n = 0; n < kTurns; ++n) piece[n] = (lane & (kPieces - 1)) ^ swap_along(row_of(wave * kLoads + n));
            read = c * kInner * 2 + ((h ^ swap_along(c)) << 4);
            read2 = 0;
        } else {
            const int row = h * 8 + (i >> 2), q = g * 2 + ((i & 3) >> 1);
            read = row * 256 + ((q ^ swap_across(row)) << 4) + (i & 1) * 8;
            read2 = (row + 4) * 256 + ((q ^ swap_across(row + 4)) << 4) + (i & 1) * 8;
        }
    }

    // Loads the tile that begins at inner index k; zeros behind the last one.
    __device__ __forceinline__ void load(const Operand& x, int k, char* lds, int wave) const {
        const int left = max(min(x.inner - k, kInner), 0);
        if constexpr (ALONG) {
            const char* base = scalar(x.p + (int64_t)k * 2);
            const uint32_t bytes = scalar(left > 0 ? (uint32_t)((int64_t)(min(x.outer, R) - 1) * x.stride) + (left + 7) / 8 * 16 : 0);
#pragma unroll
            for (int n = 0; n < kLoads; ++n)
                load_lds<ONCE>(base, bytes, piece[n & (kTurns - 1)] * 8 < left ? at[n] : kNowhere, lds + (wave * kLoads + n) * 1024);
        } else {
            const char* base = scalar(x.p + (int64_t)k * x.stride);
            const uint32_t bytes = scalar(left > 0 ? (uint32_t)((int64_t)(left - 1) * x.stride) + min(x.outer, R) * 2 : 0);
#pragma unroll
            for (int n = 0; n < kLoads; ++n) load_lds<ONCE>(base, bytes, at[n], lds + (wave * kLoads + n) * 1024);
        }
    }

    // Outer indices 32 b .. of the tile at inner indices 16 ks ..: an operand of the
    // matrix unit, lane's outer index lane & 31, inner ones (lane >> 5) * 8 ...
    __device__ __forceinline__ u32x4 operand(const char* lds, int b, int ks) const {
        if constexpr (ALONG) {
            return *reinterpret_cast<const u32x4*>(lds + b * 64 * kInner + (read ^ (ks << 5)));
        } else {
            const char* p = lds + (b >> 2) * (kInner * 256) + ks * 4096;
            const u32x2 lo = read_turned(p + (read ^ ((b & 3) << 6))), hi = read_turned(p + (read2 ^ ((b & 3) << 6)));
            return u32x4{lo.x, lo.y, hi.x, hi.y};
        }
    }
};

// An object in LDS for each number: the compiler would wait for loads to one before it
// reads another if they were parts of one object.
template <int ID, int BYTES>
__device__ __forceinline__ char* lds_object() {
    __shared__ __attribute__((aligned(1024))) char bytes[BYTES];
    return bytes;
}

template <typename T, int WM, int WN, int MB, int NB, bool A_ALONG, bool B_ALONG>
struct Product {
    static constexpr int kWM = WM, kWaves = WM * WN, kThreads = kWaves * 64;
    static constexpr int TM = WM * MB * 32, TN = WN * NB * 32;
    using TileA = Tile<TM, A_ALONG, kWaves>;
    using TileB = Tile<TN, B_ALONG, kWaves>;
    static constexpr int kLoads = TileA::kLoads + TileB::kLoads;       // of a wave and stage

    // Block mb, nb of the wave, register i: m and n inside the tile.
    static __device__ __forceinline__ int m_of(int mb, int i) {
        const int wave = threadIdx.x >> 6, h = (threadIdx.x >> 5) & 1;
        return (wave % WM * MB + mb) * 32 + (i & 3) + 8 * (i >> 2) + 4 * h;
    }
    static __device__ __forceinline__ int n_of(int nb) {
        return ((threadIdx.x >> 6) / WM * NB + nb) * 32 + (threadIdx.x & 31);
    }

    template <int S>
    static __device__ __forceinline__ char* lds_a() { return lds_object<2 * S, TileA::kBytes>(); }
    template <int S>
    static __device__ __forceinline__ char* lds_b() { return lds_object<2 * S + 1, TileB::kBytes>(); }
    // kWaveBytes of LDS for each wave, behind run().
    static constexpr int kWaveBytes = (TileA::kBytes < TileB::kBytes ? TileA::kBytes : TileB::kBytes) * 4 / kWaves;
    static __device__ __forceinline__ char* lds_of_wave(int wave) {
        constexpr int kShare = kWaves / 4;
        const int which = wave / kShare;
        char* p = which == 0 ? lds_a<0>() : which == 1 ? lds_a<1>() : which == 2 ? lds_b<0>() : lds_b<1>();
        return p + wave % kShare * kWaveBytes;
    }

    struct Operands {
        u32x4 a[MB], b[NB];
    };

    // The loads to the next tile have landed, and every wave of the workgroup is here.
    template <int LEFT>
    static __device__ __forceinline__ void landed() {
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LEFT) : "memory");
    }

    static __device__ __forceinline__ void multiply(f32x16 (&acc)[MB][NB], const Operands& f) {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = mfma_32x32x16<T>(f.a[i], f.b[j], acc[i][j]);
    }

    // Adds the product over the operands' inner indices (both have the same).  LDS is free
    // to use behind it.  With MORE, that of a second pair of operands across the inner index
    // behind it in the same loop: a2 with a's outer indices and stride, b2 with any.  Which
    // pair a load takes is chosen without a branch, which would part the loads from what runs
    // beside them (dweight of 8,192 tokens, 32,768 rows of 4,096: 1,590 us without a second
    // pair, 1,660 with one of a tile as a rule, 1,860 with the branch).
    template <bool MORE = false>
    static __device__ __forceinline__ void run(f32x16 (&acc)[MB][NB], const Operand& a, const Operand& b,
                                               const Operand& a2 = {}, const Operand& b2 = {}) {
        static_assert(!MORE || (!A_ALONG && !B_ALONG), "operands across the inner index");
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int am = wave % WM * MB, bn = wave / WM * NB;
        const int first = MORE ? (max(a.inner, 0) + kInner - 1) / kInner * kInner : a.inner;
        const int inner = MORE ? first + max(a2.inner, 0) : first;
        const TileA ta(a, wave);
        const TileB tb(b, wave), tb2(MORE ? b2 : b, wave);
        if (inner <= 0) return;
        const auto load = [&](int k, char* la, char* lb) {
            if constexpr (MORE) {
                const bool more = k >= first;
                const Operand oa{more ? a2.p : a.p, a.stride, a.outer, more ? a2.inner : a.inner};
                const Operand ob{more ? b2.p : b.p, more ? b2.stride : b.stride, more ? b2.outer : b.outer, oa.inner};
                TileB t = tb;
#pragma unroll
                for (int n = 0; n < TileB::kLoads; ++n) t.at[n] = more ? tb2.at[n] : tb.at[n];
                ta.load(oa, more ? k - first : k, la, wave);
                t.load(ob, more ? k - first : k, lb, wave);
            } else {
                ta.load(a, k, la, wave);
                tb.load(b, k, lb, wave);
            }
        };
        Operands f[2];
        const auto read = [&](Operands& to, const char* la, const char* lb, int ks) {
#pragma unroll
            for (int i = 0; i < MB; ++i) to.a[i] = ta.operand(la, am + i, ks);
#pragma unroll
            for (int j = 0; j < NB; ++j) to.b[j] = tb.operand(lb, bn + j, ks);
        };
        // The operands of 16 inner indices are read while the 16 before are multiplied, and
        // a tile's first 16 while the last of the tile before are: the matrix units have
        // operands at hand on both sides of the barrier.  The barrier also says that every
        // wave has read the last of a tile, whose place is loaded next.
        const auto step = [&](int k, char* la, char* lb, const char* next_a, const char* next_b) {
#pragma unroll
            for (int ks = 0; ks < kInner / 16 - 1; ++ks) {
                read(f[(ks + 1) & 1], la, lb, ks + 1);
                multiply(acc, f[ks & 1]);
                __builtin_amdgcn_sched_barrier(0);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            landed<0>();
            load(k + 2 * kInner, la, lb);
            read(f[0], next_a, next_b, 0);
            multiply(acc, f[1]);
            __builtin_amdgcn_sched_barrier(0);
        };
        load(0, lds_a<0>(), lds_b<0>());
        load(kInner, lds_a<1>(), lds_b<1>());
        landed<kLoads>();
        read(f[0], lds_a<0>(), lds_b<0>(), 0);
        __builtin_amdgcn_sched_barrier(0);
        // both stages in a turn; zeros behind the last tile, or with MORE, where one more tile
        // is the rule, half a turn for the last
        int k = 0;
        for (; k < (MORE ? inner - kInner : inner); k += 2 * kInner) {
            step(k, lds_a<0>(), lds_b<0>(), lds_a<1>(), lds_b<1>());
            step(k + kInner, lds_a<1>(), lds_b<1>(), lds_a<0>(), lds_b<0>());
        }
        if (MORE && k < inner) step(k, lds_a<0>(), lds_b<0>(), lds_a<1>(), lds_b<1>());
        landed<0>();
    }
};

// Writes a wave's sums as rows n of 16-bit elements m: each lane has four neighbours in m
// of one row, so the wave turns its part in LDS, 32 rows at a time, and stores whole rows
// of MB * 64 bytes.  value(j, i, r): element of block i, j, register r as T; row(n): where
// m = 0 of the tile's row n is, or null; elements from m_left on (a multiple of 8) are not
// there.  The rows go past the caches, which hold the operands that other workgroups share
// (the loss of 8 tokens over 32,000 rows of 4,096, forward and back: 252 us, and 220 so).
// Behind Product::run.
template <typename P, typename T, int MB, int NB, typename Value, typename Row>
__device__ __forceinline__ void store_rows(int m_left, Value value, Row row) {
    constexpr int kPieces = MB * 4;
    static_assert(32 * kPieces * 16 <= P::kWaveBytes, "room for the turn");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    char* lds = P::lds_of_wave(wave);
    const int m0 = wave % P::kWM * MB * 32, n0 = wave / P::kWM * NB * 32;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int n = lane & 31;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                AlignedPack<T, 4> v;
#pragma unroll
                for (int r = 0; r < 4; ++r) v.v[r] = value(j, i, 4 * q + r);
                *reinterpret_cast<AlignedPack<T, 4>*>(lds + (n * kPieces + ((i * 4 + q) ^ (n & (kPieces - 1)))) * 16 + h * 8) = v;
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int t = 0; t < 32 * kPieces / 64; ++t) {
            const int q = t * 64 + lane, r = q / kPieces, piece = q % kPieces;
            const u32x4 v = *reinterpret_cast<const u32x4*>(lds + (r * kPieces + (piece ^ (r & (kPieces - 1)))) * 16);
            T* to = row(n0 + j * 32 + r);
            if (to == nullptr || m0 + piece * 8 >= m_left) continue;
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(to + m0 + piece * 8));
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// Which tile a workgroup takes: the eight dies take workgroups in turn, and each gets a
// run of the tiles of its own, in which `group` tiles of the first index run fastest, so
// that the tiles that a die works on at one time share their operands.
constexpr uint32_t kTileGroup = 4;
__device__ __forceinline__ bool tile_at(uint32_t first, uint32_t second, uint32_t group_size, uint32_t v, uint32_t& i,
                                        uint32_t& j) {      // the v-th of the workgroup's die
    const uint32_t total = first * second, each = (total + 7) / 8;
    const uint32_t t = blockIdx.x % 8 * each + v;
    if (v >= each || t >= total) return false;
    const uint32_t group = t / (group_size * second), in = t - group * group_size * second;
    const uint32_t high = min(group_size, first - group * group_size);
    i = group * group_size + in % high;
    j = in / high;
    return true;
}
__device__ __forceinline__ bool tile_of(uint32_t first, uint32_t second, uint32_t group_size, uint32_t& i, uint32_t& j) {
    return tile_at(first, second, group_size, blockIdx.x / 8, i, j);
}
inline unsigned tile_blocks(int64_t first, int64_t second) { return (unsigned)((first * second + 7) / 8 * 8); }

}  // namespace c3
