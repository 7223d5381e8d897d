// Products of two 16-bit matrices on the matrix units, as tiles that kernels put an
// epilogue of their own behind: acc[n][m] = sum over k of a(m, k) b(n, k).
//
// A workgroup holds TM x TN sums in registers, each wave MB x NB blocks of 32 x 32.
// Tiles of kInner inner indices come into LDS straight from memory, two of each operand
// in turn: while one pair is multiplied the next is on its way.  An operand lies in
// memory along the inner index (rows of k) or across it (rows of m or n); the latter is
// turned by the reads from LDS, so that no operand is copied in another order first.
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

// 16 bytes a lane from memory to LDS; zeros from `bytes` on.
__device__ __forceinline__ void load_lds(const char* base, uint32_t bytes, uint32_t offset, char* lds) {
    const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, (int)bytes, 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds), 16, (int)offset, 0, 0,
                                             0);
}
constexpr uint32_t kNowhere = 0xFFFFFF00u;

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
//   ALONG: R rows of 128 bytes; the 16-byte pieces of a row change places with bits 1 to
//   3 of the row, so that 16 rows' reads of one piece spread over all banks.
//   Across: for each 128 outer indices kInner rows of 256 bytes; the pieces of a row
//   change places with its low four bits, so that a turned read's four rows, 64 bytes of
//   each, do too.
template <int R, bool ALONG, int WAVES>
struct Tile {
    static constexpr int kLoads = R / 8 / WAVES;        // of a wave, 1 KiB each
    static constexpr int kBytes = R * kInner * 2;
    static_assert(kLoads * WAVES * 8 == R && (ALONG || R % 128 == 0), "rows of a tile");
    uint32_t at[kLoads];        // byte offset of a lane's piece
    int piece[2];               // ALONG: which piece, in even and odd loads
    int read, read2;            // byte offsets of a lane's reads

    static __device__ __forceinline__ int swap_along(int row) {
        return (((row >> 1) & 1) << 2) | (((row >> 2) & 1) << 1) | ((row >> 3) & 1);
    }
    static __device__ __forceinline__ int swap_across(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }

    // wave: which of the WAVES that load the tile
    __device__ __forceinline__ Tile(const Operand& x, int wave) {
        const int lane = threadIdx.x & 63;
        const int h = lane >> 5, c = lane & 31, i = lane & 15, g = (lane >> 4) & 1;
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const int load = wave * kLoads + n;
            if constexpr (ALONG) {
                const int row = load * 8 + lane / 8, q = (lane & 7) ^ swap_along(row);
                at[n] = row < x.outer ? (uint32_t)(row * x.stride) + q * 16 : kNowhere;
            } else {
                const int row = load % 16 * 4 + lane / 16, col = load / 16 * 128 + ((lane & 15) ^ swap_across(row)) * 8;
                at[n] = col < x.outer ? (uint32_t)(row * x.stride) + col * 2 : kNowhere;
            }
        }
        if constexpr (ALONG) {
            piece[0] = (lane & 7) ^ swap_along(wave * kLoads * 8 + lane / 8);
            piece[1] = (lane & 7) ^ swap_along((wave * kLoads + 1) * 8 + lane / 8);
            read = c * 128 + ((h ^ swap_along(c)) << 4);
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
            const char* base = x.p + (int64_t)k * 2;
            const uint32_t bytes = left > 0 ? (uint32_t)((int64_t)(min(x.outer, R) - 1) * x.stride) + (left + 7) / 8 * 16 : 0;
#pragma unroll
            for (int n = 0; n < kLoads; ++n)
                load_lds(base, bytes, piece[n & 1] * 8 < left ? at[n] : kNowhere, lds + (wave * kLoads + n) * 1024);
        } else {
            const char* base = x.p + (int64_t)k * x.stride;
            const uint32_t bytes = left > 0 ? (uint32_t)((int64_t)(left - 1) * x.stride) + min(x.outer, R) * 2 : 0;
#pragma unroll
            for (int n = 0; n < kLoads; ++n) load_lds(base, bytes, at[n], lds + (wave * kLoads + n) * 1024);
        }
    }

    // Outer indices 32 b .. of the tile at inner indices 16 ks ..: an operand of the
    // matrix unit, lane's outer index lane & 31, inner ones (lane >> 5) * 8 ...
    __device__ __forceinline__ u32x4 operand(const char* lds, int b, int ks) const {
        if constexpr (ALONG) {
            return *reinterpret_cast<const u32x4*>(lds + b * 4096 + (read ^ (ks << 5)));
        } else {
            const char* p = lds + (b >> 2) * (kInner * 256) + ks * 4096;
            const u32x2 lo = read_turned(p + (read ^ ((b & 3) << 6))), hi = read_turned(p + (read2 ^ ((b & 3) << 6)));
            return u32x4{lo.x, lo.y, hi.x, hi.y};
        }
    }
};

// The wave's loads to LDS have landed, and every wave of the workgroup is here.
__device__ __forceinline__ void loads_ready() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

template <typename T, int WM, int WN, int MB, int NB, bool A_ALONG, bool B_ALONG>
struct Product {
    static constexpr int kWM = WM, kWaves = WM * WN, kThreads = kWaves * 64;
    static constexpr int TM = WM * MB * 32, TN = WN * NB * 32;
    using TileA = Tile<TM, A_ALONG, kWaves>;
    using TileB = Tile<TN, B_ALONG, kWaves>;

    // Block mb, nb of the wave, register i: m and n inside the tile.
    static __device__ __forceinline__ int m_of(int mb, int i) {
        const int wave = threadIdx.x >> 6, h = (threadIdx.x >> 5) & 1;
        return (wave % WM * MB + mb) * 32 + (i & 3) + 8 * (i >> 2) + 4 * h;
    }
    static __device__ __forceinline__ int n_of(int nb) {
        return ((threadIdx.x >> 6) / WM * NB + nb) * 32 + (threadIdx.x & 31);
    }

    static __device__ __forceinline__ void step(f32x16 (&acc)[MB][NB], const TileA& ta, const TileB& tb, const char* a,
                                                const char* b) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int am = wave % WM * MB, bn = wave / WM * NB;
        // the operands of the next 16 inner indices are read while these are multiplied
        u32x4 fa[2][MB], fb[2][NB];
        auto read = [&](int ks) {
#pragma unroll
            for (int i = 0; i < MB; ++i) fa[ks & 1][i] = ta.operand(a, am + i, ks);
#pragma unroll
            for (int j = 0; j < NB; ++j) fb[ks & 1][j] = tb.operand(b, bn + j, ks);
        };
        read(0);
#pragma unroll
        for (int ks = 0; ks < kInner / 16; ++ks) {
            __builtin_amdgcn_sched_barrier(0);      // no operands further ahead: registers are short
            if (ks + 1 < kInner / 16) read(ks + 1);
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = mfma_32x32x16<T>(fa[ks & 1][i], fb[ks & 1][j], acc[i][j]);
        }
        __builtin_amdgcn_sched_barrier(0);
    }

    // Adds the product over the operands' inner indices (both have the same).  The four
    // buffers are objects of their own, or the compiler would wait for loads to one
    // before it reads another.  LDS is free to use behind the next barrier.
    static __device__ __forceinline__ void run(f32x16 (&acc)[MB][NB], const Operand& a, const Operand& b, char* a0,
                                               char* b0, char* a1, char* b1) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const TileA ta(a, wave);
        const TileB tb(b, wave);
        const int inner = a.inner;
        if (inner <= 0) return;
        ta.load(a, 0, a0, wave);
        tb.load(b, 0, b0, wave);
        // two tiles a turn; a last one of zeros where their number is odd
        for (int k = 0; k < inner; k += 2 * kInner) {
            loads_ready();
            ta.load(a, k + kInner, a1, wave);
            tb.load(b, k + kInner, b1, wave);
            step(acc, ta, tb, a0, b0);
            loads_ready();
            if (k + 2 * kInner < inner) {
                ta.load(a, k + 2 * kInner, a0, wave);
                tb.load(b, k + 2 * kInner, b0, wave);
            }
            step(acc, ta, tb, a1, b1);
        }
    }
};

// Writes a wave's sums as rows n of 16-bit elements m: each lane has four neighbours in m
// of one row, so the wave turns its part in LDS, which it has to itself, and stores whole
// rows of MB * 64 bytes.  value(j, i, r): element of block i, j, register r as T; row(n):
// where m = 0 of the tile's row n is, or null; elements from m_left on (a multiple of 8)
// are not there.  The buffers are those of Product::run, behind a barrier.
template <typename P, typename T, int MB, int NB, typename Value, typename Row>
__device__ __forceinline__ void store_rows(char* a0, char* b0, char* a1, char* b1, int m_left, Value value, Row row) {
    constexpr int kPieces = MB * 4, kPart = NB * 32 * kPieces * 16, kShare = P::kWaves / 4;
    static_assert(kShare * kPart <= P::TileA::kBytes && kShare * kPart <= P::TileB::kBytes, "room for the turn");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int which = wave / kShare;
    char* lds = (which == 0 ? a0 : which == 1 ? b0 : which == 2 ? a1 : b1) + wave % kShare * kPart;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int n = j * 32 + (lane & 31);
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                AlignedPack<T, 4> v;
#pragma unroll
                for (int r = 0; r < 4; ++r) v.v[r] = value(j, i, 4 * q + r);
                *reinterpret_cast<AlignedPack<T, 4>*>(lds + (n * kPieces + ((i * 4 + q) ^ (n & (kPieces - 1)))) * 16 + h * 8) = v;
            }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    const int m0 = wave % P::kWM * MB * 32, n0 = wave / P::kWM * NB * 32;
#pragma unroll
    for (int t = 0; t < NB * 32 * kPieces / 64; ++t) {
        const int at = t * 64 + lane, n = at / kPieces, piece = at % kPieces;
        const u32x4 v = *reinterpret_cast<const u32x4*>(lds + (n * kPieces + (piece ^ (n & (kPieces - 1)))) * 16);
        T* to = row(n0 + n);
        if (to != nullptr && m0 + piece * 8 < m_left) *reinterpret_cast<u32x4*>(to + m0 + piece * 8) = v;
    }
}

// Which tile a workgroup takes: the eight dies take workgroups in turn, and each gets a
// run of the tiles of its own, in which kGroup tiles of the first index run fastest, so
// that the tiles that a die works on at one time share their operands.
constexpr int kTileGroup = 4;
__device__ __forceinline__ bool tile_of(uint32_t first, uint32_t second, uint32_t& i, uint32_t& j) {
    const uint32_t total = first * second, each = (total + 7) / 8;
    const uint32_t t = blockIdx.x % 8 * each + blockIdx.x / 8;
    if (blockIdx.x / 8 >= each || t >= total) return false;
    const uint32_t group = t / (kTileGroup * second), in = t - group * kTileGroup * second;
    const uint32_t high = min((uint32_t)kTileGroup, first - group * kTileGroup);
    i = group * kTileGroup + in % high;
    j = in / high;
    return true;
}
inline unsigned tile_blocks(int64_t first, int64_t second) { return (unsigned)((first * second + 7) / 8 * 8); }

}  // namespace c3
