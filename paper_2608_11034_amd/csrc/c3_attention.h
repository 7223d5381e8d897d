// What the attention kernels share: the work list, LDS tiles, fragments and the
// masked product.
//
// Rows.  The query heads that share a key head are taken together: row r of a
// sequence and key head is query r / group and head r % group of the group, so
// a tile of rows reads a key tile once for all of them, and a token's row of a
// group of 8 fills a quarter of a matrix operand.
//
// Matrix operands.  v_mfma_f32_32x32x16 takes, from lane l = 32 h + c, eight
// elements k = 8 h .. 8 h + 7 of row c of A (of column c of B), and leaves in
// register i row 8 (i / 4) + 4 h + i % 4 of column c.  A product whose 32 rows
// are the next product's inner index therefore feeds it without any movement:
// registers 8 j .. 8 j + 7, rounded, are its B operand for inner indices
//     16 j + 4 h + {0 .. 3}  and  16 j + 8 + 4 h + {0 .. 3},
// and the A operand is read in that order.  So scores are computed with keys as
// rows where the next product sums over keys (forward, dq) and with queries as
// rows where it sums over queries (dk, dv), and probabilities never leave the
// registers.  A operands along a tile's rows are 16-byte LDS reads; those across
// them (values in the forward, for instance) are ds_read_b64_tr_b16 reads, which
// hand lane c elements of four rows of column c.
//
// LDS tiles hold rows of DP elements in 16-byte pieces, piece p of row r at
// p ^ swizzle(r), which spreads both kinds of reads over all banks.  They are
// filled by buffer loads straight to LDS; a piece outside the sequence or
// behind the head size reads as zeros by the buffer's bound.
#pragma once

#include <algorithm>
#include <initializer_list>

#include "c3_internal.h"
#include "c3_replay_types.h"

namespace c3 {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = kAttnThreads / 64;
constexpr uint32_t kDirect = 256;
constexpr int64_t kDirectKeys = 256;

struct AttnSeq {
    int32_t b;              // sequence
    int32_t q_start, q_len, k_start, k_len;
    int32_t unit0[2];       // its first unit of one key head, by rows and by keys
};

// Sequences that go along as a kernel's argument (4,096 bytes at most in all);
// longer lists are staged, which a capture cannot record.
constexpr int kAttnArgSeqs = C3_ATTENTION_CAPTURE_SEQUENCES;

struct AttnTable {
    int32_t n;              // 0: every sequence has q_tokens and k_tokens
    const AttnSeq* staged;  // or null: seq
    AttnSeq seq[kAttnArgSeqs];
};

struct AttnTensor {
    char* ptr;
    int64_t sb, st, sh;     // bytes: batch, token, head
};

// How one pass divides its work.
struct AttnSide {
    uint32_t units;         // units of one key head, all sequences
    FastDiv splits;         // parts of one unit's walk (the forward: at most)
    uint32_t* marks;        // per workgroup: repeat it with care
    float* part;            // results of the parts
    int64_t part_rows;      // rows of one part
};

struct AttnArgs {
    AttnTensor q, k, v, o, d_o, dq, dk, dv;
    float* lse;
    float* lse2;            // per row, as lse: in powers of two, +inf where a row sees nothing
    float* delta;           // per row: the sum of dout * out
    float* part_ml;         // maxima (scaled, in powers of two) and sums of parts of the forward
    FastDiv group;          // query heads of a key head
    FastDiv kv, batch;      // key heads and sequences
    AttnSide side[2];       // units that are tiles of rows, and blocks of keys
    int32_t heads, kv_heads, dim, causal, window, packed;
    int32_t q_tokens, k_tokens;
    int32_t split_keys;     // keys of a split, where splits go by the length
    float scale;
};

// One unit: a sequence, a key head and the number of the unit in them.
struct AttnUnit {
    int32_t b, q_start, q_len, q_pad, k_start, k_len, hk;
    uint32_t unit;
};

// Key heads and sequences run fastest, units slowest.  Units are numbered from the
// longest walk under a causal mask, so that the short ones fill the end; and workgroups
// go to the eight dies in turn, so that where heads times sequences are a multiple of
// eight (or divide it) a die meets the keys of an eighth of them only and shares them in
// its L2.  With a head's units in one run on a die instead, 16,384 causal tokens of 2 key
// heads gave one die 1.75 times its share.
__device__ __forceinline__ AttnUnit attn_unit(const AttnArgs& a, const AttnTable& tab, int side,
                                              uint32_t block) {
    AttnUnit w;
    const uint32_t u = a.kv.quot(block);
    w.hk = (int32_t)(block - u * a.kv.d);
    if (tab.n == 0) {
        w.unit = a.batch.quot(u);
        w.b = (int32_t)(u - w.unit * a.batch.d);
        w.q_start = w.k_start = 0;
        w.q_len = a.q_tokens;
        w.k_len = a.k_tokens;
    } else {
        int lo = 0, hi = tab.n - 1;             // the last sequence with unit0 <= u
        AttnSeq s;
        if (tab.staged != nullptr) {
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if ((uint32_t)tab.staged[mid].unit0[side] <= u) lo = mid; else hi = mid - 1;
            }
            s = tab.staged[lo];
        } else {
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if ((uint32_t)tab.seq[mid].unit0[side] <= u) lo = mid; else hi = mid - 1;
            }
            s = tab.seq[lo];
        }
        w.b = s.b;
        w.q_start = s.q_start;
        w.q_len = s.q_len;
        w.k_start = s.k_start;
        w.k_len = s.k_len;
        w.unit = u - (uint32_t)s.unit0[side];
    }
    // the same for every lane, kept in scalar registers
    w.b = __builtin_amdgcn_readfirstlane(w.b);
    w.q_start = __builtin_amdgcn_readfirstlane(w.q_start);
    w.q_len = __builtin_amdgcn_readfirstlane(w.q_len);
    w.k_start = __builtin_amdgcn_readfirstlane(w.k_start);
    w.k_len = __builtin_amdgcn_readfirstlane(w.k_len);
    w.unit = __builtin_amdgcn_readfirstlane(w.unit);
    w.hk = __builtin_amdgcn_readfirstlane(w.hk);
    w.q_pad = a.packed ? w.q_len : a.q_tokens;
    return w;
}

// First token's head `head` of a sequence.
__device__ __forceinline__ char* seq_base(const AttnTensor& t, int packed, int b, int start, int head) {
    return t.ptr + (packed ? (int64_t)0 : (int64_t)b * t.sb) + (int64_t)start * t.st + (int64_t)head * t.sh;
}

// Index into lse of query 0, head 0 of a sequence, in rows of `heads`.
__device__ __forceinline__ int64_t seq_row(const AttnArgs& a, const AttnUnit& w) {
    return ((int64_t)(a.packed ? 0 : w.b) * a.q_tokens + w.q_start) * a.heads;
}

// ---------------------------------------------------------------------------
// fragments
// ---------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c);
template <>
__device__ __forceinline__ f32x16 mfma<__bf16>(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x16 mfma<_Float16>(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Registers 8 j .. 8 j + 7 of a product as the B operand of the next: rounded to
// the 16 bits that the matrix units take (nearest, ties to even); the sums that
// they enter stay in fp32.
template <typename T>
__device__ __forceinline__ u32x4 operand(const f32x16& x, int j) {
    T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = (T)x[8 * j + i];
    u32x4 r;
    __builtin_memcpy(&r, e, 16);
    return r;
}

__device__ __forceinline__ u32x2 read_tr(const char* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(p)));
}

// Pieces of a row of DP elements; the shift spreads rows over the 256 bytes that
// the 64 banks span.
template <int DP>
__host__ __device__ constexpr int swizzle(int row) {
    if constexpr (DP == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
    return (((row >> 1) & 1) << 2) | (((row >> 2) & 1) << 1) | ((row >> 3) & 1);
}

// A lane's reads in a tile.  The piece of a row that is read enters the address
// only through the exclusive or, so each read is one of two base offsets with
// constant bits flipped.
template <int DP>
struct TileReads {
    int row;            // A operand along rows: lane's row, piece h
    int col;            // across rows: rows 4 h + .., columns 0 ..
    __device__ __forceinline__ TileReads() {
        const int lane = threadIdx.x & 63, h = lane >> 5, c = lane & 31, i = lane & 15, g = (lane >> 4) & 1;
        row = c * DP * 2 + ((h ^ swizzle<DP>(c)) << 4);
        const int r = h * 4 + (i >> 2);
        col = r * DP * 2 + (((g * 2 + ((i & 3) >> 1)) ^ swizzle<DP>(r)) << 4) + (i & 1) * 8;
    }
    // Rows 0..31 of `tile`, inner step ks.
    __device__ __forceinline__ u32x4 along(const char* tile, int ks) const {
        return *reinterpret_cast<const u32x4*>(tile + (row ^ (ks << 5)));
    }
    // Elements d .. d + 3 of a row.
    __device__ __forceinline__ const char* four(const char* tile, int r, int d) const {
        return tile + r * DP * 2 + (((d >> 3) ^ swizzle<DP>(r)) << 4) + (d & 7) * 2;
    }
    // Columns 32 db .. of rows 0..15 of `tile`, as the A operand over them.
    __device__ __forceinline__ u32x4 across(const char* tile, int db) const {
        constexpr int kFlip = (swizzle<DP>(8) << 4) | (8 * DP * 2);
        const u32x2 lo = read_tr(tile + (col ^ (db << 6))), hi = read_tr(tile + (col ^ (db << 6) ^ kFlip));
        return u32x4{lo.x, lo.y, hi.x, hi.y};
    }
};

// The second layout: for each 32 rows and inner step ks 1 KiB with 32 bytes of
// every row.  Every read then is one of a few lane offsets plus a constant, without a
// register for each; the loads that fill it take 32 bytes of a row at a time, half of
// what a compute unit's vector cache could deliver.  Plainly laid out, every read
// would meet its banks twice (half of the reads' cycles in the gradient's second
// pass): so the two pieces of rows 8 .. 15 and 24 .. 31 change places, which parts 16
// rows' reads of one piece, and rows r of odd steps stand at r ^ 4, which parts the
// two steps that a read across rows takes together.
template <int DP>
struct StepReads {
    int row[2], col[2];
    __device__ __forceinline__ StepReads() {
        const int lane = threadIdx.x & 63, h = lane >> 5, c = lane & 31, i = lane & 15, g = (lane >> 4) & 1;
        row[0] = piece(c, 0, h);
        row[1] = piece(c, 1, h);
        col[0] = g * 1024 + piece(h * 4 + (i >> 2), g, (i & 3) >> 1) + (i & 1) * 8;
        col[1] = g * 1024 + piece(h * 4 + (i >> 2) + 8, g, (i & 3) >> 1) + (i & 1) * 8;
    }
    // Where a row's piece stands in a step's 1 KiB.
    static __device__ __forceinline__ int piece(int row, int ks, int half) {
        return (row ^ ((ks & 1) << 2)) * 32 + ((half ^ ((row >> 3) & 1)) << 4);
    }
    // The row and the half that a lane loads of a step.
    static __device__ __forceinline__ int load_row(int lane, int ks) { return (lane >> 1) ^ ((ks & 1) << 2); }
    static __device__ __forceinline__ int load_half(int lane) { return (lane & 1) ^ ((lane >> 4) & 1); }
    // Rows 0..31 of the 32 rows at `sub`, inner step ks, as the A or B operand.
    __device__ __forceinline__ u32x4 along(const char* sub, int ks) const {
        return *reinterpret_cast<const u32x4*>(sub + row[ks & 1] + ks * 1024);
    }
    // Elements d .. d + 3 of a row.
    __device__ __forceinline__ const char* four(const char* sub, int r, int d) const {
        return sub + (d >> 4) * 1024 + piece(r, d >> 4, (d >> 3) & 1) + (d & 7) * 2;
    }
    // Columns 32 db .. of rows 16 j .. 16 j + 15, as the A operand over them.
    __device__ __forceinline__ u32x4 across(const char* sub, int j, int db) const {
        const char* p = sub + db * 2048 + j * 512;
        const u32x2 lo = read_tr(p + col[0]), hi = read_tr(p + col[1]);
        return u32x4{lo.x, lo.y, hi.x, hi.y};
    }
};

// A lane's 16-byte pieces 2 ks + h of one row, from memory; zeros behind the head
// size or for a row that does not exist.
template <int DP>
__device__ __forceinline__ void load_row(u32x4 (&f)[DP / 16], const char* row, bool there, int dim) {
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks) {
        f[ks] = u32x4{0, 0, 0, 0};
        if (there && (2 * ks + h) * 8 < dim) f[ks] = *reinterpret_cast<const u32x4*>(row + (2 * ks + h) * 16);
    }
}

// ---------------------------------------------------------------------------
// tiles
// ---------------------------------------------------------------------------
// ROWS rows of DP elements to LDS, each wave its part.  The byte offsets of a
// lane's pieces from the tile's first row are those of `Offsets`.
template <int DP, int ROWS>
struct TileLoads {
    static constexpr int kPieces = DP / 8;                  // of a row
    static constexpr int kStepRows = 64 / kPieces;          // rows of one load of a wave
    static constexpr int kSteps = ROWS / kStepRows / kAttnWaves;
    static constexpr int kBytes = ROWS * DP * 2;
    static_assert(kSteps * kStepRows * kAttnWaves == ROWS, "rows of a tile");
};

// Offsets of pieces of consecutive tokens, `st` bytes apart.
template <int DP, int ROWS>
struct TokenOffsets {
    uint32_t at[TileLoads<DP, ROWS>::kSteps];
    __device__ __forceinline__ TokenOffsets(int64_t st, int dim) {
        using L = TileLoads<DP, ROWS>;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int n = 0; n < L::kSteps; ++n) {
            const int row = (wave * L::kSteps + n) * L::kStepRows + lane / L::kPieces;
            const int piece = (lane % L::kPieces) ^ swizzle<DP>(row);
            at[n] = piece * 8 < dim ? (uint32_t)((int64_t)row * st) + piece * 16 : 0xFFFFFF00u;
        }
    }
};

__device__ __forceinline__ void load_piece_lds(const char* base, uint32_t bytes, uint32_t offset, char* lds) {
    const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, (int)bytes, 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds), 16,
                                             (int)offset, 0, 0, 0);
}

// Loads `rows` (those left of the sequence, any number) of a tile; `base` is its
// first row's head.
template <int DP, int ROWS>
__device__ __forceinline__ void load_tile(const char* base, int64_t st, int dim, int rows,
                                          const TokenOffsets<DP, ROWS>& off, char* lds) {
    using L = TileLoads<DP, ROWS>;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n_rows = min(rows, ROWS);
    const uint32_t bytes = n_rows > 0 ? (uint32_t)((int64_t)(n_rows - 1) * st) + dim * 2 : 0;
#pragma unroll
    for (int n = 0; n < L::kSteps; ++n)
        load_piece_lds(base, bytes, off.at[n], lds + (wave * L::kSteps + n) * 1024);
}

// The wave's loads to LDS have landed and every wave of the workgroup is here.
__device__ __forceinline__ void tiles_ready() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// ---------------------------------------------------------------------------
// the masked product
// ---------------------------------------------------------------------------
// Bits 15 and 31 where a half of x is an infinity or NaN.
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t x) {
    if constexpr (__is_same(T, __bf16)) return (x & 0x7F807F80u) + 0x00800080u;
    return (x & 0x7C007C00u) + 0x04000400u;
}
template <typename T>
__device__ __forceinline__ uint32_t not_finite(u32x4 x) {
    return not_finite<T>(x[0]) | not_finite<T>(x[1]) | not_finite<T>(x[2]) | not_finite<T>(x[3]);
}
// Bits 15 and 31 set where the operands row(0 .. n - 1), which cover a tile, hold an
// infinity or NaN.
template <typename T, typename F>
__device__ __forceinline__ uint32_t tile_not_finite(int n, F row) {
    uint32_t bad = 0;
#pragma unroll 1
    for (int i = 0; i < n; ++i) bad |= not_finite<T>(row(i));
    return bad & 0x80008000u;
}

// Care for infinities and NaN that the mask hides takes registers that the walks
// have none of to spare.  So a workgroup only notes whether a tile that its mask
// cuts held one, and a further kernel repeats the noted units with care: hardly ever
// any, and then it ends at once.  (A grid of at most kDirect workgroups, one a compute
// unit, with walks of at most kDirectKeys takes care from the start, a launch less: 64
// causal tokens of 8 heads 8.6 -> 6.6 us, their gradient 20.5 -> 17.9; at 512 tokens of
// heads of 128 the care in the walk cost the forward 1.2.)  A thread looks at one mark at a time, so that few
// workgroups look at all `blocks` of them.
template <typename F>
__device__ __forceinline__ void repeat_marked(const uint32_t* marks, uint32_t blocks, uint32_t group,
                                              uint32_t groups, F unit) {
    __shared__ uint32_t set[kAttnThreads];
    for (uint32_t first = 0; first < blocks; first += groups * kAttnThreads) {
        const uint32_t mine = first + threadIdx.x * groups + group;
        const uint32_t mark = mine < blocks ? marks[mine] : 0;
        if (!__syncthreads_or(mark != 0)) continue;
        set[threadIdx.x] = mark;
        __syncthreads();
        for (int i = 0; i < kAttnThreads; ++i) {
            if (set[i] == 0) continue;
            unit(first + i * groups + group);
            __syncthreads();
        }
    }
}

// x with its infinities and NaN as zeros.
template <typename T>
__device__ __forceinline__ u32x4 finite_part(u32x4 x) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = x[i] & ~(((not_finite<T>(x[i]) & 0x80008000u) >> 15) * 0xFFFFu);
    return r;
}

// The product acc[db] += A[db] x over 32 inner indices with a mask, where A holds
// infinities or NaN: a hidden pair must add nothing, and 0 times those is NaN in a
// matrix product.  So the matrix units take the finite part of A, with which columns
// that see none of the others keep their bits, and each inner index in turn adds its
// infinities and NaN to the columns that see it.  `x` is a product's result, a column
// per lane, zero where hidden; bit i of `seen` says that its register i is not hidden;
// `words` has room for 32 x 32 elements, the wave's own; four(k, d) are elements
// d .. d + 3 of A's inner index k, across(j, db) A's operand for its indices 16 j ...
template <typename T, int NDB, typename F, typename G>
__device__ __forceinline__ void masked_product(f32x16 (&acc)[NDB], const f32x16& x, uint32_t seen, T* words,
                                               F four, G across) {
    const int lane = threadIdx.x & 63, h = lane >> 5, c = lane & 31;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const u32x4 p = operand<T>(x, j);
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
            acc[db] = mfma<T>(finite_part<T>(across(j, db)), p, acc[db]);
            __builtin_amdgcn_sched_barrier(0);      // no operands ahead: registers are short here
        }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)        // -0 stands for a hidden pair
        words[((i >> 2) * 8 + h * 4 + (i & 3)) * 32 + c] = (seen >> i) & 1 ? (T)(x[i] + 0.0f) : (T)-0.0f;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 1
    for (int k = 0; k < 32; ++k) {
        const float p = to_f32(words[k * 32 + c]);
        const bool hidden = __builtin_bit_cast(uint32_t, p) == 0x80000000u;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                T v[4];
                __builtin_memcpy(v, four(k, db * 32 + q * 8 + h * 4), 8);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float f = to_f32(v[i]);
                    const float sum = fmaf(p, f, acc[db][4 * q + i]);
                    acc[db][4 * q + i] = hidden || f - f == 0.0f ? acc[db][4 * q + i] : sum;
                }
            }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // before the words are written again
}

// fp16 holds 6e-8 to 65,504, and dS = P (dP - delta) is about the output's gradient over
// the number of keys: below that range for ordinary gradients and a few thousand keys,
// above it for large ones and few keys.  So dS enters its product times a power of two,
// each column's own.  It starts at kDsFactor, of which no product of finite numbers
// passes fp32, and falls where an entry would pass 2^14, to leave the largest at 2^8: its
// column keeps what is 2^-32 of it or more.  Every step is exact, so results change only
// where fp16 would lose bits.  4,096 keys, an output gradient of 1e-3: dq is off by 7e-4 in
// the norm, its own rounding, and was by 5e-3.  bf16 has fp32's range and goes without.  It costs 2%: 2 x
// 2,048 causal tokens of 32 heads of 128 on 8, forward and back, 454 -> 465 us.
constexpr float kDsFactor = 0x1p64f;
template <typename T>
constexpr bool kDsScaled = __is_same(T, _Float16);

// Fits the entries x, times `factor` already, and the sums that they enter; returns the
// powers of two by which the lane's factor fell.
template <int NDB>
__device__ __forceinline__ float fit_ds(f32x16& x, f32x16 (&acc)[NDB], float& factor) {
    constexpr float kMost = 0x1p14f;
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(x[i]));
    if (!__any(top > kMost)) return 0.0f;
    top = fmaxf(top, __shfl_xor(top, 32));          // the column's other half
    const int k = top > kMost ? (int)(__builtin_bit_cast(uint32_t, top) >> 23) - 127 - 8 : 0;
    const float f = __builtin_bit_cast(float, (uint32_t)(127 - k) << 23);
    factor *= f;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] *= f;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[db][i] *= f;
    return (float)k;
}

// ---------------------------------------------------------------------------
// host side (c3_attention.hip)
// ---------------------------------------------------------------------------
// Checked sizes of a call and the list of its sequences, longest first.
struct AttnPlan {
    AttnArgs args;
    AttnTable table;
    int64_t rows;               // query rows of all heads: entries of lse
    int64_t key_rows;           // key rows of all key heads
    int64_t max_q, max_k;       // the longest of each
    AttnSeq* seqs;              // heap copy where more than kAttnArgSeqs, else null
    AttnPlan() : args(), table(), seqs(nullptr) {}
    AttnPlan(const AttnPlan&) = delete;
    ~AttnPlan() { delete[] seqs; }
    AttnSeq* list() { return seqs != nullptr ? seqs : table.seq; }
};

// How a tensor's tiles are addressed: row by row with 64 bits, or with 31 from the first
// of 64 tokens of a head, or of all heads that share a key head.
enum class Tiles { kNone, kHead, kGroup };

int attn_plan(const c3_attention_t* a, AttnPlan& p);
int attn_tensor(const c3_attn_tensor_t* t, const AttnPlan& p, bool keys, Tiles tiles, AttnTensor& to);
// Numbers the units of each sequence on one side, of which `units_of(queries, k_len,
// keys)` (queries and keys with the padding of a dense batch) gives the count, and
// returns those of one key head, or -1 where a launch of kAttnThreads threads a unit and
// key head would pass the 2^32 that its dimension holds.  Not to be launched: the number
// alone, whatever it is.
template <typename F>
int64_t attn_number(AttnPlan& p, int batch, int side, F units_of, bool launched = true) {
    AttnSide& d = p.args.side[side];
    int64_t n = 0;
    if (p.table.n == 0) {
        const int64_t u = units_of(p.args.q_tokens, p.args.k_tokens, p.args.k_tokens);
        n = u * batch;
    } else {
        AttnSeq* s = p.list();
        for (int i = 0; i < p.table.n && n >= 0; ++i) {
            s[i].unit0[side] = (int32_t)n;
            n += units_of(p.args.packed ? s[i].q_len : p.args.q_tokens, s[i].k_len,
                          p.args.packed ? s[i].k_len : p.args.k_tokens);
            if (launched && n >= (1ll << 31)) return -1;
        }
    }
    if (!launched) return n;
    if (n >= (1ll << 31) || n * p.args.kv_heads >= (1ll << 32) / kAttnThreads) return -1;
    d.units = (uint32_t)(n < 1 ? 1 : n);
    return n;
}
// Whether one of `results` starts where another or one of `inputs` does: units that are
// repeated read their rows again after others were written.
bool attn_overlap(std::initializer_list<const AttnTensor*> results, std::initializer_list<const AttnTensor*> inputs);
size_t attn_table_bytes(const c3_attention_t* a);
// Stages a list of sequences that does not go along as an argument at `to`; refuses
// a stream under capture.
int attn_stage(const c3_attention_t* a, AttnPlan& p, char* to, hipStream_t s);

// The passes of the gradient; the plan's units are numbered.
hipError_t launch_attn_dq(const AttnPlan& p, bool bf16, hipStream_t s);
hipError_t launch_attn_dkv(const AttnPlan& p, bool bf16, hipStream_t s);
// Workgroups of a pass, and whether it takes care of hidden infinities itself.
inline uint32_t attn_blocks(const AttnPlan& p, int side) {
    return p.args.side[side].units * (uint32_t)p.args.kv_heads;
}
inline bool attn_direct(const AttnPlan& p, int side) {
    return (p.args.causal || p.args.window) && attn_blocks(p, side) <= kDirect &&
           std::max(p.max_q, p.max_k) <= kDirectKeys;
}

}  // namespace c3
