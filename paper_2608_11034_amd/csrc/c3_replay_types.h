// Element types, wide loads and small helpers of the replay operators.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/c3_replay.h"

namespace c3 {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// V elements of one load: 16 bytes on the wide paths, one element otherwise.
template <typename T, int V>
struct alignas(sizeof(T) * V) AlignedPack {
    T v[V];
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__bf16 x) { return (float)x; }
__device__ __forceinline__ float to_f32(_Float16 x) { return (float)x; }

// An fp32 result rounded to T.  In fp16 the compiler may join a last product or sum with
// the rounding, which then rounds once instead of twice; where it does goes by how the
// stores are laid out, and the bits must not: what is rounded is an fp32 value in a register.
template <typename T>
__device__ __forceinline__ T from_f32(float x) {
    if constexpr (sizeof(T) == 2) asm("" : "+v"(x));
    return (T)x;
}

// Division by a run-time constant d of numbers below 2^31: q = (mulhi(n, m) +
// n) >> s, with s = ceil(log2 d) and m = ceil(2^32 (2^s - d) / d) (Granlund and
// Montgomery, division by invariant integers, 1994).
struct FastDiv {
    uint32_t d, m, s;
    FastDiv() : d(1), m(0), s(0) {}
    explicit FastDiv(uint32_t div) : d(div), s(0) {
        while ((1ull << s) < div) ++s;
        m = (uint32_t)((((1ull << 32) * ((1ull << s) - div)) + div - 1) / div);
    }
    __device__ __forceinline__ uint32_t quot(uint32_t n) const {
        return (__umulhi(n, m) + n) >> s;       // m < 2^32, so the sum is below 2 n
    }
};

// A launch dimension holds fewer than 2^32 threads, and one with more is cut off without
// an error.  So grids that may pass that have two dimensions; the last workgroups of
// the second may have nothing to do.
inline dim3 wide_grid(uint64_t blocks, unsigned threads = 256) {
    const uint64_t kRow = (1u << 30) / threads;
    return blocks <= kRow ? dim3((unsigned)blocks) : dim3((unsigned)kRow, (unsigned)((blocks + kRow - 1) / kRow));
}
__device__ __forceinline__ int64_t wide_block() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }
__device__ __forceinline__ int64_t wide_blocks() { return (int64_t)gridDim.y * gridDim.x; }

inline int replay_elem_size(int dtype) {
    return dtype == C3_F32 ? 4 : dtype == C3_BF16 || dtype == C3_F16 ? 2 : 0;
}

}  // namespace c3
