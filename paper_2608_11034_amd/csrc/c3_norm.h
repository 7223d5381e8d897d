// What the residual norm and its gradient share: rows in registers and their sums.
#pragma once

#include <algorithm>

#include "c3_internal.h"
#include "c3_replay_types.h"

namespace c3 {

constexpr int E = 8;                // elements of a thread's piece

struct Rows {
    char* p;
    int64_t stride;                 // in elements
};

// 8 elements of a row as they lie in memory; zeros behind `hidden`.  Where widths or
// addresses are not in 16 bytes (WIDE), loads and stores of whole pieces still are, at the
// element's alignment, which the memory units take (16,384 tokens of 4,097 in bf16: 127 us
// forward and 275 back, 333 and 456 element by element).
template <typename T>
struct Raw {
    T v[E];
};

template <typename T, bool WIDE>
__device__ __forceinline__ Raw<T> fetch8(const Rows& r, int64_t row, int at, int hidden) {
    const T* p = reinterpret_cast<const T*>(r.p) + row * r.stride;
    Raw<T> x;
    if constexpr (WIDE) {
        constexpr int V = 16 / sizeof(T);
        u32x4 v[E / V];
#pragma unroll
        for (int i = 0; i < E / V; ++i) v[i] = at < hidden ? reinterpret_cast<const u32x4*>(p + at)[i] : u32x4{};
        __builtin_memcpy(&x, v, sizeof(x));
    } else if (at + E <= hidden) {
        __builtin_memcpy(&x, p + at, sizeof(x));
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) x.v[i] = at + i < hidden ? p[at + i] : (T)0.0f;
    }
    return x;
}

template <typename T>
__device__ __forceinline__ void expand8(const Raw<T>& r, float (&x)[E]) {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = to_f32(r.v[i]);
}

template <typename T, bool WIDE>
__device__ __forceinline__ void load8(const Rows& r, int64_t row, int at, int hidden, float (&x)[E]) {
    expand8(fetch8<T, WIDE>(r, row, at, hidden), x);
}

template <typename T, bool WIDE>
__device__ __forceinline__ void store8(const Rows& r, int64_t row, int at, int hidden, const float (&x)[E]) {
    T* p = reinterpret_cast<T*>(r.p) + row * r.stride;
    if constexpr (WIDE) {
        constexpr int V = 16 / sizeof(T);
        if (at >= hidden) return;
#pragma unroll
        for (int i = 0; i < E; i += V) {
            AlignedPack<T, V> v;
#pragma unroll
            for (int j = 0; j < V; ++j) v.v[j] = from_f32<T>(x[i + j]);
            *reinterpret_cast<AlignedPack<T, V>*>(p + at + i) = v;
        }
    } else if (at + E <= hidden) {
        Raw<T> y;
#pragma unroll
        for (int i = 0; i < E; ++i) y.v[i] = from_f32<T>(x[i]);
        __builtin_memcpy(p + at, &y, sizeof(y));
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (at + i < hidden) p[at + i] = from_f32<T>(x[i]);
    }
}

// The sum over the TPR threads of a row, the same in each of them.
template <int TPR>
__device__ __forceinline__ float row_sum(float x, float* lds) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    if constexpr (TPR > 64) {
        constexpr int kWaves = TPR / 64;
        const int wave = threadIdx.x >> 6, first = wave / kWaves * kWaves;
        __syncthreads();                    // the last sum's readers are through
        if ((threadIdx.x & 63) == 0) lds[wave] = x;
        __syncthreads();
        x = lds[first];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) x += lds[first + w];
    }
    return x;
}

struct NormArgs {
    Rows x, y, gate, h, n;                      // forward
    Rows dn, dh, dx, dy, dgate;                 // gradient
    Rows weight, post;                          // one row each
    float* stats;
    float* parts;                               // [kinds][groups][hidden]
    float* sums;                                // [3][hidden]
    int64_t tokens;
    int64_t groups;                             // of rows walked together, for the parts
    int hidden, gate_kind;
    float scale, eps;
};

template <int TPR>
constexpr int rows_of_block() { return TPR < 256 ? 256 / TPR : 1; }

// Threads that share a row: as few as hold it in two pieces each.
inline int norm_threads(int64_t hidden) {
    int t = 64;
    while (t < 1024 && t * 2 * E < hidden) t *= 2;
    return t;
}

// In the gradient one piece each, as its sums over tokens take registers too.
inline int norm_grad_threads(int64_t hidden) {
    int t = 64;
    while (t < 1024 && t * E < hidden) t *= 2;
    return t;
}

// The gradient of one pair of types (residual, block): c3_norm_grad_*.hip.
template <typename R, typename B>
hipError_t launch_norm_grad(const NormArgs& a, bool wide, unsigned blocks, hipStream_t s);

}  // namespace c3
