// Rotary positions (include/c3_replay.h).
//
// Pair i of every head of a token is turned by position * freqs[i].  One pass:
// each element is read and written once, so HBM bounds it.  The cosines and
// sines of a token are shared by all its heads: a workgroup takes as many
// tokens as give its 256 threads about two items each, puts the tokens'
// rot / 2 pairs of (cos, sin) into LDS once, and turns the heads of both tensors
// with them.  An item is one 16-byte piece of a head (both halves of it where
// the pair's elements are half a head apart).  The first items are loaded before the
// cosines and sines are formed, and few of them a thread keep many waves on a compute
// unit.  4 x 4,096 tokens of 64 heads of 128 in bf16: 103 us, 5.2 TB/s, what a large copy
// reaches (four items a thread 112); 16,383 tokens of 36 heads of 64 in fp32, a quarter
// turned: 53 us, 5.7 TB/s (60; trigonometry before any load 81).
//
// The angle is formed in fp64 in whole turns and only its fraction is rounded
// to fp32: at position 131,072 an fp32 angle is off by up to 0.004 radians.
#include "c3_internal.h"
#include "c3_replay_types.h"

namespace c3 {
namespace {

constexpr int kThreads = 256;
constexpr int kItems = 2;

struct RotaryArgs {
    c3_heads_t t[2];
    const void* pos;
    int64_t pos_stride[2];
    const double* freqs;
    int64_t tokens;          // batch * length
    FastDiv length;          // tokens of a sequence
    FastDiv items;           // items of a head
    FastDiv token_items;     // items of a token, both tensors
    uint32_t heads0;         // heads of the first tensor
    int32_t dim, rot, pos_bytes, interleaved;
    int32_t block_tokens;
    float amplitude, sign;
};

template <typename T, int V>
__device__ __forceinline__ AlignedPack<T, V> load_piece(const T* p) {
    return *reinterpret_cast<const AlignedPack<T, V>*>(p);
}
template <typename T, int V>
__device__ __forceinline__ void store_piece(T* p, const AlignedPack<T, V>& x) {
    *reinterpret_cast<AlignedPack<T, V>*>(p) = x;
}

// Items of a head.  V > 1: rot / 2 / V pieces of both halves (or rot / V pieces
// of neighbouring pairs), then (dim - rot) / V pieces that are copied.  V = 1:
// rot / 2 pairs, then dim - rot elements.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
    extern __shared__ float2 turn[];        // [block_tokens][rot / 2]
    const int half = a.rot / 2;
    const int64_t tok0 = wide_block() * a.block_tokens;
    if (tok0 >= a.tokens) return;
    const int nt = (int)min((int64_t)a.block_tokens, a.tokens - tok0);
    const bool pairs_apart = V == 1 || !a.interleaved;
    const int turned = pairs_apart ? half / V : a.rot / V;
    const uint32_t n = (uint32_t)nt * a.token_items.d;

    AlignedPack<T, V> x[kItems], y[kItems];
    T* out[kItems];
    int first[kItems], second[kItems], cs[kItems];
    auto load = [&](uint32_t base) {
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            const uint32_t i = base + u * kThreads;
            out[u] = nullptr;
            if (i >= n) continue;
            const uint32_t t = a.token_items.quot(i), r = i - t * a.token_items.d;
            uint32_t head = a.items.quot(r);
            const int c = (int)(r - head * a.items.d);
            const bool other = head >= a.heads0;
            if (other) head -= a.heads0;
            const c3_heads_t& h = other ? a.t[1] : a.t[0];
            const uint32_t tok = (uint32_t)(tok0 + t), b = a.length.quot(tok);
            const int64_t s = tok - b * a.length.d;
            const T* in = (const T*)h.in + (int64_t)b * h.in_stride[0] + s * h.in_stride[1] +
                          (int64_t)head * h.in_stride[2];
            out[u] = (T*)h.out + (int64_t)b * h.out_stride[0] + s * h.out_stride[1] +
                     (int64_t)head * h.out_stride[2];
            cs[u] = -1;
            second[u] = -1;
            if (c >= turned) {
                first[u] = a.rot + (c - turned) * V;
                if (h.in == h.out) { out[u] = nullptr; continue; }    // in place already
            } else if (pairs_apart) {
                const int p = c * V;
                const bool near = V == 1 && a.interleaved;
                first[u] = near ? 2 * p : p;
                second[u] = near ? 2 * p + 1 : p + half;
                cs[u] = (int)t * half + p;
                y[u] = load_piece<T, V>(in + second[u]);
            } else {
                first[u] = c * V;
                cs[u] = (int)t * half + c * (V / 2);
            }
            x[u] = load_piece<T, V>(in + first[u]);
        }
    };

    // the first items are on their way while the cosines and sines are formed
    load(threadIdx.x);
    for (int i = threadIdx.x; i < nt * half; i += kThreads) {
        const int t = i / half, p = i - t * half;
        const uint32_t tok = (uint32_t)(tok0 + t), b = a.length.quot(tok);
        const int64_t at = (int64_t)b * a.pos_stride[0] + (int64_t)(tok - b * a.length.d) * a.pos_stride[1];
        const double pos = a.pos_bytes == 8 ? (double)((const int64_t*)a.pos)[at]
                                            : (double)((const int32_t*)a.pos)[at];
        const double turns = pos * a.freqs[p] * 0.15915494309189533577;
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        turn[i] = make_float2(c * a.amplitude, s * a.amplitude * a.sign);
    }
    __syncthreads();
    for (uint32_t base = threadIdx.x; base < n; base += kThreads * kItems) {
        if (base >= kThreads * kItems) load(base);
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            if (out[u] == nullptr) continue;
            if (cs[u] >= 0) {
                if (pairs_apart) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float2 w = turn[cs[u] + j];
                        const float p = to_f32(x[u].v[j]), q = to_f32(y[u].v[j]);
                        x[u].v[j] = (T)fmaf(p, w.x, -q * w.y);
                        y[u].v[j] = (T)fmaf(q, w.x, p * w.y);
                    }
                    store_piece<T, V>(out[u] + second[u], y[u]);
                } else {
#pragma unroll
                    for (int j = 0; j < V / 2; ++j) {
                        const float2 w = turn[cs[u] + j];
                        const float p = to_f32(x[u].v[2 * j]), q = to_f32(x[u].v[2 * j + (V > 1)]);
                        x[u].v[2 * j] = (T)fmaf(p, w.x, -q * w.y);
                        x[u].v[2 * j + (V > 1)] = (T)fmaf(q, w.x, p * w.y);
                    }
                }
            }
            store_piece<T, V>(out[u] + first[u], x[u]);
        }
    }
}

inline bool multiple(int64_t x, int64_t of) { return x % of == 0; }

template <typename T, int V>
hipError_t launch(const RotaryArgs& a, hipStream_t s) {
    const int64_t blocks = (a.tokens + a.block_tokens - 1) / a.block_tokens;
    const size_t lds = sizeof(float2) * (size_t)a.block_tokens * (size_t)(a.rot / 2);
    rotary_kernel<T, V><<<wide_grid((uint64_t)blocks), dim3(kThreads), lds, s>>>(a);
    return hipGetLastError();
}

}  // namespace
}  // namespace c3

extern "C" int c3_rotary(const c3_heads_t* tensors, int n, int dtype, int64_t batch, int64_t length,
                         int64_t dim, const void* positions, int pos_bytes,
                         const int64_t pos_stride[2], const double* freqs, int64_t rot, int layout,
                         int inverse, double amplitude, c3_stream_t stream) {
    using namespace c3;
    const int es = replay_elem_size(dtype);
    if (tensors == nullptr || n < 1 || n > 2 || batch < 0 || length < 0 || dim < 1 || dim > 4096 ||
        rot < 2 || rot > dim || rot % 2 != 0 || pos_stride == nullptr ||
        (pos_bytes != 4 && pos_bytes != 8) ||
        (layout != C3_ROTARY_HALF && layout != C3_ROTARY_INTERLEAVED) || !(amplitude - amplitude == 0))
        return C3_E_INVAL;
    if (es == 0) return C3_E_UNSUPPORTED;
    // each bounded before their product, which then cannot overflow
    if (batch >= (1ll << 31) || length >= (1ll << 31) || batch * length >= (1ll << 31))
        return C3_E_INVAL;
    int64_t heads = 0;
    for (int i = 0; i < n; ++i) {
        if (tensors[i].heads < 0 || tensors[i].heads > 65536) return C3_E_INVAL;
        heads += tensors[i].heads;
    }
    if (batch * length == 0 || heads == 0) return C3_OK;
    if (positions == nullptr || freqs == nullptr) return C3_E_INVAL;
    if ((uintptr_t)positions % pos_bytes != 0 || (uintptr_t)freqs % 8 != 0) return C3_E_ALIGN;
    RotaryArgs a{};
    const int v = 16 / es;
    // 16-byte pieces where every head starts on one and no piece straddles
    // the two halves or the end of what is turned; single elements otherwise
    bool wide = multiple(dim, v) && multiple(layout == C3_ROTARY_HALF ? rot / 2 : rot, v) &&
                multiple(rot, v);
    for (int i = 0; i < n; ++i) {
        const c3_heads_t& t = tensors[i];
        if (t.heads == 0) continue;
        if (t.in == nullptr || t.out == nullptr) return C3_E_INVAL;
        if ((uintptr_t)t.in % es != 0 || (uintptr_t)t.out % es != 0) return C3_E_ALIGN;
        wide = wide && (uintptr_t)t.in % 16 == 0 && (uintptr_t)t.out % 16 == 0;
        const int64_t entries[3] = {batch, length, t.heads};
        for (int j = 0; j < 3; ++j) {
            if (entries[j] == 1) continue;          // its stride says nothing
            if (t.in == t.out && t.in_stride[j] != t.out_stride[j]) return C3_E_INVAL;
            wide = wide && multiple(t.in_stride[j], v) && multiple(t.out_stride[j], v);
        }
    }
    a.t[0] = tensors[0];
    a.t[1] = tensors[n - 1];
    a.pos = positions;
    a.pos_stride[0] = pos_stride[0];
    a.pos_stride[1] = pos_stride[1];
    a.pos_bytes = pos_bytes;
    a.freqs = freqs;
    a.tokens = batch * length;
    a.length = FastDiv((uint32_t)length);
    a.dim = (int32_t)dim;
    a.rot = (int32_t)rot;
    a.interleaved = layout == C3_ROTARY_INTERLEAVED;
    a.heads0 = (uint32_t)tensors[0].heads;
    a.amplitude = (float)amplitude;
    a.sign = inverse ? -1.0f : 1.0f;
    const int64_t per_head = !wide ? rot / 2 + dim - rot
                             : (layout == C3_ROTARY_HALF ? rot / 2 : rot) / v + (dim - rot) / v;
    if (per_head * heads >= (1ll << 24)) return C3_E_INVAL;
    a.items = FastDiv((uint32_t)per_head);
    a.token_items = FastDiv((uint32_t)(per_head * heads));
    int64_t bt = kThreads * kItems / (per_head * heads);
    bt = bt < 1 ? 1 : bt > 16 ? 16 : bt;
    // at most 32 KiB of cosines and sines
    while (bt > 1 && bt * (rot / 2) * 8 > 32768) bt /= 2;
    a.block_tokens = (int32_t)bt;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    hipError_t e;
    if (dtype == C3_F32)
        e = wide ? launch<float, 4>(a, s) : launch<float, 1>(a, s);
    else if (dtype == C3_BF16)
        e = wide ? launch<__bf16, 8>(a, s) : launch<__bf16, 1>(a, s);
    else
        e = wide ? launch<_Float16, 8>(a, s) : launch<_Float16, 1>(a, s);
    return e == hipSuccess ? C3_OK : C3_E_HIP;
}
