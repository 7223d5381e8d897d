// The gradient of the residual norm.
//
// A workgroup walks every so many-th group of rows, the next row's elements on their way
// while one is worked on, and keeps its sums over tokens in registers.
#pragma once

#include "c3_norm.h"

namespace c3 {
namespace {

// BLOCK, POST: whether y and post are there; GATE: a c3_gate_t.  Their code and sums
// cost registers, so each form is a kernel of its own.
template <typename R, typename B, bool WIDE, int TPR, int PK, bool BLOCK, bool POST, int GATE>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void residual_norm_grad_kernel(NormArgs a) {
    constexpr int RPB = rows_of_block<TPR>();
    constexpr bool AHEAD = PK == 1;         // two pieces leave sixteen waves no registers for it
    __shared__ float lds[16];
    const int tid = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const float inv = 1.0f / (float)a.hidden;
    float s_weight[PK][E] = {}, s_post[POST ? PK : 1][E] = {}, s_gate[GATE == C3_GATE_CHANNELS ? PK : 1][E] = {};
    const int64_t walk = (int64_t)gridDim.x * RPB;
    // every thread takes part in the sums: groups behind the last row work on that again
    const auto row_of = [&](int64_t first) { return min(first + sub, a.tokens - 1); };
    struct Row {
        Raw<R> x[PK], dh[PK];
        Raw<B> dn[PK], y[BLOCK ? PK : 1], gate[GATE == C3_GATE_TOKENS ? PK : 1];
        float2 st;
    };
    const auto fetch = [&](int64_t row) {
        Row r;
        r.st = *reinterpret_cast<const float2*>(a.stats + 2 * row);
#pragma unroll
        for (int k = 0; k < PK; ++k) {
            const int at = (k * TPR + tid) * E;
            r.x[k] = fetch8<R, WIDE>(a.x, row, at, a.hidden);
            r.dn[k] = fetch8<B, WIDE>(a.dn, row, at, a.hidden);
            if constexpr (BLOCK) r.y[k] = fetch8<B, WIDE>(a.y, row, at, a.hidden);
            if constexpr (GATE == C3_GATE_TOKENS) r.gate[k] = fetch8<B, WIDE>(a.gate, row, at, a.hidden);
            if (a.dh.p != nullptr) r.dh[k] = fetch8<R, WIDE>(a.dh, row, at, a.hidden);
            else r.dh[k] = Raw<R>{};
        }
        return r;
    };
    // the rows that all tokens share stay in registers
    Raw<B> weight[PK], post[POST ? PK : 1], channels[GATE == C3_GATE_CHANNELS ? PK : 1];
#pragma unroll
    for (int k = 0; k < PK; ++k) {
        const int at = (k * TPR + tid) * E;
        weight[k] = fetch8<B, WIDE>(a.weight, 0, at, a.hidden);
        if constexpr (POST) post[k] = fetch8<B, WIDE>(a.post, 0, at, a.hidden);
        if constexpr (GATE == C3_GATE_CHANNELS) channels[k] = fetch8<B, WIDE>(a.gate, 0, at, a.hidden);
    }
    Row next;
    if constexpr (AHEAD) next = fetch(row_of((int64_t)blockIdx.x * RPB));
    for (int64_t first = (int64_t)blockIdx.x * RPB; first < a.tokens; first += walk) {
        const bool there = first + sub < a.tokens;
        const int64_t row = row_of(first);
        Row cur;
        if constexpr (AHEAD) {
            cur = next;
            next = fetch(row_of(first + walk < a.tokens ? first + walk : first));
        } else {
            cur = fetch(row);
        }
        const float rh = cur.st.x, ry = cur.st.y;
        const auto gate_of = [&](int k, float (&w)[E]) {
            if constexpr (GATE == C3_GATE_TOKENS) expand8(cur.gate[k], w);
            if constexpr (GATE == C3_GATE_CHANNELS) expand8(channels[k], w);
        };
        float d[PK][E], h[PK][E], y[BLOCK ? PK : 1][E], w[E];
        // h as in the forward pass
#pragma unroll
        for (int k = 0; k < PK; ++k) {
            expand8(cur.x[k], h[k]);
            expand8(cur.dn[k], d[k]);
        }
        if constexpr (BLOCK) {
#pragma unroll
            for (int k = 0; k < PK; ++k) {
                expand8(cur.y[k], y[k]);
                float z[E];
                if constexpr (POST) expand8(post[k], w);
#pragma unroll
                for (int i = 0; i < E; ++i) z[i] = POST ? y[k][i] * ry * w[i] : y[k][i];
                if constexpr (GATE != C3_GATE_NONE) {
                    gate_of(k, w);
#pragma unroll
                    for (int i = 0; i < E; ++i) z[i] *= w[i];
                }
#pragma unroll
                for (int i = 0; i < E; ++i) h[k][i] = fmaf(a.scale, z[i], h[k][i]);
            }
        }
        // d becomes the gradient of h
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < PK; ++k) {
            expand8(weight[k], w);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                h[k][i] *= rh;
                if (there) s_weight[k][i] = fmaf(d[k][i], h[k][i], s_weight[k][i]);
                d[k][i] *= w[i];
                sum = fmaf(d[k][i], h[k][i], sum);
            }
        }
        const float mean = row_sum<TPR>(sum, lds) * inv;
#pragma unroll
        for (int k = 0; k < PK; ++k) {
            expand8(cur.dh[k], w);
#pragma unroll
            for (int i = 0; i < E; ++i) d[k][i] = fmaf(rh, fmaf(-h[k][i], mean, d[k][i]), w[i]);
            if (there) store8<R, WIDE>(a.dx, row, (k * TPR + tid) * E, a.hidden, d[k]);
        }
        if constexpr (BLOCK) {
            // d becomes the gradient of z, then of y
            sum = 0.0f;
#pragma unroll
            for (int k = 0; k < PK; ++k) {
                const int at = (k * TPR + tid) * E;
                float p[E];
                if constexpr (POST) {
                    expand8(post[k], p);
#pragma unroll
                    for (int i = 0; i < E; ++i) y[k][i] *= ry;
                }
#pragma unroll
                for (int i = 0; i < E; ++i) d[k][i] *= a.scale;
                if constexpr (GATE != C3_GATE_NONE) {
                    float dg[E];
#pragma unroll
                    for (int i = 0; i < E; ++i) dg[i] = d[k][i] * (POST ? y[k][i] * p[i] : y[k][i]);
                    if constexpr (GATE == C3_GATE_CHANNELS) {
#pragma unroll
                        for (int i = 0; i < E; ++i)
                            if (there) s_gate[k][i] += dg[i];
                    } else if (there) {
                        store8<B, WIDE>(a.dgate, row, at, a.hidden, dg);
                    }
                    gate_of(k, w);
#pragma unroll
                    for (int i = 0; i < E; ++i) d[k][i] *= w[i];
                }
                if constexpr (POST) {
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        if (there) s_post[k][i] = fmaf(d[k][i], y[k][i], s_post[k][i]);
                        d[k][i] *= p[i];
                        sum = fmaf(d[k][i], y[k][i], sum);
                    }
                }
            }
            if constexpr (POST) {
                const float mean_y = row_sum<TPR>(sum, lds) * inv;
#pragma unroll
                for (int k = 0; k < PK; ++k)
#pragma unroll
                    for (int i = 0; i < E; ++i) d[k][i] = ry * fmaf(-y[k][i], mean_y, d[k][i]);
            }
            if (there)
#pragma unroll
                for (int k = 0; k < PK; ++k) store8<B, WIDE>(a.dy, row, (k * TPR + tid) * E, a.hidden, d[k]);
        }
    }
    // the workgroup's parts
    const int64_t group = (int64_t)blockIdx.x * RPB + sub;
    auto part = [&](int kind, const float (*s)[E]) {
        float* to = a.parts + (kind * a.groups + group) * a.hidden;
#pragma unroll
        for (int k = 0; k < PK; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i)
                if ((k * TPR + tid) * E + i < a.hidden) to[(k * TPR + tid) * E + i] = s[k][i];
    };
    part(0, s_weight);
    if constexpr (POST) part(1, s_post);
    if constexpr (GATE == C3_GATE_CHANNELS) part(2, s_gate);
}

template <typename R, typename B, bool WIDE, int TPR, int PK>
hipError_t by_form(const NormArgs& a, unsigned blocks, hipStream_t s) {
    const dim3 grid(blocks), block(TPR < 256 ? 256 : TPR);
    const int form = a.y.p == nullptr ? 0 : a.post.p == nullptr ? 1 + a.gate_kind : 4 + a.gate_kind;
    switch (form) {
        case 0: residual_norm_grad_kernel<R, B, WIDE, TPR, PK, false, false, 0><<<grid, block, 0, s>>>(a); break;
        case 1: residual_norm_grad_kernel<R, B, WIDE, TPR, PK, true, false, 0><<<grid, block, 0, s>>>(a); break;
        case 2: residual_norm_grad_kernel<R, B, WIDE, TPR, PK, true, false, 1><<<grid, block, 0, s>>>(a); break;
        case 3: residual_norm_grad_kernel<R, B, WIDE, TPR, PK, true, false, 2><<<grid, block, 0, s>>>(a); break;
        case 4: residual_norm_grad_kernel<R, B, WIDE, TPR, PK, true, true, 0><<<grid, block, 0, s>>>(a); break;
        case 5: residual_norm_grad_kernel<R, B, WIDE, TPR, PK, true, true, 1><<<grid, block, 0, s>>>(a); break;
        default: residual_norm_grad_kernel<R, B, WIDE, TPR, PK, true, true, 2><<<grid, block, 0, s>>>(a); break;
    }
    return hipGetLastError();
}

template <typename R, typename B, bool WIDE>
hipError_t grad_by_width(const NormArgs& a, unsigned blocks, hipStream_t s) {
    switch (norm_grad_threads(a.hidden)) {
        case 64: return by_form<R, B, WIDE, 64, 1>(a, blocks, s);
        case 128: return by_form<R, B, WIDE, 128, 1>(a, blocks, s);
        case 256: return by_form<R, B, WIDE, 256, 1>(a, blocks, s);
        case 512: return by_form<R, B, WIDE, 512, 1>(a, blocks, s);
        default:
            return a.hidden <= 1024 * E ? by_form<R, B, WIDE, 1024, 1>(a, blocks, s)
                                        : by_form<R, B, WIDE, 1024, 2>(a, blocks, s);
    }
}

}  // namespace

template <typename R, typename B>
hipError_t launch_norm_grad(const NormArgs& a, bool wide, unsigned blocks, hipStream_t s) {
    return wide ? grad_by_width<R, B, true>(a, blocks, s) : grad_by_width<R, B, false>(a, blocks, s);
}

}  // namespace c3
