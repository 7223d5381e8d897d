// The residual sum with the norms around a block, and its gradient
// (include/c3_replay.h).
//
// Both are bound by HBM: every row is read once and held in registers between its
// sums and its results.  TPR threads share a row, each with PK times 8 elements in a
// row of the width; sums over a row run over a thread's elements, a butterfly over the
// wave, then the waves in order.  An odd width or alignment changes how the elements
// are loaded, not which thread has them, so the bits do not go by it.
//
// The gradient's sums over tokens stay in a thread's registers while a workgroup walks
// every so many-th group of rows; a second launch adds up the workgroups' parts in
// order.
//
// 16,384 tokens of 4,096 in bf16: 537 MB forward in 91 us (5.9 TB/s, above a large copy's
// 5.2) and 806 MB back in 160 (5.0), 6 to add up the parts.  8 tokens: 3.7 us, of which
// most is the launch.
#include "c3_norm.h"

namespace c3 {
namespace {

template <typename R, typename B, bool WIDE, int TPR, int PK>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void residual_norm_kernel(NormArgs a) {
    constexpr int RPB = rows_of_block<TPR>();
    __shared__ float lds[16];
    const int tid = threadIdx.x % TPR;
    const int64_t want = wide_block() * RPB + threadIdx.x / TPR;
    const bool there = want < a.tokens;
    const int64_t row = there ? want : a.tokens - 1;        // every thread takes part in the sums
    const float inv = 1.0f / (float)a.hidden;
    float h[PK][E];
#pragma unroll
    for (int k = 0; k < PK; ++k) load8<R, WIDE>(a.x, row, (k * TPR + tid) * E, a.hidden, h[k]);
    float ry = 1.0f;
    if (a.y.p != nullptr) {
        float y[PK][E], w[E];
#pragma unroll
        for (int k = 0; k < PK; ++k) load8<B, WIDE>(a.y, row, (k * TPR + tid) * E, a.hidden, y[k]);
        if (a.post.p != nullptr) {
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < PK; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) sum = fmaf(y[k][i], y[k][i], sum);
            ry = 1.0f / sqrtf(row_sum<TPR>(sum, lds) * inv + a.eps);
#pragma unroll
            for (int k = 0; k < PK; ++k) {
                load8<B, WIDE>(a.post, 0, (k * TPR + tid) * E, a.hidden, w);
#pragma unroll
                for (int i = 0; i < E; ++i) y[k][i] = y[k][i] * ry * w[i];
            }
        }
        if (a.gate_kind != C3_GATE_NONE) {
#pragma unroll
            for (int k = 0; k < PK; ++k) {
                load8<B, WIDE>(a.gate, a.gate_kind == C3_GATE_TOKENS ? row : 0, (k * TPR + tid) * E, a.hidden, w);
#pragma unroll
                for (int i = 0; i < E; ++i) y[k][i] *= w[i];
            }
        }
#pragma unroll
        for (int k = 0; k < PK; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i) h[k][i] = fmaf(a.scale, y[k][i], h[k][i]);
        if (there)
#pragma unroll
            for (int k = 0; k < PK; ++k) store8<R, WIDE>(a.h, row, (k * TPR + tid) * E, a.hidden, h[k]);
    }
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < PK; ++k)
#pragma unroll
        for (int i = 0; i < E; ++i) sum = fmaf(h[k][i], h[k][i], sum);
    const float rh = 1.0f / sqrtf(row_sum<TPR>(sum, lds) * inv + a.eps);
    if (!there) return;
#pragma unroll
    for (int k = 0; k < PK; ++k) {
        float w[E];
        load8<B, WIDE>(a.weight, 0, (k * TPR + tid) * E, a.hidden, w);
#pragma unroll
        for (int i = 0; i < E; ++i) h[k][i] = h[k][i] * rh * w[i];
        store8<B, WIDE>(a.n, row, (k * TPR + tid) * E, a.hidden, h[k]);
    }
    if (tid == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(rh, ry);
}

// sums[kind][c] = the groups' parts of column c: 64 columns a workgroup, each of its
// sixteen waves a run of the groups.
__global__ __launch_bounds__(1024) void norm_parts_kernel(const float* parts, int64_t groups, int hidden,
                                                          int kinds, float* sums) {
    __shared__ float lds[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int kind = blockIdx.y;
    if (!((kinds >> kind) & 1)) return;
    const int c = blockIdx.x * 64 + lane, col = min(c, hidden - 1);
    const int64_t each = (groups + 15) / 16, begin = wave * each, end = min(groups, begin + each);
    const float* p = parts + kind * groups * hidden + col;
    float sum = 0.0f;
    for (int64_t g = begin; g < end; g += 8) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p[min(g + i, end - 1) * hidden];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += g + i < end ? v[i] : 0.0f;
    }
    lds[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || c >= hidden) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += lds[w][lane];
    sums[(int64_t)kind * hidden + c] = sum;
}

// Workgroups of the gradient, all of which the device holds at once: two a compute unit of
// up to eight waves, one of sixteen.  Three or four smaller ones a unit were slower (8,191
// gated tokens of 2,048: 122 us forward and back with 1,024 workgroups, 117 with 512): the
// registers of the gated forms leave no room for the fourth.
int64_t grad_blocks(int64_t tokens, int64_t hidden) {
    const int t = norm_grad_threads(hidden), rpb = std::max(1, 256 / t);
    return std::min<int64_t>((tokens + rpb - 1) / rpb, t <= 512 ? 512 : 256);
}
int64_t grad_groups(int64_t tokens, int64_t hidden) {
    return grad_blocks(tokens, hidden) * std::max(1, 256 / norm_grad_threads(hidden));
}

template <typename R, typename B, bool WIDE, int TPR, int PK>
hipError_t launch(const NormArgs& a, hipStream_t s) {
    constexpr int kBlock = TPR < 256 ? 256 : TPR, RPB = rows_of_block<TPR>();
    residual_norm_kernel<R, B, WIDE, TPR, PK><<<wide_grid((uint64_t)(a.tokens + RPB - 1) / RPB, kBlock), dim3(kBlock), 0, s>>>(a);
    return hipGetLastError();
}

template <typename R, typename B, bool WIDE>
hipError_t by_width(const NormArgs& a, hipStream_t s) {
    switch (norm_threads(a.hidden)) {
        case 64: return a.hidden <= 64 * E ? launch<R, B, WIDE, 64, 1>(a, s) : launch<R, B, WIDE, 64, 2>(a, s);
        case 128: return launch<R, B, WIDE, 128, 2>(a, s);
        case 256: return launch<R, B, WIDE, 256, 2>(a, s);
        case 512: return launch<R, B, WIDE, 512, 2>(a, s);
        default: return launch<R, B, WIDE, 1024, 2>(a, s);
    }
}

template <typename R, typename B>
hipError_t by_kind(const NormArgs& a, bool grad, bool wide, hipStream_t s) {
    if (!grad) return wide ? by_width<R, B, true>(a, s) : by_width<R, B, false>(a, s);
    const hipError_t e = launch_norm_grad<R, B>(a, wide, (unsigned)grad_blocks(a.tokens, a.hidden), s);
    if (e != hipSuccess) return e;
    const int kinds = 1 | (a.post.p != nullptr ? 2 : 0) | (a.gate_kind == C3_GATE_CHANNELS ? 4 : 0);
    norm_parts_kernel<<<dim3((unsigned)((a.hidden + 63) / 64), 3), dim3(1024), 0, s>>>(a.parts, a.groups, a.hidden,
                                                                                      kinds, a.sums);
    return hipGetLastError();
}

int by_type(const c3_residual_norm_t* c, NormArgs& a, bool grad, hipStream_t s) {
    a.tokens = c->tokens;
    a.hidden = (int)c->hidden;
    a.gate_kind = a.y.p != nullptr ? c->gate : C3_GATE_NONE;
    a.scale = c->scale;
    a.eps = c->eps;
    const int es = replay_elem_size(c->dtype), rs = replay_elem_size(c->residual);
    bool wide = a.hidden % E == 0;
    for (const Rows* r : {&a.x, &a.y, &a.gate, &a.h, &a.n, &a.dn, &a.dh, &a.dx, &a.dy, &a.dgate, &a.weight, &a.post}) {
        const bool residual = r == &a.x || r == &a.h || r == &a.dh || r == &a.dx;
        const int size = residual ? rs : es;
        if ((uintptr_t)r->p % size != 0) return C3_E_ALIGN;
        wide = wide && (uintptr_t)r->p % 16 == 0 && (r->stride * size) % 16 == 0;
    }
    hipError_t e;
    if (c->dtype == C3_F32)
        e = by_kind<float, float>(a, grad, wide, s);
    else if (c->dtype == C3_BF16)
        e = c->residual == C3_F32 ? by_kind<float, __bf16>(a, grad, wide, s) : by_kind<__bf16, __bf16>(a, grad, wide, s);
    else
        e = c->residual == C3_F32 ? by_kind<float, _Float16>(a, grad, wide, s)
                                  : by_kind<_Float16, _Float16>(a, grad, wide, s);
    return e == hipSuccess ? C3_OK : C3_E_HIP;
}

int check_sizes(const c3_residual_norm_t* a) {
    if (a == nullptr || a->tokens < 0 || a->tokens >= (1ll << 31) || a->hidden < 1 || a->gate < C3_GATE_NONE ||
        a->gate > C3_GATE_TOKENS || !(a->scale - a->scale == 0.0f) || !(a->eps >= 0.0f) || a->eps - a->eps != 0.0f)
        return C3_E_INVAL;
    if (replay_elem_size(a->dtype) == 0 || (a->residual != a->dtype && a->residual != C3_F32) ||
        a->hidden > C3_MAX_NORM_HIDDEN)
        return C3_E_UNSUPPORTED;
    return C3_OK;
}

// Rows that have to be there, or those that may be missing.
bool take(const c3_residual_norm_t* a, const c3_rows_t* r, bool needed, Rows* to) {
    *to = Rows{nullptr, 0};
    if (r == nullptr || r->ptr == nullptr) return !needed;
    if (a->tokens > 1 && r->stride < a->hidden) return false;
    // the stride of a single row says nothing
    *to = Rows{static_cast<char*>(r->ptr), a->tokens > 1 ? r->stride : 0};
    return true;
}
bool take_gate(const c3_residual_norm_t* a, const c3_rows_t* r, Rows* to) {
    if (a->gate == C3_GATE_TOKENS) return take(a, r, true, to);
    *to = Rows{nullptr, 0};
    if (a->gate == C3_GATE_NONE) return true;
    if (r == nullptr || r->ptr == nullptr) return false;
    to->p = static_cast<char*>(r->ptr);
    return true;
}

// Results that start where another tensor does, but for the pairs that may.
bool clash(const Rows& out, std::initializer_list<const Rows*> others, const Rows* may) {
    if (out.p == nullptr) return false;
    for (const Rows* o : others)
        if (o->p == out.p && !(o == may && o->stride == out.stride)) return true;
    return false;
}

}  // namespace
}  // namespace c3

extern "C" {

int c3_residual_norm(const c3_residual_norm_t* a, const c3_rows_t* x, const c3_rows_t* y, const c3_rows_t* gate,
                     const void* weight, const void* post, const c3_rows_t* h, const c3_rows_t* n, float* stats,
                     c3_stream_t stream) {
    using namespace c3;
    const int rc = check_sizes(a);
    if (rc != C3_OK || a->tokens == 0) return rc;
    NormArgs k{};
    if (weight == nullptr || stats == nullptr || !take(a, x, true, &k.x) || !take(a, y, false, &k.y) ||
        !take(a, h, k.y.p != nullptr, &k.h) || !take(a, n, true, &k.n))
        return C3_E_INVAL;
    if (k.y.p == nullptr) {
        if (post != nullptr || a->gate != C3_GATE_NONE) return C3_E_INVAL;
        k.h = Rows{nullptr, 0};             // h = x
    } else if (!take_gate(a, gate, &k.gate)) {
        return C3_E_INVAL;
    }
    k.weight.p = static_cast<char*>(const_cast<void*>(weight));
    k.post.p = static_cast<char*>(const_cast<void*>(post));
    if (clash(k.h, {&k.x, &k.y, &k.gate, &k.weight, &k.post}, &k.x) ||
        clash(k.n, {&k.x, &k.y, &k.gate, &k.weight, &k.post, &k.h}, nullptr))
        return C3_E_INVAL;
    if ((uintptr_t)stats % 8 != 0) return C3_E_ALIGN;
    k.stats = stats;
    return by_type(a, k, false, reinterpret_cast<hipStream_t>(stream));
}

size_t c3_residual_norm_grad_workspace_size(const c3_residual_norm_t* a) {
    using namespace c3;
    if (check_sizes(a) != C3_OK) return 0;
    const size_t n = 3 * sizeof(float) * (size_t)(grad_groups(a->tokens, a->hidden) * a->hidden);
    return n < 256 ? 256 : (n + 255) / 256 * 256;
}

int c3_residual_norm_grad(const c3_residual_norm_t* a, const c3_rows_t* dn, const c3_rows_t* dh, const c3_rows_t* x,
                          const c3_rows_t* y, const c3_rows_t* gate, const void* weight, const void* post,
                          const float* stats, const c3_rows_t* dx, const c3_rows_t* dy, const c3_rows_t* dgate,
                          float* sums, void* ws, size_t ws_bytes, c3_stream_t stream) {
    using namespace c3;
    const int rc = check_sizes(a);
    if (rc != C3_OK) return rc;
    if (weight == nullptr || sums == nullptr) return C3_E_INVAL;
    if ((uintptr_t)sums % 4 != 0) return C3_E_ALIGN;
    if (ws == nullptr || (uintptr_t)ws % 256 != 0 || ws_bytes < c3_residual_norm_grad_workspace_size(a))
        return C3_E_WORKSPACE;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (a->tokens == 0) {                   // sums over nothing
        const int kinds = 1 | (post != nullptr ? 2 : 0) | (a->gate == C3_GATE_CHANNELS ? 4 : 0);
        norm_parts_kernel<<<dim3((unsigned)((a->hidden + 63) / 64), 3), dim3(1024), 0, s>>>(
            static_cast<float*>(ws), 0, (int)a->hidden, kinds, sums);
        return hipGetLastError() == hipSuccess ? C3_OK : C3_E_HIP;
    }
    NormArgs k{};
    if (stats == nullptr || !take(a, dn, true, &k.dn) || !take(a, dh, false, &k.dh) || !take(a, x, true, &k.x) ||
        !take(a, y, false, &k.y) || !take(a, dx, true, &k.dx) || !take(a, dy, k.y.p != nullptr, &k.dy) ||
        !take(a, dgate, k.y.p != nullptr && a->gate == C3_GATE_TOKENS, &k.dgate))
        return C3_E_INVAL;
    if (a->gate != C3_GATE_TOKENS) k.dgate = Rows{nullptr, 0};
    if (k.y.p == nullptr) {
        if (post != nullptr || a->gate != C3_GATE_NONE) return C3_E_INVAL;
        k.dy = Rows{nullptr, 0};
    } else if (!take_gate(a, gate, &k.gate)) {
        return C3_E_INVAL;
    }
    k.weight.p = static_cast<char*>(const_cast<void*>(weight));
    k.post.p = static_cast<char*>(const_cast<void*>(post));
    if (clash(k.dx, {&k.dn, &k.dh, &k.x, &k.y, &k.gate, &k.weight, &k.post}, &k.dh) ||
        clash(k.dy, {&k.dn, &k.dh, &k.x, &k.y, &k.gate, &k.weight, &k.post, &k.dx}, &k.dn) ||
        clash(k.dgate, {&k.dn, &k.dh, &k.x, &k.y, &k.gate, &k.weight, &k.post, &k.dx, &k.dy}, nullptr))
        return C3_E_INVAL;
    if ((uintptr_t)stats % 8 != 0) return C3_E_ALIGN;
    k.stats = const_cast<float*>(stats);
    k.sums = sums;
    k.parts = static_cast<float*>(ws);
    k.groups = grad_groups(a->tokens, a->hidden);
    return by_type(a, k, true, s);
}

}  // extern "C"
