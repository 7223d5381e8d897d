// Second pass of attention's gradient (c3_attention_dkv.h).
#include "c3_attention_dkv.h"

namespace c3 {
namespace {

// Heads of 64 in fp16: three waves a SIMD (165 registers) make up for the care for dS's
// range, 254 -> 244 us for 2 x 2,048 causal tokens of 32 heads, forward and back.
template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, DP == 64 && kDsScaled<T> ? 3 : 2) void attn_dkv_kernel(AttnArgs a, AttnTable tab) {
    const bool bad = dkv_unit<T, DP, false>(a, tab, blockIdx.x);
    if (a.causal || a.window) {
        const int any = __syncthreads_or(bad);
        if (threadIdx.x == 0) a.side[1].marks[blockIdx.x] = any;
    }
}

template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, 1) void attn_dkv_direct_kernel(AttnArgs a, AttnTable tab) {
    dkv_unit<T, DP, true>(a, tab, blockIdx.x);
}

template <typename T, int DP>
hipError_t launch(const AttnPlan& p, hipStream_t s) {
    const dim3 grid(attn_blocks(p, 1)), block(kAttnThreads);
    if (attn_direct(p, 1))
        attn_dkv_direct_kernel<T, DP><<<grid, block, 0, s>>>(p.args, p.table);
    else
        attn_dkv_kernel<T, DP><<<grid, block, 0, s>>>(p.args, p.table);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_dkv(const AttnPlan& p, bool bf16, hipStream_t s) {
    if (bf16) return p.args.dim > 64 ? launch<__bf16, 128>(p, s) : launch<__bf16, 64>(p, s);
    return p.args.dim > 64 ? launch<_Float16, 128>(p, s) : launch<_Float16, 64>(p, s);
}

}  // namespace c3
