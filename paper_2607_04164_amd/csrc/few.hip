// The few-token layer (see few.h): gate logits, sizes, and the layers of plain weights.
#include "few.h"

namespace bmoe {
namespace {

// ---- gate logits

// TT: tokens of a workgroup. A thread takes every 256th 16-byte chunk of the expert's row. The
// first workgroup also clears the counters of few_down_kernel.
template <typename Act, int TT>
__global__ __launch_bounds__(kLogitThreads) void few_logits_kernel(const uint4* __restrict__ x,
                                                                   const uint4* __restrict__ w,
                                                                   const float* __restrict__ bias,
                                                                   double* __restrict__ logits, int T, int E, int nch,
                                                                   int32_t* __restrict__ done, int tiles) {
    constexpr int N = Vec<Act>::N;
    __shared__ double red[TT][kLogitThreads];
    const int tid = threadIdx.x, e = blockIdx.x, t0 = blockIdx.y * TT;
    if (e == 0 && t0 == 0)
        for (int i = tid; i < tiles; i += kLogitThreads) done[i] = 0;
    double acc[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[t] = 0.0;
    for (int c = tid; c < nch; c += kLogitThreads) {
        const uint4 wv = w[(size_t)e * nch + c];
        uint4 xv[TT];
#pragma unroll
        for (int t = 0; t < TT; ++t) xv[t] = x[(size_t)min(t0 + t, T - 1) * nch + c];
        float wf[N];
        Vec<Act>::load(wv, wf);
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            float xf[N];
            Vec<Act>::load(xv[t], xf);
#pragma unroll
            for (int j = 0; j < N; ++j) acc[t] = fma((double)xf[j], (double)wf[j], acc[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) red[t][tid] = acc[t];
    __syncthreads();
    const int t = tid >> 4, s = tid & 15;
    if (t < TT) {
        double v = 0.0;
        for (int j = 0; j < kLogitThreads / 16; ++j) v += red[t][s + 16 * j];
        v = group_sum<16>(v);
        if (s == 0 && t0 + t < T) logits[(t0 + t) * E + e] = v + (bias ? (double)bias[e] : 0.0);
    }
}

template <typename Act>
hipError_t launch_logits(const FewArgs& a, int32_t* done, hipStream_t s) {
    const int nch = a.d / Vec<Act>::N, tiles = ceil_div(a.d, kFewCols);
    auto go = [&](auto kernel, int tokens) {
        hipLaunchKernelGGL(kernel, dim3(a.E, ceil_div(a.T, tokens)), dim3(kLogitThreads), 0, s, (const uint4*)a.x,
                           (const uint4*)a.w.w_router, a.w.bias, (double*)a.ws, a.T, a.E, nch, done, tiles);
    };
    if (a.T == 1) go(few_logits_kernel<Act, 1>, 1);
    else if (a.T == 2) go(few_logits_kernel<Act, 2>, 2);
    else go(few_logits_kernel<Act, kLogitTokens>, kLogitTokens);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_few_logits(const FewArgs& a, int32_t* done, hipStream_t s) {
    return a.dtype == BMOE_BF16 ? launch_logits<uint16_t>(a, done, s) : launch_logits<float>(a, done, s);
}

size_t few_ws_bytes(int T, int E, int k, int d, int f, int fs) {
    return logit_bytes(T, E) + done_bytes(d) + partial_bytes(d) + ((size_t)T * k * f + (size_t)T * fs) * 4;
}

hipError_t launch_few(const FewArgs& a, hipStream_t s) {
    if (a.w.group) return launch_few_w4(a, s);
    if (a.dtype == BMOE_BF16)
        return launch_few_t<FmtBf16>(
            a, [](const bmoe_matrix& m, int64_t, int) { return FmtBf16::Stack{(const uint16_t*)m.w, false}; }, s);
    return launch_few_t<FmtF32>(
        a, [](const bmoe_matrix& m, int64_t, int) { return FmtF32::Stack{(const float*)m.w, false}; }, s);
}

}  // namespace bmoe
