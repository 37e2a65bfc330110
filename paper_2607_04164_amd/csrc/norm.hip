// RMS norms around the layer (the residual block that a MoE layer sits in):
//   pre_norm:  out = rms(x) * w
//   post_norm: r = res_scale * x + gate * n, n = rms(y) * w_post or y;
//              a = rms(r) * w_next, from r before it is rounded
// Bound by memory: every row is read once into registers (NT threads a row, CH
// 16-byte chunks a thread), the sums of squares are reduced over the row's
// threads, and the outputs are written from the registers (8192 bf16 rows of 2048 with
// every stream, 168 MB: 35 us, 4.8 TB/s; a copy reaches 4.9). Sums in fp32; a row
// whose squares overflow fp32 is summed again at 2^-100 of its values.
#include <math.h>

#include <type_traits>

#include "bmoe_common.h"
#include "chunk16.h"
#include "stream_io.h"

namespace bmoe {
namespace {

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// sum over the NT threads of a row (every thread gets the same bits)
template <int NT>
__device__ __forceinline__ float row_sum(float v, float* part) {
    v = wave_sum(v);
    if constexpr (NT > 64) {
        constexpr int W = NT / 64;
        __syncthreads();  // the partials of the sum before are read
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = part[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v += part[w];
    }
    return v;
}

// 1 / sqrt(mean of f^2 + eps) of a row. A row whose squares overflow is summed at 2^-100 of
// its values, and left at 2^-4 of them with 2^4 times the result (which would lose bits
// where it is below 2^-126).
template <int NT, int M>
__device__ __forceinline__ float inv_rms(float (&f)[M], int d, float eps, float* part) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < M; ++i) s = fmaf(f[i], f[i], s);
    s = row_sum<NT>(s, part);
    if (!(s <= 3.0e38f)) {  // (the same for every thread of the row)
        s = 0.f;
#pragma unroll
        for (int i = 0; i < M; ++i) {
            s = fmaf(f[i] * 0x1p-100f, f[i] * 0x1p-100f, s);
            f[i] *= 0x1p-4f;
        }
        s = row_sum<NT>(s, part);
        return 0x1p-96f / sqrtf(s / (float)d);
    }
    return 1.f / sqrtf(s / (float)d + eps);
}

template <typename E, int NT, int CH>
__device__ __forceinline__ void load_row(const uint4* row, int c0, int nch, float (&f)[CH * Vec<E>::N]) {
#pragma unroll
    for (int u = 0; u < CH; ++u) {
        const int c = c0 + NT * u;
        Vec<E>::load(c < nch ? row[c] : make_uint4(0, 0, 0, 0), f + u * Vec<E>::N);
    }
}

template <typename E, int NT, int CH>
__device__ __forceinline__ void store_row(uint4* row, int c0, int nch, const float (&f)[CH * Vec<E>::N]) {
#pragma unroll
    for (int u = 0; u < CH; ++u) {
        const int c = c0 + NT * u;
        if (c < nch) store_stream(row + c, Vec<E>::store(f + u * Vec<E>::N));
    }
}

template <int NT>
constexpr int rows_per_wg() { return NT > 256 ? 1 : 256 / NT; }

template <typename E, int NT, int CH>
__global__ __launch_bounds__(NT > 256 ? NT : 256) void pre_norm_kernel(const uint4* x, const uint4* w, uint4* out,
                                                                       int T, int nch, float eps) {
    constexpr int N = Vec<E>::N, R = rows_per_wg<NT>();
    __shared__ float part[NT / 64];
    const int c0 = threadIdx.x % NT;
    for (int64_t t = (int64_t)blockIdx.x * R + threadIdx.x / NT; t < T; t += (int64_t)gridDim.x * R) {
        float f[CH * N], g[CH * N];
        load_row<E, NT, CH>(x + (size_t)t * nch, c0, nch, f);
        if (w) load_row<E, NT, CH>(w, c0, nch, g);
        const float inv = inv_rms<NT>(f, nch * N, eps, part);
#pragma unroll
        for (int i = 0; i < CH * N; ++i) f[i] = w ? f[i] * inv * g[i] : f[i] * inv;
        store_row<E, NT, CH>(out + (size_t)t * nch, c0, nch, f);
    }
}

struct PostParams {
    const uint4 *y, *x, *w_post, *w_next;
    const void* gate;
    uint4 *r, *a;
    int T, nch, norm_y, gate_mode;
    float eps, res_scale;
};

template <typename E, int NT, int CH>
__global__ __launch_bounds__(NT > 256 ? NT : 256) void post_norm_kernel(PostParams p) {
    constexpr int N = Vec<E>::N, R = rows_per_wg<NT>(), M = CH * N;
    __shared__ float part[NT / 64];
    const int c0 = threadIdx.x % NT, nch = p.nch;
    for (int64_t t = (int64_t)blockIdx.x * R + threadIdx.x / NT; t < p.T; t += (int64_t)gridDim.x * R) {
        float n[M], r[M], g[M];
        load_row<E, NT, CH>(p.y + (size_t)t * nch, c0, nch, n);
        load_row<E, NT, CH>(p.x + (size_t)t * nch, c0, nch, r);
        float gt = 1.f;
        const bool wide = p.gate_mode == BMOE_GATE_CHANNEL || p.gate_mode == BMOE_GATE_FULL;
        if (wide)
            load_row<E, NT, CH>((const uint4*)p.gate + (p.gate_mode == BMOE_GATE_FULL ? (size_t)t * nch : 0), c0, nch, g);
        else if (p.gate_mode == BMOE_GATE_TOKEN)
            gt = ((const float*)p.gate)[t];
        if (p.norm_y) {
            const float inv = inv_rms<NT>(n, nch * N, p.eps, part);
            float w[M];
            if (p.w_post) load_row<E, NT, CH>(p.w_post, c0, nch, w);
#pragma unroll
            for (int i = 0; i < M; ++i) n[i] = p.w_post ? n[i] * inv * w[i] : n[i] * inv;
        }
#pragma unroll
        for (int i = 0; i < M; ++i) r[i] = fmaf(wide ? g[i] : gt, n[i], p.res_scale * r[i]);
        store_row<E, NT, CH>(p.r + (size_t)t * nch, c0, nch, r);
        if (p.a) {
            float w[M];
            if (p.w_next) load_row<E, NT, CH>(p.w_next, c0, nch, w);
            const float inv = inv_rms<NT>(r, nch * N, p.eps, part);
#pragma unroll
            for (int i = 0; i < M; ++i) r[i] = p.w_next ? r[i] * inv * w[i] : r[i] * inv;
            store_row<E, NT, CH>(p.a + (size_t)t * nch, c0, nch, r);
        }
    }
}

template <int V>
using Int = std::integral_constant<int, V>;

// f(NT, CH) with the least CH of LEAST, 2 LEAST, .. MOST that holds a thread's chunks
template <int NT, int LEAST, int MOST, typename F>
void with_chunks(int nch, F f) {
    if constexpr (LEAST < MOST) {
        if (nch > NT * LEAST) return with_chunks<NT, 2 * LEAST, MOST>(nch, f);
    }
    f(Int<NT>{}, Int<LEAST>{});
}

// runs f(NT, CH) with the row split that fits: a wave a row where there are rows for
// every wave of the chip and a lane's share of the row is at most WAVE_CHUNKS, else four
// waves; sixteen where a row needs them. WAVE_CHUNKS: 4 for pre_norm, 2 for post_norm,
// which holds three rows; with more, too few waves fit a SIMD to keep its loads going
// (8192 bf16 rows, a wave and four waves a row: pre_norm 6.8 and 10.0 us of 1024
// columns, 11.7 and 13.2 of 2048, 22.7 and 20.5 of 4096; post_norm 17.4 and 24.8, 39.7
// and 34.0, 116.7 and 70.4). Wider rows have no split that keeps both: with four waves
// bf16 post_norm of 8192 columns holds 234 registers (4096 rows with a full gate: 75 us, 4.5
// TB/s, against 5.0 at 4096 columns), of 16384 256 (2048 rows: 114 us, 2.9), and with sixteen
// waves it spills (32768 columns: 385 us, 1.7). pre_norm stays at 5.2 TB/s and more.
template <int WAVE_CHUNKS, int MAX_NCH, typename F>
hipError_t with_split(int64_t T, int nch, F f) {
    if (nch <= 64 || (nch <= 64 * WAVE_CHUNKS && T >= 1024)) with_chunks<64, 1, WAVE_CHUNKS>(nch, f);
    else if (nch <= 2048) with_chunks<256, 1, 8>(nch, f);
    else with_chunks<1024, 4, MAX_NCH / 1024>(nch, f);
    return hipGetLastError();
}

// workgroups: one pass over the rows, or a loop where a launch could not hold them
template <int NT>
unsigned grid_of(int64_t T) {
    const int64_t wgs = ceil_div64(T, rows_per_wg<NT>());
    return (unsigned)(wgs < (1 << 20) ? wgs : (1 << 20));
}

template <typename E>
hipError_t launch_pre_norm_t(const PreNormArgs& a, hipStream_t s) {
    constexpr int N = Vec<E>::N;
    const int nch = a.d / N;
    return with_split<4, BMOE_NORM_MAX_D / N>(a.T, nch, [&](auto nt, auto ch) {
        constexpr int NT = decltype(nt)::value, CH = decltype(ch)::value;
        hipLaunchKernelGGL((pre_norm_kernel<E, NT, CH>), dim3(grid_of<NT>(a.T)), dim3(NT > 256 ? NT : 256), 0, s,
                           (const uint4*)a.x, (const uint4*)a.w, (uint4*)a.out, a.T, nch, a.eps);
    });
}

template <typename E>
hipError_t launch_post_norm_t(const PostNormArgs& a, hipStream_t s) {
    constexpr int N = Vec<E>::N;
    const int nch = a.d / N;
    const PostParams p{(const uint4*)a.y, (const uint4*)a.x, (const uint4*)a.w_post, (const uint4*)a.w_next, a.gate,
                       (uint4*)a.r, (uint4*)a.a, a.T, nch, a.norm_y, a.gate_mode, a.eps, a.res_scale};
    return with_split<2, BMOE_NORM_MAX_D / N>(a.T, nch, [&](auto nt, auto ch) {
        constexpr int NT = decltype(nt)::value, CH = decltype(ch)::value;
        hipLaunchKernelGGL((post_norm_kernel<E, NT, CH>), dim3(grid_of<NT>(a.T)), dim3(NT > 256 ? NT : 256), 0, s, p);
    });
}

}  // namespace

hipError_t launch_pre_norm(const PreNormArgs& a, hipStream_t s) {
    return a.dtype == BMOE_BF16 ? launch_pre_norm_t<uint16_t>(a, s) : launch_pre_norm_t<float>(a, s);
}

hipError_t launch_post_norm(const PostNormArgs& a, hipStream_t s) {
    return a.dtype == BMOE_BF16 ? launch_post_norm_t<uint16_t>(a, s) : launch_post_norm_t<float>(a, s);
}

}  // namespace bmoe
