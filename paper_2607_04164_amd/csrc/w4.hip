// Weights in 4 bits with group scales: the quantizer and the grouped products
// of few rows (see w4.h for the arithmetic).
//
// The products are bound by reading the codes: one workgroup (4 waves) owns a
// segment and 16 output columns, its waves split K by chunks of 128 columns, and
// a segment's rows are taken 64 at a time, so that up to 64 rows share one read
// of the weights. The waves' partial tiles are added through LDS in wave order.
#include "bmoe_common.h"
#include "w4.h"

namespace bmoe {
namespace {

constexpr int kW4Threads = 256;
constexpr int kW4Waves = kW4Threads / 64;
constexpr int kW4Cols = 16;
constexpr int kW4Tiles = 4;  // tiles of 16 rows per pass

struct W4Params {
    const uint16_t* A;  // [rows_cap or a_count, K]
    W4Stack w[2];       // [n_seg, N, K] (gated: W_gate, W_up)
    uint16_t* C;        // [rows_cap, N]
    const int32_t* offsets;
    const int32_t* a_rows;
    int a_count;
    int n_seg, rows_cap, N, K;
};

template <bool GATED, int GROUP>
__global__ __launch_bounds__(kW4Threads, 2) void w4_gemm_kernel(W4Params p) {
    constexpr int NMAT = GATED ? 2 : 1, TILES = kW4Tiles, NG = W4Chunk<GROUP>::NG, STEPS = GROUP / 32;
    __shared__ __align__(16) f32x4 part[kW4Waves][NMAT * TILES][64];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int r16 = lane & 15, q = lane >> 4;
    const int K = p.K, N = p.N;
    const int ncb = ceil_div(N, kW4Cols);
    const int s = blockIdx.x / ncb, n0 = (blockIdx.x % ncb) * kW4Cols;
    const int beg = min(max(p.offsets[s], 0), p.rows_cap);
    const int end = min(max(p.offsets[s + 1], beg), p.rows_cap);
    if (end <= beg) return;
    const W4Rows<GROUP> rows0(p.w[0], (int64_t)s * N + n0, K), rows1(p.w[NMAT - 1], (int64_t)s * N + n0, K);
    const int wrow = min(r16, N - 1 - n0);
    const int nch = ceil_div(K, kW4Chunk);
    const v4u ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};

    for (int m0 = beg; m0 < end; m0 += 16 * TILES) {
        const int tiles = min(ceil_div(end - m0, 16), TILES);
        const uint16_t* xp[TILES];
#pragma unroll
        for (int nt = 0; nt < TILES; ++nt) {
            const int r = min(m0 + nt * 16 + r16, end - 1);
            xp[nt] = p.A + (size_t)gathered_row(p.a_rows, p.a_count, r) * K;
        }
        f32x4 tot[NMAT][TILES];
#pragma unroll
        for (int m = 0; m < NMAT; ++m)
#pragma unroll
            for (int nt = 0; nt < TILES; ++nt) tot[m][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int c = wave; c < nch; c += kW4Waves) {
            W4Chunk<GROUP> w[NMAT];
#pragma unroll
            for (int m = 0; m < NMAT; ++m) w[m].load(m ? rows1 : rows0, wrow, c, K, q);
#pragma unroll
            for (int m = 0; m < NMAT; ++m) w[m].codes = w4_transpose(w[m].codes);
#pragma unroll
            for (int nt = 0; nt < TILES; ++nt) {
                if (nt >= tiles) break;
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    f32x4 acc[NMAT], xs = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int m = 0; m < NMAT; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int u = g * STEPS; u < (g + 1) * STEPS; ++u) {
                        const int col = c * kW4Chunk + u * 32 + q * 8;
                        v4u x = col < K ? *(const v4u*)(xp[nt] + col) : v4u{0, 0, 0, 0};
                        x = w4_order(x);
                        xs = mfma16(x, ones, xs);
#pragma unroll
                        for (int m = 0; m < NMAT; ++m) acc[m] = mfma16(x, w4_unpack(w[m].codes[u]), acc[m]);
                    }
#pragma unroll
                    for (int m = 0; m < NMAT; ++m) {
                        const float sc = w[m].scale(g), off = w[m].offset(p.w[0].has_zeros, g);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            tot[m][nt][i] = fmaf(sc, fmaf(-off, xs[i], acc[m][i]), tot[m][nt][i]);
                    }
                }
            }
        }
#pragma unroll
        for (int nt = 0; nt < TILES; ++nt)
            if (nt < tiles) {
#pragma unroll
                for (int m = 0; m < NMAT; ++m) part[wave][m * TILES + nt][lane] = tot[m][nt];
            }
        __syncthreads();
        // wave nt finishes row tile nt: the lane holds rows 4q .. 4q+3, column r16
        if (wave < tiles && n0 + r16 < N) {
            f32x4 sum[NMAT];
#pragma unroll
            for (int m = 0; m < NMAT; ++m) {
                sum[m] = part[0][m * TILES + wave][lane];
#pragma unroll
                for (int w = 1; w < kW4Waves; ++w) sum[m] += part[w][m * TILES + wave][lane];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = m0 + wave * 16 + 4 * q + i;
                if (row >= end) continue;
                float v;
                if constexpr (GATED) v = silu_mul(sum[0][i], sum[NMAT - 1][i]);
                else v = sum[0][i];
                p.C[(size_t)row * N + n0 + r16] = f32_to_bf16(v);
            }
        }
        __syncthreads();  // the partials are rewritten by the next pass
    }
}

// ---- quantizer: 8 lanes per group of a row, each holding GROUP / 8 columns

template <typename T>
__device__ __forceinline__ float as_f32(T v);
template <>
__device__ __forceinline__ float as_f32<uint16_t>(uint16_t v) { return bf16_to_f32(v); }
template <>
__device__ __forceinline__ float as_f32<float>(float v) { return v; }

template <typename T>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const T* __restrict__ w, uint8_t* __restrict__ codes,
                                                          uint16_t* __restrict__ scales, uint8_t* __restrict__ zeros,
                                                          int64_t rows, int K, int group) {
    const int ng = ceil_div(K, group), per = group / 8, pitch = BMOE_W4_ROW_BYTES(K);
    const int64_t total = rows * ng;
    const int l = threadIdx.x & 7;
    for (int64_t i = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3); i < total; i += (int64_t)gridDim.x * 32) {
        const int64_t row = i / ng;
        const int g = (int)(i % ng);
        const int k0 = g * group + l * per;  // this lane's columns (per is a multiple of 4)
        const T* src = w + row * (int64_t)K;
        float lo = 0.f, hi = 0.f;
        for (int j = 0; j < per; ++j)
            if (k0 + j < K) {
                const float v = as_f32<T>(src[k0 + j]);
                lo = fminf(lo, v);
                hi = fmaxf(hi, v);
            }
#pragma unroll
        for (int off = 4; off; off >>= 1) {
            lo = fminf(lo, __shfl_xor(lo, off));
            hi = fmaxf(hi, __shfl_xor(hi, off));
        }
        const float want = zeros ? (hi - lo) / 15.f : fmaxf(hi, -lo) / 7.f;
        const uint16_t sb = f32_to_bf16(want);
        const float s = bf16_to_f32(sb);
        const bool some = s > 0.f;
        const float zf = !some ? 0.f : rintf(-lo / s);
        const int z = zeros ? (int)fminf(fmaxf(zf, 0.f), 15.f) : 8;
        if (l == 0) {
            scales[i] = sb;
            if (zeros) zeros[i] = (uint8_t)z;
        }
        const int least = zeros ? 0 : 1;
        uint8_t* dst = codes + row * (int64_t)pitch;
        // two columns a byte; the row's last group also writes the padding
        const int stop = g == ng - 1 ? pitch * 2 : min(K, (g + 1) * group);
        for (int j = 0; j < per; j += 2) {
            const int k = k0 + j;
            if (k >= stop) break;
            uint32_t b = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                int c = 8;  // padding
                if (k + h < K) {
                    const float v = as_f32<T>(src[k + h]);
                    const float n = some ? rintf(v / s) : 0.f;
                    c = (int)fminf(fmaxf(n + (float)z, (float)least), 15.f);
                }
                b |= (uint32_t)c << (4 * h);
            }
            dst[k >> 1] = (uint8_t)b;
        }
    }
}

template <bool GATED>
hipError_t launch_w4(const W4Params& p, int group, hipStream_t s) {
    const int64_t blocks = (int64_t)p.n_seg * ceil_div(p.N, kW4Cols);
    if (blocks > kMaxBlocks256) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks), block(kW4Threads);
    if (group == 32) hipLaunchKernelGGL((w4_gemm_kernel<GATED, 32>), grid, block, 0, s, p);
    else if (group == 64) hipLaunchKernelGGL((w4_gemm_kernel<GATED, 64>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((w4_gemm_kernel<GATED, 128>), grid, block, 0, s, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_w4_quantize(const W4QuantizeArgs& a, hipStream_t s) {
    const int64_t rows = (int64_t)a.n * a.N, groups = rows * ceil_div(a.K, a.group);
    const int64_t wgs = ceil_div64(groups, 32);
    const dim3 grid((unsigned)(wgs < (1 << 20) ? wgs : (1 << 20))), block(256);
    if (a.dtype == BMOE_BF16)
        hipLaunchKernelGGL((w4_quantize_kernel<uint16_t>), grid, block, 0, s, (const uint16_t*)a.w, a.codes,
                           (uint16_t*)a.scales, a.zeros, rows, a.K, a.group);
    else
        hipLaunchKernelGGL((w4_quantize_kernel<float>), grid, block, 0, s, (const float*)a.w, a.codes,
                           (uint16_t*)a.scales, a.zeros, rows, a.K, a.group);
    return hipGetLastError();
}

hipError_t launch_w4_gemm(const W4GemmArgs& a, hipStream_t s) {
    auto stack = [&](const bmoe_w4* w) {
        return w ? w4_stack(w->codes, w->scales, w->zeros, (int64_t)a.n_seg * a.N, a.K, w->group) : W4Stack{};
    };
    W4Params p{(const uint16_t*)a.a, {stack(a.w0), stack(a.w1)}, (uint16_t*)a.c, a.offsets, a.a_rows, a.a_count,
               a.n_seg, a.rows_cap, a.N, a.K};
    return a.w1 ? launch_w4<true>(p, a.w0->group, s) : launch_w4<false>(p, a.w0->group, s);
}

}  // namespace bmoe
