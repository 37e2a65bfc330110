// Weights in 4 bits with group scales: the quantizer and the grouped products
// of few rows (see w4.h for the arithmetic).
//
// One workgroup (8 waves) takes up to 32 rows of a segment (a pass) and 16 output
// columns; its waves split K by units of 256 columns. The passes of a segment run side
// by side: a loop over them inside a workgroup would make the longest segment's time
// the kernel's. Their weights meet in the L2 cache (column blocks of a multiple of 8
// keep them on one XCD). A wave loads WB units of weights, then takes their
// columns step by step; the activations of the next XS steps (from the L2 cache) are
// loaded while these are multiplied. The waves' partial tiles are added through LDS
// in wave order.
#include "bmoe_common.h"
#include "w4.h"

namespace bmoe {
namespace {

constexpr int kW4Threads = 512;
constexpr int kW4Waves = kW4Threads / 64;
constexpr int kW4Cols = 16;
constexpr int kW4Tiles = 2;  // tiles of 16 rows per pass

struct W4Params {
    const uint16_t* A;  // [rows_cap or a_count, K]
    W4Stack w[2];       // [n_seg, N, K] (gated: W_gate, W_up)
    uint16_t* C;        // [rows_cap, N]
    const int32_t* offsets;
    const int32_t* a_rows;
    int a_count;
    int n_seg, rows_cap, N, K;
};

// One pass: rows m0 .. m0 + 16 * TILES - 1 (fewer: the segment's last), this wave's
// units. RAGGED: K is not whole units; WB > 1 needs units that go evenly over the waves.
template <bool GATED, int GROUP, int TILES, int WB, bool RAGGED>
__device__ __forceinline__ void w4_pass(const W4Params& p, const W4Rows<GROUP>& rows0, const W4Rows<GROUP>& rows1, int wrow,
                                        int m0, int end, int wave, int r16, int q, f32x4 (*part)[64]) {
    constexpr int NMAT = GATED ? 2 : 1, GS = GROUP / 32;
    constexpr int XS = 4 / TILES, NX = WB * 8 / XS;
    const int K = p.K, units = ceil_div(K, kW4Unit);
    const v4u ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
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
    for (int u0 = wave; u0 < units; u0 += kW4Waves * WB) {
        v4u x[2][XS][TILES];
        auto load_x = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < XS; ++j) {
                const int step = i * XS + j;
                int col = (u0 + kW4Waves * (step / 8)) * kW4Unit + (step % 8) * 32 + q * 8;
                if constexpr (RAGGED) col = min(col, K - 8);
#pragma unroll
                for (int nt = 0; nt < TILES; ++nt) x[i & 1][j][nt] = *(const v4u*)(xp[nt] + col);
            }
        };
        load_x(0);
        W4Unit<GROUP> w[WB][NMAT];
#pragma unroll
        for (int b = 0; b < WB; ++b)
#pragma unroll
            for (int m = 0; m < NMAT; ++m) w[b][m].load(m ? rows1 : rows0, wrow, u0 + kW4Waves * b, K, q);
        f32x4 acc[NMAT][TILES], xs[TILES];
        v4u c[NMAT];
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (i + 1 < NX) load_x(i + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < XS; ++j) {
                const int step = i * XS + j, b = step / 8, s8 = step % 8, g = s8 / GS;
                if (s8 == 0 && RAGGED) {
#pragma unroll
                    for (int m = 0; m < NMAT; ++m) w[b][m].settle();
                }
                if (s8 % 4 == 0) {
#pragma unroll
                    for (int m = 0; m < NMAT; ++m) c[m] = w4_transpose(w[b][m].codes[s8 / 4]);
                }
                if (s8 % GS == 0) {
#pragma unroll
                    for (int nt = 0; nt < TILES; ++nt) {
                        xs[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int m = 0; m < NMAT; ++m) acc[m][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
                    }
                }
                v4u wv[NMAT];
#pragma unroll
                for (int m = 0; m < NMAT; ++m) wv[m] = w4_unpack(c[m][s8 % 4]);
#pragma unroll
                for (int nt = 0; nt < TILES; ++nt) {
                    v4u xv = x[i & 1][j][nt];
                    if constexpr (RAGGED) xv &= (u0 + kW4Waves * b) * kW4Unit + s8 * 32 + q * 8 < K ? ~0u : 0u;
                    xv = w4_order(xv);
                    xs[nt] = mfma16(xv, ones, xs[nt]);
#pragma unroll
                    for (int m = 0; m < NMAT; ++m) acc[m][nt] = mfma16(xv, wv[m], acc[m][nt]);
                }
                if (s8 % GS == GS - 1) {
#pragma unroll
                    for (int m = 0; m < NMAT; ++m) {
                        const float sc = w[b][m].scale(g), off = w[b][m].offset(p.w[0].has_zeros, g);
#pragma unroll
                        for (int nt = 0; nt < TILES; ++nt) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                tot[m][nt][e] = fmaf(sc, fmaf(-off, xs[nt][e], acc[m][nt][e]), tot[m][nt][e]);
                            asm volatile("" : "+v"(tot[m][nt]));  // here, and not where tot is used next
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);  // (registers: no step runs ahead of the one before)
            }
        }
    }
    const int lane = r16 + 16 * q;
#pragma unroll
    for (int nt = 0; nt < TILES; ++nt)
#pragma unroll
        for (int m = 0; m < NMAT; ++m) part[(wave * kW4Tiles + nt) * NMAT + m][lane] = tot[m][nt];
}

// Finds pass `at` of all segments' passes: its segment and its place among them, or
// returns the number of passes there are (`at` then past them). One wave's work, the
// same in every wave.
__device__ __forceinline__ int find_pass(const int32_t* offsets, int n_seg, int rows_cap, int at, int lane, int* seg,
                                         int* nth) {
    int before = 0;
    for (int base = 0; base < n_seg; base += 64) {
        int passes = 0;
        if (base + lane < n_seg) {
            const int beg = min(max(offsets[base + lane], 0), rows_cap);
            const int end = min(max(offsets[base + lane + 1], beg), rows_cap);
            passes = ceil_div(end - beg, 16 * kW4Tiles);
        }
        int upto = passes;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int v = __shfl_up(upto, off);
            if (lane >= off) upto += v;
        }
        const unsigned long long past = __ballot(before + upto > at);
        if (past) {
            const int l = __ffsll(past) - 1;
            *seg = __builtin_amdgcn_readfirstlane(base + l);
            *nth = __builtin_amdgcn_readfirstlane(at - before - __shfl(upto - passes, l));
            return -1;
        }
        before += __builtin_amdgcn_readfirstlane(__shfl(upto, 63));
    }
    return before;
}

template <bool GATED, int GROUP, bool RAGGED>
__global__ __launch_bounds__(kW4Threads, 4) void w4_gemm_kernel(W4Params p) {
    constexpr int NMAT = GATED ? 2 : 1;
    __shared__ __align__(16) f32x4 part[kW4Waves * kW4Tiles * NMAT][64];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int r16 = lane & 15, q = lane >> 4;
    const int K = p.K, N = p.N;
    const int ncb = ceil_div(N, kW4Cols);
    for (int64_t at = blockIdx.x;; at += gridDim.x) {  // (a launch that holds all of them makes one turn)
        const int pass = __builtin_amdgcn_readfirstlane((int)(at / ncb));
        int s, nth;
        if (find_pass(p.offsets, p.n_seg, p.rows_cap, pass, lane, &s, &nth) >= 0) return;
        const int n0 = __builtin_amdgcn_readfirstlane((int)(at - (int64_t)pass * ncb)) * kW4Cols;
        const int beg = min(max(p.offsets[s], 0), p.rows_cap);
        const int end = min(max(p.offsets[s + 1], beg), p.rows_cap);
        const W4Rows<GROUP> rows0(p.w[0], (int64_t)s * N + n0, K), rows1(p.w[NMAT - 1], (int64_t)s * N + n0, K);
        const int wrow = min(r16, N - 1 - n0);
        const int m0 = beg + nth * 16 * kW4Tiles, rows = min(end - m0, 16 * kW4Tiles);
        if (rows > 16) w4_pass<GATED, GROUP, 2, 1, RAGGED>(p, rows0, rows1, wrow, m0, end, wave, r16, q, part);
        else if (!RAGGED && K % (kW4Unit * kW4Waves * 2) == 0)
            w4_pass<GATED, GROUP, 1, 2, false>(p, rows0, rows1, wrow, m0, end, wave, r16, q, part);
        else w4_pass<GATED, GROUP, 1, 1, RAGGED>(p, rows0, rows1, wrow, m0, end, wave, r16, q, part);
        __syncthreads();
        // a thread per output of the pass
        const int row = tid >> 4, col = tid & 15, nt = row >> 4;
        if (row < rows && n0 + col < N) {
            const float* d = (const float*)&part[nt * NMAT][((row & 15) >> 2) * 16 + col] + (row & 3);
            float sum[NMAT];
#pragma unroll
            for (int m = 0; m < NMAT; ++m) {
                sum[m] = d[m * 256];
#pragma unroll
                for (int w = 1; w < kW4Waves; ++w) sum[m] += d[(w * kW4Tiles * NMAT + m) * 256];
            }
            float v;
            if constexpr (GATED) v = silu_mul(sum[0], sum[NMAT - 1]);
            else v = sum[0];
            p.C[(size_t)(m0 + row) * N + n0 + col] = f32_to_bf16(v);
        }
        __syncthreads();  // the partials are rewritten by the next turn
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
    // passes: at most one for 32 rows, and one more for the rest of each segment's rows
    const int64_t passes = (int64_t)p.rows_cap / (16 * kW4Tiles) + (p.n_seg < p.rows_cap ? p.n_seg : p.rows_cap);
    const int64_t blocks = passes * ceil_div(p.N, kW4Cols), room = (int64_t)1 << 22;
    const dim3 grid((unsigned)(blocks < room ? blocks : room)), block(kW4Threads);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, p); };
    const bool ragged = p.K % kW4Unit != 0;
    if (group == 32) ragged ? go(w4_gemm_kernel<GATED, 32, true>) : go(w4_gemm_kernel<GATED, 32, false>);
    else if (group == 64) ragged ? go(w4_gemm_kernel<GATED, 64, true>) : go(w4_gemm_kernel<GATED, 64, false>);
    else ragged ? go(w4_gemm_kernel<GATED, 128, true>) : go(w4_gemm_kernel<GATED, 128, false>);
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
