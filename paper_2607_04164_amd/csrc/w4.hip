// Weights in 4 bits with group scales: the quantizer and the grouped products
// of few rows (see w4.h for the arithmetic).
//
// One workgroup takes up to 32 rows of a segment (a pass) and four tiles of 16 weight
// rows: 32 columns of a gated product (both matrices), 64 of a plain one. Its waves
// split K by units of 256 columns. The passes of a segment run side by side: a loop over
// them inside a workgroup would make the longest segment's time the kernel's. Their
// weights meet in the L2 cache (column blocks of a multiple of 8 keep them on one XCD).
// A wave loads a unit of weights, then takes its columns step by step; the activations
// of the next steps (from the L2 cache) are loaded while these are multiplied. The
// waves' partial tiles are added through LDS in wave order.
//
// Bound by latency: a workgroup takes about 10 us (its segment 1, the first loads 3,
// products 3.3, sums and stores 2.5), one of them a CU by registers. 250 rows of 8
// segments, gate and up 1408 x 2048, down 2048 x 1408, groups of 32: 24 + 15 us for
// 43 MB; 1000 rows of 32 segments of 2048 x 2048: 50 us for 82 MB. Workgroups that stay
// and load the next item's first unit before they add this one's partials need all 256
// registers: 44 us for the second, but 39.2 against 37.4 for the first. Every pass unpacks
// its weights again, so long segments cost by their rows: a layer of 64 tokens (60 experts,
// top-4, 15 segments, d 2048, d_ff 1408) takes 57 us, 68 with bf16 weights; of 256 tokens
// 116 and 114, of 4096 1162 and 324.
// The FFN's h is rounded to bf16 and y is formed from the rounded h, as in the FFN of bf16
// weights: h is an output that the caller may read, or hand to the down product itself, and
// the two products stay one pass each. Against the unrounded h this costs 0.0024 instead of
// 0.0017 of error relative to y's size.
#include <type_traits>

#include "bmoe_common.h"
#include "chunk16.h"
#include "w4.h"

namespace bmoe {
namespace {

constexpr int kW4Tiles = 2;  // tiles of 16 rows per pass
constexpr int kW4Rows = 16 * kW4Tiles;
constexpr int w4_waves(int mt) { return mt == 1 ? 16 : 8; }  // per workgroup

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
// units. RAGGED: K is not whole units.
template <int NR, int MT, int GROUP, int TILES, bool RAGGED>
__device__ __forceinline__ void w4_pass(const W4Params& p, const W4Place<GROUP, NR, MT>& place, int m0, int end, int wave,
                                        int r16, int q, f32x4 (*part)[64]) {
    constexpr int GS = GROUP / 32, XS = 4 / TILES, NX = 8 / XS;
    const int K = p.K, units = ceil_div(K, kW4Unit);
    const v4u ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
    int row[TILES];  // (gathered while the first weights are loaded)
#pragma unroll
    for (int nt = 0; nt < TILES; ++nt) row[nt] = gathered_row(p.a_rows, p.a_count, min(m0 + nt * 16 + r16, end - 1));
    f32x4 tot[MT][TILES];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int nt = 0; nt < TILES; ++nt) tot[m][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int unit = wave; unit < units; unit += w4_waves(MT)) {
        v4u x[2][XS][TILES];
        auto load_x = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < XS; ++j) {
                int col = unit * kW4Unit + (i * XS + j) * 32 + q * 8;
                if constexpr (RAGGED) col = min(col, K - 8);
#pragma unroll
                for (int nt = 0; nt < TILES; ++nt) x[i & 1][j][nt] = *(const v4u*)(p.A + (size_t)row[nt] * K + col);
            }
        };
        W4Unit<GROUP, MT> w;
        w.load(place, unit, K, q);
        __builtin_amdgcn_sched_barrier(0);
        load_x(0);
        load_x(1);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (RAGGED) w.settle(unit * kW4Unit, K);
        const W4Spread<GROUP, MT> groups(w, p.w[0].has_zeros);
        f32x4 acc[MT][TILES], xs[TILES];
        float xa[TILES];  // xs of group 4i + q
#pragma unroll
        for (int nt = 0; nt < TILES; ++nt) xa[nt] = 0.f;
        v4u c[MT];
#pragma unroll
        for (int i = 0; i < NX; ++i) {
#pragma unroll
            for (int j = 0; j < XS; ++j) {
                const int step = i * XS + j, g = step / GS;
                if (step % 4 == 0) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) c[m] = w4_transpose(w.codes[m][step / 4]);
                }
                if (step % GS == 0) {
#pragma unroll
                    for (int nt = 0; nt < TILES; ++nt) {
                        xs[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int m = 0; m < MT; ++m) acc[m][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
                    }
                }
                v4u xv[TILES];
#pragma unroll
                for (int nt = 0; nt < TILES; ++nt) {
                    xv[nt] = x[i & 1][j][nt];
                    if constexpr (RAGGED) xv[nt] &= unit * kW4Unit + step * 32 + q * 8 < K ? ~0u : 0u;
                    xv[nt] = w4_order(xv[nt]);
                    xs[nt] = mfma16(ones, xv[nt], xs[nt]);
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const v4u wv = w4_unpack(c[m][step % 4]);
#pragma unroll
                    for (int nt = 0; nt < TILES; ++nt) acc[m][nt] = mfma16(xv[nt], wv, acc[m][nt]);
                }
                if (step % GS == GS - 1) {
#pragma unroll
                    for (int nt = 0; nt < TILES; ++nt) xa[nt] = q == (g & 3) ? xs[nt][0] : xa[nt];
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        const float sc = groups.scale(m, g);
#pragma unroll
                        for (int nt = 0; nt < TILES; ++nt) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) tot[m][nt][e] = fmaf(sc, acc[m][nt][e], tot[m][nt][e]);
                            if (g % 4 == 3 || step == 7) tot[m][nt] = groups.add_offset(tot[m][nt], xa[nt], m, g);
                            asm volatile("" : "+v"(tot[m][nt]));  // here, and not where tot is used next
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);  // (registers: no step runs ahead of the one before)
            }
            if (i + 2 < NX) load_x(i + 2);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    const int lane = r16 + 16 * q;
#pragma unroll
    for (int nt = 0; nt < TILES; ++nt)
#pragma unroll
        for (int m = 0; m < MT; ++m) part[(wave * kW4Tiles + nt) * MT + m][lane] = tot[m][nt];
}

// inclusive sum over the lanes of a wave
__device__ __forceinline__ int wave_prefix(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // lane 15 to row 1, lane 47 to row 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2 and 3
    return v;
}

struct W4Pass {
    int seg, beg, end;  // the pass's rows; seg -1: there are fewer passes
};
// Pass `at` of all segments' passes. One wave's work, the same in every wave.
__device__ __forceinline__ W4Pass find_pass(const int32_t* offsets, int n_seg, int rows_cap, int at, int lane) {
    int before = 0;
    for (int base = 0; base < n_seg; base += 64) {
        const int s = min(base + lane, n_seg - 1);
        const int beg = min(max(offsets[s], 0), rows_cap), end = min(max(offsets[s + 1], beg), rows_cap);
        const int passes = base + lane < n_seg ? ceil_div(end - beg, kW4Rows) : 0;
        const int upto = before + wave_prefix(passes);
        const unsigned long long past = __ballot(upto > at);
        if (past) {
            const int l = __ffsll(past) - 1;
            const int nth = at - __builtin_amdgcn_readlane(upto - passes, l);
            const int from = __builtin_amdgcn_readlane(beg, l) + nth * kW4Rows, last = __builtin_amdgcn_readlane(end, l);
            return {base + l, from, min(from + kW4Rows, last)};
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return {-1, 0, 0};
}

template <int NR, int MT, int GROUP, bool RAGGED>
__global__ __launch_bounds__(64 * w4_waves(MT), w4_waves(MT) / 4) void w4_gemm_kernel(W4Params p) {
    constexpr int WAVES = w4_waves(MT), COLS = 16 * MT / NR;
    __shared__ __align__(16) f32x4 part[WAVES * kW4Tiles * MT][64];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int r16 = lane & 15, q = lane >> 4;
    const int K = p.K, N = p.N;
    for (int pass = blockIdx.y;; pass += gridDim.y) {  // (a launch that holds all of them makes one turn)
        const W4Pass at = find_pass(p.offsets, p.n_seg, p.rows_cap, pass, lane);
        if (at.seg < 0) return;
        const int n0 = blockIdx.x * COLS, rows = at.end - at.beg;
        W4Place<GROUP, NR, MT> place;
        place.set(p.w[0], p.w[NR - 1], (int64_t)at.seg * N + n0, N - n0, K, r16, q);
        if (rows > 16) w4_pass<NR, MT, GROUP, 2, RAGGED>(p, place, at.beg, at.end, wave, r16, q, part);
        else w4_pass<NR, MT, GROUP, 1, RAGGED>(p, place, at.beg, at.end, wave, r16, q, part);
        __syncthreads();
        // a thread: one lane's four rows of a tile of each matrix
        for (int i = tid; i < kW4Tiles * MT / NR * 64; i += 64 * WAVES) {
            const int l = i & 63, t = (i >> 6) % (MT / NR), nt = (i >> 6) / (MT / NR);
            const int row = nt * 16 + (l >> 4) * 4, col = n0 + t * 16 + (l & 15);
            if (row >= rows || col >= N) continue;
            f32x4 sum[NR];
#pragma unroll
            for (int m = 0; m < NR; ++m) {
                const f32x4* d = &part[nt * MT + t * NR + m][l];
                sum[m] = d[0];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) sum[m] += d[w * kW4Tiles * MT * 64];
            }
            unsigned again = 0;  // rows whose result is not finite
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = NR == 2 ? silu_mul(sum[0][e], sum[NR - 1][e]) : sum[0][e];
                again |= isfinite(v) ? 0u : 1u << e;
                if (row + e < rows) p.C[(size_t)(at.beg + row + e) * N + col] = f32_to_bf16(v);
            }
            for (; __builtin_expect(again != 0, 0); again &= again - 1) {
                const int r = at.beg + row + __ffs(again) - 1;
                if (r >= at.end) break;
                const uint4* x = (const uint4*)(p.A + (size_t)gathered_row(p.a_rows, p.a_count, r) * K);
                auto load = [&](int k, float* f) { Vec<uint16_t>::load(x[k / 8], f); };
                float v = (float)w4_defined<GROUP>(p.w[0], (int64_t)at.seg * N + col, K, load);
                if constexpr (NR == 2) v = silu_mul(v, (float)w4_defined<GROUP>(p.w[1], (int64_t)at.seg * N + col, K, load));
                p.C[(size_t)r * N + col] = f32_to_bf16(v);
            }
        }
        __syncthreads();  // the partials are rewritten by the next turn
    }
}

// ---- quantizer: 8 lanes per group of a row, each holding PER = group / 8 columns in
// registers, loaded 4 at a time (K is a multiple of 8, so four columns are inside a row or
// past it together). Bound by memory: 15 matrices of 1408 x 2048 take 30 us from bf16 with
// groups of 128 (108 MB, 3.6 TB/s), 48 with groups of 32 (a lane stores 2 bytes), 44 and 49
// from fp32 (195 MB).

template <typename T>
__device__ __forceinline__ void load4(const T* p, float (&f)[4]);
template <>
__device__ __forceinline__ void load4<uint16_t>(const uint16_t* p, float (&f)[4]) {
    const uint2 v = *(const uint2*)p;
    f[0] = __uint_as_float(v.x << 16);
    f[1] = __uint_as_float(v.x & 0xffff0000u);
    f[2] = __uint_as_float(v.y << 16);
    f[3] = __uint_as_float(v.y & 0xffff0000u);
}
template <>
__device__ __forceinline__ void load4<float>(const float* p, float (&f)[4]) {
    const float4 v = *(const float4*)p;
    f[0] = v.x;
    f[1] = v.y;
    f[2] = v.z;
    f[3] = v.w;
}

template <typename T, int PER>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const T* __restrict__ w, uint8_t* __restrict__ codes,
                                                          uint16_t* __restrict__ scales, uint8_t* __restrict__ zeros,
                                                          int64_t rows, int K) {
    constexpr int GROUP = 8 * PER;
    const int ng = ceil_div(K, GROUP), pitch = BMOE_W4_ROW_BYTES(K);
    const int64_t total = rows * ng;
    const int l = threadIdx.x & 7;
    for (int64_t i = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3); i < total; i += (int64_t)gridDim.x * 32) {
        const int64_t row = i / ng;
        const int g = (int)(i - row * ng);
        const int k0 = g * GROUP + l * PER;  // this lane's columns
        const T* src = w + row * (int64_t)K;
        float f[PER / 4][4];
        float lo = 0.f, hi = 0.f, odd = 0.f;  // odd: NaN once a value is not finite
#pragma unroll
        for (int c = 0; c < PER / 4; ++c) {
            load4<T>(src + min(k0 + 4 * c, K - 4), f[c]);
            if (k0 + 4 * c < K) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    lo = fminf(lo, f[c][j]);
                    hi = fmaxf(hi, f[c][j]);
                    odd = fmaf(f[c][j], 0.f, odd);
                }
            }
        }
        hi = isnan(odd) ? INFINITY : hi;  // (neither minimum nor maximum keeps a NaN)
#pragma unroll
        for (int off = 4; off; off >>= 1) {
            lo = fminf(lo, __shfl_xor(lo, off));
            hi = fmaxf(hi, __shfl_xor(hi, off));
        }
        float want = zeros ? (hi - lo) / 15.f : fmaxf(hi, -lo) / 7.f;
        // infinite with finite values: zeros, and the range is past the largest value
        if (__builtin_expect(isinf(want), 0)) want = isinf(fmaxf(hi, -lo)) ? NAN : (0.5f * hi - 0.5f * lo) / 7.5f;
        const uint16_t sb = f32_to_bf16(want);
        const float s = bf16_to_f32(sb);
        const bool some = s > 0.f;
        const float zf = !some ? 0.f : rintf(-lo / s);
        const int z = zeros ? (int)fminf(fmaxf(zf, 0.f), 15.f) : 8;
        if (l == 0) {
            scales[i] = sb;
            if (zeros) zeros[i] = (uint8_t)z;
        }
        const float least = zeros ? 0.f : 1.f;
        uint16_t packed[PER / 4];
#pragma unroll
        for (int c = 0; c < PER / 4; ++c) {
            uint32_t b = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float n = some ? rintf(f[c][j] / s) : 0.f;
                b |= (uint32_t)fminf(fmaxf(n + (float)z, least), 15.f) << (4 * j);
            }
            packed[c] = (uint16_t)(k0 + 4 * c < K ? b : 0x8888u);  // (padding)
        }
        // (rows of codes are whole multiples of 32 columns)
        if (k0 < 2 * pitch) __builtin_memcpy(__builtin_assume_aligned(codes + row * (int64_t)pitch + k0 / 2, PER / 2), packed, PER / 2);
    }
}

template <int NR, int MT>
hipError_t launch_w4_tiles(const W4Params& p, int group, int64_t passes, hipStream_t s) {
    const int blocks = ceil_div(p.N, 16 * MT / NR);
    // (a launch counts its threads in 32 bits, and at most 65535 rows of workgroups)
    int64_t room = ((int64_t)1 << 21) / blocks;
    room = room < 1 ? 1 : room > 65535 ? 65535 : room;
    const dim3 grid((unsigned)blocks, (unsigned)(passes < room ? passes : room)), block(64 * w4_waves(MT));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, p); };
    const bool ragged = p.K % kW4Unit != 0;
    if (group == 32) ragged ? go(w4_gemm_kernel<NR, MT, 32, true>) : go(w4_gemm_kernel<NR, MT, 32, false>);
    else if (group == 64) ragged ? go(w4_gemm_kernel<NR, MT, 64, true>) : go(w4_gemm_kernel<NR, MT, 64, false>);
    else ragged ? go(w4_gemm_kernel<NR, MT, 128, true>) : go(w4_gemm_kernel<NR, MT, 128, false>);
    return hipGetLastError();
}

template <int NR>
hipError_t launch_w4(const W4Params& p, int group, hipStream_t s) {
    // passes: at most one for 32 rows, and one more for the rest of each segment's rows
    const int64_t passes = (int64_t)p.rows_cap / kW4Rows + (p.n_seg < p.rows_cap ? p.n_seg : p.rows_cap);
    // fewer workgroups than CUs: one tile of each matrix a wave (one row of 4096 x 4096, groups of
    // 128: 7.0 us, with four tiles 9.5; where there are more, the FFN above takes 24.8 + 16.1 with two)
    if (passes * ceil_div(p.N, 64 / NR) < persistent_workgroups()) return launch_w4_tiles<NR, NR>(p, group, passes, s);
    return launch_w4_tiles<NR, 4>(p, group, passes, s);
}

}  // namespace

hipError_t launch_w4_quantize(const W4QuantizeArgs& a, hipStream_t s) {
    const int64_t rows = (int64_t)a.n * a.N, groups = rows * ceil_div(a.K, a.group);
    const int64_t wgs = ceil_div64(groups, 32);
    const dim3 grid((unsigned)(wgs < (1 << 20) ? wgs : (1 << 20))), block(256);
    auto go = [&](auto kernel, auto* w) {
        hipLaunchKernelGGL(kernel, grid, block, 0, s, w, a.codes, (uint16_t*)a.scales, a.zeros, rows, a.K);
    };
    auto typed = [&](auto* w) {
        typedef std::remove_cv_t<std::remove_pointer_t<decltype(w)>> T;
        if (a.group == 32) go(w4_quantize_kernel<T, 4>, w);
        else if (a.group == 64) go(w4_quantize_kernel<T, 8>, w);
        else go(w4_quantize_kernel<T, 16>, w);
    };
    if (a.dtype == BMOE_BF16) typed((const uint16_t*)a.w);
    else typed((const float*)a.w);
    return hipGetLastError();
}

hipError_t launch_w4_gemm(const W4GemmArgs& a, hipStream_t s) {
    auto stack = [&](const bmoe_w4* w) {
        return w ? w4_stack(w->codes, w->scales, w->zeros, (int64_t)a.n_seg * a.N, a.K, w->group) : W4Stack{};
    };
    W4Params p{(const uint16_t*)a.a, {stack(a.w0), stack(a.w1)}, (uint16_t*)a.c, a.offsets, a.a_rows, a.a_count,
               a.n_seg, a.rows_cap, a.N, a.K};
    return a.w1 ? launch_w4<2>(p, a.w0->group, s) : launch_w4<1>(p, a.w0->group, s);
}

}  // namespace bmoe
