// Rows in 8 bits with a scale for each row: activations by token, weights by output channel.
//   scale = max|x| / 127,   code = round(x / scale)   (to nearest even, of the true quotient)
// The grouped products with them are those of ffn.hip and ffn_skinny.hip on int8 MFMA (their sums are exact in int32:
// 131072 * 127^2 < 2^31), but for very few rows (few8_kernel).
//
// The quantizer is bound by memory: a row is read once into registers (NT threads a row, CH units of 16 values a
// thread; longer rows are read again for what does not fit), its largest magnitude is reduced over the row's threads,
// and the codes go out 16 bytes a thread. 30000 bf16 rows of 1408 (127 MB) 28 to 32 us, 4.0 to 4.5 TB/s; 8192 rows of
// 14336, which the last-level cache holds in part, 59 us (5.9 TB/s); up to 512 rows 2.5 to 4 us of latency.
#include "bmoe_common.h"
#include "chunk16.h"
#include "stream_io.h"

namespace bmoe {
namespace {

// Scales below this are taken as 0 (the row reads zeros): above it the remainders below are exact.
constexpr float kMinScale = 0x1p-120f;

// 16 values of a row from value 16 u on (zeros past K, a multiple of 8)
template <typename E>
__device__ __forceinline__ void load_unit(const uint4* row, int u, int K, float (&f)[16]) {
    constexpr int N = Vec<E>::N, C = 16 / N;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const bool in = u * 16 + i * N < K;
        Vec<E>::load(in ? row[u * C + i] : make_uint4(0, 0, 0, 0), f + i * N);
    }
}

// magnitude bits: ordered like the magnitudes, with infinities and then NaN above them
__device__ __forceinline__ uint32_t magnitude(float f) { return __float_as_uint(f) & 0x7fffffffu; }

// round(x / s) for |x| <= 127 s: floor of an approximate quotient, then the side of the half step that x is on (the
// fma's sign is exact, so ties and near ties come out as the true quotient's; an approximation that falls to the
// other side of a whole number changes nothing)
__device__ __forceinline__ int code_of(float x, float s, float inv) {
    const float k = floorf(x * inv);
    const float over = fmaf(-s, k + 0.5f, x);
    const int i = (int)k;
    return i + (over > 0.f ? 1 : over == 0.f ? i & 1 : 0);
}

__device__ __forceinline__ uint4 codes_of(const float (&f)[16], float s, float inv) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        w[j] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[j] |= ((uint32_t)code_of(f[4 * j + i], s, inv) & 0xffu) << (8 * i);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// the scale of a row whose largest magnitude bits are m, and its reciprocal (0: the codes are 0)
__device__ __forceinline__ float row_scale(uint32_t m, float& inv) {
    const float s = __uint_as_float(m) / 127.f;
    const bool finite = m < 0x7f800000u, live = finite && s >= kMinScale;
    inv = live ? 1.f / s : 0.f;
    return live ? s : finite ? 0.f : __builtin_nanf("");
}

template <typename E, int NT, int CH>
__global__ __launch_bounds__(NT > 256 ? NT : 256) void q8_rows_kernel(W8QuantizeArgs a) {
    constexpr int R = NT > 256 ? 1 : 256 / NT;  // rows of a workgroup
    constexpr int W = NT / 64;
    __shared__ uint32_t part[W];
    const int64_t r = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * R + threadIdx.x / NT;
    // (one row of a workgroup where its threads have a barrier: they leave together)
    if (r >= a.rows) return;
    const int K = a.K, t = threadIdx.x % NT;
    const int units = (int)(w8_pitch(K) / 16);
    const uint4* row = (const uint4*)((const E*)a.x + (size_t)r * K);
    float f[CH][16];
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        load_unit<E>(row, t + NT * c, K, f[c]);
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, magnitude(f[c][i]));
    }
    for (int u = t + NT * CH; u < units; u += NT) {
        float g[16];
        load_unit<E>(row, u, K, g);
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, magnitude(g[i]));
    }
    // (rows of no segment: their loads do not wait for the offsets)
    if (a.offsets && (r < a.offsets[0] || r >= a.offsets[a.n_seg])) return;
#pragma unroll
    for (int off = 32; off; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) m = max(m, part[w]);
    }
    float inv;
    const float s = row_scale(m, inv);
    uint4* out = (uint4*)(a.codes + (size_t)r * w8_pitch(K));
    const uint4 none = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int u = t + NT * c;
        if (u < units) out[u] = inv > 0.f ? codes_of(f[c], s, inv) : none;
    }
    for (int u = t + NT * CH; u < units; u += NT) {
        float g[16];
        load_unit<E>(row, u, K, g);
        out[u] = inv > 0.f ? codes_of(g, s, inv) : none;
    }
    if (t == 0) a.scales[r] = s;
}

template <typename E, int NT, int CH>
hipError_t launch_q8(const W8QuantizeArgs& a, hipStream_t s) {
    constexpr int R = NT > 256 ? 1 : 256 / NT;
    // (2^24 of these workgroups are too many for one dimension of a grid)
    const int64_t blocks = ceil_div64(a.rows, R), across = min(blocks, (int64_t)1 << 22);
    hipLaunchKernelGGL((q8_rows_kernel<E, NT, CH>), dim3((unsigned)across, (unsigned)ceil_div64(blocks, across)),
                       dim3(NT > 256 ? NT : 256), 0, s, a);
    return hipGetLastError();
}

// Rows of 65 to 128 units: 256 threads a row up to this many rows, 64 above. us, 64 / 256 threads (captured, bf16, three
// inputs in turn): K = 2048 256 rows 3.5 / 3.1, 512 rows 3.5 / 3.2, 768 rows 3.6 / 3.4, 1024 rows 3.7 / 3.8, 2048 rows 4.4 /
// 5.4, 16384 rows 19.8 / 25.4; K = 1032 512 rows 4.2 / 3.3, 768 rows 4.3 / 3.4, 1024 rows 4.3 / 3.8, 2048 rows 4.4 / 5.1,
// 16384 rows 16.1 / 23.9. (The two sides meet at about 900 rows of 128 units and 1400 of 72, so that between 512 and
// those the rule gives away up to 0.9 us.)
constexpr int kShortRows = 512;

template <typename E>
hipError_t pick_q8(const W8QuantizeArgs& a, hipStream_t s) {
    const int units = (int)(w8_pitch(a.K) / 16);
    // (few rows: a workgroup each, for their latency)
    if (units <= 64) return launch_q8<E, 64, 1>(a, s);
    if (units <= 128 && a.rows > kShortRows) return launch_q8<E, 64, 2>(a, s);
    if (units <= 256) return launch_q8<E, 256, 1>(a, s);
    if (units <= 512) return launch_q8<E, 256, 2>(a, s);
    return launch_q8<E, 256, 4>(a, s);
}

// ---- products of a few rows that round their activations themselves
//
// One launch instead of two where rows_cap * K is small: every workgroup rounds its segment's rows (at most
// kFewValues values, from the L2 cache) into LDS while its first weights are on their way, and then multiplies as
// skinny_reg_kernel does: 16 output columns, K split over the four waves (128-column pairs of MFMA steps, PAIRS of
// them in flight a wave), the waves' sums added in LDS. Bound by a chain of latencies (offsets, rows, their maximum,
// codes, sums) beside the weights' load: a row through 4096 x 4096 6.9 us, 2.4 TB/s; one token's four rows on four of 15
// segments, d = 2048, d_ff = 1408, gate/up 10, down 6 us. Every load whose address the kernel's arguments give is issued
// before the offsets are there (source rows, the scales, one segment's weights).
constexpr int kFewThreads = 256;
constexpr int kFewRows = 16;
constexpr int kFewValues = 16384;                              // rows_cap * pitch, at most
constexpr int kFewUnits = kFewValues / 16 / kFewThreads;       // units of 16 values a thread
constexpr int kFewPad = 16;                                    // bytes between rows in LDS: rows on other banks

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

struct Few8Params {
    const uint16_t* A;
    const int8_t* B0;
    const int8_t* B1;
    const float* sb0;
    const float* sb1;
    uint16_t* C;
    const int32_t* offsets;
    const int32_t* a_rows;
    int a_count, n_seg, rows_cap, N, K;
};

template <bool GATED, int PAIRS>
__global__ __launch_bounds__(kFewThreads, 2) void few8_kernel(Few8Params p) {
    constexpr int NMAT = GATED ? 2 : 1;
    __shared__ __align__(16) char s_x[kFewValues + kFewRows * kFewPad];
    __shared__ __align__(16) i32x4 s_part[4][NMAT][64];
    __shared__ uint32_t s_max[kFewRows];
    __shared__ float s_scale[kFewRows];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int N = p.N, K = p.K, P = (int)w8_pitch(K);
    const int ncb = ceil_div(N, 16), s = blockIdx.x / ncb, n0 = (blockIdx.x % ncb) * 16;
    const int r16 = lane & 15, q = lane >> 4;
    const size_t wrow = (size_t)s * N + min(n0 + r16, N - 1);
    const char* wp[NMAT];
    wp[0] = (const char*)p.B0 + wrow * P + q * 16;
    if constexpr (GATED) wp[NMAT - 1] = (const char*)p.B1 + wrow * P + q * 16;
    const int npairs = P / 128;
    // step u of the batch from pair p0: bytes 64 (u & 1) .. of pair p0 + 4 (u / 2)
    v4u w[2 * PAIRS][NMAT];
    auto load_weights = [&](int p0) {
#pragma unroll
        for (int u = 0; u < 2 * PAIRS; ++u)
            if (p0 + 4 * (u >> 1) < npairs) {
#pragma unroll
                for (int mat = 0; mat < NMAT; ++mat)
                    w[u][mat] = *(const v4u*)(wp[mat] + (p0 + 4 * (u >> 1)) * 128 + (u & 1) * 64);
            }
    };
    // (one segment has rows, whatever its offsets: its weights need not wait for them)
    const bool early = p.n_seg == 1;
    if (early) load_weights(wave);
    // the source of row `lane` (rows_cap <= kFewRows), loaded beside the offsets
    const int source = gathered_row(p.a_rows, p.a_count, min(lane, p.rows_cap - 1));
    const int beg = min(max(p.offsets[s], 0), p.rows_cap);
    const int end = min(max(p.offsets[s + 1], beg), p.rows_cap);
    const int rows = end - beg;  // (rows_cap of them at most, so kFewRows, and rows * P <= kFewValues)
    if (rows <= 0) return;
    // the rows' values, a unit of 16 a thread and round
    const int upr = P / 16, units = rows * upr;
    uint4 x[kFewUnits][2];
#pragma unroll
    for (int i = 0; i < kFewUnits; ++i) {
        const int j = tid + kFewThreads * i, r = j / upr, u = j - r * upr;
        x[i][0] = x[i][1] = make_uint4(0, 0, 0, 0);
        const int from = __shfl(source, min(beg + r, kFewRows - 1));
        if (j < units) {
            const uint4* row = (const uint4*)(p.A + (size_t)from * K);
            if (u * 16 < K) x[i][0] = row[2 * u];
            if (u * 16 + 8 < K) x[i][1] = row[2 * u + 1];
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (!early) load_weights(wave);
    const int col = n0 + 4 * q;  // (N is a multiple of 8: the scales are a quarter of a row's)
    const size_t at = (size_t)s * N + min(col, N - 4);
    const float4 c0 = *(const float4*)(p.sb0 + at), c1 = GATED ? *(const float4*)(p.sb1 + at) : c0;
    __builtin_amdgcn_sched_barrier(0);
    if (tid < kFewRows) s_max[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kFewUnits; ++i) {
        const int j = tid + kFewThreads * i;
        if (j >= units) break;
        uint32_t m = 0;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const uint32_t v[4] = {x[i][c].x, x[i][c].y, x[i][c].z, x[i][c].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) m = max(m, max(v[e] << 16 & 0x7fff0000u, v[e] & 0x7fff0000u));
        }
        atomicMax(&s_max[j / upr], m);  // (whatever the order)
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kFewUnits; ++i) {
        const int j = tid + kFewThreads * i, r = j / upr, u = j - r * upr;
        if (j >= units) break;
        float inv;
        const float sc = row_scale(s_max[r], inv);
        float f[16];
        Vec<uint16_t>::load(x[i][0], f);
        Vec<uint16_t>::load(x[i][1], f + 8);
        *(uint4*)(s_x + r * (P + kFewPad) + u * 16) = inv > 0.f ? codes_of(f, sc, inv) : make_uint4(0, 0, 0, 0);
        if (u == 0) s_scale[r] = sc;
    }
    __syncthreads();
    i32x4 acc[NMAT];
#pragma unroll
    for (int mat = 0; mat < NMAT; ++mat) acc[mat] = i32x4{0, 0, 0, 0};
    // (lanes past the last row repeat it: their results are not stored)
    const char* xp = s_x + min(r16, rows - 1) * (P + kFewPad) + q * 16;
    for (int p0 = wave; p0 < npairs; p0 += 4 * PAIRS) {
        if (p0 != wave) load_weights(p0);
#pragma unroll
        for (int u = 0; u < 2 * PAIRS; ++u)
            if (p0 + 4 * (u >> 1) < npairs) {
                const v4u xv = *(const v4u*)(xp + (p0 + 4 * (u >> 1)) * 128 + (u & 1) * 64);
#pragma unroll
                for (int mat = 0; mat < NMAT; ++mat) acc[mat] = OpI8::mma16(w[u][mat], xv, acc[mat]);
            }
    }
#pragma unroll
    for (int mat = 0; mat < NMAT; ++mat) s_part[wave][mat][lane] = acc[mat];
    __syncthreads();
    // the lane holds columns n0 + 4 q .. + 3 of row r16
    if (wave != 0 || r16 >= rows) return;
    if (col >= N) return;
    i32x4 sum[NMAT];
#pragma unroll
    for (int mat = 0; mat < NMAT; ++mat)
        sum[mat] = s_part[0][mat][lane] + s_part[1][mat][lane] + s_part[2][mat][lane] + s_part[3][mat][lane];
    const float rs = s_scale[r16];
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = scaled(sum[0][i], rs, ((const float*)&c0)[i]);
        if (GATED) v[i] = silu_mul(v[i], scaled(sum[NMAT - 1][i], rs, ((const float*)&c1)[i]));
    }
    *(uint2*)(p.C + (size_t)(beg + r16) * N + col) =
        make_uint2(pack_bf16x2_hw(v[0], v[1]), pack_bf16x2_hw(v[2], v[3]));
}

template <bool GATED, int PAIRS>
hipError_t launch_few8(const Few8Params& p, hipStream_t s) {
    hipLaunchKernelGGL((few8_kernel<GATED, PAIRS>), dim3((unsigned)(p.n_seg * ceil_div(p.N, 16))), dim3(kFewThreads), 0, s,
                       p);
    return hipGetLastError();
}

}  // namespace

// Half as many values where all rows are one segment's (every workgroup then rounds all of them). us, this kernel / the
// quantizer and the product, weights of three sets in turn: 1 segment, d = 2048, d_ff = 1408 gate/up 4 rows 7.5 / 8.5, 8
// rows 9.2 / 9.0; N = K = 4096, 2 rows 8.7 / 10.0, 4 rows 10.5 / 10.2; N = K = 1024, 8 rows 5.7 / 6.6, 16 rows 7.6 / 6.8;
// 15 segments, gate/up 4 rows 9.9 / 12.2, 8 rows 11.5 / 17.2, down 8 rows 8.8 / 11.1; 4 segments, N = K = 4096, 4 rows
// 13.8 / 14.7. (Room for 32768 values costs the smaller calls 0.3 to 1 us by its registers.)
bool w8_few_fits(const W8GemmArgs& a) {
    // (the most segments of the widest matrices: the other kernels' workgroups have more columns)
    if (!grid_holds((int64_t)a.n_seg * ceil_div(a.N, 16), kFewThreads)) return false;
    return a.rows_cap <= kFewRows && a.rows_cap * w8_pitch(a.K) <= (a.n_seg == 1 ? kFewValues / 2 : kFewValues);
}

hipError_t launch_w8_few(const W8GemmArgs& a, const void* x, hipStream_t s) {
    const Few8Params p{(const uint16_t*)x, a.w0.codes, a.w1.codes, a.w0.scales, a.w1.scales, (uint16_t*)a.c,
                       a.offsets, a.a_rows, a.a_count, a.n_seg, a.rows_cap, a.N, a.K};
    return a.w1.codes ? launch_few8<true, 4>(p, s) : launch_few8<false, 8>(p, s);
}

hipError_t launch_w8_quantize(const W8QuantizeArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    return a.dtype == BMOE_BF16 ? pick_q8<uint16_t>(a, s) : pick_q8<float>(a, s);
}

}  // namespace bmoe
