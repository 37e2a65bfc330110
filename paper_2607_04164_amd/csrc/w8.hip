// Rows in 8 bits with a scale for each row: activations by token, weights by output channel.
//   scale = max|x| / 127,   code = round(x / scale)   (to nearest even, of the true quotient)
// The grouped products with them are those of ffn.hip and ffn_skinny.hip on int8 MFMA.
//
// Bound by memory: a row is read once into registers (NT threads a row, CH units of 16 values a thread; longer
// rows are read again for what does not fit), its largest magnitude is reduced over the row's threads, and the
// codes go out 16 bytes a thread.
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

template <typename E, int NT, int CH>
__global__ __launch_bounds__(NT > 256 ? NT : 256) void q8_rows_kernel(W8QuantizeArgs a) {
    constexpr int R = NT > 256 ? 1 : 256 / NT;  // rows of a workgroup
    constexpr int W = NT / 64;
    __shared__ uint32_t part[W];
    int64_t r = (int64_t)blockIdx.x * R + threadIdx.x / NT;
    // (one row of a workgroup where its threads have a barrier: they leave together)
    if (r >= a.rows) return;
    if (a.offsets && (r < a.offsets[0] || r >= a.offsets[a.n_seg])) return;
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
#pragma unroll
    for (int off = 32; off; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) m = max(m, part[w]);
    }
    float s = __uint_as_float(m) / 127.f, inv = 0.f;
    const bool finite = m < 0x7f800000u;
    if (finite && s >= kMinScale) inv = 1.f / s;
    else s = finite ? 0.f : __builtin_nanf("");
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
    const int64_t blocks = ceil_div64(a.rows, R);
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL((q8_rows_kernel<E, NT, CH>), dim3((unsigned)blocks), dim3(NT > 256 ? NT : 256), 0, s, a);
    return hipGetLastError();
}

template <typename E>
hipError_t pick_q8(const W8QuantizeArgs& a, hipStream_t s) {
    const int units = (int)(w8_pitch(a.K) / 16);
    if (units <= 64) return launch_q8<E, 64, 1>(a, s);
    if (units <= 128) return launch_q8<E, 64, 2>(a, s);
    if (units <= 256) return launch_q8<E, 256, 1>(a, s);
    if (units <= 512) return launch_q8<E, 256, 2>(a, s);
    return launch_q8<E, 256, 4>(a, s);
}

}  // namespace

hipError_t launch_w8_quantize(const W8QuantizeArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    return a.dtype == BMOE_BF16 ? pick_q8<uint16_t>(a, s) : pick_q8<float>(a, s);
}

}  // namespace bmoe
