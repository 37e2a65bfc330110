// The whole layer for at most 16 tokens (Sec. 2.1 with the map of Eq. 2).
//
// With so few tokens all of them fit one MFMA tile, so nothing is permuted: a
// reached segment's weights are multiplied with every token, and a token that
// does not call the segment is left out where its hidden values would be stored.
//   few_up_kernel    one workgroup per 16 hidden columns of a reached segment (or
//                    of the shared experts): silu(Wg x) * (Wu x), times the
//                    token's gate of that segment, to the workspace;
//   few_down_kernel  one workgroup per 16 output columns: the sum over the reached
//                    segments and their hidden columns is one long K, so the
//                    gate-weighted sum over experts falls out of it.
// Both are bound by reading the weights. A workgroup's waves split K, each holding
// several units of the weight rows in flight, and add their partial tiles through
// LDS in wave order. The tokens are the A operand, the weight rows the B operand:
// D[token 4q+i][weight row r16] in element i of lane (r16, q).
// A unit is the columns that a wave takes at once, UK of them: 64 of bf16 and 32
// of fp32 weights (a 128-byte line of each row), 128 of 4-bit ones (see w4.h).
// Hidden values of bf16 layers are kept as the sum of two bf16 (16 bits of
// significand) and multiplied as such, since the matrix cores idle here anyway;
// so the layer's output is rounded once.
#include "bmoe_common.h"
#include "w4.h"

namespace bmoe {
namespace {

constexpr int kFewTok = BMOE_FEW_MAX_TOKENS;
constexpr int kFewCols = 16;
constexpr int kUpThreads = 512, kDownThreads = 1024;
static_assert(kFewTok == 16, "one MFMA tile of tokens");

// Weights of one format. A wave's unit: load() fetches it, multiply() adds its
// products with the activations of NX parts (their sum is the value) to acc.
struct FmtBf16 {
    typedef uint16_t Act;
    static constexpr int UK = 64, LD = 2, NX = 2;
    struct Stack { const uint16_t* w; };
    struct Unit {
        v4u w[LD];
        __device__ __forceinline__ void load(const Stack& st, size_t row, int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < LD; ++u) {
                const int col = k + u * 32 + q * 8;
                w[u] = col < K ? *(const v4u*)(st.w + row * K + col) : v4u{0, 0, 0, 0};
            }
        }
    };
    // activations of a unit: column k + 32u + 8q ..
    struct X {
        v4u x[LD];
        __device__ __forceinline__ void load(const Act* xr, bool some, int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < LD; ++u) {
                const int col = k + u * 32 + q * 8;
                x[u] = some && col < K ? *(const v4u*)(xr + col) : v4u{0, 0, 0, 0};
            }
        }
    };
    template <int NM, int NP>
    __device__ static __forceinline__ void multiply(f32x4 (&tot)[NM], const Unit (&w)[NM], const X (&x)[NP]) {
#pragma unroll
        for (int u = 0; u < LD; ++u)
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int m = 0; m < NM; ++m) tot[m] = mfma16(x[p].x[u], w[m].w[u], tot[m]);
    }
};

struct FmtF32 {
    typedef float Act;
    static constexpr int UK = 32, LD = 2, NX = 1;
    struct Stack { const float* w; };
    struct Unit {
        f32x4 w[LD];
        __device__ __forceinline__ void load(const Stack& st, size_t row, int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < LD; ++u) {
                const int col = k + u * 16 + q * 4;
                w[u] = col < K ? *(const f32x4*)(st.w + row * K + col) : f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
    };
    struct X {
        f32x4 x[LD];
        __device__ __forceinline__ void load(const Act* xr, bool some, int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < LD; ++u) {
                const int col = k + u * 16 + q * 4;
                x[u] = some && col < K ? *(const f32x4*)(xr + col) : f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
    };
    template <int NM, int NP>
    __device__ static __forceinline__ void multiply(f32x4 (&tot)[NM], const Unit (&w)[NM], const X (&x)[NP]) {
        static_assert(NP == 1, "fp32 activations are whole");
#pragma unroll
        for (int u = 0; u < LD; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int m = 0; m < NM; ++m)
                    tot[m] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[0].x[u][j], w[m].w[u][j], tot[m], 0, 0, 0);
    }
};

template <int GROUP>
struct FmtW4 {
    typedef uint16_t Act;
    static constexpr int UK = kW4Chunk, LD = 1, NX = 2, NG = W4Chunk<GROUP>::NG, STEPS = GROUP / 32;
    typedef W4Stack Stack;
    struct Unit {
        W4Chunk<GROUP> w;
        __device__ __forceinline__ void load(const Stack& st, size_t row, int k, int K, int q) {
            w.load(st, row, k / kW4Chunk, K, q);
        }
    };
    struct X {
        v4u x[4];
        __device__ __forceinline__ void load(const Act* xr, bool some, int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int col = k + u * 32 + q * 8;
                x[u] = some && col < K ? *(const v4u*)(xr + col) : v4u{0, 0, 0, 0};
            }
        }
    };
    template <int NM, int NP>
    __device__ static __forceinline__ void multiply(f32x4 (&tot)[NM], const Unit (&w)[NM], const X (&x)[NP]) {
        const v4u ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        v4u c[NM];
#pragma unroll
        for (int m = 0; m < NM; ++m) c[m] = w4_transpose(w[m].w.codes);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            f32x4 acc[NM], xs = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < NM; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = g * STEPS; u < (g + 1) * STEPS; ++u) {
                v4u b[NM];
#pragma unroll
                for (int m = 0; m < NM; ++m) b[m] = w4_unpack(c[m][u]);
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const v4u a = w4_order(x[p].x[u]);
                    xs = mfma16(a, ones, xs);
#pragma unroll
                    for (int m = 0; m < NM; ++m) acc[m] = mfma16(a, b[m], acc[m]);
                }
            }
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                const float sc = bf16_to_f32(w[m].w.s[g]), off = 16.f + (float)w[m].w.z[g];
#pragma unroll
                for (int i = 0; i < 4; ++i) tot[m][i] = fmaf(sc, fmaf(-off, xs[i], acc[m][i]), tot[m][i]);
            }
        }
    }
};

template <class F>
struct FewParams {
    typedef typename F::Act Act;
    typename F::Stack gate, up, down, gate_sh, up_sh, down_sh;
    const Act* x;
    const int32_t* slot_group;
    const float* slot_gate;
    // hidden values, [T*k, f] of the slots then [T, fs] of the shared experts;
    // bf16 layers: the high parts, then as many low parts
    Act* h;
    Act* out;
    int T, k, G, d, f, fs;
    int64_t h_part;  // elements of one part
};

// sum of the waves' partials of D element (token, col)
__device__ __forceinline__ float tile_sum(const f32x4 (*part)[64], int waves, int token, int col) {
    const float* p = (const float*)&part[0][(token >> 2) * 16 + col] + (token & 3);
    float v = p[0];
    for (int w = 1; w < waves; ++w) v += p[w * 256];
    return v;
}

__device__ __forceinline__ void store_hidden(float* h, int64_t, int64_t at, float v) { h[at] = v; }
__device__ __forceinline__ void store_hidden(uint16_t* h, int64_t part, int64_t at, float v) {
    const uint16_t hi = f32_to_bf16(v);
    const float rest = v - bf16_to_f32(hi);
    h[at] = hi;
    h[part + at] = isfinite(rest) ? f32_to_bf16(rest) : (uint16_t)0;  // (an infinite value stays one)
}

template <class F>
__global__ __launch_bounds__(kUpThreads, 2) void few_up_kernel(FewParams<F> p) {
    constexpr int WAVES = kUpThreads / 64, BATCH = 4;
    __shared__ __align__(16) f32x4 part[2][WAVES][64];
    __shared__ int present[BMOE_MAX_EXPERTS], seg_s, slot_of[kFewTok];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int r16 = lane & 15, q = lane >> 4;
    const int T = p.T, k = p.k, d = p.d;
    const int sh_tiles = ceil_div(p.fs, kFewCols), tiles = ceil_div(p.f, kFewCols);
    const bool shared = (int)blockIdx.x < sh_tiles;
    int seg = 0, n0 = blockIdx.x * kFewCols;
    if (!shared) {
        // the reached segments ascending; this workgroup takes columns n0 .. of the a-th
        const int a = (blockIdx.x - sh_tiles) / tiles;
        n0 = (blockIdx.x - sh_tiles) % tiles * kFewCols;
        if (tid < BMOE_MAX_EXPERTS) present[tid] = 0;
        if (tid < kFewTok) slot_of[tid] = -1;
        if (tid == 0) seg_s = -1;
        __syncthreads();
        const int g = tid < T * k ? p.slot_group[tid] : -1;
        const bool valid = (unsigned)g < (unsigned)p.G;
        if (valid) present[g] = 1;
        __syncthreads();
        if (wave == 0) {
            int before = 0;
            for (int b = 0; b < BMOE_MAX_EXPERTS; b += 64) {
                const bool in = present[b + lane] != 0;
                const unsigned long long m = __ballot(in);
                if (in && before + __popcll(m & ((1ull << lane) - 1)) == a) seg_s = b + lane;
                before += __popcll(m);
            }
        }
        __syncthreads();
        seg = seg_s;
        if (seg < 0) return;  // fewer segments are reached
        if (valid && g == seg) slot_of[tid / k] = tid;
        // (read after the barrier that follows the products)
    }
    const int N = shared ? p.fs : p.f;
    const size_t wrow = (size_t)seg * N + min(n0 + r16, N - 1);
    const typename F::Act* xr = p.x + (size_t)min(r16, T - 1) * d;
    const int units = ceil_div(d, F::UK);
    f32x4 tot[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    for (int u0 = wave; u0 < units; u0 += WAVES * BATCH) {
        typename F::Unit w[BATCH][2];
        typename F::X x[BATCH][1];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int u = u0 + WAVES * b;
            if (u < units) {
                w[b][0].load(shared ? p.gate_sh : p.gate, wrow, u * F::UK, d, q);
                w[b][1].load(shared ? p.up_sh : p.up, wrow, u * F::UK, d, q);
                x[b][0].load(xr, true, u * F::UK, d, q);
            }
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
            if (u0 + WAVES * b < units) F::multiply(tot, w[b], x[b]);
    }
    part[0][wave][lane] = tot[0];
    part[1][wave][lane] = tot[1];
    __syncthreads();
    const int token = tid >> 4, col = tid & 15;
    if (token < T && n0 + col < N) {
        const int slot = shared ? token : slot_of[token];
        if (slot >= 0) {
            const float g = tile_sum(part[0], WAVES, token, col), u = tile_sum(part[1], WAVES, token, col);
            const float v = silu_mul(g, u) * (shared ? 1.f : p.slot_gate[slot]);
            const int64_t at = (shared ? (int64_t)T * k * p.f : 0) + (int64_t)slot * N + n0 + col;
            store_hidden(p.h, p.h_part, at, v);
        }
    }
}

template <class F>
__global__ __launch_bounds__(kDownThreads) void few_down_kernel(FewParams<F> p) {
    constexpr int WAVES = kDownThreads / 64, BATCH = 2;
    __shared__ __align__(16) f32x4 part[WAVES][64];
    __shared__ int present[BMOE_MAX_EXPERTS];
    __shared__ int16_t segs[BMOE_MAX_EXPERTS];               // the reached segments, ascending
    __shared__ int16_t slot_of[BMOE_MAX_EXPERTS][kFewTok];   // [i][token]: slot of segs[i], or -1
    __shared__ int reached_s;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int r16 = lane & 15, q = lane >> 4;
    const int T = p.T, k = p.k, d = p.d, f = p.f, fs = p.fs;
    const int n0 = blockIdx.x * kFewCols;
    if (tid < BMOE_MAX_EXPERTS) present[tid] = 0;
    for (int i = tid; i < BMOE_MAX_EXPERTS * kFewTok / 2; i += kDownThreads) ((int*)slot_of)[i] = -1;
    __syncthreads();
    const int g = tid < T * k ? p.slot_group[tid] : -1;
    const bool valid = (unsigned)g < (unsigned)p.G;
    if (valid) present[g] = 1;
    __syncthreads();
    if (wave == 0) {
        int before = 0;
        for (int b = 0; b < BMOE_MAX_EXPERTS; b += 64) {
            const bool in = present[b + lane] != 0;
            const unsigned long long m = __ballot(in);
            const int at = before + __popcll(m & ((1ull << lane) - 1));
            if (in) {
                segs[at] = (int16_t)(b + lane);
                present[b + lane] = at;  // from here on: the segment's place
            }
            before += __popcll(m);
        }
        if (lane == 0) reached_s = before;
    }
    __syncthreads();
    if (valid) slot_of[present[g]][tid / k] = (int16_t)tid;
    __syncthreads();
    const int per = ceil_div(f, F::UK), routed = reached_s * per, units = routed + ceil_div(fs, F::UK);
    const int wr = min(n0 + r16, d - 1);
    f32x4 tot[1] = {{0.f, 0.f, 0.f, 0.f}};
    for (int u0 = wave; u0 < units; u0 += WAVES * BATCH) {
        typename F::Unit w[BATCH][1];
        typename F::X x[BATCH][F::NX];
        int place[BATCH];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int u = u0 + WAVES * b;
            place[b] = -1;
            if (u >= units) continue;
            const bool sh = u >= routed;
            const int a = sh ? 0 : u / per;
            const int kk = (sh ? u - routed : u - a * per) * F::UK;
            const int width = sh ? fs : f;
            const int slot = sh ? (r16 < T ? r16 : -1) : slot_of[a][r16];
            const int64_t at = (sh ? (int64_t)T * k * f : 0) + (int64_t)max(slot, 0) * width;
            if (!sh) place[b] = a;
            w[b][0].load(sh ? p.down_sh : p.down, (size_t)(sh ? 0 : segs[a]) * d + wr, kk, width, q);
#pragma unroll
            for (int i = 0; i < F::NX; ++i) x[b][i].load(p.h + i * p.h_part + at, slot >= 0, kk, width, q);
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            if (u0 + WAVES * b >= units) break;
            f32x4 acc[1] = {{0.f, 0.f, 0.f, 0.f}};
            F::multiply(acc, w[b], x[b]);
            // a token that does not call the segment takes nothing of its products
            // (its zero activations against an infinite weight would be NaN)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (place[b] < 0 || slot_of[place[b]][4 * q + i] >= 0) tot[0][i] += acc[0][i];
        }
    }
    part[wave][lane] = tot[0];
    __syncthreads();
    const int token = tid >> 4, col = tid & 15;
    if (token < T && n0 + col < d) {
        const float v = tile_sum(part, WAVES, token, col);
        typename F::Act* o = p.out + (size_t)token * d + n0 + col;
        if constexpr (sizeof(typename F::Act) == 2) *o = f32_to_bf16(v);
        else *o = v;
    }
}

int64_t up_workgroups(int T, int k, int G, int f, int fs) {
    const int64_t slots = (int64_t)T * k, most = slots < G ? slots : G;
    return most * ceil_div(f, kFewCols) + ceil_div(fs, kFewCols);
}

template <class F>
hipError_t launch_few_t(const FewArgs& a, const FewParams<F>& p, hipStream_t s) {
    const int64_t up = up_workgroups(a.T, a.k, a.G, a.f, a.fs);
    hipLaunchKernelGGL((few_up_kernel<F>), dim3((unsigned)up), dim3(kUpThreads), 0, s, p);
    hipLaunchKernelGGL((few_down_kernel<F>), dim3((unsigned)ceil_div(a.d, kFewCols)), dim3(kDownThreads), 0, s, p);
    return hipGetLastError();
}

template <class F, class ToStack>
FewParams<F> params_of(const FewArgs& a, ToStack st) {
    typedef typename F::Act Act;
    FewParams<F> p;
    p.gate = st(a.w.gate);
    p.up = st(a.w.up);
    p.down = st(a.w.down);
    p.gate_sh = st(a.w.gate_sh);
    p.up_sh = st(a.w.up_sh);
    p.down_sh = st(a.w.down_sh);
    p.x = (const Act*)a.x;
    p.slot_group = a.slot_group;
    p.slot_gate = a.slot_gate;
    p.h = (Act*)a.ws;
    p.out = (Act*)a.out;
    p.T = a.T;
    p.k = a.k;
    p.G = a.G;
    p.d = a.d;
    p.f = a.f;
    p.fs = a.fs;
    p.h_part = (int64_t)a.T * a.k * a.f + (int64_t)a.T * a.fs;
    return p;
}

}  // namespace

size_t few_ws_bytes(int T, int k, int f, int fs) { return ((size_t)T * k * f + (size_t)T * fs) * 4; }

// (a launch counts its threads in 32 bits)
bool few_grid_fits(int T, int k, int G, int f, int fs) {
    return up_workgroups(T, k, G, f, fs) * kUpThreads < ((int64_t)1 << 32);
}

hipError_t launch_few(const FewArgs& a, hipStream_t s) {
    RouteArgs r{a.x, a.w.w_router, a.w.bias, nullptr, a.w.e2g, a.topk_idx, a.topk_w, a.slot_group, a.slot_gate,
                nullptr, a.T, a.d, a.E, a.k, a.G, a.norm, a.dtype};
    hipError_t e = launch_route(r, s);
    if (e != hipSuccess) return e;
    if (a.w.group) {
        auto st = [](const bmoe_matrix& m) {
            return W4Stack{(const uint8_t*)m.w, (const uint16_t*)m.scales, m.zeros};
        };
        if (a.w.group == 32) return launch_few_t<FmtW4<32>>(a, params_of<FmtW4<32>>(a, st), s);
        if (a.w.group == 64) return launch_few_t<FmtW4<64>>(a, params_of<FmtW4<64>>(a, st), s);
        return launch_few_t<FmtW4<128>>(a, params_of<FmtW4<128>>(a, st), s);
    }
    if (a.dtype == BMOE_BF16)
        return launch_few_t<FmtBf16>(
            a, params_of<FmtBf16>(a, [](const bmoe_matrix& m) { return FmtBf16::Stack{(const uint16_t*)m.w}; }), s);
    return launch_few_t<FmtF32>(
        a, params_of<FmtF32>(a, [](const bmoe_matrix& m) { return FmtF32::Stack{(const float*)m.w}; }), s);
}

}  // namespace bmoe
