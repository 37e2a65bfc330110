// The whole layer for at most 16 tokens (Sec. 2.1 with the map of Eq. 2).
//
// With so few tokens all of them fit one MFMA tile, so nothing is permuted: a
// reached segment's weights are multiplied with every token, and a token that
// does not call the segment is left out where its hidden values would be stored.
//   few_logits_kernel  one workgroup per expert (and four tokens): the gate logits
//                      in float64 (bf16 and fp32 products are exact there), so
//                      near ties need no second look;
//   few_up_kernel      items of 16 hidden columns of a reached segment (or of the
//                      shared experts), dealt out to the workgroups. Every
//                      workgroup selects the top-k from the logits by itself, which
//                      costs less than another launch: silu(Wg x) * (Wu x), times
//                      the token's gate of that segment, to the workspace;
//   few_down_kernel    16 output columns a workgroup: the sum over the reached
//                      segments and their hidden columns is one long K, so the
//                      gate-weighted sum over experts falls out of it. K is split
//                      over several workgroups where the columns alone are too few
//                      for the chip; the last one to finish adds the parts in order.
// The last two are bound by reading the weights. A workgroup's waves split K; each
// wave reads units of the weight rows into one register buffer while it multiplies
// the other. Their partial tiles are added through LDS in wave order. The tokens
// are the A operand, the weight rows the B operand: D[token 4q+i][weight row r16] in
// element i of lane (r16, q). Rows of the A operand past the last token (or of
// tokens that do not call the segment) hold what is at hand: a row of D depends on
// its own row of A alone, and theirs are not used.
// A unit is the columns that a wave takes at once, UK of them: 64 of bf16 and 32
// of fp32 weights (a 128-byte line of each row), 128 of 4-bit ones (see w4.h).
// Hidden values of bf16 layers are kept as the sum of two bf16 (16 bits of
// significand) and multiplied as such, since the matrix cores idle here anyway;
// so the layer's output is rounded once. Up to eight tokens have their high parts
// in rows 0..7 of the A operand and their low parts in rows 8..15.
#include <math.h>

#include "bmoe_common.h"
#include "chunk16.h"
#include "route_select.h"
#include "w4.h"

namespace bmoe {
namespace {

constexpr int kFewTok = BMOE_FEW_MAX_TOKENS;
constexpr int kFewCols = 16;
constexpr int kLogitThreads = 256, kUpThreads = 512, kDownThreads = 256;
constexpr int kUpWgsPerCu = 2, kDownWgsPerCu = 3;  // by their registers
constexpr int kSplitMax = 8;     // workgroups that share 16 output columns
constexpr int kLogitTokens = 4;  // tokens of a few_logits_kernel workgroup
constexpr int kMaxSlots = kFewTok * BMOE_MAX_TOPK;
static_assert(kFewTok == 16, "one MFMA tile of tokens");
constexpr int kTile = kFewTok * kFewCols;  // outputs of a tile, a thread each
static_assert(kMaxSlots <= kTile && BMOE_MAX_EXPERTS <= kTile, "a thread per slot and per expert");
static_assert(kTile <= kUpThreads && kTile == kDownThreads, "a thread per output");

// A value that the wave shares, in a scalar register: left to itself the compiler
// keeps some of them, and the addresses that follow from them, in vector registers
// (up kernel: 203 registers, 130 this way).
__device__ __forceinline__ int scalar(int v) {
    asm("" : "+v"(v));  // (nothing is known of v here, so the next step stays)
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int div_uniform(int a, int b) { return scalar((int)((unsigned)a / (unsigned)b)); }

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

// ---- selection and the reached segments
//
// The 16 lanes of a row of lanes hold one token's logits, V each (experts s, s + 16, ..).

constexpr int kSetWords = BMOE_MAX_EXPERTS / 32;

struct SelectSmem {
    int pk[kFewTok][BMOE_MAX_TOPK];    // picks, best first
    float pe[kFewTok][BMOE_MAX_TOPK];  // exp(logit - best)
    float sum[kFewTok];                // of exp(logit - best) over all experts
    float gate[kMaxSlots];             // by slot, of a segment's first slot of the token
    uint32_t reached[kSetWords];       // the reached segments as a bit set
    int16_t segs[BMOE_MAX_EXPERTS];    // and ascending
    int16_t slot_of[BMOE_MAX_EXPERTS][kFewTok];  // [place in segs][token], -1: does not call it
};

__device__ __forceinline__ int members_below(const uint32_t* set, int g) {
    int n = 0;
    for (int i = 0; i < g >> 5; ++i) n += __popc(set[i]);
    return n + __popc(set[g >> 5] & ((1u << (g & 31)) - 1));
}
__device__ __forceinline__ int members(const uint32_t* set) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < kSetWords; ++i) n += __popc(set[i]);
    return scalar(n);
}

// picks of tokens 4 * wave .. 4 * wave + 3; the set was cleared before
template <int V>
__device__ __forceinline__ void few_select(const double* logits, const int32_t* e2g, SelectSmem& sm, int T, int E, int G,
                                           int k, int wave, int lane) {
    const int s = lane & 15, t = wave * 4 + (lane >> 4), tl = min(t, T - 1);
    const int vpl = (E - s + 15) / 16;
    double v[V];
    int key[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int e = min(s + 16 * j, E - 1);
        v[j] = logits[tl * E + e];
        key[j] = (e << 16) | (e2g[e] + 1);
    }
    unsigned taken = vpl >= V ? 0u : ~0u << vpl;
    double top = 0.0;
    for (int r = 0; r < k; ++r) {
        // ascending expert order, strict >: the lower index wins a tie; the first
        // untaken one is taken even at -inf
        double bv = -INFINITY;
        int be = kNoPick;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const bool in = !((taken >> j) & 1u) && (v[j] > bv || be == kNoPick);
            bv = in ? v[j] : bv;
            be = in ? key[j] : be;
        }
        group_argmax<16>(bv, be);
        const int e = pick_expert(be);
        if ((e & 15) == s) taken |= 1u << ((e >> 4) & 31);
        top = r == 0 ? bv : top;
        if (s == 0) {
            sm.pk[t][r] = be;
            sm.pe[t][r] = __expf((float)(bv - top));
            const int g = pick_group(be);
            if (t < T && (unsigned)g < (unsigned)G) atomicOr(&sm.reached[g >> 5], 1u << (g & 31));
        }
    }
    float se = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) se += j < vpl ? __expf((float)(v[j] - top)) : 0.f;
    se = group_sum<16>(se);
    if (s == 0) sm.sum[t] = se;
}

// ---- weights of one format
//
// Rows: 16 weight rows (fewer at the matrix's end) of K columns; Unit: a wave's UK
// columns of them, loaded at lane row r and the unit's first column; X: the same
// columns of the tokens, from an address that the wave shares and the lane's row's
// byte offset. Columns past K read the row's last ones and tail() zeroes them (in
// every unit: a branch would cost copies of the buffers). multiply() adds the products with NP parts of the activations (their sum is the value) to
// tot. PARTS: parts of a hidden value; BATCH: units of a register buffer.
struct FmtBf16 {
    typedef uint16_t Act;
    static constexpr int UK = 64, LD = 2, PARTS = 2, BATCH = 2;
    struct Stack { const uint16_t* w; };
    struct Rows {
        const uint16_t* w;
        __device__ __forceinline__ Rows(const Stack& st, int64_t first, int K) : w(st.w + first * K) {}
    };
    struct X {
        v4u x[LD];
        __device__ __forceinline__ void load(const Act* base, uint32_t row, int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < LD; ++u) x[u] = load_at(base, row + 2 * min(k + u * 32 + q * 8, K - 8));
        }
        __device__ __forceinline__ void tail(int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < LD; ++u) x[u] &= k + u * 32 + q * 8 < K ? ~0u : 0u;
        }
    };
    struct Unit {
        X w;
        __device__ __forceinline__ void load(const Rows& rows, int r, int k, int K, int q) {
            w.load(rows.w, (uint32_t)(r * K) * 2, k, K, q);
        }
        __device__ __forceinline__ void tail(int k, int K, int q) { w.tail(k, K, q); }
    };
    template <int NM, int NP>
    __device__ static __forceinline__ void multiply(f32x4 (&tot)[NM], const Unit (&w)[NM], const X (&x)[NP],
                                                    const Stack&) {
#pragma unroll
        for (int u = 0; u < LD; ++u)
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int m = 0; m < NM; ++m) tot[m] = mfma16(x[p].x[u], w[m].w.x[u], tot[m]);
    }
};

struct FmtF32 {
    typedef float Act;
    static constexpr int UK = 32, LD = 2, PARTS = 1, BATCH = 2;
    struct Stack { const float* w; };
    struct Rows {
        const float* w;
        __device__ __forceinline__ Rows(const Stack& st, int64_t first, int K) : w(st.w + first * K) {}
    };
    struct X {
        v4u x[LD];
        __device__ __forceinline__ void load(const Act* base, uint32_t row, int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < LD; ++u) x[u] = load_at(base, row + 4 * min(k + u * 16 + q * 4, K - 4));
        }
        __device__ __forceinline__ void tail(int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < LD; ++u) x[u] &= k + u * 16 + q * 4 < K ? ~0u : 0u;
        }
    };
    struct Unit {
        X w;
        __device__ __forceinline__ void load(const Rows& rows, int r, int k, int K, int q) {
            w.load(rows.w, (uint32_t)(r * K) * 4, k, K, q);
        }
        __device__ __forceinline__ void tail(int k, int K, int q) { w.tail(k, K, q); }
    };
    template <int NM, int NP>
    __device__ static __forceinline__ void multiply(f32x4 (&tot)[NM], const Unit (&w)[NM], const X (&x)[NP],
                                                    const Stack&) {
        static_assert(NP == 1, "fp32 activations are whole");
#pragma unroll
        for (int u = 0; u < LD; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int m = 0; m < NM; ++m)
                    tot[m] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[0].x[u][j]),
                                                                  __uint_as_float(w[m].w.x[u][j]), tot[m], 0, 0, 0);
    }
};

template <int GROUP>
struct FmtW4 {
    typedef uint16_t Act;
    static constexpr int UK = kW4Chunk, PARTS = 2, BATCH = 1;
    static constexpr int NG = W4Chunk<GROUP>::NG, STEPS = GROUP / 32;
    typedef W4Stack Stack;
    typedef W4Rows<GROUP> Rows;
    struct X {
        v4u x[4];
        __device__ __forceinline__ void load(const Act* base, uint32_t row, int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = load_at(base, row + 2 * min(k + u * 32 + q * 8, K - 8));
        }
        __device__ __forceinline__ void tail(int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] &= k + u * 32 + q * 8 < K ? ~0u : 0u;
        }
    };
    struct Unit {
        W4Chunk<GROUP> w;
        __device__ __forceinline__ void load(const Rows& rows, int r, int k, int K, int q) {
            w.load(rows, r, k / kW4Chunk, K, q);
        }
        __device__ __forceinline__ void tail(int, int, int) {}  // codes are finite
    };
    template <int NM, int NP>
    __device__ static __forceinline__ void multiply(f32x4 (&tot)[NM], const Unit (&w)[NM], const X (&x)[NP],
                                                    const Stack& st) {
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
                const float sc = w[m].w.scale(g), off = w[m].w.offset(st.has_zeros, g);
#pragma unroll
                for (int i = 0; i < 4; ++i) tot[m][i] = fmaf(sc, fmaf(-off, xs[i], acc[m][i]), tot[m][i]);
            }
        }
    }
};

// one of two by value (a conditional between two kernel arguments themselves would
// become a load through a chosen address, which waits for every load before it)
template <typename T>
__device__ __forceinline__ T pick(bool first, T a, T b) { return first ? a : b; }
__device__ __forceinline__ FmtBf16::Stack pick(bool first, FmtBf16::Stack a, FmtBf16::Stack b) {
    return {pick(first, a.w, b.w)};
}
__device__ __forceinline__ FmtF32::Stack pick(bool first, FmtF32::Stack a, FmtF32::Stack b) {
    return {pick(first, a.w, b.w)};
}
__device__ __forceinline__ W4Stack pick(bool first, W4Stack a, W4Stack b) {
    return {pick(first, a.codes, b.codes), pick(first, a.scales, b.scales), pick(first, a.zeros, b.zeros),
            pick(first, a.groups, b.groups), a.has_zeros};
}

template <class F>
struct FewParams {
    typedef typename F::Act Act;
    typename F::Stack up[2], up_sh[2], down, down_sh;  // up: W_gate, W_up
    const Act* x;
    const double* logits;  // [T, E]
    const int32_t* e2g;
    int32_t* topk_idx;
    float* topk_w;
    int32_t* slot_group;
    float* slot_gate;
    // hidden values, [T*k, f] of the slots then [T, fs] of the shared experts;
    // bf16 layers: the high parts, then as many low parts
    Act* h;
    Act* out;
    int32_t* done;   // [tiles of d] workgroups that have finished, when split > 1
    float* partial;  // [tiles of d][split][16 tokens][16 columns]
    int T, k, G, E, d, f, fs, norm, split;
    int64_t h_part;  // elements of one part
};

// Runs n steps over two register buffers: load(buffer, step) of step i + 2 follows
// multiply(buffer, step) of step i. Every load of the loop is issued on every path
// (a step past the last loads the last one again), so that the compiler can count
// the loads that are younger than the ones it has to wait for.
template <class Buf, class Load, class Multiply>
__device__ __forceinline__ void pingpong(int n, Load load, Multiply multiply) {
    if (n <= 0) return;
    Buf b0, b1;
    // Neither loads nor multiplies move past here. (The memory clobber keeps the
    // loads in front of the loop and at its end from being merged into ones at its
    // start, which would be waited for at once.)
    auto fence = [] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    load(b0, 0);
    load(b1, min(1, n - 1));
    fence();
    int i = 0;
    for (; i + 2 < n; i += 2) {
        multiply(b0, i);
        fence();
        load(b0, i + 2);
        fence();
        multiply(b1, i + 1);
        fence();
        load(b1, min(i + 3, n - 1));
        fence();
    }
    multiply(b0, i);
    if (i + 1 < n) multiply(b1, i + 1);
}

template <class F, int NM, int NP>
struct FewBuf {
    typename F::Unit w[F::BATCH][NM];
    typename F::X x[F::BATCH][NP];
};

// sum of the waves' partials of D element (row, col)
template <int WAVES>
__device__ __forceinline__ float tile_sum(const f32x4 (*part)[64], int row, int col) {
    const float* p = (const float*)&part[0][(row >> 2) * 16 + col] + (row & 3);
    float v = p[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += p[w * 256];
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
__global__ __launch_bounds__(kUpThreads, kUpWgsPerCu * kUpThreads / 256) void few_up_kernel(FewParams<F> p) {
    constexpr int WAVES = kUpThreads / 64, BATCH = F::BATCH;
    __shared__ __align__(16) f32x4 part[2][2][WAVES][64];  // [parity of the item][matrix]
    __shared__ SelectSmem sm;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int r16 = lane & 15, q = lane >> 4;
    const int T = p.T, k = p.k, d = p.d, f = p.f, fs = p.fs;
    const int sh_tiles = ceil_div(fs, kFewCols), tiles = ceil_div(f, kFewCols);

    // the picks, the reached segments, and where each token's gate of a segment is
    if (tid < kSetWords) sm.reached[tid] = 0;
    for (int i = tid; i < BMOE_MAX_EXPERTS * kFewTok / 2; i += kUpThreads) ((uint32_t*)sm.slot_of)[i] = ~0u;
    __syncthreads();
    if (wave * 4 < T) {
        if (p.E <= 64) few_select<4>(p.logits, p.e2g, sm, T, p.E, p.G, k, wave, lane);
        else few_select<16>(p.logits, p.e2g, sm, T, p.E, p.G, k, wave, lane);
    }
    __syncthreads();
    if (tid < p.G && (sm.reached[tid >> 5] >> (tid & 31)) & 1u) sm.segs[members_below(sm.reached, tid)] = (int16_t)tid;
    if (tid < T * k) {
        const int t = tid / k, i = tid - t * k;
        const int g = pick_group(sm.pk[t][i]);
        const bool known = (unsigned)g < (unsigned)p.G;
        float mine = 0.f, all = 0.f;
        bool first = known;
        for (int j = 0; j < k; ++j) {
            const float e = sm.pe[t][j];
            const bool same = pick_group(sm.pk[t][j]) == g;
            all += e;
            if (same && j < i) first = false;
            mine += same && j >= i ? e : 0.f;
        }
        const float inv = 1.f / (p.norm ? all : sm.sum[t]);
        sm.gate[tid] = mine * inv;
        if (first) sm.slot_of[members_below(sm.reached, g)][t] = (int16_t)tid;
        if (blockIdx.x == 0) {
            p.topk_idx[tid] = pick_expert(sm.pk[t][i]);
            p.topk_w[tid] = sm.pe[t][i] * inv;
            p.slot_group[tid] = first ? g : -1;
            p.slot_gate[tid] = first ? mine * inv : 0.f;
        }
    }
    const int items = sh_tiles + members(sm.reached) * tiles;
    __syncthreads();

    const uint32_t xr = (uint32_t)(min(r16, T - 1) * d) * sizeof(typename F::Act);
    const int units = ceil_div(d, F::UK), steps = ceil_div(ceil_div(units, WAVES), BATCH);  // steps of an item
    // (kept in scalar registers: the addresses of every load follow from them)
    const int wg = scalar(blockIdx.x), wgs = scalar(gridDim.x);
    const int mine = scalar(wg < items ? div_uniform(items - 1 - wg, wgs) + 1 : 0);
    typedef FewBuf<F, 2, 1> Buf;
    auto load = [&](Buf& b, int at) __attribute__((always_inline)) {
        const int of = div_uniform(at, steps), step = at - of * steps, l_item = wg + of * wgs;
        const bool sh = l_item < sh_tiles;
        const int a = sh ? 0 : div_uniform(l_item - sh_tiles, tiles), N = pick(sh, fs, f);
        const int n0 = (sh ? l_item : l_item - sh_tiles - a * tiles) * kFewCols;
        const int seg = sh ? 0 : scalar(sm.segs[a]);
        const typename F::Rows gate(pick(sh, p.up_sh[0], p.up[0]), (int64_t)seg * N + n0, d);
        const typename F::Rows up(pick(sh, p.up_sh[1], p.up[1]), (int64_t)seg * N + n0, d);
        const int r = min(r16, N - 1 - n0);
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int u = min(wave + WAVES * (BATCH * step + i), units - 1);
            b.w[i][0].load(gate, r, u * F::UK, d, q);
            b.w[i][1].load(up, r, u * F::UK, d, q);
            b.x[i][0].load(p.x, xr, u * F::UK, d, q);
        }
    };
    f32x4 tot[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    int item = wg, step = 0, parity = 0;
    auto multiply = [&](Buf& b, int) __attribute__((always_inline)) {
        const bool sh = item < sh_tiles;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int kk = (wave + WAVES * (BATCH * step + i)) * F::UK;
            b.w[i][0].tail(kk, d, q);
            b.w[i][1].tail(kk, d, q);
            b.x[i][0].tail(kk, d, q);
            F::multiply(tot, b.w[i], b.x[i], p.up[0]);
        }
        if (++step < steps) return;
        step = 0;
        part[parity][0][wave][lane] = tot[0];
        part[parity][1][wave][lane] = tot[1];
        tot[0] = tot[1] = f32x4{0.f, 0.f, 0.f, 0.f};
        // one barrier an item: the other parity's partials were read before it
        lds_reads_done();
        wg_barrier();
        const int a = sh ? 0 : div_uniform(item - sh_tiles, tiles), N = pick(sh, fs, f);
        const int col = (sh ? item : item - sh_tiles - a * tiles) * kFewCols + (tid & 15), token = tid >> 4;
        if (token < T && col < N) {
            const int slot = sh ? token : sm.slot_of[a][token];
            if (slot >= 0) {
                const float g = tile_sum<WAVES>(part[parity][0], token, tid & 15), u = tile_sum<WAVES>(part[parity][1], token, tid & 15);
                const float v = silu_mul(g, u) * (sh ? 1.f : sm.gate[slot]);
                const int64_t at = (sh ? (int64_t)T * k * f : 0) + (int64_t)slot * N + col;
                store_hidden(p.h, p.h_part, at, v);
            }
        }
        parity ^= 1;
        item += wgs;
    };
    pingpong<Buf>(mine * steps, load, multiply);
}

// PACK: at most 8 tokens, both parts of their hidden values in one A operand
template <class F, bool PACK>
__global__ __launch_bounds__(kDownThreads, kDownWgsPerCu * kDownThreads / 256) void few_down_kernel(FewParams<F> p) {
    constexpr int WAVES = kDownThreads / 64, BATCH = F::BATCH, NP = PACK ? 1 : F::PARTS;
    __shared__ __align__(16) f32x4 part[WAVES][64];
    __shared__ uint32_t reached[kSetWords];
    // by place among the reached segments (ascending): the segment, the tokens that
    // call it, each token's slot (0 where it has none)
    __shared__ int16_t segs[BMOE_MAX_EXPERTS];
    __shared__ uint32_t callers[BMOE_MAX_EXPERTS];
    __shared__ uint8_t slot_of[BMOE_MAX_EXPERTS][kFewTok];
    __shared__ int last_s;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int r16 = lane & 15, q = lane >> 4;
    const int T = p.T, k = p.k, d = p.d, f = p.f, fs = p.fs;
    const int wg = scalar(blockIdx.x), tile = div_uniform(wg, p.split), n0 = tile * kFewCols;
    const int g = tid < T * k ? p.slot_group[tid] : -1;
    const bool valid = (unsigned)g < (unsigned)p.G;
    if (tid < kSetWords) reached[tid] = 0;
    callers[tid] = 0;
    for (int i = tid; i < BMOE_MAX_EXPERTS * kFewTok / 4; i += kDownThreads) ((uint32_t*)slot_of)[i] = 0;
    __syncthreads();
    if (valid) atomicOr(&reached[g >> 5], 1u << (g & 31));
    __syncthreads();
    if (valid) {
        const int place = members_below(reached, g), t = tid / k;
        segs[place] = (int16_t)g;
        atomicOr(&callers[place], 1u << t);
        slot_of[place][t] = (uint8_t)tid;
    }
    const int per = ceil_div(f, F::UK), routed = members(reached) * per, units = routed + ceil_div(fs, F::UK);
    __syncthreads();
    // the waves of the tile's workgroups take the units in turn
    const int first = (wg - tile * p.split) * WAVES + wave, stride = p.split * WAVES;
    const int steps = ceil_div(div_uniform(units + stride - 1, stride), BATCH);
    const int wr = min(r16, d - 1 - n0), token = PACK ? r16 & 7 : r16;
    typedef FewBuf<F, 1, NP> Buf;
    auto load = [&](Buf& b, int step) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int u = min(first + stride * (BATCH * step + i), units - 1);
            const bool sh = u >= routed;
            const int a = sh ? 0 : div_uniform(u, per);
            const int kk = (sh ? u - routed : u - a * per) * F::UK, width = pick(sh, fs, f);
            const int slot = sh ? min(token, T - 1) : slot_of[a][token];
            const int seg = sh ? 0 : scalar(segs[a]);
            const typename F::Rows rows(pick(sh, p.down_sh, p.down), (int64_t)seg * d + n0, width);
            b.w[i][0].load(rows, wr, kk, width, q);
            // (hidden values are below 2^32 bytes: 16 tokens, 16 slots, 2^20 columns)
            const uint32_t hr = (uint32_t)((sh ? (int64_t)T * k * f : 0) + (int64_t)slot * width +
                                           (PACK && r16 >= 8 ? p.h_part : 0)) * sizeof(typename F::Act);
#pragma unroll
            for (int j = 0; j < NP; ++j) b.x[i][j].load(p.h + j * p.h_part, hr, kk, width, q);
        }
    };
    f32x4 tot = {0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](Buf& b, int step) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int u = first + stride * (BATCH * step + i);
            const bool sh = u >= routed;
            const int a = sh ? 0 : div_uniform(u, per), width = pick(sh, fs, f);
            const int kk = u < units ? (sh ? u - routed : u - a * per) * F::UK : width;
            b.w[i][0].tail(kk, width, q);
#pragma unroll
            for (int j = 0; j < NP; ++j) b.x[i][j].tail(kk, width, q);
            f32x4 acc[1] = {{0.f, 0.f, 0.f, 0.f}};
            F::multiply(acc, b.w[i], b.x[i], p.down);
            // only the tokens that call the segment take its products
            const uint32_t who = sh ? 0xffffu : callers[a];
#pragma unroll
            for (int j = 0; j < 4; ++j) tot[j] += (who >> ((PACK ? 4 * (q & 1) : 4 * q) + j)) & 1u ? acc[0][j] : 0.f;
        }
    };
    pingpong<Buf>(steps, load, multiply);
    part[wave][lane] = tot;
    __syncthreads();
    const int t = tid >> 4, col = tid & 15;
    float v = tile_sum<WAVES>(part, t, col);
    if constexpr (PACK) v += t < 8 ? tile_sum<WAVES>(part, t + 8, col) : 0.f;
    if (p.split > 1) {
        // the parts meet in memory; the workgroup that finishes last adds them in
        // order. Relaxed accesses of agent scope go past the caches of one XCD, and
        // the wait orders them; fences would write back and drop whole L2 caches
        // (81 us instead of 11 for one token of the fine-grained layer).
        float* mine = p.partial + (size_t)blockIdx.x * kDownThreads;
        __hip_atomic_store(mine + tid, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        wait_vmcnt<0>();  // (this wave's part is written)
        __syncthreads();
        if (tid == 0)
            last_s = __hip_atomic_fetch_add(p.done + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == p.split - 1;
        __syncthreads();
        if (!last_s) return;
        const float* all = p.partial + (size_t)tile * p.split * kDownThreads;
        float parts[kSplitMax];
#pragma unroll
        for (int i = 0; i < kSplitMax; ++i)
            if (i < p.split)
                parts[i] = __hip_atomic_load(all + i * kDownThreads + tid, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        v = parts[0];
#pragma unroll
        for (int i = 1; i < kSplitMax; ++i)
            if (i < p.split) v += parts[i];
    }
    if (t < T && n0 + col < d) {
        typename F::Act* o = p.out + (size_t)t * d + n0 + col;
        if constexpr (sizeof(typename F::Act) == 2) *o = f32_to_bf16(v);
        else *o = v;
    }
}

// items of few_up_kernel, at most
int64_t up_items(int T, int k, int G, int f, int fs) {
    const int64_t slots = (int64_t)T * k, most = slots < G ? slots : G;
    return most * ceil_div(f, kFewCols) + ceil_div(fs, kFewCols);
}

// Workgroups that share 16 output columns: as many as the chip holds at once, where
// the columns are fewer
int most_splits(int d) {
    const int tiles = ceil_div(d, kFewCols), n = kDownWgsPerCu * 256 / tiles;
    return n < 1 ? 1 : n > kSplitMax ? kSplitMax : n;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
size_t logit_bytes(int T, int E) { return round256((size_t)T * E * sizeof(double)); }
size_t done_bytes(int d) { return round256((size_t)ceil_div(d, kFewCols) * sizeof(int32_t)); }
size_t partial_bytes(int d) {
    return most_splits(d) == 1 ? 0 : (size_t)ceil_div(d, kFewCols) * most_splits(d) * kTile * sizeof(float);
}

template <typename Act>
void launch_logits(const FewArgs& a, int32_t* done, hipStream_t s) {
    const int nch = a.d / Vec<Act>::N, tiles = ceil_div(a.d, kFewCols);
    auto go = [&](auto kernel, int tokens) {
        hipLaunchKernelGGL(kernel, dim3(a.E, ceil_div(a.T, tokens)), dim3(kLogitThreads), 0, s, (const uint4*)a.x,
                           (const uint4*)a.w.w_router, a.w.bias, (double*)a.ws, a.T, a.E, nch, done, tiles);
    };
    if (a.T == 1) go(few_logits_kernel<Act, 1>, 1);
    else if (a.T == 2) go(few_logits_kernel<Act, 2>, 2);
    else go(few_logits_kernel<Act, kLogitTokens>, kLogitTokens);
}

template <class F, class ToStack>
hipError_t launch_few_t(const FewArgs& a, ToStack st, hipStream_t s) {
    typedef typename F::Act Act;
    FewParams<F> p;
    p.up[0] = st(a.w.gate, (int64_t)a.G * a.f, a.d);
    p.up[1] = st(a.w.up, (int64_t)a.G * a.f, a.d);
    p.down = st(a.w.down, (int64_t)a.G * a.d, a.f);
    p.up_sh[0] = st(a.w.gate_sh, a.fs, a.d);
    p.up_sh[1] = st(a.w.up_sh, a.fs, a.d);
    p.down_sh = st(a.w.down_sh, a.d, a.fs);
    p.x = (const Act*)a.x;
    p.logits = (const double*)a.ws;
    p.e2g = a.w.e2g;
    p.topk_idx = a.topk_idx;
    p.topk_w = a.topk_w;
    p.slot_group = a.slot_group;
    p.slot_gate = a.slot_gate;
    char* ws = (char*)a.ws + logit_bytes(a.T, a.E);
    p.done = (int32_t*)ws;
    ws += done_bytes(a.d);
    p.partial = (float*)ws;
    p.h = (Act*)(ws + partial_bytes(a.d));
    p.out = (Act*)a.out;
    p.T = a.T;
    p.k = a.k;
    p.G = a.G;
    p.E = a.E;
    p.d = a.d;
    p.f = a.f;
    p.fs = a.fs;
    p.norm = a.norm;
    p.h_part = (int64_t)a.T * a.k * a.f + (int64_t)a.T * a.fs;
    const int64_t slots = (int64_t)a.T * a.k, most = slots < a.G ? slots : a.G;
    const int64_t units = most * ceil_div(a.f, F::UK) + ceil_div(a.fs, F::UK);
    p.split = most_splits(a.d);
    if (units < (int64_t)p.split * (kDownThreads / 64)) p.split = (int)ceil_div64(units, kDownThreads / 64);  // a unit a wave
    launch_logits<Act>(a, p.done, s);
    const int64_t items = up_items(a.T, a.k, a.G, a.f, a.fs), room = (int64_t)kUpWgsPerCu * persistent_workgroups();
    hipLaunchKernelGGL((few_up_kernel<F>), dim3((unsigned)(items < room ? items : room)), dim3(kUpThreads), 0, s, p);
    const dim3 grid((unsigned)(ceil_div(a.d, kFewCols) * p.split));
    if (F::PARTS == 2 && a.T <= 8) hipLaunchKernelGGL((few_down_kernel<F, F::PARTS == 2>), grid, dim3(kDownThreads), 0, s, p);
    else hipLaunchKernelGGL((few_down_kernel<F, false>), grid, dim3(kDownThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace

size_t few_ws_bytes(int T, int E, int k, int d, int f, int fs) {
    return logit_bytes(T, E) + done_bytes(d) + partial_bytes(d) + ((size_t)T * k * f + (size_t)T * fs) * 4;
}

hipError_t launch_few(const FewArgs& a, hipStream_t s) {
    auto w4 = [&](const bmoe_matrix& m, int64_t rows, int K) {
        return w4_stack(m.w, m.scales, m.zeros, rows, K, a.w.group);
    };
    if (a.w.group == 32) return launch_few_t<FmtW4<32>>(a, w4, s);
    if (a.w.group == 64) return launch_few_t<FmtW4<64>>(a, w4, s);
    if (a.w.group == 128) return launch_few_t<FmtW4<128>>(a, w4, s);
    if (a.dtype == BMOE_BF16)
        return launch_few_t<FmtBf16>(
            a, [](const bmoe_matrix& m, int64_t, int) { return FmtBf16::Stack{(const uint16_t*)m.w}; }, s);
    return launch_few_t<FmtF32>(
        a, [](const bmoe_matrix& m, int64_t, int) { return FmtF32::Stack{(const float*)m.w}; }, s);
}

}  // namespace bmoe
