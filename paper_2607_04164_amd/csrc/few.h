// The whole layer for at most 16 tokens (Sec. 2.1 with the map of Eq. 2).
//
// With so few tokens all of them fit one MFMA tile, so nothing is permuted: a
// reached segment's weights are multiplied with every token, and a token that
// does not call the segment is left out where its hidden values would be stored.
//   few_logits_kernel  one workgroup per expert (and four tokens): the gate logits
//                      in float64 (bf16 and fp32 products are exact there), so
//                      near ties need no second look;
//   few_up_kernel      items of 16 or 32 hidden columns of a reached segment (or of
//                      the shared experts), dealt out to the workgroups. Every
//                      workgroup selects the top-k from the logits by itself, which
//                      costs less than another launch: silu(Wg x) * (Wu x), times
//                      the token's gate of that segment, to the workspace;
//   few_down_kernel    16 to 64 output columns a workgroup: the sum over the reached
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
// of fp32 weights, 256 of 4-bit ones (see w4.h): a 128-byte line of each row.
// Hidden values of bf16 layers are kept as the sum of two bf16 (16 bits of
// significand) and multiplied as such, since the matrix cores idle here anyway;
// so the layer's output is rounded once. Up to eight tokens have their high parts
// in rows 0..7 of the A operand and their low parts in rows 8..15. In 4-bit layers
// hidden values and outputs that are not finite are formed again as they are
// defined (see w4.h).
//
// d 2048, 60 experts, top-4, 15 segments, d_ff 1408, kernel by kernel (medians over
// three sets of weights in turn, part of which stays in the last-level cache): one token
// 3.0 + 14.4 + 8.9 us (63 MB on average; of the second 3.5 before its first weights), 16
// tokens 4.6 + 29.4 + 18.7 (177 MB), one token in 4 bits 2.8 + 10.4 + 7.8 (17 MB: latency).
// Two tokens of d 4096, d_ff 14336 that reach three or four segments: 4.6 + 122 + 64 (1060
// to 1410 MB); six of them in 4 bits 4.8 + 63 + 42 (331 MB: two waves a SIMD by registers,
// each with one unit on its way). Down of more than eight tokens is short of registers: at
// three waves a SIMD bf16 spills 8 bytes a lane, at two 4-bit groups of 32 spill 44.
#pragma once

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
constexpr int kSplitMax = 8;  // workgroups that share their output columns
constexpr int kLogitTokens = 4;  // tokens of a few_logits_kernel workgroup
constexpr int kMaxSlots = kFewTok * BMOE_MAX_TOPK;
static_assert(kFewTok == 16, "one MFMA tile of tokens");
constexpr int kTile = kFewTok * kFewCols;  // outputs of a tile
static_assert(kMaxSlots <= kTile && BMOE_MAX_EXPERTS <= kTile, "a thread per slot and per expert");
static_assert(2 * kTile <= kUpThreads && kTile == kDownThreads, "a thread per output of a tile");

// A value that the wave shares, in a scalar register: left to itself the compiler
// keeps some of them, and the addresses that follow from them, in vector registers
// (up kernel: 203 registers, 130 this way).
__device__ __forceinline__ int scalar(int v) {
    asm("" : "+v"(v));  // (nothing is known of v here, so the next step stays)
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int div_uniform(int a, int b) { return scalar((int)((unsigned)a / (unsigned)b)); }

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
        const int g = e2g[e];  // (outside [0, G): sent nowhere, as brownout_moe_route takes it)
        key[j] = (e << 16) | ((unsigned)g < (unsigned)G ? g + 1 : 0);
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
// Place: tiles of 16 rows (fewer at the matrix's end) of NR matrices, from row `first`
// of each on; tile m is rows 16 (m / NR) .. of matrix m % NR. Set: a wave's unit of UK
// columns of NM such tiles; X: the same columns of the tokens, from an address that the
// wave shares and the lane's row's byte offset. RAGGED: columns past K read the row's
// last ones and tail() zeroes them (in every unit: a branch would cost copies of the
// buffers). multiply() adds the products with NP parts of the activations (their sum is
// the value) to tot. PARTS: parts of a hidden value; DOWN_BATCH: units of a register
// buffer there; UP_TILES (at most), DOWN_TILES: tiles of 16 columns that a wave takes with
// the same activations, PACK_TILES: for up to eight tokens; UP_WAVES, DOWN_WAVES: waves per
// SIMD, by registers. 4-bit weights are a quarter of the bytes, and with one tile the
// activations' loads, not the weights', bound them: 86 and 58 us for six tokens of wide
// experts. bf16, down: two tiles take 58.6 us for the layer of 16 tokens, one 63.2, but
// 28.7 against 27.1 for the layer of one token, where they leave fewer waves.

// bf16 and fp32 weights: 16 bytes of a row are EPC columns
template <typename ActT>
struct FmtPlain {
    typedef ActT Act;
    static constexpr bool kBf16 = sizeof(Act) == 2;
    static constexpr int EPC = 16 / sizeof(Act), LD = 2, UK = 4 * EPC * LD, PARTS = kBf16 ? 2 : 1;
    static constexpr bool PAIRS = true, X_IN_LDS = false, OFFSET = false;
    static constexpr int UP_TILES = PARTS, UP_WAVES = 4;  // (at most, of bf16)
    static constexpr int DOWN_TILES = PARTS, PACK_TILES = 1, DOWN_BATCH = 2, DOWN_WAVES = 3;
    struct Stack {
        const Act* w;
        bool has_zeros;  // (no meaning here)
    };
    template <int NR, int NM>
    struct Place {
        const Act* w[NR];
        uint32_t row[NM / NR];  // the lane's row of a tile, in bytes
        __device__ __forceinline__ void set(const Stack& s0, const Stack& s1, int64_t first, int left, int K, int r16, int) {
            w[0] = s0.w + first * K;
            if constexpr (NR == 2) w[NR - 1] = s1.w + first * K;
#pragma unroll
            for (int t = 0; t < NM / NR; ++t) row[t] = (uint32_t)(min(16 * t + r16, left - 1) * K) * sizeof(Act);
        }
    };
    struct X {
        v4u x[LD];
        template <bool RAGGED>
        __device__ __forceinline__ void load(const void* base, uint32_t row, int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < LD; ++u) {
                const int col = k + (u * 4 + q) * EPC;
                x[u] = load_at(base, row + sizeof(Act) * (RAGGED ? min(col, K - EPC) : col));
            }
        }
        __device__ __forceinline__ void tail(int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < LD; ++u) x[u] &= k + (u * 4 + q) * EPC < K ? ~0u : 0u;
        }
    };
    template <int NM>
    struct Set {
        X w[NM];
        template <bool RAGGED, int NR>
        __device__ __forceinline__ void load(const Place<NR, NM>& at, int k, int K, int q) {
#pragma unroll
            for (int m = 0; m < NM; ++m) w[m].template load<RAGGED>(at.w[m % NR], at.row[m / NR], k, K, q);
        }
        __device__ __forceinline__ void tail(int k, int K, int q) {
#pragma unroll
            for (int m = 0; m < NM; ++m) w[m].tail(k, K, q);
        }
    };
    template <int NM, int NP>
    __device__ static __forceinline__ void multiply(f32x4 (&tot)[NM], const Set<NM>& w, const X (&x)[NP], bool) {
#pragma unroll
        for (int u = 0; u < LD; ++u)
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                if constexpr (kBf16) {
#pragma unroll
                    for (int m = 0; m < NM; ++m) tot[m] = mfma16(x[p].x[u], w.w[m].x[u], tot[m]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int m = 0; m < NM; ++m)
                            tot[m] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                                __uint_as_float(x[p].x[u][j]), __uint_as_float(w.w[m].x[u][j]), tot[m], 0, 0, 0);
                }
            }
    }
};
typedef FmtPlain<uint16_t> FmtBf16;
typedef FmtPlain<float> FmtF32;

template <int GROUP>
struct FmtW4 {
    typedef uint16_t Act;
    static constexpr int UK = kW4Unit, LD = UK / 32, PARTS = 2;
    static constexpr bool PAIRS = false, X_IN_LDS = true, OFFSET = true;
    static constexpr int UP_TILES = 2, UP_WAVES = 2;
    static constexpr int DOWN_TILES = 4, PACK_TILES = 4, DOWN_BATCH = 1, DOWN_WAVES = 2;
    static constexpr int NG = W4Unit<GROUP>::NG, STEPS = GROUP / 32;
    typedef W4Stack Stack;
    // the product of a row of W with x (the sum of PARTS_OF_X parts, `part` apart), as defined
    template <int PARTS_OF_X>
    __device__ static __forceinline__ double defined(const Stack& w, int64_t row, int K, const uint16_t* x, int64_t part) {
        return w4_defined<GROUP>(w, row, K, [&](int k, float* f) {
            Vec<uint16_t>::load(*(const uint4*)(x + k), f);
            if constexpr (PARTS_OF_X == 2) {
                float low[8];
                Vec<uint16_t>::load(*(const uint4*)(x + part + k), low);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] += low[j];  // (exact: 16 bits)
            }
        });
    }
    template <int NR, int NM>
    using Place = W4Place<GROUP, NR, NM>;
    struct X {
        v4u x[LD];
        template <bool RAGGED>
        __device__ __forceinline__ void load(const void* base, uint32_t row, int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < LD; ++u)
                x[u] = load_at(base, row + 2 * (RAGGED ? min(k + u * 32 + q * 8, K - 8) : k + u * 32 + q * 8));
        }
        __device__ __forceinline__ void tail(int k, int K, int q) {
#pragma unroll
            for (int u = 0; u < LD; ++u) x[u] &= k + u * 32 + q * 8 < K ? ~0u : 0u;
        }
    };
    template <int NM>
    struct Set {
        static_assert(NM == 4, "four tiles");
        W4Unit<GROUP> w;
        template <bool RAGGED, int NR>
        __device__ __forceinline__ void load(const Place<NR, NM>& at, int k, int K, int q) {
            w.load(at, k / kW4Unit, K, q);
        }
        __device__ __forceinline__ void tail(int k, int K, int) { w.settle(k, K); }  // (codes are finite)
    };
    template <int NM, int NP>
    __device__ static __forceinline__ void multiply(f32x4 (&tot)[NM], const Set<NM>& w, const X (&x)[NP], bool has_zeros) {
        const v4u ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        const W4Spread<GROUP> groups(w.w, has_zeros);
        const int q = (threadIdx.x & 63) >> 4;
        v4u c[NM];
        // A group is scaled while the next one is multiplied. (The fences keep the
        // compiler from running more groups side by side than there are registers.)
        f32x4 acc[2][NM], xs[2];
        float xa = 0.f;  // xs of group 4i + q
        auto flush = [&](int g) __attribute__((always_inline)) {
            xa = q == (g & 3) ? xs[g & 1][0] : xa;
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                const float sc = groups.scale(m, g);
#pragma unroll
                for (int i = 0; i < 4; ++i) tot[m][i] = fmaf(sc, acc[g & 1][m][i], tot[m][i]);
                if (g % 4 == 3 || g == NG - 1) tot[m] = groups.add_offset(tot[m], xa, m, g);
                asm volatile("" : "+v"(tot[m]));  // here, and not where tot is used next
            }
        };
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            xs[g & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < NM; ++m) acc[g & 1][m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = g * STEPS; u < (g + 1) * STEPS; ++u) {
                if (u % 4 == 0) {
#pragma unroll
                    for (int m = 0; m < NM; ++m) c[m] = w4_transpose(w.w.codes[m][u / 4]);
                }
                v4u b[NM];
#pragma unroll
                for (int m = 0; m < NM; ++m) b[m] = w4_unpack(c[m][u % 4]);
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const v4u a = w4_order(x[p].x[u]);
                    xs[g & 1] = mfma16(ones, a, xs[g & 1]);
#pragma unroll
                    for (int m = 0; m < NM; ++m) acc[g & 1][m] = mfma16(a, b[m], acc[g & 1][m]);
                }
            }
            if (g > 0) flush(g - 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        flush(NG - 1);
    }
};

// one of two by value (a conditional between two kernel arguments themselves would
// become a load through a chosen address, which waits for every load before it)
template <typename T>
__device__ __forceinline__ T pick(bool first, T a, T b) { return first ? a : b; }
template <typename Act>
__device__ __forceinline__ typename FmtPlain<Act>::Stack pick_stack(bool first, typename FmtPlain<Act>::Stack a,
                                                                    typename FmtPlain<Act>::Stack b) {
    return {pick(first, a.w, b.w), false};
}
__device__ __forceinline__ FmtBf16::Stack pick(bool first, FmtBf16::Stack a, FmtBf16::Stack b) {
    return pick_stack<uint16_t>(first, a, b);
}
__device__ __forceinline__ FmtF32::Stack pick(bool first, FmtF32::Stack a, FmtF32::Stack b) {
    return pick_stack<float>(first, a, b);
}
__device__ __forceinline__ W4Stack pick(bool first, W4Stack a, W4Stack b) {
    return {pick(first, a.codes, b.codes), pick(first, a.scales, b.scales), pick(first, a.zeros, b.zeros),
            pick(first, a.groups, b.groups), pick(first, a.has_zeros, b.has_zeros)};
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

// Neither loads nor multiplies move past a fence. (The memory clobber keeps the
// loads in front of a loop and at its end from being merged into ones at its start,
// which would be waited for at once.)
__device__ __forceinline__ void step_fence() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Both run n steps over two register buffers of weights. Every load of their loops
// is issued on every path (a step past the last loads the last one again), so that
// the compiler can count the loads that are younger than the ones it waits for.
//
// stream_pairs: the activations have two buffers too; the loads of step i + 2 follow
// the multiply of step i.
template <class W, class X, class LoadW, class LoadX, class Multiply>
__device__ __forceinline__ void stream_pairs(int n, LoadW load_w, LoadX load_x, Multiply multiply) {
    W w0, w1;
    X x0, x1;
    load_w(w0, 0);
    load_x(x0, 0);
    load_w(w1, min(1, n - 1));
    load_x(x1, min(1, n - 1));
    step_fence();
    int i = 0;
    for (; i + 2 < n; i += 2) {
        multiply(w0, x0);
        step_fence();
        load_w(w0, i + 2);
        load_x(x0, i + 2);
        step_fence();
        multiply(w1, x1);
        step_fence();
        load_w(w1, min(i + 3, n - 1));
        load_x(x1, min(i + 3, n - 1));
        step_fence();
    }
    multiply(w0, x0);
    if (i + 1 < n) multiply(w1, x1);
}
// stream_weights: one buffer of activations, which come from the L2 cache; they are
// loaded just before the next step's weights (loads return in order: after them they
// would be waited for together).
template <class W, class X, class LoadW, class LoadX, class Multiply>
__device__ __forceinline__ void stream_weights(int n, LoadW load_w, LoadX load_x, Multiply multiply) {
    W w0, w1;
    X x;
    load_w(w0, 0);
    step_fence();
    int i = 0;
    for (; i + 1 < n; i += 2) {
        load_x(x, i);
        step_fence();
        load_w(w1, i + 1);
        step_fence();
        multiply(w0, x);
        step_fence();
        load_x(x, i + 1);
        step_fence();
        load_w(w0, min(i + 2, n - 1));
        step_fence();
        multiply(w1, x);
        step_fence();
    }
    if (i < n) {
        load_x(x, i);
        multiply(w0, x);
    }
}
// Plain weights: 15.7 us (one token, up) by pairs, 19.0 with one buffer of
// activations; 4-bit weights, whose units hold four times the columns, have no
// registers for the second one.
template <class F, class W, class X, class LoadW, class LoadX, class Multiply>
__device__ __forceinline__ void stream_steps(int n, LoadW load_w, LoadX load_x, Multiply multiply) {
    if (n <= 0) return;
    if constexpr (F::PAIRS) stream_pairs<W, X>(n, load_w, load_x, multiply);
    else stream_weights<W, X>(n, load_w, load_x, multiply);
}

template <class F, int BATCH, int NM>
struct FewW {
    typename F::template Set<NM> w[BATCH];
};
template <class F, int BATCH, int NP>
struct FewX {
    typename F::X x[BATCH][NP];
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

// What a workgroup of few_up_kernel works on: item i is `cols` hidden columns, of the
// shared experts first, then of the reached segments in turn.
struct UpItem {
    bool shared;
    int place, n0;  // place among the reached segments
    __device__ __forceinline__ UpItem(int i, int cols, int sh_tiles, int tiles) {
        shared = i < sh_tiles;
        place = shared ? 0 : div_uniform(i - sh_tiles, tiles);
        n0 = (shared ? i : i - sh_tiles - place * tiles) * cols;
    }
};

// TILES: of a matrix an item has; a register buffer holds two units, of one tile or one of
// each of two. RAGGED: d is not whole units, or they do not go evenly over the waves' buffers
// X_LDS: the tokens are kept in LDS (up to kXBytes of them)
constexpr int kXPad = 16;  // bytes between the rows there, so that they start on other banks
constexpr int kXBytes = 16 * (2 * 2048 + kXPad);
template <class F, int TILES, bool RAGGED, bool X_LDS>
__global__ __launch_bounds__(kUpThreads, F::UP_WAVES) void few_up_kernel(FewParams<F> p) {
    constexpr int WAVES = kUpThreads / 64, BATCH = 2 / TILES, COLS = TILES * kFewCols;
    __shared__ __align__(16) f32x4 part[2][2 * TILES][WAVES][64];  // [parity of the item][matrix, tile]
    __shared__ SelectSmem sm;
    __shared__ __align__(16) char x_lds[X_LDS ? kXBytes : 16];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int r16 = lane & 15, q = lane >> 4;
    const int T = p.T, k = p.k, d = p.d, f = p.f, fs = p.fs;
    const int sh_tiles = ceil_div(fs, COLS), tiles = ceil_div(f, COLS);

    // the picks, the reached segments, and where each token's gate of a segment is
    if (tid < kSetWords) sm.reached[tid] = 0;
    __syncthreads();
    const int selecting = ceil_div(T, 4) * 64, idle = tid - selecting;
    if (idle < 0) {
        if (p.E <= 64) few_select<4>(p.logits, p.e2g, sm, T, p.E, p.G, k, wave, lane);
        else few_select<16>(p.logits, p.e2g, sm, T, p.E, p.G, k, wave, lane);
    } else {
        for (int i = idle; i < BMOE_MAX_EXPERTS * kFewTok / 2; i += kUpThreads - selecting)
            ((uint32_t*)sm.slot_of)[i] = ~0u;
        if constexpr (X_LDS) {
            const int nch = d * (int)sizeof(typename F::Act) / 16;
            for (int i = idle; i < T * nch; i += kUpThreads - selecting) {
                const int t = i / nch;
                *(v4u*)(x_lds + t * (nch * 16 + kXPad) + (i - t * nch) * 16) = ((const v4u*)p.x)[i];
            }
        }
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

    const uint32_t xr = min(r16, T - 1) * (d * (uint32_t)sizeof(typename F::Act) + (X_LDS ? kXPad : 0));
    const int units = ceil_div(d, F::UK), steps = ceil_div(ceil_div(units, WAVES), BATCH);  // steps of an item
    const int wg = scalar(blockIdx.x), wgs = scalar(gridDim.x);
    const int mine = scalar(wg < items ? div_uniform(items - 1 - wg, wgs) + 1 : 0);
    // A workgroup starts an item at a step of its own and goes around: rows are often a
    // power of two long, and from one column the workgroups would ask a few memory
    // channels for all of them.
    const int turn = scalar((int)((unsigned)wg % (unsigned)steps));
    auto turned = [&](int s) __attribute__((always_inline)) { return s + turn < steps ? s + turn : s + turn - steps; };
    typedef FewW<F, BATCH, 2 * TILES> W;
    typedef FewX<F, BATCH, 1> X;
    // the place of the loads: step l_step of item l_item
    int l_item = wg, l_step = 0, l_at = 0;
    typename F::template Place<2, 2 * TILES> rows;  // of W_gate and W_up
    auto enter = [&]() __attribute__((always_inline)) {
        const UpItem it(l_item, COLS, sh_tiles, tiles);
        const int seg = it.shared ? 0 : scalar(sm.segs[it.place]), N = pick(it.shared, fs, f);
        rows.set(pick(it.shared, p.up_sh[0], p.up[0]), pick(it.shared, p.up_sh[1], p.up[1]), (int64_t)seg * N + it.n0,
                 N - it.n0, d, r16, q);
    };
    auto load_w = [&](W& b, int at) __attribute__((always_inline)) {
        if (at != l_at) {
            l_at = at;
            if (++l_step == steps) {
                l_step = 0;
                l_item += wgs;
                enter();
            }
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            int u = wave + WAVES * (BATCH * turned(l_step) + i);
            if constexpr (RAGGED) u = min(u, units - 1);
            b.w[i].template load<RAGGED>(rows, u * F::UK, d, q);
        }
    };
    f32x4 tot[2 * TILES];
#pragma unroll
    for (int m = 0; m < 2 * TILES; ++m) tot[m] = f32x4{0.f, 0.f, 0.f, 0.f};
    int item = wg, step = 0, parity = 0;
    int x_at = 0, x_step = 0;  // and of the activations'
    auto load_x = [&](X& b, int at) __attribute__((always_inline)) {
        if (at != x_at) {
            x_at = at;
            if (++x_step == steps) x_step = 0;
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            int u = wave + WAVES * (BATCH * turned(x_step) + i);
            if constexpr (RAGGED) u = min(u, units - 1);
            b.x[i][0].template load<RAGGED>(X_LDS ? (const void*)x_lds : (const void*)p.x, xr, u * F::UK, d, q);
        }
    };
    auto multiply = [&](W& b, X& x) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            if constexpr (RAGGED) {
                const int kk = (wave + WAVES * (BATCH * turned(step) + i)) * F::UK;
                b.w[i].tail(kk, d, q);
                x.x[i][0].tail(kk, d, q);
            }
            F::multiply(tot, b.w[i], x.x[i], p.up[0].has_zeros);
        }
        if (++step < steps) return;
        step = 0;
#pragma unroll
        for (int m = 0; m < 2 * TILES; ++m) {
            part[parity][m][wave][lane] = tot[m];
            tot[m] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        // one barrier an item: the other parity's partials were read before it
        lds_reads_done();
        wg_barrier();
        const UpItem it(item, COLS, sh_tiles, tiles);
        const int N = pick(it.shared, fs, f), at_col = tid % COLS, col = it.n0 + at_col, token = tid / COLS;
        if (token < T && col < N) {
            const int slot = it.shared ? token : sm.slot_of[it.place][token];
            if (slot >= 0) {
                const float g = tile_sum<WAVES>(part[parity][2 * (at_col >> 4)], token, at_col & 15);
                const float u = tile_sum<WAVES>(part[parity][2 * (at_col >> 4) + 1], token, at_col & 15);
                const float gate = it.shared ? 1.f : sm.gate[slot];
                float v = silu_mul(g, u) * gate;
                if (__builtin_expect(!isfinite(v), 0)) {
                    float g1 = g, u1 = u;
                    if constexpr (F::OFFSET) {
                        const int64_t row = (int64_t)(it.shared ? 0 : sm.segs[it.place]) * N + col;
#pragma clang loop unroll(disable)
                        for (int m = 0; m < 2; ++m) {  // W_gate, then W_up
                            g1 = u1;
                            u1 = (float)F::template defined<1>(pick(it.shared, p.up_sh[m], p.up[m]), row, d,
                                                               p.x + (size_t)token * d, 0);
                        }
                    }
                    v = silu_mul(g1, u1 * gate);  // (may be finite where silu(g) u is not)
                }
                const int64_t at = (it.shared ? (int64_t)T * k * f : 0) + (int64_t)slot * N + col;
                store_hidden(p.h, p.h_part, at, v);
            }
        }
        parity ^= 1;
        item += wgs;
    };
    if (mine > 0) enter();
    stream_steps<F, W, X>(mine * steps, load_w, load_x, multiply);
}

// The long K of few_down_kernel: unit k of place a among the reached segments; a ==
// segments: of the shared experts.
struct DownUnit {
    int a, k;
    __device__ __forceinline__ void advance(int n, int segments, int per) {
        k += n;
#pragma clang loop unroll(disable) vectorize(disable)
        while (a < segments && k >= per) {
            k -= per;
            ++a;
        }
    }
};

// column c of token t's output from the stored hidden values, as defined
template <class F>
__device__ __forceinline__ float defined_output(const FewParams<F>& p, int t, int c) {
    double sum = 0.0;
#pragma clang loop unroll(disable)
    for (int i = 0; i <= p.k && !isnan(sum); ++i) {  // (the last one: the shared experts)
        const bool sh = i == p.k;
        const int slot = t * p.k + min(i, p.k - 1), g = sh ? 0 : p.slot_group[slot], width = pick(sh, p.fs, p.f);
        if (sh ? p.fs == 0 : (unsigned)g >= (unsigned)p.G) continue;
        const int64_t at = sh ? (int64_t)p.T * p.k * p.f + (int64_t)t * p.fs : (int64_t)slot * p.f;
        sum += F::template defined<2>(pick(sh, p.down_sh, p.down), (int64_t)g * p.d + c, width, p.h + at, p.h_part);
    }
    return (float)sum;
}

// PACK: at most 8 tokens, both parts of their hidden values in one A operand
// RAGGED: d_ff or d_ff_shared is not whole units
template <class F, bool PACK, bool RAGGED>
__global__ __launch_bounds__(kDownThreads, F::DOWN_WAVES) void few_down_kernel(FewParams<F> p) {
    constexpr int WAVES = kDownThreads / 64, BATCH = F::DOWN_BATCH, NP = PACK ? 1 : F::PARTS;
    constexpr int TILES = PACK ? F::PACK_TILES : F::DOWN_TILES, COLS = TILES * kFewCols;
    __shared__ __align__(16) f32x4 part[TILES][WAVES][64];
    __shared__ uint32_t reached[kSetWords];
    // by place among the reached segments (ascending): the segment, the tokens that
    // call it, each token's slot (0 where it has none)
    __shared__ int16_t segs[BMOE_MAX_EXPERTS];
    __shared__ uint32_t callers[BMOE_MAX_EXPERTS + 1];
    __shared__ uint8_t slot_of[BMOE_MAX_EXPERTS][kFewTok];
    __shared__ int last_s;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int r16 = lane & 15, q = lane >> 4;
    const int T = p.T, k = p.k, d = p.d, f = p.f, fs = p.fs;
    const int wg = scalar(blockIdx.x), tile = div_uniform(wg, p.split), n0 = tile * COLS;
    const int g = tid < T * k ? p.slot_group[tid] : -1;
    const bool valid = (unsigned)g < (unsigned)p.G;
    if (tid < kSetWords) reached[tid] = 0;
    if (tid == 0) segs[0] = 0;  // (read for its address where no segment is reached)
    callers[tid] = 0;
    for (int i = tid; i < BMOE_MAX_EXPERTS * kFewTok / 4; i += kDownThreads) ((uint32_t*)slot_of)[i] = 0;
    __syncthreads();
    if (valid) atomicOr(&reached[g >> 5], 1u << (g & 31));
    __syncthreads();
    const int segments = members(reached);
    if (valid) {
        const int place = members_below(reached, g), t = tid / k;
        segs[place] = (int16_t)g;
        atomicOr(&callers[place], 1u << t);
        slot_of[place][t] = (uint8_t)tid;
    }
    if (tid == 0) callers[segments] = 0xffffu;  // the shared experts
    const int per = ceil_div(f, F::UK), per_sh = ceil_div(fs, F::UK), units = segments * per + per_sh;
    __syncthreads();
    // the waves of the tile's workgroups take the units in turn
    const int first = (wg - tile * p.split) * WAVES + wave, stride = p.split * WAVES;
    const int steps = ceil_div(div_uniform(units + stride - 1, stride), BATCH);
    const int token = PACK ? r16 & 7 : r16;
    typedef FewW<F, BATCH, TILES> W;
    typedef FewX<F, BATCH, NP> X;
    DownUnit lu{0, 0}, xu, mu;  // of the weights' loads, the activations' and the products
    lu.advance(first, segments, per);
    xu = mu = lu;
    int l_at = 0, x_at = 0;
    auto load_w = [&](W& b, int at) __attribute__((always_inline)) {
        if (at != l_at) {
            l_at = at;
            lu.advance(stride, segments, per);
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            if (i) lu.advance(stride, segments, per);
            // (past the last unit: the first one again, its products are dropped)
            const bool past = lu.a == segments && lu.k >= per_sh, sh = lu.a == segments && !past;
            const int seg = sh ? 0 : scalar(segs[past ? 0 : lu.a]), width = pick(sh, fs, f);
            typename F::template Place<1, TILES> rows;
            const typename F::Stack st = pick(sh, p.down_sh, p.down);
            rows.set(st, st, (int64_t)seg * d + n0, d - n0, width, r16, q);
            b.w[i].template load<RAGGED>(rows, past ? 0 : lu.k * F::UK, width, q);
        }
    };
    auto load_x = [&](X& b, int at) __attribute__((always_inline)) {
        if (at != x_at) {
            x_at = at;
            xu.advance(stride, segments, per);
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            if (i) xu.advance(stride, segments, per);
            const bool past = xu.a == segments && xu.k >= per_sh, sh = xu.a == segments && !past;
            const int slot = sh ? min(token, T - 1) : slot_of[past ? 0 : xu.a][token], width = pick(sh, fs, f);
            // (hidden values are below 2^32 bytes: 16 tokens, 16 slots, 2^20 columns)
            const uint32_t hr = (uint32_t)((sh ? (int64_t)T * k * f : 0) + (int64_t)slot * width +
                                           (PACK && r16 >= 8 ? p.h_part : 0)) * sizeof(typename F::Act);
#pragma unroll
            for (int j = 0; j < NP; ++j)
                b.x[i][j].template load<RAGGED>(p.h + j * p.h_part, hr, past ? 0 : xu.k * F::UK, width, q);
        }
    };
    f32x4 tot[TILES];
#pragma unroll
    for (int m = 0; m < TILES; ++m) tot[m] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](W& b, X& x) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const bool past = mu.a == segments && mu.k >= per_sh;
            if constexpr (RAGGED) {
                const int kk = mu.k * F::UK, width = pick(mu.a == segments, fs, f);
                b.w[i].tail(kk, width, q);
#pragma unroll
                for (int j = 0; j < NP; ++j) x.x[i][j].tail(kk, width, q);
            }
            f32x4 acc[TILES];
#pragma unroll
            for (int m = 0; m < TILES; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
            F::multiply(acc, b.w[i], x.x[i], p.down.has_zeros);
            // only the tokens that call the segment take its products
            const uint32_t who = past ? 0u : callers[mu.a];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool takes = (who >> ((PACK ? 4 * (q & 1) : 4 * q) + j)) & 1u;
#pragma unroll
                for (int m = 0; m < TILES; ++m) tot[m][j] += takes ? acc[m][j] : 0.f;
            }
            mu.advance(stride, segments, per);
        }
    };
    stream_steps<F, W, X>(steps, load_w, load_x, multiply);
#pragma unroll
    for (int m = 0; m < TILES; ++m) part[m][wave][lane] = tot[m];
    __syncthreads();
    const int t = tid >> 4, col = tid & 15;
    float v[TILES];
#pragma unroll
    for (int m = 0; m < TILES; ++m) {
        v[m] = tile_sum<WAVES>(part[m], t, col);
        if constexpr (PACK) v[m] += t < 8 ? tile_sum<WAVES>(part[m], t + 8, col) : 0.f;
    }
    if (p.split > 1) {
        // the parts meet in memory; the workgroup that finishes last adds them in
        // order. Relaxed accesses of agent scope go past the caches of one XCD, and
        // the wait orders them; fences would write back and drop whole L2 caches
        // (81 us instead of 9 for one token of the fine-grained layer).
        float* mine = p.partial + (size_t)wg * (TILES * kTile) + tid;
#pragma unroll
        for (int m = 0; m < TILES; ++m)
            __hip_atomic_store(mine + m * kTile, v[m], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        wait_vmcnt<0>();  // (this wave's part is written)
        __syncthreads();
        if (tid == 0)
            last_s = __hip_atomic_fetch_add(p.done + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == p.split - 1;
        __syncthreads();
        if (!last_s) return;
        const float* all = p.partial + (size_t)tile * p.split * (TILES * kTile) + tid;
        float parts[kSplitMax][TILES];
#pragma unroll
        for (int i = 0; i < kSplitMax; ++i)
            if (i < p.split) {
#pragma unroll
                for (int m = 0; m < TILES; ++m)
                    parts[i][m] = __hip_atomic_load(all + (i * TILES + m) * kTile, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
#pragma unroll
        for (int m = 0; m < TILES; ++m) {
            v[m] = parts[0][m];
#pragma unroll
            for (int i = 1; i < kSplitMax; ++i)
                if (i < p.split) v[m] += parts[i][m];
        }
    }
#pragma unroll
    for (int m = 0; m < TILES; ++m) {
        const int c = n0 + 16 * m + col;
        if (t < T && c < d) {
            if constexpr (F::OFFSET) {
                if (__builtin_expect(!isfinite(v[m]), 0)) v[m] = defined_output(p, t, c);
            }
            typename F::Act* o = p.out + (size_t)t * d + c;
            if constexpr (sizeof(typename F::Act) == 2) *o = f32_to_bf16(v[m]);
            else *o = v[m];
        }
    }
}

// Workgroups that share `cols` output columns: as many as two or three a CU, where the
// columns are fewer
constexpr int kMostCus = 256;  // that the workspace is for; a launch counts no more of them
inline int most_splits(int d, int cols, int per_cu, int cus) {
    const int tiles = ceil_div(d, cols), n = per_cu * (cus < kMostCus ? cus : kMostCus) / tiles;
    return n < 1 ? 1 : n > kSplitMax ? kSplitMax : n;
}

inline size_t round256(size_t n) { return (n + 255) / 256 * 256; }
inline size_t logit_bytes(int T, int E) { return round256((size_t)T * E * sizeof(double)); }
inline size_t done_bytes(int d) { return round256((size_t)ceil_div(d, kFewCols) * sizeof(int32_t)); }
// (of the partials, enough for any format: 1, 2 or 4 tiles of columns, 2 or 3 workgroups a CU)
inline size_t partial_bytes(int d) {
    size_t most = 0;
    for (int tiles = 1; tiles <= 4; tiles *= 2) {
        const int split = most_splits(d, tiles * kFewCols, 3, kMostCus);
        const size_t n = split == 1 ? 0 : (size_t)ceil_div(d, tiles * kFewCols) * split * tiles * kTile * sizeof(float);
        most = n > most ? n : most;
    }
    return most;
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
    const bool pack = F::PARTS == 2 && a.T <= 8;
    const int down_cols = (pack ? F::PACK_TILES : F::DOWN_TILES) * kFewCols;
    const int cus = persistent_workgroups();
    p.split = most_splits(a.d, down_cols, F::DOWN_WAVES, cus);
    if (units < (int64_t)p.split * (kDownThreads / 64)) p.split = (int)ceil_div64(units, kDownThreads / 64);  // a unit a wave
    hipError_t e = launch_few_logits(a, p.done, s);
    if (e != hipSuccess) return e;
    // Pairs of tiles of bf16 weights: for many tokens, whose activations they save loads of
    // (16 tokens: 52.1 us for the layer, single tiles 55.3), and where they leave a CU no
    // more than one workgroup (one token: 25.5 and 26.7). In between single tiles keep the
    // workgroups' shares closer (two tokens of wide experts: 206 and 228).
    auto items_of = [&](int tiles) {
        const int cols = tiles * kFewCols;
        return most * ceil_div(a.f, cols) + ceil_div(a.fs, cols);
    };
    const int up_tiles = F::PAIRS && a.T <= 8 && items_of(F::UP_TILES) > cus ? 1 : F::UP_TILES;
    const int64_t items = items_of(up_tiles);
    const int64_t room = (int64_t)F::UP_WAVES * 256 / kUpThreads * cus;
    const dim3 up((unsigned)(items < room ? items : room)), down((unsigned)(ceil_div(a.d, down_cols) * p.split));
    const bool up_ragged = a.d % (F::UK * (2 / up_tiles) * (kUpThreads / 64)) != 0;
    const bool down_ragged = a.f % F::UK != 0 || a.fs % F::UK != 0;
    const bool x_fits = F::X_IN_LDS && (int64_t)a.T * (a.d * (int)sizeof(Act) + kXPad) <= kXBytes;
    auto go_up = [&](auto kernel) { hipLaunchKernelGGL(kernel, up, dim3(kUpThreads), 0, s, p); };
    constexpr int kSingle = F::PAIRS ? 1 : F::UP_TILES;
    if (x_fits) {
        if (up_ragged) go_up(few_up_kernel<F, F::UP_TILES, true, F::X_IN_LDS>);
        else go_up(few_up_kernel<F, F::UP_TILES, false, F::X_IN_LDS>);
    } else if (up_tiles == F::UP_TILES) {
        if (up_ragged) go_up(few_up_kernel<F, F::UP_TILES, true, false>);
        else go_up(few_up_kernel<F, F::UP_TILES, false, false>);
    } else {
        if (up_ragged) go_up(few_up_kernel<F, kSingle, true, false>);
        else go_up(few_up_kernel<F, kSingle, false, false>);
    }
    constexpr bool kParts = F::PARTS == 2;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, down, dim3(kDownThreads), 0, s, p); };
    if (pack) {
        if (down_ragged) go(few_down_kernel<F, kParts, true>);
        else go(few_down_kernel<F, kParts, false>);
    } else {
        if (down_ragged) go(few_down_kernel<F, false, true>);
        else go(few_down_kernel<F, false, false>);
    }
    return hipGetLastError();
}

}  // namespace
}  // namespace bmoe
