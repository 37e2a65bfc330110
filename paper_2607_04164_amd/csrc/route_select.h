// What the top-k selections share: arg-max and sum over a group of lanes that
// holds a token's logits, and the form in which a pick is kept.
#pragma once

#include "bmoe_common.h"

namespace bmoe {

__device__ __forceinline__ bool better(float v, int e, float bv, int be) {
    return v > bv || (v == bv && e < be);
}
__device__ __forceinline__ bool better(double v, int e, double bv, int be) {
    return v > bv || (v == bv && e < be);
}

// ---- lane exchanges. Within rows of 16 lanes, DPP row permutations (quad
// xor 1, quad xor 2, half-row mirror, row mirror) run on the VALU; they pair
// every lane with a lane of the other half of its group at each step, so
// after log2(S) steps all S lanes of an aligned group hold the reduction.
// Steps across rows (16, 32) go through ds_bpermute (__shfl_xor).
template <int CTRL>
__device__ __forceinline__ int dpp_i(int v) {
    return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, false);
}
template <int CTRL>
__device__ __forceinline__ float dpp_f(float v) {
    return __int_as_float(dpp_i<CTRL>(__float_as_int(v)));
}
template <int CTRL>
__device__ __forceinline__ double dpp_d(double v) {
    return __hiloint2double(dpp_i<CTRL>(__double2hiint(v)), dpp_i<CTRL>(__double2loint(v)));
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;

template <int CTRL, typename V>
__device__ __forceinline__ void argmax_step(V& bv, int& be) {
    V ov;
    if constexpr (sizeof(V) == 8) ov = dpp_d<CTRL>(bv);
    else ov = dpp_f<CTRL>(bv);
    const int oe = dpp_i<CTRL>(be);
    if (better(ov, oe, bv, be)) { bv = ov; be = oe; }
}

// arg-max (ties: lower index) over aligned groups of S lanes, S in {1,2,4,...,64}
template <int S, typename V>
__device__ __forceinline__ void group_argmax(V& bv, int& be) {
    if constexpr (S >= 2) argmax_step<kDppXor1>(bv, be);
    if constexpr (S >= 4) argmax_step<kDppXor2>(bv, be);
    if constexpr (S >= 8) argmax_step<kDppHalfMirror>(bv, be);
    if constexpr (S >= 16) argmax_step<kDppMirror>(bv, be);
#pragma unroll
    for (int off = 16; off < S; off <<= 1) {
        V ov = __shfl_xor(bv, off);
        int oe = __shfl_xor(be, off);
        if (better(ov, oe, bv, be)) { bv = ov; be = oe; }
    }
}

// sum over aligned groups of S lanes (every lane gets the same bits: each
// step adds two values in an order-independent way)
template <int S, typename V>
__device__ __forceinline__ V group_sum(V v) {
    if constexpr (sizeof(V) == 8) {
        if constexpr (S >= 2) v += dpp_d<kDppXor1>(v);
        if constexpr (S >= 4) v += dpp_d<kDppXor2>(v);
        if constexpr (S >= 8) v += dpp_d<kDppHalfMirror>(v);
        if constexpr (S >= 16) v += dpp_d<kDppMirror>(v);
    } else {
        if constexpr (S >= 2) v += dpp_f<kDppXor1>(v);
        if constexpr (S >= 4) v += dpp_f<kDppXor2>(v);
        if constexpr (S >= 8) v += dpp_f<kDppHalfMirror>(v);
        if constexpr (S >= 16) v += dpp_f<kDppMirror>(v);
    }
#pragma unroll
    for (int off = 16; off < S; off <<= 1) v += __shfl_xor(v, off);
    return v;
}

// A pick in a token's pick list: expert id in the high bits, united expert + 1
// in the low 16 bits (0: the map sends the expert nowhere, so the slot calls
// none). Keys of distinct experts order like their expert ids, so the packed
// value serves as the tie-break index of an arg-max.
constexpr int kNoPick = 0x7fff0000;  // out-of-range expert, no united expert
__device__ __forceinline__ int pack_pick(int e, const int* e2g_s, int E) {
    const int g = (unsigned)e < (unsigned)E ? e2g_s[e] : -1;  // NaN logits pick nothing
    return ((e & 0x7fff) << 16) | (g + 1);
}
__device__ __forceinline__ int pick_expert(int pk) { return pk >> 16; }
__device__ __forceinline__ int pick_group(int pk) { return (pk & 0xffff) - 1; }

}  // namespace bmoe
