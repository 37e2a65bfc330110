// 4-bit weights with group scales on the bf16 matrix cores: w = s (q - z).
//
// A code q becomes the bf16 value 16 + q by placing its four bits on top of the
// mantissa of 16 (one shift, one and-or for two codes); q and 16 + q are exact in
// bf16. Per group of columns the matrix cores form
//   acc = sum_k x_k (16 + q_k)   and   xs = sum_k x_k   (A operand of ones),
// and the group adds s acc - s (16 + z) xs to the total, in fp32: the first term by
// one multiply-add an element, the second as a product over the groups on the fp32
// matrix cores, four groups an instruction (s (16 + z) is exact in fp32; the vector
// units, not the matrix cores, bound a product of more than a few rows). The offset
// costs about 5 times the rounding of the plain sum (16 + q against q - z), far
// below the bf16 output's.
// Where the terms leave fp32 though the product itself does not (activations near the
// largest value), or an activation is infinite (acc and its offset are then infinities
// of opposite signs), the result is not finite: such a result is computed again as it
// is defined (w4_defined).
//
// A wave owns MT = 4 tiles of 16 rows of W (the B operands; of one matrix, or two of
// each of two; where that makes too few workgroups, one tile of each matrix) and one
// or two tiles of 16 activation rows (the A operands). It takes the columns in units
// of 256, a 128-byte line of each row: lane (r, q) loads the 16 bytes of columns 32q .. 32q+31 and of
// 128 + 32q .., row r. Two exchanges of lane rows then give step u of a half (one
// MFMA of 32 columns) the columns 32u .. 32u+31, eight of them in each lane, so that
// a group of 32 is one step. In a lane the eight codes come out as columns
// 0,4,1,5,2,6,3,7; the activations are put into the same order (w4_order). The scales
// of a unit are one load: lane row q brings those of tile q, and three exchanges hand
// them to all lanes; the zero points likewise, into the fp32 product's B operand. (Loads are what is scarce: an
// instruction of 64 lanes takes 16 cycles of the address unit however little it brings.)
#pragma once

#include "bmoe_common.h"

namespace bmoe {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));  // native vector: stays in registers

constexpr int kW4Unit = 256;  // columns per unit

__device__ __forceinline__ v4u w4_unpack(uint32_t c) {
    constexpr uint32_t kMask = 0x00780078u;
    // (in a vector register: an instruction takes one scalar operand, and with both
    // constants scalar the and and the or would be two)
    uint32_t sixteen;
    asm("v_mov_b32 %0, 0x41804180" : "=v"(sixteen));
    return v4u{((c << 3) & kMask) | sixteen, ((c >> 1) & kMask) | sixteen, ((c >> 5) & kMask) | sixteen,
               ((c >> 9) & kMask) | sixteen};
}

// eight activations in the order of w4_unpack
__device__ __forceinline__ v4u w4_order(v4u x) {
    return v4u{__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u),
               __builtin_amdgcn_perm(x[3], x[1], 0x05040100u), __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
}

// c[j] of lane row q -> c[q] of lane row j (lane rows: 16 lanes)
__device__ __forceinline__ v4u w4_transpose(v4u c) {
    typedef uint32_t v2u __attribute__((ext_vector_type(2)));
    const v2u a = __builtin_amdgcn_permlane16_swap(c[0], c[1], false, false);
    const v2u b = __builtin_amdgcn_permlane16_swap(c[2], c[3], false, false);
    const v2u e = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false);
    const v2u f = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
    return v4u{e[0], f[0], e[1], f[1]};
}

__device__ __forceinline__ f32x4 mfma16(v4u a, v4u b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
}

// One matrix stack.
struct W4Stack {
    const uint8_t* codes;
    const uint16_t* scales;
    const uint8_t* zeros;  // where there are none: any memory that can be read like them
    int64_t groups;        // of all rows
    int has_zeros;
};

inline W4Stack w4_stack(const void* codes, const void* scales, const uint8_t* zeros, int64_t rows, int K, int group) {
    return W4Stack{(const uint8_t*)codes, (const uint16_t*)scales, zeros ? zeros : (const uint8_t*)scales,
                   rows * ceil_div(K, group), zeros != nullptr};
}

// 16 bytes at a 32-bit offset from an address that the whole wave shares
__device__ __forceinline__ v4u load_at(const void* base, uint32_t off) {
    return *(const v4u*)((const char*)base + off);
}

// N bytes of group values from any address
template <int N>
struct W4Groups {
    static constexpr int WORDS = (N + 3) / 4;
    uint32_t v[WORDS];
    __device__ __forceinline__ void load(const void* p) {
        if constexpr (N == 2) {
            uint16_t h;
            __builtin_memcpy(&h, p, 2);
            v[0] = h;
        } else {
            __builtin_memcpy(v, p, N);
        }
    }
    // drops the first `bits` of the first word (below 32)
    template <int BITS>
    __device__ __forceinline__ void drop() {
#pragma unroll
        for (int j = 0; j < WORDS; ++j) v[j] = v[j] >> BITS | (j + 1 < WORDS ? v[j + 1 < WORDS ? j + 1 : j] << (32 - BITS) : 0u);
    }
};

// MT tiles of 16 rows: of NR stacks, from row `first` of each on, `left` rows there
// (at least 8). Tile m is rows 16 (m / NR) .. of stack m % NR.
template <int GROUP, int NR, int MT = 4>
struct W4Place {
    static constexpr int NG = kW4Unit / GROUP;
    const uint8_t* codes[NR];  // the first row
    uint32_t row[MT / NR];     // the lane's row of a tile, in bytes
    const uint16_t* scales;    // the lane's row of tile q % MT
    const uint8_t* zeros;
    int last;                  // from there: the stack's last NG groups

    __device__ __forceinline__ void set(const W4Stack& s0, const W4Stack& s1, int64_t first, int left, int K, int r16, int q) {
        const int pitch = BMOE_W4_ROW_BYTES(K), ng = ceil_div(K, GROUP);
        codes[0] = s0.codes + first * pitch;
        if constexpr (NR == 2) codes[NR - 1] = s1.codes + first * pitch;
#pragma unroll
        for (int t = 0; t < MT / NR; ++t) row[t] = (uint32_t)(min(16 * t + r16, left - 1) * pitch);
        const bool second = NR == 2 && (q & 1);
        const int64_t j = (first + min(16 * (q % MT / NR) + r16, left - 1)) * ng;
        scales = (second ? s1.scales : s0.scales) + j;
        zeros = (second ? s1.zeros : s0.zeros) + j;
        const int64_t rest = s0.groups - NG - j;
        last = (int)(rest < 0x7fffffff ? rest : 0x7fffffff);
    }
};

// out[i]: lane row i's value in every lane row, where row q has the value of q % MT
template <int MT>
__device__ __forceinline__ void w4_spread(uint32_t v, uint32_t (&out)[MT]) {
    typedef uint32_t v2u __attribute__((ext_vector_type(2)));
    out[0] = v;
    if constexpr (MT == 2) {
        const v2u a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        out[0] = a[0];
        out[MT - 1] = a[1];
    }
    if constexpr (MT != 4) return;
    const v2u a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const v2u b = __builtin_amdgcn_permlane16_swap(a[0], a[0], false, false);
    const v2u c = __builtin_amdgcn_permlane16_swap(a[1], a[1], false, false);
    out[0] = b[0];
    out[MT > 1 ? 1 : 0] = b[1];
    out[MT > 2 ? 2 : 0] = c[0];
    out[MT > 3 ? 3 : 0] = c[1];
}

// A unit of the tiles: 256 columns' codes (the lane's 64 of them) and the unit's
// groups, without a branch (zeros are loaded where there are none too). Rows of groups
// have any alignment.
template <int GROUP, int MT = 4>
struct W4Unit {
    static constexpr int NG = kW4Unit / GROUP;
    typedef W4Groups<2 * NG> Scales;
    typedef W4Groups<NG> Zeros;
    v4u codes[MT][2];
    Scales s;  // of tile q % MT
    Zeros z;
    int back;  // groups that s and z start before the unit's first one

    template <int NR>
    __device__ __forceinline__ void load(const W4Place<GROUP, NR, MT>& w, int c, int K, int q) {
        const int pitch = BMOE_W4_ROW_BYTES(K);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                codes[m][h] = load_at(w.codes[m % NR], w.row[m / NR] + min(128 * c + 64 * h + 16 * q, pitch - 16));
        // Groups past the row's last one are another row's: their activations are
        // zero. A unit that would reach past the stack's end starts further back (a
        // stack has at least 8 rows).
        const int from = min(c * NG, w.last);
        back = c * NG - from;
        s.load(w.scales + from);
        z.load(w.zeros + from);
    }
    // After the load, where K is not whole units: moves the groups to their places and
    // clears the scales of those past column K (another row's may be infinite).
    __device__ __forceinline__ void settle(int k, int K) {
#pragma unroll
        for (int i = 0; i < NG; ++i)
            if (i < back) {
                s.template drop<16>();
                z.template drop<8>();
            }
#pragma unroll
        for (int i = 0; i < NG; ++i)
            if (k + i * GROUP >= K) s.v[i / 2] &= i & 1 ? 0xffffu : 0xffff0000u;
    }
};

// the groups of all tiles: their scales in every lane, and - s (16 + z) as B operands
// of the fp32 matrix cores (group 4 i + q in lane row q of offset[i])
template <int GROUP, int MT = 4>
struct W4Spread {
    static constexpr int NG = kW4Unit / GROUP, NC = (NG + 3) / 4;
    uint32_t s[(2 * NG + 3) / 4][MT];
    v4u offset[NC];  // of tiles 0 .. 3 (beyond MT: repeated)
    __device__ __forceinline__ W4Spread(const W4Unit<GROUP, MT>& u, bool has_zeros) {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            v4u own = {0u, 0u, 0u, 0u};  // of the tile of this lane row, groups 4 i .. 4 i + 3
#pragma unroll
            for (int j = 0; j < 4 && 4 * i + j < NG; ++j) {
                const int g = 4 * i + j;
                const float z = has_zeros ? (float)((u.z.v[i] >> (8 * j)) & 0xffu) : 8.f;
                own[j] = __float_as_uint(-value(u.s.v[g >> 1], g) * (16.f + z));
            }
            offset[i] = w4_transpose(own);
        }
#pragma unroll
        for (int i = 0; i < (2 * NG + 3) / 4; ++i) w4_spread<MT>(u.s.v[i], s[i]);
    }
    __device__ __forceinline__ static float value(uint32_t pair, int g) {
        return __uint_as_float(g & 1 ? pair & 0xffff0000u : pair << 16);
    }
    __device__ __forceinline__ float scale(int m, int g) const { return value(s[g >> 1][m], g); }
    // after group g, the last or every fourth: adds the offsets' part of tile m; xs:
    // the A operand, group 4 (g / 4) + q's sum of the token r16 in lane (r16, q)
    __device__ __forceinline__ f32x4 add_offset(f32x4 tot, float xs, int m, int g) const {
        return __builtin_amdgcn_mfma_f32_16x16x4f32(xs, __uint_as_float(offset[g >> 2][m]), tot, 0, 0, 0);
    }
};

// sum over k of x_k s (q_k - z) for one row of W as it is defined, in float64 (every term
// is exact there). load(k, f): columns k .. k + 7 of x. One lane's work, for the few
// results that are not finite.
template <int GROUP, class Load>
__device__ __forceinline__ double w4_defined(const W4Stack& w, int64_t row, int K, Load load) {
    const int ng = ceil_div(K, GROUP);
    const uint8_t* codes = w.codes + row * BMOE_W4_ROW_BYTES(K);
    double sum = 0.0;
#pragma clang loop unroll(disable)
    for (int k = 0; k < K && !isnan(sum); k += 8) {
        const int64_t g = row * ng + k / GROUP;
        const double s = bf16_to_f32(w.scales[g]);
        const int z = w.has_zeros ? w.zeros[g] : 8;
        uint32_t c = *(const uint32_t*)(codes + k / 2);
        float f[8];
        load(k, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum = fma(s * ((int)(c & 15u) - z), (double)f[j], sum);
            c >>= 4;
        }
    }
    return sum;
}

}  // namespace bmoe
