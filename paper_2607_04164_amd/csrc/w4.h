// 4-bit weights with group scales on the bf16 matrix cores: w = s (q - z).
//
// A code q becomes the bf16 value 16 + q by placing its four bits on top of the
// mantissa of 16 (one shift, one and-or for two codes); q and 16 + q are exact in
// bf16. Per group of columns the matrix cores form
//   acc = sum_k x_k (16 + q_k)   and   xs = sum_k x_k   (B operand of ones),
// and the group adds s (acc - (16 + z) xs) to the total, in fp32. The offset
// costs about 5 times the rounding of the plain sum (16 + q against q - z), far
// below the bf16 output's.
//
// A wave owns 16 rows of W (the B operand) and up to TILES tiles of 16
// activation rows (the A operand). It takes the columns in units of 256, a 128-byte
// line of each row: lane (r, q) loads the 16 bytes of columns 32q .. 32q+31 and of
// 128 + 32q .., row r. Two exchanges of lane rows then give step u of a half (one
// MFMA of 32 columns) the columns 32u .. 32u+31, eight of them in each lane, so that
// a group of 32 is one step. In a lane the eight codes come out as columns
// 0,4,1,5,2,6,3,7; the activations are put into the same order (w4_order). A unit's
// scales are one load of each lane, and so are its zero points.
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

// 16 rows of a stack (fewer at its end), from row `first` on
template <int GROUP>
struct W4Rows {
    static constexpr int NG = kW4Unit / GROUP;
    const uint8_t* codes;
    const uint16_t* scales;
    const uint8_t* zeros;
    int last;  // the place of the stack's last NG groups, from the first row's first
    W4Rows() = default;
    __device__ __forceinline__ W4Rows(const W4Stack& w, int64_t first, int K) {
        const int64_t j = first * ceil_div(K, GROUP);
        codes = w.codes + first * BMOE_W4_ROW_BYTES(K);
        scales = w.scales + j;
        zeros = w.zeros + j;
        last = (int)(w.groups - NG - j < 0x7fffffff ? w.groups - NG - j : 0x7fffffff);
    }
};

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

// A unit of one lane's W row: 256 columns' codes (the lane's 64 of them) and the
// unit's groups, without a branch (zeros are loaded where there are none too). Rows
// of groups have any alignment.
template <int GROUP>
struct W4Unit {
    static constexpr int NG = kW4Unit / GROUP;
    v4u codes[2];
    W4Groups<2 * NG> s;
    W4Groups<NG> z;
    int back;  // groups that s and z start before the unit's first one

    // unit c of row r of the rows; K columns
    __device__ __forceinline__ void load(const W4Rows<GROUP>& w, int r, int c, int K, int q) {
        const int pitch = BMOE_W4_ROW_BYTES(K), ng = ceil_div(K, GROUP);
#pragma unroll
        for (int h = 0; h < 2; ++h)
            codes[h] = load_at(w.codes, (uint32_t)(r * pitch + min(128 * c + 64 * h + 16 * q, pitch - 16)));
        // Groups past the row's last one are another row's: their activations are
        // zero. A unit that would reach past the stack's end starts further back (a
        // stack has at least 8 rows).
        const int j = r * ng + c * NG, from = min(j, w.last);
        back = j - from;
        s.load((const char*)w.scales + (uint32_t)(from * 2));
        z.load(w.zeros + (uint32_t)from);
    }
    // moves the groups to their places: after the load, where K is not whole units
    __device__ __forceinline__ void settle() {
#pragma unroll
        for (int i = 0; i < NG; ++i)
            if (i < back) {
                s.template drop<16>();
                z.template drop<8>();
            }
    }
    __device__ __forceinline__ float scale(int g) const {
        return __uint_as_float(g & 1 ? s.v[g >> 1] & 0xffff0000u : s.v[g >> 1] << 16);
    }
    // 16 + the zero point of group g
    __device__ __forceinline__ float offset(bool has_zeros, int g) const {
        return has_zeros ? 16.f + (float)((z.v[g >> 2] >> (8 * (g & 3))) & 0xffu) : 24.f;
    }
};

}  // namespace bmoe
