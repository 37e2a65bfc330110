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
// activation rows (the A operand). It takes the columns in chunks of 128: lane
// (r, q) loads the 16 bytes of row r, columns 32q .. 32q+31. Two exchanges of
// lane rows then give step u (one MFMA of 32 columns) the columns 32u .. 32u+31,
// eight of them in each lane, so that a group of 32 is one step. In a lane the
// eight codes come out as columns 0,4,1,5,2,6,3,7; the activations are put into
// the same order (w4_order).
#pragma once

#include "bmoe_common.h"

namespace bmoe {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));  // native vector: stays in registers

constexpr int kW4Chunk = 128;  // columns per chunk

__device__ __forceinline__ v4u w4_unpack(uint32_t c) {
    constexpr uint32_t kMask = 0x00780078u, kSixteen = 0x41804180u;
    return v4u{((c << 3) & kMask) | kSixteen, ((c >> 1) & kMask) | kSixteen, ((c >> 5) & kMask) | kSixteen,
               ((c >> 9) & kMask) | kSixteen};
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

// the unsigned integer of N bytes
template <int N>
struct UintOf;
template <>
struct UintOf<1> { typedef uint8_t type; };
template <>
struct UintOf<2> { typedef uint16_t type; };
template <>
struct UintOf<4> { typedef uint32_t type; };
template <>
struct UintOf<8> { typedef uint64_t type; };

// 16 bytes at a 32-bit offset from an address that the whole wave shares
__device__ __forceinline__ v4u load_at(const void* base, uint32_t off) {
    return *(const v4u*)((const char*)base + off);
}

// 16 rows of a stack (fewer at its end), from row `first` on
template <int GROUP>
struct W4Rows {
    static constexpr int NG = kW4Chunk / GROUP;
    const uint8_t* codes;
    const uint16_t* scales;
    const uint8_t* zeros;
    int last;  // the place of the stack's last NG groups, from the first row's first
    __device__ __forceinline__ W4Rows(const W4Stack& w, int64_t first, int K) {
        const int64_t j = first * ceil_div(K, GROUP);
        codes = w.codes + first * BMOE_W4_ROW_BYTES(K);
        scales = w.scales + j;
        zeros = w.zeros + j;
        last = (int)(w.groups - NG - j < 0x7fffffff ? w.groups - NG - j : 0x7fffffff);
    }
};

// A chunk of one lane's W row: 128 columns' codes (the lane's 32 of them) and the
// chunk's groups, in one load each and without a branch (zeros are loaded where
// there are none too). Rows of groups have any alignment.
template <int GROUP>
struct W4Chunk {
    static constexpr int NG = kW4Chunk / GROUP;
    v4u codes;
    typename UintOf<2 * NG>::type s;
    typename UintOf<NG>::type z;

    // chunk c of row r of the rows; K columns
    __device__ __forceinline__ void load(const W4Rows<GROUP>& w, int r, int c, int K, int q) {
        const int pitch = BMOE_W4_ROW_BYTES(K), ng = ceil_div(K, GROUP);
        codes = load_at(w.codes, (uint32_t)(r * pitch + min(64 * c + 16 * q, pitch - 16)));
        // groups past the row's last one are another row's, or 0 past the stack's
        // end (a stack has at least 8 rows): their activations are zero
        const int j = r * ng + c * NG, from = min(j, w.last);
        __builtin_memcpy(&s, (const char*)w.scales + (uint32_t)(from * 2), sizeof s);
        __builtin_memcpy(&z, w.zeros + (uint32_t)from, sizeof z);
        if constexpr (NG > 1) {
            s = (decltype(s))(s >> (16 * (j - from)));
            z = (decltype(z))(z >> (8 * (j - from)));
        }
    }
    __device__ __forceinline__ float scale(int g) const { return bf16_to_f32((uint16_t)(s >> (16 * g))); }
    // 16 + the zero point of group g
    __device__ __forceinline__ float offset(bool has_zeros, int g) const {
        return has_zeros ? 16.f + (float)(uint8_t)(z >> (8 * g)) : 24.f;
    }
};

}  // namespace bmoe
