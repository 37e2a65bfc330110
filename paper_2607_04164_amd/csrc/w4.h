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

// One matrix stack and the sizes that address it.
struct W4Stack {
    const uint8_t* codes;
    const uint16_t* scales;
    const uint8_t* zeros;  // or nullptr
};

// A chunk of one lane's W row: 128 columns' codes (the lane's 32 of them) and the chunk's groups.
template <int GROUP>
struct W4Chunk {
    static constexpr int NG = kW4Chunk / GROUP;
    v4u codes;
    uint16_t s[NG];
    uint8_t z[NG];

    // chunk c of matrix row `row` (of all rows of the stack); K columns
    __device__ __forceinline__ void load(const W4Stack& w, size_t row, int c, int K, int q) {
        const int pitch = BMOE_W4_ROW_BYTES(K), ng = ceil_div(K, GROUP);
        const int at = 64 * c + 16 * q;
        codes = *(const v4u*)(w.codes + row * pitch + (at < pitch ? at : 0));
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            // (groups past the last one: their activations are zero)
            const size_t j = row * ng + min(c * NG + g, ng - 1);
            s[g] = w.scales[j];
            z[g] = w.zeros ? w.zeros[j] : (uint8_t)8;
        }
    }
};

}  // namespace bmoe
