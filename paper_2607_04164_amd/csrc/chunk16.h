// 16-byte chunks of rows as fp32 values: 8 bf16 or 4 floats.
#pragma once

#include "bmoe_common.h"

namespace bmoe {

template <typename T>
struct Vec;
template <>
struct Vec<uint16_t> {  // 8 bf16 per chunk
    static constexpr int N = 8;
    __device__ static void load(const uint4& v, float* f) {
        const uint32_t* u = (const uint32_t*)&v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(u[i] << 16);
            f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
    __device__ static uint4 store(const float* f) {
        uint4 v;
        v.x = pack_bf16x2(f[0], f[1]);
        v.y = pack_bf16x2(f[2], f[3]);
        v.z = pack_bf16x2(f[4], f[5]);
        v.w = pack_bf16x2(f[6], f[7]);
        return v;
    }
};
template <>
struct Vec<float> {  // 4 floats per chunk
    static constexpr int N = 4;
    __device__ static void load(const uint4& v, float* f) {
        f[0] = __uint_as_float(v.x);
        f[1] = __uint_as_float(v.y);
        f[2] = __uint_as_float(v.z);
        f[3] = __uint_as_float(v.w);
    }
    __device__ static uint4 store(const float* f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                          __float_as_uint(f[3]));
    }
};

}  // namespace bmoe
