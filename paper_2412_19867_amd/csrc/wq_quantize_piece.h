// Rows of any float type in pieces of eight elements a lane, and the group quantizer over adjacent lanes.
#pragma once

#include "wq_device.h"
#include "wq.h"

namespace {   // every including file has its own

template <int TYPE>
struct Elem;
template <>
struct Elem<WQ_FP32> {
    using type = float;
};
template <>
struct Elem<WQ_BF16> {
    using type = __bf16;
};
template <>
struct Elem<WQ_FP16> {
    using type = _Float16;
};

// Eight adjacent elements (aligned to 16 bytes) as fp32, and back.
template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8]) {
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
        const vec t = ((const vec *)p)[k];
#pragma unroll
        for (int j = 0; j < 16 / (int)sizeof(T); ++j) v[k * 16 / sizeof(T) + j] = (float)t[j];
    }
}
// The same of elements that are aligned to themselves only.
template <typename T>
__device__ __forceinline__ void load8_anywhere(const T *p, float (&v)[8]) {
    T t[8];
    __builtin_memcpy(t, p, sizeof t);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)t[j];
}
// (stored past the caches: what comes next reads the codes)
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
        vec t;
#pragma unroll
        for (int j = 0; j < 16 / (int)sizeof(T); ++j) t[j] = (T)v[k * 16 / sizeof(T) + j];
        __builtin_nontemporal_store(t, (vec *)p + k);
    }
}

// A lane's eight codes and the scale of its group of g elements = g / 8 adjacent lanes (32 to 512: all of one wave).
__device__ __forceinline__ uint2 quantize_piece(const float (&v)[8], int g, float &s) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
    top = dpp_max<0xB1>(top);   // quad_perm [1,0,3,2]
    top = dpp_max<0x4E>(top);   // quad_perm [2,3,0,1]: the 4 lanes of 32 elements
    if (g > 32) top = dpp_max<0x141>(top);   // row_half_mirror: 8 lanes
    if (g > 64) top = dpp_max<0x140>(top);   // row_mirror: 16 lanes
    if (g > 128) top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    if (g > 256) top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    float r;
    group_scale(__uint_as_float(top), s, r);
    return make_uint2(quant_code(v[0], r) | (quant_code(v[1], r) << 8) | (quant_code(v[2], r) << 16) | (quant_code(v[3], r) << 24),
                      quant_code(v[4], r) | (quant_code(v[5], r) << 8) | (quant_code(v[6], r) << 16) | (quant_code(v[7], r) << 24));
}

}  // namespace
