// Stored NVFP4 weights as bf16 in registers, for the operators that apply a
// stored layer (adapt.hip, experts.hip).
#pragma once

#include "common.h"

namespace {

// The E4M3 value of a scale code times 2^e, exact and without a branch: the
// code's fields moved to those of an fp32 stand for the value times 2^-120, the
// subnormal ones among them.
__device__ __forceinline__ float scale_value(uint32_t code, int e) {
    return ldexpf(__uint_as_float(code << 20), 120 + e);
}

// Two E2M1 values of byte K of `src` times l, as a pair of bf16: exact.
template <int K>
__device__ __forceinline__ uint32_t stored_pair(uint32_t src, float l) {
    const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(src, 1.0f, K);
    return __builtin_amdgcn_perm(__float_as_uint(v[1] * l), __float_as_uint(v[0] * l), 0x07060302);
}

__device__ __forceinline__ u32x4 stored_eight(uint32_t src, float l) {
    return u32x4{stored_pair<0>(src, l), stored_pair<1>(src, l), stored_pair<2>(src, l), stored_pair<3>(src, l)};
}

// The same with 2^e on the values' side, where the conversion multiplies by it
// at no cost: `two_e` is 2^e, `l` an E4M3 value.
template <int K>
__device__ __forceinline__ uint32_t scaled_pair(uint32_t src, float two_e, float l) {
    const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(src, two_e, K);
    return __builtin_amdgcn_perm(__float_as_uint(v[1] * l), __float_as_uint(v[0] * l), 0x07060302);
}

__device__ __forceinline__ u32x4 scaled_eight(uint32_t src, float two_e, float l) {
    return u32x4{scaled_pair<0>(src, two_e, l), scaled_pair<1>(src, two_e, l), scaled_pair<2>(src, two_e, l),
                 scaled_pair<3>(src, two_e, l)};
}

}  // namespace
