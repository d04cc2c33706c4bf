// Reductions over the lanes of a wavefront and conversions shared by the kernels around the layer.
#pragma once
#include "common.h"

// 8-bit values are e4m3 (largest 448) with an fp32 scale per row or block: scale = max / 448, code = value / scale.
// A row or block whose largest magnitude is below Q8_TINY has scale 0 and codes 0 (its reciprocal would overflow).
constexpr float Q8_MAX = 448.0f, Q8_TINY = 1e-30f;

// what lane (l ^ 1, l ^ 2, 7 - l and 15 - l inside groups of 8 and 16) holds: the first four steps of a butterfly without
// an LDS round trip.  The mirrors are as good as l ^ 4 and l ^ 8 once all lanes of a group of 4 or 8 hold the same.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;

// Op over the LANES (8, 16, 32 or 64) neighbouring lanes, the result in every one of them
template <int LANES, class Op>
__device__ __forceinline__ uint32_t lanes_reduce(uint32_t v, Op op) {
    v = op(v, dpp<DPP_XOR1>(v));
    v = op(v, dpp<DPP_XOR2>(v));
    v = op(v, dpp<DPP_HALF_MIRROR>(v));
    if constexpr (LANES >= 16) v = op(v, dpp<DPP_MIRROR>(v));
    if constexpr (LANES >= 32) v = op(v, (uint32_t)__shfl_xor((int)v, 16));
    if constexpr (LANES >= 64) v = op(v, (uint32_t)__shfl_xor((int)v, 32));
    return v;
}
struct AddF32 {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }
};
// magnitudes as bit patterns: infinity is above every number and NaN above infinity, so neither gets lost
struct MaxBits {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) { return __uint_as_float(lanes_reduce<LANES>(__float_as_uint(v), AddF32())); }
template <int LANES>
__device__ __forceinline__ float lanes_max_abs(float v) {      // v's sign bit is clear
    return __uint_as_float(lanes_reduce<LANES>(__float_as_uint(v), MaxBits()));
}
__device__ __forceinline__ float max_abs(float top, float v) {
    const uint32_t a = __float_as_uint(top), b = __float_as_uint(v) & 0x7FFFFFFFu;
    return __uint_as_float(a > b ? a : b);
}

// scale and its reciprocal from the largest magnitude
struct Q8Scale { float scale, inv; };
__device__ __forceinline__ Q8Scale q8_scale(float top) {
    const bool none = top < Q8_TINY;                            // false for NaN
    return {none ? 0.0f : top * (1.0f / Q8_MAX), none ? 0.0f : (1.0f / top) * Q8_MAX};
}

struct F8 { float v[8]; };
__device__ __forceinline__ F8 unpack_bf16(u32x4 p) {
    F8 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o.v[2 * i] = __uint_as_float(p[i] << 16);
        o.v[2 * i + 1] = __uint_as_float(p[i] & 0xFFFF0000u);
    }
    return o;
}
__device__ __forceinline__ u32x4 pack_bf16(const F8& x) {      // nearest, ties to even
    union { __bf16 h[8]; u32x4 u; } o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.h[i] = (__bf16)x.v[i];
    return o.u;
}
// nearest, ties to even; the caller keeps magnitudes below 464, which is where rounding passes 448
__device__ __forceinline__ u32x2 pack_e4m3(const F8& x) {
    u32x2 o;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(x.v[4 * i], x.v[4 * i + 1], 0, false);
        o[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x.v[4 * i + 2], x.v[4 * i + 3], p, true);
    }
    return o;
}
typedef float f32x2 __attribute__((ext_vector_type(2)));
