// Microscaled 4-bit rows: their format, and how it is made and read.  Not part
// of the public ABI.
//
// 32 consecutive elements of a row share a power of two 2^(s - 127) of one byte
// s; an element is a sign, two bits of exponent and one of mantissa: 0, 0.5, 1,
// 1.5, 2, 3, 4 or 6.  A block's power is that of its largest element less 2, the
// power of 4: x = 2^(s - 127) * e, e rounded to the nearest (ties to the even
// code) and 6 at most.
#pragma once

#include "psc_ops.hpp"

namespace psc {

constexpr int kMxBlock = 32;       // elements of a scale
constexpr int kMxNaN = 255;        // the scale of a block with an infinity or a NaN
constexpr int kVec = 8;            // elements that a thread takes at once

// Elements d .. d + 7 of a row of D, zeros from D on.
template <bool kBf16>
__device__ __forceinline__ void load_eight(const void *row, int64_t d, int64_t D, float (&v)[kVec]) {
    using T = typename Logit<kBf16>::type;
    const T *p = static_cast<const T *>(row) + d;
    T t[kVec] = {};
    if (d + kVec <= D) __builtin_memcpy(t, p, sizeof t);
    else
        for (int k = 0; k < kVec; k++)
            if (d + k < D) t[k] = p[k];
#pragma unroll
    for (int k = 0; k < kVec; k++) {
        if constexpr (kBf16) v[k] = from_bf16(t[k]);
        else v[k] = t[k];
    }
}

// Elements d .. d + 7 of a row to memory, those from D on left out.
template <bool kBf16>
__device__ __forceinline__ void store_eight(void *row, int64_t d, int64_t D, const float (&v)[kVec]) {
    using T = typename Logit<kBf16>::type;
    T *p = static_cast<T *>(row) + d;
    T t[kVec];
#pragma unroll
    for (int k = 0; k < kVec; k++) {
        if constexpr (kBf16) t[k] = to_bf16(v[k]);
        else t[k] = v[k];
    }
    if (d + kVec <= D) __builtin_memcpy(p, t, sizeof t);
    else
        for (int k = 0; k < kVec; k++)
            if (d + k < D) p[k] = t[k];
}

// Eight elements of a block to codes, lowest first; four neighbouring lanes
// hold a block, and all of them take part.  The quotient by the scale is exact,
// the conversion rounds once.
__device__ __forceinline__ uint32_t to_mx4(const float (&v)[kVec], uint32_t &scale) {
    uint32_t most = 0;             // of the absolute values' bits: a NaN's are above an infinity's
#pragma unroll
    for (int k = 0; k < kVec; k++) most = max(most, __builtin_bit_cast(uint32_t, v[k]) & 0x7FFFFFFFu);
    most = max(most, dpp_from<0xB1, 0xF>(most, 0u));       // lane ^ 1
    most = max(most, dpp_from<0x4E, 0xF>(most, 0u));       // lane ^ 2
    if (most >= 0x7F800000u) {
        scale = kMxNaN;
        return 0;
    }
    // the exponent's bits of the largest; numbers below 2^-126 have the power of a scale of 0 at most
    scale = max(most >> 23, 2u) - 2;
    const float by = __builtin_bit_cast(float, (254 - scale) << 23);       // 2^(127 - scale)
    uint32_t out = 0;
#pragma unroll
    for (int k = 0; k < kVec; k += 2) {
        switch (k) {
            case 0: out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, v[k] * by, v[k + 1] * by, 1.0f, 0); break;
            case 2: out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, v[k] * by, v[k + 1] * by, 1.0f, 1); break;
            case 4: out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, v[k] * by, v[k + 1] * by, 1.0f, 2); break;
            default: out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, v[k] * by, v[k + 1] * by, 1.0f, 3); break;
        }
    }
    return out;
}

// A scale as a float of that exponent: what the conversions and matrix
// instructions take a power of two by (0 stands for 2^-127, an infinity for NaN).
__device__ __forceinline__ float mx_power(uint32_t scale) { return __builtin_bit_cast(float, scale << 23); }

// Eight codes as pairs of bfloat16, scaled: no rounding from 2^-133 on, the smallest bfloat16; from 2^128 on infinite (4 and 6
// with a scale of 253, 2 and more with one of 254).
__device__ __forceinline__ void from_mx4(uint32_t codes, float power, uint32_t (&out)[4]) {
    out[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 0));
    out[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 1));
    out[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 2));
    out[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 3));
}

}  // namespace psc
