// What the device files of the operators around a step's logits share
// (psc_head.hip, psc_penalize.hip, psc_sample.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "psc_internal.hpp"

namespace psc {

constexpr int kWave = 64;
constexpr float kMinusInf = -__builtin_huge_valf();

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// A raw buffer resource over `bytes` bytes at p: accesses at an offset >=
// bytes are dropped by the hardware (a load gives zeros).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int32_t)bytes, 0x00020000);
}

// The value of another lane, moved by a DPP control into the rows of kRowMask;
// `none` where there is no such lane.
template <int kCtrl, int kRowMask, class T>
__device__ __forceinline__ T dpp_from(T v, T none) {
    static_assert(sizeof(T) == 4, "one register");
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), kCtrl,
                                                             kRowMask, 0xF, false));
}

// op over the lanes up to this one, in a fixed order; `none` is op's neutral
// element.  Shifts by 1, 2, 4 and 8 within rows of 16 lanes, then lane 15 into
// the rows after its own pair's first (row_bcast:15) and lane 31 into the
// upper half.  Every lane of the wavefront takes part.
template <class T, class Op>
__device__ __forceinline__ T wave_scan(T v, T none, const Op &op) {
    v = op(v, dpp_from<0x111, 0xF>(v, none));
    v = op(v, dpp_from<0x112, 0xF>(v, none));
    v = op(v, dpp_from<0x114, 0xF>(v, none));
    v = op(v, dpp_from<0x118, 0xF>(v, none));
    v = op(v, dpp_from<0x142, 0xA>(v, none));
    return op(v, dpp_from<0x143, 0xC>(v, none));
}

template <class T>
__device__ __forceinline__ T lane_value(T v, int lane) {      // `lane` is uniform
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// op over the wavefront's lanes, uniform.
template <class T, class Op>
__device__ __forceinline__ T wave_all(T v, T none, const Op &op) {
    return lane_value(wave_scan(v, none, op), kWave - 1);
}

constexpr auto kAdd = [](auto a, auto b) { return a + b; };
constexpr auto kMax = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
constexpr auto kMin = [](uint32_t a, uint32_t b) { return a < b ? a : b; };

// Logits are float32 or bfloat16; the arithmetic on them is float32.
template <bool kBf16>
struct Logit {
    using type = float;
};
template <>
struct Logit<true> {
    using type = uint16_t;
};

__device__ __forceinline__ float from_bf16(uint16_t u) { return __builtin_bit_cast(float, (uint32_t)u << 16); }
// Round to nearest, ties to even.
__device__ __forceinline__ uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

template <bool kBf16>
__device__ __forceinline__ float load_logit(const void *row, int64_t v) {
    if (kBf16) return from_bf16(static_cast<const uint16_t *>(row)[v]);
    return static_cast<const float *>(row)[v];
}
template <bool kBf16>
__device__ __forceinline__ void store_logit(void *row, int64_t v, float f) {
    if (kBf16) static_cast<uint16_t *>(row)[v] = to_bf16(f);
    else static_cast<float *>(row)[v] = f;
}

// ---------------------------------------------------------------- host side

inline psc_status refuse(const char *what, const std::string &why) {
    set_error(std::string(what) + ": " + why);
    return PSC_E_INVALID_ARG;
}

inline psc_status launched_op(const char *what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return PSC_OK;
    set_error(std::string(what) + ": " + hipGetErrorString(e));
    return PSC_E_DEVICE;
}

inline bool is_dtype(psc_dtype d) { return d == PSC_F32 || d == PSC_BF16; }
inline int64_t size_of(psc_dtype d) { return d == PSC_BF16 ? 2 : 4; }
inline bool aligned_to(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// The checks of logits [B][V] with rows `stride` elements apart.
inline psc_status check_rows(const char *what, const void *logits, psc_dtype dtype, int64_t stride, int32_t B, int32_t V) {
    if (!is_dtype(dtype)) return refuse(what, "bad dtype");
    if (B < 0 || V < 0) return refuse(what, "negative size");
    if (B > 0 && V > 0 && !logits) return refuse(what, "null logits");
    if (B > 1 && stride < V) return refuse(what, "rows overlap (stride < V)");
    if (!aligned_to(logits, size_of(dtype))) return refuse(what, "logits off their elements' alignment");
    return PSC_OK;
}

}  // namespace psc
