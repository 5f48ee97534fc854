// What the device files of the operators around a step's logits share
// (psc_head.hip, psc_head_mx.hip, psc_rows.hip, psc_penalize.hip, psc_sample.hip).
// Not part of the public ABI.
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

// ---------------------------------------------------------------- masking

// Rows are masked in tiles of kTileBytes of memory, cut at 128-byte lines, so
// that full lines are written whole whatever a row's alignment.
constexpr int kTileBytes = 4096, kLineBytes = 128;
constexpr int32_t tiles_of_row(int64_t V, int32_t elem) {      // for any alignment of the row
    return (int32_t)(((int64_t)V * elem + kLineBytes - elem + kTileBytes - 1) / kTileBytes);
}

// -inf in the forbidden logits of tiles t0 .. t0 + kTiles - 1 of a row, by one
// wavefront, with stores alone: other logits are neither read nor written.  The
// words of all the tiles are loaded first.  Lane l has the bits of elements 32 l
// .. 32 l + 31 of a tile, put together from the two words that they lie in; a
// line that is forbidden whole is written in vectors, of the others 64
// elements at a time, whose bits are the store's execution mask.
template <bool kBf16, int kTiles>
__device__ __forceinline__ void forbid_tiles(void *row, const uint32_t *__restrict__ words, int32_t V, int32_t W, int32_t t0, int lane) {
    constexpr int kElem = kBf16 ? 2 : 4, kWords = kTileBytes / kElem / 32, kVecsPerWord = 2 * kElem;
    const uintptr_t addr = reinterpret_cast<uintptr_t>(row);
    char *const line = reinterpret_cast<char *>(addr & ~(uintptr_t)(kLineBytes - 1));
    const int32_t delta = (int32_t)(addr & (kLineBytes - 1)) / kElem;      // elements of the line before the row
    const int32_t before = (delta + 31) / 32, shift = before * 32 - delta;
    uint32_t drop[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; i++) {
        const int64_t w = (int64_t)(t0 + i) * kWords + lane - before;
        const bool mine = lane < kWords;
        const uint32_t lo = mine && w >= 0 && w < W ? words[w] : 0, hi = mine && shift && w >= -1 && w + 1 < W ? words[w + 1] : 0;
        const int64_t p0 = ((int64_t)(t0 + i) * kWords + lane) * 32, left = (int64_t)delta + V - p0;
        uint32_t inside = mine ? ~0u : 0u;
        if (p0 < delta) inside &= delta - p0 >= 32 ? 0u : ~0u << (delta - p0);
        if (left < 32) inside &= left <= 0 ? 0u : ~(~0u << left);
        drop[i] = ~__builtin_amdgcn_alignbit(hi, lo, shift) & inside;
    }
    constexpr uint32_t kInf = kBf16 ? 0xFF80FF80u : 0xFF800000u;
    // written through at device scope (16), whole lines as a stream (2): they need not stay in a cache
    constexpr int kWhole = 16 | 2, kPart = 16;
#pragma unroll
    for (int i = 0; i < kTiles; i++) {
        if (!__ballot(drop[i])) continue;
        const __amdgpu_buffer_rsrc_t rsrc = buffer_of(line + (int64_t)(t0 + i) * kTileBytes, kTileBytes);
        const uint32_t other = kBf16 ? dpp_from<0xB1, 0xF>(drop[i], 0u) : ~0u;      // a bfloat16 line is two words: the pair's other lane
        const bool full = drop[i] == ~0u && other == ~0u;
        const uint64_t lines = __ballot(full);
        const u32x4 inf = {kInf, kInf, kInf, kInf};
#pragma unroll
        for (int j = 0; j < kTileBytes / 16 / kWave; j++) {
            const int v = j * kWave + lane;
            if ((lines >> (v / kVecsPerWord)) & 1) __builtin_amdgcn_raw_buffer_store_b128(inf, rsrc, (uint32_t)v * 16u, 0, kWhole);
        }
        const uint32_t rest = full ? 0u : drop[i];
        const uint64_t some = __ballot(rest != 0);
        if (!some) continue;
#pragma unroll
        for (int k = 0; k < kWords; k += 2) {
            if (!((some >> k) & 3)) continue;
            const uint64_t bits = lane_value(rest, k) | (uint64_t)lane_value(rest, k + 1) << 32;
            if (__builtin_amdgcn_inverse_ballot_w64(bits)) {
                const uint32_t at = (uint32_t)(k * 32 + lane) * kElem;
                if (kBf16) __builtin_amdgcn_raw_buffer_store_b16((short)0xFF80, rsrc, at, 0, kPart);
                else __builtin_amdgcn_raw_buffer_store_b32(0xFF800000u, rsrc, at, 0, kPart);
            }
        }
    }
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
