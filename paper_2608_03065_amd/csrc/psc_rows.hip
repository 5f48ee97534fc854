// Operators on quantised rows: microscaled 4-bit rows made (psc_quantize_mx),
// rows of a quantised table read by token (psc_lookup_rows), and the
// root-mean-square norm with the residual's addition whose result goes to any
// of the forms (psc_add_rms_norm).
#include <algorithm>
#include <type_traits>

#include "psc_mx.hpp"

using namespace psc;

namespace {

constexpr int kBlock = 256;
// Workgroups of one launch: a grid's threads are fewer than 2^32 in each dimension.
constexpr int64_t kMostGrid = ((int64_t)1 << 32) / kBlock - 1;

// n / d for n < 2^32 by a multiplication: `magic` is 2^64 / d, rounded up.
struct Divisor {
    uint64_t magic;
    uint32_t d;
    explicit Divisor(uint32_t by) : magic(by > 1 ? ~0ull / by + 1 : 0), d(by) {}
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return d > 1 ? (uint32_t)__umul64hi(magic, n) : n; }
};

// ---------------------------------------------------------------- rows to 4 bits

// A thread takes eight elements, four threads a block.  A row has `eights` of
// them, whole blocks, zeros from D on.  Bound by memory: 128,256 x 4,096 from bfloat16
// take 236 us, 1.3 GB, 5.6 TB/s.
template <bool kBf16>
__global__ void __launch_bounds__(kBlock)
quantize_mx_kernel(const void *__restrict__ x, int64_t x_stride, int32_t D, Divisor eights, uint32_t units,
                   uint8_t *__restrict__ q, int64_t q_stride, uint8_t *__restrict__ scales, int64_t scales_stride) {
    const uint32_t u = blockIdx.x * kBlock + threadIdx.x;
    if (u >= units) return;
    const uint32_t r = eights.quotient(u), k = u - r * eights.d;
    float v[kVec];
    load_eight<kBf16>(static_cast<const char *>(x) + r * x_stride * (kBf16 ? 2 : 4), (int64_t)k * kVec, D, v);
    uint32_t scale;
    const uint32_t codes = to_mx4(v, scale);
    __builtin_memcpy(q + r * q_stride + (int64_t)k * 4, &codes, 4);
    if (k % 4 == 0) scales[r * scales_stride + k / 4] = (uint8_t)scale;
}

// ---------------------------------------------------------------- rows of a table

struct LookupArgs {
    const void *q, *scales;
    int64_t q_stride, scales_stride, n_rows;
    const int32_t *ids;
    void *out;
    int64_t out_stride;
    int64_t first;                // row of the launch's first unit
    int32_t D;
};

// A thread takes eight elements of a row; a row of no table's is zeros.  kStream:
// whole vectors, stored past the caches, which are not to hold what is read once
// after it all: 128,256 x 4,096 from 4 bits to bfloat16 take 259 us (361 by ordinary
// stores), 8,192 x 4,096 from 8 bits 16.3 (22.2), 6.2 TB/s.
template <bool kMx, bool kBf16, bool kStream>
__global__ void __launch_bounds__(kBlock)
lookup_kernel(const LookupArgs a, Divisor eights, uint32_t units) {
    const uint32_t u = blockIdx.x * kBlock + threadIdx.x;
    if (u >= units) return;
    const uint32_t r = eights.quotient(u), k = u - r * eights.d;
    const int64_t at = a.first + r, id = a.ids ? a.ids[at] : at;
    float v[kVec] = {};
    if (id >= 0 && id < a.n_rows) {
        const uint8_t *row = static_cast<const uint8_t *>(a.q) + id * a.q_stride;
        if constexpr (kMx) {
            uint32_t codes, pairs[4];
            __builtin_memcpy(&codes, row + (int64_t)k * 4, 4);
            const uint32_t scale = static_cast<const uint8_t *>(a.scales)[id * a.scales_stride + k / 4];
            from_mx4(codes, mx_power(scale), pairs);
#pragma unroll
            for (int e = 0; e < kVec; e++) v[e] = from_bf16((uint16_t)(pairs[e / 2] >> (16 * (e % 2))));
        } else {
            int8_t t[kVec];
            __builtin_memcpy(t, row + (int64_t)k * kVec, sizeof t);
            const float scale = static_cast<const float *>(a.scales)[id];
#pragma unroll
            for (int e = 0; e < kVec; e++) v[e] = (float)t[e] * scale;
        }
    }
    char *const out = static_cast<char *>(a.out) + at * a.out_stride * (kBf16 ? 2 : 4);
    if constexpr (kStream) {
        constexpr int kStores = kBf16 ? 1 : 2;
        u32x4 t[kStores];
#pragma unroll
        for (int e = 0; e < kVec; e++) {
            if constexpr (kBf16) t[0][e / 2] = e % 2 ? t[0][e / 2] | (uint32_t)to_bf16(v[e]) << 16 : to_bf16(v[e]);
            else t[e / 4][e % 4] = __builtin_bit_cast(uint32_t, v[e]);
        }
#pragma unroll
        for (int i = 0; i < kStores; i++) __builtin_nontemporal_store(t[i], reinterpret_cast<u32x4 *>(out) + (int64_t)k * kStores + i);
    } else store_eight<kBf16>(out, (int64_t)k * kVec, a.D, v);
}

// ---------------------------------------------------------------- the norm

struct NormArgs {
    const void *x;
    void *residual;
    const float *gain;
    void *out, *scales;
    int64_t x_stride, residual_stride, out_stride, scales_stride, n_rows;
    int32_t D, padded;            // padded: elements of the result's row that are written
    float eps;
    bool x_bf16;
};

// Sum or maximum over a row's threads, the same in all of them.
template <int kThreads, class T, class Op>
__device__ __forceinline__ T row_all(T v, T none, const Op &op, T *s_part) {
    v = wave_all(v, none, op);
    if constexpr (kThreads > kWave) {
        if (threadIdx.x % kWave == 0) s_part[threadIdx.x / kWave] = v;
        __syncthreads();
        v = s_part[0];
#pragma unroll
        for (int i = 1; i < kThreads / kWave; i++) v = op(v, s_part[i]);
    }
    return v;
}

// kThreads threads take a row, eight elements a thread at a time.  A row of up to
// kTurns times that is read once and stays in registers, up to twice its gain too; of a
// longer one (kTurns 0) the sum is read again from the residual, or x where there
// is none.  kResidual: none, float32, bfloat16.
//
// Bound by memory where there are many rows: 8,192 x 4,096 with a bfloat16 residual to
// 8 bits take 50.7 us, 235 MB, 4.6 TB/s, what a large copy reaches; one of 2,048 by its
// chain of waits, 3.0 us.
template <psc_form kTo, int kResidual, int kThreads, int kTurns>
__global__ void __launch_bounds__(kThreads > kBlock ? kThreads : kBlock)
norm_kernel(const NormArgs a) {
    constexpr int kRows = kThreads < kBlock ? kBlock / kThreads : 1;      // rows of a workgroup
    constexpr int kParts = kThreads / kWave;
    constexpr bool kHeld = kTurns > 0, kGains = kTurns == 1 || kTurns == 2, kRBf16 = kResidual == 2;
    __shared__ float s_sum[kParts], s_again[kParts];
    __shared__ uint32_t s_most[kParts];
    const int t = threadIdx.x % kThreads;
    const int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / kThreads;
    if (r >= a.n_rows) return;            // whole wavefronts, and where there are barriers, whole workgroups
    const char *const x = static_cast<const char *>(a.x) + r * a.x_stride * (a.x_bf16 ? 2 : 4);
    char *const residual = kResidual ? static_cast<char *>(a.residual) + r * a.residual_stride * (kRBf16 ? 2 : 4) : nullptr;
    const auto load_x = [&](int64_t d, float (&v)[kVec]) {
        if (a.x_bf16) load_eight<true>(x, d, a.D, v);
        else load_eight<false>(x, d, a.D, v);
    };
    const auto load_gain = [&](int64_t d, float (&g)[kVec]) {
        if (a.gain) load_eight<false>(a.gain, d, a.D, g);
        else
#pragma unroll
            for (int k = 0; k < kVec; k++) g[k] = 1.0f;
    };
    // the residual's sum is rounded to its own type before anything is made of it
    const auto add = [&](int64_t d, float (&v)[kVec], const float (&y)[kVec]) {
#pragma unroll
        for (int k = 0; k < kVec; k++) {
            v[k] += y[k];
            if constexpr (kRBf16) v[k] = from_bf16(to_bf16(v[k]));
        }
        store_eight<kRBf16>(residual, d, a.D, v);
    };
    float held[kHeld ? kTurns : 1][kVec], gains[kGains ? kTurns : 1][kVec];
    if constexpr (kHeld) {
        float y[kTurns][kVec];
#pragma unroll
        for (int i = 0; i < kTurns; i++) {
            const int64_t d = ((int64_t)i * kThreads + t) * kVec;
            load_x(d, kResidual ? y[i] : held[i]);
            if constexpr (kResidual != 0) load_eight<kRBf16>(residual, d, a.D, held[i]);
            if constexpr (kGains) load_gain(d, gains[i]);
        }
        if constexpr (kResidual != 0)
#pragma unroll
            for (int i = 0; i < kTurns; i++) add(((int64_t)i * kThreads + t) * kVec, held[i], y[i]);
    }
    // f(first element, the sum there, its gain) for all of the thread's
    const auto each = [&](auto &&f, bool first) {
        if constexpr (kHeld) {
#pragma unroll
            for (int i = 0; i < kTurns; i++) {
                const int64_t d = ((int64_t)i * kThreads + t) * kVec;
                if (!kGains && !first) load_gain(d, gains[0]);
                f(d, held[i], gains[kGains ? i : 0]);
            }
        } else {
            for (int64_t d = (int64_t)t * kVec; d < a.padded; d += kThreads * kVec) {
                if constexpr (kResidual == 0) load_x(d, held[0]);
                else {
                    load_eight<kRBf16>(residual, d, a.D, held[0]);
                    if (first) {
                        float y[kVec];
                        load_x(d, y);
                        add(d, held[0], y);
                    }
                }
                if (!first) load_gain(d, gains[0]);
                f(d, held[0], gains[0]);
            }
        }
    };
    float sum = 0;
    each([&](int64_t, const float (&v)[kVec], const float (&)[kVec]) {
#pragma unroll
        for (int k = 0; k < kVec; k++) sum = __builtin_fmaf(v[k], v[k], sum);
    }, true);
    sum = row_all<kThreads>(sum, 0.0f, kAdd, s_sum);
    // Squares, or their mean with eps, past float32's range: the same of the numbers
    // times 2^-80, or 2^80 where eps is too small to hide it.  An element much smaller
    // than the row's largest would lose bits to 2^-80: it goes with the quotient, all
    // of it but the quarter that keeps that from the subnormal numbers.
    float before = 1, after = 1, eps = a.eps;
    if (!(sum / (float)a.D + eps < __builtin_huge_valf()) || (sum < 0x1p-40f && eps < 0x1p-80f)) {
        const float by = sum < 1 ? 0x1p80f : 0x1p-80f;
        before = sum < 1 ? by : 0x1p-2f;
        after = sum < 1 ? 1.0f : 0x1p-78f;
        eps = eps * by * by;
        sum = 0;
        each([&](int64_t, const float (&v)[kVec], const float (&)[kVec]) {
#pragma unroll
            for (int k = 0; k < kVec; k++) sum = __builtin_fmaf(v[k] * by, v[k] * by, sum);
        }, false);
        sum = row_all<kThreads>(sum, 0.0f, kAdd, s_again);
    }
    const float inverse = 1.0f / __builtin_sqrtf(sum / (float)a.D + eps) * after;
    const auto norm = [&](const float (&v)[kVec], const float (&g)[kVec], float (&y)[kVec]) {
#pragma unroll
        for (int k = 0; k < kVec; k++) y[k] = v[k] * before * inverse * g[k];
    };
    if constexpr (kTo == PSC_FORM_F32 || kTo == PSC_FORM_BF16) {
        constexpr bool kBf16 = kTo == PSC_FORM_BF16;
        char *const out = static_cast<char *>(a.out) + r * a.out_stride * (kBf16 ? 2 : 4);
        each([&](int64_t d, const float (&v)[kVec], const float (&g)[kVec]) {
            if (d >= a.padded) return;
            float y[kVec];
            norm(v, g, y);
            store_eight<kBf16>(out, d, a.D, y);
        }, false);
    } else if constexpr (kTo == PSC_FORM_MX4) {
        uint8_t *const out = static_cast<uint8_t *>(a.out) + r * a.out_stride;
        uint8_t *const scales = static_cast<uint8_t *>(a.scales) + r * a.scales_stride;
        each([&](int64_t d, const float (&v)[kVec], const float (&g)[kVec]) {
            if (d >= a.padded) return;            // whole blocks
            float y[kVec];
            norm(v, g, y);
            if (d + kVec > a.D)
#pragma unroll
                for (int k = 0; k < kVec; k++) y[k] = d + k < a.D ? y[k] : 0.0f;      // 0 times an infinite factor is none
            uint32_t scale;
            const uint32_t codes = to_mx4(y, scale);
            __builtin_memcpy(out + d / 2, &codes, 4);
            if (t % 4 == 0) scales[d / kMxBlock] = (uint8_t)scale;
        }, false);
    } else {
        uint32_t most = 0;            // of the absolute values' bits: a NaN's are above an infinity's
        each([&](int64_t d, const float (&v)[kVec], const float (&g)[kVec]) {
            if (d >= a.D) return;
            float y[kVec];
            norm(v, g, y);
#pragma unroll
            for (int k = 0; k < kVec; k++)
                if (d + k < a.D) most = max(most, __builtin_bit_cast(uint32_t, y[k]) & 0x7FFFFFFFu);
        }, false);
        most = row_all<kThreads>(most, 0u, kMax, s_most);
        const bool finite = most < 0x7F800000u;
        const float scale = finite ? __builtin_bit_cast(float, most) / 127.0f : __builtin_nanf("");
        if (t == 0) static_cast<float *>(a.scales)[r] = scale;
        int8_t *const out = static_cast<int8_t *>(a.out) + r * a.out_stride;
        // Quotients by the scale's reciprocal and one correction by the remainder, which is exact, a division's
        // result in three operations for its ten; a scale whose reciprocal or remainders leave the range divides.
        const bool divides = !(scale > 0x1p-100f);
        const float reciprocal = 1.0f / scale;
        each([&](int64_t d, const float (&v)[kVec], const float (&g)[kVec]) {
            if (d >= a.padded) return;
            float y[kVec];
            norm(v, g, y);
            uint64_t codes = 0;
#pragma unroll
            for (int k = 0; k < kVec; k++) {
                const float near = y[k] * reciprocal;
                float f = __builtin_fmaf(__builtin_fmaf(-near, scale, y[k]), reciprocal, near);
                if (divides) f = scale > 0 ? y[k] / scale : 0.0f;
                f = d + k < a.D ? __builtin_rintf(f) : 0.0f;
                codes |= (uint64_t)(uint8_t)(int8_t)(int)fminf(fmaxf(f, -127.0f), 127.0f) << (8 * k);
            }
            __builtin_memcpy(out + d, &codes, sizeof codes);
        }, false);
    }
}

// ---------------------------------------------------------------- host side

// f(first row, units) for launches that hold all rows of `eights` units each.
template <class F>
void by_launches(int64_t n_rows, int64_t eights, const F &f) {
    const int64_t most = std::max<int64_t>(1, kMostGrid * kBlock / eights);
    for (int64_t r = 0; r < n_rows; r += most) f(r, (uint32_t)(std::min(most, n_rows - r) * eights));
}

dim3 grid_of(uint32_t units) { return dim3((units + kBlock - 1) / kBlock); }

constexpr int32_t kMostD = 1 << 30;

bool is_form(int32_t f) { return f >= PSC_FORM_F32 && f <= PSC_FORM_MX4; }
int64_t whole(int64_t n, int64_t of) { return (n + of - 1) / of * of; }

// Rows of 4-bit codes and of their scales.
psc_status check_mx(const char *what, const void *q, int64_t q_stride, const void *scales, int64_t scales_stride, int64_t D) {
    if (!q || !scales) return refuse(what, "null pointer");
    if (q_stride % 16 || q_stride < (D + 1) / 2 || !aligned_to(q, 16)) return refuse(what, "rows of q start at 16 bytes and hold D elements");
    if (scales_stride % 4 || scales_stride < (D + kMxBlock - 1) / kMxBlock || !aligned_to(scales, 4))
        return refuse(what, "rows of scales start at 4 bytes and hold one of every 32 elements");
    return PSC_OK;
}

psc_status check_i8(const char *what, const void *q, int64_t q_stride, const void *scales, int64_t D) {
    if (!q || !scales) return refuse(what, "null pointer");
    if (q_stride % 16 || q_stride < D || !aligned_to(q, 16)) return refuse(what, "rows of q start at 16 bytes and hold D elements");
    if (!aligned_to(scales, 4)) return refuse(what, "scales off their elements' alignment");
    return PSC_OK;
}

template <psc_form kTo, int kResidual>
void launch_norm(const NormArgs &all, hipStream_t s) {
    NormArgs a = all;
    const auto go = [&](auto kernel, int threads, int rows) {
        for (int64_t left = all.n_rows; left > 0;) {
            const int64_t n = std::min<int64_t>(left, (((int64_t)1 << 32) / threads - 1) * rows);
            a.n_rows = n;
            hipLaunchKernelGGL(kernel, dim3((uint32_t)((n + rows - 1) / rows)), dim3(threads), 0, s, a);
            left -= n;
            a.x = static_cast<const char *>(a.x) + n * a.x_stride * (a.x_bf16 ? 2 : 4);
            if (kResidual) a.residual = static_cast<char *>(a.residual) + n * a.residual_stride * (kResidual == 2 ? 2 : 4);
            constexpr int kSize = kTo == PSC_FORM_F32 ? 4 : kTo == PSC_FORM_BF16 ? 2 : 1;
            a.out = static_cast<char *>(a.out) + n * a.out_stride * kSize;
            if (kTo == PSC_FORM_I8) a.scales = static_cast<float *>(a.scales) + n;
            if (kTo == PSC_FORM_MX4) a.scales = static_cast<char *>(a.scales) + n * a.scales_stride;
        }
    };
    // Threads of a row: a wavefront where it holds the row in two turns, else the fewest that hold it.
    const int64_t vectors = (a.padded + kVec - 1) / kVec;
    if (vectors <= 64 * 2) go(norm_kernel<kTo, kResidual, 64, 2>, kBlock, kBlock / 64);
    else if (vectors <= 256) go(norm_kernel<kTo, kResidual, 256, 1>, 256, 1);
    else if (vectors <= 256 * 2) go(norm_kernel<kTo, kResidual, 256, 2>, 256, 1);
    else if (vectors <= 256 * 4) go(norm_kernel<kTo, kResidual, 256, 4>, 256, 1);
    else if (vectors <= 1024 * 2) go(norm_kernel<kTo, kResidual, 1024, 2>, 1024, 1);
    else if (vectors <= 1024 * 4) go(norm_kernel<kTo, kResidual, 1024, 4>, 1024, 1);
    else go(norm_kernel<kTo, kResidual, 1024, 0>, 1024, 1);
}

template <psc_form kTo>
void launch_norm(const NormArgs &a, int residual, hipStream_t s) {
    if (residual == 0) launch_norm<kTo, 0>(a, s);
    else if (residual == 1) launch_norm<kTo, 1>(a, s);
    else launch_norm<kTo, 2>(a, s);
}

}  // namespace

extern "C" psc_status psc_quantize_mx(const void *x, psc_dtype dtype, int64_t x_stride, int64_t n_rows, int32_t D, uint8_t *q,
                                      int64_t q_stride, uint8_t *scales, int64_t scales_stride, void *stream) {
    const char *what = "psc_quantize_mx";
    if (!is_dtype(dtype)) return refuse(what, "bad dtype");
    if (n_rows < 0 || D < 0) return refuse(what, "negative size");
    if (n_rows == 0 || D == 0) return PSC_OK;
    if (n_rows > INT32_MAX) return refuse(what, "more than 2^31 - 1 rows");
    if (D > kMostD) return refuse(what, "D > 2^30");
    if (!x) return refuse(what, "null pointer");
    if (x_stride < 0 || !aligned_to(x, size_of(dtype))) return refuse(what, "negative stride, or x off its elements' alignment");
    if (psc_status st = check_mx(what, q, q_stride, scales, scales_stride, D)) return st;
    const int64_t eights = whole(D, kMxBlock) / kVec;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    by_launches(n_rows, eights, [&](int64_t r, uint32_t units) {
        const auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid_of(units), dim3(kBlock), 0, s, static_cast<const char *>(x) + r * x_stride * size_of(dtype), x_stride,
                               D, Divisor((uint32_t)eights), units, q + r * q_stride, q_stride, scales + r * scales_stride, scales_stride);
        };
        if (dtype == PSC_BF16) go(quantize_mx_kernel<true>);
        else go(quantize_mx_kernel<false>);
    });
    return launched_op(what);
}

extern "C" psc_status psc_lookup_rows(psc_form form, const void *q, int64_t q_stride, const void *scales, int64_t scales_stride,
                                      int64_t n_rows, int32_t D, const int32_t *ids, int64_t n, void *out, psc_dtype dtype,
                                      int64_t out_stride, void *stream) {
    const char *what = "psc_lookup_rows";
    if (form != PSC_FORM_I8 && form != PSC_FORM_MX4) return refuse(what, "bad form");
    if (!is_dtype(dtype)) return refuse(what, "bad dtype");
    if (n_rows < 0 || D < 0 || n < 0) return refuse(what, "negative size");
    if (n == 0 || D == 0) return PSC_OK;
    if (n > INT32_MAX || n_rows > INT32_MAX) return refuse(what, "more than 2^31 - 1 rows");
    if (D > kMostD) return refuse(what, "D > 2^30");
    if (!ids && n > n_rows) return refuse(what, "more rows than the table has");
    if (!out) return refuse(what, "null pointer");
    if (n > 1 && out_stride < D) return refuse(what, "rows of out overlap (stride < D)");
    if (!aligned_to(out, size_of(dtype)) || (ids && !aligned_to(ids, 4))) return refuse(what, "out or ids off their elements' alignment");
    if (n_rows > 0)        // of a table without rows nothing is read
        if (psc_status st = form == PSC_FORM_MX4 ? check_mx(what, q, q_stride, scales, scales_stride, D) : check_i8(what, q, q_stride, scales, D)) return st;
    const int64_t eights = (D + kVec - 1) / kVec;
    const bool streams = D % kVec == 0 && aligned_to(out, 16) && (n == 1 || out_stride * size_of(dtype) % 16 == 0);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    by_launches(n, eights, [&](int64_t r, uint32_t units) {
        const LookupArgs a{q, scales, q_stride, scales_stride, n_rows, ids, out, out_stride, r, D};
        const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid_of(units), dim3(kBlock), 0, s, a, Divisor((uint32_t)eights), units); };
        const auto of = [&](auto mx, auto bf16) {
            if (streams) go(lookup_kernel<mx, bf16, true>);
            else go(lookup_kernel<mx, bf16, false>);
        };
        constexpr std::true_type yes;
        constexpr std::false_type no;
        if (form == PSC_FORM_MX4) {
            if (dtype == PSC_BF16) of(yes, yes);
            else of(yes, no);
        } else {
            if (dtype == PSC_BF16) of(no, yes);
            else of(no, no);
        }
    });
    return launched_op(what);
}

extern "C" psc_status psc_add_rms_norm(const void *x, psc_dtype x_dtype, int64_t x_stride, void *residual, psc_dtype residual_dtype,
                                       int64_t residual_stride, int64_t n_rows, int32_t D, const float *gain, float eps, psc_form to,
                                       void *out, int64_t out_stride, void *scales, int64_t scales_stride, void *stream) {
    const char *what = "psc_add_rms_norm";
    if (!is_dtype(x_dtype) || (residual && !is_dtype(residual_dtype))) return refuse(what, "bad dtype");
    if (!is_form(to)) return refuse(what, "bad form");
    if (n_rows < 0 || D < 0) return refuse(what, "negative size");
    if (!(eps >= 0)) return refuse(what, "eps is a number of at least 0");
    if (n_rows == 0 || D == 0) return PSC_OK;
    if (n_rows > INT32_MAX) return refuse(what, "more than 2^31 - 1 rows");
    if (D > kMostD) return refuse(what, "D > 2^30");
    if (!x || !out) return refuse(what, "null pointer");
    if (x_stride < 0 || !aligned_to(x, size_of(x_dtype))) return refuse(what, "negative stride, or x off its elements' alignment");
    if (residual && ((n_rows > 1 && residual_stride < D) || !aligned_to(residual, size_of(residual_dtype))))
        return refuse(what, "rows of the residual overlap, or it is off its elements' alignment");
    if (!aligned_to(gain, 4)) return refuse(what, "gain off its elements' alignment");
    NormArgs a{x, residual, gain, out, scales, x_stride, residual_stride, out_stride, scales_stride, n_rows, D, D, eps, x_dtype == PSC_BF16};
    if (to == PSC_FORM_MX4) {
        if (psc_status st = check_mx(what, out, out_stride, scales, scales_stride, D)) return st;
        a.padded = (int32_t)whole(D, kMxBlock);
    } else if (to == PSC_FORM_I8) {
        if (psc_status st = check_i8(what, out, out_stride, scales, D)) return st;
        a.padded = (int32_t)whole(D, 16);
    } else {
        const int64_t size = to == PSC_FORM_BF16 ? 2 : 4;
        if ((n_rows > 1 && out_stride < D) || !aligned_to(out, size)) return refuse(what, "rows of out overlap, or it is off its elements' alignment");
    }
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const int kind = !residual ? 0 : residual_dtype == PSC_BF16 ? 2 : 1;
    switch (to) {
        case PSC_FORM_F32: launch_norm<PSC_FORM_F32>(a, kind, s); break;
        case PSC_FORM_BF16: launch_norm<PSC_FORM_BF16>(a, kind, s); break;
        case PSC_FORM_I8: launch_norm<PSC_FORM_I8>(a, kind, s); break;
        default: launch_norm<PSC_FORM_MX4>(a, kind, s); break;
    }
    return launched_op(what);
}
