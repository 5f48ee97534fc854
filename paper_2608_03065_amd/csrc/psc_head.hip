// The output projection in 8-bit integers (psc_quantize_rows, psc_head_logits):
// rows of int8 with one scale each on both sides, products summed exactly in
// 32-bit integers by the matrix cores, and one epilogue that scales, adds the
// bias, applies the grammar mask and rounds once.
#include "psc_ops.hpp"

#include <algorithm>

using namespace psc;

namespace {

// ---------------------------------------------------------------- rows to int8

// x[d] = scale * q[d]: scale = max |x| / 127 and q = rint(x / scale) (ties to
// even), both divisions in float32.  A row of zeros has scale 0; a row with an
// infinity or a NaN has scale NaN and q 0, so that every product with it is NaN.
constexpr int kQuantBlock = 256;
constexpr int kQuantVec = 8;      // elements per load

template <bool kBf16>
__device__ __forceinline__ void load_vec(const void *row, int64_t d, int32_t D, float (&v)[kQuantVec]) {
    using T = typename Logit<kBf16>::type;
    const T *p = static_cast<const T *>(row) + d;
    T t[kQuantVec] = {};
    if (d + kQuantVec <= D) __builtin_memcpy(t, p, sizeof t);
    else
        for (int k = 0; k < kQuantVec; k++)
            if (d + k < D) t[k] = p[k];
#pragma unroll
    for (int k = 0; k < kQuantVec; k++) {
        if constexpr (kBf16) v[k] = from_bf16(t[k]);
        else v[k] = t[k];
    }
}

// One workgroup per row; q[D .. padded) become zeros.
template <bool kBf16>
__global__ void __launch_bounds__(kQuantBlock)
quantize_kernel(const void *__restrict__ x, int64_t x_stride, int32_t D, int32_t padded, int8_t *__restrict__ q,
                int64_t q_stride, float *__restrict__ scales) {
    __shared__ uint32_t s_most[kQuantBlock / kWave];
    const int64_t r = blockIdx.x;
    const char *row = static_cast<const char *>(x) + r * x_stride * (kBf16 ? 2 : 4);
    uint32_t most = 0;            // of the absolute values' bits: a NaN's are above an infinity's
    float v[kQuantVec];
    for (int32_t d = threadIdx.x * kQuantVec; d < D; d += kQuantBlock * kQuantVec) {
        load_vec<kBf16>(row, d, D, v);
#pragma unroll
        for (int k = 0; k < kQuantVec; k++) most = max(most, __builtin_bit_cast(uint32_t, v[k]) & 0x7FFFFFFFu);
    }
    for (int o = kWave / 2; o > 0; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o, kWave));
    if (threadIdx.x % kWave == 0) s_most[threadIdx.x / kWave] = most;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kQuantBlock / kWave; k++) most = max(most, s_most[k]);
    const bool finite = most < 0x7F800000u;
    const float scale = finite ? __builtin_bit_cast(float, most) / 127.0f : __builtin_nanf("");
    if (threadIdx.x == 0) scales[r] = scale;
    int8_t *to = q + r * q_stride;
    for (int32_t d = threadIdx.x * kQuantVec; d < padded; d += kQuantBlock * kQuantVec) {
        load_vec<kBf16>(row, d, D, v);
        uint64_t out = 0;
#pragma unroll
        for (int k = 0; k < kQuantVec; k++) {
            // past D the element is 0; a scale too small for its row's maximum (a subnormal one) is clamped
            const float f = scale > 0 ? __builtin_rintf(v[k] / scale) : 0.0f;
            out |= (uint64_t)(uint8_t)(int8_t)(int)fminf(fmaxf(f, -127.0f), 127.0f) << (8 * k);
        }
        __builtin_memcpy(to + d, &out, sizeof out);
    }
}

// ---------------------------------------------------------------- the product

constexpr int kStep = 128;        // bytes of a row per step along D: one line
constexpr int kChunk = 16;        // bytes per lane of a load and of a matrix instruction's operand
constexpr int kChunks = kStep / kChunk;

struct HeadArgs {
    const int8_t *x;              // quantised states, rows x_stride apart, zeros from D up to whole steps
    int64_t x_stride;
    const float *x_scales;
    const int8_t *w;
    int64_t w_stride;
    const float *w_scales, *bias;
    const uint32_t *bitmask;
    void *y;
    int64_t y_stride;
    int32_t B, D, V, W;
    int32_t steps, m_tiles;
};

// Wait until at most n of the wavefront's loads are outstanding and its reads
// of LDS are done, then for the other wavefronts of the workgroup.
template <int n>
__device__ __forceinline__ void wait_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(n) : "memory");
}

// One workgroup computes kM states by kN tokens.  Steps of 128 bytes of all
// its rows go straight from memory into one of kStages buffers in LDS, kStages
// - 1 steps ahead.  A row's 16-byte chunk c lies at place c ^ (row & 7) of its
// 128 bytes, so that the 16 rows that a matrix instruction reads at one chunk
// fall into different banks; since a load puts lane l's chunk at place l, the
// lane fetches the chunk that belongs there.
template <int kM, int kN, int kWavesM, int kWavesN, int kStages, bool kBf16>
__global__ void __launch_bounds__(kWave * kWavesM * kWavesN)
head_kernel(const HeadArgs a) {
    constexpr int kWaves = kWavesM * kWavesN, kRows = kM + kN;
    constexpr int kLoads = kRows * kChunks / (kWaves * kWave);
    static_assert(kLoads * kWaves * kWave == kRows * kChunks && kN % 8 == 0, "every wavefront loads as much");
    constexpr int kTm = kM / kWavesM / 16, kTn = kN / kWavesN / 16;   // 16 x 16 blocks of a wavefront
    __shared__ __align__(1024) int8_t lds[kStages][kRows * kStep];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave % kWavesM, wn = wave / kWavesM;
    const int32_t m0 = (int32_t)(blockIdx.x % a.m_tiles) * kM, n0 = (int32_t)(blockIdx.x / a.m_tiles) * kN;

    const int64_t w_bytes = (int64_t)(a.V - n0 - 1) * a.w_stride + (a.D + kChunk - 1) / kChunk * kChunk;
    const __amdgpu_buffer_rsrc_t rw = buffer_of(a.w + (int64_t)n0 * a.w_stride, (uint32_t)min(w_bytes, (int64_t)INT32_MAX));
    const int64_t x_bytes = (int64_t)(a.B - m0) * a.x_stride;
    const __amdgpu_buffer_rsrc_t rx = buffer_of(a.x + (int64_t)m0 * a.x_stride, (uint32_t)min(x_bytes, (int64_t)INT32_MAX));
    uint32_t from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int row = (i * kWaves + wave) * 8 + lane / 8, chunk = (lane & 7) ^ (row & 7);
        from[i] = (row < kN ? (uint32_t)row * (uint32_t)a.w_stride : (uint32_t)(row - kN) * (uint32_t)a.x_stride) + chunk * kChunk;
    }
    auto fetch = [&](int32_t step) {
        int8_t *to = lds[step % kStages];
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int first = (i * kWaves + wave) * 8;
            // past the last step nothing is read, and the number of accesses stays the same
            const uint32_t off = step < a.steps ? from[i] + (uint32_t)step * kStep : 0x80000000u;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(first < kN ? rw : rx,
                                                     (__attribute__((address_space(3))) void *)(to + first * kStep),
                                                     kChunk, off, 0, 0, 0);
        }
    };
    i32x4 acc[kTn][kTm] = {};
#pragma unroll
    for (int s = 0; s < kStages - 1; s++) fetch(s);
    const int r16 = lane % 16, quad = lane / 16;
    for (int32_t step = 0; step < a.steps; step++) {
        wait_and_meet<(kStages - 2) * kLoads>();   // the step has landed, and its predecessor's buffer is free
        fetch(step + kStages - 1);
        const int8_t *from_lds = lds[step % kStages];
#pragma unroll
        for (int k = 0; k < kStep / 64; k++) {
            i32x4 fw[kTn], fx[kTm];
#pragma unroll
            for (int i = 0; i < kTn; i++) {
                const int row = (wn * kTn + i) * 16 + r16;
                fw[i] = *reinterpret_cast<const i32x4 *>(from_lds + row * kStep + (((k * 4 + quad) ^ (row & 7)) * kChunk));
            }
#pragma unroll
            for (int j = 0; j < kTm; j++) {
                const int row = kN + (wm * kTm + j) * 16 + r16;
                fx[j] = *reinterpret_cast<const i32x4 *>(from_lds + row * kStep + (((k * 4 + quad) ^ (row & 7)) * kChunk));
            }
#pragma unroll
            for (int i = 0; i < kTn; i++)
#pragma unroll
                for (int j = 0; j < kTm; j++)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[i], fx[j], acc[i][j], 0, 0, 0);
        }
    }
    // lane: state r16 of a block, tokens 4 quad .. 4 quad + 3
#pragma unroll
    for (int i = 0; i < kTn; i++) {
        const int32_t v0 = n0 + (wn * kTn + i) * 16 + quad * 4;
        if (v0 >= a.V) continue;
        float ws[4], bias[4] = {};
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int32_t v = min(v0 + e, a.V - 1);
            ws[e] = a.w_scales[v];
            if (a.bias) bias[e] = a.bias[v];
        }
#pragma unroll
        for (int j = 0; j < kTm; j++) {
            const int32_t b = m0 + (wm * kTm + j) * 16 + r16;
            if (b >= a.B) continue;
            const float xs = a.x_scales[b];
            uint32_t bits = 15;
            if (a.bitmask) bits = a.bitmask[(int64_t)b * a.W + (v0 >> 5)] >> (v0 & 31);
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; e++) y[e] = (bits >> e) & 1 ? (float)acc[i][j][e] * xs * ws[e] + bias[e] : kMinusInf;
            using T = typename Logit<kBf16>::type;
            T *to = static_cast<T *>(a.y) + (int64_t)b * a.y_stride + v0;
            T out[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if constexpr (kBf16) out[e] = to_bf16(y[e]);
                else out[e] = y[e];
            }
            if (v0 + 4 <= a.V) __builtin_memcpy(to, out, sizeof out);
            else
                for (int e = 0; e < 4; e++)
                    if (v0 + e < a.V) to[e] = out[e];
        }
    }
}

template <int kM, int kN, int kWavesM, int kWavesN, int kStages>
void launch_head(HeadArgs a, bool bf16, hipStream_t s) {
    a.m_tiles = (a.B + kM - 1) / kM;
    const dim3 grid((uint32_t)a.m_tiles * (uint32_t)((a.V + kN - 1) / kN)), block(kWave * kWavesM * kWavesN);
    if (bf16) hipLaunchKernelGGL((head_kernel<kM, kN, kWavesM, kWavesN, kStages, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((head_kernel<kM, kN, kWavesM, kWavesN, kStages, false>), grid, block, 0, s, a);
}

void launch_quantize(const void *x, psc_dtype dtype, int64_t x_stride, int64_t n_rows, int32_t D, int32_t padded,
                     int8_t *q, int64_t q_stride, float *scales, hipStream_t s) {
    const dim3 grid((uint32_t)n_rows);
    if (dtype == PSC_BF16)
        hipLaunchKernelGGL(quantize_kernel<true>, grid, dim3(kQuantBlock), 0, s, x, x_stride, D, padded, q, q_stride, scales);
    else
        hipLaunchKernelGGL(quantize_kernel<false>, grid, dim3(kQuantBlock), 0, s, x, x_stride, D, padded, q, q_stride, scales);
}

constexpr int32_t kMostD = 131072;       // |sum| <= 127 * 128 * D stays below 2^31
int32_t whole_steps(int32_t D) { return (D + kStep - 1) / kStep * kStep; }
// The workspace: quantised states [B][whole_steps(D)], then their scales.
size_t states_bytes(int32_t B, int32_t D) { return (size_t)B * (size_t)whole_steps(D); }

}  // namespace

extern "C" psc_status psc_quantize_rows(const void *x, psc_dtype dtype, int64_t x_stride, int64_t n_rows, int32_t D,
                                        int8_t *q, int64_t q_stride, float *scales, void *stream) {
    const char *what = "psc_quantize_rows";
    if (!is_dtype(dtype)) return refuse(what, "bad dtype");
    if (n_rows < 0 || D < 0) return refuse(what, "negative size");
    if (n_rows == 0) return PSC_OK;
    const int64_t padded = ((int64_t)D + kChunk - 1) / kChunk * kChunk;
    if ((D > 0 && (!x || !q)) || !scales) return refuse(what, "null pointer");
    if (n_rows > INT32_MAX) return refuse(what, "more than 2^31 - 1 rows");
    if (x_stride < 0 || !aligned_to(x, size_of(dtype))) return refuse(what, "negative stride, or x off its elements' alignment");
    if (q_stride % kChunk || q_stride < padded || !aligned_to(q, kChunk))
        return refuse(what, "rows of q start at 16 bytes and hold D elements");
    launch_quantize(x, dtype, x_stride, n_rows, D, (int32_t)padded, q, q_stride, scales, reinterpret_cast<hipStream_t>(stream));
    return launched_op(what);
}

extern "C" size_t psc_head_workspace(int32_t B, int32_t D, int32_t V) {
    (void)V;
    return B <= 0 || D < 0 ? 0 : states_bytes(B, D) + (size_t)B * sizeof(float);
}

extern "C" psc_status psc_head_logits(const void *x, psc_dtype x_dtype, int64_t x_stride, int32_t B, int32_t D,
                                      const int8_t *w, int64_t w_stride, const float *w_scales, int32_t V,
                                      const float *bias, const uint32_t *bitmask, void *logits, psc_dtype dtype,
                                      int64_t stride, void *workspace, size_t workspace_bytes, void *stream) {
    const char *what = "psc_head_logits";
    if (psc_status st = check_rows(what, logits, dtype, stride, B, V)) return st;
    if (!is_dtype(x_dtype)) return refuse(what, "bad dtype of x");
    if (D < 1 || D > kMostD) return refuse(what, "D outside [1, 131072]");
    if (B == 0 || V == 0) return PSC_OK;
    if (!x || !w || !w_scales || !workspace) return refuse(what, "null pointer");
    if (x_stride < 0 || !aligned_to(x, size_of(x_dtype))) return refuse(what, "negative stride, or x off its elements' alignment");
    if (w_stride % kChunk || w_stride < D || w_stride > INT32_MAX / 512 || !aligned_to(w, kChunk))
        return refuse(what, "rows of w start at 16 bytes and hold D elements");
    if (workspace_bytes < psc_head_workspace(B, D, V) || !aligned_to(workspace, kChunk))
        return refuse(what, "the workspace is too small or not 16-byte aligned");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    HeadArgs a{};
    int8_t *q = static_cast<int8_t *>(workspace);
    float *scales = reinterpret_cast<float *>(q + states_bytes(B, D));
    launch_quantize(x, x_dtype, x_stride, B, D, whole_steps(D), q, whole_steps(D), scales, s);
    if (psc_status st = launched_op(what)) return st;
    a.x = q;
    a.x_stride = whole_steps(D);
    a.x_scales = scales;
    a.w = w;
    a.w_stride = w_stride;
    a.w_scales = w_scales;
    a.bias = bias;
    a.bitmask = bitmask;
    a.y = logits;
    a.y_stride = stride;
    a.B = B;
    a.D = D;
    a.V = V;
    a.W = (int32_t)(((int64_t)V + 31) / 32);
    a.steps = whole_steps(D) / kStep;
    const bool bf16 = dtype == PSC_BF16;
    if (B <= 16) launch_head<16, 64, 1, 2, 4>(a, bf16, s);
    else if (B <= 64) launch_head<64, 128, 2, 2, 3>(a, bf16, s);
    else launch_head<256, 256, 2, 4, 2>(a, bf16, s);
    return launched_op(what);
}
