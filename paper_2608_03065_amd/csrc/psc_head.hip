// The output projection in 8-bit integers (psc_quantize_rows, psc_head_logits):
// rows of int8 with one scale each on both sides, products summed exactly in
// 32-bit integers by the matrix cores, and one epilogue that scales, adds the
// bias, applies the grammar mask and rounds once.
//
// A call launches prepare_kernel (the states to 8 bits and, under a mask, the
// list of tokens that any row allows), then the product: small_kernel for up to
// 128 rows, and for more where the large tiles would be too few (takes_wide),
// wide_kernel for the others.  Where the mask leaves few tokens, the product is
// taken of the listed tokens' weights only (small_kernel, `gather`; beside
// wide_kernel in a launch of its own).  Where there are too few tiles for the GPU, D
// is split over workgroups; the last one of a tile to end adds their sums, which
// are integers: any order gives the same.
//
// Few rows are bound by the weights' bytes, each read once: 64 x 151,665 x 2,048
// takes 73 us, 4.5 TB/s, where a large copy reaches 4.8.  Many rows are bound by
// the matrix cores: 2,048 x 128,256 x 4,096 takes 900 to 935 us, 2.3 to 2.4 P
// integer operations a second.  Calls that need few tokens' weights (8 rows, 160
// tokens: 11 us) are bound by their chain of waits: the list, the weights, the
// parts' sums.
#include "psc_head.hpp"

using namespace psc;

namespace {

// ---------------------------------------------------------------- rows to int8

// x[d] = scale * q[d]: scale = max |x| / 127 and q = rint(x / scale) (ties to
// even), both divisions in float32.  A row of zeros has scale 0; a row with an
// infinity or a NaN has scale NaN and q 0, so that every product with it is NaN.
// Weights of 128,256 x 4,096 take 453 us from float32 (2.6 GB, 5.8 TB/s), and 432
// from bfloat16, of 1.6 GB: there a row's chain is the bound, loads, maximum,
// barrier and the divisions, which are the same in number.
constexpr int kQuantBlock = kPrepareBlock;
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

// The row by one workgroup; q[D .. padded) become zeros.
template <bool kBf16>
__device__ __forceinline__ void quantize_row(const void *__restrict__ x, int64_t x_stride, int64_t r, int32_t D, int32_t padded,
                                             int8_t *__restrict__ q, int64_t q_stride, float *__restrict__ scales,
                                             uint32_t *s_most) {
    const char *row = static_cast<const char *>(x) + r * x_stride * (kBf16 ? 2 : 4);
    uint32_t most = 0;            // of the absolute values' bits: a NaN's are above an infinity's
    // a row of up to kHeld elements is read once
    constexpr int kTurns = 4, kHeld = kTurns * kQuantBlock * kQuantVec;
    float held[kTurns][kQuantVec], v[kQuantVec];
    const bool once = D <= kHeld;
    if (once) {
#pragma unroll
        for (int i = 0; i < kTurns; i++) load_vec<kBf16>(row, (i * kQuantBlock + (int)threadIdx.x) * kQuantVec, D, held[i]);
#pragma unroll
        for (int i = 0; i < kTurns; i++)
#pragma unroll
            for (int k = 0; k < kQuantVec; k++) most = max(most, __builtin_bit_cast(uint32_t, held[i][k]) & 0x7FFFFFFFu);
    } else {
        for (int32_t d = threadIdx.x * kQuantVec; d < D; d += kQuantBlock * kQuantVec) {
            load_vec<kBf16>(row, d, D, v);
#pragma unroll
            for (int k = 0; k < kQuantVec; k++) most = max(most, __builtin_bit_cast(uint32_t, v[k]) & 0x7FFFFFFFu);
        }
    }
    most = wave_all(most, 0u, kMax);
    if (threadIdx.x % kWave == 0) s_most[threadIdx.x / kWave] = most;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kQuantBlock / kWave; k++) most = max(most, s_most[k]);
    const bool finite = most < 0x7F800000u;
    const float scale = finite ? __builtin_bit_cast(float, most) / 127.0f : __builtin_nanf("");
    if (threadIdx.x == 0) scales[r] = scale;
    int8_t *to = q + r * q_stride;
    const auto put = [&](int32_t d, const float(&f8)[kQuantVec]) {
        uint64_t out = 0;
#pragma unroll
        for (int k = 0; k < kQuantVec; k++) {
            // past D the element is 0; a scale too small for its row's maximum (a subnormal one) is clamped
            const float f = scale > 0 ? __builtin_rintf(f8[k] / scale) : 0.0f;
            out |= (uint64_t)(uint8_t)(int8_t)(int)fminf(fmaxf(f, -127.0f), 127.0f) << (8 * k);
        }
        __builtin_memcpy(to + d, &out, sizeof out);
    };
    if (once) {
#pragma unroll
        for (int i = 0; i < kTurns; i++) {
            const int32_t d = (i * kQuantBlock + (int)threadIdx.x) * kQuantVec;
            if (d < padded) put(d, held[i]);
        }
    } else {
        for (int32_t d = threadIdx.x * kQuantVec; d < padded; d += kQuantBlock * kQuantVec) {
            load_vec<kBf16>(row, d, D, v);
            put(d, v);
        }
    }
}

template <bool kBf16>
__global__ void __launch_bounds__(kQuantBlock)
quantize_kernel(const void *__restrict__ x, int64_t x_stride, int32_t D, int32_t padded, int8_t *__restrict__ q,
                int64_t q_stride, float *__restrict__ scales) {
    __shared__ uint32_t s_most[kQuantBlock / kWave];
    quantize_row<kBf16>(x, x_stride, blockIdx.x, D, padded, q, q_stride, scales, s_most);
}

// ---------------------------------------------------------------- the product's arguments, and what is prepared for it

struct HeadArgs : HeadBase {
    const int8_t *x;              // quantised states, rows x_stride apart, zeros from D up to whole steps
    int64_t x_stride;
    const float *x_scales;
    const int8_t *w;
    int64_t w_stride;
    const float *w_scales;
};

// Workgroups 0 .. rows - 1: a row of states each; the others a block of needed
// tokens each; all of them clear the arrival counters.
template <bool kBf16>
__global__ void __launch_bounds__(kQuantBlock)
prepare_kernel(const HeadArgs a, int32_t rows, const void *__restrict__ x, int64_t x_stride, int8_t *__restrict__ q,
               float *__restrict__ scales, int32_t *__restrict__ counts, int32_t *__restrict__ ids) {
    __shared__ uint32_t shared[kQuantBlock / kWave][kBlockWords];
    for (int64_t i = (int64_t)blockIdx.x * kQuantBlock + threadIdx.x; i < a.arrivals_most; i += (int64_t)gridDim.x * kQuantBlock)
        a.arrivals[i] = 0;
    if ((int32_t)blockIdx.x < rows) quantize_row<kBf16>(x, x_stride, blockIdx.x, a.D, (int32_t)a.x_stride, q, a.x_stride, scales, shared[0]);
    else needed_block(a, (int32_t)blockIdx.x - rows, counts, ids, shared);
}

// |sum| <= 127 * 128 * D stays below 2^31 for every row but one of -128 alone, which is at 2^31 with weights of -128.
constexpr int32_t kMostD = 131072;

// The same of states that are in 8 bits already: rows `first` .. are copied, zeros behind them.  A row of kMostD times
// -128 becomes one of -64 with twice its scale, the same numbers, whose sums fit 32 bits.
__global__ void __launch_bounds__(kQuantBlock)
copy_kernel(const HeadArgs a, int32_t first, int32_t rows, const int8_t *__restrict__ x, int64_t x_stride, const float *__restrict__ x_scales,
            int8_t *__restrict__ q, float *__restrict__ scales, int32_t *__restrict__ counts, int32_t *__restrict__ ids) {
    __shared__ uint32_t shared[kQuantBlock / kWave][kBlockWords];
    if (first == 0)
        for (int64_t i = (int64_t)blockIdx.x * kQuantBlock + threadIdx.x; i < a.arrivals_most; i += (int64_t)gridDim.x * kQuantBlock) a.arrivals[i] = 0;
    if ((int32_t)blockIdx.x >= rows) {
        needed_block(a, (int32_t)blockIdx.x - rows, counts, ids, shared);
        return;
    }
    const int64_t r = (int64_t)first + blockIdx.x;
    bool halves = false;
    if (a.D == kMostD) {
        uint32_t off = 0;
        for (int32_t d = threadIdx.x * kChunk; d < kMostD; d += kQuantBlock * kChunk) {
            uint32_t t[4];
            __builtin_memcpy(t, x + r * x_stride + d, sizeof t);
#pragma unroll
            for (int k = 0; k < 4; k++) off |= t[k] ^ 0x80808080u;
        }
        halves = !__syncthreads_or(off != 0);
    }
    for (int32_t d = threadIdx.x * kChunk; d < (int32_t)a.x_stride; d += kQuantBlock * kChunk) {
        uint32_t t[4] = {};
        if (d < a.D) __builtin_memcpy(t, x + r * x_stride + d, sizeof t);
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int32_t left = a.D - d - 4 * k;
            if (left < 4) t[k] &= left > 0 ? ~(~0u << (8 * left)) : 0u;
            if (halves) t[k] = 0xC0C0C0C0u;
        }
        __builtin_memcpy(q + r * a.x_stride + d, t, sizeof t);
    }
    if (threadIdx.x == 0) {
        const float scale = x_scales[r], twice = 2 * scale;
        // a scale whose double passes float32 makes every sum but 0 infinite as it is
        scales[r] = halves && __builtin_isfinite(twice) ? twice : scale;
    }
}

// ---------------------------------------------------------------- results

// sum * xs * ws + bias: the sum and its product with xs rounded to float32, the
// product with ws and the bias as one operation with one rounding.  Named, so
// that every kernel rounds alike.
__device__ __forceinline__ float scaled(int32_t sum, float xs, float ws, float bias) { return __builtin_fmaf((float)sum * xs, ws, bias); }

// Four consecutive logits of a row from token v on, a multiple of 4; bit e of
// `allowed` is token v + e's.
template <bool kBf16>
__device__ __forceinline__ void put_four(const HeadArgs &a, int32_t b, int32_t v, const i32x4 &sum, float xs, const float (&ws)[4],
                                         const float (&bias)[4], uint32_t allowed) {
    using T = typename Logit<kBf16>::type;
    T out[4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const float y = (allowed >> e) & 1 ? scaled(sum[e], xs, ws[e], bias[e]) : kMinusInf;
        if constexpr (kBf16) out[e] = to_bf16(y);
        else out[e] = y;
    }
    T *to = static_cast<T *>(a.y) + (int64_t)b * a.y_stride + v;
    if (v + 4 <= a.V) __builtin_memcpy(to, out, sizeof out);
    else
        for (int e = 0; e < 4; e++)
            if (v + e < a.V) to[e] = out[e];
}

// What kTn by kTm blocks of 16 tokens by 16 states need besides their sums.
// The lane's tokens of block i are v + 16 i .. + 3, its state of block j is
// m0 + b + 16 j.  All of it is loaded at once, by small_kernel before the
// product, without a branch: places outside, a bias or a mask that there is not
// give zeros.  kPlain: neither a bias nor a mask.
template <int kTn, int kTm, bool kPlain>
struct Factors {
    float ws[kTn][4], bias[kTn][4], xs[kTm];
    uint32_t words[kTn][kTm];

    __device__ __forceinline__ void load(const HeadArgs &a, int32_t v, int32_t m0, int32_t b) {
        const uint32_t tokens = (uint32_t)a.V * 4u;
        const __amdgpu_buffer_rsrc_t from_ws = buffer_of(a.w_scales, tokens), from_bias = buffer_of(a.bias, a.bias ? tokens : 0);
        const __amdgpu_buffer_rsrc_t from_xs = buffer_of(a.x_scales + m0, (uint32_t)min(a.B - m0, kMostRows) * 4u);
        const __amdgpu_buffer_rsrc_t from_mask = mask_from(a, m0);
#pragma unroll
        for (int j = 0; j < kTm; j++) xs[j] = __builtin_bit_cast(float, load_word(from_xs, b + j * 16));
#pragma unroll
        for (int i = 0; i < kTn; i++) {
#pragma unroll
            for (int e = 0; e < 4; e++) {
                ws[i][e] = __builtin_bit_cast(float, load_word(from_ws, v + i * 16 + e));
                bias[i][e] = kPlain ? 0.0f : __builtin_bit_cast(float, load_word(from_bias, v + i * 16 + e));
            }
            if (!kPlain)
#pragma unroll
                for (int j = 0; j < kTm; j++) words[i][j] = load_word(from_mask, (b + j * 16) * a.W + ((v + i * 16) >> 5));
        }
    }

    template <bool kBf16>
    __device__ __forceinline__ void put(const HeadArgs &a, int32_t v, int32_t b, const i32x4 (&sum)[kTn][kTm]) const {
        const uint32_t all = kPlain || !a.bitmask ? 15u : 0u;
#pragma unroll
        for (int i = 0; i < kTn; i++)
#pragma unroll
            for (int j = 0; j < kTm; j++)
                if (v + i * 16 < a.V && b + j * 16 < a.B)
                    put_four<kBf16>(a, b + j * 16, v + i * 16, sum[i][j], xs[j], ws[i], bias[i],
                                    kPlain ? 15u : words[i][j] >> ((v + i * 16) & 31) | all);
    }
};

// ---------------------------------------------------------------- up to 128 rows

// The weights from row `row` on, up to the first multiple of 16 bytes at or
// after the last row's D elements: nothing behind that is touched.
__device__ __forceinline__ int64_t weight_bytes(const HeadArgs &a, int32_t row) {
    return (int64_t)(a.V - row - 1) * a.w_stride + (a.D + kChunk - 1) / kChunk * kChunk;
}

// One workgroup computes kM states by kN tokens over a part of D.  Steps of
// 128 bytes of all its rows go straight from memory into one of kStages buffers
// in LDS, kStages - 1 steps ahead.  A row's 16-byte chunk c lies at place c ^
// (row & 7) of its 128 bytes, so that the 16 rows that a matrix instruction
// reads at one chunk fall into different banks; since a load puts lane l's
// chunk at place l, the lane fetches the chunk that belongs there.  What is
// read past a row's D elements is multiplied by the states' zeros.
template <int kM, int kN, int kWavesM, int kWavesN, int kStages, bool kBf16, bool kPlain>
__device__ __forceinline__ void small_body(const HeadArgs &a, bool gather_only) {
    constexpr int kWaves = kWavesM * kWavesN, kRows = kM + kN;
    constexpr int kLoads = kRows * kChunks / (kWaves * kWave);
    static_assert(kLoads * kWaves * kWave == kRows * kChunks && kN % 8 == 0, "every wavefront loads as much");
    constexpr int kTm = kM / kWavesM / 16, kTn = kN / kWavesN / 16;   // 16 x 16 blocks of a wavefront
    static_assert(kTm * kWavesM * 16 == kM && kTn * kWavesN * 16 == kN, "whole blocks");
    __shared__ __align__(1024) int8_t lds[kStages][kRows * kStep];
    __shared__ int32_t s_ids[kN];
    __shared__ uint32_t s_arrived;
    // until the first loads into lds: the needed tokens before each block
    int32_t *const s_before = reinterpret_cast<int32_t *>(&lds[0][0]);
    static_assert(sizeof lds >= (kMostBlocks + 1) * sizeof(int32_t), "room for the blocks");
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave % kWavesM, wn = wave / kWavesM;

    int32_t total = 0, count[kShare];
    if (!kPlain && a.counts) {
        const int32_t upto = needed_upto(a, lane, count);
        total = lane_value(upto, kWave - 1);
        if (total <= a.gather_most && wave == 0) {
            int32_t before = upto;
#pragma unroll
            for (int i = kShare - 1; i >= 0; i--) {
                s_before[lane * kShare + i + 1] = before;
                before -= count[i];
            }
            if (lane == 0) s_before[0] = 0;
        }
    }
    Plan plan = plan_of<kM, kN>(a, total);
    if (kPlain) plan.gather = false;
    if (gather_only && !plan.gather) return;
    const bool fill = plan.gather && !gather_only;        // else wide_kernel does it
    const int32_t tiles = plan.tiles * a.m_tiles;
    if ((int32_t)blockIdx.x >= tiles * plan.splits) {
        if (fill) fill_forbidden<kBf16, 1>(a, blockIdx.x, gridDim.x);
        return;
    }
    const int32_t split = (int32_t)blockIdx.x / tiles, tile = (int32_t)blockIdx.x - split * tiles;
    const int32_t m0 = tile % a.m_tiles * kM, n0 = tile / a.m_tiles * kN;
    const int32_t first = a.steps * split / plan.splits, steps = a.steps * (split + 1) / plan.splits;

    if (plan.gather) {
        // token n0 + i of the needed ones: its block by bisection of the sums before each
        __syncthreads();
        for (int i = threadIdx.x; i < kN; i += kWaves * kWave) {
            int32_t id = -1;
            if (n0 + i < plan.columns) {
                int32_t lo = 0, hi = a.blocks;
                while (hi - lo > 1) {
                    const int32_t mid = (lo + hi) / 2;
                    if (s_before[mid] <= n0 + i) lo = mid;
                    else hi = mid;
                }
                id = a.ids[(int64_t)lo * kBlockTokens + n0 + i - s_before[lo]];
            }
            s_ids[i] = id;
        }
        __syncthreads();
    }
    const int32_t w_row = plan.gather ? 0 : n0;
    const u32x4 rw = rows_from(a.w + (int64_t)w_row * a.w_stride, weight_bytes(a, w_row));
    const u32x4 rx = rows_from(a.x + (int64_t)m0 * a.x_stride, (int64_t)(a.B - m0) * a.x_stride);
    uint32_t from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int row = (i * kWaves + wave) * 8 + lane / 8, chunk = (lane & 7) ^ (row & 7);
        uint32_t at;
        if (row >= kN) at = (uint32_t)(row - kN) * (uint32_t)a.x_stride;
        else if (!plan.gather) at = (uint32_t)row * (uint32_t)a.w_stride;
        else at = s_ids[row] >= 0 ? (uint32_t)s_ids[row] * (uint32_t)a.w_stride : kNowhere;
        from[i] = at == kNowhere ? at : at + chunk * kChunk;
    }
    const auto fetch = [&](int32_t step) {
        const uint32_t to = lds_byte(lds) + (uint32_t)(step % kStages) * (kRows * kStep);
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int row = (i * kWaves + wave) * 8;
            // past the last step nothing is read, and the number of accesses stays the same
            const uint32_t off = step < steps && from[i] != kNowhere ? from[i] + (uint32_t)step * kStep : kNowhere;
            load_to_lds(row < kN ? rw : rx, off, to + (uint32_t)row * kStep);
        }
    };
    i32x4 acc[kTn][kTm] = {};
    const int r16 = lane % 16, quad = lane / 16;
    const int32_t v0 = n0 + wn * kTn * 16 + quad * 4, b0 = m0 + wm * kTm * 16 + r16;    // the lane's first token and state
    Factors<kTn, kTm, kPlain> factors;
    if (!plan.gather && plan.splits == 1) factors.load(a, v0, m0, b0 - m0);
#pragma unroll
    for (int s = 0; s < kStages - 1; s++) fetch(first + s);
    if (fill) fill_forbidden<kBf16, 1>(a, blockIdx.x, gridDim.x);
    for (int32_t step = first; step < steps; step++) {
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
    if (plan.splits > 1) {
        // The sums go to memory at device scope, which every XCD sees alike, and
        // only when they are there does the workgroup count itself in; the
        // last one of the tile reads them all.
        constexpr uint32_t kPart = kM * kN * sizeof(int32_t);
        constexpr int kDevice = 16;        // the accesses' scope (sc1)
        const __amdgpu_buffer_rsrc_t sums = buffer_of(a.partials + (int64_t)tile * plan.splits * (kM * kN), (uint32_t)plan.splits * kPart);
        const auto place = [&](int i, int j) { return (uint32_t)(((i * kTm + j) * kWaves * kWave + (int)threadIdx.x) * 16); };
#pragma unroll
        for (int i = 0; i < kTn; i++)
#pragma unroll
            for (int j = 0; j < kTm; j++)
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[i][j]), sums, (uint32_t)split * kPart + place(i, j), 0, kDevice);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) s_arrived = __hip_atomic_fetch_add(a.arrivals + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (s_arrived != (uint32_t)plan.splits - 1) return;
        if (!plan.gather) factors.load(a, v0, m0, b0 - m0);
        constexpr int kAtOnce = 4;
        for (int32_t part = 0; part < plan.splits; part += kAtOnce) {
            u32x4 t[kAtOnce][kTn][kTm];
#pragma unroll
            for (int n = 0; n < kAtOnce; n++)
#pragma unroll
                for (int i = 0; i < kTn; i++)
#pragma unroll
                    for (int j = 0; j < kTm; j++) {
                        // its own sum it has; parts that there are not give zeros
                        const bool other = part + n < plan.splits && part + n != split;
                        t[n][i][j] = __builtin_amdgcn_raw_buffer_load_b128(sums, other ? (uint32_t)(part + n) * kPart + place(i, j) : kNowhere, 0, kDevice);
                    }
#pragma unroll
            for (int n = 0; n < kAtOnce; n++)
#pragma unroll
                for (int i = 0; i < kTn; i++)
#pragma unroll
                    for (int j = 0; j < kTm; j++) acc[i][j] += __builtin_bit_cast(i32x4, t[n][i][j]);
        }
    }
    if (!plan.gather) {
        factors.template put<kBf16>(a, v0, b0, acc);
        return;
    }
    // few of a tile's logits are allowed: first all the bits, at once, then those
    const __amdgpu_buffer_rsrc_t mask = mask_from(a, m0);
    uint32_t allowed[kTm] = {};
#pragma unroll
    for (int i = 0; i < kTn; i++) {
        uint32_t words[kTm][4];
        int32_t v[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            v[e] = s_ids[(wn * kTn + i) * 16 + quad * 4 + e];
#pragma unroll
            for (int j = 0; j < kTm; j++)
                words[j][e] = __builtin_amdgcn_raw_buffer_load_b32(mask, v[e] < 0 ? kNowhere : (uint32_t)((b0 - m0 + j * 16) * a.W + (v[e] >> 5)) * 4u, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < kTm; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) allowed[j] |= (words[j][e] >> (v[e] & 31) & 1u) << (i * 4 + e);
    }
#pragma unroll
    for (int j = 0; j < kTm; j++) {
        const int32_t b = b0 + j * 16;
        if (b >= a.B || !allowed[j]) continue;
        const float xs = a.x_scales[b];
        using T = typename Logit<kBf16>::type;
        T *const row = static_cast<T *>(a.y) + (int64_t)b * a.y_stride;
#pragma unroll
        for (int i = 0; i < kTn; i++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if (!((allowed[j] >> (i * 4 + e)) & 1)) continue;
                const int32_t v = s_ids[(wn * kTn + i) * 16 + quad * 4 + e];
                store_logit<kBf16>(row, v, scaled(acc[i][j][e], xs, a.w_scales[v], a.bias ? a.bias[v] : 0.0f));
            }
    }
}

template <int kM, int kN, int kWavesM, int kWavesN, int kStages, bool kBf16, bool kPlain>
__global__ void __launch_bounds__(kWave * kWavesM * kWavesN, 2)
small_kernel(const HeadArgs a, bool gather_only) {
    small_body<kM, kN, kWavesM, kWavesN, kStages, kBf16, kPlain>(a, gather_only);
}

// ---------------------------------------------------------------- more than 128 rows

// 256 states by kN tokens a tile, 8 wavefronts of 64 states by kN / 2 tokens, a
// workgroup per compute unit that goes through tiles until none are left, its
// loads running ahead into the next tile.
//
// The matrix cores are fed by two groups of four wavefronts, one of each per
// SIMD, half a turn apart: while one group multiplies (64 bytes of D, 32 or 40
// matrix instructions a wavefront), the other reads its next operands from LDS
// and issues loads, and a barrier ends each turn.
//
// LDS holds kRing steps of weights, which come from HBM, and two of states,
// which come from L2.  A load covers whole 128-byte lines: with 64-byte pieces
// the loads alone took 507 us of 2,048 x 128,256 x 4,096, with lines 322.
//
// XCDs take workgroups in turn; ids are dealt so that the tiles of one block of
// tokens (all blocks of states) run on one XCD and share its L2.
template <int kN, int kRing, bool kBf16, bool kPlain>
__device__ __forceinline__ void wide_body(const HeadArgs &a) {
    constexpr int kM = 256, kWavesM = 4, kWavesN = 2, kWaves = 8;
    constexpr int kLoadsW = kN * kChunks / (kWaves * kWave), kLoadsX = kM * kChunks / (kWaves * kWave);
    static_assert(kLoadsW * kWaves * kWave == kN * kChunks && kN % 64 == 0, "every wavefront loads as much");
    static_assert(kRing == 2 || kRing == 3, "only the newest weights may be outstanding");
    constexpr int kTm = kM / kWavesM / 16, kTn = kN / kWavesN / 16, kPairs = kTn / 2;
    __shared__ __align__(1024) int8_t lds_w[kRing * kN * kStep], lds_x[2 * kM * kStep];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave % kWavesM, wn = wave / kWavesM;
    if (!kPlain && a.counts) {
        int32_t count[kShare];
        if (lane_value(needed_upto(a, lane, count), kWave - 1) <= a.gather_most) {
            fill_forbidden<kBf16, 4>(a, blockIdx.x, gridDim.x);      // the product was small_kernel's
            return;
        }
    }
    const int32_t n_tiles = (a.V + kN - 1) / kN, tiles = n_tiles * a.m_tiles, whole = n_tiles / 8 * 8 * a.m_tiles;
    const auto corner = [&](int32_t id, int32_t &m0, int32_t &n0) {
        n0 = (id < whole ? id / 8 / a.m_tiles * 8 + id % 8 : id / a.m_tiles) * kN;
        m0 = (id < whole ? id / 8 % a.m_tiles : id % a.m_tiles) * kM;
    };
    const int row8 = wave * 8 + lane / 8;
    const uint32_t chunk = ((lane & 7) ^ (row8 & 7)) * kChunk;
    const uint32_t base_w = (uint32_t)row8 * (uint32_t)a.w_stride + chunk, base_x = (uint32_t)row8 * (uint32_t)a.x_stride + chunk;
    const uint32_t turn_w = kWaves * 8 * (uint32_t)a.w_stride, turn_x = kWaves * 8 * (uint32_t)a.x_stride;
    // the loads' own tile and step; past the last tile they read nothing, and their number stays the same
    int32_t id_w = blockIdx.x, id_x = blockIdx.x, step_w = 0, step_x = 0, to_w = 0, to_x = 0;
    u32x4 rw, rx;
    const auto point_w = [&]() {
        int32_t m0, n0;
        corner(id_w, m0, n0);
        rw = id_w < tiles ? rows_from(a.w + (int64_t)n0 * a.w_stride, weight_bytes(a, n0)) : rows_from(a.w, 0);
    };
    const auto point_x = [&]() {
        int32_t m0, n0;
        corner(id_x, m0, n0);
        rx = id_x < tiles ? rows_from(a.x + (int64_t)m0 * a.x_stride, (int64_t)(a.B - m0) * a.x_stride) : rows_from(a.x, 0);
    };
    const auto fetch_w = [&]() {
#pragma unroll
        for (int i = 0; i < kLoadsW; i++)
            load_to_lds(rw, base_w + i * turn_w + (uint32_t)step_w * kStep, lds_byte(lds_w) + (uint32_t)(to_w * kN + (i * kWaves + wave) * 8) * kStep);
        to_w = to_w == kRing - 1 ? 0 : to_w + 1;
        if (++step_w == a.steps) {
            step_w = 0;
            id_w += (int32_t)gridDim.x;
            point_w();
        }
    };
    const auto fetch_x = [&]() {
#pragma unroll
        for (int i = 0; i < kLoadsX; i++)
            load_to_lds(rx, base_x + i * turn_x + (uint32_t)step_x * kStep, lds_byte(lds_x) + (uint32_t)(to_x * kM + (i * kWaves + wave) * 8) * kStep);
        to_x ^= 1;
        if (++step_x == a.steps) {
            step_x = 0;
            id_x += (int32_t)gridDim.x;
            point_x();
        }
    };
    point_w();
    point_x();
    fetch_x();
    for (int i = 0; i < kRing - 1; i++) fetch_w();
    const int r16 = lane % 16, quad = lane / 16;
    // the newest step of weights, fetched after the states of its turn, need not have landed where there are three
    constexpr int kLeft = kRing == 3 ? kLoadsW : 0;
    wait_and_meet<kLeft>();
    if (wave >= kWaves / 2) asm volatile("s_barrier" ::: "memory");      // the second group, one turn later
    int32_t at_w = 0, at_x = 0;
    for (int32_t id = blockIdx.x; id < tiles; id += (int32_t)gridDim.x) {
        i32x4 acc[kTn][kTm] = {};
        for (int32_t s = 0; s < a.steps; s++) {
            const int8_t *const pw = lds_w + (at_w * kN + wn * kTn * 16 + r16) * kStep;
            const int8_t *const px = lds_x + (at_x * kM + wm * kTm * 16 + r16) * kStep;
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const int place = ((k * 4 + quad) ^ (r16 & 7)) * kChunk;
                i32x4 fw[kTn], fx[kTm];
#pragma unroll
                for (int i = 0; i < kTn; i++) fw[i] = *reinterpret_cast<const i32x4 *>(pw + i * 16 * kStep + place);
#pragma unroll
                for (int j = 0; j < kTm; j++) fx[j] = *reinterpret_cast<const i32x4 *>(px + j * 16 * kStep + place);
                // Into the buffers of the step before.  The second group read the
                // last of them in the turn that has just ended: its wait for these
                // reads and that turn's barrier are all that lies between.
                if (k == 0) {
                    fetch_x();
                    fetch_w();
                }
                __builtin_amdgcn_sched_barrier(0);
                if (k == 0) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                else wait_and_meet<kLeft>();       // this wavefront's part of the next step has landed
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int i = 0; i < kTn; i++)
#pragma unroll
                    for (int j = 0; j < kTm; j++)
                        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[i], fx[j], acc[i][j], 0, 0, 0);
                __builtin_amdgcn_s_setprio(0);
                __builtin_amdgcn_sched_barrier(0);
                asm volatile("s_barrier" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
            }
            at_w = at_w == kRing - 1 ? 0 : at_w + 1;
            at_x ^= 1;
        }
        int32_t m0, n0;
        corner(id, m0, n0);
        const int32_t v0 = n0 + wn * kTn * 16;       // the wavefront's first token
        if (m0 + kM <= a.B && n0 + kN <= a.V) {
            // Whole tiles.  A lane has four consecutive tokens of every block:
            // 16 bytes of float32.  Of bfloat16 it gets eight: of two blocks
            // of 16 tokens, lanes 16 apart swap halves.  Either way a store
            // writes 64 bytes of every state's row.
            using T = typename Logit<kBf16>::type;
            const int32_t mine = kBf16 ? (quad & 1) * 16 + (quad >> 1) * 8 : quad * 4;
            float xs[kTm];
            T *to[kTm];
            const uint32_t *words[kTm];
#pragma unroll
            for (int j = 0; j < kTm; j++) {
                const int32_t b = m0 + (wm * kTm + j) * 16 + r16;
                xs[j] = a.x_scales[b];
                to[j] = static_cast<T *>(a.y) + (int64_t)b * a.y_stride + v0 + mine;
                if (!kPlain && a.bitmask) words[j] = a.bitmask + (int64_t)b * a.W + (v0 >> 5);
            }
#pragma unroll
            for (int p = 0; p < kPairs; p++) {
                float ws[2][4], bias[2][4] = {};
                uint32_t word[kTm];
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const int32_t v = v0 + (2 * p + h) * 16 + quad * 4;
                    __builtin_memcpy(ws[h], a.w_scales + v, sizeof ws[h]);
                    if (!kPlain && a.bias) __builtin_memcpy(bias[h], a.bias + v, sizeof bias[h]);
                }
#pragma unroll
                for (int j = 0; j < kTm; j++) word[j] = !kPlain && a.bitmask ? words[j][p] >> mine : ~0u;
#pragma unroll
                for (int j = 0; j < kTm; j++) {
                    float y[2][4];
#pragma unroll
                    for (int h = 0; h < 2; h++)
#pragma unroll
                        for (int e = 0; e < 4; e++) y[h][e] = scaled(acc[2 * p + h][j][e], xs[j], ws[h][e], bias[h][e]);
                    if constexpr (kBf16) {
                        uint32_t o[2][2];
#pragma unroll
                        for (int h = 0; h < 2; h++)
#pragma unroll
                            for (int e = 0; e < 2; e++)
                                o[h][e] = (uint32_t)to_bf16(y[h][2 * e]) | (uint32_t)to_bf16(y[h][2 * e + 1]) << 16;
                        const auto s0 = __builtin_amdgcn_permlane16_swap(o[0][0], o[1][0], false, false);
                        const auto s1 = __builtin_amdgcn_permlane16_swap(o[0][1], o[1][1], false, false);
                        u32x4 t = {(uint32_t)s0[0], (uint32_t)s1[0], (uint32_t)s0[1], (uint32_t)s1[1]};
                        if (!kPlain)
#pragma unroll
                            for (int e = 0; e < 4; e++) {
                                const uint32_t lo = (uint32_t)((int32_t)(word[j] << (31 - 2 * e)) >> 31);
                                const uint32_t hi = (uint32_t)((int32_t)(word[j] << (30 - 2 * e)) >> 31);
                                const uint32_t keep = (lo & 0xFFFFu) | (hi & 0xFFFF0000u);
                                t[e] = (t[e] & keep) | (0xFF80FF80u & ~keep);
                            }
                        __builtin_memcpy(to[j] + p * 32, &t, sizeof t);
                    } else {
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            if (!kPlain)
#pragma unroll
                                for (int e = 0; e < 4; e++) y[h][e] = (word[j] >> (h * 16 + e)) & 1 ? y[h][e] : kMinusInf;
                            __builtin_memcpy(to[j] + p * 32 + h * 16, y[h], sizeof y[h]);
                        }
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kTn; i++) {
                const int32_t v = v0 + i * 16 + quad * 4, b = m0 + wm * kTm * 16 + r16;
                Factors<1, kTm, kPlain> factors;
                factors.load(a, v, m0, b - m0);
                factors.template put<kBf16>(a, v, b, reinterpret_cast<const i32x4 (&)[1][kTm]>(acc[i]));
            }
            // no load of this branch is left for the compiler to wait for after the other, where a wait is one for all stores
            __builtin_amdgcn_s_waitcnt(0x0F70);     // vmcnt(0)
        }
    }
    if (wave < kWaves / 2) asm volatile("s_barrier" ::: "memory");
}

// kPlain: neither a mask nor a bias.
template <int kN, int kRing, bool kBf16, bool kPlain>
__global__ void __launch_bounds__(kWave * 8, 2)
wide_kernel(const HeadArgs a) {
    wide_body<kN, kRing, kBf16, kPlain>(a);
}

// ---------------------------------------------------------------- host side

constexpr int32_t kWideRows = 128;

// Rows to 8 bits, a workgroup each, in as many launches as that takes.
void launch_quantize(const void *x, psc_dtype dtype, int64_t x_stride, int64_t n_rows, int32_t D, int32_t padded, int8_t *q,
                     int64_t q_stride, float *scales, hipStream_t s) {
    for (int64_t r = 0; r < n_rows; r += kMostGrid) {
        const dim3 grid((uint32_t)std::min(kMostGrid, n_rows - r)), block(kQuantBlock);
        const void *from = static_cast<const char *>(x) + r * x_stride * size_of(dtype);
        const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, from, x_stride, D, padded, q + r * q_stride, q_stride, scales + r); };
        if (dtype == PSC_BF16) go(quantize_kernel<true>);
        else go(quantize_kernel<false>);
    }
}

// prepare_kernel with the rows that fit beside the blocks, then the others alone.
void launch_prepare(const HeadArgs &a, const void *x, psc_dtype dtype, int64_t x_stride, int8_t *q, float *scales, int32_t *counts,
                    int32_t *ids, hipStream_t s) {
    const int32_t rows = (int32_t)std::min<int64_t>(a.B, kMostGrid - a.blocks);
    const dim3 grid((uint32_t)(rows + a.blocks)), block(kQuantBlock);
    if (dtype == PSC_BF16) hipLaunchKernelGGL(prepare_kernel<true>, grid, block, 0, s, a, rows, x, x_stride, q, scales, counts, ids);
    else hipLaunchKernelGGL(prepare_kernel<false>, grid, block, 0, s, a, rows, x, x_stride, q, scales, counts, ids);
    launch_quantize(static_cast<const char *>(x) + rows * x_stride * size_of(dtype), dtype, x_stride, a.B - rows, a.D, (int32_t)a.x_stride,
                    q + rows * a.x_stride, a.x_stride, scales + rows, s);
}

// copy_kernel with the rows that fit beside the blocks, then the others alone.
void launch_copy(const HeadArgs &all, const int8_t *x, int64_t x_stride, const float *x_scales, int8_t *q, float *scales, int32_t *counts,
                 int32_t *ids, hipStream_t s) {
    HeadArgs a = all;
    for (int32_t first = 0; first < all.B; a.blocks = 0) {
        const int32_t rows = (int32_t)std::min<int64_t>(all.B - first, kMostGrid - a.blocks);
        hipLaunchKernelGGL(copy_kernel, dim3((uint32_t)(rows + a.blocks)), dim3(kQuantBlock), 0, s, a, first, rows, x, x_stride, x_scales, q, scales,
                           counts, ids);
        first += rows;
    }
}

template <int kM, int kN, int kWavesM, int kWavesN, int kStages>
void launch_small(HeadArgs a, bool bf16, bool gather_only, hipStream_t s) {
    shape_small<kM, kN>(a, gather_only);
    const dim3 grid((uint32_t)a.units), block(kWave * kWavesM * kWavesN);
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a, gather_only); };
    if (a.bitmask || a.bias) {
        if (bf16) go(small_kernel<kM, kN, kWavesM, kWavesN, kStages, true, false>);
        else go(small_kernel<kM, kN, kWavesM, kWavesN, kStages, false, false>);
    } else {
        if (bf16) go(small_kernel<kM, kN, kWavesM, kWavesN, kStages, true, true>);
        else go(small_kernel<kM, kN, kWavesM, kWavesN, kStages, false, true>);
    }
}

template <int kN, int kRing>
void launch_wide(HeadArgs a, bool bf16, hipStream_t s) {
    a.m_tiles = up(a.B, 256);
    const dim3 grid((uint32_t)std::min<int64_t>(kComputeUnits, (int64_t)a.m_tiles * up(a.V, kN))), block(kWave * 8);
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
    if (a.bitmask || a.bias) {
        if (bf16) go(wide_kernel<kN, kRing, true, false>);
        else go(wide_kernel<kN, kRing, false, false>);
    } else {
        if (bf16) go(wide_kernel<kN, kRing, true, true>);
        else go(wide_kernel<kN, kRing, false, true>);
    }
}

// wide_kernel's calls: above kWideRows rows, unless its tiles would leave most
// compute units idle.  us by wide_kernel and by small_kernel: 160 x 128,256 x
// 4,096 169 and 193, 256 x 40,000 x 4,096 (157 tiles) 69 and 82, 1,194 x 7,168 x
// 640 (140 tiles of five steps) 32 and 28.
bool takes_wide(const HeadArgs &a) {
    return a.B > kWideRows && (int64_t)up(a.B, 256) * up(a.V, 256) >= kComputeUnits / 2;
}

// Of the two widths of wide_kernel the one that ends first: rounds of tiles
// over the compute units times a tile's width.  256 states x 151,936 tokens x
// 4,096: 3 rounds of 256 take 221 us, 2 of 320 201; 2,048 x 128,256: 16 of 256
// 922, 13 of 320 936.
//
// The tiles of small_kernel grow with the rows.  us by tiles of 32 x 64, 64 x 128 and 128
// x 128, times 128,256 x 4,096: 32 rows 111, 124, 128; 33 rows 169, 124, 128; 64 rows 174,
// 129, 133; 65 rows 221, 153, 134; 128 rows 349, 167, 146.  Above 64 rows on small
// vocabularies the middle ones are ahead: 128 x 32,000 x 2,048 43, 28, 32.
//
// Beside wide_kernel the needed tokens' launch is made before it is known whether
// they are few.  Where they are not, it takes 4.5 us, and the list and it together 12
// of the 222 of 256 x 151,936 x 4,096.
void launch_product(const HeadArgs &a, bool bf16, hipStream_t s) {
    if (a.B <= 32) return launch_small<32, 64, 1, 4, 4>(a, bf16, false, s);
    if (a.B <= 64) return launch_small<64, 128, 1, 4, 3>(a, bf16, false, s);
    if (!takes_wide(a)) return launch_small<128, 128, 2, 4, 3>(a, bf16, false, s);
    if (a.counts) launch_small<64, 128, 1, 4, 3>(a, bf16, true, s);
    const int64_t rounds256 = up((int64_t)up(a.B, 256) * up(a.V, 256), kComputeUnits),
                  rounds320 = up((int64_t)up(a.B, 256) * up(a.V, 320), kComputeUnits);
    if (rounds320 * 320 < rounds256 * 256) launch_wide<320, 2>(a, bf16, s);
    else launch_wide<256, 3>(a, bf16, s);
}

int32_t whole_steps(int32_t D) { return up(D, kStep) * kStep; }

// The workspace: quantised states [B][whole_steps(D)], their scales, the needed
// tokens, the arrival counters, the partial sums; each from a multiple of 16
// bytes on.
struct Workspace {
    size_t scales, counts, ids, arrivals, partials, total;
    int32_t partials_most;
    Workspace(int32_t B, int32_t D, int32_t V) {
        const auto whole = [](size_t n) { return (n + 15) / 16 * 16; };
        const int64_t blocks = up(V, kBlockTokens);
        scales = (size_t)B * (size_t)whole_steps(D);
        counts = scales + whole((size_t)B * sizeof(float));
        ids = counts + whole(blocks <= kMostBlocks ? blocks * sizeof(int32_t) : 0);
        arrivals = ids + (blocks <= kMostBlocks ? blocks * kBlockTokens * sizeof(int32_t) : 0);
        partials = arrivals + kMostArrivals * sizeof(uint32_t);
        // twice the compute units' number of the largest tiles
        partials_most = (int32_t)std::min<int64_t>((int64_t)kMostArrivals * 128 * 128, (int64_t)16 * up(B, 16) * 16 * (up(V, 128) * 128));
        total = partials + (size_t)partials_most * sizeof(int32_t);
    }
};

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
    if (D > INT32_MAX - 8 * kQuantBlock * kQuantVec) return refuse(what, "D too large");
    if (x_stride < 0 || !aligned_to(x, size_of(dtype))) return refuse(what, "negative stride, or x off its elements' alignment");
    if (q_stride % kChunk || q_stride < padded || !aligned_to(q, kChunk))
        return refuse(what, "rows of q start at 16 bytes and hold D elements");
    launch_quantize(x, dtype, x_stride, n_rows, D, (int32_t)padded, q, q_stride, scales, reinterpret_cast<hipStream_t>(stream));
    return launched_op(what);
}

extern "C" size_t psc_head_workspace(int32_t B, int32_t D, int32_t V) {
    return B <= 0 || D <= 0 || D > kMostD || V <= 0 || V > kMostV ? 0 : Workspace(B, D, V).total;
}

namespace {

// What the caller gives as states: numbers of `dtype`, or where `scales` is not null 8-bit integers.
struct States {
    const void *x;
    psc_dtype dtype;
    int64_t stride;
    const float *scales;
};

psc_status head_logits(const char *what, const States &x, int32_t B, int32_t D, const int8_t *w, int64_t w_stride, const float *w_scales,
                       int32_t V, const float *bias, const uint32_t *bitmask, void *logits, psc_dtype dtype, int64_t stride,
                       void *workspace, size_t workspace_bytes, void *stream) {
    if (D < 1 || D > kMostD) return refuse(what, "D outside [1, 131072]");
    if (V > kMostV) return refuse(what, "V > 2^26");
    if (B == 0 || V == 0) return PSC_OK;
    if ((int64_t)up(B, 64) * up(V, 512) > kMostGrid) return refuse(what, "ceil(B / 64) * ceil(V / 512) >= 2^24");
    if (!x.x || !w || !w_scales || !workspace) return refuse(what, "null pointer");
    if (x.scales) {
        if (x.stride % kChunk || x.stride < D || !aligned_to(x.x, kChunk) || !aligned_to(x.scales, 4))
            return refuse(what, "rows of q start at 16 bytes and hold D elements");
    } else if (x.stride < 0 || !aligned_to(x.x, size_of(x.dtype))) return refuse(what, "negative stride, or x off its elements' alignment");
    if (w_stride % kChunk || w_stride < D || w_stride > INT32_MAX / 512 || !aligned_to(w, kChunk))
        return refuse(what, "rows of w start at 16 bytes and hold D elements");
    if (workspace_bytes < psc_head_workspace(B, D, V) || !aligned_to(workspace, kChunk))
        return refuse(what, "the workspace is too small or not 16-byte aligned");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const Workspace ws(B, D, V);
    char *at = static_cast<char *>(workspace);
    HeadArgs a{};
    a.x = reinterpret_cast<int8_t *>(at);
    a.x_stride = whole_steps(D);
    a.x_scales = reinterpret_cast<float *>(at + ws.scales);
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
    a.W = up(V, 32);
    a.steps = whole_steps(D) / kStep;
    a.partials = reinterpret_cast<int32_t *>(at + ws.partials);
    a.partials_most = ws.partials_most;
    a.arrivals = reinterpret_cast<uint32_t *>(at + ws.arrivals);
    a.arrivals_most = kMostArrivals;
    // The needed tokens are listed where offsets of all weights fit 32 bits.
    int32_t *counts = nullptr, *ids = nullptr;
    if (bitmask && up(V, kBlockTokens) <= kMostBlocks && (int64_t)V * w_stride < kMostBytes) {
        a.blocks = up(V, kBlockTokens);
        a.counts = counts = reinterpret_cast<int32_t *>(at + ws.counts);
        a.ids = ids = reinterpret_cast<int32_t *>(at + ws.ids);
        // Half of them; a quarter where wide_kernel, which is closer to the compute units' rate, takes all.  us with
        // the needed ones only and with all: 8 x 128,256 x 4,096 74 and 108 where half are needed, 83 and 107 at 0.6; 64 x
        // 151,665 x 2,048 69 and 78 at a half, 77 and 78 at 0.6, 86 and 78 at 0.8; by wide_kernel 256 x 151,936 x 4,096 146
        // and 220 at 0.2, 195 and 216 at 0.3, 240 and 216 at 0.4; 512 x 128,256 x 2,048 109 and 182 at 0.1, 176 and 173 at 0.2.
        a.gather_most = takes_wide(a) ? V / 4 : V / 2;
    }
    int8_t *const q = reinterpret_cast<int8_t *>(at);
    float *const scales = reinterpret_cast<float *>(at + ws.scales);
    if (x.scales) launch_copy(a, static_cast<const int8_t *>(x.x), x.stride, x.scales, q, scales, counts, ids, s);
    else launch_prepare(a, x.x, x.dtype, x.stride, q, scales, counts, ids, s);
    // the product would go by whatever the workspace holds
    if (psc_status st = launched_op(what)) return st;
    launch_product(a, dtype == PSC_BF16, s);
    return launched_op(what);
}

}  // namespace

extern "C" psc_status psc_head_logits(const void *x, psc_dtype x_dtype, int64_t x_stride, int32_t B, int32_t D,
                                      const int8_t *w, int64_t w_stride, const float *w_scales, int32_t V,
                                      const float *bias, const uint32_t *bitmask, void *logits, psc_dtype dtype,
                                      int64_t stride, void *workspace, size_t workspace_bytes, void *stream) {
    const char *what = "psc_head_logits";
    if (psc_status st = check_rows(what, logits, dtype, stride, B, V)) return st;
    if (!is_dtype(x_dtype)) return refuse(what, "bad dtype of x");
    return head_logits(what, {x, x_dtype, x_stride, nullptr}, B, D, w, w_stride, w_scales, V, bias, bitmask, logits, dtype, stride, workspace,
                       workspace_bytes, stream);
}

extern "C" psc_status psc_head_logits_quantized(const int8_t *q, int64_t q_stride, const float *scales, int32_t B, int32_t D,
                                         const int8_t *w, int64_t w_stride, const float *w_scales, int32_t V,
                                         const float *bias, const uint32_t *bitmask, void *logits, psc_dtype dtype,
                                         int64_t stride, void *workspace, size_t workspace_bytes, void *stream) {
    const char *what = "psc_head_logits_quantized";
    if (psc_status st = check_rows(what, logits, dtype, stride, B, V)) return st;
    if (!scales && B > 0 && V > 0) return refuse(what, "null pointer");
    return head_logits(what, {q, PSC_F32, q_stride, scales}, B, D, w, w_stride, w_scales, V, bias, bitmask, logits, dtype, stride, workspace,
                       workspace_bytes, stream);
}
