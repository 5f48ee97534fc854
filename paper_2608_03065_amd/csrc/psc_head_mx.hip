// The output projection by microscaled 4-bit weights (psc_head_logits_mx):
// states in 4 bits too, or in bfloat16.
//
// The matrix instruction of 4-bit operands takes 128 elements of a row, a lane
// 32 of them: a block, 16 bytes of codes, with the block's power of two.  For
// bfloat16 states the same 16 bytes are converted to bfloat16 times their power,
// which holds them exactly, and go through four matrix instructions of 32
// elements each, of which a lane has 8.  Products are exact, sums float32.  (The
// same instruction takes states in 8-bit floating point, whose sums it cuts off
// near 2^-13 of the largest product: no form of states here.)
//
// A call launches prepare_mx_kernel (the states to what is multiplied, and under a
// mask the list of tokens that any row allows) unless the states can be read
// where they are, there is no mask, and D is not split; then the product:
// small_mx_kernel for up to 128 rows and where the large tiles would be few
// (takes_wide), wide_mx_kernel for the others.  Where the mask leaves few tokens,
// the product is taken of the listed tokens' weights only (small_mx_kernel,
// `gather`; beside wide_mx_kernel in a launch of its own).  Where there are too few
// tiles for the GPU, D is split over workgroups, and the last one of a tile to end
// adds their sums in the order of the parts: the same call gives the same bits.
//
// Few rows are bound by the weights' bytes, each read once: 1 x 128,256 x 4,096
// takes 50 us, 5.6 TB/s, where a large copy reaches 4.7; 64 x 128,256 x 4,096 66 us of
// states in 4 bits, 4.5 TB/s, but 118 of bfloat16, whose lines are three times the
// weights' bytes on their way from L2 to LDS.  Many rows, by box and by what ran
// before: 2,048 x 128,256 x 4,096 takes 577 to 648 us in 4 bits, 3.3 to 3.7 P
// operations a second (the library's product of that size without scales' variety, a
// mask or a bias 820), 256 x 151,936 x 4,096 of bfloat16 271 to 307.  Their matrix
// instructions alone would take 228 and 160; the rest is about equally the waits for
// what is read from LDS, for the lines from L2, and the stores of the logits, which
// all compute units write at once.
#include <type_traits>

#include "psc_head.hpp"
#include "psc_mx.hpp"

using namespace psc;

namespace {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kStepElems = kStep * 2;              // a line of codes
constexpr int kStepScales = kStepElems / kMxBlock; // and its scales, in bytes
constexpr int kPairScales = 2 * kStepScales;       // those of two lines are loaded at once
constexpr int kScaleRows = 256;                    // the states' are held in tiles of so many rows: [tiles][pairs of lines][rows][16]
constexpr int kWideStep = kStepElems * 2;          // the same elements in bfloat16
constexpr uint32_t kOne = 127;                     // the scale of 1

struct MxArgs : HeadBase {
    const void *x;                // states: codes or bfloat16, zeros from D up to whole steps
    int64_t x_stride;             // in bytes
    const uint8_t *x_scales;      // of codes, whole pairs of steps, in tiles
    const uint8_t *w;
    int64_t w_stride;
    const uint8_t *w_scales;
    int64_t w_scales_stride;
    int32_t w_blocks;             // scales of a row
};

// ---------------------------------------------------------------- prepare

// The byte of a state's scale.
__host__ __device__ __forceinline__ int64_t scale_at(int32_t steps, int64_t row, int32_t block) {
    const int64_t pairs = (steps + 1) / 2;
    return ((row / kScaleRows * pairs + block / kPairScales) * kScaleRows + row % kScaleRows) * kPairScales + block % kPairScales;
}

// Workgroups 0 .. rows - 1: a row of states each, to codes, or to bfloat16, or
// copied codes; the others a block of needed tokens each; all of them clear
// the arrival counters.
enum class From { kF32, kBf16, kMx };

template <From kFrom, bool kMx>
__device__ __forceinline__ void prepare_row(const MxArgs &a, int64_t r, const void *__restrict__ x, int64_t x_stride,
                                            const uint8_t *__restrict__ x_scales, int64_t x_scales_stride, uint8_t *__restrict__ q,
                                            uint8_t *__restrict__ scales) {
    const int32_t padded = a.steps * kStepElems, blocks = (a.D + kMxBlock - 1) / kMxBlock;
    uint8_t *const to = q + r * a.x_stride;
    const auto put_scale = [&](int32_t block, uint32_t scale) { scales[scale_at(a.steps, r, block)] = (uint8_t)scale; };
    for (int32_t d = threadIdx.x * kVec; d < padded; d += kPrepareBlock * kVec) {
        if constexpr (kFrom == From::kMx) {
            const uint8_t *const from = static_cast<const uint8_t *>(x) + r * x_stride;
            uint32_t codes = 0;
            if (d < a.D) __builtin_memcpy(&codes, from + d / 2, 4);
            if (d + kVec > a.D) codes &= d < a.D ? ~(~0u << (4 * (a.D - d))) : 0u;
            __builtin_memcpy(to + d / 2, &codes, 4);
            if (threadIdx.x % 4 == 0) put_scale(d / kMxBlock, d / kMxBlock < blocks ? x_scales[r * x_scales_stride + d / kMxBlock] : 0);
        } else {
            float v[kVec];
            load_eight<kFrom == From::kBf16>(static_cast<const char *>(x) + r * x_stride * (kFrom == From::kBf16 ? 2 : 4), d, a.D, v);
            if constexpr (kMx) {
                uint32_t scale;
                const uint32_t codes = to_mx4(v, scale);
                __builtin_memcpy(to + d / 2, &codes, 4);
                if (threadIdx.x % 4 == 0) put_scale(d / kMxBlock, scale);
            } else {
                store_eight<true>(to, d, padded, v);
            }
        }
    }
}

template <From kFrom, bool kMx>
__global__ void __launch_bounds__(kPrepareBlock)
prepare_mx_kernel(const MxArgs a, int32_t first, int32_t rows, const void *__restrict__ x, int64_t x_stride, const uint8_t *__restrict__ x_scales,
                  int64_t x_scales_stride, uint8_t *__restrict__ q, uint8_t *__restrict__ scales, int32_t *__restrict__ counts,
                  int32_t *__restrict__ ids) {
    __shared__ uint32_t shared[kPrepareBlock / kWave][kBlockWords];
    if (first == 0)
        for (int64_t i = (int64_t)blockIdx.x * kPrepareBlock + threadIdx.x; i < a.arrivals_most; i += (int64_t)gridDim.x * kPrepareBlock) a.arrivals[i] = 0;
    if ((int32_t)blockIdx.x < rows) prepare_row<kFrom, kMx>(a, (int64_t)first + blockIdx.x, x, x_stride, x_scales, x_scales_stride, q, scales);
    else if ((int32_t)blockIdx.x - rows < a.blocks) needed_block(a, (int32_t)blockIdx.x - rows, counts, ids, shared);
}

// ---------------------------------------------------------------- results

// Four consecutive logits of a row from token v on, a multiple of 4; bit e of
// `allowed` is token v + e's.
template <bool kBf16>
__device__ __forceinline__ void put_four(const HeadBase &a, int32_t b, int32_t v, const f32x4 &sum, const float (&bias)[4], uint32_t allowed) {
    using T = typename Logit<kBf16>::type;
    T out[4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const float y = (allowed >> e) & 1 ? sum[e] + bias[e] : kMinusInf;
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
// The lane's tokens of block i are v + 16 i .. + 3, its state of block j is m0 +
// b + 16 j.  Places outside, a bias or a mask that there is not give zeros.
template <int kTn, int kTm, bool kPlain>
struct Extras {
    float bias[kTn][4];
    uint32_t words[kTn][kTm];

    __device__ __forceinline__ void load(const HeadBase &a, int32_t v, int32_t m0, int32_t b) {
        if (kPlain) return;
        const __amdgpu_buffer_rsrc_t from_bias = buffer_of(a.bias, a.bias ? (uint32_t)a.V * 4u : 0), from_mask = mask_from(a, m0);
#pragma unroll
        for (int i = 0; i < kTn; i++) {
#pragma unroll
            for (int e = 0; e < 4; e++) bias[i][e] = __builtin_bit_cast(float, load_word(from_bias, v + i * 16 + e));
#pragma unroll
            for (int j = 0; j < kTm; j++) words[i][j] = load_word(from_mask, (b + j * 16) * a.W + ((v + i * 16) >> 5));
        }
    }

    template <bool kBf16>
    __device__ __forceinline__ void put(const HeadBase &a, int32_t v, int32_t b, const f32x4 (&sum)[kTn][kTm]) const {
        const uint32_t all = kPlain || !a.bitmask ? 15u : 0u;
        const float none[4] = {};
#pragma unroll
        for (int i = 0; i < kTn; i++)
#pragma unroll
            for (int j = 0; j < kTm; j++)
                if (v + i * 16 < a.V && b + j * 16 < a.B)
                    put_four<kBf16>(a, b + j * 16, v + i * 16, sum[i][j], kPlain ? none : bias[i],
                                    kPlain ? 15u : words[i][j] >> ((v + i * 16) & 31) | all);
    }
};

// ---------------------------------------------------------------- products

// Of the scales, byte kByte.
template <int kByte>
__device__ __forceinline__ f32x4 product(const u32x4 &w, uint32_t w_scale, const u32x4 &x, uint32_t x_scale, const f32x4 &sum) {
    const i32x8 a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0}, b = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, sum, 4, 4, kByte, (int)w_scale, kByte, (int)x_scale);
}

__device__ __forceinline__ f32x4 product(const bf16x8 &w, const bf16x8 &x, const f32x4 &sum) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, sum, 0, 0, 0);
}

__device__ __forceinline__ bf16x8 widened(uint32_t codes, float power) {
    uint32_t pairs[4];
    from_mx4(codes, power, pairs);
    return __builtin_bit_cast(bf16x8, pairs);
}

// The weights' rows from `row` on, up to the end of the last one's last block,
// and their scales: nothing behind that is touched but what shares 4 bytes with it.
__device__ __forceinline__ int64_t code_bytes(const MxArgs &a, int32_t row) {
    return (int64_t)(a.V - row - 1) * a.w_stride + (int64_t)a.w_blocks * (kMxBlock / 2);
}
__device__ __forceinline__ int64_t scale_bytes(const MxArgs &a, int32_t row) {
    return (int64_t)(a.V - row - 1) * a.w_scales_stride + (a.w_blocks + 3) / 4 * 4;
}

// A row's codes past D in its last block, in LDS, to zeros: its scale could make them infinite in bfloat16, and these
// no zeros of the states' take out.  `line` holds the row's last step.
__device__ __forceinline__ void clear_behind(const MxArgs &a, uint8_t *line, int row) {
    const int block = a.w_blocks - 1 - (a.steps - 1) * kStepScales, n = a.D % kMxBlock;
    uint32_t *const at = reinterpret_cast<uint32_t *>(line + ((block ^ (row & 7)) * kChunk));
    for (int e = n / kVec; e < kMxBlock / kVec; e++) at[e] &= ~(~0u << (4 * max(n - e * kVec, 0)));
}

// One workgroup computes kM states by kN tokens over a part of D.  Steps of 256
// elements of all its rows go straight from memory into one of kStages buffers
// in LDS, kStages - 1 steps ahead: a line of codes of every token, and of every
// state the same or four lines of bfloat16; with every second step, 16 bytes of
// scales of each row of codes, those of both.  A
// row's 16-byte chunk c lies at place c ^ (row & 7) of its line, and of a state in
// bfloat16 at c ^ (row & 15), so that the 16 rows that a matrix instruction reads
// at one chunk fall into different banks; since a load puts lane l's chunk at
// place l, the lane fetches the chunk that belongs there.  Blocks past a row's D
// elements are multiplied by the states' zeros, and by a scale of 1.
template <int kM, int kN, int kWavesM, int kWavesN, int kStages, bool kMx, bool kBf16, bool kPlain>
__device__ __forceinline__ void small_mx_body(const MxArgs &a, bool gather_only) {
    constexpr int kWaves = kWavesM * kWavesN, kXStep = kMx ? kStep : kWideStep;
    constexpr int kTm = kM / kWavesM / 16, kTn = kN / kWavesN / 16;   // 16 x 16 blocks of a wavefront
    static_assert(kTm * kWavesM * 16 == kM && kTn * kWavesN * 16 == kN, "whole blocks");
    // loads of a step: of the codes, the states, the scales of the tokens and those of the states
    constexpr int kLoadsW = kN * kStep / 1024 / kWaves;
    static_assert(kLoadsW * kWaves * 1024 == kN * kStep, "every wavefront loads as much");
    constexpr int kX1024 = kM * kXStep / 1024, kLoadsX = (kX1024 + kWaves - 1) / kWaves;
    constexpr int kRowsS = kN + (kMx ? kM : 0), kS1024 = (kRowsS + kWave - 1) / kWave, kLoadsS = (kS1024 + kWaves - 1) / kWaves;
    static_assert(kN % kWave == 0, "a load has the scales of tokens, or of states");
    constexpr int kLoads = kLoadsW + kLoadsX;
    static_assert(kStages == 3 || kStages == 4, "what is waited for");
    static_assert(2 * kLoads + kLoadsS < 64, "the counter's range");
    constexpr int kAtX = kN * kStep, kStage = kAtX + kX1024 * 1024;
    constexpr int kGroups = kStages == 3 ? 2 : 3, kAtS = kStages * kStage;       // pairs of steps whose scales are held
    constexpr int kRest = kAtS + kGroups * kS1024 * 1024;                       // where loads of nothing go
    __shared__ __align__(1024) uint8_t lds[kRest + 1024];
    __shared__ int32_t s_ids[kN];
    __shared__ uint32_t s_arrived;
    // until the first loads into lds: the needed tokens before each block
    int32_t *const s_before = reinterpret_cast<int32_t *>(lds);
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
    const bool fill = plan.gather && !gather_only;        // else the wide kernel does it
    const int32_t tiles = plan.tiles * a.m_tiles;
    if ((int32_t)blockIdx.x >= tiles * plan.splits) {
        if (fill) fill_forbidden<kBf16, 1>(a, blockIdx.x, gridDim.x);
        return;
    }
    const int32_t split = (int32_t)blockIdx.x / tiles, tile = (int32_t)blockIdx.x - split * tiles;
    const int32_t m0 = tile % a.m_tiles * kM, n0 = tile / a.m_tiles * kN;
    const int32_t pairs = (a.steps + 1) / 2;          // a part is whole pairs of steps
    const int32_t first = pairs * split / plan.splits * 2, steps = min(a.steps, pairs * (split + 1) / plan.splits * 2);

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
    const u32x4 rw = rows_from(a.w + (int64_t)w_row * a.w_stride, code_bytes(a, w_row));
    const u32x4 rs = rows_from(a.w_scales + (int64_t)w_row * a.w_scales_stride, scale_bytes(a, w_row));
    const u32x4 rx = rows_from(static_cast<const char *>(a.x) + (int64_t)m0 * a.x_stride, (int64_t)(a.B - m0 - 1) * a.x_stride + (int64_t)a.steps * kXStep);
    // from the tile's first pair on, its rows from m0 on
    const u32x4 rt = kMx ? rows_from(a.x_scales + scale_at(a.steps, m0, 0), (int64_t)pairs * kScaleRows * kPairScales - m0 % kScaleRows * kPairScales) : rs;
    // offsets of the lane's loads; past the last step, and for rows that there are not, they read nothing
    uint32_t from_w[kLoadsW], from_x[kLoadsX], from_s[kLoadsS];
    const auto token = [&](int row, int64_t stride) {
        if (!plan.gather) return (uint32_t)row * (uint32_t)stride;
        return s_ids[row] >= 0 ? (uint32_t)s_ids[row] * (uint32_t)stride : kNowhere;
    };
#pragma unroll
    for (int i = 0; i < kLoadsW; i++) {
        const int row = (i * kWaves + wave) * 8 + lane / 8;
        const uint32_t at = token(row, a.w_stride);
        from_w[i] = at == kNowhere ? at : at + (((lane & 7) ^ (row & 7)) * kChunk);
    }
#pragma unroll
    for (int i = 0; i < kLoadsX; i++) {
        constexpr int kLanes = kXStep / kChunk;       // that take a row
        const int row = (i * kWaves + wave) * (kWave / kLanes) + lane / kLanes, c = lane % kLanes;
        from_x[i] = row < kM && m0 + row < a.B ? (uint32_t)row * (uint32_t)a.x_stride + (uint32_t)((kMx ? c ^ (row & 7) : c ^ (row & 15)) * kChunk) : kNowhere;
    }
#pragma unroll
    for (int i = 0; i < kLoadsS; i++) {
        const int row = (i * kWaves + wave) * kWave + lane;
        if (row < kN) from_s[i] = token(row, a.w_scales_stride);
        else from_s[i] = row < kRowsS ? (uint32_t)(row - kN) * kPairScales : kNowhere;
    }
    const auto fetch = [&](int32_t step, bool even) {
        const uint32_t base = lds_byte(lds), to = base + (uint32_t)(step % kStages) * kStage;
        const auto off = [&](uint32_t from, uint32_t bytes) { return step < steps && from != kNowhere ? from + bytes : kNowhere; };
        if (even)
#pragma unroll
            for (int i = 0; i < kLoadsS; i++) {
                const int n = i * kWaves + wave;
                const bool states = n * kWave >= kN;
                load_to_lds(states ? rt : rs, off(from_s[i], (uint32_t)(step / 2) * (states ? kScaleRows * kPairScales : kPairScales)),
                            n < kS1024 ? base + kAtS + (uint32_t)(step / 2 % kGroups * kS1024 + n) * 1024u : base + kRest);
            }
#pragma unroll
        for (int i = 0; i < kLoadsW; i++) load_to_lds(rw, off(from_w[i], (uint32_t)step * kStep), to + (uint32_t)(i * kWaves + wave) * 1024u);
#pragma unroll
        for (int i = 0; i < kLoadsX; i++) {
            const int n = i * kWaves + wave;
            load_to_lds(rx, off(from_x[i], (uint32_t)step * kXStep), n < kX1024 ? to + kAtX + (uint32_t)n * 1024u : base + kRest);
        }
    };
    f32x4 acc[kTn][kTm] = {};
    const int r16 = lane % 16, quad = lane / 16;
    const int32_t v0 = n0 + wn * kTn * 16 + quad * 4, b0 = m0 + wm * kTm * 16 + r16;    // the lane's first token and state
    Extras<kTn, kTm, kPlain> extras;
    if (!plan.gather && plan.splits == 1) extras.load(a, v0, m0, b0 - m0);
#pragma unroll
    for (int s = 0; s < kStages - 1; s++) fetch(first + s, s % 2 == 0);
    if (fill) fill_forbidden<kBf16, 1>(a, blockIdx.x, gridDim.x);
    const auto turn = [&](int32_t step, bool even) {
        const uint8_t *const at = lds + step % kStages * kStage, *const scales = lds + kAtS + step / 2 % kGroups * kS1024 * 1024 + (even ? 0 : kStepScales);
        const int left = a.w_blocks - step * kStepScales - quad;       // of the lane's first block: blocks up to the row's end
#pragma unroll
        for (int k = 0; k < kStepElems / 128; k++) {
            u32x4 fw[kTn];
            uint32_t sw[kTn];
#pragma unroll
            for (int i = 0; i < kTn; i++) {
                const int row = (wn * kTn + i) * 16 + r16;
                fw[i] = *reinterpret_cast<const u32x4 *>(at + row * kStep + (((k * 4 + quad) ^ (row & 7)) * kChunk));
                const uint32_t word = *reinterpret_cast<const uint32_t *>(scales + row * kPairScales + k * 4);
                sw[i] = left > k * 4 ? (word >> (8 * quad)) & 255u : kOne;
            }
            if constexpr (kMx) {
                u32x4 fx[kTm];
                uint32_t sx[kTm];
#pragma unroll
                for (int j = 0; j < kTm; j++) {
                    const int row = (wm * kTm + j) * 16 + r16;
                    fx[j] = *reinterpret_cast<const u32x4 *>(at + kAtX + row * kStep + (((k * 4 + quad) ^ (row & 7)) * kChunk));
                    sx[j] = *reinterpret_cast<const uint32_t *>(scales + (kN + row) * kPairScales + k * 4) >> (8 * quad);
                }
#pragma unroll
                for (int i = 0; i < kTn; i++)
#pragma unroll
                    for (int j = 0; j < kTm; j++) acc[i][j] = product<0>(fw[i], sw[i], fx[j], sx[j], acc[i][j]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    bf16x8 fx[kTm];
#pragma unroll
                    for (int j = 0; j < kTm; j++) {
                        const int row = (wm * kTm + j) * 16 + r16;
                        fx[j] = *reinterpret_cast<const bf16x8 *>(at + kAtX + row * kWideStep + (((k * 16 + quad * 4 + e) ^ (row & 15)) * kChunk));
                    }
#pragma unroll
                    for (int i = 0; i < kTn; i++) {
                        const bf16x8 w = widened(fw[i][e], mx_power(sw[i]));
#pragma unroll
                        for (int j = 0; j < kTm; j++) acc[i][j] = product(w, fx[j], acc[i][j]);
                    }
                }
            }
        }
    };
    const auto settle = [&](int32_t step) {
        if (kMx || a.D % kMxBlock == 0 || step + 1 != a.steps) return;
        for (int row = threadIdx.x; row < kN; row += kWaves * kWave) clear_behind(a, lds + step % kStages * kStage + row * kStep, row);
        wait_and_meet<63>();
    };
    // of the loads after the step's own: kStages - 2 steps of them, of which scales come with the even ones
    for (int32_t step = first; step < steps; step += 2) {
        wait_and_meet<(kStages - 2) * kLoads + (kStages == 4 ? kLoadsS : 0)>();   // the step has landed, and its predecessor's buffer is free
        fetch(step + kStages - 1, kStages == 3);
        settle(step);
        turn(step, true);
        if (step + 1 == steps) break;
        wait_and_meet<(kStages - 2) * kLoads + kLoadsS>();
        fetch(step + kStages, kStages == 4);
        settle(step + 1);
        turn(step + 1, false);
    }
    if (plan.splits > 1) {
        // The sums go to memory at device scope, which every XCD sees alike, and
        // only when they are there does the workgroup count itself in; the
        // last one of the tile adds them all, in the order of the parts.
        constexpr uint32_t kPart = kM * kN * sizeof(float);
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
        if (!plan.gather) extras.load(a, v0, m0, b0 - m0);
#pragma unroll
        for (int i = 0; i < kTn; i++)
#pragma unroll
            for (int j = 0; j < kTm; j++) acc[i][j] = f32x4{};
        constexpr int kAtOnce = 4;
        for (int32_t part = 0; part < plan.splits; part += kAtOnce) {
            u32x4 t[kAtOnce][kTn][kTm];
#pragma unroll
            for (int n = 0; n < kAtOnce; n++)
#pragma unroll
                for (int i = 0; i < kTn; i++)
#pragma unroll
                    for (int j = 0; j < kTm; j++)      // parts that there are not give zeros
                        t[n][i][j] = __builtin_amdgcn_raw_buffer_load_b128(sums, part + n < plan.splits ? (uint32_t)(part + n) * kPart + place(i, j) : kNowhere, 0, kDevice);
#pragma unroll
            for (int n = 0; n < kAtOnce; n++)
#pragma unroll
                for (int i = 0; i < kTn; i++)
#pragma unroll
                    for (int j = 0; j < kTm; j++) acc[i][j] += __builtin_bit_cast(f32x4, t[n][i][j]);
        }
    }
    if (!plan.gather) {
        extras.template put<kBf16>(a, v0, b0, acc);
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
        using T = typename Logit<kBf16>::type;
        T *const row = static_cast<T *>(a.y) + (int64_t)b * a.y_stride;
#pragma unroll
        for (int i = 0; i < kTn; i++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if (!((allowed[j] >> (i * 4 + e)) & 1)) continue;
                const int32_t v = s_ids[(wn * kTn + i) * 16 + quad * 4 + e];
                store_logit<kBf16>(row, v, acc[i][j][e] + (a.bias ? a.bias[v] : 0.0f));
            }
    }
}

template <int kM, int kN, int kWavesM, int kWavesN, int kStages, bool kMx, bool kBf16, bool kPlain>
__global__ void __launch_bounds__(kWave * kWavesM * kWavesN)
small_mx_kernel(const MxArgs a, bool gather_only) {
    small_mx_body<kM, kN, kWavesM, kWavesN, kStages, kMx, kBf16, kPlain>(a, gather_only);
}

// ---------------------------------------------------------------- many rows

// 256 states by kN tokens a tile, 8 wavefronts of 64 states by kN / 2 tokens, two
// on each SIMD, a workgroup per compute unit that goes through tiles until none
// are left, its loads running ahead into the next tile.  Two, because matrix
// instructions of one alone come 24 cycles apart, of two 16.
//
// LDS holds two lines of every state, two of every token's codes, and their
// scales.  A line of codes is 256 elements: one line of a state in 4 bits, four
// of one in bfloat16.  A line of states is multiplied in two halves.  While one
// is, the operands of the next are read, weights into the place of those that
// have been multiplied; between the two, when the line has been read by all
// wavefronts, the line after the next is fetched into its place.
//
// Of 4-bit states lane quad q takes block 2 q + k of the line's eight in half k, so
// that its scales of both halves are two bytes in a row, of which the matrix
// instruction picks one.  Of bfloat16 a half is 32 elements, one block of each
// token: a lane has 8 of the block's codes, 4 bytes, and converts them beside the
// matrix instructions, which leave the time.
//
// XCDs take workgroups in turn; ids are dealt so that the tiles of one block of
// tokens (all blocks of states) run on one XCD and share its L2.
template <int kN, bool kMx, bool kBf16, bool kPlain>
__device__ __forceinline__ void wide_mx_body(const MxArgs &a) {
    constexpr int kM = 256, kWavesM = 4, kWavesN = 2, kWaves = 8;
    constexpr int kSubs = kMx ? 1 : 4;                 // lines of a state per line of codes
    constexpr int kLoadsW = kN * kChunks / (kWaves * kWave), kLoadsX = kM * kChunks / (kWaves * kWave);
    static_assert(kLoadsW * kWaves * kWave == kN * kChunks && kN % 64 == 0, "every wavefront loads as much");
    constexpr int kRowsS = kN + (kMx ? kM : 0), kS1024 = kRowsS / kWave;
    static_assert(kS1024 <= kWaves && kN % kWave == 0, "a load has the scales of tokens, or of states");
    constexpr int kTm = kM / kWavesM / 16, kTn = kN / kWavesN / 16, kPairs = kTn / 2;
    static_assert(kTn % 2 == 0 && kTm < kTn && kLoadsX + kLoadsW <= kTn, "the reads and loads that go with a block's products");
    constexpr int kScales = kRowsS * kPairScales;
    static_assert(kM == kScaleRows, "a tile of states is one of scales");
    constexpr int kStores = kBf16 ? kPairs * kTm : kTn * kTm;      // of a whole tile
    __shared__ __align__(1024) uint8_t lds_w[2 * kN * kStep], lds_x[2 * kM * kStep], lds_s[2 * kScales];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave % kWavesM, wn = wave / kWavesM;
    if (!kPlain && a.counts) {
        int32_t count[kShare];
        if (lane_value(needed_upto(a, lane, count), kWave - 1) <= a.gather_most) {
            fill_forbidden<kBf16, 4>(a, blockIdx.x, gridDim.x);      // the product was the small kernel's
            return;
        }
    }
    const int32_t n_tiles = (a.V + kN - 1) / kN, tiles = n_tiles * a.m_tiles, whole = n_tiles / 8 * 8 * a.m_tiles;
    const auto corner = [&](int32_t id, int32_t &m0, int32_t &n0) {
        n0 = (id < whole ? id / 8 / a.m_tiles * 8 + id % 8 : id / a.m_tiles) * kN;
        m0 = (id < whole ? id / 8 % a.m_tiles : id % a.m_tiles) * kM;
    };
    // What is loaded next of the codes and of the states.  Past the last tile nothing is read, and the number of loads
    // stays the same.
    const uint32_t turn_w = kWaves * 8 * (uint32_t)a.w_stride, turn_x = kWaves * 8 * (uint32_t)a.x_stride;
    const int32_t x_lines = a.steps * kSubs;
    int32_t id_w = blockIdx.x, id_x = blockIdx.x, step_w = 0, line_x = 0, to_w = 0, to_x = 0, to_s = 0;
    u32x4 rw, rs, rx, rt;
    const auto point_w = [&]() {
        int32_t m0 = 0, n0 = 0;
        const bool some = id_w < tiles;
        if (some) corner(id_w, m0, n0);
        rw = rows_from(a.w + (int64_t)n0 * a.w_stride, some ? code_bytes(a, n0) : 0);
        rs = rows_from(a.w_scales + (int64_t)n0 * a.w_scales_stride, some ? scale_bytes(a, n0) : 0);
        if (kMx) rt = rows_from(a.x_scales + scale_at(a.steps, m0, 0), some ? (int64_t)((a.steps + 1) / 2) * kScaleRows * kPairScales : 0);
    };
    const auto point_x = [&]() {
        int32_t m0 = 0, n0 = 0;
        const bool some = id_x < tiles;
        if (some) corner(id_x, m0, n0);
        rx = rows_from(static_cast<const char *>(a.x) + (int64_t)m0 * a.x_stride, some ? (int64_t)(a.B - m0 - 1) * a.x_stride + (int64_t)x_lines * kStep : 0);
    };
    // a sum of scalars that the compiler keeps as one, in place of sums per lane that outlive the loop
    const auto uniform = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };
    // The lane, anew: what is worked out of it then is not kept in registers beside the sums, which would not fit.
    const auto this_lane = [&]() {
        int32_t l = threadIdx.x % kWave;
        asm volatile("" : "+v"(l));
        return l;
    };
    // of the lane's row and chunk in a load of eight rows
    const auto base = [&](int64_t stride) {
        const int l = this_lane(), row8 = wave * 8 + l / 8;
        return (uint32_t)row8 * (uint32_t)stride + ((l & 7) ^ (row8 & 7)) * kChunk;
    };
    // with every second line of codes the scales of both: 64 rows a load, tokens first, then states
    const auto fetch_s = [&]() {
        if (step_w % 2) return;
        const uint32_t pair = (uint32_t)step_w / 2;
        const uint32_t row = (uint32_t)(wave * kWave + this_lane()), to = lds_byte(lds_s) + (uint32_t)(to_s * kScales + wave * 1024);
        if (kMx && wave * kWave >= kN) load_to_lds(rt, row * kPairScales + uniform((pair * kScaleRows - kN) * kPairScales), to);
        else if (wave < kS1024) load_to_lds(rs, row * (uint32_t)a.w_scales_stride + uniform(pair * kPairScales), to);
        to_s ^= 1;
    };
    // Load i of a line; `base` is the lane's place in the first one.
    const auto fetch_w = [&](uint32_t base, int i) {
        load_to_lds(rw, base + uniform(i * turn_w + (uint32_t)step_w * kStep), lds_byte(lds_w) + (uint32_t)(to_w * kN + (i * kWaves + wave) * 8) * kStep);
    };
    const auto fetch_x = [&](uint32_t base, int i) {
        load_to_lds(rx, base + uniform(i * turn_x + (uint32_t)line_x * kStep), lds_byte(lds_x) + (uint32_t)(to_x * kM + (i * kWaves + wave) * 8) * kStep);
    };
    const auto fetched_w = [&]() {
        to_w ^= 1;
        if (++step_w == a.steps) {
            step_w = 0;
            id_w += (int32_t)gridDim.x;
            point_w();
        }
    };
    const auto fetched_x = [&]() {
        to_x ^= 1;
        if (++line_x == x_lines) {
            line_x = 0;
            id_x += (int32_t)gridDim.x;
            point_x();
        }
    };
    // What is read next: half k of line `sub` of the states' of step `step_r`.
    int32_t step_r = 0, sub_r = 0, at_w = 0, at_x = 0, at_s = 0;
    u32x4 fx[2][kTm], fw[2][kMx ? kTn : 1];
    uint32_t codes[2][kMx ? 1 : kTn], sw[kTn], sx[2][kMx ? kTm : 1];
    const uint8_t *px, *pw, *ps;
    const auto look = [&](int k) {
        const int l = this_lane(), r16 = l % 16, quad = l / 16;
        const int place = ((kMx ? quad * 2 + k : k * 4 + quad) ^ (r16 & 7)) * kChunk;
        px = lds_x + (at_x * kM + wm * kTm * 16 + r16) * kStep + place;
        pw = lds_w + (at_w * kN + wn * kTn * 16 + r16) * kStep + (kMx ? place : ((sub_r * 2 + k) ^ (r16 & 7)) * kChunk + quad * 4);
    };
    const auto read_w = [&](int k, int i) {
        if constexpr (kMx) fw[k][i] = *reinterpret_cast<const u32x4 *>(pw + i * 16 * kStep);
        else codes[k][i] = *reinterpret_cast<const uint32_t *>(pw + i * 16 * kStep);
    };
    const auto read_x = [&](int k, int j) { fx[k][j] = *reinterpret_cast<const u32x4 *>(px + j * 16 * kStep); };
    // the scales of both halves of a line
    const auto look_s = [&]() {
        const int l = this_lane(), r16 = l % 16, quad = l / 16;
        ps = lds_s + at_s * kScales + (wn * kTn * 16 + r16) * kPairScales + step_r % 2 * kStepScales + (kMx ? quad * 2 : sub_r * 2);
    };
    const auto read_s = [&](int i) { sw[i] = *reinterpret_cast<const uint16_t *>(ps + i * 16 * kPairScales); };
    const auto read_t = [&]() {
        if constexpr (kMx)
#pragma unroll
            for (int j = 0; j < kTm; j++) sx[1][j] = *reinterpret_cast<const uint16_t *>(ps + (kN + (wm * kTm - wn * kTn + j) * 16) * kPairScales);
    };
    // A block past the row's end counts with a power of 2^-127, whatever its scale: it is multiplied by zeros.  For
    // 4-bit states the bytes that count of the lane's two; for bfloat16 the bits of each half's power.
    uint32_t inside[2];
    const auto look_inside = [&]() {
        const int left = a.w_blocks - step_r * kStepScales;       // blocks up to the row's end
        if constexpr (kMx) {
            inside[1] = 0xFFFFu;
            if (left < kStepScales) {
                const int first = this_lane() / 16 * 2;
                inside[1] = (first < left ? 0xFFu : 0u) | (first + 1 < left ? 0xFF00u : 0u);
            }
        } else {
            inside[0] = sub_r * 2 < left ? 0x7F800000u : 0u;
            inside[1] = sub_r * 2 + 1 < left ? 0x7F800000u : 0u;
        }
    };
    const auto renew = [&]() {
        if constexpr (kMx) {
#pragma unroll
            for (int j = 0; j < kTm; j++) sx[0][j] = sx[1][j];
#pragma unroll
            for (int i = 0; i < kTn; i++) sw[i] &= inside[1];
        }
    };
    f32x4 acc[kTn][kTm] = {};
    bf16x8 w[2];
    const auto convert = [&](int k, int i) {
        if constexpr (!kMx) {
            const uint32_t power = (k ? sw[i] << 15 : sw[i] << 23) & inside[k];
            w[i % 2] = widened(codes[k][i], __builtin_bit_cast(float, power));
        }
    };
    // Half k, a block of 16 tokens after the other, the next one's weights converted meanwhile; with each of them,
    // what `with` does with its number.  The products are pinned to their place: the compiler would take them along
    // over the branches that follow.
    const auto multiply = [&](auto half, auto &&with) {
        constexpr int k = decltype(half)::value;
#pragma unroll
        for (int i = 0; i < kTn; i++) {
            with(i);
#pragma unroll
            for (int j = 0; j < kTm; j++) {
                if constexpr (kMx) acc[i][j] = product<k>(fw[k][i], sw[i], fx[k][j], sx[0][j], acc[i][j]);
                else acc[i][j] = product(w[i % 2], __builtin_bit_cast(bf16x8, fx[k][j]), acc[i][j]);
            }
            if (i + 1 < kTn) convert(k, i + 1);
#pragma unroll
            for (int j = 0; j < kTm; j++) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
#pragma unroll
            for (int j = 0; j < kTm; j++) asm volatile("" : "+v"(acc[i][j]));
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    constexpr std::integral_constant<int, 0> kFirst;
    constexpr std::integral_constant<int, 1> kSecond;
    point_w();
    point_x();
#pragma unroll
    for (int n = 0; n < 2; n++) {
        if (kMx || n == 0) {
            fetch_s();
#pragma unroll
            for (int i = 0; i < kLoadsW; i++) fetch_w(base(a.w_stride), i);
            fetched_w();
        }
#pragma unroll
        for (int i = 0; i < kLoadsX; i++) fetch_x(base(a.x_stride), i);
        fetched_x();
    }
    wait_and_meet<0>();
    const bool ragged = !kMx && a.D % kMxBlock != 0;
    const auto settle = [&](int buffer) {
        if ((int)threadIdx.x < kN) clear_behind(a, lds_w + (buffer * kN + (int)threadIdx.x) * kStep, threadIdx.x);
    };
    if (ragged && a.steps == 1) {
        settle(0);
        wait_and_meet<0>();
    }
    look(0);
    look_s();
    look_inside();
#pragma unroll
    for (int i = 0; i < kTn; i++) {
        read_w(0, i);
        read_s(i);
    }
#pragma unroll
    for (int j = 0; j < kTm; j++) read_x(0, j);
    read_t();
    renew();
    convert(0, 0);
    bool stored = false;       // stores of a whole tile were the last accesses
    for (int32_t id = blockIdx.x; id < tiles; id += (int32_t)gridDim.x) {
#pragma clang loop unroll(disable)
        for (int32_t line = 0; line < x_lines; line++) {
            multiply(kFirst, [&](int i) {
                // read before the last blocks, so that nothing is waited for at the barrier
                if (i == 0) look(1);
                if (i < kTm) read_x(1, i);
                if (i < kTn / 2) {
                    read_w(1, 2 * i);
                    read_w(1, 2 * i + 1);
                }
            });
            convert(1, 0);
            // The next line has landed: all but what was issued after it, the stores of the tile before, or codes.
            // And this one has been read by all.
            if (line == 0 && stored) wait_and_meet<(kStores < 63 ? kStores : 63)>();
            else if (!kMx && sub_r == 1) wait_and_meet<kLoadsW>();
            else wait_and_meet<0>();
            // The next line of codes, which is first read after the next barrier.
            if (ragged && sub_r == 2 && (step_r + 1 == a.steps ? 1 : step_r + 2) == a.steps) settle(at_w ^ 1);
            __builtin_amdgcn_sched_barrier(0);
            const bool codes_too = kMx || sub_r == 0;
            const uint32_t base_x = base(a.x_stride), base_w = base(a.w_stride);
            multiply(kSecond, [&](int i) {
                if (i == 0) {
                    if (codes_too) fetch_s();
                    at_x ^= 1;
                    if (kSubs > 1) sub_r = (sub_r + 1) % kSubs;
                    if (sub_r == 0) {
                        at_w ^= 1;
                        if (++step_r == a.steps) step_r = 0;
                        if (step_r % 2 == 0) at_s ^= 1;
                    }
                    look(0);
                    look_s();
                }
                if (i < kLoadsX) fetch_x(base_x, i);
                if (i >= kLoadsX && i < kLoadsX + kLoadsW && codes_too) fetch_w(base_w, i - kLoadsX);
                if (i > 0) {
                    read_s(i - 1);
                    if (i <= kTm) read_x(0, i - 1);
                    if (i <= kTn / 2) {
                        read_w(0, 2 * i - 2);
                        read_w(0, 2 * i - 1);
                    }
                }
                if (i == kTm) read_t();
            });
            read_s(kTn - 1);
            fetched_x();
            if (codes_too) fetched_w();
            look_inside();
            renew();
            convert(0, 0);
        }
        int32_t m0, n0;
        corner(id, m0, n0);
        const int32_t v0 = n0 + wn * kTn * 16;       // the wavefront's first token
        const int l = this_lane(), r16 = l % 16, quad = l / 16;
        stored = m0 + kM <= a.B && n0 + kN <= a.V;
        if (stored) {
            // Whole tiles.  A lane has four consecutive tokens of every block:
            // 16 bytes of float32.  Of bfloat16 it gets eight: of two blocks
            // of 16 tokens, lanes 16 apart swap halves.  Either way a store
            // writes 64 bytes of every state's row.
            using T = typename Logit<kBf16>::type;
            const int32_t mine = kBf16 ? (quad & 1) * 16 + (quad >> 1) * 8 : quad * 4;
            T *to[kTm];
            const uint32_t *words[kTm];
#pragma unroll
            for (int j = 0; j < kTm; j++) {
                const int32_t b = m0 + (wm * kTm + j) * 16 + r16;
                to[j] = static_cast<T *>(a.y) + (int64_t)b * a.y_stride + v0 + mine;
                if (!kPlain && a.bitmask) words[j] = a.bitmask + (int64_t)b * a.W + (v0 >> 5);
            }
#pragma unroll
            for (int p = 0; p < kPairs; p++) {
                float bias[2][4] = {};
                uint32_t word[kTm];
                if (!kPlain && a.bias)
#pragma unroll
                    for (int h = 0; h < 2; h++) __builtin_memcpy(bias[h], a.bias + v0 + (2 * p + h) * 16 + quad * 4, sizeof bias[h]);
#pragma unroll
                for (int j = 0; j < kTm; j++) word[j] = !kPlain && a.bitmask ? words[j][p] >> mine : ~0u;
#pragma unroll
                for (int j = 0; j < kTm; j++) {
                    float y[2][4];
#pragma unroll
                    for (int h = 0; h < 2; h++)
#pragma unroll
                        for (int e = 0; e < 4; e++) y[h][e] = kPlain ? acc[2 * p + h][j][e] : acc[2 * p + h][j][e] + bias[h][e];
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
                Extras<1, kTm, kPlain> extras;
                extras.load(a, v, m0, b - m0);
                extras.template put<kBf16>(a, v, b, reinterpret_cast<const f32x4 (&)[1][kTm]>(acc[i]));
            }
            // no load of this branch is left for the compiler to wait for after the other, where a wait is one for all stores
            __builtin_amdgcn_s_waitcnt(0x0F70);     // vmcnt(0)
        }
#pragma unroll
        for (int i = 0; i < kTn; i++)
#pragma unroll
            for (int j = 0; j < kTm; j++) acc[i][j] = f32x4{};
    }
}

// kPlain: neither a mask nor a bias.
template <int kN, bool kMx, bool kBf16, bool kPlain>
__global__ void __launch_bounds__(kWave * 8, 2)
wide_mx_kernel(const MxArgs a) {
    wide_mx_body<kN, kMx, kBf16, kPlain>(a);
}

// ---------------------------------------------------------------- host side

template <int kM, int kN, int kWavesM, int kWavesN, int kStages, bool kMx>
struct Small {
    static void shape(MxArgs &a, bool gather_only) { shape_small<kM, kN>(a, gather_only); }
    static void launch(const MxArgs &a, bool bf16, bool gather_only, hipStream_t s) {
        const dim3 grid((uint32_t)a.units), block(kWave * kWavesM * kWavesN);
        const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a, gather_only); };
        if (a.bitmask || a.bias) {
            if (bf16) go(small_mx_kernel<kM, kN, kWavesM, kWavesN, kStages, kMx, true, false>);
            else go(small_mx_kernel<kM, kN, kWavesM, kWavesN, kStages, kMx, false, false>);
        } else {
            if (bf16) go(small_mx_kernel<kM, kN, kWavesM, kWavesN, kStages, kMx, true, true>);
            else go(small_mx_kernel<kM, kN, kWavesM, kWavesN, kStages, kMx, false, true>);
        }
    }
};

template <int kN, bool kMx>
void launch_wide(MxArgs a, bool bf16, hipStream_t s) {
    a.m_tiles = up(a.B, 256);
    const dim3 grid((uint32_t)std::min<int64_t>(kComputeUnits, (int64_t)a.m_tiles * up(a.V, kN))), block(kWave * 8);
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
    if (a.bitmask || a.bias) {
        if (bf16) go(wide_mx_kernel<kN, kMx, true, false>);
        else go(wide_mx_kernel<kN, kMx, false, false>);
    } else {
        if (bf16) go(wide_mx_kernel<kN, kMx, true, true>);
        else go(wide_mx_kernel<kN, kMx, false, true>);
    }
}

// wide_mx_kernel's calls: above 128 rows, unless its tiles would leave most compute units idle.  us by wide_mx_kernel and by
// small_mx_kernel, times 128,256 x 4,096: states in 4 bits 96 rows 83 and 86, 128 89 and 88, 160 91 and 151; bfloat16 96
// rows 213 and 212, 128 225 and 223, 160 229 and 317.  256 x 40,000 x 4,096 (157 tiles) 44 and 62, 111 and 138;
// 256 x 24,000 (94 tiles) 39 and 41, 106 and 83.
bool takes_wide(const MxArgs &a) {
    return a.B > 128 && (int64_t)up(a.B, 256) * up(a.V, 256) >= kComputeUnits / 2;
}

constexpr int32_t kMostD = 131072;
int32_t steps_of(int32_t D) { return up(D, kStepElems); }

// The workspace: states [B] of whole steps, their scales, the needed tokens, the
// arrival counters, the partial sums; each from a multiple of 16 bytes on.
struct Workspace {
    size_t scales, counts, ids, arrivals, partials, total;
    int64_t x_stride;
    int32_t partials_most;
    Workspace(int32_t B, int32_t D, int32_t V, bool mx) {
        const auto whole = [](size_t n) { return (n + 15) / 16 * 16; };
        const int64_t blocks = up(V, kBlockTokens);
        x_stride = (int64_t)steps_of(D) * (mx ? kStep : kWideStep);
        scales = (size_t)B * (size_t)x_stride;
        counts = scales + (mx ? (size_t)scale_at(steps_of(D), (int64_t)up(B, kScaleRows) * kScaleRows, 0) : 0);
        ids = counts + whole(blocks <= kMostBlocks ? blocks * sizeof(int32_t) : 0);
        arrivals = ids + (blocks <= kMostBlocks ? blocks * kBlockTokens * sizeof(int32_t) : 0);
        partials = arrivals + kMostArrivals * sizeof(uint32_t);
        // twice the compute units' number of the largest tiles
        partials_most = (int32_t)std::min<int64_t>((int64_t)kMostArrivals * 128 * 128, (int64_t)16 * up(B, 16) * 16 * (up(V, 128) * 128));
        total = partials + (size_t)partials_most * sizeof(float);
    }
};

// What the caller gives as states.
struct States {
    const void *x;
    psc_form form;
    int64_t stride;
    const uint8_t *scales;
    int64_t scales_stride;
};

// The rows that fit beside the blocks, then the others alone.
template <bool kMx>
void launch_prepare(const MxArgs &a, const States &x, int32_t rows, uint8_t *q, uint8_t *scales, int32_t *counts, int32_t *ids, hipStream_t s) {
    for (int32_t first = 0; first == 0 || first < rows;) {
        MxArgs part = a;
        if (first) part.blocks = 0;
        const int32_t n = (int32_t)std::min<int64_t>(rows - first, kMostGrid - part.blocks);
        const dim3 grid((uint32_t)std::max(n + part.blocks, 1)), block(kPrepareBlock);
        const auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, block, 0, s, part, first, n, x.x, x.stride, x.scales, x.scales_stride, q, scales, counts, ids);
        };
        if (x.form == PSC_FORM_MX4) {
            if constexpr (kMx) go(prepare_mx_kernel<From::kMx, true>);
        } else if (x.form == PSC_FORM_BF16) go(prepare_mx_kernel<From::kBf16, kMx>);
        else go(prepare_mx_kernel<From::kF32, kMx>);
        first += n;
        if (n == 0) break;
    }
}

template <bool kMx>
psc_status head_mx(const char *what, MxArgs &a, const States &x, bool bf16, uint8_t *q, uint8_t *scales, int32_t *counts, int32_t *ids, bool direct, hipStream_t s) {
    const auto prepare = [&](bool needed) {
        if (!needed) return PSC_OK;
        launch_prepare<kMx>(a, x, direct ? 0 : a.B, q, scales, counts, ids, s);
        return launched_op(what);      // the product would go by whatever the workspace holds
    };
    const auto run = [&](auto small) {
        small.shape(a, false);
        if (psc_status st = prepare(!direct || a.counts || a.splits > 1)) return st;
        small.launch(a, bf16, false, s);
        return launched_op(what);
    };
    // Of bfloat16 states the width whose rounds of tiles over the compute units end first: 256 x 151,936 x 4,096 takes 314 us
    // in 3 rounds of 256, 278 in 2 of 320.  Sums and operands in 4 bits of 320 would not fit the registers.
    if (takes_wide(a)) {
        if (psc_status st = prepare(!direct || a.counts)) return st;
        if (a.counts) {
            using Gather = std::conditional_t<kMx, Small<64, 128, 2, 4, 3, true>, Small<64, 128, 1, 8, 3, false>>;
            MxArgs few = a;
            Gather::shape(few, true);
            Gather::launch(few, bf16, true, s);
        }
        if constexpr (!kMx) {
            const int64_t rounds256 = up((int64_t)up(a.B, 256) * up(a.V, 256), kComputeUnits),
                          rounds320 = up((int64_t)up(a.B, 256) * up(a.V, 320), kComputeUnits);
            if (rounds320 * 320 < rounds256 * 256) {
                launch_wide<320, false>(a, bf16, s);
                return launched_op(what);
            }
        }
        launch_wide<256, kMx>(a, bf16, s);
        return launched_op(what);
    }
    // The tiles grow with the rows.  us of states in 4 bits by tiles of 64 x 64 and 64 x 128, the latter by wavefronts of 64
    // and of 32 states: 64 x 128,256 x 4,096 72, 66, 66; 64 x 151,665 x 2,048 under masks 61, 54, 51.  Of bfloat16: 1 x 128,256 x
    // 4,096 by 16 x 64, three steps in LDS, three workgroups a compute unit 50, four steps 55; 32 rows by 32 x 64 82, by
    // 32 x 128 of eight wavefronts 74; 64 rows by 64 x 64 of four 163, by 64 x 128 of eight 118.
    if constexpr (kMx) {
        if (a.B <= 32) return run(Small<32, 64, 1, 4, 4, true>{});
        if (a.B <= 64) return run(Small<64, 128, 2, 4, 3, true>{});
        return run(Small<128, 128, 2, 4, 3, true>{});
    } else {
        if (a.B <= 16) return run(Small<16, 64, 1, 4, 3, false>{});
        if (a.B <= 32) return run(Small<32, 128, 1, 8, 3, false>{});
        return run(Small<64, 128, 1, 8, 3, false>{});
    }
}

}  // namespace

extern "C" size_t psc_head_mx_workspace(int32_t B, int32_t D, int32_t V, psc_form states) {
    if (B <= 0 || D <= 0 || D > kMostD || V <= 0 || V > kMostV || (states != PSC_FORM_BF16 && states != PSC_FORM_MX4)) return 0;
    return Workspace(B, D, V, states == PSC_FORM_MX4).total;
}

extern "C" psc_status psc_head_logits_mx(const void *x, psc_form x_form, int64_t x_stride, const uint8_t *x_scales, int64_t x_scales_stride,
                                         int32_t B, int32_t D, psc_form states, const uint8_t *w, int64_t w_stride,
                                         const uint8_t *w_scales, int64_t w_scales_stride, int32_t V, const float *bias,
                                         const uint32_t *bitmask, void *logits, psc_dtype dtype, int64_t stride, void *workspace,
                                         size_t workspace_bytes, void *stream) {
    const char *what = "psc_head_logits_mx";
    if (psc_status st = check_rows(what, logits, dtype, stride, B, V)) return st;
    if (states != PSC_FORM_BF16 && states != PSC_FORM_MX4) return refuse(what, "states are multiplied in bfloat16 or in 4 bits");
    if (x_form != PSC_FORM_F32 && x_form != PSC_FORM_BF16 && !(x_form == PSC_FORM_MX4 && states == PSC_FORM_MX4))
        return refuse(what, "bad form of x");
    if (D < 1 || D > kMostD) return refuse(what, "D outside [1, 131072]");
    if (V > kMostV) return refuse(what, "V > 2^26");
    if (B == 0 || V == 0) return PSC_OK;
    // workgroups of 512 threads, where needed tokens are taken beside wide_mx_kernel
    if ((int64_t)up(B, 64) * up(V, 512) > kMostGrid / 2) return refuse(what, "ceil(B / 64) * ceil(V / 512) >= 2^23");
    if (!x || !w || !w_scales || !workspace) return refuse(what, "null pointer");
    const int64_t blocks = up(D, kMxBlock);
    if (x_form == PSC_FORM_MX4) {
        if (!x_scales) return refuse(what, "null pointer");
        if (x_stride % 16 || x_stride < blocks * 16 || !aligned_to(x, 16) || x_scales_stride < blocks)
            return refuse(what, "rows of x start at 16 bytes and hold D elements, its scales one of every 32");
    } else if (x_stride < 0 || !aligned_to(x, x_form == PSC_FORM_BF16 ? 2 : 4)) return refuse(what, "negative stride, or x off its elements' alignment");
    if (w_stride % 16 || w_stride < blocks * 16 || w_stride > INT32_MAX / 512 || !aligned_to(w, 16))
        return refuse(what, "rows of w start at 16 bytes and hold D elements");
    if (w_scales_stride % 4 || w_scales_stride < blocks || w_scales_stride > INT32_MAX / 512 || !aligned_to(w_scales, 4))
        return refuse(what, "rows of w_scales start at 4 bytes and hold one of every 32 elements");
    if (workspace_bytes < psc_head_mx_workspace(B, D, V, states) || !aligned_to(workspace, kChunk))
        return refuse(what, "the workspace is too small or not 16-byte aligned");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const bool mx = states == PSC_FORM_MX4;
    const Workspace ws(B, D, V, mx);
    uint8_t *const at = static_cast<uint8_t *>(workspace);
    MxArgs a{};
    a.x = at;
    a.x_stride = ws.x_stride;
    a.x_scales = at + ws.scales;
    // States in bfloat16 that are whole steps at 16-byte addresses are read where they are.
    const bool direct = !mx && x_form == PSC_FORM_BF16 && D % kStepElems == 0 && aligned_to(x, 16) && x_stride % 8 == 0 && (x_stride >= D || B == 1) &&
                        x_stride <= (1 << 22);
    if (direct) {
        a.x = x;
        a.x_stride = x_stride * 2;
    }
    a.w = w;
    a.w_stride = w_stride;
    a.w_scales = w_scales;
    a.w_scales_stride = w_scales_stride;
    a.w_blocks = (int32_t)blocks;
    a.bias = bias;
    a.bitmask = bitmask;
    a.y = logits;
    a.y_stride = stride;
    a.B = B;
    a.D = D;
    a.V = V;
    a.W = up(V, 32);
    a.steps = steps_of(D);
    a.partials = reinterpret_cast<int32_t *>(at + ws.partials);
    a.partials_most = ws.partials_most;
    a.arrivals = reinterpret_cast<uint32_t *>(at + ws.arrivals);
    a.arrivals_most = kMostArrivals;
    // The needed tokens are listed where offsets of all weights fit 32 bits.
    int32_t *counts = nullptr, *ids = nullptr;
    if (bitmask && up(V, kBlockTokens) <= kMostBlocks && (int64_t)V * w_stride < kMostBytes && (int64_t)V * w_scales_stride < kMostBytes) {
        a.blocks = up(V, kBlockTokens);
        a.counts = counts = reinterpret_cast<int32_t *>(at + ws.counts);
        a.ids = ids = reinterpret_cast<int32_t *>(at + ws.ids);
        // Half of them, of states in 4 bits a third; a quarter where wide_mx_kernel takes all.  us with the needed ones only
        // and with all: 8 x 128,256 x 4,096 of bfloat16 45 and 62 where half are needed, 64 rows 90 and 121, at 0.6 119 and
        // 121; 64 x 151,665 x 2,048 in 4 bits 47 and 49 at 0.3, 52 and 49 at 0.4; by wide_mx_kernel 256 x 151,936 x 4,096 in 4 bits
        // 124 and 153 at 0.2, 157 and 154 at 0.3, of bfloat16 256 and 300 at 0.3, 319 and 302 at 0.4; 512 x 128,256 x 2,048 in
        // 4 bits 123 and 125 at 0.1, 162 and 126 at 0.2.
        a.gather_most = takes_wide(a) ? V / 4 : mx ? V / 3 : V / 2;
    }
    const States given{x, x_form, x_stride, x_scales, x_scales_stride};
    uint8_t *const scales = at + ws.scales;
    return mx ? head_mx<true>(what, a, given, dtype == PSC_BF16, at, scales, counts, ids, direct, s)
              : head_mx<false>(what, a, given, dtype == PSC_BF16, at, scales, counts, ids, direct, s);
}
