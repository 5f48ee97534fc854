// What the output projections share (psc_head.hip, psc_head_mx.hip): how a call is
// carried out, the list of tokens that any row allows, loads to LDS, and the
// logits that a mask forbids.  Not part of the public ABI.
#pragma once

#include <algorithm>

#include "psc_ops.hpp"

namespace psc {

constexpr int kPrepareBlock = 256;

// ---------------------------------------------------------------- the product's arguments

constexpr int kStep = 128;        // bytes of a row per step along D: one line
constexpr int kChunk = 16;        // bytes per lane of a load and of a matrix instruction's operand
constexpr int kChunks = kStep / kChunk;
constexpr uint32_t kNowhere = 0xFFFF8000u;        // an offset past any resource: the hardware drops the access
constexpr uint32_t kMostBytes = 0xFFFF0000u;      // of a resource
constexpr int32_t kMostRows = 256;                // of a tile

// The tokens that any row allows, in blocks of kBlockWords mask words: each
// block's number of them, and their ids in ascending order.
constexpr int kBlockWords = 64, kBlockTokens = kBlockWords * 32;
constexpr int kMostBlocks = 512;                  // V up to 1,048,576

// What every output projection is told about its logits and how it is carried out.
struct HeadBase {
    const float *bias;
    const uint32_t *bitmask;
    void *y;
    int64_t y_stride;
    int32_t B, D, V, W;
    int32_t steps, m_tiles;
    int32_t splits;               // parts of D, where all tokens are taken
    const int32_t *counts, *ids;  // needed tokens: [blocks], [blocks][kBlockTokens]; null without a mask
    int32_t blocks;
    int32_t gather_most;          // most needed tokens at which only they are taken
    int32_t units;                // workgroups there are for tiles times parts
    int32_t *partials;            // [tiles][parts][kM * kN] sums, where D is split
    int32_t partials_most;        // their room
    uint32_t *arrivals;           // [tiles] parts that have ended: cleared before the product
    int32_t arrivals_most;
};

// Parts of D at most.  us with at most 4, 8 and 16: 64 x 128,256 x 8,192 with few
// tokens needed 34.5, 32.5, 35.1; 32 x 32,000 x 2,048 17.6, 17.0, 17.4; but 64 x 8,000
// x 4,096 18.3, 20.9, 20.9 and 1 x 4,096 x 8,192 14.1, 15.9, 16.0.
constexpr int32_t kMostSplits = 8;

// How a call is carried out: which columns (all tokens, or the needed ones),
// and in how many parts of D each.  Every workgroup works it out alike.
struct Plan {
    bool gather;
    int32_t columns, tiles, splits;
};

// What is read is the wavefront's; `total` is the last lane's needed_upto.
template <int kM, int kN>
__device__ __forceinline__ Plan plan_of(const HeadBase &a, int32_t total) {
    Plan p{false, a.V, (a.V + kN - 1) / kN, a.splits};
    if (a.counts && total <= a.gather_most) {
        p.gather = true;
        p.columns = total;
        p.tiles = (total + kN - 1) / kN;
        const int32_t tiles = max(p.tiles * a.m_tiles, 1);
        const int32_t room = tiles > a.arrivals_most ? 1 : a.partials_most / (tiles * kM * kN);
        // of at least two steps; one or four make no difference (8 x 128,256 x 4,096 with 160 tokens needed: 14.0, 14.1)
        p.splits = max(1, min(min(a.units / tiles, room), min(a.steps / 2, kMostSplits)));
    }
    return p;
}

// Sum of the blocks' counts up to and with the lane's share of them, kShare
// consecutive blocks a lane.
constexpr int kShare = kMostBlocks / kWave;
__device__ __forceinline__ int32_t needed_upto(const HeadBase &a, int lane, int32_t (&count)[kShare]) {
    int32_t sum = 0;
#pragma unroll
    for (int i = 0; i < kShare; i++) {
        const int32_t at = lane * kShare + i;
        count[i] = at < a.blocks ? a.counts[at] : 0;
        sum += count[i];
    }
    return wave_scan(sum, 0, kAdd);
}

// ---------------------------------------------------------------- needed tokens

// Block `block` of the needed tokens: the OR of the rows' words, by one
// workgroup, its wavefronts over every fourth row.  Most masks allow almost all
// tokens; as soon as a block has all of its bits, the other rows are not read.
__device__ __forceinline__ void needed_block(const HeadBase &a, int32_t block, int32_t *__restrict__ counts,
                                             int32_t *__restrict__ ids, uint32_t (*s_words)[kBlockWords]) {
    constexpr int kWaves = kPrepareBlock / kWave, kAhead = 16;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int32_t w = block * kBlockWords + lane;
    const int32_t left = a.V - w * 32;        // tokens from the word's first on
    const uint32_t inside = left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1;
    uint32_t any = 0;
    for (int32_t b = wave; b < a.B; b += kWaves * kAhead) {
        uint32_t word[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const int32_t row = b + i * kWaves;
            word[i] = inside && row < a.B ? a.bitmask[(int64_t)row * a.W + w] : 0;
        }
#pragma unroll
        for (int i = 0; i < kAhead; i++) any |= word[i];
        if (!__ballot((any & inside) != inside)) break;
    }
    s_words[wave][lane] = any & inside;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int i = 1; i < kWaves; i++) any |= s_words[i][lane];
    any &= inside;
    const int32_t n = __popc(any), upto = wave_scan(n, 0, kAdd);
    if (lane == kWave - 1) counts[block] = upto;
    int32_t *to = ids + (int64_t)block * kBlockTokens + upto - n;
    for (; any; any &= any - 1) *to++ = w * 32 + __ffs((int)any) - 1;
}

__device__ __forceinline__ uint32_t load_word(__amdgpu_buffer_rsrc_t from, int32_t at) {
    return __builtin_amdgcn_raw_buffer_load_b32(from, (uint32_t)at * 4u, 0, 0);
}

// The mask's words from row m0 on; nothing without a mask.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t mask_from(const HeadBase &a, int32_t m0) {
    const int64_t rows = a.bitmask ? min(a.B - m0, kMostRows) : 0;
    return buffer_of(a.bitmask + (a.bitmask ? (int64_t)m0 * a.W : 0), (uint32_t)min(rows * a.W * 4, (int64_t)kMostBytes));
}

// -inf in the forbidden logits and nothing else: the allowed ones are written
// by other workgroups.  `part` of `parts` workgroups; each wavefront takes
// kTiles tiles of a row at a time.
template <bool kBf16, int kTiles>
__device__ __forceinline__ void fill_forbidden(const HeadBase &a, int32_t part, int32_t parts) {
    constexpr int kElem = kBf16 ? 2 : 4;
    const int32_t waves = (int32_t)blockDim.x / kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int32_t pieces = (tiles_of_row(a.V, kElem) + kTiles - 1) / kTiles;
    const int64_t all = (int64_t)a.B * pieces;
    for (int64_t u = (int64_t)part * waves + wave; u < all; u += (int64_t)parts * waves) {
        const int64_t b = u >> 32 ? u / pieces : (int64_t)((uint32_t)u / (uint32_t)pieces);
        forbid_tiles<kBf16, kTiles>(static_cast<char *>(a.y) + b * a.y_stride * kElem, a.bitmask + b * a.W, a.V, a.W,
                                    (int32_t)(u - b * pieces) * kTiles, threadIdx.x % kWave);
    }
}

// ---------------------------------------------------------------- loads to LDS

// Wait until at most n of the wavefront's loads are outstanding and its reads
// of LDS are done, then for the other wavefronts of the workgroup.
template <int n>
__device__ __forceinline__ void wait_and_meet() {
    static_assert(n < 64, "the counter's range");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(n) : "memory");
}

// 16 bytes per lane from the resource straight to LDS: lane l's to place l from
// byte `to` of LDS on (M0; the hardware wants an instruction between its write
// and the load).  In assembly, because the compiler would wait for all such
// loads before any read of LDS; wait_and_meet waits for the ones that are due.
__device__ __forceinline__ void load_to_lds(u32x4 from, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(from)
                 : "memory", "m0");
}

// The byte of LDS that a pointer into it names.
__device__ __forceinline__ uint32_t lds_byte(const void *p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}

// The words of buffer_of's resource.
__device__ __forceinline__ u32x4 rows_from(const void *p, int64_t bytes) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    return u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, (uint32_t)min(max(bytes, (int64_t)0), (int64_t)kMostBytes), 0x00020000u};
}

// ---------------------------------------------------------------- host side

constexpr int32_t kComputeUnits = 256;
inline int32_t up(int64_t n, int64_t d) { return (int32_t)((n + d - 1) / d); }

// Workgroups of one launch: a grid's threads are fewer than 2^32 in each dimension.
constexpr int64_t kMostGrid = ((int64_t)1 << 32) / kPrepareBlock - 1;

constexpr int32_t kMostV = 1 << 26;      // offsets into a tile's rows of the mask fit 32 bits
static_assert((int64_t)kMostRows * (kMostV / 32) * 4 < kMostBytes, "and are inside a resource");
constexpr int32_t kMostArrivals = 2 * kComputeUnits;

// How a small kernel is launched: its tiles of kM by kN, the parts of D, and the
// workgroups, of which there are enough to split D further when few tokens are needed.
template <int kM, int kN>
void shape_small(HeadBase &a, bool gather_only) {
    a.m_tiles = up(a.B, kM);
    const int64_t tiles = (int64_t)a.m_tiles * up(a.V, kN);
    // Parts of D where the tiles alone would leave compute units idle, of at
    // least four steps each.  us in parts of at least 1, 4 and 8 steps, and whole:
    // 64 x 16,000 x 1,024 18.7, 15.3, 11.8, 11.9; 128 x 4,000 x 2,048 20.1, 16.0, 16.7,
    // 16.6; 16 x 2,000 x 4,096 11.3, 11.3, 10.5, 13.2; 1 x 4,096 x 8,192 16.0, 15.9,
    // 15.9, 19.8.  128 x 16,000 x 4,096, 125 tiles, would be better off whole: 40.1 in
    // parts, 29.7.
    const int64_t room = tiles > a.arrivals_most ? 1 : a.partials_most / (tiles * kM * kN);
    a.splits = gather_only ? 1 : (int32_t)std::max<int64_t>(1, std::min<int64_t>({2 * kComputeUnits / tiles, a.steps / 4, kMostSplits, room}));
    // the entry point has seen to it that units of 256 threads fit a launch (V / 4 tokens at most, where only needed ones are taken)
    a.units = (int32_t)std::max<int64_t>(gather_only ? (int64_t)a.m_tiles * up(a.gather_most, kN) : tiles * a.splits, 2 * kComputeUnits);
}

}  // namespace psc
