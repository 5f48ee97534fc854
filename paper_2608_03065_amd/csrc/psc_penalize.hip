// What a request changes in its logits (psc_penalize): penalties of repeated
// tokens, biases of single tokens, and the grammar mask, in place; and the
// token history that the penalties read (psc_append_tokens).
#include "psc_ops.hpp"

#include <algorithm>
#include <type_traits>

using namespace psc;

namespace {

constexpr int kBlock = 256;

// ---------------------------------------------------------------- mask

// A wavefront per kMaskTiles tiles of a row.  Bound by the stores: 256 rows of
// 151,936 bf16 under masks of every kind (70 MB, of which 5 are the masks) take
// 14.3 us, 4.9 TB/s.
constexpr int kMaskTiles = 2;

template <bool kBf16>
__global__ void __launch_bounds__(kBlock)
forbid_kernel(void *__restrict__ logits, int64_t stride, int32_t V, const uint32_t *__restrict__ bitmask, int32_t W) {
    const int32_t wave = (int32_t)blockIdx.x * (kBlock / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t b = blockIdx.y;
    forbid_tiles<kBf16, kMaskTiles>(static_cast<char *>(logits) + b * stride * (kBf16 ? 2 : 4), bitmask + b * W, V, W, wave * kMaskTiles,
                                    threadIdx.x % kWave);
}

// ---------------------------------------------------------------- penalties and biases

constexpr int kPenBlock = 1024;
constexpr int kPenWaves = kPenBlock / kWave;
constexpr int kCounterWords = 38784;   // with kListed places a wavefront nearly all 160 KB of LDS
constexpr int32_t kMostBiases = kPenBlock;
constexpr int kChunk = 2 * kWave;                 // counters that a wavefront looks through at a time
constexpr int kListed = 2 * kWave + kChunk;       // places that its list holds

// Counters of kSlice consecutive tokens of the vocabulary: 2 * occurrences after the
// prompt + (occurs in the prompt), in half a word each where a history is short
// enough (kHalf: up to kHalfCap tokens), so that a slice holds twice as many.
constexpr int32_t kHalfCap = 32767;
template <bool kHalf>
struct Counters {
    static constexpr int kSlice = kCounterWords * (kHalf ? 2 : 1);
    uint32_t *words;      // kCounterWords + kWave: the last ones are the lanes' own, for what is not to be counted

    static __device__ __forceinline__ uint32_t nobody(int lane) { return kSlice + (uint32_t)lane * (kHalf ? 2 : 1); }
    __device__ __forceinline__ uint32_t *word(uint32_t at) const { return words + (kHalf ? at >> 1 : at); }
    static __device__ __forceinline__ int shift(uint32_t at) { return kHalf ? (int)(at & 1) * 16 : 0; }
    // before anything is counted: a neighbour's counter may be cleared with it
    __device__ __forceinline__ void clear(uint32_t at) const { *word(at) = 0; }
    __device__ __forceinline__ void in_prompt(uint32_t at, bool is) const { atomicOr(word(at), (is ? 1u : 0u) << shift(at)); }
    __device__ __forceinline__ void after_prompt(uint32_t at, bool is) const { atomicAdd(word(at), (is ? 2u : 0u) << shift(at)); }
    __device__ __forceinline__ uint32_t get(uint32_t at) const { return kHalf ? *word(at) >> shift(at) & 0xFFFFu : *word(at); }
    // the counter, which becomes 0
    __device__ __forceinline__ uint32_t take(uint32_t at) const {
        if (!kHalf) return atomicExch(word(at), 0u);
        return atomicAnd(word(at), 0xFFFFu << (16 - shift(at))) >> shift(at) & 0xFFFFu;
    }
};

struct PenArgs {
    void *logits;
    int64_t stride;
    const uint32_t *bitmask;
    const int32_t *history, *lens, *prompt_lens;
    const float *repetition, *presence, *frequency;
    const int32_t *bias_ids;
    const float *bias_values;
    int32_t cap, n_bias, V, W;
};

// `parts` workgroups per row go through slices of it: they count the history's
// tokens that lie in the slice in LDS, then change the logits.  A thread holds
// kHeld tokens of the history, so that one of up to kHeld * 1,024 tokens is read
// once.  Two ways, by the row's history:
//
//  Few tokens: only their logits are read and written.  The history is gone
//  through once more, and the first occurrence that takes a token's counter
//  away changes its logit; a counter is cleared only where a token stands.  The
//  mask is applied by tiles, with stores alone.  No branch parts the lanes on
//  this way (what a lane has nothing to do with goes to a counter or an offset
//  of nobody's), so that a lane's accesses are under way together.  Bound by
//  them: each token reads and writes a piece of a line of its own, 256 rows of
//  151,665 bf16 with 300 biases take 19 us with 1,000 tokens each, 40 with 4,000,
//  59 with 8,000.
//
//  At least 3.5 tokens per 128-byte line of the row (`in_order`): the history's
//  tokens stand in no order, and going by them fetches every line several times.
//  Then each wavefront goes through counters in order, lists those that are not
//  0, and changes the listed logits two a lane, neighbours by neighbours: the
//  same rows with 9,400 tokens take 47 us, the other way 66, and under masks of
//  every kind both 52; with 4,000 41 and 40, under masks 47 and 39.  In float32
//  it is ahead from fewer tokens on: 2 a line, without biases, 72 and 82.  (Three a
//  lane took 65 for 62 us, for their list takes LDS from the counters.  Going
//  through the logits themselves, 16 bytes with their counters at a time, took
//  73: its arithmetic is done for all the tokens that do not change.)
//  The number is that of large vocabularies.  All counters are cleared and dealt
//  to the wavefronts however many of them there are tokens for, so that on small
//  ones this way takes longer: 256 rows of 32,000 bf16 with 1,750 tokens 14.9 us and
//  the other way 12.6, with 3,500 17.1 and 15.2; of 5,000 with 273 tokens 10.5 and 4.5.
//
// A workgroup takes all LDS of a compute unit; two or four a compute unit, with
// fewer slices each, took 75 and 83 us where this split took 65.
//
// The biased tokens' logits are written by the threads that hold the biases,
// which take their counters away before.
template <bool kBf16, int kHeld, bool kHalf>
__global__ void __launch_bounds__(kPenBlock)
penalize_kernel(const PenArgs a) {
    constexpr int kElem = kBf16 ? 2 : 4;
    using C = Counters<kHalf>;
    constexpr int kSlice = C::kSlice;
    __shared__ __align__(16) uint32_t s_counters[kCounterWords + kWave];
    // the biases' ids first, then the wavefronts' lists
    __shared__ __align__(16) uint32_t s_shared[kPenWaves * kListed / 2];
    static_assert(sizeof s_shared >= kMostBiases * sizeof(int32_t), "room for the biases");
    int32_t *const s_bias_ids = reinterpret_cast<int32_t *>(s_shared);
    const C counters{s_counters};
    const int64_t b = blockIdx.y;
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int32_t part = blockIdx.x, parts = gridDim.x;
    using T = typename Logit<kBf16>::type;
    T *row = static_cast<T *>(a.logits) + b * a.stride;
    const uint32_t *words = a.bitmask ? a.bitmask + b * a.W : nullptr;
    const bool counts = (int64_t)part * kSlice < a.V;       // whether the workgroup has a slice
    const int32_t *history = a.history + b * a.cap;
    int32_t held[kHeld], n = 0, prompt = 0;
    float r = 1, presence = 0, frequency = 0, bias = 0;
    int32_t bias_id = -1;
    if (a.lens) n = min(max(a.lens[b], 0), a.cap);
    if (counts) {
        if (a.lens) {
            // The first ones are loaded before the length is known: what lies past
            // the history's end, in the buffer, is not used.
            constexpr int kFirst = kHeld < 4 ? kHeld : 4;
            const __amdgpu_buffer_rsrc_t rsrc = buffer_of(history, (uint32_t)min(a.cap, kFirst * kPenBlock) * 4u);
#pragma unroll
            for (int k = 0; k < kFirst; k++)
                held[k] = (int32_t)__builtin_amdgcn_raw_buffer_load_b32(rsrc, (uint32_t)(k * kPenBlock + tid) * 4u, 0, 0);
            const __amdgpu_buffer_rsrc_t rest = buffer_of(history, (uint32_t)min(n, kHeld * kPenBlock) * 4u);
#pragma unroll
            for (int k = kFirst; k < kHeld; k++)
                held[k] = (int32_t)__builtin_amdgcn_raw_buffer_load_b32(rest, (uint32_t)(k * kPenBlock + tid) * 4u, 0, 0);
            prompt = a.prompt_lens ? min(max(a.prompt_lens[b], 0), n) : 0;
        }
        if (a.repetition) r = a.repetition[b];
        if (a.presence) presence = a.presence[b];
        if (a.frequency) frequency = a.frequency[b];
        if (tid < a.n_bias) {
            bias_id = a.bias_ids[b * a.n_bias + tid];
            bias = a.bias_values[b * a.n_bias + tid];
            if (bias_id >= a.V) bias_id = -1;
        }
        if (a.n_bias) s_bias_ids[tid] = bias_id;
    }
    const bool in_order = 2 * (int64_t)n * kLineBytes >= 7 * (int64_t)a.V * kElem;
    if (words) {
        const int32_t pieces = (tiles_of_row(a.V, kElem) + kMaskTiles - 1) / kMaskTiles;
        for (int32_t u = part * kPenWaves + wave; u < pieces; u += parts * kPenWaves)
            forbid_tiles<kBf16, kMaskTiles>(row, words, a.V, a.W, u * kMaskTiles, lane);
    }
    if (!counts || (n == 0 && a.n_bias == 0)) return;
    if (a.n_bias) {
        // of a token's entries the last one counts; places behind n_bias hold -1
        __syncthreads();
        bool last = bias_id >= 0;
        if (__ballot(last)) {
            constexpr int kAtOnce = 16;
            for (int32_t j = wave * kWave; j < a.n_bias; j += kAtOnce) {
                int32_t id[kAtOnce];
#pragma unroll
                for (int e = 0; e < kAtOnce; e++) id[e] = s_bias_ids[j + e];
#pragma unroll
                for (int e = 0; e < kAtOnce; e++) last &= id[e] != bias_id || j + e <= tid;
            }
        }
        if (!last) bias_id = -1;
    }
    const __amdgpu_buffer_rsrc_t logits = buffer_of(row, (uint32_t)a.V * kElem);
    const __amdgpu_buffer_rsrc_t mask = buffer_of(words, words ? (uint32_t)a.W * 4u : 0);
    constexpr uint32_t kNowhere = 0xFFFF8000u;
    // the value of a changed logit: its token's counter, and what is added last
    const auto changed = [&](float x, uint32_t count, float add) {
        float y = x;
        if (count) y = y > 0 ? y / r : y * r;
        if (count >= 2) y = y - (float)(count >> 1) * frequency - presence;
        return y + add;
    };
    const auto load = [&](int32_t t, bool is) {
        const uint32_t at = is ? (uint32_t)t * kElem : kNowhere;
        if constexpr (kBf16) return from_bf16((uint16_t)__builtin_amdgcn_raw_buffer_load_b16(logits, at, 0, 0));
        else return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(logits, at, 0, 0));
    };
    const auto store = [&](int32_t t, bool is, float y) {
        const uint32_t at = is ? (uint32_t)t * kElem : kNowhere;
        if constexpr (kBf16) __builtin_amdgcn_raw_buffer_store_b16((short)to_bf16(y), logits, at, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, y), logits, at, 0, 0);
    };
    const uint32_t all = words ? 0u : ~0u;
    const auto word_at = [&](int32_t w, bool is) { return __builtin_amdgcn_raw_buffer_load_b32(mask, is ? (uint32_t)w * 4u : kNowhere, 0, 0) | all; };
    // a biased token's mask and logit, which this thread alone changes
    const bool has_bias = bias_id >= 0;
    const uint32_t bias_word = word_at(bias_id >> 5, has_bias);
    const float bias_logit = load(bias_id, has_bias);
    const bool bias_counts = has_bias && (bias_word >> (bias_id & 31) & 1) && bias_logit != kMinusInf;
    for (int64_t start = (int64_t)part * kSlice; start < a.V; start += (int64_t)parts * kSlice) {
        const int32_t v0 = (int32_t)start;
        const uint32_t size = (uint32_t)min(kSlice, a.V - v0);
        // the slice's counter of token t, or the lane's own
        const auto place = [&](int32_t t, bool is) {
            const uint32_t at = (uint32_t)t - (uint32_t)v0;
            return is && at < size ? at : C::nobody(lane);
        };
        const uint32_t bias_at = place(bias_id, has_bias);
        const bool biased = bias_at < size;
        if (in_order) {
            for (int32_t i = tid * 4; i < kCounterWords; i += kPenBlock * 4) *reinterpret_cast<u32x4 *>(s_counters + i) = u32x4{};
        } else {
#pragma unroll
            for (int k = 0; k < kHeld; k++)
                if (k * kPenBlock < n) counters.clear(place(held[k], k * kPenBlock + tid < n));
            for (int32_t i = kHeld * kPenBlock + tid; i < n; i += kPenBlock) counters.clear(place(history[i], true));
            if (biased) counters.clear(bias_at);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kHeld; k++) {
            if (k * kPenBlock >= n) continue;
            const int32_t i = k * kPenBlock + tid;
            const uint32_t at = place(held[k], i < n);
            if (k * kPenBlock < prompt) counters.in_prompt(at, i < prompt);
            if ((k + 1) * kPenBlock > prompt) counters.after_prompt(at, i >= prompt);
        }
        for (int32_t i = kHeld * kPenBlock + tid; i < n; i += kPenBlock) {
            const uint32_t at = place(history[i], true);
            if (i < prompt) counters.in_prompt(at, true);
            else counters.after_prompt(at, true);
        }
        __syncthreads();
        if (a.n_bias) {
            // takes the token's count away from the history's occurrences, and changes the logit by both
            if (biased) store(bias_id, bias_counts, changed(bias_logit, counters.take(bias_at), bias));
            __syncthreads();
        }
        if (in_order) {
            uint16_t *const list = reinterpret_cast<uint16_t *>(s_shared) + wave * kListed;
            uint32_t listed = 0;
            // the wavefront's part of the slice; a list's entries are places in it
            const uint32_t share = (kSlice / kPenWaves + kChunk - 1) / kChunk * kChunk, first = (uint32_t)wave * share,
                           end = min(size, first + share);
            static_assert(kSlice / kPenWaves + kChunk <= 0x10000 && kSlice % 2 == 0, "an entry's 16 bits, whole pairs");
            const auto change = [&](uint32_t from, uint32_t n_of) {
                uint32_t at[2], count[2], word[2];
                float x[2];
                asm volatile("" ::: "memory");      // the list is the other lanes' too
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const uint32_t e = (uint32_t)(i * kWave + lane);
                    const bool is = e < n_of;
                    at[i] = first + (is ? list[from + e] : 0u);
                    count[i] = is ? counters.get(at[i]) : 0;
                    word[i] = word_at((v0 + (int32_t)at[i]) >> 5, is);
                }
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const int32_t t = v0 + (int32_t)at[i];
                    count[i] = word[i] >> (t & 31) & 1 ? count[i] : 0;
                    x[i] = load(t, count[i] != 0);
                }
#pragma unroll
                for (int i = 0; i < 2; i++)
                    store(v0 + (int32_t)at[i], count[i] != 0 && x[i] != kMinusInf, changed(x[i], count[i], 0.0f));
                asm volatile("" ::: "memory");
            };
            constexpr int kAtOnce = 4;      // chunks whose counters are read together
            for (uint32_t at = first; at < end; at += kChunk * kAtOnce) {
                uint32_t two[kAtOnce][2];
#pragma unroll
                for (int i = 0; i < kAtOnce; i++) {
                    // counters of the slice past its tokens are 0
                    const uint32_t mine = at + (uint32_t)(i * kChunk + lane * 2);
                    const bool is = mine < min(first + share, (uint32_t)kSlice);
                    if (kHalf) {
                        const uint32_t w = is ? *counters.word(mine) : 0;
                        two[i][0] = w & 0xFFFFu;
                        two[i][1] = w >> 16;
                    } else {
                        two[i][0] = is ? *counters.word(mine) : 0;
                        two[i][1] = is ? *counters.word(mine + 1) : 0;
                    }
                }
#pragma unroll
                for (int i = 0; i < kAtOnce; i++) {
                    const uint32_t mine = at - first + (uint32_t)(i * kChunk + lane * 2);
                    const uint32_t n_mine = (two[i][0] != 0) + (two[i][1] != 0), upto = wave_scan(n_mine, 0u, kAdd);
                    uint32_t to = listed + upto - n_mine;
                    if (two[i][0]) list[to++] = (uint16_t)mine;
                    if (two[i][1]) list[to] = (uint16_t)(mine + 1);
                    listed += lane_value(upto, kWave - 1);
                    if (listed >= 2 * kWave) {
                        listed -= 2 * kWave;
                        change(listed, 2 * kWave);
                    }
                }
            }
            change(0, listed);
            __syncthreads();
            continue;
        }
        // kGroup of the held tokens together from the g-th on; of all 16 at once
        // the values would not fit the registers.
        const auto change_held = [&](auto group, int g) {
            constexpr int kGroup = decltype(group)::value;
            uint32_t count[kGroup], word[kGroup];
            float x[kGroup];
#pragma unroll
            for (int e = 0; e < kGroup; e++) {
                const int k = g + e;
                count[e] = k * kPenBlock < n ? counters.take(place(held[k], k * kPenBlock + tid < n)) : 0;
            }
            // nothing is loaded of logits that another occurrence or a bias has taken, or that are forbidden
#pragma unroll
            for (int e = 0; e < kGroup; e++) {
                const int k = g + e;
                const bool mine = k * kPenBlock + tid < n && place(held[k], true) < size;
                count[e] = mine ? count[e] : 0;
                word[e] = word_at(held[k] >> 5, count[e] != 0);
            }
#pragma unroll
            for (int e = 0; e < kGroup; e++) {
                const int32_t t = held[g + e];
                count[e] = word[e] >> (t & 31) & 1 ? count[e] : 0;
                x[e] = load(t, count[e] != 0);
            }
#pragma unroll
            for (int e = 0; e < kGroup; e++) store(held[g + e], count[e] != 0 && x[e] != kMinusInf, changed(x[e], count[e], 0.0f));
        };
        // Accesses to nowhere cost time too: a short history in a long buffer goes
        // alone (256 rows of 500 tokens of 16,384: 10.7 us, by eight 13.4).
        if (n <= kPenBlock) {
            change_held(std::integral_constant<int, 1>{}, 0);
        } else if constexpr (kHeld == 4) {
            change_held(std::integral_constant<int, 4>{}, 0);
        } else if constexpr (kHeld == 16) {
            change_held(std::integral_constant<int, 8>{}, 0);
            if (n > 8 * kPenBlock) change_held(std::integral_constant<int, 8>{}, 8);
        }
        static_assert(kHeld == 1 || kHeld == 4 || kHeld == 16, "the numbers handled here");
        for (int32_t i = kHeld * kPenBlock + tid; i < n; i += kPenBlock) {
            const int32_t t = history[i];
            const uint32_t at = place(t, true);
            if (at >= size) continue;
            const uint32_t c = counters.take(at);
            if (!c || !(word_at(t >> 5, true) >> (t & 31) & 1)) continue;
            const float y = load(t, true);
            store(t, y != kMinusInf, changed(y, c, 0.0f));
        }
        __syncthreads();
    }
}

// One wait and one store: 1.5 us for 256 rows.
__global__ void __launch_bounds__(kBlock)
append_kernel(int32_t *__restrict__ history, int32_t cap, int32_t *__restrict__ lens, int32_t B,
              const int32_t *__restrict__ tokens, int32_t *__restrict__ status) {
    const int64_t b = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (b >= B) return;
    const int32_t t = tokens[b], n = lens[b];
    int32_t st = PSC_ADV_OK;
    if (t < 0) st = PSC_ADV_SKIPPED;
    else if (n < 0) st = PSC_ADV_BAD_INPUT;
    else if (n >= cap) st = PSC_ADV_OVERFLOW;
    else {
        history[b * cap + n] = t;
        lens[b] = n + 1;
    }
    if (status) status[b] = st;
}

constexpr int32_t kMostRows = 65535;      // the grid's second dimension
constexpr int32_t kComputeUnits = 256;

template <bool kBf16>
void launch_penalize(const PenArgs &a, int32_t B, hipStream_t s) {
    // b passes 31 bits after the last rows
    for (int64_t b = 0; b < B; b += kMostRows) {
        const int32_t rows = (int32_t)std::min<int64_t>(kMostRows, B - b);
        PenArgs p = a;
        p.logits = static_cast<char *>(a.logits) + b * a.stride * (kBf16 ? 2 : 4);
        if (a.bitmask) p.bitmask = a.bitmask + b * a.W;
        const int32_t tiles = tiles_of_row(a.V, kBf16 ? 2 : 4);
        if (!a.lens && !a.n_bias) {
            constexpr int kTiles = kMaskTiles * kBlock / kWave;
            if (a.bitmask)
                hipLaunchKernelGGL(forbid_kernel<kBf16>, dim3((tiles + kTiles - 1) / kTiles, rows), dim3(kBlock), 0, s, p.logits, a.stride,
                                   a.V, p.bitmask, a.W);
            continue;
        }
        if (a.lens) p.history = a.history + b * a.cap, p.lens = a.lens + b;
        if (a.prompt_lens) p.prompt_lens = a.prompt_lens + b;
        if (a.repetition) p.repetition = a.repetition + b;
        if (a.presence) p.presence = a.presence + b;
        if (a.frequency) p.frequency = a.frequency + b;
        if (a.n_bias) p.bias_ids = a.bias_ids + b * a.n_bias, p.bias_values = a.bias_values + b * a.n_bias;
        // As many workgroups a row as it has slices, or shares of tiles to mask,
        // up to one per compute unit in all.
        const bool half = a.cap <= kHalfCap;
        const int32_t slice = half ? Counters<true>::kSlice : Counters<false>::kSlice;
        const int32_t slices = (int32_t)(((int64_t)a.V + slice - 1) / slice);
        const int32_t shares = a.bitmask ? (tiles + kMaskTiles * kPenWaves - 1) / (kMaskTiles * kPenWaves) : 1;
        const int32_t parts = std::max(1, std::min(std::max(slices, shares), (kComputeUnits + rows - 1) / rows));
        const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(parts, rows), dim3(kPenBlock), 0, s, p); };
        if (a.cap <= kPenBlock) go(penalize_kernel<kBf16, 1, true>);
        else if (a.cap <= kPenBlock * 4) go(penalize_kernel<kBf16, 4, true>);
        else if (half) go(penalize_kernel<kBf16, 16, true>);
        else go(penalize_kernel<kBf16, 16, false>);
    }
}

}  // namespace

extern "C" psc_status psc_penalize(void *logits, psc_dtype dtype, int64_t stride, int32_t B, int32_t V,
                                   const psc_penalties *penalties, const uint32_t *bitmask, void *stream) {
    const char *what = "psc_penalize";
    if (psc_status st = check_rows(what, logits, dtype, stride, B, V)) return st;
    if ((int64_t)V * size_of(dtype) >= (int64_t)1 << 31) return refuse(what, "rows of 2 GiB or more");
    PenArgs a{};
    if (penalties) {
        const psc_penalties &p = *penalties;
        if (p.cap < 0 || p.n_bias < 0) return refuse(what, "negative size");
        if (p.cap > (1 << 30)) return refuse(what, "a history of more than 2^30 tokens");
        if (p.n_bias > kMostBiases) return refuse(what, "more than 1,024 biases a row");
        if (p.cap > 0 && B > 0) {
            if (!p.history || !p.lens) return refuse(what, "null history or lengths");
            a.history = p.history;
            a.lens = p.lens;
            a.prompt_lens = p.prompt_lens;
            a.cap = p.cap;
        }
        if (p.n_bias > 0 && B > 0) {
            if (!p.bias_ids || !p.bias_values) return refuse(what, "null biases");
            a.bias_ids = p.bias_ids;
            a.bias_values = p.bias_values;
            a.n_bias = p.n_bias;
        }
        a.repetition = p.repetition;
        a.presence = p.presence;
        a.frequency = p.frequency;
    }
    if (B == 0 || V == 0) return PSC_OK;
    a.logits = logits;
    a.stride = stride;
    a.bitmask = bitmask;
    a.V = V;
    a.W = (int32_t)(((int64_t)V + 31) / 32);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (dtype == PSC_BF16) launch_penalize<true>(a, B, s);
    else launch_penalize<false>(a, B, s);
    return launched_op(what);
}

extern "C" psc_status psc_append_tokens(int32_t *history, int32_t cap, int32_t *lens, int32_t B, const int32_t *tokens,
                                        int32_t *status, void *stream) {
    const char *what = "psc_append_tokens";
    if (B < 0 || cap < 0) return refuse(what, "negative size");
    if (B == 0) return PSC_OK;
    if ((cap > 0 && !history) || !lens || !tokens) return refuse(what, "null pointer");
    hipLaunchKernelGGL(append_kernel, dim3((uint32_t)(((int64_t)B + kBlock - 1) / kBlock)), dim3(kBlock), 0,
                       reinterpret_cast<hipStream_t>(stream), history, cap, lens, B, tokens, status);
    return launched_op(what);
}
