// From logits to a token (psc_sample): the log of the sum of the allowed
// tokens' exponentials, the k best tokens with their log-probabilities, and
// one token drawn from these under temperature, top-k, top-p and min-p.
//
// Two kernels.  The scan reads every allowed logit once and leaves, per 4 KB of
// a row, its maximum and the sum of exponentials below it, and per group of 64
// tokens the group's maximum.  The k best tokens lie in the k groups with the
// largest maxima (ties to the lower group): any token outside them is preceded
// by those groups' k maxima, which are larger, or equal and of lower id.  So
// the second kernel, a workgroup per row, selects groups that hold these k,
// reads them again, orders their best tokens and draws.
//
// The scan is bound by memory: 512 rows of 128,256 bf16 (131 MB) take 30 us, 4.4
// TB/s, where a large copy reaches 4.8; under masks by two waits in a row, for
// the words and then for the logits that they allow (whole 128-byte lines of
// them: 96 rows of 262,145 float32 of which 37 MB are allowed fetch 66 MB in 21
// us).  The pick is a chain of waits and barriers, 6 us for a row of 32,000 and 8
// to 9.5 for 64 to 512 rows at once.  One launch for both, each row's workgroup scanning it alone, takes
// 0.7 us less up to 32 KB a row and 2 more at 128 KB, where that unit's reads
// are the bound.
//
// Log-probabilities are off by 1.2e-7 (rms) where the best token has nearly all
// of the probability: by the roundings of sums that hold its 1.
#include "psc_ops.hpp"

#include <algorithm>
#include <cfloat>

using namespace psc;

namespace {

constexpr int kScanBlock = 256;
constexpr int kGroup = 64;                          // tokens per group
constexpr int kVecs = kTileBytes / 16 / kWave;      // 16-byte vectors per lane
constexpr uint32_t kOffSkip = 0x80000000u;
constexpr int kMostK = kWave;

struct SampleArgs {
    const void *logits;
    int64_t stride;
    const uint32_t *bitmask;
    int32_t V, W, k, tiles;
    const float *temperature, *top_p, *min_p, *noise;
    const int32_t *top_k;
    uint32_t *group_keys;        // [B][tiles * Row::kTileGroups]
    float2 *parts;               // [B][tiles] (maximum, sum)
    int32_t *tokens, *ids;
    float *logprobs, *id_logprobs;
};

// An order-preserving key of a logit: larger number, larger key, a NaN above
// every number, -0 as +0; 0 for -inf, which is never drawn.
__device__ __forceinline__ uint32_t key_of(float f) {
    const uint32_t u = __builtin_bit_cast(uint32_t, f + 0.0f);
    if (f != f) return ~0u;
    if (f == kMinusInf) return 0;
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t key) {
    if (key == 0) return kMinusInf;
    return __builtin_bit_cast(float, key == ~0u ? 0x7FC00000u : key >> 31 ? key & 0x7FFFFFFFu : ~key);
}

// 1 / temperature as the exponentials' factor; a temperature that is not
// above zero means the best token, with the probabilities of temperature 1.
// The bounds keep 0 * inf out of the products.
__device__ __forceinline__ float inverse_temperature(const float *temperature, int64_t b) {
    const float t = temperature ? temperature[b] : 1.0f;
    return t > 0 ? fminf(fmaxf(1.0f / t, 1e-30f), 1e30f) : 1.0f;
}

constexpr float kLog2e = 1.44269504088896340736f;
// exp(x * c) for x <= 0
__device__ __forceinline__ float exp_scaled(float x, float c) { return __builtin_amdgcn_exp2f(x * c * kLog2e); }

// The larger of two floats; a NaN wins.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

constexpr auto kLarger = [](float a, float b) { return larger(a, b); };

// Row b: `line` is the 128-byte line that holds its first element, the delta
// elements before it there are not the row's.
template <bool kBf16>
struct Row {
    static constexpr int kElem = kBf16 ? 2 : 4, kPerVec = 16 / kElem;
    static constexpr int kTileGroups = kTileBytes / (kGroup * kElem), kGroupLanes = kGroup / kPerVec;
    const char *line;
    int32_t delta;
    __device__ __forceinline__ Row(const SampleArgs &a, int64_t b) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(a.logits) + (uintptr_t)(b * a.stride) * kElem;
        line = reinterpret_cast<const char *>(at & ~(uintptr_t)(kLineBytes - 1));
        delta = (int32_t)(at & (kLineBytes - 1)) / kElem;
    }
};

// Bits of the `count` tokens from v on (v may be negative): 1 where a token
// is in the vocabulary and allowed.  Without branches, so that the words' loads
// overlap what else is loaded.
__device__ __forceinline__ uint32_t allowed_bits(const uint32_t *__restrict__ words, int32_t v, int count, int32_t V, int32_t W) {
    uint32_t in = (1u << count) - 1;
    if (v < 0) in = v > -count ? in & ~0u << -v : 0;
    if (v + count > V) in = v < V ? in & ((1u << (V - v)) - 1) : 0;
    if (!words) return in;
    const int32_t w = v >> 5, last = W - 1;
    const uint32_t lo = words[min(max(w, 0), last)], hi = words[min(max(w + 1, 0), last)];
    return __builtin_amdgcn_alignbit(hi, lo, (uint32_t)v & 31) & in;
}

template <bool kBf16>
__global__ void __launch_bounds__(kScanBlock)
scan_kernel(const SampleArgs a) {
    using R = Row<kBf16>;
    const int lane = threadIdx.x % kWave;
    const int64_t b = blockIdx.y;
    const int32_t t = blockIdx.x * (kScanBlock / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (t >= a.tiles) return;
    const R row(a, b);
    const char *tile = row.line + (int64_t)t * kTileBytes;
    const uint32_t *words = a.bitmask ? a.bitmask + b * a.W : nullptr;
    const float c = inverse_temperature(a.temperature, b) * kLog2e;
    const __amdgpu_buffer_rsrc_t rsrc = buffer_of(tile, kTileBytes);
    uint32_t keep[kVecs];
    u32x4 x[kVecs];
    bool edge = false;
#pragma unroll
    for (int j = 0; j < kVecs; j++) {
        const int at = (j * kWave + lane) * R::kPerVec;
        const int32_t v = t * (kTileBytes / R::kElem) + at - row.delta;
        keep[j] = allowed_bits(words, v, R::kPerVec, a.V, a.W);
        // a vector that reaches out of the row is read by element
        const bool whole = v >= 0 && v + R::kPerVec <= a.V;
        edge |= keep[j] && !whole;
        x[j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, keep[j] && whole ? (uint32_t)at * R::kElem : kOffSkip, 0, 2);
    }
    if (__ballot(edge)) {
#pragma unroll
        for (int j = 0; j < kVecs; j++) {
            const int at = (j * kWave + lane) * R::kPerVec;
            const int32_t v = t * (kTileBytes / R::kElem) + at - row.delta;
            if (!keep[j] || (v >= 0 && v + R::kPerVec <= a.V)) continue;
#pragma unroll
            for (int e = 0; e < R::kPerVec; e++) {
                if (!((keep[j] >> e) & 1)) continue;
                if constexpr (kBf16) x[j][e / 2] |= (uint32_t) reinterpret_cast<const uint16_t *>(tile)[at + e] << (e % 2 * 16);
                else x[j][e] = reinterpret_cast<const uint32_t *>(tile)[at + e];
            }
        }
    }
    // -inf in place of what is not allowed; most tiles without a mask have none
    constexpr uint32_t kWhole = (1u << R::kPerVec) - 1;
    bool part = false;
#pragma unroll
    for (int j = 0; j < kVecs; j++) part |= keep[j] != kWhole;
    if (__ballot(part)) {
#pragma unroll
        for (int j = 0; j < kVecs; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const auto bit = [&](int i) { return (uint32_t)((int32_t)(keep[j] << (31 - i)) >> 31); };
                const uint32_t is = kBf16 ? (bit(2 * e) & 0xFFFFu) | (bit(2 * e + 1) & 0xFFFF0000u) : bit(e);
                x[j][e] = (x[j][e] & is) | ((kBf16 ? 0xFF80FF80u : 0xFF800000u) & ~is);
            }
    }
    const auto value = [&](int j, int e) {
        return __builtin_bit_cast(float, kBf16 ? (e % 2 ? x[j][e / 2] & 0xFFFF0000u : x[j][e / 2] << 16) : x[j][e]);
    };
    float most = kMinusInf;
    uint32_t *keys = a.group_keys + (b * a.tiles + t) * R::kTileGroups;
#pragma unroll
    for (int j = 0; j < kVecs; j++) {
        float m = kMinusInf;
#pragma unroll
        for (int e = 0; e < R::kPerVec; e++) m = larger(m, value(j, e));
        // over the 8 or 16 lanes that hold a group
        m = larger(m, dpp_from<0xB1, 0xF>(m, m));     // quad_perm [1,0,3,2]
        m = larger(m, dpp_from<0x4E, 0xF>(m, m));     // quad_perm [2,3,0,1]
        m = larger(m, dpp_from<0x141, 0xF>(m, m));    // row_half_mirror
        if (!kBf16) m = larger(m, dpp_from<0x140, 0xF>(m, m));    // row_mirror
        if (lane % R::kGroupLanes == 0) keys[(j * kWave + lane) / R::kGroupLanes] = key_of(m);
        most = larger(most, m);
    }
    most = wave_all(most, kMinusInf, kLarger);
    float sum = 0;
    if (most > kMinusInf || most != most) {
#pragma unroll
        for (int j = 0; j < kVecs; j++)
#pragma unroll
            for (int e = 0; e < R::kPerVec; e++) sum += __builtin_amdgcn_exp2f((value(j, e) - most) * c);
    }
    sum = wave_all(sum, 0.0f, kAdd);
    if (lane == 0) a.parts[b * a.tiles + t] = make_float2(most, sum);
}

// ---------------------------------------------------------------- selection

constexpr int kPickBlock = 256;
constexpr int kPickWaves = kPickBlock / kWave;
constexpr int kBinsEach = 4, kBins = kPickBlock * kBinsEach;
constexpr int kMostGroups = 128;
constexpr int kMostFound = kPickBlock;                    // a multiple of 16

struct PickShared {
    __align__(16) uint32_t bins[kBins];
    uint32_t waves[kPickWaves];
    float2 parts[kPickWaves];
    uint32_t least[kPickWaves], most[kPickWaves];
    uint32_t lo, hi, count, bin, above, in_bin, n_groups, n_found;
    int32_t groups[kMostGroups];
    __align__(16) uint64_t found[kMostFound];
    uint64_t best[kMostK];
};

// Larger for a larger key, and of equal keys for the lower token.
__device__ __forceinline__ uint64_t ranked(uint32_t key, int32_t id) { return (uint64_t)key << 32 | ~(uint32_t)id; }

// The sum of v over the threads before this one.  Every thread calls it.
__device__ __forceinline__ uint32_t block_before(uint32_t v, PickShared &s) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const uint32_t upto = wave_scan(v, 0u, kAdd);
    if (lane == kWave - 1) s.waves[wave] = upto;
    __syncthreads();
    uint32_t before = upto - v;
#pragma unroll
    for (int i = 0; i < kPickWaves; i++) before += i < wave ? s.waves[i] : 0;
    return before;
}

// One round of the search for the k-th largest of the workgroup's keys, of
// which more than k lie in [lo, hi] or above: a histogram of the keys in [lo,
// hi] over equal bins.  [lo, hi] becomes the bin in which the number of keys
// from the top reaches k; `above` keys are larger, in_bin lie in it.
// bins are zero before and after.
template <int kPer>
__device__ __forceinline__ void narrow(const uint32_t (&key)[kPer], uint32_t k, PickShared &s, uint32_t &lo, uint32_t &hi,
                                       uint32_t &above, uint32_t &in_bin) {
    const uint32_t range = hi - lo;
    const int shift = range < kBins ? 0 : 32 - __builtin_clz(range) - 10;
    static_assert(kBins == 1 << 10, "range >> shift < kBins");
#pragma unroll
    for (int i = 0; i < kPer; i++)
        if (key[i] >= lo && key[i] <= hi) atomicAdd(&s.bins[(hi - key[i]) >> shift], 1u);
    __syncthreads();
    static_assert(kBinsEach == 4, "a vector of a thread's bins");
    u32x4 &bins = reinterpret_cast<u32x4 *>(s.bins)[threadIdx.x];
    const u32x4 mine = bins;
    bins = u32x4{};
    uint32_t before = above + block_before(mine.x + mine.y + mine.z + mine.w, s);
#pragma unroll
    for (int i = 0; i < kBinsEach; i++) {
        if (before < k && before + mine[i] >= k) {
            s.bin = threadIdx.x * kBinsEach + i;
            s.above = before;
            s.in_bin = mine[i];
        }
        before += mine[i];
    }
    __syncthreads();
    above = s.above;
    in_bin = s.in_bin;
    hi -= s.bin << shift;
    const uint32_t span = (1u << shift) - 1;
    lo = hi - lo > span ? hi - span : lo;
    __syncthreads();
}

// Of the workgroup's non-zero keys: a threshold t and the number `above` of
// keys > t such that the k largest are those and k - above of the keys equal to
// t.  t = 0 if there are no more than k.
template <int kPer>
__device__ uint32_t kth_key(const uint32_t (&key)[kPer], uint32_t k, PickShared &s, uint32_t &above) {
    uint32_t most = 0, least = ~0u, count = 0;
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        most = max(most, key[i]);
        if (key[i]) least = min(least, key[i]), count++;
    }
    __syncthreads();
    reinterpret_cast<u32x4 *>(s.bins)[threadIdx.x] = u32x4{};
    if (threadIdx.x == 0) s.hi = 0, s.lo = ~0u, s.count = 0;
    __syncthreads();
    atomicMax(&s.hi, most);
    atomicMin(&s.lo, least);
    atomicAdd(&s.count, count);
    __syncthreads();
    uint32_t lo = s.lo, hi = s.hi, in_bin = 0;
    above = 0;
    if (s.count <= k) return 0;
    while (lo != hi) {
        narrow<kPer>(key, k, s, lo, hi, above, in_bin);
        if (above + in_bin == k) {
            above = k;
            return lo - 1;
        }
    }
    return lo;
}

// Places for each lane's n entries in a list of *count so far: the first of them.
__device__ __forceinline__ uint32_t reserve(uint32_t *count, uint32_t n, int lane) {
    const uint32_t upto = wave_scan(n, 0u, kAdd), all = lane_value(upto, kWave - 1);
    uint32_t at = 0;
    if (all && lane == 0) at = atomicAdd(count, all);
    return lane_value(at, 0) + upto - n;
}

// The next two are for few rows, and calls, for pick_kernel's length is time in
// every row: with both inlined it took 25 us for 256 rows of 8,000 float32, 12
// without.  They take values only, as a reference to the kernel's arguments
// would have them all copied to memory, and a caller passes a barrier after
// them: the compiler may otherwise keep what it has read of LDS over the call.

// Exactly the k best tokens into s.found, whatever the row: the k groups, then
// k of their tokens, ties to the lower ones.  Groups and tokens are dealt to
// the threads in ascending order, so that a sum over the threads before this
// one is a place in that order.
template <bool kBf16, int kPer>
__device__ __attribute__((noinline)) void pick_exactly(Row<kBf16> row, const uint32_t *words, int32_t V, int32_t W, uint32_t k,
                                                       int32_t groups, const uint32_t *keys, PickShared *shared) {
    PickShared &s = *shared;
    const int tid = threadIdx.x;
    uint32_t key[kPer];
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        const int32_t l = tid * kPer + i;
        key[i] = l < groups ? keys[l] : 0;
    }
    s.found[tid] = 0;
    uint32_t above;
    uint32_t t = kth_key<kPer>(key, k, s, above);
    uint32_t n = 0;      // those above t, and, << 16, those equal to it
#pragma unroll
    for (int i = 0; i < kPer; i++) n += key[i] > t ? 1u : key[i] == t && t ? 1u << 16 : 0u;
    __syncthreads();
    uint32_t before = block_before(n, s);
    uint32_t gt = before & 0xFFFF, eq = before >> 16, quota = k - above;
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        const bool more = key[i] > t, same = key[i] == t && t;
        if (more || (same && eq < quota)) s.groups[gt + min(eq, quota)] = tid * kPer + i;
        gt += more;
        eq += same;
    }
    if (tid == kPickBlock - 1) s.n_groups = gt + min(eq, quota);
    __syncthreads();
    constexpr int kMine = kMostK * kGroup / kPickBlock;
    uint32_t mine[kMine] = {};
    int32_t v = 0;
    const uint32_t g = (uint32_t)tid / (kGroup / kMine);
    if (g < s.n_groups) {
        const int32_t at = s.groups[g] * kGroup + (tid % (kGroup / kMine)) * kMine;
        v = at - row.delta;
        const uint32_t keep = allowed_bits(words, v, kMine, V, W);
#pragma unroll
        for (int e = 0; e < kMine; e++)
            if ((keep >> e) & 1) mine[e] = key_of(load_logit<kBf16>(row.line, at + e));
    }
    t = kth_key<kMine>(mine, k, s, above);
    n = 0;
#pragma unroll
    for (int e = 0; e < kMine; e++) n += mine[e] > t ? 1u : mine[e] == t && t ? 1u << 16 : 0u;
    __syncthreads();
    before = block_before(n, s);
    gt = before & 0xFFFF, eq = before >> 16, quota = k - above;
#pragma unroll
    for (int e = 0; e < kMine; e++) {
        const bool more = mine[e] > t, same = mine[e] == t && t;
        if (more || (same && eq < quota)) s.found[gt + min(eq, quota)] = ranked(mine[e], v + e);
        gt += more;
        eq += same;
    }
    if (tid == kPickBlock - 1) s.n_found = gt + min(eq, quota);
    __syncthreads();
}

// s.found anew, where more than kMostFound of the groups' tokens have a key of
// at least lo: those from a higher threshold on, found among the tokens' keys
// themselves.  hi: the row's largest key.
template <bool kBf16>
__device__ __attribute__((noinline)) void thin_out(Row<kBf16> row, const uint32_t *words, int32_t V, uint32_t k, uint32_t lo, uint32_t hi,
                                                   PickShared *shared) {
    PickShared &s = *shared;
    const int tid = threadIdx.x, lane = tid % kWave;
    constexpr int kMine = kMostGroups * kGroup / kPickBlock;
    const int32_t tokens = (int32_t)s.n_groups * kGroup;
    uint32_t key[kMine];
    const auto id_of = [&](int i) {
        const int32_t n = i * kPickBlock + tid;
        return n < tokens ? s.groups[n / kGroup] * kGroup + n % kGroup - row.delta : -1;
    };
#pragma unroll
    for (int i = 0; i < kMine; i++) {
        const int32_t v = id_of(i);
        const bool is = v >= 0 && v < V;
        const float x = is ? load_logit<kBf16>(row.line, (int64_t)v + row.delta) : 0;
        key[i] = is && (!words || words[v >> 5] >> (v & 31) & 1) ? key_of(x) : 0;
    }
    __syncthreads();
    s.found[tid] = 0;
    if (tid == 0) s.n_found = 0;
    uint32_t above = 0, in_bin;
    do narrow<kMine>(key, k, s, lo, hi, above, in_bin);
    while (above + in_bin > kMostFound && lo != hi);
    uint32_t hits = 0;
    static_assert(kMine <= 32, "a bit per token of a thread");
#pragma unroll
    for (int i = 0; i < kMine; i++) hits |= (uint32_t)(key[i] >= lo) << i;
    uint32_t to = reserve(&s.n_found, __popc(hits), lane);
    for (; hits; hits &= hits - 1, to++) {
        const int32_t v = id_of(__ffs((int)hits) - 1);
        if (to < kMostFound) s.found[to] = ranked(key_of(load_logit<kBf16>(row.line, (int64_t)v + row.delta)), v);
    }
    __syncthreads();
}

template <bool kBf16, int kPer>
__global__ void __launch_bounds__(kPickBlock)
pick_kernel(const SampleArgs a) {
    using R = Row<kBf16>;
    __shared__ PickShared s;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int64_t b = blockIdx.x;
    const uint32_t k = (uint32_t)a.k;
    const int32_t groups = a.tiles * R::kTileGroups;
    uint32_t key[kPer];
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        const int32_t l = i * kPickBlock + tid;
        key[i] = l < groups ? a.group_keys[b * groups + l] : 0;
    }
    // what the first wavefront needs at the end is on its way from the start
    const float c = inverse_temperature(a.temperature, b);
    const bool cold = a.temperature && !(a.temperature[b] > 0);
    const int32_t top_k = a.top_k ? a.top_k[b] : 0;
    const float top_p = a.top_p ? a.top_p[b] : 1.0f, min_p = a.min_p ? a.min_p[b] : 0.0f;
    const float noise = wave == 0 && lane < a.k && a.noise ? a.noise[b * a.k + lane] : 1.0f;
    // the row's maximum and sum: tile t by thread t, and on
    float2 part = make_float2(kMinusInf, 0.0f);
    for (int32_t t = tid; t < a.tiles; t += kPickBlock) {
        const float2 p = a.parts[b * a.tiles + t];
        const float m = larger(part.x, p.x);
        if (m != kMinusInf)
            part.y = (part.x == kMinusInf ? 0.0f : part.y * exp_scaled(part.x - m, c)) +
                     (p.x == kMinusInf ? 0.0f : p.y * exp_scaled(p.x - m, c));
        part.x = m;
    }
    reinterpret_cast<u32x4 *>(s.bins)[tid] = u32x4{};
    s.found[tid] = 0;
    if (tid == 0) s.n_groups = s.n_found = 0, s.bin = kBins - 1, s.above = 0, s.in_bin = 0;
    // Every lane of a wavefront has a key that is at least the wavefront's
    // least lane maximum: kMostK keys lie at or above it.
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kPer; i++) most = max(most, key[i]);
    const uint32_t least = wave_all(most, ~0u, kMin);
    most = wave_all(most, 0u, kMax);
    const float top = wave_all(part.x, kMinusInf, kLarger);
    const float sum_here = wave_all(part.x == kMinusInf ? 0.0f : part.y * exp_scaled(part.x - top, c), 0.0f, kAdd);
    if (lane == 0) {
        s.parts[wave] = make_float2(top, sum_here);
        s.most[wave] = most;
        s.least[wave] = least;
    }
    __syncthreads();
    uint32_t lo = 1, hi = 0;
#pragma unroll
    for (int i = 0; i < kPickWaves; i++) {
        hi = max(hi, s.most[i]);
        lo = max(lo, s.least[i]);
    }
    const bool some = hi != 0;
    const uint32_t largest_key = hi;
    uint32_t above = 0, in_bin = 0;
    // One round mostly leaves little more than k groups; where the keys' range
    // crosses zero its bins are coarse.  Where a row has fewer than k, all of
    // them are taken.
    if (some) {
        do narrow<kPer>(key, k, s, lo, hi, above, in_bin);
        while (above + in_bin > kMostGroups && lo != hi);
        if (!in_bin) lo = 1;
    }
    {
        uint64_t hits = 0;
#pragma unroll
        for (int i = 0; i < kPer; i++) hits |= (uint64_t)(some && key[i] >= lo) << i;
        uint32_t to = reserve(&s.n_groups, __popcll(hits), lane);
        for (; hits; hits &= hits - 1, to++)
            if (to < kMostGroups) s.groups[to] = (__ffsll((long long)hits) - 1) * kPickBlock + tid;
    }
    __syncthreads();
    const uint32_t n_groups = s.n_groups;
    // their tokens, kMine at a time; every load is under way before the first is used
    constexpr int kMine = 8, kParts = kGroup / kMine, kTurns = kMostGroups * kParts / kPickBlock;
    const R row(a, b);
    const uint32_t *words = a.bitmask ? a.bitmask + b * a.W : nullptr;
    if (n_groups <= kMostGroups) {
        constexpr int kVecsMine = kMine / R::kPerVec;
        const __amdgpu_buffer_rsrc_t rsrc = buffer_of(row.line, (uint32_t)a.tiles * kTileBytes);
        u32x4 x[kTurns][kVecsMine];
        uint32_t keep[kTurns];
        int32_t first[kTurns];       // of the tokens, in the row
        bool ends = false;
#pragma unroll
        for (int i = 0; i < kTurns; i++) {
            const int n = i * kPickBlock + tid;
            const bool mine = (uint32_t)n / kParts < n_groups;
            const int32_t at = mine ? s.groups[n / kParts] * kGroup + n % kParts * kMine : 0;
            first[i] = mine ? at - row.delta : a.V;
            const bool whole = first[i] >= 0 && first[i] <= a.V - kMine;
            ends |= !whole && first[i] < a.V;
#pragma unroll
            for (int j = 0; j < kVecsMine; j++)
                x[i][j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, whole ? (uint32_t)at * R::kElem + 16 * j : kOffSkip, 0, 0);
            keep[i] = allowed_bits(words, first[i], kMine, a.V, a.W);
        }
        if (__ballot(ends)) {        // what reaches out of the row is read by element
#pragma unroll
            for (int i = 0; i < kTurns; i++) {
                if (first[i] >= a.V || (first[i] >= 0 && first[i] <= a.V - kMine)) continue;
                const char *from = row.line + ((int64_t)first[i] + row.delta) * R::kElem;
#pragma unroll
                for (int e = 0; e < kMine; e++) {
                    if (!((keep[i] >> e) & 1)) continue;
                    if constexpr (kBf16) x[i][0][e / 2] |= (uint32_t) reinterpret_cast<const uint16_t *>(from)[e] << (e % 2 * 16);
                    else x[i][e / 4][e % 4] = reinterpret_cast<const uint32_t *>(from)[e];
                }
            }
        }
        // a bit per token that is not below the threshold (a NaN is not)
        const float least_value = lo < 0x00800000u ? -FLT_MAX : of_key(lo);
        uint32_t hits = 0;
        static_assert(kTurns * kMine <= 32, "a bit per token of a thread");
#pragma unroll
        for (int i = 0; i < kTurns; i++) {
#pragma unroll
            for (int e = 0; e < kMine; e++) {
                const uint32_t u = kBf16 ? (e % 2 ? x[i][0][e / 2] & 0xFFFF0000u : x[i][0][e / 2] << 16) : x[i][e / 4 % kVecsMine][e % 4];
                hits |= (uint32_t)!(__builtin_bit_cast(float, u) < least_value) << (i * kMine + e);
            }
            hits &= ~(((1u << kMine) - 1) << (i * kMine)) | keep[i] << (i * kMine);
        }
        // few are: those are read again rather than picked out of registers,
        // for the code's length is time where a launch runs it once
        uint32_t to = reserve(&s.n_found, __popc(hits), lane);
        for (; hits; hits &= hits - 1, to++) {
            const int bit = __ffs((int)hits) - 1, i = bit / kMine;
            const int32_t v = (i < 2 ? i < 1 ? first[0] : first[1] : i < 3 ? first[2] : first[3]) + bit % kMine;
            static_assert(kTurns == 4, "the turns named here");
            if (to < kMostFound) s.found[to] = ranked(key_of(load_logit<kBf16>(row.line, (int64_t)v + row.delta)), v);
        }
    }
    __syncthreads();
    if (s.n_found > kMostFound) {        // fewer than k groups, or many tokens about as large as the k-th
        thin_out<kBf16>(row, words, a.V, k, lo, largest_key, &s);
        __syncthreads();
    }
    if (n_groups > kMostGroups || s.n_found > kMostFound) {        // many equal ones
        pick_exactly<kBf16, kPer>(row, words, a.V, a.W, k, groups, a.group_keys + b * groups, &s);
        __syncthreads();
    }
    // the place of every token found, by counting those before it
    const uint32_t n_found = s.n_found;
    if ((uint32_t)tid < n_found) {
        const uint64_t mine = s.found[tid];
        uint32_t rank = 0;
        constexpr int kAtOnce = 16;      // what lies behind the last one is 0
        for (uint32_t j = 0; j < n_found; j += kAtOnce) {
            uint64_t other[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; i++) other[i] = s.found[j + i];
#pragma unroll
            for (int i = 0; i < kAtOnce; i++) rank += other[i] > mine;
        }
        if (rank < k) s.best[rank] = mine;
    }
    __syncthreads();
    if (wave) return;
    // one wavefront: lane j has the j-th best
    const uint32_t live = min(n_found, k);
    const bool is = (uint32_t)lane < live;
    const uint64_t mine = is ? s.best[lane] : 0;
    const int32_t id = is ? (int32_t)~(uint32_t)mine : -1;
    const float x = of_key((uint32_t)(mine >> 32)), x0 = lane_value(x, 0);
    float sum = 0;
#pragma unroll
    for (int i = 0; i < kPickWaves; i++)
        if (s.parts[i].x != kMinusInf) sum += s.parts[i].y * exp_scaled(s.parts[i].x - x0, c);
    const float z = (x - x0) * c;
    const float logprob = is ? z - __builtin_logf(sum) : kMinusInf;
    const bool in_top = is && (top_k <= 0 || lane < top_k);
    const float weight = in_top ? exp_scaled(x - x0, c) : 0.0f;
    const float upto = wave_scan(weight, 0.0f, kAdd), all = lane_value(upto, kWave - 1);
    const bool kept = weight > 0 && (top_p >= 1 || upto - weight < top_p * all || lane == 0) && (weight >= min_p || lane == 0);
    int at = 0;
    if (a.noise && !cold && sum < INFINITY) {
        const float score = kept ? weight / noise : -1.0f;
        const float largest = wave_all(score, -1.0f, [](float p, float q) { return fmaxf(p, q); });
        const uint64_t where = __ballot(score == largest);
        if (largest >= 0 && where) at = __ffsll((long long)where) - 1;
    }
    if (lane == at) {
        a.tokens[b] = id;
        if (a.logprobs) a.logprobs[b] = logprob;
    }
    if (lane < a.k) {
        if (a.ids) a.ids[b * a.k + lane] = id;
        if (a.id_logprobs) a.id_logprobs[b * a.k + lane] = logprob;
    }
}

int32_t tiles_of(int32_t V, psc_dtype dtype) { return tiles_of_row(V, (int32_t)size_of(dtype)); }

template <bool kBf16>
void launch_sample(const SampleArgs &a, int32_t B, hipStream_t s) {
    constexpr int kWaves = kScanBlock / kWave;
    hipLaunchKernelGGL(scan_kernel<kBf16>, dim3((a.tiles + kWaves - 1) / kWaves, B), dim3(kScanBlock), 0, s, a);
    const int32_t groups = a.tiles * Row<kBf16>::kTileGroups;
    const dim3 rows(B), block(kPickBlock);
    if (groups <= kPickBlock * 4) hipLaunchKernelGGL((pick_kernel<kBf16, 4>), rows, block, 0, s, a);
    else if (groups <= kPickBlock * 10) hipLaunchKernelGGL((pick_kernel<kBf16, 10>), rows, block, 0, s, a);
    else if (groups <= kPickBlock * 20) hipLaunchKernelGGL((pick_kernel<kBf16, 20>), rows, block, 0, s, a);
    else hipLaunchKernelGGL((pick_kernel<kBf16, 64>), rows, block, 0, s, a);
}

constexpr int32_t kMostTiles = kPickBlock * 64 / Row<true>::kTileGroups;       // 2 MiB of logits a row, less a line

}  // namespace

extern "C" size_t psc_sample_workspace(int32_t B, int32_t V, psc_dtype dtype) {
    if (B <= 0 || V <= 0 || !is_dtype(dtype)) return 0;
    return (size_t)B * (size_t)tiles_of(V, dtype) * (sizeof(float2) + Row<true>::kTileGroups * sizeof(uint32_t));
}

extern "C" psc_status psc_sample(const void *logits, psc_dtype dtype, int64_t stride, int32_t B, int32_t V,
                                 const uint32_t *bitmask, const psc_sampling *sampling, int32_t k, int32_t *tokens,
                                 float *logprobs, int32_t *ids, float *id_logprobs, void *workspace,
                                 size_t workspace_bytes, void *stream) {
    const char *what = "psc_sample";
    if (psc_status st = check_rows(what, logits, dtype, stride, B, V)) return st;
    if (k < 1 || k > kMostK) return refuse(what, "k outside [1, 64]");
    if (B > 65535) return refuse(what, "B > 65535");
    if (B == 0) return PSC_OK;
    if (V == 0) return refuse(what, "an empty vocabulary");
    if (!tokens || !workspace) return refuse(what, "null pointer");
    if (tiles_of(V, dtype) > kMostTiles) return refuse(what, "rows of more than 2 MiB less 128 bytes");
    if (workspace_bytes < psc_sample_workspace(B, V, dtype) || !aligned_to(workspace, 16))
        return refuse(what, "the workspace is too small or not 16-byte aligned");
    SampleArgs a{};
    a.logits = logits;
    a.stride = stride;
    a.bitmask = bitmask;
    a.V = V;
    a.W = (int32_t)(((int64_t)V + 31) / 32);
    a.k = k;
    a.tiles = tiles_of(V, dtype);
    if (sampling) {
        a.temperature = sampling->temperature;
        a.top_k = sampling->top_k;
        a.top_p = sampling->top_p;
        a.min_p = sampling->min_p;
        a.noise = sampling->noise;
    }
    a.parts = static_cast<float2 *>(workspace);
    a.group_keys = reinterpret_cast<uint32_t *>(a.parts + (size_t)B * a.tiles);
    a.tokens = tokens;
    a.logprobs = logprobs;
    a.ids = ids;
    a.id_logprobs = id_logprobs;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (dtype == PSC_BF16) launch_sample<true>(a, B, s);
    else launch_sample<false>(a, B, s);
    return launched_op(what);
}
