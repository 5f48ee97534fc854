// From logits to a token (psc_sample): the log of the sum of the allowed
// tokens' exponentials, the k best tokens with their log-probabilities, and
// one token drawn from these under temperature, top-k, top-p and min-p.
//
// Two kernels.  The scan reads every allowed logit once and leaves, per 4 KB of
// a row, its maximum and the sum of exponentials below it, and per 128-byte
// line the line's maximum.  The k best tokens lie in the k lines with the
// largest maxima (ties to the lower line): any token outside them is preceded
// by those lines' k maxima, which are larger, or equal and of lower id.  So the
// second kernel, a workgroup per row, selects k lines, reads them again,
// selects k of their tokens, orders them and draws.
#include "psc_ops.hpp"

#include <algorithm>
#include <cfloat>

using namespace psc;

namespace {

constexpr int kScanBlock = 256;
constexpr int kTileBytes = 4096;
constexpr int kLineBytes = 128;
constexpr int kTileLines = kTileBytes / kLineBytes;
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
    uint32_t *line_keys;         // [B][tiles * kTileLines]
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

template <int kCtrl>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl, 0xF, 0xF, false));
}

// Row b: `line` is the 128-byte line that holds its first element, the delta
// elements before it there are not the row's.
template <bool kBf16>
struct Row {
    static constexpr int kElem = kBf16 ? 2 : 4, kPerVec = 16 / kElem;
    const char *line;
    int32_t delta;
    __device__ __forceinline__ Row(const SampleArgs &a, int64_t b) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(a.logits) + (uintptr_t)(b * a.stride) * kElem;
        line = reinterpret_cast<const char *>(at & ~(uintptr_t)(kLineBytes - 1));
        delta = (int32_t)(at & (kLineBytes - 1)) / kElem;
    }
};

// Bits of the `count` tokens from v on (v may be negative): 1 where a token
// is in the vocabulary and allowed.
__device__ __forceinline__ uint32_t allowed_bits(const uint32_t *__restrict__ words, int64_t v, int count, int32_t V, int32_t W) {
    uint32_t in = (1u << count) - 1;
    if (v < 0) in = v > -count ? in & ~0u << -v : 0;
    if (v + count > V) in = v < V ? in & ((1u << (V - v)) - 1) : 0;
    if (!words || !in) return in;
    const int64_t w = v >> 5;
    const int shift = (int)(v & 31);
    const uint32_t lo = w >= 0 && w < W ? words[w] : 0, hi = shift + count > 32 && w + 1 >= 0 && w + 1 < W ? words[w + 1] : 0;
    return __builtin_amdgcn_alignbit(hi, lo, shift) & in;
}

template <bool kBf16>
__global__ void __launch_bounds__(kScanBlock)
scan_kernel(const SampleArgs a) {
    using R = Row<kBf16>;
    constexpr uint32_t kAll = (1u << R::kPerVec) - 1;
    const int lane = threadIdx.x % kWave;
    const int64_t b = blockIdx.y;
    const int32_t t = blockIdx.x * (kScanBlock / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (t >= a.tiles) return;
    const R row(a, b);
    const char *tile = row.line + (int64_t)t * kTileBytes;
    const uint32_t *words = a.bitmask ? a.bitmask + b * a.W : nullptr;
    const float c = inverse_temperature(a.temperature, b);
    const __amdgpu_buffer_rsrc_t rsrc = buffer_of(tile, kTileBytes);
    uint32_t keep[kVecs];
    u32x4 x[kVecs];
    bool edge = false;
#pragma unroll
    for (int j = 0; j < kVecs; j++) {
        const int at = (j * kWave + lane) * R::kPerVec;
        const int64_t v = (int64_t)t * (kTileBytes / R::kElem) + at - row.delta;
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
            const int64_t v = (int64_t)t * (kTileBytes / R::kElem) + at - row.delta;
            if (!keep[j] || (v >= 0 && v + R::kPerVec <= a.V)) continue;
#pragma unroll
            for (int e = 0; e < R::kPerVec; e++) {
                if (!((keep[j] >> e) & 1)) continue;
                if constexpr (kBf16) x[j][e / 2] |= (uint32_t) reinterpret_cast<const uint16_t *>(tile)[at + e] << (e % 2 * 16);
                else x[j][e] = reinterpret_cast<const uint32_t *>(tile)[at + e];
            }
        }
    }
    const auto value = [&](int j, int e) {
        const uint32_t u = kBf16 ? (e % 2 ? x[j][e / 2] & 0xFFFF0000u : x[j][e / 2] << 16) : x[j][e];
        return (keep[j] >> e) & 1 ? __builtin_bit_cast(float, u) : kMinusInf;
    };
    float most = kMinusInf;
    uint32_t *keys = a.line_keys + (b * a.tiles + t) * kTileLines;
#pragma unroll
    for (int j = 0; j < kVecs; j++) {
        float m = kMinusInf;
#pragma unroll
        for (int e = 0; e < R::kPerVec; e++) m = larger(m, value(j, e));
        // over the 8 lanes that hold a line
        m = larger(m, dpp<0xB1>(m));     // quad_perm [1,0,3,2]
        m = larger(m, dpp<0x4E>(m));     // quad_perm [2,3,0,1]
        m = larger(m, dpp<0x141>(m));    // row_half_mirror
        if (lane % 8 == 0) keys[j * 8 + lane / 8] = key_of(m);
        most = larger(most, m);
    }
#pragma unroll
    for (int o = 8; o < kWave; o *= 2) most = larger(most, __shfl_xor(most, o, kWave));
    float sum = 0;
    if (most > kMinusInf || most != most) {
#pragma unroll
        for (int j = 0; j < kVecs; j++)
#pragma unroll
            for (int e = 0; e < R::kPerVec; e++) sum += exp_scaled(value(j, e) - most, c);
    }
#pragma unroll
    for (int o = 1; o < kWave; o *= 2) sum += __shfl_xor(sum, o, kWave);
    if (lane == 0) a.parts[b * a.tiles + t] = make_float2(most, sum);
}

// ---------------------------------------------------------------- selection

constexpr int kPickBlock = 1024;
constexpr int kPickWaves = kPickBlock / kWave;
constexpr int kBins = kPickBlock;

struct PickShared {
    uint32_t bins[kBins];
    uint32_t waves[kPickWaves];
    uint32_t least, most, bin, above, in_bin;
    int32_t lines[kMostK];
    uint32_t keys[kMostK];
    int32_t ids[kMostK];
    float2 part;
};

__device__ __forceinline__ uint32_t wave_inclusive(uint32_t v, int lane) {
#pragma unroll
    for (int o = 1; o < kWave; o *= 2) {
        const uint32_t u = __shfl_up(v, o, kWave);
        if (lane >= o) v += u;
    }
    return v;
}

// The sum of v over the threads before this one.  Every thread calls it.
__device__ __forceinline__ uint32_t block_before(uint32_t v, PickShared &s) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const uint32_t upto = wave_inclusive(v, lane);
    __syncthreads();
    if (lane == kWave - 1) s.waves[wave] = upto;
    __syncthreads();
    uint32_t before = upto - v;
    for (int i = 0; i < wave; i++) before += s.waves[i];
    return before;
}

// Of the workgroup's non-zero keys (n of them per thread): a threshold t and
// the number `above` of keys > t such that the k largest are those above t and
// k - above of those equal to t (or all of them, if there are fewer than k:
// t = 0).  Histograms of the keys between two bounds, which close in on the
// k-th largest key by a factor of kBins a round.
template <int kPer>
__device__ __forceinline__ uint32_t kth_key(const uint32_t (&key)[kPer], uint32_t k, PickShared &s, uint32_t &above) {
    uint32_t lo = 1, hi = 0;
    uint32_t count = 0;
    {
        uint32_t most = 0, least = ~0u;
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            most = max(most, key[i]);
            if (key[i]) least = min(least, key[i]), count++;
        }
        if (threadIdx.x == 0) s.most = 0, s.least = ~0u, s.in_bin = 0;
        __syncthreads();
#pragma unroll
        for (int o = 1; o < kWave; o *= 2) {
            most = max(most, (uint32_t)__shfl_xor((int)most, o, kWave));
            least = min(least, (uint32_t)__shfl_xor((int)least, o, kWave));
            count += __shfl_xor(count, o, kWave);
        }
        if (threadIdx.x % kWave == 0 && count) {
            atomicMax(&s.most, most);
            atomicMin(&s.least, least);
            atomicAdd(&s.in_bin, count);
        }
        __syncthreads();
        lo = s.least;
        hi = s.most;
        count = s.in_bin;
    }
    above = 0;
    if (count <= k) return 0;
    // the k - above largest keys in [lo, hi] are wanted, of more than there are
    for (;;) {
        if (lo == hi) return lo;
        const uint32_t range = hi - lo;
        int shift = 0;
        while ((range >> shift) >= kBins) shift++;
        __syncthreads();
        s.bins[threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPer; i++)
            if (key[i] >= lo && key[i] <= hi) atomicAdd(&s.bins[(hi - key[i]) >> shift], 1u);
        __syncthreads();
        const uint32_t mine = s.bins[threadIdx.x];
        const uint32_t before = block_before(mine, s);
        if (above + before < k && above + before + mine >= k) {
            s.bin = threadIdx.x;
            s.above = above + before;
            s.in_bin = mine;
        }
        __syncthreads();
        above = s.above;
        const uint32_t in_bin = s.in_bin, bin = s.bin;
        const uint32_t top = hi - (bin << shift);
        const uint32_t span = (1u << shift) - 1;
        lo = max(lo, top - min(span, top));
        hi = top;
        if (above + in_bin == k) {      // the whole bin is wanted
            above = k;
            return lo - 1;
        }
    }
}

template <bool kBf16, int kPer>
__global__ void __launch_bounds__(kPickBlock)
pick_kernel(const SampleArgs a) {
    using R = Row<kBf16>;
    __shared__ PickShared s;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int64_t b = blockIdx.x;
    const float c = inverse_temperature(a.temperature, b);
    const int32_t lines = a.tiles * kTileLines;
    // the row's maximum and sum
    float most = kMinusInf, sum = 0;
    for (int32_t t = tid; t < a.tiles; t += kPickBlock) {
        const float2 p = a.parts[b * a.tiles + t];
        const float m = larger(most, p.x);
        if (m > kMinusInf || m != m) sum = sum * (most > kMinusInf ? exp_scaled(most - m, c) : 0.0f) + (p.x > kMinusInf || p.x != p.x ? p.y * exp_scaled(p.x - m, c) : 0.0f);
        most = m;
    }
    // in a fixed order, so that the same row gives the same sum
    __shared__ float2 s_parts[kPickWaves];
#pragma unroll
    for (int o = 1; o < kWave; o *= 2) {
        const float m2 = __shfl_xor(most, o, kWave), s2 = __shfl_xor(sum, o, kWave);
        const float m = larger(most, m2);
        const float f = most > kMinusInf || most != most ? exp_scaled(most - m, c) * sum : 0.0f;
        const float g = m2 > kMinusInf || m2 != m2 ? exp_scaled(m2 - m, c) * s2 : 0.0f;
        sum = f + g;
        most = m;
    }
    if (lane == 0) s_parts[wave] = make_float2(most, sum);
    __syncthreads();
    most = kMinusInf;
    for (int i = 0; i < kPickWaves; i++) most = larger(most, s_parts[i].x);
    sum = 0;
    for (int i = 0; i < kPickWaves; i++)
        if (s_parts[i].x > kMinusInf || s_parts[i].x != s_parts[i].x) sum += s_parts[i].y * exp_scaled(s_parts[i].x - most, c);

    // the k lines, in ascending order
    const uint32_t *line_keys = a.line_keys + b * lines;
    uint32_t key[kPer];
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        const int32_t l = tid * kPer + i;
        key[i] = l < lines ? line_keys[l] : 0;
    }
    const uint32_t k = (uint32_t)a.k;
    uint32_t above;
    uint32_t t = kth_key<kPer>(key, k, s, above);
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < kPer; i++) n += key[i] > t ? 1u : key[i] == t && t ? 1u << 16 : 0u;
    uint32_t before = block_before(n, s);
    uint32_t n_lines;
    {
        uint32_t gt = before & 0xFFFF, eq = before >> 16;
        const uint32_t quota = k - above;
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            const bool more = key[i] > t, same = key[i] == t && t;
            if (more || (same && eq < quota)) s.lines[gt + min(eq, quota)] = tid * kPer + i;
            gt += more;
            eq += same;
        }
        if (tid == kPickBlock - 1) s.in_bin = gt + min(eq, quota);
        __syncthreads();
        n_lines = s.in_bin;
    }
    // their tokens: 8 bytes a thread, 16 threads a line
    constexpr int kMine = 8 / R::kElem;
    uint32_t mine[kMine] = {};
    int64_t v = 0;
    if ((uint32_t)tid / 16 < n_lines) {
        const R row(a, b);
        const int64_t at = (int64_t)s.lines[tid / 16] * (kLineBytes / R::kElem) + (tid % 16) * kMine;
        v = at - row.delta;
        const uint32_t keep = allowed_bits(a.bitmask ? a.bitmask + b * a.W : nullptr, v, kMine, a.V, a.W);
        const char *from = row.line + at * R::kElem;
#pragma unroll
        for (int e = 0; e < kMine; e++)
            if ((keep >> e) & 1) mine[e] = key_of(load_logit<kBf16>(from, e));
    }
    t = kth_key<kMine>(mine, k, s, above);
    n = 0;
#pragma unroll
    for (int e = 0; e < kMine; e++) n += mine[e] > t ? 1u : mine[e] == t && t ? 1u << 16 : 0u;
    before = block_before(n, s);
    {
        uint32_t gt = before & 0xFFFF, eq = before >> 16;
        const uint32_t quota = k - above;
#pragma unroll
        for (int e = 0; e < kMine; e++) {
            const bool more = mine[e] > t, same = mine[e] == t && t;
            if (more || (same && eq < quota)) {
                s.keys[gt + min(eq, quota)] = mine[e];
                s.ids[gt + min(eq, quota)] = (int32_t)(v + e);
            }
            gt += more;
            eq += same;
        }
        if (tid == kPickBlock - 1) s.in_bin = gt + min(eq, quota);
        __syncthreads();
    }
    if (wave) return;
    // one wavefront: lane j takes the j-th best
    const uint32_t live = s.in_bin;
    const uint32_t my_key = (uint32_t)lane < live ? s.keys[lane] : 0;
    const int32_t my_id = (uint32_t)lane < live ? s.ids[lane] : -1;
    int rank = 0;
    for (int j = 0; j < (int)live; j++) {
        const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)my_key, j);
        rank += other > my_key || (other == my_key && j < lane);
    }
    // the lanes past the live ones keep their places behind them
    if ((uint32_t)lane >= live) rank = lane;
    const uint32_t best_key = (uint32_t)__builtin_amdgcn_ds_permute(rank * 4, (int)my_key);
    const int32_t id = __builtin_amdgcn_ds_permute(rank * 4, my_id);
    const bool is = (uint32_t)lane < live;
    const float x = of_key(best_key), x0 = __shfl(x, 0, kWave);
    const float z = is ? (x - x0) * c : kMinusInf;
    const float logprob = is ? z - __builtin_logf(sum) : kMinusInf;
    const int32_t top_k = a.top_k ? a.top_k[b] : 0;
    const bool in_top = is && (top_k <= 0 || lane < top_k);
    const float weight = in_top ? exp_scaled(x - x0, c) : 0.0f;
    float upto = weight;
#pragma unroll
    for (int o = 1; o < kWave; o *= 2) {
        const float u = __shfl_up(upto, o, kWave);
        if (lane >= o) upto += u;
    }
    const float all = __shfl(upto, kWave - 1, kWave);
    const float top_p = a.top_p ? a.top_p[b] : 1.0f, min_p = a.min_p ? a.min_p[b] : 0.0f;
    const bool kept = weight > 0 && (top_p >= 1 || upto - weight < top_p * all || lane == 0) && (weight >= min_p || lane == 0);
    const bool greedy = !a.noise || (a.temperature && !(a.temperature[b] > 0)) || !(sum < INFINITY);
    float score = kept && !greedy ? weight / a.noise[b * a.k + lane] : -1.0f;
    int at = lane;
#pragma unroll
    for (int o = 1; o < kWave; o *= 2) {
        const float other = __shfl_xor(score, o, kWave);
        const int other_at = __shfl_xor(at, o, kWave);
        if (other > score || (other == score && other_at < at)) score = other, at = other_at;
    }
    if (greedy || !(score >= 0)) at = 0;
    if (lane == at) {
        a.tokens[b] = id;
        if (a.logprobs) a.logprobs[b] = logprob;
    }
    if (lane < a.k) {
        if (a.ids) a.ids[b * a.k + lane] = id;
        if (a.id_logprobs) a.id_logprobs[b * a.k + lane] = logprob;
    }
}

int32_t tiles_of(int32_t V, psc_dtype dtype) {
    return (int32_t)(((int64_t)V * size_of(dtype) + kLineBytes - 1 + kTileBytes - 1) / kTileBytes);
}

template <bool kBf16>
void launch_sample(const SampleArgs &a, int32_t B, hipStream_t s) {
    constexpr int kWaves = kScanBlock / kWave;
    hipLaunchKernelGGL(scan_kernel<kBf16>, dim3((a.tiles + kWaves - 1) / kWaves, B), dim3(kScanBlock), 0, s, a);
    const int32_t lines = a.tiles * kTileLines;
    if (lines <= kPickBlock * 2) hipLaunchKernelGGL((pick_kernel<kBf16, 2>), dim3(B), dim3(kPickBlock), 0, s, a);
    else if (lines <= kPickBlock * 5) hipLaunchKernelGGL((pick_kernel<kBf16, 5>), dim3(B), dim3(kPickBlock), 0, s, a);
    else hipLaunchKernelGGL((pick_kernel<kBf16, 16>), dim3(B), dim3(kPickBlock), 0, s, a);
}

constexpr int32_t kMostTiles = kPickBlock * 16 / kTileLines;       // 2 MiB of logits a row

}  // namespace

extern "C" size_t psc_sample_workspace(int32_t B, int32_t V, psc_dtype dtype) {
    if (B <= 0 || V <= 0 || !is_dtype(dtype)) return 0;
    return (size_t)B * (size_t)tiles_of(V, dtype) * (sizeof(float2) + kTileLines * sizeof(uint32_t));
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
    if (tiles_of(V, dtype) > kMostTiles) return refuse(what, "rows of more than 2 MiB");
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
    a.line_keys = reinterpret_cast<uint32_t *>(a.parts + (size_t)B * a.tiles);
    a.tokens = tokens;
    a.logprobs = logprobs;
    a.ids = ids;
    a.id_logprobs = id_logprobs;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (dtype == PSC_BF16) launch_sample<true>(a, B, s);
    else launch_sample<false>(a, B, s);
    return launched_op(what);
}
