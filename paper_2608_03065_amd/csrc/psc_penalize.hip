// What a request changes in its logits (psc_penalize): penalties of repeated
// tokens, biases of single tokens, and the grammar mask, in place; and the
// token history that the penalties read (psc_append_tokens).
#include "psc_ops.hpp"

#include <algorithm>

using namespace psc;

namespace {

constexpr int kBlock = 256;

// ---------------------------------------------------------------- mask

// One workgroup per row and kMaskTokens tokens: forbidden logits become -inf;
// nothing is read of the logits.
constexpr int kMaskTokens = 8192;

template <bool kBf16>
__global__ void __launch_bounds__(kBlock)
forbid_kernel(void *__restrict__ logits, int64_t stride, int32_t V, const uint32_t *__restrict__ bitmask, int32_t W) {
    using T = typename Logit<kBf16>::type;
    const int64_t b = blockIdx.y;
    T *row = static_cast<T *>(logits) + b * stride;
    const uint32_t *words = bitmask + b * W;
    const int32_t end = (int32_t)min((int64_t)V, ((int64_t)blockIdx.x + 1) * kMaskTokens);
    for (int32_t v = blockIdx.x * kMaskTokens + threadIdx.x; v < end; v += kBlock)
        if (!((words[v >> 5] >> (v & 31)) & 1)) store_logit<kBf16>(row, v, kMinusInf);
}

// ---------------------------------------------------------------- penalties and biases

constexpr int kPenBlock = 1024;
constexpr int kSlice = 32768;          // tokens of the vocabulary per workgroup, a counter each
constexpr uint32_t kBiased = 0x80000000u;
constexpr int32_t kMostBiases = kPenBlock;

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

// Only logits of tokens that the history or the biases name change, so only
// those are read and written.  One workgroup per row and slice of the
// vocabulary: it counts the history's tokens that lie in its slice in LDS and
// then goes through the history once more; the first occurrence that takes a
// token's counter away changes its logit.  A counter is cleared only where a
// token stands, so that a short history costs little.
// counter: 2 * occurrences after the prompt + (occurs in the prompt)
template <bool kBf16>
__global__ void __launch_bounds__(kPenBlock)
penalize_kernel(const PenArgs a) {
    __shared__ uint32_t counters[kSlice];
    const int64_t b = blockIdx.y;
    const int32_t v0 = blockIdx.x * kSlice, size = min(kSlice, a.V - v0);
    const int32_t n = a.lens ? min(max(a.lens[b], 0), a.cap) : 0;
    const int32_t prompt = a.prompt_lens ? min(max(a.prompt_lens[b], 0), n) : 0;
    const int32_t *history = a.history + b * a.cap;
    const float r = a.repetition ? a.repetition[b] : 1.0f, presence = a.presence ? a.presence[b] : 0.0f,
                frequency = a.frequency ? a.frequency[b] : 0.0f;
    using T = typename Logit<kBf16>::type;
    T *row = static_cast<T *>(a.logits) + b * a.stride;
    const uint32_t *words = a.bitmask ? a.bitmask + b * a.W : nullptr;
    // the slice's counter of token t, or a number past it
    const auto place = [&](int32_t t) { return (uint32_t)t - (uint32_t)v0; };
    const auto change = [&](uint32_t at, uint32_t count, float bias) {
        const int32_t v = v0 + (int32_t)at;
        if (words && !((words[v >> 5] >> (v & 31)) & 1)) return;     // forbidden
        const float x = load_logit<kBf16>(row, v);
        if (x == kMinusInf) return;
        float y = x;
        if (count) y = y > 0 ? y / r : y * r;
        if (count >= 2) y = y - (float)(count >> 1) * frequency - presence;
        store_logit<kBf16>(row, v, y + bias);
    };
    uint32_t bias_at = ~0u;
    float bias = 0;
    if ((int)threadIdx.x < a.n_bias) {
        bias_at = place(a.bias_ids[b * a.n_bias + threadIdx.x]);
        bias = a.bias_values[b * a.n_bias + threadIdx.x];
    }
    const bool has_bias = bias_at < (uint32_t)size;
    for (int32_t i = threadIdx.x; i < n; i += kPenBlock) {
        const uint32_t at = place(history[i]);
        if (at < (uint32_t)size) counters[at] = 0;
    }
    if (has_bias) counters[bias_at] = 0;
    __syncthreads();
    for (int32_t i = threadIdx.x; i < n; i += kPenBlock) {
        const uint32_t at = place(history[i]);
        if (at >= (uint32_t)size) continue;
        if (i < prompt) atomicOr(&counters[at], 1u);
        else atomicAdd(&counters[at], 2u);
    }
    __syncthreads();
    if (a.n_bias) {
        // of a token's entries the last one counts: it changes the logit, with the token's count
        const uint32_t count = has_bias ? counters[bias_at] : 0;
        __syncthreads();
        if (has_bias) atomicMax(&counters[bias_at], kBiased | threadIdx.x);
        __syncthreads();
        if (has_bias && counters[bias_at] == (kBiased | threadIdx.x)) change(bias_at, count, bias);
        __syncthreads();
    }
    for (int32_t i = threadIdx.x; i < n; i += kPenBlock) {
        const uint32_t at = place(history[i]);
        if (at >= (uint32_t)size) continue;
        const uint32_t count = atomicExch(&counters[at], 0u);
        if (count && !(count & kBiased)) change(at, count, 0.0f);
    }
}

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

template <bool kBf16>
void launch_penalize(const PenArgs &a, int32_t B, hipStream_t s) {
    for (int32_t b = 0; b < B; b += kMostRows) {
        const int32_t rows = std::min(kMostRows, B - b);
        PenArgs p = a;
        p.logits = static_cast<char *>(a.logits) + b * a.stride * (kBf16 ? 2 : 4);
        if (a.bitmask) p.bitmask = a.bitmask + (int64_t)b * a.W;
        if (a.bitmask)
            hipLaunchKernelGGL(forbid_kernel<kBf16>, dim3((a.V + kMaskTokens - 1) / kMaskTokens, rows), dim3(kBlock), 0, s,
                               p.logits, a.stride, a.V, p.bitmask, a.W);
        if (!a.lens && !a.n_bias) continue;
        if (a.lens) p.history = a.history + (int64_t)b * a.cap, p.lens = a.lens + b;
        if (a.prompt_lens) p.prompt_lens = a.prompt_lens + b;
        if (a.repetition) p.repetition = a.repetition + b;
        if (a.presence) p.presence = a.presence + b;
        if (a.frequency) p.frequency = a.frequency + b;
        if (a.n_bias) p.bias_ids = a.bias_ids + (int64_t)b * a.n_bias, p.bias_values = a.bias_values + (int64_t)b * a.n_bias;
        hipLaunchKernelGGL(penalize_kernel<kBf16>, dim3((a.V + kSlice - 1) / kSlice, rows), dim3(kPenBlock), 0, s, p);
    }
}

}  // namespace

extern "C" psc_status psc_penalize(void *logits, psc_dtype dtype, int64_t stride, int32_t B, int32_t V,
                                   const psc_penalties *penalties, const uint32_t *bitmask, void *stream) {
    const char *what = "psc_penalize";
    if (psc_status st = check_rows(what, logits, dtype, stride, B, V)) return st;
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
