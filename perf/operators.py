"""Performance cases of the operators around a decoding step's logits: the projection that makes them, what a request
changes in them, and the token that is drawn from them.

  head      hidden states -> logits: states quantised to 8 bits with a scale per sequence, times 8-bit weights with a scale
            per token of the vocabulary, plus a bias per token, forbidden tokens set to -inf
  penalize  penalties of repeated tokens, biases of single tokens and the grammar mask, in place
  sample    log-probabilities over the allowed tokens, the k best of them, and one token drawn from these under
            a temperature, top-k, top-p and min-p

Vocabulary sizes are those of common tokenizers (32,000, 128,256, 151,665, 151,936, 262,144, 262,145), two of them odd.
Hidden sizes are powers of two and, among the drawn cases, any number.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
#: No drawn case is larger than the largest listed one of its operator in any of these.
MOST_PRODUCTS = 2048 * 128256 * 4096
MOST_WEIGHTS = 151936 * 4096
MOST_HEAD_LOGITS = 2048 * 128256
MOST_LOGITS = 256 * 262144 * 2        # bytes of logits that a penalize or sample case holds
MOST_HISTORY = 256 * 16384            # tokens of history
KINDS = ("none", "mixed", "few")      # no mask; rows of every kind; rows that allow a few tokens each
FEW = 40


# ---------------------------------------------------------------- cases

def head(B, D, V, dtype="bf16", mask="none", bias=False, name=None):
    c = {"op": "head", "B": B, "D": D, "V": V, "dtype": dtype, "mask": mask, "bias": bias}
    return dict(c, name=name) if name else c


def penalize(B, V, cap, biases, dtype="bf16", mask="none", name=None):
    c = {"op": "penalize", "B": B, "V": V, "cap": cap, "biases": biases, "dtype": dtype, "mask": mask}
    return dict(c, name=name) if name else c


def sample(B, V, k, dtype="bf16", mask="none", name=None):
    c = {"op": "sample", "B": B, "V": V, "k": k, "dtype": dtype, "mask": mask}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's stream on a small model: the weights are read for a single row
        head(1, 2048, 32000, "f32", name="head_single"),
        # function calling, every stream inside a fixed key or an enumeration: few tokens are needed at all
        head(8, 4096, 128256, mask="few", name="head_schema_8"),
        # a server's batch on an unpadded vocabulary, the streams in all kinds of grammar states
        head(64, 2048, 151665, mask="mixed", bias=True, name="head_odd_64"),
        # a large decoding batch: products and weights weigh the same
        head(256, 4096, 151936, name="head_256"),
        # scores of every position of a prompt: the largest product
        head(2048, 4096, 128256, name="head_prompt_2048"),
        # one stream with the text of a short chat
        penalize(1, 32000, 512, 0, "f32", name="penalize_single"),
        # function calling with biased tokens under grammar masks
        penalize(64, 151936, 4096, 32, mask="mixed", name="penalize_64"),
        # long documents on an unpadded vocabulary, the largest histories
        penalize(256, 151665, 16384, 300, mask="mixed", name="penalize_long_odd_256"),
        # one user's stream
        sample(1, 32000, 20, "f32", name="sample_single"),
        # function calling under strict masks
        sample(64, 151936, 50, mask="few", name="sample_schema_64"),
        # fp32 logits of an unpadded vocabulary under masks of every kind
        sample(96, 262145, 64, "f32", "mixed", name="sample_odd_96"),
        # a large batch without a grammar
        sample(512, 128256, 64, name="sample_512"),
    ]


def spread(rng, low, high):
    return int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))


def draw(rng):
    op = rng.choice(("head", "penalize", "sample"))
    dtype, mask = rng.choice(("bf16", "f32")), rng.choice(KINDS)
    V = spread(rng, 513, 262145)
    if rng.random() < 0.5:
        V = max(544, V // 32 * 32)
    V += V == 3072
    if op == "head":
        D = spread(rng, 64, 8192)
        if rng.random() < 0.6:
            D = D // 64 * 64
        D = min(D, MOST_WEIGHTS // V)
        D += D == 3072
        most = min(2048, MOST_PRODUCTS // (V * D), MOST_HEAD_LOGITS // V // (1 if dtype == "bf16" else 2))
        return head(spread(rng, 1, most), D, V, dtype, mask, rng.random() < 0.4)
    most = min(1024, MOST_LOGITS // (V * DTYPES[dtype].itemsize))
    B = spread(rng, 1, most)
    if op == "penalize":
        cap = min(spread(rng, 16, 32768), MOST_HISTORY // B)
        cap += cap == 3072
        return penalize(B, V, cap, rng.choice((0, 0, 1, spread(rng, 1, 300))), dtype, mask)
    return sample(B, V, rng.choice((1, 20, 64, rng.randint(1, 64))), dtype, mask)


# ---------------------------------------------------------------- inputs

def bitmask_of(c, g):
    """int32 [B, ceil(V / 32)], bit v & 31 of word v >> 5 set where token v is allowed.  Rows of few tokens (inside a key
    of a schema), of some (an expression is expected), of most (inside a string), and, where the kinds are mixed, now and
    then of none (a stream that is done)."""
    if c["mask"] == "none":
        return None
    B, V, W = c["B"], c["V"], (c["V"] + 31) // 32
    few = torch.rand(B, generator=g, device=DEVICE) * (FEW / V)
    share = few
    if c["mask"] == "mixed":
        pick = torch.rand(B, generator=g, device=DEVICE)
        share = torch.where(pick < 0.3, few, torch.where(pick < 0.6, 0.04, torch.where(pick < 0.97, 0.96, 0.0)))
    out = torch.empty(B, W, dtype=torch.int32, device=DEVICE)
    weights = torch.ones(32, dtype=torch.int64, device=DEVICE) << torch.arange(32, device=DEVICE)
    for at in range(0, B, 128):
        part = share[at:at + 128, None]
        bits = torch.zeros(part.shape[0], W * 32, dtype=torch.bool, device=DEVICE)
        bits[:, :V] = torch.rand(part.shape[0], V, generator=g, device=DEVICE) < part
        words = (bits.view(part.shape[0], W, 32) * weights).sum(-1)
        out[at:at + 128] = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
    return out


def logits_of(c, g):
    """Most logits in a bell around zero, and in each row some tens of tokens that the model favours."""
    x = torch.randn(c["B"], c["V"], generator=g, device=DEVICE).mul_(2)
    at = torch.randint(0, c["V"], (c["B"], 40), generator=g, device=DEVICE)
    x.scatter_reduce_(1, at, 12 + 3 * torch.randn(c["B"], 40, generator=g, device=DEVICE), "amax")
    return x.to(DTYPES[c["dtype"]])


def uniform(c, g, low, high):
    return low + (high - low) * torch.rand(c["B"], generator=g, device=DEVICE)


def prepare(c, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)
    B, V = c["B"], c["V"]
    s = {"op": c["op"], "V": V, "bitmask": bitmask_of(c, g)}
    if c["op"] == "head":
        D, stride = c["D"], (c["D"] + 15) // 16 * 16       # a row of weights starts at 16 bytes
        # hidden states have a few channels far larger than the others
        x = torch.randn(B, D, generator=g, device=DEVICE)
        x[:, torch.randint(0, D, (max(1, D // 256),), generator=g, device=DEVICE)] *= 8
        s["x"] = x.to(torch.bfloat16)
        w = torch.randint(-63, 64, (V, stride), generator=g, device=DEVICE, dtype=torch.int8)
        w += torch.randint(-63, 64, (V, stride), generator=g, device=DEVICE, dtype=torch.int8)
        s["w"] = w[:, :D]
        s["w_scales"] = (0.5 + torch.rand(V, generator=g, device=DEVICE)) / (40 * math.sqrt(D))
        s["bias"] = torch.randn(V, generator=g, device=DEVICE) if c["bias"] else None
        s["dtype"] = DTYPES[c["dtype"]]
        return s
    s["logits"] = logits_of(c, g)
    if c["op"] == "penalize":
        # text repeats itself: the tokens' frequencies fall off as a power of their rank
        rank = torch.rand(B, c["cap"], generator=g, device=DEVICE).pow_(3).mul_(V - 1).to(torch.int64)
        s["history"] = ((rank * 7919 + 11) % V).to(torch.int32)
        s["lens"] = uniform(c, g, 0, c["cap"] + 1).to(torch.int32).clamp_(max=c["cap"])
        s["prompt_lens"] = (s["lens"] * torch.rand(B, generator=g, device=DEVICE)).to(torch.int32)
        s["repetition"], s["presence"] = uniform(c, g, 0.9, 1.5), uniform(c, g, -0.5, 1.5)
        s["frequency"] = uniform(c, g, 0, 0.5)
        s["bias_ids"] = s["bias_values"] = None
        if c["biases"]:
            s["bias_ids"] = torch.randint(-1, V, (B, c["biases"]), generator=g, device=DEVICE, dtype=torch.int32)
            s["bias_values"] = 3 * torch.randn(B, c["biases"], generator=g, device=DEVICE)
        return s
    s["k"] = c["k"]
    s["temperature"] = uniform(c, g, 0.5, 1.5)
    s["temperature"][uniform(c, g, 0, 1) < 0.1] = 0         # greedy streams
    s["top_k"] = torch.randint(1, c["k"] + 1, (B,), generator=g, device=DEVICE, dtype=torch.int32)
    s["top_p"] = uniform(c, g, 0.7, 1.05)
    s["min_p"] = uniform(c, g, 0, 0.1)
    s["noise"] = torch.empty(B, c["k"], device=DEVICE).exponential_(generator=g)
    return s


# ---------------------------------------------------------------- the plain forms

def allowed(s):
    """The mask as booleans [B, V]."""
    words = s["bitmask"]
    bits = (words[:, :, None] >> torch.arange(32, dtype=torch.int32, device=words.device)) & 1
    return bits.reshape(words.shape[0], -1)[:, :s["V"]].bool()


def plain_head(s):
    x = s["x"].float()
    scales = x.abs().amax(1, keepdim=True)
    scales = scales / torch.full_like(scales, 127)      # by a plain 127 torch would multiply with its reciprocal
    q = torch.where(scales > 0, torch.round(x / scales), 0)
    y = (q @ s["w"].float().T) * scales * s["w_scales"]
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["bitmask"] is not None:
        y = y.masked_fill(~allowed(s), -math.inf)
    return y.to(s["dtype"])


def plain_penalize(s):
    x = s["logits"].float()
    places = torch.arange(s["history"].shape[1], device=x.device)
    said = places < s["lens"][:, None]
    answered = said & (places >= s["prompt_lens"][:, None])
    ids = s["history"].long()
    seen = torch.zeros_like(x).scatter_add_(1, ids, said.float()) > 0
    count = torch.zeros_like(x).scatter_add_(1, ids, answered.float())
    r = s["repetition"][:, None]
    y = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    y = y - count * s["frequency"][:, None] - (count > 0) * s["presence"][:, None]
    if s["bias_ids"] is not None:
        # of a token's entries the last one counts
        ids = s["bias_ids"].long()
        at = torch.arange(ids.shape[1], device=x.device).expand_as(ids)
        last = torch.full_like(x, -1, dtype=torch.int64)
        last.scatter_reduce_(1, ids.clamp(min=0), torch.where(ids >= 0, at, -1), "amax")
        y = y + torch.where(last >= 0, s["bias_values"].gather(1, last.clamp(min=0)), 0)
    if s["bitmask"] is not None:
        y = y.masked_fill(~allowed(s), -math.inf)
    s["logits"].copy_(y)
    return s["logits"]


def plain_sample(s):
    x, k = s["logits"].float(), s["k"]
    if s["bitmask"] is not None:
        x = x.masked_fill(~allowed(s), -math.inf)
    best, ids = x.sort(dim=1, descending=True, stable=True)     # ties to the lowest token
    best, ids = best[:, :k], ids[:, :k]
    live = best > -math.inf
    t = s["temperature"][:, None]
    greedy = t <= 0
    t = torch.where(greedy, 1, t)
    top = torch.where(live[:, :1], best[:, :1], 0)
    total = ((x - top) / t).exp().sum(1, keepdim=True)
    z = (best - top) / t
    logprobs = torch.where(live, z - total.log(), -math.inf)
    j = torch.arange(k, device=x.device)
    w = torch.where(live & (j < s["top_k"][:, None]), z.exp(), 0)
    before = w.cumsum(1) - w
    p = s["top_p"][:, None]
    kept = (w > 0) & ((p >= 1) | (before < p * w.sum(1, keepdim=True)) | (j == 0)) & (w >= s["min_p"][:, None])
    score = torch.where(kept, w / s["noise"], -1)
    at = torch.where(greedy, 0, score.max(1, keepdim=True).indices)
    ids = torch.where(live, ids, -1).to(torch.int32)
    return ids.gather(1, at)[:, 0], logprobs.gather(1, at)[:, 0], ids, logprobs


PLAIN = {"head": plain_head, "penalize": plain_penalize, "sample": plain_sample}


def run(s):
    if not own:
        return PLAIN[s["op"]](s)
    from paper_2608_03065_amd import psc
    if s["op"] == "head":
        return psc.head_logits(s["x"], s["w"], s["w_scales"], dtype=s["dtype"], bias=s["bias"], bitmask=s["bitmask"])
    if s["op"] == "penalize":
        return psc.penalize(s["logits"], s["history"], s["lens"], prompt_lens=s["prompt_lens"], repetition=s["repetition"],
                            presence=s["presence"], frequency=s["frequency"], bias_ids=s["bias_ids"],
                            bias_values=s["bias_values"], bitmask=s["bitmask"])
    return psc.sample(s["logits"], s["k"], bitmask=s["bitmask"], temperature=s["temperature"], top_k=s["top_k"],
                      top_p=s["top_p"], min_p=s["min_p"], noise=s["noise"])


# ---------------------------------------------------------------- what a pass cannot do without

def work(c):
    """Every input read once and every output written once, less what the mask makes needless: weights of tokens that no
    row allows, logits of tokens that the row does not allow, and, in place, logits that stay as they are."""
    B, V, size = c["B"], c["V"], DTYPES[c["dtype"]].itemsize
    words = 0 if c["mask"] == "none" else 4 * B * ((V + 31) // 32)
    share = {"none": 1.0, "few": FEW / 2 / V, "mixed": 0.3 * FEW / 2 / V + 0.3 * 0.04 + 0.37 * 0.96}[c["mask"]]
    if c["op"] == "head":
        rows = min(V, B * FEW / 2) if c["mask"] == "few" else V
        return {"bytes": rows * (c["D"] + 4 + 4 * c["bias"]) + 2 * B * c["D"] + words + B * V * size,
                "flops": 2 * B * V * share * c["D"]}
    if c["op"] == "penalize":
        history = B * c["cap"] / 2
        touched = min(B * V, history + B * c["biases"]) * share
        return {"bytes": 4 * history + 8 * B * c["biases"] + words + 2 * size * touched + (1 - share) * B * V * size,
                "flops": 0}
    return {"bytes": share * B * V * size + words + 12 * B * c["k"] + 8 * B, "flops": 3 * share * B * V}


# ---------------------------------------------------------------- the definitions in 64 bits

def host(t):
    return None if t is None else t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def allowed_on_host(s):
    bits = np.unpackbits(np.ascontiguousarray(host(s["bitmask"])).view(np.uint8), axis=1, bitorder="little")
    return bits[:, :s["V"]].astype(bool)


def exact_head(s):
    x = host(s["x"]).astype(np.float32)
    # a scale and a quotient are 32-bit values by definition; what follows them is exact
    scales = np.abs(x).max(1, keepdims=True) / np.float32(127)
    q = np.rint(np.divide(x, scales, out=np.zeros_like(x), where=scales > 0)).astype(np.float64)
    w, y = host(s["w"]), np.empty((x.shape[0], s["V"]))
    for at in range(0, s["V"], 16384):
        y[:, at:at + 16384] = q @ w[at:at + 16384].astype(np.float64).T
    y *= scales.astype(np.float64) * host(s["w_scales"])
    if s["bias"] is not None:
        y += host(s["bias"])
    if s["bitmask"] is not None:
        y[~allowed_on_host(s)] = -np.inf
    return y


def exact_penalize(s):
    y, history, lens, starts = host(s["logits"]), host(s["history"]), host(s["lens"]), host(s["prompt_lens"])
    r, presence, frequency = host(s["repetition"]), host(s["presence"]), host(s["frequency"])
    ids, values = host(s["bias_ids"]), host(s["bias_values"])
    for b in range(y.shape[0]):
        seen = np.unique(history[b, :lens[b]])
        y[b, seen] = np.where(y[b, seen] > 0, y[b, seen] / r[b], y[b, seen] * r[b])
        said, count = np.unique(history[b, starts[b]:lens[b]], return_counts=True)
        y[b, said] -= count * frequency[b] + presence[b]
        if ids is not None:
            for v, a in {v: a for v, a in zip(ids[b].tolist(), values[b].tolist()) if v >= 0}.items():
                y[b, v] += a
    if s["bitmask"] is not None:
        y[~allowed_on_host(s)] = -np.inf
    return y


def exact_sample(s):
    x, k = host(s["logits"]), s["k"]
    if s["bitmask"] is not None:
        x[~allowed_on_host(s)] = -np.inf
    B = x.shape[0]
    out = np.full(B, -1, np.int32), np.full(B, -np.inf), np.full((B, k), -1, np.int32), np.full((B, k), -np.inf)
    tokens, logprob, ids, logprobs = out
    temperature, top_k, top_p = host(s["temperature"]), host(s["top_k"]), host(s["top_p"])
    min_p, noise = host(s["min_p"]), host(s["noise"])
    for b in range(B):
        least = np.partition(x[b], x.shape[1] - k)[x.shape[1] - k]
        best = np.nonzero((x[b] >= least) & (x[b] > -np.inf))[0]
        best = best[np.argsort(-x[b, best], kind="stable")][:k]
        if not best.size:
            continue
        greedy = temperature[b] <= 0
        z = (x[b] - x[b, best[0]]) / (1 if greedy else temperature[b])
        ids[b, :best.size], logprobs[b, :best.size] = best, z[best] - np.log(np.exp(z).sum())
        w = np.exp(z[best])[:top_k[b]]
        before = np.concatenate([[0], np.cumsum(w)[:-1]])
        kept = (w >= min_p[b]) & ((top_p[b] >= 1) | (before < top_p[b] * w.sum()) | (np.arange(w.size) == 0))
        at = 0 if greedy else int(np.argmax(np.where(kept, w / noise[b, :w.size], -1)))
        tokens[b], logprob[b] = ids[b, at], logprobs[b, at]
    return out


def exact(c, seed):
    if c["op"] == "head" and c["B"] * c["V"] * c["D"] > 2e11:
        return None        # over 20 seconds
    s = prepare(c, seed)
    return {"head": exact_head, "penalize": exact_penalize, "sample": exact_sample}[c["op"]](s)
