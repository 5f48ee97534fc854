#!/usr/bin/env python3
"""Constrained generation, whole steps on the GPU: the operators around the
logits together with the grammar's masks.

Each step of B streams, on one HIP stream and without a copy to the host:

  DecodeStates.compute_masks   the tokens that each stream's grammar state allows
  psc.head_logits              hidden states -> logits by 8-bit weights, forbidden tokens -inf
  psc.penalize                 repeated tokens made less likely, the end of text more likely
  psc.sample                   a token by temperature, top-k, top-p and min-p
  psc.append_tokens            onto the history that the penalties read
  DecodeStates.advance         the lexer and parser states past the token

The model is a stand-in with random weights, hidden = decay * hidden +
embedding[token], since the text's form comes from the grammar.

With --weights mx4 the output projection and the embedding share one table in
4 bits, and a norm stands before the projection, whose states are in 4 bits too:

  psc.lookup_rows              the last token's embedding out of the table
  psc.add_rms_norm             its addition to the hidden state, the norm, and the result in 4 bits
  psc.head_logits_mx           these states -> logits by the table's weights

  python examples/generate.py --workload json --batch 4 --tokens 48 [--weights mx4]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from inputs import configs  # noqa: E402
from paper_2608_03065_amd import psc  # noqa: E402


class Generator:
    """B streams of at most `cap` tokens under clf's grammar, from a seed."""

    def __init__(self, clf, eos_id, B, cap, D=1024, k=50, temperature=1.0, top_p=0.95, min_p=0.02, repetition=1.1,
                 presence=0.2, frequency=0.1, eos_bias=2.0, seed=0, weights="i8"):
        dev = clf.device
        self.g = torch.Generator(dev).manual_seed(seed)
        self.clf, self.k = clf, k
        self.states = psc.DecodeStates(clf, B, 4096, dev)
        self.tied = weights == "mx4"
        embedding = torch.randn(clf.V, D, generator=self.g, device=dev)
        if self.tied:
            # once: the table in 4 bits, a power of two per 32 elements
            self.weights, self.scales = psc.quantize_mx(embedding / D ** 0.5)
            self.gain, self.last = torch.ones(D, device=dev), torch.zeros(B, D, dtype=torch.bfloat16, device=dev)
        else:
            self.embedding = embedding
            # once: the output projection's weights in 8 bits, a scale per token
            self.weights, self.scales = psc.quantize_rows(torch.randn(clf.V, D, generator=self.g, device=dev) / D ** 0.5)
        self.hidden = torch.randn(B, D, generator=self.g, device=dev)
        self.history = torch.zeros(B, cap, dtype=torch.int32, device=dev)
        self.lens = torch.zeros(B, dtype=torch.int32, device=dev)
        self.done = torch.zeros(B, dtype=torch.bool, device=dev)
        self.eos = torch.full((B, 1), eos_id, dtype=torch.int32, device=dev)
        row = lambda value: torch.full((B,), value, device=dev)  # noqa: E731
        self.penalties = dict(repetition=row(repetition), presence=row(presence), frequency=row(frequency),
                              bias_ids=self.eos, bias_values=row(eos_bias)[:, None].contiguous())
        self.draw = dict(temperature=row(temperature), top_p=row(top_p), min_p=row(min_p))
        self.noise = torch.empty(B, k, device=dev)

    def step(self):
        """One token per stream; returns (tokens, log-probabilities, masks), token -1 for a stream that is done."""
        masks = self.states.compute_masks().masked_fill_(self.done[:, None], 0)
        if self.tied:
            state, powers = psc.add_rms_norm(self.last, self.gain, residual=self.hidden.mul_(0.8), to="mx4")
            logits = psc.head_logits_mx(state, self.weights, self.scales, x_scales=powers, bitmask=masks)
        else:
            logits = psc.head_logits(self.hidden.to(torch.bfloat16), self.weights, self.scales, bitmask=masks)
        psc.penalize(logits, self.history, self.lens, bitmask=masks, **self.penalties)
        self.noise.exponential_(generator=self.g)
        tokens, logprobs, _, _ = psc.sample(logits, self.k, bitmask=masks, noise=self.noise, **self.draw)
        psc.append_tokens(self.history, self.lens, tokens)
        self.done |= self.states.advance(tokens) != psc.ADV_OK
        if self.tied:
            self.last = psc.lookup_rows(self.weights, self.scales, tokens)
        else:
            self.hidden.mul_(0.8).add_(self.embedding[tokens.clamp(min=0)])
        return tokens, logprobs, masks


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workload", default="json", choices=sorted(configs.WORKLOADS))
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=48)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--weights", default="i8", choices=("i8", "mx4"))
    args = ap.parse_args()
    wl = configs.get(args.workload)
    clf = psc.Classifier(wl.grammar, wl.vocab).bind("cuda:0")
    gen = Generator(clf, wl.vocab.eos_id, args.batch, args.tokens, D=args.hidden, seed=args.seed,
                    weights=args.weights)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    score = torch.zeros(args.batch, device="cuda:0")
    for n in range(args.tokens):
        if n == 1:      # the first step loads the kernels
            start.record()
        tokens, logprobs, _ = gen.step()
        score += torch.where(tokens >= 0, logprobs, 0)
    end.record()
    torch.cuda.synchronize()
    history, lens, done, score = (t.cpu().tolist() for t in (gen.history, gen.lens, gen.done, score))
    for b in range(args.batch):
        text = b"".join(wl.vocab.tokens[t] for t in history[b][:lens[b]])
        print(f"[{b}] {lens[b]} tokens, log p {score[b]:.1f}, {'ended' if done[b] else 'cut off'}: {text.decode('utf-8', 'replace')}")
    if args.tokens > 1:
        print(f"{start.elapsed_time(end) * 1e3 / (args.tokens - 1):.0f} us a step of {args.batch} streams, V={clf.V}, D={args.hidden}")


if __name__ == "__main__":
    main()
