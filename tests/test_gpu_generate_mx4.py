"""The example with one table in 4 bits for the output projection and the embedding: every step's masks against the
oracle, its tokens under them, and the history they leave; a second run of the same seed is the same."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from examples.generate import Generator  # noqa: E402

pytestmark = pytest.mark.gpu
B, STEPS = 5, 30


@pytest.mark.parametrize("name,D", [("arithmetic", 200), ("json", 512)])
def test_generated_tokens_obey_the_grammar(built, name, D):
    wl, clf, orc = built(name)
    gen = Generator(clf, wl.vocab.eos_id, B, STEPS, D=D, k=20, seed=4, weights="mx4")
    states, said, done = gen.states.host_states(), [[] for _ in range(B)], [False] * B
    for _ in range(STEPS):
        tokens, logprobs, masks = (t.cpu().numpy() for t in gen.step())
        masks, want = masks.view(np.uint32), orc.masks(states)
        for b, t in enumerate(tokens.tolist()):
            if done[b]:
                assert t == -1 and np.isneginf(logprobs[b]) and not masks[b].any() and not bool(gen.last[b].any())
                continue
            assert np.array_equal(masks[b], want[b]) and t >= 0 and masks[b, t >> 5] >> np.uint32(t & 31) & 1 and logprobs[b] <= 0
            said[b].append(t)
            code, new = orc.advance(states[b], t, 4096)
            if code == 0:
                states[b] = new
            else:
                done[b] = True
                assert t == wl.vocab.eos_id
    assert gen.lens.tolist() == [len(s) for s in said] and bool(torch.isfinite(gen.hidden).all())
    assert [gen.history[b, :len(s)].tolist() for b, s in enumerate(said)] == said
    again = Generator(clf, wl.vocab.eos_id, B, STEPS, D=D, k=20, seed=4, weights="mx4")
    for _ in range(STEPS):
        again.step()
    assert torch.equal(gen.history, again.history) and torch.equal(gen.hidden, again.hidden)
