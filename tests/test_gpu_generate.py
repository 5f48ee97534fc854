"""The example that runs the operators around the logits with the grammar's masks: every step's masks against the
oracle, its tokens under them, and the history they leave; a second run of the same seed is the same."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from examples.generate import Generator  # noqa: E402

pytestmark = pytest.mark.gpu
B, STEPS = 6, 40


def allowed(masks, b, t):
    return masks[b, t >> 5] >> np.uint32(t & 31) & 1


@pytest.mark.parametrize("name", ["arithmetic", "json"])
def test_generated_tokens_obey_the_grammar(built, name):
    wl, clf, orc = built(name)
    gen = Generator(clf, wl.vocab.eos_id, B, STEPS, D=200, k=20, seed=3)
    states, said, done = gen.states.host_states(), [[] for _ in range(B)], [False] * B
    for _ in range(STEPS):
        tokens, logprobs, masks = (t.cpu().numpy() for t in gen.step())
        masks, want = masks.view(np.uint32), orc.masks(states)
        for b in range(B):
            if done[b]:
                assert tokens[b] == -1 and np.isneginf(logprobs[b]) and not masks[b].any()
                continue
            t = int(tokens[b])
            assert np.array_equal(masks[b], want[b]) and t >= 0 and allowed(masks, b, t) and logprobs[b] <= 0
            said[b].append(t)
            code, new = orc.advance(states[b], t, 4096)
            if code == 0:
                states[b] = new
            else:
                done[b] = True
                assert t == wl.vocab.eos_id
    assert gen.lens.tolist() == [len(s) for s in said]
    assert [gen.history[b, :len(s)].tolist() for b, s in enumerate(said)] == said
    assert gen.done.tolist() == done
    again = Generator(clf, wl.vocab.eos_id, B, STEPS, D=200, k=20, seed=3)
    for _ in range(STEPS):
        again.step()
    assert torch.equal(gen.history, again.history) and torch.equal(gen.lens, again.lens)
