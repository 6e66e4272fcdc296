"""Attention over shared prompts where the caches themselves change, or are one and the same.  Tolerances: those of
test_gpu_prefix, whose definition in 64 bits this uses."""

import pytest
import torch

import paper_2605_14037_amd as spkv
from tests.test_gpu_prefix import Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch", [2, 20])
def test_another_threshold(batch):
    """Raised on the prompts' cache: the gates of the ring follow at once, the kept pairs once they are pruned."""
    s = Setup([700, 300], [5 + b for b in range(batch)], [b % 2 for b in range(batch)], 8, 2, 64, window=64, tau=0.3, keep=0.5, seed=batch)
    s.decode()
    logits, old = s.prompt[2], s.theta
    s.prefix.set_tau(0.6)
    new = s.prefix.threshold_logit()
    assert new > old

    def on(passes):                                      # the gates as the definition takes them
        s.prompt[2] = [torch.where(passes(f), 40.0, -40.0).double() for f in logits]

    # still in the lists: what passed the old threshold and had left the window by then; the ring's are new decisions
    on(lambda f: torch.where((torch.arange(len(f)) < len(f) - 64)[:, None], f >= old, f >= new))
    s.decode()
    s.prefix.prune()
    on(lambda f: f >= new)
    s.decode()


@pytest.mark.parametrize("batch", [3, 30])
def test_prompts_that_grow(batch):
    """More tokens on a prompt, then its cache in a larger arena, between steps of those who continue it."""
    s = Setup([200, 90], [1 + b for b in range(batch)], [b % 2 for b in range(batch)], 8, 2, 64, keep=0.4, seed=batch, extra=200)
    s.decode()
    s._feed(s.prefix, s.prompt, [150, 1])
    s.decode()
    s.prefix.grow(max_context=3000, max_total_kept_tokens=20000)
    s.decode()
    s._feed(s.prefix, s.prompt, [1700, 40])
    s.decode()
    s.append([3] * batch)
    s.decode()


@pytest.mark.parametrize("own", [40, 2500], ids=["short", "long"])
@pytest.mark.parametrize("batch", [3, 30])
def test_one_cache_in_both_roles(batch, own):
    """Sequence 0 is the prompt of the others, in the same cache, and is served itself."""
    counts = [700] + [own + b for b in range(batch - 1)]
    s = Setup([1], counts, [-1] + [0] * (batch - 1), 8, 2, 64, keep=0.6, seed=batch)
    s.sharing = spkv.PrefixSharing(s.cache, s.member)
    for t, mine in zip(s.prompt, s.own):
        t[0] = mine[0]
    q, out, lse = s.decode()
    alone, alone_lse = s.cache.decode_attention(q, want_lse=True)
    out, lse = s.cache.prefix_attention(s.sharing, q, None, alone, alone_lse)
    s.check(out, lse, s.reference(q, [1] * batch), "joined")
    assert torch.equal(out[0], alone[0]) and torch.equal(lse[0], alone_lse[0])
    s.append([1] * batch)                                # the prompt grows too
    for t, mine in zip(s.prompt, s.own):
        t[0] = mine[0]
    s.decode()
