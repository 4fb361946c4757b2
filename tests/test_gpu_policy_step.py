"""The example that runs the trainer-side operators together with the delta
path: the loss falls, and the receivers follow the trainer's weights through
sparse deltas alone."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab,hidden,tokens", [(1000, 64, 200), (6002, 256, 1024)])
def test_policy_step(vocab, hidden, tokens):
    from policy_step import Policy

    print("case: policy step", vocab, hidden, tokens, flush=True)
    policy = Policy(vocab, hidden)
    gen = torch.Generator(device="cuda").manual_seed(1)
    weights = torch.full((tokens,), 1.0 / tokens, device="cuda")
    first = None
    for _ in range(12):
        ids = torch.randint(0, 64, (tokens,), generator=gen, device="cuda")
        target = (ids * 31 + 7) % vocab
        target[::9] = -1
        loss, changed = policy.step(ids, target, weights)
        mean = float(loss[target >= 0].mean())
        first = mean if first is None else first
        assert bool((loss[target < 0] == 0).all())
        assert 0 < changed <= policy.p.numel()
    assert mean < first
    # the reconstruction's rounding may miss a change where it lands on the
    # other side of a BF16 rounding boundary: its error is a few binary32 ulps
    # of a weight, such boundaries are 2^16 of them apart, so a few in 2^14 of
    # the changes, over 12 steps
    assert policy.stale() <= policy.p.numel() * 12 * 2.0 ** -14
