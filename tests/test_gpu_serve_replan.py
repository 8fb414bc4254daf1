"""A plan that changes while requests run: what they found stays in place until they are through."""

import numpy as np
import pytest
import torch

from examples import prefix_cache as E

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", [torch.bfloat16, torch.float8_e4m3fn])
def test_running_requests_keep_their_chunks(cache):
    print(f"\n[case] {cache}", flush=True)
    layer = E.Layer.random()
    parent, target, words, leaf, prompts = E.make_inputs(seed=2, requests=12, n=60, resident=25)
    other = E.plan_one(parent, np.where(target > 0, 1, 1000).astype(np.int64), 25)   # what was not wanted before
    none = np.zeros_like(target)
    outs = []
    for plans in (None, {2: other, 4: target, 5: none, 6: other}):
        worker = E.Worker(layer, parent, target, words.shape[1], words, requests=12, max_len=max(map(len, prompts)) + 9,
                          cache=cache, spare=30)
        tokens, o, computed, found = E.serve(worker, leaf, prompts, 9, 64, plans=plans)
        outs.append((tokens, torch.cat(o), computed, found))
    assert outs[0][3] > 0
    assert ((target > 0) & (other == 0)).any() and ((other > 0) & (target == 0)).any()
    assert outs[0][0] == outs[1][0] and outs[0][2:] == outs[1][2:]
    assert torch.equal(outs[0][1], outs[1][1])


def test_slots_that_are_given_away():
    """Without the running requests' chunks in the target their slots go to others in the same call."""
    layer = E.Layer.random()
    parent, target, words, leaf, prompts = E.make_inputs(seed=2, requests=12, n=60, resident=25)
    worker = E.Worker(layer, parent, target, words.shape[1], words, requests=12, max_len=max(map(len, prompts)))
    before = worker.held.copy()
    other = E.plan_one(parent, np.where(target > 0, 1, 1000).astype(np.int64), 25)
    worker.place_chunks(other)
    gone = before[(target > 0) & (other == 0)]
    new = worker.held[(target == 0) & (other > 0)]
    assert np.intersect1d(gone, new).size > 0
