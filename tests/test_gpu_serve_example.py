"""The prefix cache's operators together: requests served behind resident chunks against plain
attention in 64 bits over the same tokens."""

import math

import pytest
import torch

from examples import prefix_cache as E

pytestmark = pytest.mark.gpu


def plain(layer, tokens, first, window, k_scale):
    """Attention of tokens first.. of one request, in 64 bits on the layer's rounded rows."""
    t = torch.tensor(tokens, device="cuda")
    n = t.shape[0]
    q, k, v = (x.float() for x in layer.project(t, torch.arange(n, device="cuda")))
    if k_scale:
        k, v = ((x / k_scale).to(torch.float8_e4m3fn).float() * k_scale for x in (k, v))
    G = layer.heads // layer.kv_heads
    q, k, v = (x.double().cpu() for x in (q[first:], k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)))
    s = (q.transpose(0, 1) @ k.permute(1, 2, 0)) / math.sqrt(layer.dim)
    i, j = torch.arange(first, n)[:, None], torch.arange(n)[None, :]
    hidden = (j > i) | ((j <= i - window) if window else torch.zeros_like(j, dtype=torch.bool))
    return (torch.softmax(s.masked_fill(hidden, -math.inf), 2) @ v.transpose(0, 1)).transpose(0, 1)


@pytest.mark.parametrize("cache,window,max_new", [(torch.bfloat16, 0, 64), (torch.bfloat16, 100, 37), (torch.float8_e4m3fn, 0, 256)])
def test_requests_behind_resident_chunks(cache, window, max_new):
    print(f"\n[case] {cache} window {window} max_new {max_new}", flush=True)
    layer = E.Layer.random()
    parent, target, words, leaf, prompts = E.make_inputs(seed=window, requests=12, n=60, resident=25)
    worker = E.Worker(layer, parent, target, words.shape[1], words, requests=12, max_len=max(map(len, prompts)) + 4,
                      cache=cache, window=window)
    tokens, outs, computed, found = E.serve(worker, leaf, prompts, 4, max_new)
    assert found > 0 and found + computed == sum(len(t) for t in tokens)
    for t, p, o in zip(tokens, prompts, outs):
        assert o.shape[0] == 5 and len(t) == len(p) + 4 and t[:len(p)] == p.tolist()
        want = plain(layer, t, len(p) - 1, window, 1 / 16 if cache == torch.float8_e4m3fn else None)
        # weights and the output are rounded to bf16 (2^-9 of each), and values stay below 8; the projection
        # of a batch of another shape may differ by one bf16 rounding of a value, a key or a query (2^-8 of
        # itself; scores of some 8 move by 2^-4 at most where all their terms do)
        assert (o.double().cpu() - want).abs().max() < 0.25


def test_prefixes_change_nothing():
    """Tokens computed behind found chunks see what they see where nothing is resident."""
    layer = E.Layer.random()
    parent, target, words, leaf, prompts = E.make_inputs(seed=5, requests=6, n=40, resident=20)
    outs, founds = [], []
    for t in (target, target * 0):
        worker = E.Worker(layer, parent, t, words.shape[1], words, requests=6, max_len=max(map(len, prompts)) + 1)
        _, o, _, found = E.serve(worker, leaf, prompts, 0, 512)
        outs.append(torch.cat(o).double())
        founds.append(found)
    assert founds[0] > 0 and founds[1] == 0
    assert (outs[0] - outs[1]).abs().max() < 0.25
