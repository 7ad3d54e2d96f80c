"""rest_accept_sampled on rows whose logits are one fp32 step apart, so that the rounding of their weights
decides nothing: the nucleus goes by the logits."""
import numpy as np
import pytest
import torch

import paper_2311_08252_b200 as rest
import sampled_util
from gpu_util import to_dev

pytestmark = pytest.mark.gpu


def run(logits, tokens, parents, nodes, uni, temp, top_p, depth, workspace=None):
    got = rest.rest_accept_sampled(to_dev(logits), to_dev(tokens), to_dev(parents), to_dev(nodes), to_dev(uni),
                                   to_dev(temp), to_dev(top_p), depth, workspace=workspace)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in got]


def check(logits, tokens, parents, nodes, uni, temp, top_p, depth):
    """Both forms against the walk in 64 bits, none of whose comparisons the weights' rounding could turn."""
    B = len(tokens)
    want = [sampled_util.walk(logits[b].astype(np.float64), tokens[b], parents[b], nodes[b], uni[b], temp[b], top_p[b], depth)
            for b in range(B)]
    assert min(w[2] for w in want) > 1
    for workspace in (None, False):
        n, an, ot = run(logits, tokens, parents, nodes, uni, temp, top_p, depth, workspace)
        for b in range(B):
            path, out, _ = want[b]
            assert an[b, :n[b]].tolist() == path and ot[b, :n[b] + 1].tolist() == out, (
                b, logits[b, 0].tolist() if logits.shape[2] < 10 else b, float(uni[b, 0]), an[b].tolist(), ot[b].tolist(), want[b])


def pairs(rng, B, near, far):
    """Logits x and the next fp32 number above it, x near `near`."""
    low = (near + rng.uniform(-far, far, B)).astype(np.float32)
    return low, np.nextafter(low, np.float32(np.inf))


@pytest.mark.parametrize("order", [(0, 1, 2), (0, 2, 1), (2, 1, 0), (1, 2, 0)])
@pytest.mark.parametrize("top_p", [0.9, 0.5])
def test_two_logits_one_step_apart(order, top_p):
    """Three tokens, the second and third one step apart.  0.9 keeps all three, 0.5 the first two: neither
    may lose a token whose mass was counted, nor take one in whose mass was not."""
    B = 60
    rng = np.random.default_rng(1)
    low, high = pairs(rng, B, 0.01, 0.004)
    low[0], high[0] = np.float32(0.0102107851), np.float32(0.010210786)
    low[1], high[1] = high[0], np.nextafter(high[0], np.float32(1))
    logits = np.stack([np.full(B, 0.02, np.float32), high, low], 1)[:, order][:, None].repeat(2, 1)
    none = np.zeros(B, np.int32)
    tokens = np.full((B, 1), order.index(1), np.int32)
    one = np.ones(B, np.float32)
    for u0 in (0.05, 0.3, 0.45, 0.6, 0.8, 0.95):
        uni = np.stack([np.full(B, u0), np.full(B, 0.2)], 1).astype(np.float32)
        check(logits, tokens, np.full((B, 1), -1, np.int32), none, uni, one, np.full(B, top_p, np.float32), 1)
    # the same with the second token drafted: accepted at 0.2, refused at 0.7 and then not drawn
    for u1 in (0.2, 0.7):
        uni = np.stack([np.full(B, 0.6), np.full(B, u1)], 1).astype(np.float32)
        check(logits, tokens, np.full((B, 1), -1, np.int32), none + 1, uni, one, np.full(B, top_p, np.float32), 1)


@pytest.mark.parametrize("V", [3, 4, 17, 300, 2000])
@pytest.mark.parametrize("temp,top", [(0.6, 0.0), (1.0, 5.0), (2.0, 20.0), (0.9, 12.0)])
def test_many_logits_a_step_apart(V, temp, top):
    """One largest logit and pairs one step apart around 0, the cut in the midst of them; rows of more than
    512 tokens that share a bin among them."""
    B = 40 if V > 100 else 250
    rng = np.random.default_rng(V + int(10 * temp))
    # the row's other tokens weigh as much as the largest one, or less where they are few
    k = (V - 1) // 2
    low, high = pairs(rng, B * k, 0.0, 0.004)
    logits = np.zeros((B, 2, V), np.float32)
    body = np.concatenate([low.reshape(B, k), high.reshape(B, k)], 1)
    logits[:, :, 0] = top
    logits[:, :, 1:1 + 2 * k] = rng.permuted(body, axis=1)[:, None]
    share = V * np.exp(-top / temp)
    top_p = (1 - rng.uniform(0.05, 0.95, B) * min(share, 0.9) / (1 + share)).astype(np.float32)
    tokens = rng.integers(0, V, (B, 1)).astype(np.int32)
    uni = rng.random((B, 2)).astype(np.float32)
    t = np.full(B, temp, np.float32)
    check(logits, tokens, np.full((B, 1), -1, np.int32), rng.integers(0, 2, B).astype(np.int32), uni, t, top_p, 1)
