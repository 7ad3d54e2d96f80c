"""rest_rotary where positions and values are at their ends, against 64 bits (bounds as in test_gpu_rotary.py)."""
import numpy as np
import pytest
import torch

import paper_2311_08252_b200 as rest
from test_gpu_rotary import cuda, inputs, near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("far", [1 << 29, 1 << 30, (1 << 31) - 1])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("F", [64, 61])
def test_the_bound_holds_for_every_position(F, interleaved, far):
    """32-bit rows of quickly turning pairs: what is lost of the angle shows in them."""
    x, pos, _ = inputs(F, 4, 64, 4, 128, F, torch.float32)
    rng = np.random.default_rng(far)
    pos = rng.integers(far - far // 8, far, pos.shape) * rng.choice([-1, 1], pos.shape)
    pos[0, :4] = far, -far, far - 1, 1 - far
    if far == (1 << 31) - 1:
        pos[1, 0] = -1 << 31
    freq = (10000.0 ** (-0.05 * rng.random(F))).astype(np.float32)
    freq[0] = 1
    pos = pos.astype(np.int32)
    near(rest.rest_rotary(x.cuda(), cuda(pos), cuda(freq), interleaved=interleaved), x, pos, freq, interleaved, 1.0)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("F", [1, 5, 8, 13, 16, 32])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_what_is_not_finite_stays_with_its_pair(F, interleaved, dtype, bad):
    """In either half of a pair, at the border of the halves, in lanes that hold turned and copied elements; in place, too."""
    for f in sorted({0, F // 2, F - 1, min(7, F - 1)}):
        where = [2 * f, 2 * f + 1] if interleaved else [f, F + f]
        for at in where:
            x, pos, freq = inputs(F, 1, 5, 3, 64, F, dtype)
            freq[:] = 0.7
            pos[0] = np.arange(3, 8)                    # (no angle whose sine or cosine is 0)
            x[0, 2, 1, at] = bad
            xd = x.cuda()
            for out in (None, xd):
                got = rest.rest_rotary(xd, cuda(pos), cuda(freq), interleaved=interleaved, out=out)
                assert (~got.isfinite()).nonzero().tolist() == [[0, 2, 1, w] for w in where]
