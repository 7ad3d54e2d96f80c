"""The appends and the commit in codes where values and pages are at their ends, against the plain models."""
import numpy as np
import pytest
import torch

import paper_2311_08252_b200 as rest
import scaled_util as plain
from test_gpu_append import BF16, cuda, scaled_state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("F,amplitude,value", [(32, 1.0, 3.3e38), (32, 2.0, 2e38), (13, 1.0, 3.3e38), (13, -3.0, 3e38), (32, 1e6, 1e37)])
def test_finite_values_that_32_bits_do_not_hold(F, amplitude, value, interleaved):
    """Pairs that a rotation or the amplitude takes beyond the largest 32-bit number saturate as other large ones do;
    what is not finite beside them becomes NaN."""
    kv_len = [20]
    rng, pk, pv, ks, vs, raw, scales, table = scaled_state(5, 1, 2, 64, 16, kv_len, 4)
    new = torch.zeros((1, 4, 2, 64), dtype=BF16)
    one, two = (6, 7) if interleaved else (3, F + 3)
    new[0, 1, 0, one], new[0, 1, 0, two] = value, value
    new[0, 2, 1, one], new[0, 2, 1, two] = -value, value
    new[0, 3, 1, one + 2 if interleaved else one + 1] = float("inf")
    pos = np.array([[0, 1, 2, 3]], np.int32)
    freq = np.full(F, 0.7853981633974483, np.float32)
    rest.rest_paged_kv_append_scaled(pk, pv, ks, vs, cuda(table), cuda(np.array(kv_len, np.int32)), new.cuda(), new.cuda(),
                                     cuda(pos), cuda(freq), interleaved, amplitude)
    with np.errstate(invalid="ignore"):
        k = plain.turn(new.double().numpy(), pos, freq, interleaved, amplitude)
    assert np.abs(k[np.isfinite(k)]).max() > np.finfo(np.float32).max
    for i, (codes, sc, x) in enumerate(((pk, ks, k), (pv, vs, new.double().numpy()))):
        plain.write(raw[i], scales[i], table, kv_len, x, [4])
        assert np.array_equal(sc.cpu().numpy(), scales[i]) and plain.same_codes(codes, raw[i])
