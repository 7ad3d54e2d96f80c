"""rest_paged_attention_scaled with scales of keys at their ends, against 64 bits."""
import pytest

from test_gpu_paged_attention_scaled import BF16, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,H", [(1, 4), (4, 4), (20, 1), (20, 4), (70, 4)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ks,q,scale", [(-60, 57, -7), (-60, 57, -12), (60, -50, -18), (40, 0, -48), (-20, 0, 12), (0, 20, -28)])
def test_scales_of_keys_at_their_ends(N, H, D, ks, q, scale):
    """Sizes of keys, queries and of the scale of scores that only together make scores of ordinary size."""
    c = make(70, 2, N, H, 1, D, 32, [150, 33])
    c["ks"][:] = 2.0 ** ks
    c["q"] = (c["q"].float() * 2.0 ** q).to(BF16)
    check(c, scale=2.0 ** scale)
    check(c, window=60, sinks=3, scale=2.0 ** scale)
