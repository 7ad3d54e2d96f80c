"""What the calls of the rotation and of the cache in codes refuse, before anything is launched, and the frequencies."""
import ctypes
import math

import numpy as np
import pytest

import paper_2311_08252_b200 as rest
import scaled_util as plain

OK, INVALID, UNSUPPORTED = 0, 1, 2


def strides(*s):
    return (ctypes.c_int64 * len(s))(*s)


ROWS = strides(4096, 1024, 128)


def rotary(x=256, s=ROWS, dtype=0, pos=256, freq=256, pairs=64, amp=1.0, B=1, H=8, N=4, D=128, out=256, os=ROWS):
    return rest.lib().rest_rotary(x, s, dtype, pos, freq, pairs, 0, amp, None, B, H, N, D, out, os, None)


def test_rotary_refuses():
    assert rotary(B=0) == OK and rotary(N=0) == OK
    assert rotary(x=None) == INVALID and rotary(x=264) == INVALID and rotary(out=264) == INVALID
    assert rotary(dtype=3) == INVALID and rotary(H=0) == INVALID and rotary(D=0) == INVALID and rotary(B=-1) == INVALID
    assert rotary(D=120, pairs=60) == UNSUPPORTED and rotary(D=528, pairs=4) == UNSUPPORTED
    assert rotary(pairs=65) == INVALID and rotary(pairs=-1) == INVALID and rotary(pos=None) == INVALID and rotary(freq=None) == INVALID
    assert rotary(amp=float("inf")) == INVALID and rotary(amp=float("nan")) == INVALID
    assert rotary(s=strides(4096, 1024, 124)) == INVALID and rotary(os=strides(4096, 64, 128)) == INVALID
    assert rotary(s=strides(4096, 1024, -128)) == INVALID and rotary(s=None) == INVALID


def append(k=256, s=strides(8 * 16 * 128, 16 * 128, 128), scale=256, P=4, page=16, table=256, ts=3, cols=3, new=ROWS, dtype=0,
           pairs=64, q=256, H=8, B=1, H_kv=8, N=4, D=128, scaled=True, pos=256):
    L = rest.lib()
    tail = (P, page, table, ts, cols, 256, 256, 256, new, None, dtype, pos, 256, pairs, 0, 1.0, q, ROWS, 256, ROWS, H, B, H_kv, N, D,
            None)
    return L.rest_paged_kv_append_scaled(k, 256, s, scale, scale, *tail) if scaled else L.rest_paged_kv_append(k, 256, s, *tail)


@pytest.mark.parametrize("scaled", [False, True])
def test_appends_refuse(scaled):
    a = lambda **kw: append(scaled=scaled, **kw)  # noqa: E731
    assert a(B=0) == OK and a(N=0) == OK
    assert a(k=None) == INVALID and a(k=264) == INVALID and a(page=24) == UNSUPPORTED and a(D=96) == UNSUPPORTED
    assert a(s=strides(16384, 2048, 120)) == INVALID and a(s=strides(0, 2048, 128)) == INVALID
    assert a(table=None) == INVALID and a(ts=2) == INVALID and a(P=0) == INVALID
    assert a(new=strides(4096, 1024, 4)) == INVALID and a(dtype=2) == INVALID and a(pairs=65) == INVALID
    assert a(q=None) == INVALID and a(q=None, H=0, B=0) == OK and a(H=-1) == INVALID and a(pos=None) == INVALID
    # rows of codes start on 16 bytes: strides of 8 elements do for 16-bit pages alone
    assert a(s=strides(16384 + 8, 2048 + 8, 136), B=1, table=None) == INVALID
    if scaled:
        assert a(scale=None) == INVALID and a(s=strides(16384, 2048, 136)) == INVALID


def test_commits_and_copies_refuse():
    L, s = rest.lib(), strides(8 * 16 * 128, 16 * 128, 128)
    c = lambda depth=4, B=1, page=16, nodes=256, scale=256: L.rest_paged_kv_commit_scaled(  # noqa: E731
        256, 256, s, scale, scale, 4, page, 256, 3, 3, 256, nodes, 256, B, 8, 64, 128, depth, None, None)
    assert c(B=0) == OK and c(depth=17) == UNSUPPORTED and c(depth=0) == INVALID and c(page=20) == UNSUPPORTED
    assert c(nodes=None) == INVALID and c(scale=None) == INVALID
    y = lambda n=1, D=128, src=256, scale=256: L.rest_pages_copy_scaled(256, 256, s, scale, scale, 4, 16, 8, D, src, 256, n, None)  # noqa: E731
    assert y(n=0) == OK and y(n=-1) == INVALID and y(D=32) == UNSUPPORTED and y(src=None) == INVALID and y(scale=None) == INVALID


def test_python_refuses():
    torch = pytest.importorskip("torch")
    x, i = torch.zeros((1, 2, 3, 64)), torch.zeros((1, 2), dtype=torch.int32)
    f = torch.zeros(32)
    with pytest.raises(rest.RestError):
        rest.rest_rotary(x, i, f)                       # on the host
    with pytest.raises(rest.RestError, match="x must be"):
        rest.rest_rotary(x.double(), i, f)
    with pytest.raises(rest.RestError, match="together"):
        rest.rest_rotary(x, None, f)
    with pytest.raises(rest.RestError, match="at most"):
        rest.rest_rotary(x, i, torch.zeros(33))
    codes, scales = torch.zeros((2, 1, 16, 64), dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros((2, 1, 1))
    with pytest.raises(rest.RestError, match="float8"):
        rest.rest_pages_copy_scaled(x, x, scales, scales, i[0], i[0])
    with pytest.raises(rest.RestError, match="k_scales"):
        rest.rest_pages_copy_scaled(codes, codes, scales[:, :, :0], scales, i[0], i[0])


def test_frequencies():
    f, a = rest.rotary_frequencies(64)
    assert a == 1.0 and np.allclose(f.numpy(), 10000.0 ** (-np.arange(32) / 32), rtol=2e-7)
    g, a = rest.rotary_frequencies(64, scaling="linear", factor=4.0)
    assert a == 1.0 and np.allclose(g.numpy(), f.numpy() / 4, rtol=2e-7)
    g, _ = rest.rotary_frequencies(64, scaling="base", factor=8.0)
    assert g[0] == 1 and math.isclose(float(f[-1] / g[-1]), 8.0, rel_tol=1e-5)
    g, a = rest.rotary_frequencies(64, scaling="parts", factor=8.0, original_len=4096)
    assert math.isclose(a, 0.1 * math.log(8.0) + 1) and g[0] == f[0] and math.isclose(float(f[-1] / g[-1]), 8.0, rel_tol=1e-5)
    turns = 4096 * f.double().numpy() / (2 * math.pi)
    ratio = (g.double() / f.double()).numpy()
    assert (np.diff(ratio[turns < 32]) <= 1e-7).all() and (abs(ratio[turns >= 32] - 1) < 1e-6).all()
    for bad in (dict(dim=63), dict(dim=0), dict(dim=64, scaling="other"), dict(dim=64, factor=0.5),
                dict(dim=64, scaling="parts", factor=2.0), dict(dim=64, base=0.0)):
        with pytest.raises(rest.RestError):
            rest.rotary_frequencies(**bad)


def test_the_plain_model():
    """The model itself: 448 fits a scale of 1, 449 needs 2; older rows move to a larger scale, never to a smaller."""
    assert plain.fitting(448.0) == 1 and plain.fitting(449.0) == 2 and plain.fitting(0.0) == 2.0 ** -60
    codes, scales = np.zeros((1, 1, 16, 16), np.uint8), np.ones((1, 1, 1), np.float32)
    table = np.zeros((1, 1), np.int32)
    plain.write(codes, scales, table, [0], np.full((1, 1, 1, 16), 7.0), [1])
    assert scales[0, 0, 0] == 2.0 ** -6 and (plain.decode(codes[0, 0, 0]) == 448).all()
    plain.write(codes, scales, table, [1], np.full((1, 1, 1, 16), 28.0), [1])
    assert scales[0, 0, 0] == 2.0 ** -4 and (plain.decode(codes[0, 0, :2]) == [[112.0] * 16, [448.0] * 16]).all()
    plain.write(codes, scales, table, [2], np.full((1, 1, 1, 16), 1.0), [1])
    assert scales[0, 0, 0] == 2.0 ** -4 and (plain.decode(codes[0, 0, 2]) == 16).all()


def attend(st=None, dtype=0, P=4, page=16, ts=3, cols=3, H=8, H_kv=2, N=4, D=128, window=0, sinks=0, scale=1.0, q=256,
           scales=256, B=1):
    st = strides(4096, 1024, 128, 4096, 2048, 128, 4096, 1024, 128) if st is None else st
    return rest.lib().rest_paged_attention_scaled(q, 256, 256, st, scales, 256, dtype, P, page, 256, ts, cols, 256, None, 256, B, H,
                                                  H_kv, N, D, window, sinks, scale, 256, None, None, 0, None)


def test_attention_refuses():
    assert attend(B=0) == OK
    assert attend(D=96) == UNSUPPORTED and attend(N=257) == UNSUPPORTED and attend(H_kv=3) == UNSUPPORTED
    assert attend(page=8) == UNSUPPORTED and attend(page=48) == UNSUPPORTED
    assert attend(dtype=2) == INVALID and attend(dtype=-1) == INVALID and attend(scales=None) == INVALID
    assert attend(scale=0.0) == INVALID and attend(scale=float("inf")) == INVALID and attend(scale=float("nan")) == INVALID
    assert attend(window=-1) == INVALID and attend(sinks=-1) == INVALID and attend(P=0) == INVALID
    assert attend(q=None) == INVALID and attend(q=264) == INVALID and attend(ts=2) == INVALID
    assert attend(strides(4096, 1024, 128, 4096, 2048, 136, 4096, 1024, 128)) == INVALID     # rows of codes off 16 bytes
    assert attend(strides(4096, 1024, 128, 4096, 2048, 64, 4096, 1024, 128)) == INVALID      # rows that overlap
    assert attend() == INVALID                                                               # no scratch
