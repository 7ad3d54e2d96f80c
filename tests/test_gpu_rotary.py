"""rest_rotary against 64 bits, and as its own inverse and gradient.

Bound of an element: its cosine and sine are rounded to 32 bits, one product and the multiply-add are rounded: three
times 2^-24 of a (|x1| + |x2|), below 2^-22 of it; then half a step of the type."""
import numpy as np
import pytest
import torch

import paper_2311_08252_b200 as rest
import scaled_util as plain

pytestmark = pytest.mark.gpu
EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def inputs(seed, B, N, H, D, F, dtype, far=5000):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.normal(size=(B, N, H, D))).to(dtype)
    pos = rng.integers(-far, far, (B, N)).astype(np.int32)
    freq = (10000.0 ** (-np.arange(F) / max(F, 1))).astype(np.float32)
    return x, pos, freq


def near(got, x, pos, freq, interleaved, amplitude):
    xs = x.double().numpy()
    want = plain.turn(xs, pos, freq, interleaved, amplitude)
    size = plain.turn(np.abs(xs), np.zeros_like(pos), freq, interleaved, amplitude)      # a |x1|, a |x2|
    F = len(freq)
    one, two = (slice(0, 2 * F, 2), slice(1, 2 * F, 2)) if interleaved else (slice(0, F), slice(F, 2 * F))
    both = np.zeros_like(size)
    both[..., one] = both[..., two] = size[..., one] + size[..., two]
    over = np.abs(got.double().cpu().numpy() - want) - EPS[x.dtype] * np.abs(want) - 2.0 ** -22 * both - (
        2.0 ** -25 if x.dtype == torch.float16 else 0)
    assert over.max() <= 0, over.max()


def cuda(a):
    return torch.from_numpy(a).cuda()


SHAPES = [(1, 1, 1, 16, 8), (2, 5, 3, 64, 32), (1, 64, 32, 128, 64), (3, 17, 5, 128, 32), (2, 33, 2, 128, 13),
          (2, 16, 7, 80, 40), (1, 9, 3, 96, 24), (2, 3, 2, 256, 128), (1, 20, 2, 512, 256), (1, 19, 1, 512, 9),
          (2, 4, 3, 48, 1), (1, 3, 2, 64, 0), (5, 256, 1, 64, 16)]


@pytest.mark.parametrize("dtype", list(EPS))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_rotation(shape, interleaved, dtype):
    x, pos, freq = inputs(sum(shape), *shape, dtype)
    out = rest.rest_rotary(x.cuda(), cuda(pos), cuda(freq), interleaved=interleaved, amplitude=1.25)
    near(out, x, pos, freq, interleaved, 1.25)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("F", [64, 32, 13])
def test_far_positions_strides_and_in_place(F, interleaved):
    """Positions of millions, heads before rows in memory, with gaps; in place gives the same."""
    x, pos, freq = inputs(F, 2, 21, 6, 128, F, torch.bfloat16, far=1 << 30)
    big = torch.zeros((2, 6, 21, 144), dtype=x.dtype, device="cuda")
    view = big[..., :128].transpose(1, 2)
    view.copy_(x)
    out = rest.rest_rotary(view, cuda(pos), cuda(freq), interleaved=interleaved)
    near(out, x, pos, freq, interleaved, 1.0)
    got = rest.rest_rotary(view, cuda(pos), cuda(freq), interleaved=interleaved, out=view)
    assert got is view and torch.equal(view, out) and not big[..., 128:].any()


def test_rows_behind_the_tree_stay():
    x, pos, freq = inputs(3, 4, 20, 2, 64, 32, torch.float16)
    out = torch.full_like(x, 7).cuda()
    nodes = np.array([0, 20, 3, -5], np.int32)
    rest.rest_rotary(x.cuda(), cuda(pos), cuda(freq), out=out, n_nodes=cuda(nodes))
    whole = rest.rest_rotary(x.cuda(), cuda(pos), cuda(freq))
    for b, n in enumerate(nodes):
        n = max(n, 0)
        assert torch.equal(out[b, :n], whole[b, :n]) and (out[b, n:] == 7).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("F", [0, 5, 8, 16])
def test_what_is_not_finite_stays_with_its_pair(F, interleaved):
    x, pos, freq = inputs(F, 1, 3, 2, 64, F, torch.bfloat16)
    x[0, 1, 0, 40], x[0, 2, 1, 63] = float("inf"), float("nan")
    out = rest.rest_rotary(x.cuda(), cuda(pos), cuda(freq), interleaved=interleaved).cpu()
    assert torch.equal(out[..., 2 * F:].view(torch.int16), x[..., 2 * F:].view(torch.int16)) and out[..., :2 * F].isfinite().all()


def test_inverse_and_gradient():
    """The call with -inv_freq undoes the rotation; with the amplitude kept it is the gradient, by autograd of the
    formula and by differences."""
    x, pos, freq = inputs(5, 2, 7, 3, 64, 32, torch.float32)
    p, f = cuda(pos), cuda(freq)
    y = rest.rest_rotary(x.cuda(), p, f, amplitude=2.0)
    back = rest.rest_rotary(y, p, -f, amplitude=0.5)
    assert (back.cpu() - x).abs().max() <= 8 * 2.0 ** -22 * 2 * x.abs().max()
    g = torch.from_numpy(np.random.default_rng(6).normal(size=x.shape)).float()
    dx = rest.rest_rotary(g.cuda(), p, -f, amplitude=2.0).double().cpu()
    a = x.double().requires_grad_()
    t = torch.from_numpy(pos).double()[:, :, None, None] * torch.from_numpy(freq).double()
    z = 2.0 * torch.cat([a[..., :32] * t.cos() - a[..., 32:] * t.sin(), a[..., 32:] * t.cos() + a[..., :32] * t.sin()], -1)
    (z * g.double()).sum().backward()
    assert (dx - a.grad).abs().max() <= 2.0 ** -22 * 4 * g.abs().max()
    d = torch.from_numpy(np.random.default_rng(7).normal(size=x.shape))
    run = lambda v: (torch.from_numpy(plain.turn(v.numpy(), pos, freq, False, 2.0)) * g.double()).sum()  # noqa: E731
    slope = (run(x.double() + 1e-3 * d) - run(x.double() - 1e-3 * d)) / 2e-3
    assert abs(float((dx * d).sum() - slope)) <= 2.0 ** -20 * float((dx * d).abs().sum())


def test_captured_and_on_another_stream():
    x, pos, freq = inputs(9, 2, 11, 4, 128, 64, torch.bfloat16)
    xd, p, f, out = x.cuda(), cuda(pos), cuda(freq), torch.zeros_like(x).cuda()
    want = rest.rest_rotary(xd, p, f)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = rest.rest_rotary(xd, p, f, stream=s)
    s.synchronize()
    assert torch.equal(other, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rest.rest_rotary(xd, p, f, out=out)
    xd.copy_(-x.cuda())
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, -want)
