"""Rotary positions against the rotation in 64 bits: layouts, parts of the head, far and negative
positions, strides, in place, inverse (the gradient), scaled frequencies."""
import numpy as np
import pytest

import decoding_reference as R

pytestmark = pytest.mark.gpu


def _rng(*seed):
    return np.random.Generator(np.random.PCG64(list(seed)))


def _freqs(rot, **kw):
    import paper_2509_26436_amd as q
    return q.rotary_frequencies(rot, **kw)


def _check(got, x, positions, freqs, layout, **kw):
    y, far = R.rotate(x, positions, freqs.cpu().numpy(), layout, **kw)
    off = np.abs(R.host(got) - y)
    assert (off <= R.HALF_BF16 * np.abs(y) + (1 + R.HALF_BF16) * far).all(), off.max()
    rot = 2 * freqs.numel()
    np.testing.assert_array_equal(R.host(got)[..., rot:], x[..., rot:])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,H,d,rot", [(1, 1, 64, 64), (3, 5, 128, 128), (17, 4, 128, 64), (5, 7, 64, 20), (9, 3, 80, 80),
                                       (2, 9, 256, 32), (300, 2, 96, 96), (4, 3, 6, 2), (7, 2, 64, 0)])
def test_rotary(T, H, d, rot, layout):
    import torch
    import paper_2509_26436_amd as q
    print(f"rotary {T} x {H} x {d} rot {rot} {layout}", flush=True)
    rng = _rng(1, T, H, d, rot)
    x = R.bf16(rng.normal(0, 2, (T, H, d)))
    positions = rng.integers(0, 1 << 20, T)
    positions[0] = 0
    f, p = _freqs(rot), torch.from_numpy(positions.astype(np.int32)).cuda()
    xd = R.device(x)
    got = q.rotary(xd, p, f, layout)
    _check(got, x, positions, f, layout)
    np.testing.assert_array_equal(R.host(xd), x)
    assert q.rotary(xd, p, f, layout, out=xd) is xd                     # in place
    np.testing.assert_array_equal(R.host(xd), R.host(got))
    # [heads, tokens, d] in memory
    hd = R.device(x.transpose(1, 0, 2).copy()).transpose(0, 1)
    by_head = q.rotary(hd, p, f, layout)
    np.testing.assert_array_equal(R.host(by_head), R.host(got))
    # rows of wider tensors, at an odd offset
    wide = torch.full((T, H + 1, d + 6), 3.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :H, 3:3 + d] = R.device(x)
    out = torch.full((T, H + 2, d + 2), 9.0, dtype=torch.bfloat16, device="cuda")
    q.rotary(wide[:, :H, 3:3 + d], p, f, layout, out=out[:, 1:H + 1, 1:d + 1])
    np.testing.assert_array_equal(R.host(out[:, 1:H + 1, 1:d + 1]), R.host(got))
    out[:, 1:H + 1, 1:d + 1] = 9.0
    assert (out == 9.0).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_and_negative_positions(layout):
    import torch
    import paper_2509_26436_amd as q
    positions = np.array([2 ** 31 - 1, -2 ** 31, -1, -12345, 2 ** 24 + 1, 2 ** 30])
    x = R.bf16(_rng(2).normal(0, 1, (len(positions), 2, 128)))
    f = _freqs(128)
    got = q.rotary(R.device(x), torch.from_numpy(positions.astype(np.int32)).cuda(), f, layout)
    _check(got, x, positions, f, layout)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot", [128, 36])
def test_inverse_is_the_gradient(layout, rot):
    """<g, rotary(x)> = <inverse(g), x>, the formula's transpose, and central differences of the
    map (it is linear: exact but for the bf16 roundings)."""
    import torch
    import paper_2509_26436_amd as q
    rng = _rng(3, rot)
    T, H, d, magnitude = 6, 3, 128, 1.25
    x, g = (R.bf16(rng.normal(0, 1, (T, H, d))) for _ in range(2))
    positions = rng.integers(0, 5000, T)
    p, f = torch.from_numpy(positions.astype(np.int32)).cuda(), _freqs(rot)
    back = q.rotary(R.device(g), p, f, layout, inverse=True, magnitude=magnitude)
    y, far = R.rotate(g, positions, f.cpu().numpy(), layout, inverse=True, magnitude=magnitude)
    assert (np.abs(R.host(back) - y) <= R.HALF_BF16 * np.abs(y) + (1 + R.HALF_BF16) * far).all()
    step = 0.5
    for _ in range(8):
        t, h, i = rng.integers(0, T), rng.integers(0, H), rng.integers(0, d)
        up, down = x.copy(), x.copy()
        up[t, h, i], down[t, h, i] = R.bf16(x[t, h, i] + step), R.bf16(x[t, h, i] - step)
        hi, lo = (R.host(q.rotary(R.device(a), p, f, layout, magnitude=magnitude)) for a in (up, down))
        width = up[t, h, i] - down[t, h, i]
        slope = ((hi - lo) * g).sum() / width
        # only the pair's two outputs differ: each is rounded twice
        changed = hi != lo
        far = (R.HALF_BF16 * (np.abs(hi) + np.abs(lo)) * np.abs(g))[changed].sum() / width
        want = R.host(back)[t, h, i]
        assert abs(slope - want) <= far + R.HALF_BF16 * abs(want) + 1e-4


def test_magnitude_and_scaled_frequencies():
    import torch
    import paper_2509_26436_amd as q
    x = R.bf16(_rng(4).normal(0, 1, (5, 2, 64)))
    positions = np.array([0, 1, 999, 32768, 131071])
    p = torch.from_numpy(positions.astype(np.int32)).cuda()
    for scaling in ("linear", "base", "parts"):
        f = _freqs(64, base=500000.0, scaling=scaling, factor=8.0, low=1.0, high=4.0, original=8192.0)
        _check(q.rotary(R.device(x), p, f, magnitude=1.2079), x, positions, f, "half", magnitude=1.2079)


def test_graph_and_stream():
    import torch
    import paper_2509_26436_amd as q
    rng = _rng(5)
    f = _freqs(128)
    xs = [R.device(R.bf16(rng.normal(0, 1, (33, 4, 128)))) for _ in range(2)]
    ps = [torch.from_numpy(rng.integers(0, 9000, 33).astype(np.int32)).cuda() for _ in range(2)]
    want = [q.rotary(x, p, f) for x, p in zip(xs, ps)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    y = q.rotary(xs[1], ps[1], f, stream=stream)
    stream.synchronize()
    assert torch.equal(y, want[1])
    x, p, out = xs[0].clone(), ps[0].clone(), torch.empty_like(xs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q.rotary(x, p, f, out=out)
    for i in (0, 1, 0):
        x.copy_(xs[i])
        p.copy_(ps[i])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
