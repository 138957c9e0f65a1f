"""Norms of query and key heads with their rotary positions: shapes, strides, axes, against the
definition in 64 bits."""
import numpy as np
import pytest

import decoding_reference as R
import prompt_reference as T

pytestmark = pytest.mark.gpu


def _check(got, x, weight, eps, positions, axes, freqs, layout, magnitude=1.0):
    y, far = T.head_norm(x, weight, eps)
    want, far = T.turned(y, far, positions, axes, freqs.cpu().numpy(), layout, magnitude)
    off = np.abs(R.host(got) - want)
    assert (off <= far).all(), (np.nanmax(off / far), np.unravel_index(np.argmax(~(off <= far)), off.shape))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("tokens,heads,kv,d,rot", [(1, 1, 1, 64, 64), (33, 32, 8, 128, 128), (5, 5, 3, 256, 64), (7, 3, 2, 72, 72),
                                                   (9, 4, 4, 80, 20), (3, 7, 1, 16, 16), (4, 2, 2, 512, 512), (4, 1, 9, 510, 130),
                                                   (6, 2, 1, 2, 2), (11, 6, 5, 96, 0), (300, 1, 1, 128, 96)])
def test_shapes(tokens, heads, kv, d, rot, layout):
    import paper_2509_26436_amd as q
    print(f"head norms {tokens} x {heads} + {kv} x {d}, {rot} turned, {layout}", flush=True)
    g = T.rng(1, tokens, heads, d, rot)
    x = [R.bf16(g.normal(0, 1, (tokens, n, d)) * np.exp(g.normal(0, 2, (tokens, n, 1)))) for n in (heads, kv)]
    w = [R.bf16(1 + 0.3 * g.normal(size=d)) for _ in range(2)]
    p, freqs = g.integers(-(1 << 31), (1 << 31) - 1, tokens), q.rotary_frequencies(rot)
    out = q.head_norm_rotary(R.device(x[0]), R.device(x[1]), T.int32(p), freqs, R.device(w[0]), R.device(w[1]), layout=layout)
    for i in range(2):
        _check(out[i], x[i], w[i], 1e-6, [p], [0] * (rot // 2), freqs, layout)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,parts", [(128, (16, 56, 56)), (64, (20, 22)), (72, (24, 24, 24)), (128, (32, 32, 32, 30))])
def test_axes(d, parts, layout):
    """Frequencies of each axis' own pairs one after the other; an axis that is none leaves its pairs."""
    import torch
    import paper_2509_26436_amd as q
    g = T.rng(2, d)
    tokens, heads = 21, 6
    freqs = torch.cat([q.rotary_frequencies(n) for n in parts])
    axes = np.repeat(np.arange(len(parts)), [n // 2 for n in parts])
    axes[-1] = 77
    axes[1] = -1
    p = g.integers(0, 1 << 20, (len(parts), tokens + 4))
    x, w = R.bf16(g.normal(0, 2, (tokens, heads, d))), R.bf16(1 + 0.3 * g.normal(size=d))
    y, none = q.head_norm_rotary(R.device(x), None, T.int32(p)[:, 2:-2], freqs, R.device(w), eps=1e-5, axes=T.int32(axes),
                                 layout=layout, magnitude=1.25)
    assert none is None
    _check(y, x, w, 1e-5, p[:, 2:-2], axes, freqs, layout, 1.25)


@pytest.mark.parametrize("eps,weighted", [(None, False), (1e-6, False), (0.0, True), (0.5, True)])
def test_without_norm_or_weights(eps, weighted):
    import paper_2509_26436_amd as q
    g = T.rng(3)
    x, w = R.bf16(g.normal(0, 1e-3, (10, 3, 128))), R.bf16(g.normal(size=128))
    p, freqs = g.integers(0, 5000, 10), q.rotary_frequencies(128)
    y, _ = q.head_norm_rotary(R.device(x), None, T.int32(p), freqs, R.device(w) if weighted else None, eps=eps)
    _check(y, x, w if weighted else None, eps, [p], [0] * 64, freqs, "half")
    if eps is None:
        import torch
        assert torch.equal(y, q.rotary(R.device(x), T.int32(p), freqs))


@pytest.mark.parametrize("offset", [0, 1, 2, 8])
def test_views_of_one_projection(offset):
    """Queries and keys side by side in one tensor: read in place, written beside it and in place."""
    import torch
    import paper_2509_26436_amd as q
    g = T.rng(4)
    tokens, H, KV, d = 19, 6, 2, 128
    flat = torch.zeros(tokens * ((H + 2 * KV) * d + offset) + offset, device="cuda", dtype=torch.bfloat16)
    qkv = flat.as_strided((tokens, H + 2 * KV, d), ((H + 2 * KV) * d + offset, d, 1), offset)
    x = R.bf16(g.normal(0, 1, qkv.shape))
    qkv.copy_(R.device(x))
    w = [R.bf16(1 + 0.3 * g.normal(size=d)) for _ in range(2)]
    p, freqs = g.integers(0, 9000, tokens), q.rotary_frequencies(d)
    args = T.int32(p), freqs, R.device(w[0]), R.device(w[1])
    out = torch.zeros(H, tokens, d, device="cuda", dtype=torch.bfloat16).transpose(0, 1)     # head by head
    a, b = q.head_norm_rotary(qkv[:, :H], qkv[:, H:H + KV], *args, out=(out, None))
    assert a.data_ptr() == out.data_ptr()
    q.head_norm_rotary(qkv[:, :H], qkv[:, H:H + KV], *args, out=(qkv[:, :H], qkv[:, H:H + KV]))
    assert torch.equal(qkv[:, :H], a) and torch.equal(qkv[:, H:H + KV], b)
    assert np.array_equal(R.host(qkv[:, H + KV:]), x[:, H + KV:])
    _check(a, x[:, :H], w[0], 1e-6, [p], [0] * 64, freqs, "half")
    _check(b, x[:, H:H + KV], w[1], 1e-6, [p], [0] * 64, freqs, "half")


def test_infinities_nan_and_zero_heads():
    import torch
    import paper_2509_26436_amd as q
    x = torch.ones(4, 2, 64, device="cuda", dtype=torch.bfloat16)
    x[0, 0, 3], x[1, 1, 5], x[2, 0] = float("nan"), float("inf"), 0.0
    y, _ = q.head_norm_rotary(x, None, T.int32([0, 1, 2, 3]), q.rotary_frequencies(64))
    assert y[0, 0].isnan().all() and y[1, 1].isnan().any() and (y[2, 0] == 0).all()
    y[0, 0] = y[1, 1] = 0
    assert y.isfinite().all()


def test_nothing_to_do_and_graphs():
    import torch
    import paper_2509_26436_amd as q
    freqs = q.rotary_frequencies(64)
    none = torch.empty(0, 2, 64, device="cuda", dtype=torch.bfloat16)
    assert q.head_norm_rotary(none, none, T.int32([]), freqs)[0].shape == (0, 2, 64)
    g = T.rng(5)
    x, p = R.device(R.bf16(g.normal(size=(8, 4, 64)))), T.int32(np.arange(8))
    out = torch.empty_like(x)
    q.head_norm_rotary(x, None, p, freqs, out=(out, None))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q.head_norm_rotary(x, None, p, freqs, out=(out, None))
    for i in range(3):
        p.copy_(T.int32(np.arange(8) * 7 * i))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, q.head_norm_rotary(x, None, p, freqs)[0])
