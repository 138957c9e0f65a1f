"""MXFP4 quantizer, decoder and linear layer against the format's definition in 64 bits: codes,
scales and decoded values exactly, the layer within its bf16 rounding and fp32 sums."""
import numpy as np
import pytest

import decoding_reference as R

pytestmark = pytest.mark.gpu


def _rng(*seed):
    return np.random.Generator(np.random.PCG64(list(seed)))


def _tokens(rng, M, K, spread=4.0):
    x = rng.normal(0, 1, (M, K)) * np.exp2(rng.uniform(-spread, spread, (M, K)))
    x[:, rng.integers(0, K, 2)] *= 40.0
    return R.bf16(x)


def _tensor(code, byte):
    import torch
    import paper_2509_26436_amd as q
    codes, scales = R.mx_pack(code, byte)
    return q.MxTensor(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), *code.shape)


def _check_codes(t, code, byte):
    codes, scales = R.mx_pack(code, byte)
    good = np.repeat(byte != 255, 16, axis=1).reshape(code.shape[0], -1, 16).transpose(1, 0, 2)
    np.testing.assert_array_equal(np.where(good, t.codes.cpu().numpy(), 0), np.where(good, codes, 0))
    K = code.shape[1]
    got = t.scales.cpu().numpy().transpose(1, 0, 2).reshape(code.shape[0], -1)[:, :K // 32]
    np.testing.assert_array_equal(got, byte)


@pytest.mark.parametrize("M,K", [(1, 64), (1, 4096), (15, 192), (16, 128), (17, 1088), (33, 320), (257, 64)])
def test_quantize(M, K):
    import paper_2509_26436_amd as q
    print(f"mxfp4 quantize {M} x {K}", flush=True)
    x = _tokens(_rng(1, M, K), M, K)
    x[M // 2, :64] = 0.0
    code, byte = R.mx_quantize(x)
    t = q.mxfp4_quantize(R.device(x))
    _check_codes(t, code, byte)
    np.testing.assert_array_equal(R.host(q.mxfp4_dequantize(t)), R.mx_values(code, byte))


def test_every_bf16_value_as_maximum_and_beside_one():
    """Each finite bf16 magnitude as a block's maximum, with values around the rounding borders of
    its block, and each infinity and NaN."""
    import torch
    import paper_2509_26436_amd as q
    bits = np.arange(0x8000, dtype=np.uint32)
    top = (bits << 16).view(np.float32).astype(np.float64)
    x = np.zeros((bits.size, 64))
    x[:, 0] = top
    finite = np.isfinite(top)
    for i in range(1, 32):
        x[finite, i] = R.bf16(top[finite] * i / 32) * (-1) ** i
    x[:, 32:] = np.where(np.isfinite(x[:, :32]), -x[:, :32], 1.0)   # a block without the NaN
    code, byte = R.mx_quantize(x)
    raw = (x.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    raw[:, 0] = bits
    t = q.mxfp4_quantize(torch.from_numpy(raw.view(np.int16)).cuda().view(torch.bfloat16))
    assert (byte[~finite, 0] == 255).all()
    _check_codes(t, code, byte)
    got = R.host(q.mxfp4_dequantize(t))
    np.testing.assert_array_equal(np.isnan(got[:, :32]), np.repeat(~finite[:, None], 32, 1))
    np.testing.assert_array_equal(got[finite], R.mx_values(code, byte)[finite])


def test_decode_every_code_and_scale():
    import paper_2509_26436_amd as q
    code = np.tile(np.arange(64) % 16, (256, 1))
    byte = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 2, 1)
    want = R.mx_values(code, byte)
    want[np.abs(want) >= 2.0 ** 128] *= np.inf      # past bf16's range
    np.testing.assert_array_equal(R.host(q.mxfp4_dequantize(_tensor(code, byte))), want)


def test_strides_and_what_is_beside():
    """Rows of a wider tensor in, rows of a wider tensor out; nothing else is touched."""
    import torch
    import paper_2509_26436_amd as q
    x = _tokens(_rng(2), 19, 256)
    wide = R.device(x)[:, 64:192]
    code, byte = R.mx_quantize(x[:, 64:192])
    t = q.mxfp4_quantize(wide)
    _check_codes(t, code, byte)
    out = torch.full((21, 144), 7.0, dtype=torch.bfloat16, device="cuda")
    q.mxfp4_dequantize(t, out=out[1:20, 8:136])
    want = np.full((21, 144), 7.0)
    want[1:20, 8:136] = R.mx_values(code, byte)
    np.testing.assert_array_equal(R.host(out), want)


SHAPES = [(1, 1, 64), (1, 17, 64), (1, 4096, 1088), (3, 100, 192), (16, 33, 256), (17, 250, 320), (31, 1000, 2048),
          (64, 64, 64), (65, 66, 128), (130, 129, 1152), (333, 1000, 576), (257, 3, 448)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("act,with_bias", [(0, True), (1, True), (0, False)])
def test_linear(M, N, K, act, with_bias):
    """From bf16 and from an MxTensor, into a wider output whose other columns stay."""
    import torch
    import paper_2509_26436_amd as q
    print(f"mxfp4 linear {M} x {N} x {K} act {act} bias {with_bias}", flush=True)
    rng = _rng(3, M, N, K)
    x = _tokens(rng, M, K, 1.0)
    a = R.mx_values(*R.mx_quantize(x))
    wc, wb = R.mx_quantize(R.bf16(rng.normal(0, 0.05, (N, K))))
    bias = R.bf16(rng.normal(0, 1, N)) if with_bias else None
    y, far = R.linear(a, R.mx_values(wc, wb), bias, act)
    w, b = _tensor(wc, wb), None if bias is None else R.device(bias)
    for given in (R.device(x), q.mxfp4_quantize(R.device(x))):
        got = q.mxfp4_linear(given, w, b, act)
        assert got.shape == (M, N)
        assert (np.abs(R.host(got) - y) <= far).all(), np.abs(R.host(got) - y).max()
        out = torch.full((M, N + 9), 5.0, dtype=torch.bfloat16, device="cuda")
        q.mxfp4_linear(given, w, b, act, out=out[:, :N])
        np.testing.assert_array_equal(R.host(out[:, :N]), R.host(got))
        assert (out[:, N:] == 5.0).all()


@pytest.mark.parametrize("M,N,K,tile", [(2048, 2048, 256, (128, 128)), (1999, 2100, 320, (128, 128)),
                                        (4090, 4093, 64, (128, 128)), (4000, 1100, 2112, (128, 128)),
                                        (4090, 4093, 1216, (256, 256)), (4090, 4093, 2048, (256, 256)),
                                        (2304, 4100, 1152, (192, 256)), (2300, 4100, 448, (192, 256)),
                                        (4600, 8190, 448, (128, 128)),
                                        (8190, 4599, 832, (256, 192)),
                                        (200, 4000, 2112, (32, 32)), (300, 3001, 4096, (64, 64))])
def test_linear_large(M, N, K, tile):
    """Sizes of the larger tiles, ragged, with K of one step, shorter than the ring of stages, and with
    a last stage of one step; sampled rows."""
    import paper_2509_26436_amd as q
    kernel = q.mxfp4_linear_kernel(M, N, K)
    assert (kernel["rows"], kernel["cols"]) == tile
    print(f"mxfp4 large {M} x {N} x {K}", flush=True)
    rng = _rng(4, M, N, K)
    x = _tokens(rng, M, K, 1.0)
    wc, wb = R.mx_quantize(R.bf16(rng.normal(0, 0.05, (N, K))))
    bias = R.bf16(rng.normal(0, 1, N))
    got = R.host(q.mxfp4_linear(R.device(x), _tensor(wc, wb), R.device(bias)))
    rows = np.unique(np.r_[0:3, M - 70:M, rng.integers(0, M, 200)])
    a = R.mx_values(*R.mx_quantize(x[rows]))
    y, far = R.linear(a, R.mx_values(wc, wb), bias)
    assert (np.abs(got[rows] - y) <= far).all()
    assert np.isfinite(got).all()


def test_exact_integers():
    """Codes of small integers: every sum is an integer below 256, so bf16 holds it exactly."""
    import paper_2509_26436_amd as q
    rng = _rng(5)
    for M, N, K in [(5, 300, 512), (40, 300, 512), (2100, 2100, 192)]:
        a = rng.choice([0, 0, 0, 0, 0, 1, -1], (M, K)) * 1.0
        a[:, ::32] = 4.0
        w = rng.choice([0, 0, 0, 1, -1], (N, K)) * 1.0
        w[:, ::32] = 0.0
        w[:, 5::32] = 4.0
        a[:, 5::32] = 0.0
        y = a @ w.T
        assert np.abs(y).max() < 256
        wt = q.mxfp4_quantize(R.device(w))
        np.testing.assert_array_equal(R.host(q.mxfp4_linear(R.device(a), wt)), y)


@pytest.mark.parametrize("M", [4, 40, 2304])
def test_nan_stays_in_its_row(M):
    import paper_2509_26436_amd as q
    rng = _rng(6, M)
    N, K = (2304, 256) if M > 1000 else (96, 256)
    x, w = _tokens(rng, M, K, 1.0), R.bf16(rng.normal(0, 0.05, (N, K)))
    x[M - 2, 77], w[3, 200] = np.nan, np.inf
    got = R.host(q.mxfp4_linear(R.device(x), q.mxfp4_quantize(R.device(w))))
    bad = np.zeros((M, N), bool)
    bad[M - 2] = bad[:, 3] = True
    np.testing.assert_array_equal(np.isnan(got), bad)


def test_nothing_to_do():
    import torch
    import paper_2509_26436_amd as q
    x = torch.empty((0, 128), dtype=torch.bfloat16, device="cuda")
    w = q.mxfp4_quantize(torch.ones((5, 128), dtype=torch.bfloat16, device="cuda"))
    assert q.mxfp4_linear(x, w).shape == (0, 5)
    assert q.mxfp4_dequantize(q.mxfp4_quantize(x)).shape == (0, 128)
    assert q.mxfp4_linear(torch.ones((3, 128), dtype=torch.bfloat16, device="cuda"), q.mxfp4_quantize(x)).shape == (3, 0)


@pytest.mark.parametrize("M", [1, 100, 2100])
def test_graph_stream_and_shared_workspace(M):
    """Captured on another stream with the caller's workspace, replayed with new activations
    between eager calls that use the same workspace."""
    import torch
    import paper_2509_26436_amd as q
    rng = _rng(7, M)
    N, K = 2112, 320
    w = q.mxfp4_quantize(R.device(R.bf16(rng.normal(0, 0.05, (N, K)))))
    xs = [R.device(_tokens(rng, M, K, 1.0)) for _ in range(3)]
    want = [q.mxfp4_linear(x, w) for x in xs]
    x, ws = xs[0].clone(), q.mxfp4_workspace(M, K, "cuda")
    out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    q.mxfp4_linear(x, w, out=out, stream=stream, workspace=ws)
    stream.synchronize()
    assert torch.equal(out, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q.mxfp4_linear(x, w, out=out, workspace=ws)
    for i in (1, 2, 0, 1):
        x.copy_(xs[i])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
        assert torch.equal(q.mxfp4_linear(xs[i - 1], w, workspace=ws), want[i - 1])


@pytest.mark.parametrize("M,K,kernel", [(65535 * 32, 64, "direct"), (65535 * 32 + 1, 64, "tiled"),
                                        ((1 << 32) // 512 + 40, 1024, "tiled")])
def test_very_many_tokens(M, K, kernel):
    """As many tokens as a direct kernel's grid holds, one more, and codes past 2^32 bytes: rows from
    all over against the same rows by themselves."""
    import torch
    import paper_2509_26436_amd as q
    print(f"mxfp4 {M} tokens x {K}", flush=True)
    assert q.mxfp4_linear_kernel(M, 20, K)["kernel"] == kernel
    rng = _rng(8, M)
    rows = np.unique(np.r_[0:40, M - 60:M, rng.integers(0, M, 100)])
    some = R.device(_tokens(rng, len(rows), K, 1.0))
    at = torch.from_numpy(rows).cuda()
    x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    x[at] = some
    w = q.mxfp4_quantize(R.device(R.bf16(rng.normal(0, 0.05, (20, K)))))
    bias = R.device(R.bf16(rng.normal(0, 1, 20)))
    t, few = q.mxfp4_quantize(x), q.mxfp4_quantize(some)
    assert torch.equal(t.codes[:, at], few.codes) and torch.equal(t.scales[:, at], few.scales)
    y, want = q.mxfp4_linear(t, w, bias), q.mxfp4_linear(few, w, bias)
    # the kernels differ in the order of their sums, which fp32 rounds: at most K 2^-24 of the
    # products' magnitudes, then one rounding to bf16 on either side
    far = (q.mxfp4_dequantize(few).double().abs() @ q.mxfp4_dequantize(w).double().abs().T + bias.double().abs()) * K * 2.0 ** -23
    off = (y[at].double() - want.double()).abs()
    assert (off <= far + want.double().abs() * 2.0 ** -7 + far * 2.0 ** -7).all()
    del x
    back = q.mxfp4_dequantize(t)
    assert torch.equal(back[at], q.mxfp4_dequantize(few))
    mask = torch.ones(M, dtype=torch.bool, device="cuda")
    mask[at] = False
    assert not back.view(torch.int16).any(1).logical_and(mask).any()
    assert (y[mask][:1000] == bias).all()
