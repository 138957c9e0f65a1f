"""Attention over the paged cache where small errors show: values that cancel under nearly equal
weights, against the definition in 64 bits with bounds that count the steps in fp32."""
import math

import numpy as np
import pytest

import decoding_reference as R
import test_gpu_paged as P

pytestmark = pytest.mark.gpu


def _bounds(q, k, v, scale):
    """One sequence and cache head: (o, how far it may be) with weights that hold 16 bits or more."""
    n, d = k.shape
    s = scale * (q @ k.T)
    size = abs(scale) * (np.abs(q) @ np.abs(k).T)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    o, weight = p @ v, p @ np.abs(v)
    # the score's additions and three roundings; the exponent's argument, up to 128 in base 2, rounded
    # once more; a weight's own rounding to two bf16 parts (2^-16) in the product and in the sum; the
    # additions of n weighted values and of n weights
    off = ((d + 8) * R.ADD * size + 4 * 2.0 ** -24 * (np.abs(s) + 1)).max(-1, keepdims=True)
    far = weight * (2 * np.expm1(off) + 2 * 2.0 ** -16 + 2.0 ** -20 + 2 * (2 * n + 8) * R.ADD)
    # a weight under fp32's normal range may be zero (the largest is 1, so that the others' relative
    # bound says nothing there): at most 2^-126 of each value; an output there too
    far = far + 2.0 ** -126 * (np.abs(v).sum(0) + 1)
    return o, R.HALF_BF16 * np.abs(o) + (1 + R.HALF_BF16) * far


@pytest.mark.parametrize("width", [None, 4096])
@pytest.mark.parametrize("kv,group,d,fp8", [(2, 4, 128, False), (2, 4, 128, True), (1, 3, 64, False),
                                            (3, 1, 64, True), (1, 20, 256, False), (1, 2, 256, True)])
def test_weights_of_cancelling_values(kv, group, d, fp8, width):
    """Neighbouring keys hold a value and its negative under weights that differ a little: what is
    left is the weights' difference, which a weight rounded to bf16 (off by up to 2^-8) would lose."""
    import torch
    import paper_2509_26436_amd as q
    print(f"weights: {kv} x {group} x {d} fp8 {fp8} width {width}", flush=True)
    page, lengths = 16, [2, 300, 64, 500]
    rng, table, k, v, x, cache = P._attention_case(21, lengths, kv, group, d, page, fp8,
                                                   width=None if width is None else width // page)
    kh, vh = R.host(k), R.host(v)
    kh[..., 1:] = 0.0                      # one channel scores: its products are exact
    vh[:, :, 1::2] = -vh[:, :, ::2]
    for t, h in ((k, kh), (v, vh)):
        t.copy_(torch.from_numpy(h).cuda().to(torch.bfloat16).to(t.dtype))
    x[:, :, 0] = R.bf16(rng.uniform(0.3, 1.0, x.shape[:2]))
    scale = 0.25
    assert (q.paged_attention_workspace(len(lengths), kv * group, cache) is not None) == (width is not None)
    o = R.host(q.paged_attention(R.device(x), cache, P._int32(lengths), scale=scale))
    kh, vh = R.host(k), R.host(v)
    for b, n in enumerate(lengths):
        for h in range(kv):
            kk, vv = (P._gather(t, table, b, h, n, page) for t in (kh, vh))
            rows = slice(h * group, (h + 1) * group)
            want, far = _bounds(x[b, rows], kk, vv, scale)
            off = np.abs(o[b, rows] - want)
            assert (off <= far).all(), (b, h, n, (off / far).max())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("width", [None, 4096])
@pytest.mark.parametrize("k_scale,scale,size,v_scale,v_size", [
    (1.5 * 2.0 ** -126, 2.0 ** 124, 1.0, 2.0 ** -96, 2.0 ** 80), (3.3e38, 2.0 ** -127, 1.0, 3.3e38, 2.0 ** -100),
    (1.5 * 2.0 ** 126, 1.0, 2.0 ** -124, 1.5 * 2.0 ** 126, 2.0 ** -110), (0.0371, 2.0, 1.0, 1.1, 1.0)])
def test_scales_small_and_large(k_scale, scale, size, v_scale, v_size, width, fp8):
    """The smallest and largest scales that attention takes, under scores and values of ordinary
    size: only the product of the cache's and the caller's has to be an fp32 number."""
    import torch
    import paper_2509_26436_amd as q
    print(f"scales {k_scale} {scale} {v_scale} fp8 {fp8} width {width}", flush=True)
    page, lengths, kv, group, d = 16, [3, 300, 0, 500], 2, 2, 64
    k_scale, v_scale = (float(np.float32(s)) for s in (k_scale, v_scale))
    _, table, k, v, x, cache = P._attention_case(22, lengths, kv, group, d, page, fp8, k_scale=k_scale, v_scale=v_scale,
                                                 width=None if width is None else width // page)
    x = R.bf16(x * (size / 4))             # some of them subnormal
    v_size = min(max(v_size, 2.0 ** -6), 64.0) if fp8 else v_size        # within e4m3
    v.copy_(torch.from_numpy(R.host(v) * v_size).cuda().to(torch.bfloat16).to(v.dtype))
    o = R.host(q.paged_attention(R.device(x), cache, P._int32(lengths), scale=scale))
    kh, vh = R.host(k) * k_scale, R.host(v) * v_scale
    for b, n in enumerate(lengths):
        for h in range(kv):
            kk, vv = (P._gather(t, table, b, h, n, page) for t in (kh, vh))
            rows = slice(h * group, (h + 1) * group)
            if n == 0:
                assert (o[b, rows] == 0).all()
                continue
            want, far = _bounds(x[b, rows], kk, vv, scale)
            assert (np.abs(o[b, rows] - want) <= far).all(), (b, h, n)


@pytest.mark.parametrize("kv", [1, 3])
def test_a_small_scale_over_many_keys(kv):
    """250000 equal weights, whose sum is 2^18, under the smallest scale of values.  Every step but the
    division is exact, and bf16 holds the quotients."""
    import torch
    import paper_2509_26436_amd as q
    n, page, d, v_scale = 250000, 64, 64, 1.5 * 2.0 ** -96
    pages = -(-n // page)
    k = torch.zeros((pages, kv, page, d), dtype=torch.bfloat16, device="cuda")
    values = (1 + 0.25 * (torch.arange(d, device="cuda") % 4)) * 2.0 ** 80
    v = values.to(torch.bfloat16).expand(k.shape).contiguous()
    cache = q.PagedCache(k, v, torch.arange(pages, dtype=torch.int32, device="cuda")[None], 1.0, v_scale)
    x = torch.ones((1, kv, d), dtype=torch.bfloat16, device="cuda")
    o = q.paged_attention(x, cache, P._int32([n]))
    want = R.host(values) * v_scale
    np.testing.assert_array_equal(R.host(o), np.broadcast_to(want, (1, kv, d)))


@pytest.mark.parametrize("width", [None, 4096])
@pytest.mark.parametrize("lengths", [[1, 40, 0], [128, 7, 500]])
def test_the_lowest_scores(lengths, width):
    """Scores beside fp32's lowest number still count: equal ones average the values.  (In units of
    log2, which the kernel's scores have, -1.25 2^127 is -3.07e38.)  Scores of -inf alone give 0."""
    import torch
    import paper_2509_26436_amd as q
    page, d, kv = 16, 64, 2
    _, table, k, v, x, cache = P._attention_case(23, lengths, kv, 1, d, page, False,
                                                 width=None if width is None else width // page)
    k.zero_()
    k[:, 0, :, 5], k[:, 1, :, 5] = -1.25 * 2.0 ** 64, -math.inf
    x = np.zeros_like(x)
    x[..., 5] = 2.0 ** 63
    o = R.host(q.paged_attention(R.device(x), cache, P._int32(lengths), scale=1.0))
    vh = R.host(v)
    for b, n in enumerate(lengths):
        assert (o[b, 1] == 0).all()
        if n == 0:
            assert (o[b, 0] == 0).all()
            continue
        vv = P._gather(vh, table, b, 0, n, page)
        want, far = _bounds(np.zeros((1, d)), np.zeros((n, d)), vv, 1.0)          # equal weights
        assert (np.abs(o[b, 0] - want[0]) <= far[0]).all(), (b, n)
