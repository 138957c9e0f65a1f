"""MXFP4 quantizer and decoder past the size from which inputs are read around the caches: the same
bits as of its rows in parts, which the tests of small sizes hold against the definition."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,K,extra", [(5203, 8256, 0), (41, 1 << 20, 8), (700001, 64, 0)])
def test_large_inputs_equal_their_parts(M, K, extra):
    import torch
    import paper_2509_26436_amd as q
    print(f"mxfp4 {M} x {K}", flush=True)
    assert M * K > 5 << 23
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randn((M, K + extra), generator=g, device="cuda").mul_(3).bfloat16()[:, :K]
    x[M // 2, :64], x[M - 1, K - 1] = 0.0, float("inf")
    t = q.mxfp4_quantize(x)
    y = q.mxfp4_dequantize(t)
    step = max(1, (1 << 22) // K)
    for at in range(0, M, step):
        part = q.mxfp4_quantize(x[at:at + step])
        assert torch.equal(t.codes[:, at:at + step], part.codes) and torch.equal(t.scales[:, at:at + step], part.scales)
        got, want = y[at:at + step], q.mxfp4_dequantize(part)
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))
    assert y[M - 1, K - 32:].isnan().all() and (y[M // 2, :64] == 0).all()
