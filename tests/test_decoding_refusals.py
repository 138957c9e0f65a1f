"""The decoding entry points refuse wrong arguments on the host, before anything is launched (no
GPU is needed), and the tensor helpers refuse wrong tensors."""
import math
import os

import pytest

import paper_2509_26436_amd as q

OK, ENULL, ESHAPE, EUNSUP, EALIGN, EWS = 0, 1, 2, 3, 4, 6
A = 4096      # a fake, 16-byte aligned address: never dereferenced on these paths


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(q.library_path()):
        pytest.skip("libquartz.so not built")
    return q.load()


def test_mxfp4_quantize_and_dequantize():
    def quantize(x=A, M=4, K=128, ldx=128, codes=A, scales=A):
        return q.quartz_mxfp4_quantize(x, M, K, ldx, codes, scales, None)

    def dequantize(x=A, M=4, K=128, ldx=128, codes=A, scales=A):
        return q.quartz_mxfp4_dequantize(codes, scales, M, K, x, ldx, None)
    for f in (quantize, dequantize):
        assert f(K=96) == f(K=32) == f(M=-1) == f(ldx=64) == f(ldx=(1 << 24) + 8) == ESHAPE
        assert f(K=1 << 21, ldx=1 << 21) == f(M=(1 << 28) + 1, K=64) == ESHAPE
        assert f(ldx=132) == f(x=A + 2) == f(codes=A + 8) == f(scales=A + 4) == EALIGN
        assert f(x=None) == f(codes=None) == f(scales=None) == ENULL
        assert f(M=0, x=None, codes=None, scales=None) == f(K=0, ldx=0) == OK


def test_mxfp4_linear():
    def call(ac=A, asc=A, wc=A, ws=A, bias=None, y=A, M=8, N=8, K=128, ldy=8, epi=0):
        return q.quartz_mxfp4_linear(ac, asc, wc, ws, bias, y, M, N, K, ldy, epi, None)
    assert call(epi=2) == call(epi=-1) == EUNSUP
    assert call(K=0) == call(K=96) == call(M=-1) == call(N=-1) == call(ldy=7) == call(ldy=1 << 25) == ESHAPE
    assert call(M=1 << 28, N=1 << 24, K=64, ldy=1 << 24) == ESHAPE
    for name in ("ac", "asc", "wc", "ws", "y"):
        assert call(**{name: None}) == ENULL
        assert call(**{name: A + 8}) == EALIGN
    assert call(bias=A + 2) == EALIGN
    assert call(M=0) == call(N=0, ldy=0) == OK


def test_mxfp4_linear_from_bf16():
    def call(x=A, ldx=128, wc=A, ws=A, bias=None, y=A, M=40, N=8, K=128, ldy=8, epi=0, work=A, size=None):
        size = q.quartz_mxfp4_linear_workspace_bytes(M, K) if size is None else size
        return q.quartz_mxfp4_linear_bf16(x, ldx, wc, ws, bias, y, M, N, K, ldy, epi, work, size, None)
    assert q.quartz_mxfp4_linear_workspace_bytes(40, 128) == 40 * 64 + 40 * 4
    for M, K in ((0, 128), (1, 128), (-4, 128), (40, 100), (40, 1 << 21)):
        assert q.quartz_mxfp4_linear_workspace_bytes(M, K) == 0
    assert call(epi=3) == EUNSUP
    assert call(K=100) == call(ldx=64) == call(ldx=1 << 25) == call(ldy=4) == ESHAPE
    assert call(ldx=132) == call(x=A + 4) == call(work=A + 8) == EALIGN
    assert call(x=None) == call(wc=None) == call(ws=None) == call(y=None) == ENULL
    assert call(work=None) == call(size=0) == call(size=40 * 68 - 1) == EWS
    assert call(M=0, size=0, work=None) == call(N=0, ldy=0) == OK


def test_mxfp4_linear_kernel():
    """Every kernel is some size's, and which: direct blocks for few tokens, tiles for many."""
    for M, N, K, kernel, rows, cols, fused in (
            (1, 4096, 4096, "direct", 16, 16, True), (8, 4096, 4096, "direct", 16, 16, True),
            (8, 4096, 4160, "direct", 16, 16, False), (9, 4096, 64, "direct", 16, 16, False),
            (64, 4096, 4096, "direct", 32, 32, False), (256, 4096, 4096, "direct", 64, 64, False),
            (1024, 4096, 4096, "tiled", 128, 128, False), (4096, 4096, 4096, "tiled", 256, 256, False),
            (4608, 8192, 8192, "tiled", 192, 256, False), (8192, 4608, 8192, "tiled", 256, 192, False)):
        assert q.mxfp4_linear_kernel(M, N, K) == {"kernel": kernel, "rows": rows, "cols": cols, "fused": fused}
    # more tokens than a direct kernel's grid holds
    for M in (1 << 22, 1 << 28):
        assert q.mxfp4_linear_kernel(M, 16, 64)["kernel"] == "tiled"
    assert q.quartz_mxfp4_linear_kernel(0, 8, 64, A) == q.quartz_mxfp4_linear_kernel(8, 8, 96, A) == ESHAPE
    assert q.quartz_mxfp4_linear_kernel(8, 8, 64, None) == ENULL


def test_rotary():
    def call(x=A, y=1 << 20, T=4, H=2, d=64, rot=64, xt=128, xh=64, yt=128, yh=64, pos=A, f=A, layout=0,
             inverse=0, magnitude=1.0):
        return q.quartz_rotary(x, y, T, H, d, rot, xt, xh, yt, yh, pos, f, layout, inverse, magnitude, None)
    assert call(layout=2) == call(layout=-1) == call(magnitude=math.inf) == call(magnitude=math.nan) == EUNSUP
    assert call(d=63, rot=0) == call(rot=3) == call(rot=66) == call(rot=-2) == call(d=0, rot=0) == ESHAPE
    assert call(T=-1) == call(H=-1) == call(T=1 << 32, H=64) == call(xt=1 << 41) == call(yh=-(1 << 41)) == ESHAPE
    assert call(x=None) == call(y=None) == call(pos=None) == call(f=None) == ENULL
    assert call(x=A + 1) == call(y=(1 << 20) + 1) == call(pos=A + 2) == call(f=A + 4) == EALIGN
    assert call(y=A, yt=64) == ESHAPE          # in place with other strides
    assert call(T=0, x=None) == call(H=0, pos=None) == OK


CACHE = dict(kc=A, vc=A, type=0, ks=1.0, vs=1.0, pages=4, page=16, stride=16 * 2 * 128, table=A)


def _append(k=A, v=A, T=4, H=2, d=128, kt=256, kh=128, vt=256, vh=128, pos=A, seq=A, f=A, rot=128, layout=0,
            magnitude=1.0, rows=3, width=4, row=4, **over):
    c = dict(CACHE, **over)
    return q.quartz_paged_append(k, v, T, H, d, kt, kh, vt, vh, pos, seq, f, rot, layout, magnitude, c["kc"], c["vc"],
                                 c["type"], c["ks"], c["vs"], c["pages"], c["page"], c["stride"], c["table"], rows,
                                 width, row, None)


def _attend(x=A, o=A, S=3, H=8, kv=2, d=128, qt=1024, qh=128, ot=1024, oh=128, lengths=A, scale=0.1, window=0, width=4,
            row=4, work=None, size=0, **over):
    c = dict(CACHE, **over)
    return q.quartz_paged_attention(x, o, S, H, kv, d, qt, qh, ot, oh, c["kc"], c["vc"], c["type"], c["ks"], c["vs"],
                                    c["pages"], c["page"], c["stride"], c["table"], width, row, lengths, scale, window,
                                    work, size, None)


@pytest.mark.parametrize("call", [_append, _attend])
def test_cache(call):
    assert call(type=2) == call(ks=0.0) == call(vs=-1.0) == call(ks=math.nan) == call(vs=math.inf) == EUNSUP
    assert call(ks=1e-40) == call(page=12) == call(page=4) == call(page=8192) == call(page=0) == call(page=-16) == EUNSUP
    assert call(page=1 << 62) == call(page=-(1 << 63)) == EUNSUP
    assert call(pages=0) == call(pages=-1) == call(pages=1 << 31) == call(stride=16 * 2 * 128 - 8) == ESHAPE
    assert call(row=3) == call(width=-1) == call(width=1 << 27, row=1 << 27) == ESHAPE
    assert call(kc=None) == call(vc=None) == call(table=None) == ENULL
    assert call(kc=A + 8) == call(vc=A + 2) == call(table=A + 2) == call(stride=16 * 2 * 128 + 4) == EALIGN
    assert call(type=1, stride=16 * 2 * 128 + 8) == EALIGN


def test_append():
    assert _append(layout=5) == _append(magnitude=math.inf) == _append(d=96, rot=64) == _append(d=32, rot=0) == EUNSUP
    assert _append(T=-1) == _append(H=0) == _append(rot=130) == _append(rot=7) == _append(T=1 << 24) == ESHAPE
    assert _append(rows=-1) == _append(kt=1 << 41) == _append(vh=1 << 41) == ESHAPE
    assert _append(k=None) == _append(v=None) == _append(pos=None) == _append(f=None) == ENULL
    assert _append(k=A + 1) == _append(v=A + 1) == _append(pos=A + 1) == _append(seq=A + 2) == _append(f=A + 4) == EALIGN
    assert _append(T=0, k=None, v=None, kc=None) == _append(rows=0) == _append(width=0, row=0, table=None) == OK


def test_attention():
    need = q.quartz_paged_attention_workspace_bytes
    assert need(3, 8, 2, 128, 16, 4, 0) == 0                    # 64 positions: one block a head
    assert need(3, 8, 2, 128, 16, 4096, 0) > 0
    assert need(3, 8, 2, 128, 16, 4096, 64) <= need(3, 8, 2, 128, 16, 4096, 0)
    for bad in ((3, 8, 3, 128, 16, 4, 0), (3, 8, 2, 96, 16, 4, 0), (3, 8, 2, 128, 12, 4, 0), (-1, 8, 2, 128, 16, 4, 0),
                (3, 8, 0, 128, 16, 4, 0), (3, 8, 2, 128, 16, 4, -1), (3, 8, 2, 128, 16, 1 << 40, 0)):
        assert need(*bad) == 0
    assert _attend(scale=math.nan) == _attend(d=96) == EUNSUP
    assert _attend(S=-1) == _attend(kv=3) == _attend(kv=0) == _attend(H=1) == _attend(window=-1) == ESHAPE
    assert _attend(S=1 << 24, H=8) == _attend(qt=1 << 41) == _attend(oh=-(1 << 41)) == ESHAPE
    assert _attend(x=None) == _attend(o=None) == _attend(lengths=None) == ENULL
    assert _attend(x=A + 8) == _attend(o=A + 4) == _attend(lengths=A + 2) == _attend(work=A + 8) == EALIGN
    assert _attend(qt=1028) == _attend(qh=132) == _attend(ot=1026) == _attend(oh=126) == EALIGN
    size = need(3, 8, 2, 128, 16, 4096, 0)
    long = dict(width=4096, row=4096)
    assert _attend(**long) == _attend(**long, work=A, size=size - 1) == _attend(**long, size=size) == EWS
    assert _attend(S=0, x=None, o=None, kc=None) == OK


def test_rotary_frequencies():
    import numpy as np
    # the table's unit is 2^-64 turns, a rounding to it half of that beside the float64 steps: 1e-5 / 4
    # turns are off by up to 2^-65 / 2.5e-6 = 1.1e-14 of themselves
    unit = dict(atol=2.0 ** -65)
    host = lambda **kw: q.rotary_frequencies(device="cpu", **kw).numpy().astype(object)      # noqa: E731
    for rot, base in ((2, 10000.0), (20, 10000.0), (128, 500000.0), (64, 1.0)):
        want = [base ** (-2.0 * i / rot) / (2 * math.pi) for i in range(rot // 2)]
        got = [f / 2.0 ** 64 for f in host(rot=rot, base=base)]
        np.testing.assert_allclose(got, want, rtol=1e-15, **unit)
        np.testing.assert_allclose([f / 2.0 ** 64 for f in host(rot=rot, base=base, factor=4.0)],
                                   [w / 4 for w in want], rtol=1e-15, **unit)
        if rot > 2:
            big = base * 4.0 ** (rot / (rot - 2))
            np.testing.assert_allclose([f / 2.0 ** 64 for f in host(rot=rot, base=base, scaling="base", factor=4.0)],
                                       [big ** (-2.0 * i / rot) / (2 * math.pi) for i in range(rot // 2)], rtol=1e-14,
                                       **unit)
        parts = host(rot=rot, base=base, scaling="parts", factor=8.0, low=1.0, high=4.0, original=8192.0)
        for f, w in zip(parts, want):
            keep = min(max((8192 * w - 1) / 3, 0), 1)
            assert f / 2.0 ** 64 == pytest.approx(w * keep + w / 8 * (1 - keep), rel=1e-12, abs=2.0 ** -65)
    assert host(rot=0).size == 0
    f = q.quartz_rotary_frequencies
    assert f(8, 1e4, 3, 1.0, 1.0, 2.0, 1.0, A) == f(8, 0.5, 0, 1.0, 1.0, 2.0, 1.0, A) == EUNSUP
    assert f(8, math.nan, 0, 1.0, 1.0, 2.0, 1.0, A) == f(8, 1e4, 0, 0.5, 1.0, 2.0, 1.0, A) == EUNSUP
    assert f(8, 1e4, 2, 2.0, 2.0, 2.0, 1.0, A) == f(8, 1e4, 2, 2.0, 1.0, 2.0, 0.0, A) == EUNSUP
    assert f(7, 1e4, 0, 1.0, 1.0, 2.0, 1.0, A) == f(-2, 1e4, 0, 1.0, 1.0, 2.0, 1.0, A) == ESHAPE
    assert f(8, 1e4, 0, 1.0, 1.0, 2.0, 1.0, None) == ENULL
    assert f(0, 1e4, 0, 1.0, 1.0, 2.0, 1.0, None) == OK


def test_helpers_refuse_tensors():
    import torch
    bf16, i32 = torch.bfloat16, torch.int32
    x = torch.zeros((4, 128), dtype=bf16)
    codes, scales = torch.zeros((4, 8, 16), dtype=torch.uint8), torch.zeros((1, 8, 4), dtype=torch.uint8)
    w = q.MxTensor(codes, scales, 8, 128)
    heads = torch.zeros((4, 2, 128), dtype=bf16)
    pos, f = torch.zeros(4, dtype=i32), q.rotary_frequencies(128, device="cpu")
    k = torch.zeros((3, 2, 16, 128), dtype=bf16)
    table = torch.zeros((4, 2), dtype=i32)
    cache = q.PagedCache(k, k.clone(), table)
    wrong = [
        lambda: q.MxTensor(codes[:2], scales, 8, 128), lambda: q.MxTensor(codes, scales, 8, 100),
        lambda: q.MxTensor(codes.int(), scales, 8, 128), lambda: q.MxTensor(codes, scales[:, :4], 8, 128),
        lambda: q.mxfp4_quantize(x.float()), lambda: q.mxfp4_quantize(x[:, ::2]), lambda: q.mxfp4_quantize(x[:, :96]),
        lambda: q.mxfp4_quantize(x, out=w), lambda: q.mxfp4_dequantize(w, out=x),
        lambda: q.mxfp4_linear(x[:, :64], w), lambda: q.mxfp4_linear(x, w, bias=x[0]),
        lambda: q.mxfp4_linear(x, w, out=x[:, :4]), lambda: q.mxfp4_linear(x.half(), w),
        lambda: q.rotary_frequencies(64, scaling="other", device="cpu"),
        lambda: q.rotary(x, pos, f), lambda: q.rotary(heads.float(), pos, f), lambda: q.rotary(heads, pos.long(), f),
        lambda: q.rotary(heads, pos[:3], f), lambda: q.rotary(heads, pos, f.double()),
        lambda: q.rotary(heads[:, :, :64], pos, f), lambda: q.rotary(heads, pos, f, "both"),
        lambda: q.rotary(heads, pos, f, out=heads[:3]), lambda: q.rotary(heads[:, :, ::2], pos, f[:8]),
        lambda: q.PagedCache(k, k.half(), table), lambda: q.PagedCache(k, k[:2], table),
        lambda: q.PagedCache(k, k, table.long()), lambda: q.PagedCache(k, k, table[0]),
        lambda: q.PagedCache(k.transpose(1, 2), k.transpose(1, 2), table), lambda: q.PagedCache(k.float(), k.float(), table),
        lambda: q.paged_append(cache, heads[:, :1], heads[:, :1], pos), lambda: q.paged_append(cache, heads, heads, pos[:2]),
        lambda: q.paged_append(cache, heads, heads[:3], pos), lambda: q.paged_append(cache, heads, heads, pos, pos.long()),
        lambda: q.paged_attention(heads[:3], cache, pos[:3]), lambda: q.paged_attention(heads[:, :, :64], cache, pos),
        lambda: q.paged_attention(heads[:, :1], cache, pos), lambda: q.paged_attention(heads, cache, pos.long()),
        lambda: q.paged_attention(heads, cache, pos, out=heads[:, :1]),
        # tensors that are not on a GPU
        lambda: q.mxfp4_quantize(x), lambda: q.mxfp4_dequantize(w), lambda: q.mxfp4_linear(x, w),
        lambda: q.rotary(heads, pos, f), lambda: q.paged_append(cache, heads, heads, pos),
        lambda: q.paged_attention(heads, cache, pos)]
    for i, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            print("not refused:", i)
    with pytest.raises(q.QuartzError):
        q.rotary_frequencies(64, factor=0.5, device="cpu")


def test_helpers_refuse_shared_memory():
    """Outputs that hold an element twice, or that are an input's memory; epilogues past 32 bits."""
    import torch
    x = torch.zeros((8, 128), dtype=torch.bfloat16)
    codes, scales = torch.zeros((4, 8, 16), dtype=torch.uint8), torch.zeros((1, 8, 4), dtype=torch.uint8)
    w, other = q.MxTensor(codes, scales, 8, 128), q.MxTensor(codes.clone(), scales.clone(), 8, 128)
    heads = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    pos, f = torch.zeros(4, dtype=torch.int32), q.rotary_frequencies(128, device="cpu")
    k = torch.zeros((3, 2, 16, 128), dtype=torch.bfloat16)
    cache = q.PagedCache(k, k.clone(), torch.zeros((4, 2), dtype=torch.int32))
    x16 = codes.view(-1).view(torch.bfloat16)
    wrong = [
        (lambda: q.mxfp4_linear(x, w, out=x), "share"), (lambda: q.mxfp4_linear(other, w, out=x[:1].expand(8, 128)), "twice"),
        (lambda: q.mxfp4_linear(x, w, epilogue=2 ** 32), "range"), (lambda: q.mxfp4_linear(other, w, epilogue=2 ** 32), "range"),
        (lambda: q.mxfp4_linear(other, w, out=x16[:64].view(8, 8)), "share"),
        (lambda: q.mxfp4_quantize(x16.view(2, 128), out=q.MxTensor(codes.view(-1)[:128].view(4, 2, 16), scales[:, :2].clone(), 2, 128)), "share"),
        (lambda: q.mxfp4_dequantize(q.MxTensor(codes[:, :2].clone(), scales[:, :2], 2, 128), out=torch.zeros(1, dtype=torch.bfloat16).expand(2, 128)), "twice|stride"),
        (lambda: q.rotary(heads, pos, f, out=heads[:1].expand(4, 2, 128)), "twice"),
        (lambda: q.rotary(heads[:1].expand(4, 2, 128), pos, f, out=heads[:1].expand(4, 2, 128)), "twice"),
        (lambda: q.rotary(heads.view(-1)[:512].view(2, 2, 128), pos[:2], f, out=heads.view(-1)[8:520].view(2, 2, 128)), "share"),
        (lambda: q.paged_attention(heads, cache, pos, out=heads), "share"),
        (lambda: q.paged_attention(heads, cache, pos, out=torch.zeros_like(heads[:, :1]).expand(4, 2, 128)), "twice"),
        (lambda: q.paged_attention(heads, cache, pos, out=k[0].view(-1)[:1024].view(4, 2, 128)), "share")]
    for i, (call, why) in enumerate(wrong):
        print("refused?", i)
        with pytest.raises(ValueError, match=why):
            call()


def test_helpers_take_empty_tensors_of_any_strides():
    """Strides of tensors without elements say nothing: the refusal that is left is the missing GPU."""
    import torch
    none = torch.empty_strided((0, 8), (0, 0), dtype=torch.int32)
    k = torch.zeros((3, 2, 16, 128), dtype=torch.bfloat16)
    cache = q.PagedCache(k, k.clone(), none)
    q.PagedCache(k, k.clone(), torch.empty_strided((4, 0), (0, 0), dtype=torch.int32))
    heads = torch.empty_strided((0, 2, 128), (0, 0, 0), dtype=torch.bfloat16)
    pos, f = torch.zeros(0, dtype=torch.int32), q.rotary_frequencies(128, device="cpu")
    for call in (lambda: q.mxfp4_quantize(torch.empty_strided((0, 128), (0, 0), dtype=torch.bfloat16)),
                 lambda: q.rotary(heads, pos, f), lambda: q.paged_append(cache, heads, heads, pos),
                 lambda: q.paged_attention(heads, cache, pos)):
        with pytest.raises(ValueError, match="on a GPU"):
            call()
