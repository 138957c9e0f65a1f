"""More calls that the decoding entry points refuse on the host, before anything is launched."""
import os

import pytest

import paper_2509_26436_amd as q
from test_decoding_refusals import ESHAPE, EUNSUP, EWS, _append, _attend

LONG = dict(width=4096, row=4096)     # a call that would go on to ask for its workspace


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(q.library_path()):
        pytest.skip("libquartz.so not built")
    return q.load()


def test_attention_scales_out_of_fp32():
    """The scores' factor, scale k_scale log2(e), is one fp32 number, and v_scale over the sum of 2^30
    weights stays normal."""
    attend = lambda **kw: _attend(**LONG, **kw)                          # noqa: E731
    for ks, scale in ((3.3e38, 1.25), (3.3e38, 1.0), (2.0 ** 64, -2.0 ** 64), (2.0 ** -126, 0.1), (2.0 ** -100, 2.0 ** -30)):
        assert attend(ks=ks, scale=scale) == EUNSUP, (ks, scale)
    for ks, scale in ((3.3e38, 0.5), (2.0 ** -126, 1.0), (2.0 ** -126, 0.0), (2.0 ** 64, -2.0 ** 63), (3.3e38, 2.0 ** -140)):
        assert attend(ks=ks, scale=scale) == EWS, (ks, scale)
    assert attend(vs=2.0 ** -97) == attend(vs=2.0 ** -126) == EUNSUP
    assert attend(vs=2.0 ** -96) == attend(vs=3.3e38) == EWS


def _answer(call):
    """What a helper says of CPU tensors: the refusal of shared memory, or (after it) of the device."""
    with pytest.raises(ValueError) as e:
        call()
    for word in ("share memory", "twice", "on a GPU"):
        if word in str(e.value):
            return word
    raise AssertionError(str(e.value))


def test_outputs_that_overlap_strided_inputs():
    """Views of one tensor that reach a common element, whatever their strides, and views side by side,
    which do not."""
    import torch
    bf16 = torch.bfloat16
    x = torch.zeros((8, 128), dtype=bf16)
    w = q.MxTensor(torch.zeros((4, 8, 16), dtype=torch.uint8), torch.zeros((1, 8, 4), dtype=torch.uint8), 8, 128)
    wide = torch.zeros((8, 256), dtype=bf16)
    pos, f = torch.zeros(4, dtype=torch.int32), q.rotary_frequencies(64, device="cpu")
    rows = torch.zeros((4, 6, 64), dtype=bf16)
    k = torch.zeros((3, 2, 16, 64), dtype=bf16)
    cache = q.PagedCache(k, k.clone(), torch.zeros((4, 2), dtype=torch.int32))
    assert _answer(lambda: q.mxfp4_linear(x, w, out=x[:, :8])) == "share memory"
    assert _answer(lambda: q.mxfp4_linear(wide[:, :128], w, out=wide[:, 120:130])) == "share memory"
    assert _answer(lambda: q.mxfp4_linear(wide[:, :128], w, out=wide[:, 128:136])) == "on a GPU"
    assert _answer(lambda: q.paged_attention(rows[:, :2], cache, pos, out=rows[:, 1:3])) == "share memory"
    assert _answer(lambda: q.paged_attention(rows[:, :2], cache, pos, out=rows[:, 2:4])) == "on a GPU"
    assert _answer(lambda: q.rotary(rows[:, :3], pos, f, out=rows[:, 3:])) == "on a GPU"
    assert _answer(lambda: q.rotary(rows[:, :3], pos, f, out=rows[:, 2:5])) == "share memory"
    assert _answer(lambda: q.rotary(rows[:, :3], pos, f, out=rows[:, :3])) == "on a GPU"       # in place
    assert _answer(lambda: q.rotary(rows[:, ::2], pos, f, out=rows[:, 1::2])) == "on a GPU"
    assert _answer(lambda: q.rotary(rows[:, :3], pos, f, out=rows.as_strided((4, 3, 64), (64, 64, 1)))) == "twice"
    assert _answer(lambda: q.rotary(rows[:, :3], pos, f, out=torch.zeros(4 * 6 * 64 - 1, dtype=bf16).as_strided(
        (4, 3, 64), (384, 64, 1)))) == "on a GPU"


def test_overlaps_against_all_places():
    """Random strided outputs in one storage: the same answer as listing every place does."""
    import random
    import torch
    rng = random.Random(5)
    base = torch.zeros(400, dtype=torch.bfloat16)
    pos, f = torch.zeros(3, dtype=torch.int32), q.rotary_frequencies(2, device="cpu")

    def view(last):
        while True:
            size = [rng.randint(1, 5) for _ in range(3)]
            stride = [rng.choice([0, 1, 2, 3, 4, 5, 7, 8, 12, 20, 40]) for _ in range(3)]
            if last:
                size, stride = [3, *size[1:]], [*stride[:2], 1]
            at = rng.randint(0, 100)
            places = [at + sum(i * s for i, s in zip(index, stride)) for index in
                      [(a, b, c) for a in range(size[0]) for b in range(size[1]) for c in range(size[2])]]
            if max(places) < 400 and not (last and size[2] % 2):
                return base.as_strided(size, stride, at), places
    seen = {"share memory": 0, "twice": 0, "on a GPU": 0}
    for _ in range(3000):
        (x, xs), (out, outs) = view(True), view(False)
        want = "twice" if len(set(outs)) < len(outs) else "share memory" if set(xs) & set(outs) else "on a GPU"
        if x.data_ptr() == out.data_ptr() and x.shape == out.shape:
            continue                                     # may be in place
        assert _answer(lambda: q.rotary(x, pos, f, out=out)) == want, (x.shape, x.stride(), out.shape, out.stride())
        seen[want] += 1
    assert min(seen.values()) > 200, seen


def test_overlaps_of_different_types():
    """Codes of bytes and an output of 16-bit elements in one storage."""
    import random
    import torch
    rng = random.Random(6)
    raw = torch.zeros(4000, dtype=torch.uint8)
    for _ in range(300):
        rows, stride, at, out_at = rng.randint(1, 4), rng.choice([64, 72, 200]), rng.randint(0, 700), 2 * rng.randint(0, 700)
        t = q.MxTensor(raw[at:at + 32 * rows].view(2, rows, 16), torch.zeros((1, rows, 4), dtype=torch.uint8), rows, 64)
        out = raw[out_at:].view(torch.bfloat16).as_strided((rows, 24), (stride, 1))
        places = {out_at + 2 * (r * stride + c) + b for r in range(rows) for c in range(24) for b in range(2)}
        want = "share memory" if places & set(range(at, at + 32 * rows)) else "on a GPU"
        assert _answer(lambda: q.mxfp4_dequantize(t, out=out)) == want


def test_workspaces_that_are_an_input():
    import torch
    bf16 = torch.bfloat16
    x, bias = torch.zeros((40, 128), dtype=bf16), torch.zeros(2048, dtype=bf16)
    w = q.MxTensor(torch.zeros((4, 2048, 16), dtype=torch.uint8), torch.zeros((1, 2048, 4), dtype=torch.uint8), 2048, 128)
    for bad in (x, x[10:], w.codes, w.codes[2], w.scales, bias, x.view(torch.uint8).view(-1)[17:]):
        assert _answer(lambda: q.mxfp4_linear(x, w, bias, workspace=bad)) == "share memory"
        assert _answer(lambda: q.mxfp4_linear(x, w, bias, workspace=bad, out=torch.zeros((40, 2048), dtype=bf16))) == "share memory"
    raw = torch.zeros(40 * 256 + 4096, dtype=torch.uint8)          # beside x in one storage
    assert _answer(lambda: q.mxfp4_linear(raw[:40 * 256].view(bf16).view(40, 128), w, bias, workspace=raw[40 * 256:])) == "on a GPU"
    with pytest.raises(ValueError, match="contiguous"):
        q.mxfp4_linear(x, w, workspace=torch.zeros((40, 512), dtype=torch.uint8)[:, ::2])
    rows, lengths = torch.zeros((4, 2, 64), dtype=bf16), torch.zeros(4, dtype=torch.int32)
    k = torch.zeros((3, 2, 16, 64), dtype=bf16)
    cache = q.PagedCache(k, k.clone(), torch.zeros((4, 400), dtype=torch.int32))
    for bad in (rows, cache.k, cache.v[1], cache.table, lengths, cache.table[2:]):
        assert _answer(lambda: q.paged_attention(rows, cache, lengths, workspace=bad)) == "share memory"
    assert _answer(lambda: q.paged_attention(rows, cache, lengths, workspace=torch.zeros(9, dtype=torch.uint8))) == "on a GPU"


def test_append_into_its_own_inputs():
    """A cache whose keys are its values, and new rows, positions or a table in its pages."""
    import torch
    bf16, i32 = torch.bfloat16, torch.int32
    both = torch.zeros((3, 2, 2, 16, 64), dtype=bf16)
    k, v = both[:, 0], both[:, 1]
    table, pos, f = torch.zeros((4, 2), dtype=i32), torch.zeros(4, dtype=i32), q.rotary_frequencies(64, device="cpu")
    rows = torch.zeros((4, 2, 64), dtype=bf16)
    append = lambda k, v, table=table, new=(rows, rows), pos=pos, seq=None, f=f: _answer(           # noqa: E731
        lambda: q.paged_append(q.PagedCache(k, v, table), *new, pos, seq, f))
    assert append(k, v) == "on a GPU"                    # halves of one tensor
    assert append(k, v, new=(both.view(-1)[:512].view(4, 2, 64), rows)) == "share memory"
    assert append(k, v, new=(rows, v[0, :, :4].transpose(0, 1))) == "share memory"
    assert append(k, k) == append(k, both[:, 0]) == "share memory"
    assert append(both[:, 0], both.view(-1)[1024:1024 + 2 * 4096 + 2048].as_strided((3, 2, 16, 64), (4096, 1024, 64, 1))) == "share memory"
    whole, v = k.contiguous(), v.contiguous()
    words = whole.view(-1).view(i32)
    assert append(whole, v, pos=words[:4]) == append(whole, v, seq=words[8:12]) == "share memory"
    assert append(v, whole, table=words[:8].view(4, 2)) == "share memory"
    assert append(whole, v, f=whole.view(-1).view(torch.int64)[:32]) == "share memory"
    # attention reads them only
    assert _answer(lambda: q.paged_attention(rows, q.PagedCache(whole, whole, table), pos)) == "on a GPU"


def test_append_of_tables_past_32_bits():
    for width in (-1, -(1 << 33), -(1 << 32) + 4, -(1 << 63), 1 << 31, 1 << 33):
        for row in (4, 1 << 33):
            assert _append(width=width, row=row) == ESHAPE, width


def test_columns_of_an_output_that_are_not_written():
    """Of an output wider than the layer only the first N columns count: an input may lie in the others,
    and rows may be closer than the view is wide."""
    import torch
    bf16 = torch.bfloat16
    w = q.MxTensor(torch.zeros((2, 64, 16), dtype=torch.uint8), torch.zeros((1, 64, 4), dtype=torch.uint8), 64, 64)
    rows = torch.zeros((8, 128), dtype=bf16)
    t = q.MxTensor(torch.zeros((2, 8, 16), dtype=torch.uint8), torch.zeros((1, 8, 4), dtype=torch.uint8), 8, 64)
    for call in (lambda out, x=rows[:, 64:]: q.mxfp4_linear(x, w, out=out), lambda out: q.mxfp4_linear(t, w, out=out)):
        assert _answer(lambda: call(rows)) == "on a GPU"
        assert _answer(lambda: call(rows.as_strided((8, 80), (128, 1)))) == "on a GPU"
        assert _answer(lambda: call(torch.zeros(800, dtype=bf16).as_strided((8, 100), (64, 1)))) == "on a GPU"
        assert _answer(lambda: call(torch.zeros(800, dtype=bf16).as_strided((8, 64), (63, 1)))) == "twice"
    assert _answer(lambda: q.mxfp4_linear(rows[:, :64], w, out=rows)) == "share memory"
    assert _answer(lambda: q.mxfp4_linear(rows[:, 56:120], w, out=rows)) == "share memory"
