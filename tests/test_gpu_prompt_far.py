"""Pages further apart than 32 bits reach, strides of every kind, and calls beside each other on two
streams, for the operators of prompts and drafted tokens."""
import numpy as np
import pytest

import decoding_reference as R
import prompt_reference as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
def test_pages_far_apart(fp8):
    """Pages 2^30 + 4096 elements from one to the next: offsets past 2^32 bytes."""
    import torch
    import paper_2509_26436_amd as q
    kv, d, page, step, pages = 1, 64, 16, (1 << 30) + 4096, 5
    dtype = torch.float8_e4m3fn if fp8 else torch.bfloat16
    g = T.rng(1)
    flat = [torch.empty((pages - 1) * step + kv * page * d, dtype=dtype, device="cuda") for _ in range(2)]
    k, v = (t.as_strided((pages, kv, page, d), (step, page * d, d, 1)) for t in flat)
    small = T.cache(g, pages, kv, page, d, fp8)
    k.copy_(small[0]), v.copy_(small[1])
    tab, new, lengths = np.array([[4, 0, 3], [2, 1, -1]]), [30, 3], [45, 20]
    cache = q.PagedCache(k, v, T.int32(tab))
    x = R.bf16(g.normal(0, 1.5, (33, 2, d)))
    o = q.paged_prompt_attention(R.device(x), cache, T.int32([0, 30, 33]), T.int32(lengths))
    kh, vh = R.host(small[0]), R.host(small[1])
    T.check(R.host(o), x, kh, vh, tab, [0, 30, 33], lengths, page)
    bits = np.ones((33, 64), bool)
    tree = torch.from_numpy(T.words(bits)).cuda()
    o = q.paged_tree_attention(R.device(x), cache, T.int32([0, 30, 33]), T.int32(lengths), tree)
    T.check(R.host(o), x, kh, vh, tab, [0, 30, 33], lengths, page, bits=bits)
    q.paged_keep(cache, T.int32([12, 14]), T.int32([[0, 3, 30], [5, -1, -1]]))
    for t, was in ((k, kh), (v, vh)):
        want = was.copy()
        for target, source in (((4, 0, 13), (4, 0, 15)), ((4, 0, 14), (3, 0, 10)), ((2, 0, 14), (1, 0, 3))):
            want[target] = was[source]
        assert np.array_equal(R.host(t), want)


@pytest.mark.parametrize("at", [0, 4])
def test_outputs_of_any_stride(at):
    """Outputs 8 bytes off, with strides that are multiples of 4; queries head by head."""
    import torch
    import paper_2509_26436_amd as q
    kv, group, d, page, new, lengths = 2, 2, 128, 8, [20, 4], [33, 90]
    g = T.rng(2)
    tab, pages = T.table(g, lengths, page)
    k, v = T.cache(g, pages, kv, page, d, False)
    x = R.bf16(g.normal(0, 1.5, (24, 4, d)))
    xs = torch.empty(4, 24, d, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    xs.copy_(R.device(x))
    flat = torch.full((24 * (4 * d + 12) + 64,), 5.0, device="cuda", dtype=torch.bfloat16)
    out = flat.as_strided((24, 4, d), (4 * d + 12, d, 1), at)
    cache = q.PagedCache(k, v, T.int32(tab))
    q.paged_prompt_attention(xs, cache, T.int32([0, 20, 24]), T.int32(lengths), out=out)
    T.check(R.host(out), x, R.host(k), R.host(v), tab, [0, 20, 24], lengths, page)
    rest = flat.clone()
    rest.as_strided(out.shape, out.stride(), at).fill_(5.0)
    assert (rest == 5).all()


def test_two_streams_at_once():
    """Calls with workspaces of their own run beside each other."""
    import torch
    import paper_2509_26436_amd as q
    kv, group, d, page, new, lengths = 2, 4, 128, 16, [9, 9], [3000, 1500]
    g = T.rng(3)
    tab, pages = T.table(g, lengths, page)
    k, v = T.cache(g, pages, kv, page, d, False)
    cache, x = q.PagedCache(k, v, T.int32(tab)), R.device(R.bf16(g.normal(0, 1.5, (18, 8, d))))
    starts, n = T.int32([0, 9, 18]), T.int32(lengths)
    want = [q.paged_prompt_attention(x, cache, starts, n, window=w) for w in (0, 700)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, w in enumerate((0, 700)):
            got[i].append(q.paged_prompt_attention(x, cache, starts, n, window=w, stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])


def test_gradients_are_not_recorded():
    import torch
    import paper_2509_26436_amd as q
    g = T.rng(4)
    tab, pages = T.table(g, [16], 16)
    k, v = T.cache(g, pages, 1, 16, 64, False)
    x = R.device(R.bf16(g.normal(size=(4, 1, 64)))).requires_grad_(True)
    o = q.paged_prompt_attention(x, q.PagedCache(k, v, T.int32(tab)), T.int32([0, 4]), T.int32([16]))
    y, _ = q.head_norm_rotary(x, None, T.int32([0, 1, 2, 3]), q.rotary_frequencies(64))
    assert not o.requires_grad and not y.requires_grad
