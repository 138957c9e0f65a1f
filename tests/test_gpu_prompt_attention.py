"""Attention of prompts over the paged cache: shapes, masks, caps, biases, places that do not count,
values that fp16 does not take, against the definition in 64 bits."""
import numpy as np
import pytest

import decoding_reference as R
import prompt_reference as T

pytestmark = pytest.mark.gpu


def _case(seed, new, lengths, kv, group, d, page, fp8, width=None, size=1.0, **scales):
    import paper_2509_26436_amd as q
    g = T.rng(seed, kv, group, d, page)
    tab, pages = T.table(g, lengths, page, width)
    k, v = T.cache(g, pages, kv, page, d, fp8, size)
    x = R.bf16(g.normal(0, 1.5, (sum(new), kv * group, d)))
    return g, tab, k, v, x, q.PagedCache(k, v, T.int32(tab), **scales)


def _run(x, cache, new, lengths, **kw):
    import paper_2509_26436_amd as q
    return R.host(q.paged_prompt_attention(R.device(x), cache, T.int32(T.starts_of(new)), T.int32(lengths), **kw))


# (new tokens, keys) of each sequence; fewer keys than tokens leave the first tokens without any
BATCHES = [[(1, 1)], [(3, 0), (0, 5), (2, 1)], [(33, 33), (1, 700), (17, 129)], [(65, 64), (5, 5), (64, 1000)], [(300, 333)]]


@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("kv,group,d,page,fp8", [(2, 4, 128, 16, False), (1, 1, 64, 8, False), (3, 5, 256, 64, False),
                                                 (2, 4, 128, 32, True), (1, 16, 64, 16, True), (2, 2, 256, 8, True)])
def test_causal(batch, kv, group, d, page, fp8):
    print(f"prompt attention {batch} {kv} x {group} x {d} page {page} fp8 {fp8}", flush=True)
    scales = dict(k_scale=0.75, v_scale=1.5) if fp8 else {}
    new, lengths = zip(*batch)
    _, tab, k, v, x, cache = _case(1, new, lengths, kv, group, d, page, fp8, **scales)
    o = _run(x, cache, new, lengths)
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of(new), lengths, page, **scales)


@pytest.mark.parametrize("tokens", [7, 14, 30, 200])        # tiles of 32, 64, 128 and 256 rows
@pytest.mark.parametrize("width", [None, 8192])             # a part of the keys a block, or all of them
@pytest.mark.parametrize("d,fp8", [(64, False), (64, True), (128, False), (128, True), (256, False), (256, True)])
def test_tiles_and_parts(tokens, width, d, fp8):
    import paper_2509_26436_amd as q
    kv, group, page = 2, 4, 16
    new, lengths = [tokens, tokens, tokens - 1], [2500, tokens, 777]
    print(f"prompt attention of {new} over {lengths}, {d} channels, fp8 {fp8}, width {width}", flush=True)
    _, tab, k, v, x, cache = _case(2, new, lengths, kv, group, d, page, fp8, width=None if width is None else width // page)
    assert q.paged_prompt_workspace(sum(new), kv * group, cache) is not None
    o = _run(x, cache, new, lengths)
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of(new), lengths, page)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("kw", [dict(window=1), dict(window=50), dict(window=64, prefix=True), dict(cap=30.0),
                                dict(cap=2.0, window=100, slopes=True), dict(slopes=True), dict(prefix=True),
                                dict(prefix=True, slopes=True, cap=50.0), dict(scale=-0.2), dict(scale=0.0),
                                dict(scale=3.0, cap=1024.0), dict(scale=0.1, cap=2.0 ** -10)])
def test_sight_caps_and_biases(kw, fp8):
    kv, group, d, page = 2, 3, 128, 16
    new, lengths = [40, 1, 130, 7], [40, 333, 517, 5]
    print(f"prompt attention {kw} fp8 {fp8}", flush=True)
    kw = dict(kw)
    _, tab, k, v, x, cache = _case(3, new, lengths, kv, group, d, page, fp8)
    call, want = dict(kw), dict(kw)
    if kw.get("slopes"):
        import torch
        want["slopes"] = np.float32([2.0 ** (-1.3 * (h + 1)) for h in range(kv * group)])
        call["slopes"] = torch.from_numpy(want["slopes"]).cuda()
    if kw.get("prefix"):
        want["prefix"] = [25, 0, 300, 1000]
        call["prefix"] = T.int32(want["prefix"])
    o = _run(x, cache, new, lengths, **call)
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of(new), lengths, page, **want)


@pytest.mark.parametrize("d,fp8", [(64, True), (128, False), (256, False)])
@pytest.mark.parametrize("kv,group,new,past", [(2, 4, 9, 100), (1, 2, 150, 20)])
def test_infinities_and_nan_reach_only_those_who_see_them(kv, group, new, past, d, fp8):
    """Later tokens' keys and values, places past the end and pages of nobody hold NaN and infinities;
    rows that see one of them have what the plain sums have."""
    import torch
    page, news, lengths = 16, [new, new], [past + new, past + new + 3]
    print(f"prompt attention among NaN: {kv} x {group} x {d} fp8 {fp8}, {new} tokens", flush=True)
    _, tab, k, v, x, cache = _case(4, news, lengths, kv, group, d, page, fp8, width=-(-(past + new + 3) // page) + 2)
    kh, vh = R.host(k), R.host(v)
    used = np.zeros(kh.shape[0] * page, bool)
    at = lambda b, j: tab[b, j // page] * page + j % page          # noqa: E731
    for b, n in enumerate(lengths):
        used[[at(b, j) for j in range(n)]] = True
    bad = torch.from_numpy(~used.reshape(-1, page)).cuda()
    for t in (k, v):
        t.copy_(torch.where(bad[:, None, :, None], torch.full_like(t.float(), np.nan), t.float()).to(t.dtype))
    # one token's values: NaN, or an infinity where there is one, seen from that token on; its keys too
    mark = past + new // 2
    marks = [(0, np.nan)] if fp8 else [(0, np.nan), (1, np.inf)]
    for b, what in marks:
        j = at(b, mark)
        v[j // page, :, j % page, 5] = what
        if b == 0:
            k[j // page, 0, j % page, 3] = float("nan")
    o = _run(x, cache, news, lengths)
    start = T.starts_of(news)
    for b in range(2):
        first = past + (0 if b == 0 else 3)
        clean = mark - first                                       # tokens before it see nothing of it
        rows = slice(start[b], start[b] + clean)
        sub = [0, clean, clean] if b == 0 else [0, 0, clean]
        T.check(o[rows], x[rows], kh, vh, tab, sub, [first + clean] * 2, page)
    if not fp8:
        later = o[start[1] + mark - past - 3:start[2]]
        assert (later[:, :, 5] == np.inf).all() and np.isfinite(np.delete(later, 5, 2)).all()
    later = o[start[0] + mark - past:start[1]]
    assert np.isnan(later[:, group:, 5]).all() and np.isnan(later[:, :group]).all()      # head 0's keys are NaN too
    assert kv == 1 or np.isfinite(np.delete(later[:, group:], 5, 2)).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_pages_that_are_none(fp8):
    """Positions without a page have no weight, wherever in the sequence they lie."""
    import paper_2509_26436_amd as q
    kv, group, d, page, new, lengths = 2, 2, 128, 8, [50, 20], [400, 70]
    g, tab, k, v, x, cache = _case(5, new, lengths, kv, group, d, page, fp8)
    tab[0, [0, 3, 30, 44]] = [-1, 1 << 20, -7, -1]
    tab[1, :] = -1
    cache = q.PagedCache(k, v, T.int32(tab))
    o = _run(x, cache, new, lengths)
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of(new), lengths, page)


@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** -23, 2.0 ** 9, 2.0 ** 60, "mixed", "one"])
@pytest.mark.parametrize("d,new", [(128, 5), (64, 100), (256, 60)])
def test_values_that_fp16_does_not_take(size, d, new):
    import torch
    kv, group, page, lengths = 1, 4, 16, [300, 130]
    print(f"prompt attention of values of {size}, {d} channels, {new} tokens", flush=True)
    g, tab, k, v, x, cache = _case(6, [new, new], lengths, kv, group, d, page, False)
    vh = R.host(v)
    if size == "mixed":
        vh *= np.exp2(g.integers(-60, 60, vh.shape))
    elif size == "one":
        vh[tab[0, 5], 0, 3, 7] = 2.0 ** 10
        vh[tab[0, 9], 0, 2, 1] = 2.0 ** -25
        vh[tab[1, 0], 0, 0, 0] = 2.0 ** -133
    else:
        vh *= size
    v.copy_(torch.from_numpy(vh).cuda().to(torch.bfloat16))
    o = _run(x, cache, [new, new], lengths)
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of([new, new]), lengths, page)


@pytest.mark.parametrize("d,fp8,new", [(128, False, 6), (128, True, 70), (64, False, 200), (256, True, 40)])
def test_weights_of_cancelling_values(d, fp8, new):
    """Neighbouring keys hold a value and its negative under nearly equal weights: what is left is the
    weights' difference, in which a bf16 rounding (2^-8) would show."""
    import torch
    kv, group, page, lengths = 2, 3, 16, [500, 301]
    g, tab, k, v, x, cache = _case(7, [new, new], lengths, kv, group, d, page, fp8)
    kh, vh = R.host(k), R.host(v)
    kh[..., 1:] = 0.0
    vh[:, :, 1::2] = -vh[:, :, ::2]
    for t, h in ((k, kh), (v, vh)):
        t.copy_(torch.from_numpy(h).cuda().to(torch.bfloat16).to(t.dtype))
    x[:, :, 0] = R.bf16(g.uniform(0.3, 1.0, x.shape[:2]))
    o = _run(x, cache, [new, new], lengths, scale=0.25)
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of([new, new]), lengths, page, scale=0.25)


@pytest.mark.parametrize("rise", [3.0, 9.0, 40.0])
def test_scores_that_rise(rise):
    """The maximum moves step by step, by less and by more than the slack that it is given."""
    import torch
    kv, group, d, page, new, lengths = 1, 2, 64, 16, [70], [900]
    _, tab, k, v, x, cache = _case(8, new, lengths, kv, group, d, page, False)
    kh = np.zeros(R.host(k).shape)
    for j in range(900):
        kh[tab[0, j // 16], 0, j % 16, 0] = R.bf16(rise * (j // 64))
    k.copy_(torch.from_numpy(kh).cuda().to(torch.bfloat16))
    x[:, :, 0] = 1.0
    x[10:20, :, 0] = -1.0
    o = _run(x, cache, new, lengths, scale=1.0)
    T.check(o, x, R.host(k), R.host(v), tab, [0, 70], lengths, page, scale=1.0)


@pytest.mark.parametrize("d,new", [(64, 5), (128, 100), (256, 60)])
def test_smallest_values_that_fp16_takes(d, new):
    """Values that are subnormal in fp16, all of them: taken exactly, not lost."""
    import torch
    kv, group, page, lengths = 1, 4, 16, [300, 130]
    g, tab, k, v, x, cache = _case(16, [new, new], lengths, kv, group, d, page, False)
    vh = R.bf16(np.exp2(g.uniform(-24, -21.1, R.host(v).shape)) * g.choice([-1.0, 1.0], R.host(v).shape))
    vh = np.where(np.abs(vh) < 2.0 ** -24, 2.0 ** -24, vh)
    v.copy_(torch.from_numpy(vh).cuda().to(torch.bfloat16))
    o = _run(x, cache, [new, new], lengths)
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of([new, new]), lengths, page)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new", [3, 100])
@pytest.mark.parametrize("below", [10.0, 17.25, 21.0])
def test_many_weights_far_below_the_largest(below, new, fp8):
    """One key takes nearly all the weight and has the value 0: the rest, e^-below each, is what is left."""
    import torch
    kv, group, d, page, lengths = 1, 2, 64, 16, [900]
    _, tab, k, v, x, cache = _case(17, [new], lengths, kv, group, d, page, fp8)
    kh, vh = np.zeros(R.host(k).shape), np.ones(R.host(v).shape)
    kh[..., 0] = -below if not fp8 else -round(below)
    kh[tab[0, 1], 0, 3, 0], vh[tab[0, 1], 0, 3] = 0.0, 0.0
    for t, h in ((k, kh), (v, vh)):
        t.copy_(torch.from_numpy(h).cuda().to(torch.bfloat16).to(t.dtype))
    x[:] = 0.0
    x[:, :, 0] = 1.0
    o = _run(x, cache, [new], lengths, scale=1.0)
    T.check(o, x, R.host(k), R.host(v), tab, [0, new], lengths, page, scale=1.0)
    assert (o > 0).all()


def test_views_and_rows_of_nobody():
    """Strided queries, outputs and caches; rows before the first, behind the last sequence stay."""
    import torch
    import paper_2509_26436_amd as q
    kv, group, d, page, new, lengths = 2, 4, 128, 16, [5, 40], [90, 200]
    g, tab, k, v, x, _ = _case(9, new, lengths, kv, group, d, page, False)
    both = torch.stack([k, v], 1)
    cache = q.PagedCache(both[:, 0], both[:, 1], T.int32(np.pad(tab, ((0, 0), (0, 3)), constant_values=-1))[:, :tab.shape[1]])
    wide = torch.zeros(60, kv * group + 4, d, device="cuda", dtype=torch.bfloat16)
    wide[7:52, 2:-2] = R.device(x)
    out = torch.full((kv * group, 60, d), 7.0, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    starts = T.int32([7, 12, 52])
    got = q.paged_prompt_attention(wide[:, 2:-2], cache, starts, T.int32(lengths), out=out)
    assert got.data_ptr() == out.data_ptr()
    o = R.host(out)
    assert (o[:7] == 7).all() and (o[52:] == 7).all()
    T.check(o[7:52], x, R.host(k), R.host(v), tab, [0, 5, 45], lengths, page)


def test_starts_and_lengths_out_of_range():
    """Starts outside the tokens and lengths outside the table are clamped."""
    import torch
    import paper_2509_26436_amd as q
    kv, group, d, page = 1, 2, 64, 16
    _, tab, k, v, x, cache = _case(10, [20, 20], [64, 64], kv, group, d, page, False)
    out = torch.full((40, 2, d), 7.0, device="cuda", dtype=torch.bfloat16)
    q.paged_prompt_attention(R.device(x), cache, T.int32([-5, 30, 1 << 30]), T.int32([1 << 30, -3]), out=out)
    o = R.host(out)
    T.check(o, x, R.host(k), R.host(v), tab, [0, 30, 40], [64, 0], page)
    for starts in ([30, 10, 10], [50, 60, 70], [-9, -8, -7]):
        out.fill_(7.0)
        q.paged_prompt_attention(R.device(x), cache, T.int32(starts), T.int32([64, 64]), out=out)
        assert (out == 7).all()


@pytest.mark.parametrize("S", [65, 200])
def test_many_sequences(S):
    g = T.rng(11, S)
    new = g.integers(0, 6, S)
    new[:3], new[60:70], new[-2:] = 0, 0, 0
    lengths = (new + g.integers(0, 60, S)).tolist()
    new = new.tolist()
    new[S // 2], lengths[S // 2] = 90, 1200
    _, tab, k, v, x, cache = _case(12, new, lengths, 1, 2, 64, 16, False)
    o = _run(x, cache, new, lengths)
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of(new), lengths, 16)


def test_captured_and_replayed_with_other_lengths():
    """Two graphs that share a workspace, replayed in turn with eager calls between."""
    import torch
    import paper_2509_26436_amd as q
    kv, group, d, page, new, lengths = 2, 4, 128, 16, [12, 3, 30], [700, 40, 1500]
    g, tab, k, v, x, cache = _case(13, new, lengths, kv, group, d, page, False, width=256)
    qs, starts, n = R.device(x), T.int32(T.starts_of(new)), T.int32(lengths)
    workspace = q.paged_prompt_workspace(sum(new), kv * group, cache)
    assert workspace is not None
    outs = [torch.empty_like(qs) for _ in range(2)]
    call = lambda i: q.paged_prompt_attention(qs, cache, starts, n, window=[0, 100][i], out=outs[i], workspace=workspace)   # noqa: E731
    call(0), call(1)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for i in range(2):
        with torch.cuda.graph(graphs[i]):
            call(i)
    for other, starts_now in (([700, 40, 1500], new), ([33, 1000, 64], [5, 20, 20]), ([1600, 0, 900], [0, 45, 0])):
        n.copy_(T.int32(other))
        starts.copy_(T.int32(T.starts_of(starts_now)))
        # lengths past the sequences' pages read entries of -1: no keys
        for i in (0, 1, 0):
            outs[i].zero_()
            torch.cuda.synchronize()
            graphs[i].replay()
            torch.cuda.synchronize()
            eager = q.paged_prompt_attention(qs, cache, starts, n, window=[0, 100][i], out=torch.zeros_like(qs))
            assert torch.equal(outs[i], eager)
            T.check(R.host(outs[i]), x, R.host(k), R.host(v), tab, T.starts_of(starts_now), other, page, window=[0, 100][i])


def test_on_another_stream():
    import torch
    import paper_2509_26436_amd as q
    new, lengths = [40, 9], [300, 64]
    _, tab, k, v, x, cache = _case(14, new, lengths, 2, 2, 128, 16, True)
    side = torch.cuda.Stream()
    qs, starts, n = R.device(x), T.int32(T.starts_of(new)), T.int32(lengths)
    torch.cuda.synchronize()
    o = q.paged_prompt_attention(qs, cache, starts, n, stream=side)
    side.synchronize()
    T.check(R.host(o), x, R.host(k), R.host(v), tab, T.starts_of(new), lengths, 16)


def test_nothing_to_do():
    import torch
    import paper_2509_26436_amd as q
    _, tab, k, v, x, cache = _case(15, [2], [5], 1, 1, 64, 8, False)
    none = torch.empty(0, 1, 64, device="cuda", dtype=torch.bfloat16)
    assert q.paged_prompt_attention(none, cache, T.int32([0, 0]), T.int32([5])).shape == (0, 1, 64)
    empty = q.PagedCache(k, v, torch.empty(1, 0, device="cuda", dtype=torch.int32))
    assert (q.paged_prompt_attention(R.device(x), empty, T.int32([0, 2]), T.int32([5])) == 0).all()
    nobody = q.PagedCache(k, v, torch.empty(0, 4, device="cuda", dtype=torch.int32))
    out = torch.full((2, 1, 64), 3.0, device="cuda", dtype=torch.bfloat16)
    q.paged_prompt_attention(R.device(x), nobody, T.int32([0]), T.int32([]), out=out)
    assert (out == 3).all()
