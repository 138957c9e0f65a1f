"""The paged cache: append (rotated keys, bf16 and e4m3, padding, pages that are none) and attention
of one new token a sequence, against the definitions in 64 bits."""
import math

import numpy as np
import pytest

import decoding_reference as R

pytestmark = pytest.mark.gpu


def _rng(*seed):
    return np.random.Generator(np.random.PCG64(list(seed)))


def _int32(a):
    import torch
    return torch.from_numpy(np.asarray(a, np.int32)).cuda()


def _table(rng, lengths, page, width=None, spare=2):
    """Shuffled pages for these lengths: (table with -1 where there is none, number of pages)."""
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + spare
    order = rng.permutation(pages)
    width = max(max(need), 1) if width is None else width
    table, at = np.full((len(lengths), width), -1, np.int64), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, pages


def _cache(rng, pages, heads, page, d, fp8):
    """Random keys and values, and what is stored (float64)."""
    import torch
    out = []
    for _ in range(2):
        t = torch.from_numpy(rng.normal(0, 1, (pages, heads, page, d))).cuda()
        out.append(t.to(torch.float8_e4m3fn if fp8 else torch.bfloat16))
    return out


def _gather(t, table, b, h, n, page):
    """Positions 0 .. n - 1 of sequence b and cache head h."""
    return np.concatenate([t[table[b, j], h] for j in range(-(-n // page))] + [t[0, 0, :0]])[:n]


def _check(o, q, k, v, table, lengths, page, scale=None, window=0, k_scale=1.0, v_scale=1.0):
    S, H, d = q.shape
    kv = k.shape[1]
    G = H // kv
    scale = 1 / math.sqrt(d) if scale is None else scale
    for b, n in enumerate(lengths):
        first = max(0, n - window) if window else 0
        for h in range(kv):
            kk, vv = (_gather(t, table, b, h, n, page)[first:] for t in (k, v))
            want, far = R.attention(q[b, h * G:(h + 1) * G], kk * k_scale, vv * v_scale, scale)
            off = np.abs(o[b, h * G:(h + 1) * G] - want)
            assert (off <= far).all(), (b, h, n, off.max(), far[off == off.max()])
        if n == 0:
            assert (o[b] == 0).all()


def _attention_case(seed, lengths, kv, group, d, page, fp8, window=0, width=None, **kw):
    import paper_2509_26436_amd as q
    rng = _rng(seed, kv, group, d, page)
    table, pages = _table(rng, lengths, page, width)
    k, v = _cache(rng, pages, kv, page, d, fp8)
    x = R.bf16(rng.normal(0, 1.5, (len(lengths), kv * group, d)))
    cache = q.PagedCache(k, v, _int32(table), **kw)
    return rng, table, k, v, x, cache


LENGTHS = [[1], [0], [5, 0, 33, 32, 31], [127, 128, 129, 1, 700], [2050], [64, 4097]]


@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("kv,group,d,page,fp8", [(2, 4, 128, 16, False), (1, 1, 64, 8, False), (3, 5, 256, 64, False),
                                                 (2, 4, 128, 32, True), (1, 16, 64, 16, True), (2, 2, 256, 8, True),
                                                 (1, 23, 128, 128, False), (1, 33, 64, 16, True)])
def test_attention(lengths, kv, group, d, page, fp8):
    import paper_2509_26436_amd as q
    print(f"paged attention {lengths} {kv} x {group} x {d} page {page} fp8 {fp8}", flush=True)
    kw = dict(k_scale=0.75, v_scale=1.5) if fp8 else {}
    _, table, k, v, x, cache = _attention_case(1, lengths, kv, group, d, page, fp8, **kw)
    o = q.paged_attention(R.device(x), cache, _int32(lengths))
    _check(R.host(o), x, R.host(k), R.host(v), table, lengths, page, **kw)


@pytest.mark.parametrize("S,group,fp8,d", [(300, 2, False, 64), (600, 1, True, 128), (257, 17, False, 64)])
def test_many_sequences(S, group, fp8, d):
    """More sequences than a block counts at a time, runs of empty ones, and one long one among them."""
    import paper_2509_26436_amd as q
    print(f"paged attention of {S} sequences, group {group} fp8 {fp8} d {d}", flush=True)
    rng = _rng(11, S)
    lengths = rng.integers(0, 70, S)
    lengths[:3], lengths[250:259], lengths[-2:] = 0, 0, 0
    lengths[S // 2], lengths[255], lengths[256] = 1500, 129, 600
    lengths = lengths.tolist()
    _, table, k, v, x, cache = _attention_case(12, lengths, 1, group, d, 32, fp8)
    o = q.paged_attention(R.device(x), cache, _int32(lengths))
    _check(R.host(o), x, R.host(k), R.host(v), table, lengths, 32)


@pytest.mark.parametrize("kv,group,d,fp8", [(300, 1, 64, False), (64, 3, 128, True)])
def test_many_short_heads(kv, group, d, fp8):
    """Heads enough for a block each, over more keys than one pass of it."""
    import paper_2509_26436_amd as q
    lengths = [1000, 0, 513, 31, 770]
    _, table, k, v, x, cache = _attention_case(13, lengths, kv, group, d, 16, fp8)
    o = q.paged_attention(R.device(x), cache, _int32(lengths))
    assert q.paged_attention_workspace(5, kv * group, cache) is None
    _check(R.host(o), x, R.host(k), R.host(v), table, lengths, 16)


@pytest.mark.parametrize("S,kv", [(3, 2), (90, 6)])
@pytest.mark.parametrize("group,d,fp8", [(4, 128, False), (19, 64, True), (1, 256, False), (2, 256, True)])
@pytest.mark.parametrize("longest,window", [(1, 0), (33, 0), (128, 0), (90, 20), (700, 40), (250, 0)])
def test_short_sequences(S, kv, group, d, fp8, longest, window):
    """Blocks of one, two and four waves, some of them without keys; few heads and many."""
    import paper_2509_26436_amd as q
    print(f"paged attention {S} x {kv} x {group} x {d} fp8 {fp8}, up to {longest}, window {window}", flush=True)
    lengths = _rng(17, S, longest).integers(0, longest + 1, S).tolist()
    lengths[:2] = [longest, 0]
    _, table, k, v, x, cache = _attention_case(18, lengths, kv, group, d, 16, fp8)
    o = q.paged_attention(R.device(x), cache, _int32(lengths), window=window)
    _check(R.host(o), x, R.host(k), R.host(v), table, lengths, 16, window=window)


@pytest.mark.parametrize("window", [1, 7, 32, 100, 5000])
@pytest.mark.parametrize("fp8", [False, True])
def test_window_and_scale(window, fp8):
    import paper_2509_26436_amd as q
    lengths = [0, 1, 40, 333, 900, 97]
    _, table, k, v, x, cache = _attention_case(2, lengths, 2, 3, 128, 16, fp8)
    o = q.paged_attention(R.device(x), cache, _int32(lengths), scale=0.3, window=window)
    _check(R.host(o), x, R.host(k), R.host(v), table, lengths, 16, scale=0.3, window=window)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_places_that_do_not_count_hold_nan(fp8, d):
    """Everything past a sequence's end, before its window, and in pages of nobody is NaN or infinite."""
    import torch
    import paper_2509_26436_amd as q
    lengths, page, window = [3, 40, 170, 1, 0], 16, 50
    rng, table, k, v, x, cache = _attention_case(3, lengths, 2, 4, d, page, fp8)
    kh, vh = R.host(k), R.host(v)
    counts = np.zeros((k.shape[0], page), bool)
    for b, n in enumerate(lengths):
        for p in range(max(0, n - window), n):
            counts[table[b, p // page], p % page] = True
    bad = torch.from_numpy(~counts).cuda()[:, None, :, None].expand(k.shape)
    for t, value in ((k, math.nan), (v, math.nan)):
        raw = torch.full((), value, dtype=torch.bfloat16, device="cuda").to(t.dtype)
        bits = torch.uint8 if fp8 else torch.int16
        t.view(bits)[bad] = raw.view(bits)
    if not fp8:
        v[bad & (torch.rand(v.shape, device="cuda") < 0.5)] = math.inf
    o = q.paged_attention(R.device(x), cache, _int32(lengths), window=window)
    _check(R.host(o), x, kh, vh, table, lengths, page, window=window)


@pytest.mark.parametrize("kv,group,d,fp8", [(2, 3, 128, False), (1, 20, 64, True), (1, 2, 256, False)])
@pytest.mark.parametrize("window", [0, 1500])
def test_long_sequences_with_holes(kv, group, d, fp8, window):
    """Sequences shared by blocks: NaN wherever nothing counts, pages that are none, lengths below 0
    and past the table, a window that begins inside a page."""
    import torch
    import paper_2509_26436_amd as q
    page, width = 16, 160
    lengths = [2300, 0, 1, 1700, 2560, 95, 2560]
    rng, table, k, v, x, cache = _attention_case(14, lengths, kv, group, d, page, fp8, width=width)
    table[0, 20:60] = -1
    table[3, :] = 2 ** 31 - 1
    table[4, 100] = k.shape[0]
    table[4, 0:99] = -5
    cache = q.PagedCache(k, v, _int32(table))
    kh, vh = R.host(k), R.host(v)
    have = []
    counts = np.zeros((k.shape[0], page), bool)
    for b, n in enumerate(lengths):
        places = [(table[b, p // page], p % page) for p in range(max(0, n - window) if window else 0, n)
                  if 0 <= table[b, p // page] < k.shape[0]]
        have.append(places)
        for place in places:
            counts[place] = True
    bad = torch.from_numpy(~counts).cuda()[:, None, :, None].expand(k.shape)
    raw = torch.full((), math.nan, dtype=torch.bfloat16, device="cuda").to(k.dtype)
    bits = torch.uint8 if fp8 else torch.int16
    for t in (k, v):
        t.view(bits)[bad] = raw.view(bits)
    asked = list(lengths)
    asked[1], asked[6] = -9, 2 ** 31 - 1
    o = R.host(q.paged_attention(R.device(x), cache, _int32(asked), window=window))
    for b, places in enumerate(have):
        at = tuple(np.array(places, np.int64).reshape(-1, 2).T)
        for h in range(kv):
            rows = slice(h * group, (h + 1) * group)
            want, far = R.attention(x[b, rows], kh[:, h][at], vh[:, h][at], 1 / math.sqrt(d))
            assert (np.abs(o[b, rows] - want) <= far).all(), (b, h)
    assert (o[1] == 0).all() and (o[3] == 0).all()


def test_infinities_in_long_sequences():
    """The parts of a shared sequence join as one softmax: a whole part of score -inf has no weight,
    +inf gives NaN, a NaN query gives NaN in its own head only, NaN in a counted value its column."""
    import torch
    import paper_2509_26436_amd as q
    lengths, page = [3000, 3000, 3000], 16
    _, table, k, v, x, cache = _attention_case(15, lengths, 1, 2, 64, page, False)
    x = np.abs(x)
    x[0, 1, 5] = np.nan
    v[int(table[0, 100]), 0, 3, 9] = math.nan
    k[int(table[1, 130]), 0, 3, 8] = math.inf
    lost = torch.from_numpy(table[2, :100]).cuda()
    k[lost, 0, :, 8] = -math.inf
    o = R.host(q.paged_attention(R.device(x), cache, _int32(lengths)))
    assert np.isnan(o[0, 1]).all() and np.isnan(o[0, 0, 9]) and np.isnan(o[0, 0]).sum() == 1
    assert np.isnan(o[1]).all()
    kh, vh = (_gather(R.host(t), table, 2, 0, 3000, page)[100 * page:] for t in (k, v))
    want, far = R.attention(x[2], kh, vh, 1 / math.sqrt(64))
    assert (np.abs(o[2] - want) <= far).all()


def test_tables_without_pages():
    """A table of no columns, no sequences at all; a cache of no pages is refused."""
    import torch
    import paper_2509_26436_amd as q
    k = torch.full((1, 2, 16, 64), math.nan, dtype=torch.bfloat16, device="cuda")
    x = torch.ones((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    lengths = _int32([5, 0, 3000])
    for table in (np.zeros((3, 0)), np.full((3, 200), -1)):
        assert (q.paged_attention(x, q.PagedCache(k, k.clone(), _int32(table)), lengths) == 0).all()
    cache = q.PagedCache(k, k.clone(), _int32(np.zeros((0, 8))))
    assert q.paged_attention(x[:0], cache, lengths[:0]).shape == (0, 4, 64)
    with pytest.raises(q.QuartzError):
        q.paged_attention(x, q.PagedCache(k[:0], k[:0], _int32(np.full((3, 200), -1))), lengths)


def test_two_streams_at_once():
    """Calls on two streams with workspaces of their own, while both run."""
    import torch
    import paper_2509_26436_amd as q
    lengths, page = [5000, 100, 2222], 16
    _, table, k, v, x, cache = _attention_case(16, lengths, 2, 4, 128, page, False)
    xs = [R.device(x), R.device(-x)]
    at = _int32(lengths)
    want = [q.paged_attention(t, cache, at) for t in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    outs = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs[i].append(q.paged_attention(xs[i], cache, at))
    torch.cuda.synchronize()
    for i in range(2):
        for o in outs[i]:
            assert torch.equal(o, want[i])
    _check(R.host(want[0]), x, R.host(k), R.host(v), table, lengths, page)


def test_lengths_and_pages_out_of_range():
    """Lengths below 0 and past the table are clamped; positions of pages that are none have no weight."""
    import paper_2509_26436_amd as q
    page, lengths = 16, [64, 64, 64, 64]
    _, table, k, v, x, cache = _attention_case(4, lengths, 2, 2, 128, page, False)
    bad = table.copy()
    bad[0, 1] = -7
    bad[1, :] = 10 ** 6
    bad[2, 3] = k.shape[0]
    cache = q.PagedCache(k, v, _int32(bad))
    o = R.host(q.paged_attention(R.device(x), cache, _int32([64, 64, 10 ** 6, -3])))
    kh, vh = R.host(k), R.host(v)
    for b, have in ((0, [0, 2, 3]), (1, []), (2, [0, 1, 2]), (3, [])):
        for h in range(2):
            kk, vv = (np.concatenate([t[table[b, j], h] for j in have] + [t[0, 0, :0]]) for t in (kh, vh))
            want, far = R.attention(x[b, 2 * h:2 * h + 2], kk, vv, 1 / math.sqrt(128))
            assert (np.abs(o[b, 2 * h:2 * h + 2] - want) <= far).all(), b


@pytest.mark.parametrize("d,fp8", [(128, False), (64, True)])
def test_large_scores_and_late_maxima(d, fp8):
    """Scores that grow along the sequence to hundreds, and one key far above the others."""
    import torch
    import paper_2509_26436_amd as q
    lengths, page = [600, 3000], 32
    rng, table, k, v, x, cache = _attention_case(5, lengths, 1, 4, d, page, fp8)
    kh = R.host(k)
    for b, n in enumerate(lengths):
        for j in range(-(-n // page)):
            kh[table[b, j]] *= 0.05 + 4.0 * j * page / n
    kh[table[1, 7], 0, 3] *= 30.0
    k.copy_(torch.from_numpy(np.clip(kh, -448, 448) if fp8 else kh).cuda().to(torch.bfloat16).to(k.dtype))
    o = q.paged_attention(R.device(4 * x), cache, _int32(lengths))
    _check(R.host(o), 4 * x, R.host(k), R.host(v), table, lengths, page)


def test_infinite_scores_follow_the_softmax():
    """+inf in a key that counts gives NaN, a NaN query gives NaN in its own head only, and keys of
    score -inf have no weight."""
    import torch
    import paper_2509_26436_amd as q
    lengths, page = [40, 40, 40], 16
    _, table, k, v, x, cache = _attention_case(6, lengths, 1, 2, 64, page, False)
    x = np.abs(x)
    x[0, 1, 5] = np.nan
    k[int(table[1, 0]), 0, 3, 8] = math.inf
    k[int(table[2, 0]), 0, 3, 8] = -math.inf
    o = R.host(q.paged_attention(R.device(x), cache, _int32(lengths)))
    assert np.isnan(o[0, 1]).all() and np.isfinite(o[0, 0]).all()
    assert np.isnan(o[1]).all()
    kh, vh = (np.delete(_gather(R.host(t), table, 2, 0, 40, page), 3, 0) for t in (k, v))
    want, far = R.attention(x[2], kh, vh, 1 / math.sqrt(64))
    assert (np.abs(o[2] - want) <= far).all()


def test_strides():
    """Queries inside a fused projection's rows, output into a wider tensor, pages strided, a table
    wider than it is used, lengths at an odd offset."""
    import torch
    import paper_2509_26436_amd as q
    lengths, page, kv, d = [100, 9, 300], 16, 2, 128
    rng = _rng(7)
    table, pages = _table(rng, lengths, page)
    both = torch.from_numpy(rng.normal(0, 1, (pages, 2, kv, page, d))).cuda().to(torch.bfloat16)
    wide = np.full((3, table.shape[1] + 5), 2 ** 30)
    wide[:, :table.shape[1]] = table
    cache = q.PagedCache(both[:, 0], both[:, 1], _int32(wide)[:, :table.shape[1]])
    x = R.bf16(rng.normal(0, 1, (3, 6, d)))
    rows = torch.full((3, 10, d), math.nan, dtype=torch.bfloat16, device="cuda")
    rows[:, 2:8] = R.device(x)
    out = torch.full((3, 8, d + 4), 2.0, dtype=torch.bfloat16, device="cuda")[:, :, :d]
    full = out._base
    at = _int32([9] + lengths)[1:]
    q.paged_attention(rows[:, 2:8], cache, at, out=out[:, 1:7])
    _check(R.host(out[:, 1:7]), x, R.host(both[:, 0]), R.host(both[:, 1]), table, lengths, page)
    out[:, 1:7] = 2.0
    assert (full == 2.0).all()


def test_cache_past_32_bits():
    """Pages further than 2^32 bytes into a cache."""
    import torch
    import paper_2509_26436_amd as q
    page, kv, d = 16, 1, 128
    pages = (1 << 32) // (page * kv * d * 2) + 40
    k = torch.zeros((pages, kv, page, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    rng = _rng(8)
    table = np.array([[pages - 1, 3, pages - 30, (1 << 31) // (page * d * 2) + 5]])
    positions = rng.permutation(60)
    new = [R.bf16(rng.normal(0, 1, (60, kv, d))) for _ in range(2)]
    cache = q.PagedCache(k, v, _int32(table))
    q.paged_append(cache, R.device(new[0]), R.device(new[1]), _int32(positions), _int32(np.zeros(60)))
    x = R.bf16(rng.normal(0, 1, (1, 2, d)))
    o = R.host(q.paged_attention(R.device(x), cache, _int32([60])))
    for h in range(1):
        want, far = R.attention(x[0], new[0][:, 0], new[1][:, 0], 1 / math.sqrt(d))
        assert (np.abs(o[0] - want) <= far).all()
    assert int((k != 0).any(-1).sum()) == 60


def test_graph_replays_with_other_lengths():
    """One capture serves other lengths, pages and tokens; two graphs with one workspace in turn."""
    import torch
    import paper_2509_26436_amd as q
    page, kv, G, d = 16, 2, 4, 128
    rng = _rng(9)
    steps = [[700, 3, 0, 290], [1, 1024, 512, 77], [1024, 1024, 1024, 1024]]
    table, pages = _table(rng, [1024] * 4, page)
    k, v = _cache(rng, pages, kv, page, d, False)
    cache = q.PagedCache(k, v, _int32(table))
    xs = [R.bf16(rng.normal(0, 1, (4, kv * G, d))) for _ in steps]
    x, lengths = R.device(xs[0]), _int32(steps[0])
    ws = q.paged_attention_workspace(4, kv * G, cache)
    outs = [torch.empty_like(x) for _ in range(2)]
    q.paged_attention(x, cache, lengths, out=outs[0], workspace=ws)
    graphs = []
    for out in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            q.paged_attention(x, cache, lengths, out=out, workspace=ws)
        graphs.append(g)
    for i in (1, 2, 0, 1):
        x.copy_(R.device(xs[i]))
        lengths.copy_(_int32(steps[i]))
        for g, out in zip(graphs, outs):
            out.fill_(9.0)
            g.replay()
        eager = q.paged_attention(x, cache, lengths)
        torch.cuda.synchronize()
        for out in outs:
            assert torch.equal(out, eager)
        _check(R.host(eager), xs[i], R.host(k), R.host(v), table, steps[i], page)


def _e4m3(a):
    import torch
    return torch.from_numpy(np.clip(a, -448, 448).astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kv,d,rot,page,fp8", [(1, 64, 64, 8, False), (8, 128, 128, 16, False), (3, 128, 32, 64, True),
                                               (5, 256, 256, 16, True), (2, 128, 20, 32, False), (2, 64, 0, 16, True)])
def test_append(kv, d, rot, page, fp8, layout):
    """Several sequences, tokens in any order, with padding tokens and places that are none; the rest
    of the cache stays as it was, bit for bit."""
    import torch
    import paper_2509_26436_amd as q
    print(f"append {kv} x {d} rot {rot} page {page} fp8 {fp8} {layout}", flush=True)
    rng = _rng(10, kv, d, rot, page)
    lengths = [3 * page + 1, 1, 200]
    table, pages = _table(rng, lengths, page)
    k, v = _cache(rng, pages, kv, page, d, fp8)
    before = R.host(k), R.host(v)
    kw = dict(k_scale=0.5, v_scale=1.25) if fp8 else {}
    cache = q.PagedCache(k, v, _int32(table), **kw)
    at = [(b, p) for b, n in enumerate(lengths) for p in range(n)]
    at = [at[i] for i in rng.permutation(len(at))[:77]]
    nowhere = [(0, -1), (1, page + 3), (0, table.shape[1] * page), (-1, 0), (3, 0), (2, 2 ** 31 - 1), (2 ** 30, 5)]
    at = at[:40] + nowhere + at[40:]
    T = len(at)
    rows = rng.normal(0, 1, (T, 2, kv, d)) * np.where(rng.random((T, 2, kv, d)) < 0.01, 600, 1)
    rows = R.bf16(rows)
    kv_rows = R.device(rows)
    sequences, positions = ([a[i] for a in at] for i in (0, 1))
    f = q.rotary_frequencies(rot)
    q.paged_append(cache, kv_rows[:, 0], kv_rows[:, 1], _int32(positions), _int32(sequences),
                   f if rot else None, layout, magnitude=1.1 if rot else 1.0)
    kk, kfar = R.rotate(rows[:, 0], positions, f.cpu().numpy(), layout, magnitude=1.1) if rot else (rows[:, 0], 0 * rows[:, 0])
    got_k, got_v = R.host(k), R.host(v)
    want_k, want_v = (t.copy() for t in before)
    far = np.zeros_like(want_k)
    for t, (b, p) in enumerate(at):
        if (b, p) in nowhere:
            continue
        place = table[b, p // page], slice(None), p % page
        if fp8:
            x, e = kk[t] / 0.5, kfar[t] / 0.5
            want_k[place] = np.clip(x, -448, 448)
            # half a step of e4m3, 2^-10 below its normal range
            far[place] = R.HALF_E4M3 * np.abs(want_k[place]) + 2.0 ** -10 + (1 + R.HALF_E4M3) * e
            want_v[place] = _e4m3((rows[t, 1].astype(np.float32) / np.float32(1.25)))
            if not rot:
                want_k[place], far[place] = _e4m3(x), 0
        else:
            want_k[place], want_v[place] = kk[t], rows[t, 1]
            far[place] = R.HALF_BF16 * np.abs(kk[t]) + (1 + R.HALF_BF16) * kfar[t] if rot else 0
            far[place][:, rot:] = 0
    assert (np.abs(got_k - want_k) <= far).all(), np.abs(got_k - want_k).max()
    np.testing.assert_array_equal(got_v, want_v)


def test_append_keeps_nan_and_saturates():
    import torch
    import paper_2509_26436_amd as q
    k = torch.zeros((1, 1, 8, 64), dtype=torch.float8_e4m3fn, device="cuda")
    v = torch.zeros_like(k)
    rows = np.zeros((1, 1, 64))
    rows[0, 0, :8] = [np.nan, np.inf, -np.inf, 449, -1e30, 464, 480, 0.001]
    cache = q.PagedCache(k, v, _int32([[0]]))
    q.paged_append(cache, R.device(rows), R.device(rows), _int32([3]))
    for t in (k, v):
        got = R.host(t)[0, 0, 3, :8]
        assert np.isnan(got[0])
        np.testing.assert_array_equal(got[1:7], [448, -448, 448, -448, 448, 448])
        assert abs(got[7] - 0.001) <= 2.0 ** -10


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("scale", [0.75, 1.1, 0.0371, 1.5 * 2.0 ** -126, 1.5 * 2.0 ** 126, 3.3e38])
def test_append_divides_every_value(scale, fp8):
    """Every bf16 value over a scale: the fp32 quotient, rounded to the cache's type, bit for bit.
    Below 2^-120 the quotient's remainder is no fp32 number any more, and over a scale past 2^126 the
    reciprocal is subnormal: there a value may fall to the neighbour."""
    import torch
    import paper_2509_26436_amd as q
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16)
    x = bits.view(torch.bfloat16).view(512, 1, 128).cuda()
    dtype = torch.float8_e4m3fn if fp8 else torch.bfloat16
    k = torch.zeros((32, 1, 16, 128), dtype=torch.bfloat16, device="cuda").to(dtype)
    cache = q.PagedCache(k, torch.zeros_like(k.view(torch.uint8)).view(dtype), _int32([range(32)]), scale, scale)
    q.paged_append(cache, x, x, _int32(range(512)), _int32([0] * 512))
    with np.errstate(all="ignore"):
        want = x.cpu().float().numpy() / np.float32(scale)
    want = torch.from_numpy(np.clip(want, -448, 448) if fp8 else want).to(dtype).view(-1)
    code = torch.uint8 if fp8 else torch.int16
    small = (x.cpu().float().abs().view(-1) < 2.0 ** -120) | (scale > 2.0 ** 126)
    for t in (cache.k, cache.v):
        got = t.cpu().view(-1)
        a, b = got.view(code).int(), want.view(code).int()
        both_nan = got.float().isnan() & want.float().isnan()
        assert (got.float().isnan() == want.float().isnan()).all()
        off = torch.where(both_nan, 0, (a - b).abs())
        assert (off[~small] == 0).all() and off.max() <= 1


@pytest.mark.parametrize("T", [0, 1])
def test_append_without_sequences_or_tokens(T):
    import torch
    import paper_2509_26436_amd as q
    k = torch.zeros((2, 1, 8, 64), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    new = torch.ones((T, 1, 64), dtype=torch.bfloat16, device="cuda")
    q.paged_append(q.PagedCache(k, v, _int32([[1]])), new, 2 * new, _int32([5] * T))
    assert float(k.sum()) == 64 * T and float(v[1, 0, 5].sum()) == 128 * T
    if T == 0:
        o = q.paged_attention(new, q.PagedCache(k, v, _int32([[1]])[:0]), _int32([]))
        assert o.shape == (0, 1, 64)
