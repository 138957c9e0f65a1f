"""Attention of trees of drafted tokens, the accepted ones moved behind their sequences, and a loop of
both with the norms and the append, against the definitions in 64 bits."""
import numpy as np
import pytest

import decoding_reference as R
import prompt_reference as T

pytestmark = pytest.mark.gpu


def _case(seed, new, past, kv, group, d, page, fp8, width=None, **scales):
    import paper_2509_26436_amd as q
    g = T.rng(seed, kv, group, d, page)
    lengths = [n + p for n, p in zip(new, past)]
    tab, pages = T.table(g, lengths, page, width)
    k, v = T.cache(g, pages, kv, page, d, fp8)
    x = R.bf16(g.normal(0, 1.5, (sum(new), kv * group, d)))
    bits = np.zeros((sum(new), max(new)), bool)
    for b, n in enumerate(new):
        first = T.starts_of(new)[b]
        bits[first:first + n, :n] = T.random_tree(g, n)
    return g, lengths, tab, k, v, x, bits, q.PagedCache(k, v, T.int32(tab), **scales)


def _run(x, cache, new, lengths, bits, **kw):
    import torch
    import paper_2509_26436_amd as q
    tree = torch.from_numpy(T.words(bits)).cuda()
    return R.host(q.paged_tree_attention(R.device(x), cache, T.int32(T.starts_of(new)), T.int32(lengths), tree, **kw))


@pytest.mark.parametrize("new,past", [([1], [0]), ([4, 1, 7], [0, 300, 31]), ([64, 3], [1000, 61]), ([70, 129], [5, 200]),
                                      ([26] * 5, [129, 0, 2000, 63, 64])])
@pytest.mark.parametrize("kv,group,d,page,fp8", [(2, 4, 128, 16, False), (1, 1, 64, 8, False), (1, 5, 256, 64, False),
                                                 (2, 3, 128, 32, True), (1, 8, 64, 16, True), (1, 2, 256, 8, True)])
def test_trees(new, past, kv, group, d, page, fp8):
    print(f"tree attention {new} behind {past} {kv} x {group} x {d} page {page} fp8 {fp8}", flush=True)
    scales = dict(k_scale=0.75, v_scale=1.5) if fp8 else {}
    _, lengths, tab, k, v, x, bits, cache = _case(1, new, past, kv, group, d, page, fp8, **scales)
    o = _run(x, cache, new, lengths, bits)
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of(new), lengths, page, bits=bits, **scales)


@pytest.mark.parametrize("width", [None, 1024])
@pytest.mark.parametrize("kw", [dict(cap=20.0), dict(scale=-0.3), dict(scale=0.4, cap=3.0)])
def test_caps_and_scales(kw, width):
    new, past, page = [12, 40, 1], [500, 3, 77], 16
    _, lengths, tab, k, v, x, bits, cache = _case(2, new, past, 2, 2, 128, page, False, width)
    o = _run(x, cache, new, lengths, bits, **kw)
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of(new), lengths, page, bits=bits, **kw)


def test_bits_of_any_kind():
    """Tokens that see nothing but the past, or nothing at all; words past the tree; fewer words than
    nodes; more tokens than keys."""
    new, past, page = [70, 5, 3], [40, 0, -2], 16
    g, lengths, tab, k, v, x, bits, cache = _case(3, new, past, 1, 2, 64, page, False)
    bits = g.random((78, 192)) < 0.4
    bits[10] = False
    bits[72] = False                       # nothing in the past either
    o = _run(x, cache, new, lengths, bits)
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of(new), lengths, page, bits=bits)
    assert (o[72] == 0).all()
    few = bits[:, :64]
    o = _run(x, cache, new, lengths, few)
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of(new), lengths, page, bits=few)


def test_words_in_a_wider_tensor():
    import torch
    import paper_2509_26436_amd as q
    new, past, page = [66, 9], [30, 100], 16
    _, lengths, tab, k, v, x, bits, cache = _case(4, new, past, 1, 4, 128, page, False)
    wide = torch.full((75, 7), -1, dtype=torch.int64, device="cuda")
    wide[:, 2:4] = torch.from_numpy(T.words(bits)).cuda()
    o = R.host(q.paged_tree_attention(R.device(x), cache, T.int32(T.starts_of(new)), T.int32(lengths), wide[:, 2:4]))
    T.check(o, x, R.host(k), R.host(v), tab, T.starts_of(new), lengths, page, bits=bits)


@pytest.mark.parametrize("fp8", [False, True])
def test_siblings_with_nan(fp8):
    """A drafted token's NaN reaches the nodes behind it only."""
    new, past, page, d = [20], [50], 16, 128
    _, lengths, tab, k, v, x, bits, cache = _case(5, new, past, 2, 2, d, page, fp8)
    kh, vh = R.host(k), R.host(v)
    node = 3
    j = past[0] + node
    v[tab[0, j // page], :, j % page] = float("nan")
    k[tab[0, j // page], :, j % page] = float("nan")
    o = _run(x, cache, new, lengths, bits)
    clean = ~bits[:, node]
    assert clean.any() and not clean.all()
    assert np.isnan(o[~clean]).all()
    for i in np.flatnonzero(clean):
        seen = T.sight(20, 70, bits=bits)[i:i + 1]
        for h in range(4):
            want, far = T.attention(x[i:i + 1, h], T.rows(kh, tab, 0, h // 2, 70, page), T.rows(vh, tab, 0, h // 2, 70, page),
                                    seen, d ** -0.5)
            assert (np.abs(o[i, h] - want) <= far).all(), (i, h)


# ------------------------------------------------------------------- accepted tokens

def _moved(t, tab, first, kept, page, pages):
    out = t.clone()
    most = tab.shape[1] * page

    def place(b, p):
        return (tab[b, p // page], p % page) if 0 <= p < most and 0 <= tab[b, p // page] < pages else None
    for b, f in enumerate(first):
        for i, node in enumerate(kept[b]):
            if node > i and place(b, f + node) and place(b, f + i):
                (sp, so), (tp, to) = place(b, f + node), place(b, f + i)
                out[tp, :, to] = t[sp, :, so]
    return out


@pytest.mark.parametrize("kv,d,page,fp8", [(2, 128, 16, False), (1, 64, 8, True), (3, 256, 32, False), (8, 128, 64, True), (1, 64, 8, False)])
@pytest.mark.parametrize("nodes,most", [(1, 1), (26, 7), (300, 270)])
def test_keep(kv, d, page, fp8, nodes, most):
    """Paths whose targets are other nodes' sources, entries that are none, pages that are none."""
    import torch
    import paper_2509_26436_amd as q
    g = T.rng(6, kv, d, nodes)
    first = [0, 5, 130, 17, -3]
    tab, pages = T.table(g, [max(f, 0) + nodes for f in first], page)
    tab[3, -1] = -1
    tab[3, 0] = pages + 4
    k, v = T.cache(g, pages, kv, page, d, fp8)
    kept = np.full((5, most + 2), -1)
    for b in range(5):
        count = [most, max(1, most // 2), most, most, most][b]
        path = np.sort(g.permutation(nodes)[:count])
        kept[b, :count] = path
    kept[2, ::3] = -5
    kept[1, -1] = 1 << 30
    raw = torch.uint8 if fp8 else torch.int16
    want = [_moved(t.view(raw), tab, first, kept, page, pages) for t in (k, v)]
    cache = q.PagedCache(k, v, T.int32(tab))
    q.paged_keep(cache, T.int32(first), T.int32(np.pad(kept, ((0, 0), (0, 3)), constant_values=9))[:, :most + 2])
    assert torch.equal(k.view(raw), want[0]) and torch.equal(v.view(raw), want[1])


def test_keep_nothing():
    import torch
    import paper_2509_26436_amd as q
    k = torch.randn(4, 1, 8, 64, device="cuda").bfloat16()
    v, want = k.clone(), k.clone()
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")          # noqa: E731
    q.paged_keep(q.PagedCache(k, v, i32(2, 2)), i32(2), i32(2, 0))
    q.paged_keep(q.PagedCache(k, v, i32(0, 2)), i32(0), i32(0, 3))
    q.paged_keep(q.PagedCache(k, v, i32(2, 0)), i32(2), i32(2, 3) + 5)
    q.paged_keep(q.PagedCache(k, v, i32(2, 2)), i32(2), torch.arange(6, dtype=torch.int32, device="cuda").reshape(2, 3)[:1].expand(2, 3).contiguous())
    assert torch.equal(k, want) and torch.equal(v, want)


@pytest.mark.parametrize("moved", [(), (0,), (1,), (2,), (0, 2)])
@pytest.mark.parametrize("fp8", [False, True])
def test_keep_runs_that_stay(moved, fp8):
    """384 entries, of which whole runs of 128 stay where they are; in the others each source is the
    next entry's target, and one sequence has no pages at all."""
    import torch
    import paper_2509_26436_amd as q
    g = T.rng(8)
    page, kv, d, most = 16, 2, 128, 384
    tab, pages = T.table(g, [most + 40] * 3, page)
    tab[1] = -1
    k, v = T.cache(g, pages, kv, page, d, fp8)
    kept = np.tile(np.arange(most), (3, 1))
    for run in moved:
        kept[:, 128 * run:128 * run + 128] += 1
    raw = torch.uint8 if fp8 else torch.int16
    want = [_moved(t.view(raw), tab, [3, 3, 30], kept, page, pages) for t in (k, v)]
    q.paged_keep(q.PagedCache(k, v, T.int32(tab)), T.int32([3, 3, 30]), T.int32(kept))
    assert torch.equal(k.view(raw), want[0]) and torch.equal(v.view(raw), want[1])


# ------------------------------------------------------------------- together

@pytest.mark.parametrize("captured", [False, True])
def test_draft_verify_keep(captured):
    """A prompt, then rounds of drafted trees: norms and rotation by depth, append by place, tree
    attention, the accepted path kept; at the end the cache is that of the accepted tokens alone."""
    import torch
    import paper_2509_26436_amd as q
    S, H, KV, d, page, nodes = 3, 8, 2, 128, 16, 6
    g = T.rng(7)
    freqs = q.rotary_frequencies(d)
    prompt = [37, 1, 90]
    tab = g.permutation(S * 12).reshape(S, 12)
    k = torch.full((S * 12, KV, page, d), np.nan, dtype=torch.bfloat16, device="cuda")
    cache = q.PagedCache(k, torch.full_like(k, np.nan), T.int32(tab))
    weights = [R.device(R.bf16(1 + 0.2 * g.normal(size=d))) for _ in range(2)]

    def block(qkv, turns, places, sequences):
        x, y = q.head_norm_rotary(qkv[:, :H], qkv[:, H:H + KV], turns, freqs, *weights)
        q.paged_append(cache, y, qkv[:, H + KV:], places, sequences)
        return x, y

    def tokens(n):
        return R.device(R.bf16(g.normal(0, 1.2, (n, H + 2 * KV, d))))

    stored = [np.zeros((0, 2, KV, d)) for _ in range(S)]
    qkv = tokens(sum(prompt))
    places = T.int32(np.concatenate([np.arange(n) for n in prompt]))
    sequences = T.int32(np.repeat(np.arange(S), prompt))
    x, y = block(qkv, places, places, sequences)
    o = q.paged_prompt_attention(x, cache, T.int32(T.starts_of(prompt)), T.int32(prompt))
    T.check(R.host(o), R.host(x), R.host(cache.k), R.host(cache.v), tab, T.starts_of(prompt), prompt, page)
    new = np.stack([R.host(y), R.host(qkv[:, H + KV:])], 1)
    for b in range(S):
        stored[b] = new[T.starts_of(prompt)[b]:T.starts_of(prompt)[b + 1]]

    first = np.array(prompt)
    static = dict(qkv=tokens(S * nodes), turns=T.int32(np.zeros(S * nodes)), places=T.int32(np.zeros(S * nodes)),
                  lengths=T.int32(np.zeros(S)), first=T.int32(first), kept=T.int32(np.full((S, nodes), -1)),
                  tree=torch.zeros(S * nodes, 1, dtype=torch.int64, device="cuda"))
    starts, sequences = T.int32(np.arange(S + 1) * nodes), T.int32(np.repeat(np.arange(S), nodes))
    workspace = q.paged_prompt_workspace(S * nodes, H, cache)

    def verify():
        x, y = block(static["qkv"], static["turns"], static["places"], sequences)
        return x, y, q.paged_tree_attention(x, cache, starts, static["lengths"], static["tree"], workspace=workspace)

    def keep():
        q.paged_keep(cache, static["first"], static["kept"])

    if captured:
        saved = cache.k.clone(), cache.v.clone()
        verify(), keep()
        torch.cuda.synchronize()
        graphs = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[0]):
            outs = verify()
        with torch.cuda.graph(graphs[1]):
            keep()
        cache.k.copy_(saved[0]), cache.v.copy_(saved[1])

    for step in range(4):
        trees = [T.random_tree(g, nodes) for _ in range(S)]
        depth = np.stack([t.sum(1) - 1 for t in trees])
        static["qkv"].copy_(tokens(S * nodes))
        static["turns"].copy_(T.int32((first[:, None] + depth).reshape(-1)))
        static["places"].copy_(T.int32((first[:, None] + np.arange(nodes)).reshape(-1)))
        static["lengths"].copy_(T.int32(first + nodes))
        static["first"].copy_(T.int32(first))
        bits = np.concatenate(trees)
        static["tree"].copy_(torch.from_numpy(T.words(bits)))
        if captured:
            graphs[0].replay()
            x, y, o = outs
        else:
            x, y, o = verify()
        torch.cuda.synchronize()
        T.check(R.host(o), R.host(x), R.host(cache.k), R.host(cache.v), tab, [0, nodes, 2 * nodes, 3 * nodes],
                (first + nodes).tolist(), page, bits=bits)
        leaves = g.integers(0, nodes, S)
        paths = [np.flatnonzero(trees[b][leaves[b]]) for b in range(S)]
        kept = np.full((S, nodes), -1)
        new = np.stack([R.host(y), R.host(static["qkv"][:, H + KV:])], 1)
        for b, path in enumerate(paths):
            kept[b, :len(path)] = path
            stored[b] = np.concatenate([stored[b], new[b * nodes + path]])
        static["kept"].copy_(T.int32(kept))
        if captured:
            graphs[1].replay()
        else:
            keep()
        first = first + np.array([len(p) for p in paths])
        for b in range(S):
            for t, name in ((cache.k, 0), (cache.v, 1)):
                got = np.stack([T.rows(R.host(t), tab, b, h, int(first[b]), page) for h in range(KV)], 1)
                assert np.array_equal(got, stored[b][:, name]), (step, b, name)
