"""Attention over the paged cache where blocks share the keys of many heads: runs of several units that
begin and end inside heads, parts that several blocks leave, empty sequences between, more sequences
than a block counts at once; and every key counted visibly."""
import math

import numpy as np
import pytest

import decoding_reference as R
import test_gpu_paged as P

pytestmark = pytest.mark.gpu

UNIT, TILE = 128, 32          # keys of a unit; a window's first unit begins at a multiple of 32


def _runs(lengths, parts, window, blocks):
    """How `blocks` blocks share these sequences' units in equal runs: what happens in them."""
    heads = []
    for n in lengths:
        first = (max(0, n - window) if window else 0) // TILE * TILE
        heads += [-(-(n - first) // UNIT)] * parts
    heads = [u for u in heads if u]
    total, seen = sum(heads), set()
    ends = np.cumsum(heads)
    each, more = divmod(total, blocks)
    for i in range(blocks):
        begin = i * each + min(i, more)
        end = begin + each + (i < more)
        a, b = np.searchsorted(ends, [begin, end - 1], side="right")
        inside = b - a - 1 + (begin == ends[a] - heads[a]) + (end == ends[b] and b > a)
        seen |= {"several units"} if end - begin > 1 else set()
        seen |= {"begins inside a head"} if begin > ends[a] - heads[a] else set()
        seen |= {"whole heads inside"} if inside > 0 else set()
        seen |= {"leaves two parts"} if b > a and begin > ends[a] - heads[a] and end < ends[b] else set()
        seen |= {"inside one head"} if a == b and begin > ends[a] - heads[a] and end < ends[a] else set()
    seen |= {"uneven runs"} if more else set()
    return total, seen


def _shared(cache, S, heads, d, lengths, window):
    """That the call shares the work, and how (with the most blocks that it may take)."""
    import paper_2509_26436_amd as q
    kv = cache.k.shape[1]
    ws = q.paged_attention_workspace(S, heads, cache, window)
    # two parts of 16 queries a block: d sums, a maximum and a sum each, and where to join them
    blocks = ws.numel() // (32 * (d + 2) * 4 + 24)
    parts = kv * -(-heads // kv // 16)
    total, seen = _runs(lengths, parts, window, blocks)
    assert total > 2 * blocks and "several units" in seen, (total, blocks)
    return seen


CASES = {
    # name: sequences, cache heads, group, d, page, e4m3, shortest, longest, empty one in, window
    "bf16": (24, 8, 4, 128, 16, False, 1, 4096, 5, 0),
    "e4m3": (24, 8, 5, 128, 64, True, 1, 4096, 4, 0),
    "d64": (30, 8, 2, 64, 8, False, 1, 4000, 3, 0),
    "d64 e4m3": (30, 8, 16, 64, 32, True, 100, 4000, 3, 0),
    "d256": (12, 6, 3, 256, 16, False, 1, 4096, 4, 0),
    "d256 e4m3": (20, 6, 2, 256, 16, True, 1, 4096, 6, 0),
    "two tiles": (14, 6, 20, 128, 16, False, 1, 4096, 5, 0),
    "three tiles e4m3": (18, 4, 40, 64, 128, True, 1, 4096, 5, 0),
    "window": (40, 8, 4, 128, 16, False, 0, 4096, 7, 1777),
    "window e4m3": (40, 8, 1, 64, 16, True, 0, 4096, 7, 2100),
    "many sequences": (700, 2, 2, 64, 16, False, 0, 500, 3, 0),
    "many sequences e4m3": (1100, 2, 3, 128, 32, True, 0, 700, 2, 0),
    "one long": (1, 2, 3, 64, 64, False, 70001, 70001, 0, 0),
}


def _case(name, ones):
    """Sequences over pages that they share, each page once a sequence."""
    import torch
    import paper_2509_26436_amd as q
    S, kv, group, d, page, fp8, lo, hi, empty, window = CASES[name]
    rng = P._rng(41, S, kv, group, d, page)
    lengths = rng.integers(lo, hi + 1, S)
    if empty:
        lengths[::empty] = 0
        lengths[-1], lengths[1] = hi, UNIT * (hi // UNIT)
    lengths = lengths.tolist()
    width = max(4096, hi) // page + 1                   # wide enough that blocks share
    pages = -(-hi // page) + 3
    table = np.full((S, width), -1, np.int64)
    for b, n in enumerate(lengths):
        table[b, :-(-n // page)] = rng.permutation(pages)[:-(-n // page)]
    shape = (pages, kv, page, d)
    dtype = torch.float8_e4m3fn if fp8 else torch.bfloat16
    if ones:
        k = np.zeros(shape)
        v = np.eye(d)[rng.integers(0, d, shape[:3])]
    else:
        k, v = rng.choice([-1.0, 1.0], shape), rng.normal(0, 1, shape)
    k, v = (torch.from_numpy(t).cuda().to(torch.bfloat16).to(dtype) for t in (k, v))
    cache = q.PagedCache(k, v, P._int32(table))
    seen = _shared(cache, S, kv * group, d, lengths, window)
    return rng, lengths, table, cache, seen


def test_the_cases_have_every_kind_of_run():
    seen = [_case(name, True)[-1] for name in CASES]
    for kind in ("begins inside a head", "whole heads inside", "leaves two parts", "inside one head", "uneven runs"):
        assert sum(kind in s for s in seen) >= 3, kind


def _check_counts(o, table, cache, lengths, group, window, exact=True):
    """o: outputs under equal weights of values that are 1 in one channel."""
    pages, kv, page, d = cache.v.shape
    channel = R.host(cache.v).argmax(-1)                # [pages, kv, page]
    for b, n in enumerate(lengths):
        if n == 0:
            assert (o[b] == 0).all()
            continue
        first = max(0, n - window) if window else 0
        at = channel[table[b, :-(-n // page)]].transpose(1, 0, 2).reshape(kv, -1)[:, first:n]
        counts = np.stack([np.bincount(a, minlength=d) for a in at])
        off = np.abs(o[b].reshape(kv, group, d) * (n - first) - counts[:, None])
        assert (off <= R.HALF_BF16 * counts[:, None] + 1e-3).all(), (b, n)
        assert not exact or counts.max() < 120 and (off < 0.5).all(), (b, n)


def _own_directions(rng, table, kh, lengths, group, window, d):
    """Queries, each the direction of one key that counts (of keys with channels +-1)."""
    kv, page = kh.shape[1:3]
    x = np.zeros((len(lengths), kv * group, d))
    for b, n in enumerate(lengths):
        first = max(0, n - window) if window else 0
        if n == 0:
            continue
        start = first // TILE * TILE
        borders = [first, n - 1, *(start + s + e for s in range(UNIT, n - start, UNIT) for e in (-1, 0)),
                   *(start + s + e for s in (8, 32, 64, 96) for e in (-1, 0))]
        for h in range(kv * group):
            j = borders[(h + b) % 2] if h < 2 else int(rng.choice(borders)) if h % 3 else int(rng.integers(first, n))
            j = min(max(j, first), n - 1)
            # scores of 2 d for the key, at most 2 (d - 16) for nearly all others: e^-32 each
            x[b, h] = 2 * math.sqrt(d) * kh[table[b, j // page], h // group, j % page]
    return R.bf16(x)


@pytest.mark.parametrize("name", CASES)
def test_every_key_counts_once(name):
    """Equal weights over values that are 1 in one channel: n times an output counts the keys of that
    channel, and every one of at most 120 shows (bf16 holds 1 / 256)."""
    import torch
    import paper_2509_26436_amd as q
    print(f"counted keys: {name}", flush=True)
    S, kv, group, d, page, fp8, lo, hi, empty, window = CASES[name]
    _, lengths, table, cache, _ = _case(name, True)
    o = R.host(q.paged_attention(torch.zeros((S, kv * group, d), dtype=torch.bfloat16, device="cuda"), cache,
                                 P._int32(lengths), window=window))
    _check_counts(o, table, cache, lengths, group, window, exact=name != "one long")


@pytest.mark.parametrize("name", CASES)
def test_every_query_finds_its_key(name):
    """Each query is one key's own direction, so that the output is that key's value: the first and the
    last that count, those beside the borders of units, tiles and groups of eight, and any."""
    import paper_2509_26436_amd as q
    print(f"found keys: {name}", flush=True)
    S, kv, group, d, page, fp8, lo, hi, empty, window = CASES[name]
    rng, lengths, table, cache, _ = _case(name, False)
    kh, vh = R.host(cache.k), R.host(cache.v)
    x = _own_directions(rng, table, kh, lengths, group, window, d)
    o = R.host(q.paged_attention(R.device(x), cache, P._int32(lengths), window=window))
    P._check(o, x, kh, vh, table, lengths, page, window=window)


@pytest.mark.parametrize("window", [0, 1, 50])
@pytest.mark.parametrize("longest", [128, 512])
@pytest.mark.parametrize("kv,group,d,fp8", [(2, 4, 128, False), (3, 5, 128, True), (32, 2, 64, False),
                                            (2, 20, 64, True), (4, 1, 256, False), (1, 3, 256, True)])
def test_a_block_a_head(kv, group, d, fp8, longest, window):
    """The same two in one launch: blocks of one (many heads), two and four waves; lengths around every
    border of groups of eight, tiles and steps."""
    import torch
    import paper_2509_26436_amd as q
    print(f"a block a head: {kv} x {group} x {d} fp8 {fp8} longest {longest} window {window}", flush=True)
    page = 16
    lengths = [n for n in (0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 159, 160,
                           161, 191, 255, 256, 257, 300, 383, 384, 385, 511, 512) if n <= longest]
    S, width, pages = len(lengths), longest // page, longest // page + 2
    rng = P._rng(42, kv, group, d, longest)
    table = np.stack([rng.permutation(pages)[:width] for _ in lengths])
    shape = (pages, kv, page, d)
    dtype = torch.float8_e4m3fn if fp8 else torch.bfloat16

    def cache_of(k, v):
        k, v = (torch.from_numpy(t).cuda().to(torch.bfloat16).to(dtype) for t in (k, v))
        return q.PagedCache(k, v, P._int32(table))
    cache = cache_of(np.zeros(shape), np.eye(d)[rng.integers(0, d, shape[:3])])
    assert q.paged_attention_workspace(S, kv * group, cache, window) is None
    x = torch.zeros((S, kv * group, d), dtype=torch.bfloat16, device="cuda")
    o = q.paged_attention(x, cache, P._int32(lengths), window=window)
    _check_counts(R.host(o), table, cache, lengths, group, window)
    cache = cache_of(rng.choice([-1.0, 1.0], shape), rng.normal(0, 1, shape))
    kh, vh = R.host(cache.k), R.host(cache.v)
    x = _own_directions(rng, table, kh, lengths, group, window, d)
    o = q.paged_attention(R.device(x), cache, P._int32(lengths), window=window)
    P._check(R.host(o), x, kh, vh, table, lengths, page, window=window)
