"""Attention of prompts and trees over values up to bf16's largest: sums stay finite where the answer is."""
import numpy as np
import pytest

import decoding_reference as R
import prompt_reference as T

pytestmark = pytest.mark.gpu

LARGEST = float.fromhex("0x1.fep127")
# channels and new tokens of four (two) query heads a cache head: tiles of every height, keys split or not
SHAPES = [(64, 5), (64, 14), (64, 30), (64, 70), (128, 5), (128, 14), (128, 30), (128, 70), (256, 14), (256, 30)]


def _case(seed, new, lengths, kv, group, d, width):
    import paper_2509_26436_amd as q
    page = 16
    g = T.rng(seed, kv, group, d)
    tab, pages = T.table(g, lengths, page, None if width is None else width // page)
    k, v = T.cache(g, pages, kv, page, d, False)
    x = R.bf16(g.normal(0, 1.5, (sum(new), kv * group, d)))
    return g, tab, k, v, x, q.PagedCache(k, v, T.int32(tab))


def _run(x, cache, new, lengths, trees=False, **kw):
    import torch
    import paper_2509_26436_amd as q
    args = R.device(x), cache, T.int32(T.starts_of(new)), T.int32(lengths)
    if not trees:
        return R.host(q.paged_prompt_attention(*args, **kw))
    bits = np.concatenate([np.tril(np.ones((n, max(new)), bool)) for n in new])
    return R.host(q.paged_tree_attention(*args, torch.from_numpy(T.words(bits)).cuda(), **kw))


def _set(v, values):
    import torch
    v.copy_(torch.from_numpy(R.bf16(np.clip(values, -LARGEST, LARGEST))).cuda().to(torch.bfloat16))
    return R.host(v)


@pytest.mark.parametrize("trees", [False, True])
@pytest.mark.parametrize("width", [None, 8192])             # a block a tile, or parts of its keys joined
@pytest.mark.parametrize("what", ["one", "some", "largest", 2.0 ** 64, 2.0 ** 100, 2.0 ** 114, 2.0 ** 126])
@pytest.mark.parametrize("d,new", SHAPES)
def test_values_up_to_the_largest(d, new, what, width, trees):
    kv, group, news, lengths = 1, 4, [new, new], [700, 130]
    print(f"values: {what}, {d} channels, {new} tokens, width {width}, trees {trees}", flush=True)
    g, tab, k, v, x, cache = _case(1, news, lengths, kv, group, d, width)
    values = R.host(v)
    if what == "one":                                       # one key's, in the middle and in the last place
        values[tab[0, 20], 0, 3] = LARGEST * np.where(np.arange(d) % 2, 1, -1)
        values[tab[1, 129 // 16], 0, 129 % 16, 7] = LARGEST
    elif what == "some":
        values *= np.exp2(g.integers(-60, 126, values.shape))
    elif what == "largest":
        values[:] = LARGEST * np.where(np.arange(d) % 2, 1, -1)
    else:
        values *= what
    values = _set(v, values)
    o = _run(x, cache, news, lengths, trees)
    T.check(o, x, R.host(k), values, tab, T.starts_of(news), lengths, 16)
    if what == "largest":                                   # the weights' sum and the quotient: 2^-20 at most
        assert np.isfinite(o).all() and (np.abs(o) >= LARGEST * (1 - 2.0 ** -7)).all()


@pytest.mark.parametrize("width", [None, 8192])
@pytest.mark.parametrize("size", [2.0 ** 106, 2.0 ** 114, LARGEST])
@pytest.mark.parametrize("rise", [3.0, 5.0, 9.0, 40.0, 60.0, 200.0])
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("d,new", [(64, 5), (64, 70), (128, 5), (128, 14), (128, 70), (256, 30)])
def test_large_values_under_scores_that_rise(d, new, first, rise, size, width):
    """Scores rise by less or by more than the maximum's slack; the first keys, or the last, are the large
    ones: nothing of them is left, or all."""
    kv, group, length = 1, 4, 900
    print(f"values of {size}, first {first}, scores that rise by {rise}, {d} channels, {new} tokens, width {width}", flush=True)
    _, tab, k, v, x, cache = _case(2, [new], [length], kv, group, d, width)
    keys, values = np.zeros(R.host(k).shape), R.host(v)
    for j in range(length):
        at = tab[0, j // 16], 0, j % 16
        keys[at][0] = R.bf16(rise * (j // 300))
        if (j < 300) == first and (first or j >= 600):
            values[at] *= size / 8                           # (normal values stay below 8)
            values[at][0] = size
    keys, values = _set(k, keys), _set(v, values)
    x[:, :, 0] = 1.0
    o = _run(x, cache, [new], [length], scale=1.0)
    T.check(o, x, keys, values, tab, [0, new], [length], 16, scale=1.0)


@pytest.mark.parametrize("new", [5, 70])
def test_smaller_values_beside_the_largest(new):
    """Channels of ordinary and of small values beside one of the largest: their bits stay."""
    kv, group, d, length = 1, 4, 128, 700
    g, tab, k, v, x, cache = _case(3, [new], [length], kv, group, d, None)
    values = R.host(v) * np.exp2(-np.arange(d) * 0.6)
    values[..., 0] = LARGEST
    values = _set(v, values)
    o = _run(x, cache, [new], [length])
    T.check(o, x, R.host(k), values, tab, [0, new], [length], 16)
