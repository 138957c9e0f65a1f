"""Attention of prompts and trees under scores of any size that fp32 holds: weights stay finite, and a
row's largest key keeps its weight."""
import numpy as np
import pytest

import decoding_reference as R
import prompt_reference as T

pytestmark = pytest.mark.gpu

LOG2E = 1.4426950408889634
# cache type, channels, new tokens: tiles of every height, keys split over waves and not
SHAPES = [(False, 64, 3), (True, 64, 70), (False, 128, 3), (True, 128, 12), (False, 128, 40), (True, 128, 70),
          (False, 256, 30), (True, 256, 60)]


def _case(seed, new, lengths, group, d, page, fp8, width=None):
    """Queries and keys of zeros, values from one to two: no weights give a zero."""
    import torch
    import paper_2509_26436_amd as q
    g = T.rng(seed, group, d)
    tab, pages = T.table(g, lengths, page, None if width is None else width // page)
    dtype = torch.float8_e4m3fn if fp8 else torch.bfloat16
    k = torch.zeros(pages, 1, page, d, device="cuda", dtype=dtype)
    v = torch.from_numpy(g.uniform(1, 2, k.shape)).cuda().to(dtype)
    return g, tab, k, v, np.zeros((sum(new), group, d)), q.PagedCache(k, v, T.int32(tab))


def _call(x, cache, new, lengths, tree, **kw):
    import torch
    import paper_2509_26436_amd as q
    args = R.device(x), cache, T.int32(T.starts_of(new)), T.int32(lengths)
    if tree is None:
        return R.host(q.paged_prompt_attention(*args, **kw))
    return R.host(q.paged_tree_attention(*args, torch.from_numpy(T.words(tree)).cuda(), **kw))


def _check(o, s, seen, v):
    """o [n, d] under scores s [n, L].  The addition of a score's two products is off by 2^-23 of it, its
    product with the factor (whose own rounding is every key's) by 2^-24, the maximum that is taken off by
    as much where it is not the same for all: so a weight is off by a factor of up to f = 2^(2^-22 |s| log2 e).
    Quotients of such weights move a mean by at most (f^2 - 1) / 2 of the mean distance from it, and never
    out of the values' hull.  What is left is the bound of equal scores."""
    for i in range(len(o)):
        j = np.flatnonzero(seen[i])
        p = np.exp(s[i, j] - s[i, j].max())
        p /= p.sum()
        # (keys whose weight is none, whatever their error, do not count)
        counts = p > 2.0 ** -149
        e = 2.0 ** -22 * np.abs(s[i, j][counts]).max() * LOG2E
        want = p @ v[j]
        n = len(j)
        spread = p @ np.abs(v[j] - want)
        _, far = T.attention(np.zeros((1, 1)), np.zeros((n, 1)), v[j], np.ones((1, n), bool), 1.0)
        with np.errstate(over="ignore"):
            moved = np.where(spread > 0, spread * np.expm1(2 * e * np.log(2)) / 2, 0.0)
        off = np.abs(o[i] - want)
        assert (off <= far[0] + moved).all(), (i, e, float((off - far[0] - moved).max()))
        assert (o[i] >= v[j][counts].min(0) - far[0]).all() and (o[i] <= v[j][counts].max(0) + far[0]).all(), i


@pytest.mark.parametrize("trees", [False, True])
@pytest.mark.parametrize("width", [None, 8192])
@pytest.mark.parametrize("size", [2.0 ** 19, 2.0 ** 24, 2.0 ** 28, 2.0 ** 36, 2.0 ** 126])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("fp8,d,new", SHAPES)
def test_equal_scores_average_the_values(fp8, d, new, sign, size, width, trees):
    """Every key of a row has the same score, a different one from row to row: all mantissas of bf16 from
    one to 1.25 times the size (up to 1.8 times in units of log2)."""
    import torch
    group, page, past = 2, 16, 517
    print(f"scores {sign} x {size}, {d} channels fp8 {fp8}, {new} tokens, width {width}, trees {trees}", flush=True)
    lengths = [past + new]
    _, tab, k, v, x, cache = _case(1, [new], lengths, group, d, page, fp8, width)
    k[:, 0, :, 5] = 64.0
    x[..., 5] = sign * size / 64.0 * (1 + (np.arange(new * group).reshape(new, group) % 32) / 128.0)
    bits = np.tril(np.ones((new, new), bool)) if trees else None
    o = _call(x, cache, [new], lengths, bits, scale=1.0)
    vv, seen = T.rows(R.host(v), tab, 0, 0, lengths[0], page), T.sight(new, lengths[0])
    for h in range(group):
        _check(o[:, h], np.zeros(seen.shape), seen, vv)


@pytest.mark.parametrize("rise", [3.0, 4.5, 5.5, 100.0])
@pytest.mark.parametrize("size", [2.0 ** 18, 2.0 ** 21, 2.0 ** 23, 2.0 ** 24, 2.0 ** 25])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("fp8,d,new", SHAPES)
def test_scores_that_rise_by_less_and_by_more_than_the_slack(fp8, d, new, sign, size, rise):
    """Keys whose scores lie some units above those of keys before them, at sizes where fp32 scores are a
    unit apart."""
    group, page, past = 2, 16, 900
    print(f"scores {sign} x {size} that rise by {rise}, {d} channels fp8 {fp8}, {new} tokens", flush=True)
    lengths = [past + new]
    _, tab, k, v, x, cache = _case(2, [new], lengths, group, d, page, fp8)
    level = np.floor(rise * (np.arange(lengths[0]) // 300))
    kh = np.zeros(R.host(k).shape)
    kh[..., 5] = 64.0
    for j in range(lengths[0]):
        kh[tab[0, j // page], 0, j % page, 9] = level[j]
    k.copy_(R.device(kh).to(k.dtype))
    kh = R.host(k)
    level = T.rows(kh, tab, 0, 0, lengths[0], page)[:, 9]
    x[..., 5] = sign * size / 64.0 * (1 + (np.arange(new * group).reshape(new, group) % 32) / 128.0)
    x[..., 9] = 1.0
    o = _call(x, cache, [new], lengths, None, scale=1.0)
    vv, seen = T.rows(R.host(v), tab, 0, 0, lengths[0], page), T.sight(new, lengths[0])
    for h in range(group):
        _check(o[:, h], 64.0 * x[:, h, 5:6] + level[None], seen, vv)


@pytest.mark.parametrize("fp8,d,new", [(False, 128, 3), (False, 128, 100), (False, 256, 60), (True, 64, 12)])
def test_scores_from_one_end_of_fp32_to_the_other(fp8, d, new):
    """A row's keys have scores of -3e38, 0 and, last, 3e38: the last take all of the weight."""
    group, page, past = 2, 16, 600
    lengths = [past + new]
    _, tab, k, v, x, cache = _case(3, [new], lengths, group, d, page, fp8)
    kh = np.zeros(R.host(k).shape)
    score = np.repeat([-1.0, 0.0, 1.0], 200)
    for j in range(past):
        kh[tab[0, j // page], 0, j % page, 5] = 64.0 * score[j]
    k.copy_(R.device(kh).to(k.dtype))
    x[..., 5] = 1.25 * 2.0 ** 121
    o = _call(x, cache, [new], lengths, None, scale=1.0)
    vv = T.rows(R.host(v), tab, 0, 0, lengths[0], page)
    seen = np.zeros((new, lengths[0]), bool)
    seen[:, 400:600] = True
    for h in range(group):
        _check(o[:, h], np.zeros(seen.shape), seen, vv)
