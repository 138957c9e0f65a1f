"""Attention of prompts over infinite values: a row that sees one has it, whatever its weight and wherever
among the keys it lies."""
import numpy as np
import pytest

import decoding_reference as R
import prompt_reference as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width", [None, 8192])             # a block a tile, or parts of its keys joined
@pytest.mark.parametrize("rise", [0.0, 2.0, 30.0, 200.0, -200.0])
@pytest.mark.parametrize("d,new", [(64, 5), (64, 14), (64, 70), (128, 5), (128, 14), (128, 30), (128, 70), (256, 14), (256, 30)])
def test_infinite_values_under_scores_that_rise_or_fall(d, new, rise, width):
    """Every score is finite, so every weight is above zero: a channel that holds infinities of one sign is
    one, of both NaN, and the others are as if there were none."""
    import torch
    import paper_2509_26436_amd as q
    kv, group, page, length = 1, 4, 16, 900
    print(f"infinite values, scores that rise by {rise}, {d} channels, {new} tokens, width {width}", flush=True)
    g = T.rng(1, d, new)
    tab, pages = T.table(g, [length], page, None if width is None else width // page)
    k, v = T.cache(g, pages, kv, page, d, False)
    keys, values = np.zeros(R.host(k).shape), R.host(v)
    for j in range(length):
        keys[tab[0, j // page], 0, j % page, 0] = R.bf16(rise * (j // 150))
    at = lambda j: (tab[0, j // page], 0, j % page)          # noqa: E731
    marks = [(j, 3 + i, np.inf) for i, j in enumerate((0, 100, 333, 600, 899 - new))] + [(140, 9, -np.inf), (290, 10, -np.inf),
                                                                                       (10, 11, np.inf), (600, 11, -np.inf)]
    clean = values.copy()
    for j, channel, what in marks:
        values[at(j)][channel] = what
        clean[at(j)][channel] = 0.0
    k.copy_(torch.from_numpy(keys).cuda().to(torch.bfloat16))
    v.copy_(torch.from_numpy(values).cuda().to(torch.bfloat16))
    x = np.zeros((new, group, d))
    x[:, :, 0] = 1.0
    cache = q.PagedCache(k, v, T.int32(tab))
    o = R.host(q.paged_prompt_attention(R.device(x), cache, T.int32([0, new]), T.int32([length]), scale=1.0))
    assert (o[:, :, 3:8] == np.inf).all() and (o[:, :, 9:11] == -np.inf).all() and np.isnan(o[:, :, 11]).all()
    o[:, :, [3, 4, 5, 6, 7, 9, 10, 11]] = 0.0
    clean[..., [3, 4, 5, 6, 7, 9, 10, 11]] = 0.0
    T.check(o, x, keys, clean, tab, [0, new], [length], page, scale=1.0)
