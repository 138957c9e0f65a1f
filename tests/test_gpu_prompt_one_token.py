"""One new token a sequence: as a prompt of one, as a tree of one and as a decoding step it has the same
answer, up to what each of them rounds."""
import numpy as np
import pytest

import decoding_reference as R
import prompt_reference as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,fp8", [(64, False), (64, True), (128, False), (128, True), (256, False), (256, True)])
@pytest.mark.parametrize("window", [0, 100])
def test_one_token_three_ways(d, fp8, window):
    import torch
    import paper_2509_26436_amd as q
    kv, group, page, lengths = 2, 4, 16, [1, 700, 33, 0, 129]
    print(f"one token, {d} channels fp8 {fp8}, window {window}", flush=True)
    g = T.rng(1, d, fp8)
    tab, pages = T.table(g, lengths, page)
    k, v = T.cache(g, pages, kv, page, d, fp8)
    x = R.bf16(g.normal(0, 1.5, (len(lengths), kv * group, d)))
    cache, starts, n = q.PagedCache(k, v, T.int32(tab)), T.int32(np.arange(len(lengths) + 1)), T.int32(lengths)
    step = q.paged_attention(R.device(x), cache, n, window=window)
    prompt = q.paged_prompt_attention(R.device(x), cache, starts, n, window=window)
    answers = [(step, 2.0 ** -16), (prompt, T.HALF_FP16)]
    if window == 0:
        own = torch.ones((len(lengths), 1), dtype=torch.int64, device="cuda")
        answers.append((q.paged_tree_attention(R.device(x), cache, starts, n, own), T.HALF_FP16))
        assert torch.equal(answers[2][0], prompt)
    for o, weight in answers:
        T.check(R.host(o), x, R.host(k), R.host(v), tab, list(range(len(lengths) + 1)), lengths, page, window=window,
                weight=weight)
