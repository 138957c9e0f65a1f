"""The operators together, as a decoding loop uses them: an attention block of two new tokens after
prompts, in eager steps and as one captured graph, against the same block in 64 bits."""
import math

import numpy as np
import pytest

import decoding_reference as R

pytestmark = pytest.mark.gpu

S, HIDDEN, H, KV, D, PAGE = 3, 512, 8, 2, 128, 16
WIDTH = (H + 2 * KV) * D


def _weights(rng):
    import paper_2509_26436_amd as q
    out = {}
    for name, (N, K) in {"qkv": (WIDTH, HIDDEN), "out": (HIDDEN, H * D)}.items():
        w = R.bf16(rng.normal(0, K ** -0.5, (N, K)))
        out[name] = q.mxfp4_quantize(R.device(w)), R.mx_values(*R.mx_quantize(w))
    return out


def _step(q, x, weights, cache, positions, lengths, sequences, freqs, n):
    """n new tokens a sequence: their projections and rotated queries, the last one's attention and
    block output."""
    qkv = q.mxfp4_linear(x, weights["qkv"][0]).view(-1, H + 2 * KV, D)
    turned = q.rotary(qkv[:, :H], positions, freqs)
    q.paged_append(cache, qkv[:, H:H + KV], qkv[:, H + KV:], positions, sequences, freqs)
    o = q.paged_attention(turned[n - 1::n], cache, lengths)
    return qkv, turned, o, q.mxfp4_linear(o.view(S, H * D), weights["out"][0])


def test_decoding_steps_eager_and_captured():
    import torch
    import paper_2509_26436_amd as q
    rng = np.random.Generator(np.random.PCG64(77))
    weights, freqs = _weights(rng), q.rotary_frequencies(D)
    f = freqs.cpu().numpy()
    table = torch.from_numpy(rng.permutation(S * 8).reshape(S, 8).astype(np.int32)).cuda()
    k = torch.full((S * 8, KV, PAGE, D), math.nan, dtype=torch.bfloat16, device="cuda")
    cache = q.PagedCache(k, torch.full_like(k, math.nan), table)
    int32 = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()     # noqa: E731

    def stored(t, n):
        """The first n positions of every sequence, [S, n, KV, D]."""
        pages = R.host(t)[table.cpu().numpy()]
        return pages.transpose(0, 1, 3, 2, 4).reshape(S, -1, KV, D)[:, :n]

    def check(x, qkv, turned, o, y, first, n):
        """Each operator's output from the values that the one before it stored."""
        a = R.mx_values(*R.mx_quantize(x))
        want, far = R.linear(a, weights["qkv"][1])
        assert (np.abs(R.host(qkv).reshape(-1, WIDTH) - want) <= far).all()
        rows, turned, got = R.host(qkv), R.host(turned), R.host(o)
        want, far = R.rotate(rows[:, :H + KV], np.tile(np.arange(first, first + n), S), f, "half")
        far = R.HALF_BF16 * np.abs(want) + (1 + R.HALF_BF16) * far
        assert (np.abs(turned - want[:, :H]) <= far[:, :H]).all()
        k, v = stored(cache.k, first + n), stored(cache.v, first + n)
        assert (np.abs(k[:, first:].reshape(S * n, KV, D) - want[:, H:]) <= far[:, H:]).all()
        np.testing.assert_array_equal(v[:, first:].reshape(S * n, KV, D), rows[:, H + KV:])
        for b in range(S):
            for h in range(KV):
                heads = slice(h * H // KV, (h + 1) * H // KV)
                want, far = R.attention(turned[b * n + n - 1, heads], k[b, :, h], v[b, :, h], 1 / math.sqrt(D))
                assert (np.abs(got[b, heads] - want) <= far).all()
        a = R.mx_values(*R.mx_quantize(got.reshape(S, H * D)))
        want, far = R.linear(a, weights["out"][1])
        assert (np.abs(R.host(y) - want) <= far).all()

    # prompts of 37 tokens, then a step, both eager
    first = 0
    for n in (37, 1):
        x = R.bf16(rng.normal(0, 1, (S * n, HIDDEN)))
        args = (int32(np.tile(np.arange(first, first + n), S)), int32([first + n] * S), int32(np.repeat(np.arange(S), n)))
        check(x, *_step(q, R.device(x), weights, cache, *args, freqs, n), first, n)
        first += n
    # one captured step, replayed for the next tokens
    x_in, positions, lengths = R.device(np.zeros((S, HIDDEN))), int32([0] * S), int32([0] * S)
    sequences = int32(range(S))
    saved = cache.k.clone(), cache.v.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _step(q, x_in, weights, cache, positions, lengths, sequences, freqs, 1)
    cache.k.copy_(saved[0])
    cache.v.copy_(saved[1])
    for _ in range(4):
        x = R.bf16(rng.normal(0, 1, (S, HIDDEN)))
        x_in.copy_(R.device(x))
        positions.fill_(first)
        lengths.fill_(first + 1)
        graph.replay()
        torch.cuda.synchronize()
        check(x, *outs, first, 1)
        first += 1
