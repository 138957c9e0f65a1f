"""Strides of dimensions of size one reach no element: they decide nothing."""
import math

import numpy as np
import pytest

import decoding_reference as R
import test_gpu_paged as P

pytestmark = pytest.mark.gpu


def _odd(t, dim):
    """t's elements with an odd stride along `dim`, of size one."""
    import torch
    strides = list(t.stride())
    strides[dim] = 2 * t.numel() + 3
    return torch.as_strided(t, t.shape, strides)


@pytest.mark.parametrize("S,kv,group,dim", [(1, 2, 2, 0), (3, 1, 1, 1)])
def test_attention_of_one_sequence_or_head(S, kv, group, dim):
    import torch
    import paper_2509_26436_amd as q
    lengths, page, d = [70, 33, 5][:S], 16, 128
    _, table, k, v, x, cache = P._attention_case(31, lengths, kv, group, d, page, False)
    out = _odd(torch.zeros((S, kv * group, d), dtype=torch.bfloat16, device="cuda"), dim)
    o = q.paged_attention(_odd(R.device(x), dim), cache, P._int32(lengths), out=out)
    assert o is out or o.data_ptr() == out.data_ptr()
    P._check(R.host(out), x, R.host(k), R.host(v), table, lengths, page)


@pytest.mark.parametrize("T,H,dim", [(1, 5, 0), (6, 1, 1)])
def test_rotary_of_one_token_or_head(T, H, dim):
    """In place too, where only the strides that reach no element differ."""
    import paper_2509_26436_amd as q
    rng = np.random.Generator(np.random.PCG64([32, T]))
    x, positions = R.bf16(rng.normal(0, 1, (T, H, 64))), rng.integers(0, 5000, T)
    f = q.rotary_frequencies(64)
    want, far = R.rotate(x, positions, f.cpu().numpy(), "half")
    far = R.HALF_BF16 * np.abs(want) + (1 + R.HALF_BF16) * far
    t = R.device(x)
    for y in (q.rotary(_odd(t, dim), P._int32(positions), f), q.rotary(t, P._int32(positions), f, out=_odd(t, dim))):
        assert (np.abs(R.host(y) - want) <= far).all()
    assert (np.abs(R.host(t) - want) <= far).all()


def test_append_of_one_token():
    import torch
    import paper_2509_26436_amd as q
    k = torch.zeros((2, 3, 8, 64), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    rows = R.bf16(np.random.Generator(np.random.PCG64(33)).normal(0, 1, (2, 1, 3, 64)))
    new = [_odd(R.device(r), 0) for r in rows]
    q.paged_append(q.PagedCache(k, v, P._int32([[1]])), *new, P._int32([5]))
    for cache, r in zip((k, v), rows):
        np.testing.assert_array_equal(R.host(cache)[1, :, 5], r[0])
        assert math.isclose(float(cache.float().abs().sum()), float(np.abs(r).sum()), rel_tol=1e-6)
