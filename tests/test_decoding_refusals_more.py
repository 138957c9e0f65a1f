"""More calls that the decoding entry points refuse on the host, before anything is launched."""
import os

import pytest

import paper_2509_26436_amd as q
from test_decoding_refusals import EUNSUP, EWS, _attend

LONG = dict(width=4096, row=4096)     # a call that would go on to ask for its workspace


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(q.library_path()):
        pytest.skip("libquartz.so not built")
    return q.load()


def test_attention_scales_out_of_fp32():
    """The scores' factor, scale k_scale log2(e), is one fp32 number, and v_scale over the sum of 2^30
    weights stays normal."""
    attend = lambda **kw: _attend(**LONG, **kw)                          # noqa: E731
    for ks, scale in ((3.3e38, 1.25), (3.3e38, 1.0), (2.0 ** 64, -2.0 ** 64), (2.0 ** -126, 0.1), (2.0 ** -100, 2.0 ** -30)):
        assert attend(ks=ks, scale=scale) == EUNSUP, (ks, scale)
    for ks, scale in ((3.3e38, 0.5), (2.0 ** -126, 1.0), (2.0 ** -126, 0.0), (2.0 ** 64, -2.0 ** 63), (3.3e38, 2.0 ** -140)):
        assert attend(ks=ks, scale=scale) == EWS, (ks, scale)
    assert attend(vs=2.0 ** -97) == attend(vs=2.0 ** -126) == EUNSUP
    assert attend(vs=2.0 ** -96) == attend(vs=3.3e38) == EWS
