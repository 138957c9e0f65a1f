"""The largest calls of the operators of prompts and drafted tokens are refused by their sizes, on the host
and before anything is launched."""
import os

import pytest

import paper_2509_26436_amd as q

ESHAPE = 2
A = 4096      # a fake, 16-byte aligned address: never dereferenced on these paths


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(q.library_path()):
        pytest.skip("libquartz.so not built")
    return q.load()


# sequences, heads, channels, e4m3: 2 x heads x channels x bytes / 256 blocks of 256 threads a sequence
@pytest.mark.parametrize("sequences,heads,d,fp8", [(65536, 127, 256, False), (65536, 128, 256, True), (1 << 22, 2, 128, False),
                                                   ((1 << 23) - 1, 1, 256, False)])
def test_kept_tokens_of_more_threads_than_a_grid_holds(sequences, heads, d, fp8):
    size = d * (1 if fp8 else 2)
    assert sequences * -(-2 * heads * size // 256) * 256 >= 1 << 32
    assert q.quartz_paged_keep(A, A, sequences, 4, 4, A, A, int(fp8), heads, d, 4, 16, 16 * heads * d, A, 4, 4, None) == ESHAPE
