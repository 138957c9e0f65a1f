"""The plan of attention for several new tokens a sequence, seen through its workspace (host only)."""
import os

import pytest

import paper_2509_26436_amd as q


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(q.library_path()):
        pytest.skip("libquartz.so not built")
    return q.load()


# tiles of all sequences as if they were alike: between half and all of what 256 compute units hold
@pytest.mark.parametrize("tokens,sequences,heads,kv,d,page,positions,rows", [
    (2080, 65, 16, 4, 128, 16, 131072, 128), (930, 65, 16, 2, 256, 16, 942288, 128), (256, 129, 2, 2, 64, 16, 955664, 32)])
def test_parts_of_full_devices_stay_few(tokens, sequences, heads, kv, d, page, positions, rows):
    """Where one part of every tile takes more than half of the device, four at most fill it better,
    however wide the table is: its width says nothing about the lengths."""
    size = q.quartz_paged_prompt_workspace_bytes(tokens, sequences, heads, kv, d, page, positions // page)
    tiles = tokens * (heads // kv) // rows + sequences
    part = tiles * kv * rows * (d + 2) * 4                  # a part's means, maximum and weight, in fp32
    assert size % part == 0 and size // part <= 4, size / part
