"""Attention of draft trees over pages: mixes of long and short sequences."""
import numpy as np
import pytest

import paged_reference as R
import paper_2510_15312_b200 as pkg
from test_gpu_paged import i32
from test_gpu_tree_attention import Case

pytestmark = pytest.mark.gpu


def sms():
    import torch
    return torch.cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("at,hd", [(0, 64), (31, 128), (63, 64)])
def test_merge_of_one_long_sequence_among_many_short_ones(at, hd):
    """Units of many parts, which a block merges together, and units of few, which its warps merge alone, over several rounds of a block."""
    import torch
    rows, lengths, hq, hkv = [20] * 64, [512] * 64, 28, 4
    lengths[at] = 24000
    c = Case(rows, lengths, hq, hkv, hd, 32, "float16", tree=True, seed=at)
    g, chunk = hq // hkv, 128 // (hq // hkv)
    units = ((c.n * g + 3) // 4 + c.n // chunk + len(rows)) * hkv
    tiles = [-(-(a + b) // 64) * -(-a // chunk) * hkv for a, b in zip(rows, lengths)]
    share = sum(tiles) / (2 * sms())
    assert units > 8 * 3 * sms() and -(-(24000 + 20) // 64) / share > 13     # several rounds of eight units a block; an item of more than twelve parts
    got = c.run()
    c.check(got, only=[at, 1, 62])
    for _ in range(20):
        assert torch.equal(c.run(), got)
