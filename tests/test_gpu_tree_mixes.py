"""Attention of draft trees over pages: mixes of long and short sequences, of large and small probabilities."""
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


@pytest.mark.parametrize("gap", [12, 20, 25, 28])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_a_flat_tail_behind_one_dominant_key(dtype, hd, gap):
    """One key with nearly all of the mass and the value 0, thousands of keys with 2^-gap of its share each: the output is theirs alone.  300 sequences over the same pages, so that a
    block goes through most of a sequence."""
    import torch
    t, length, page, seqs = getattr(torch, dtype), 16383, 64, 300
    rng = np.random.default_rng(gap)
    k = torch.tensor(rng.standard_normal((256, 1, page, hd)) * 0.02, device="cuda").to(t)
    v = torch.tensor(rng.standard_normal((256, 1, page, hd)) + 1.0, device="cuda").to(t)
    q = torch.zeros(seqs, 2, hd, dtype=t, device="cuda")
    q[:, 0, 0], q[:, 1, 0] = 8.0, 8.25
    k[0, 0, 0] = 0.0
    k[0, 0, 0, 0] = gap * np.log(2.0) / (8.0 * hd ** -0.5)
    v[0, 0, 0] = 0.0
    table = i32(np.arange(256)[None].repeat(seqs, 0))
    got = pkg.tree_attention(q, k, v, table, i32([length] * seqs), i32(range(seqs + 1))).double().cpu().numpy()
    kk, vv = (x.transpose(0, 1).flatten(1, 2)[:, :length + 1].double().cpu().numpy() for x in (k, v))
    exp, mass, size = R.attention(q[:1].double().cpu().numpy(), kk, vv, np.ones((1, length + 1), bool), hd ** -0.5)
    # as in Case.check, but probabilities below fp16's normal range are half a step of 2^-24 off against a largest of at least 2^7
    u, half = torch.finfo(t).eps / 2, dtype == "float16"
    eps = 2 * hd * 2.0 ** -24 * size[..., None] + 2.0 ** -21
    low, tiny = (2.0 ** -32 * np.abs(vv[0]).sum(0).max(), 2.0 ** -25) if half else (0.0, 0.0)
    assert (np.abs(got - exp) <= u * np.abs(exp) + (1 + u) * (u + eps) * mass + tiny + low).all(), float(np.abs(got / exp - 1).max())
