"""Draft distributions with entries that are no probabilities."""
import numpy as np
import pytest

import paper_2510_15312_b200 as pkg
from test_gpu_paged import check_verify, i32

pytestmark = pytest.mark.gpu


def test_negative_draft_values_count_as_zero():
    """A token without a share of the target's is never taken for it, and the rest is that of a draft with zeros there."""
    rng = np.random.default_rng(1)
    for vocab in (4, 700, 5000):
        for _ in range(30):
            p = rng.random((6, vocab)).astype(np.float32)
            p[:, rng.random(vocab) < 0.4] = 0.0
            q = (rng.random((6, vocab)) - 0.5).astype(np.float32) * 2.0
            p, q = p / p.sum(1, keepdims=True), q / np.abs(q).sum(1, keepdims=True)
            tokens, u, cu = rng.integers(0, vocab, 6).astype(np.int32), rng.random(6).astype(np.float32), np.array([0, 4, 6], np.int32)
            want = check_verify(p, tokens, cu, u, np.maximum(q, 0.0), None)
            import torch
            got = pkg.verify_sampled(torch.tensor(p, device="cuda"), i32(tokens), i32(cu), torch.tensor(u, device="cuda"), draft_probs=torch.tensor(q, device="cuda"))
            for g, w in zip(got[:3], want):
                np.testing.assert_array_equal(g.cpu().numpy(), w)


def test_a_token_without_a_share_is_rejected():
    p, q = np.array([[0.0, 0.5, 0.5]] * 2, np.float32), np.array([[0.0, 0.0, 0.0], [-0.25, 1.0, 0.25]], np.float32)
    import torch
    for u in (0.0, 0.3, 0.9):
        acc, words, _, _ = pkg.verify_sampled(torch.tensor(p, device="cuda"), i32([0, 0]), i32([0, 2]), torch.tensor([0.1, u], device="cuda"), draft_probs=torch.tensor(q, device="cuda"))
        assert acc.tolist() == [0] and words.tolist() == [2, -1]
