"""Bits of its weights that mate_attn_decode_shared keeps in the product with bf16 values: 16."""
import numpy as np
import pytest
import torch

from tests.cache_model import TEXT
from tests.test_decode_shared import i32


@pytest.mark.gpu
@pytest.mark.parametrize("behind", [0, 40, 100])
@pytest.mark.parametrize("kind", ["shared", "own"])
@pytest.mark.parametrize("H,d", [(1, 64), (16, 64), (5, 24), (1, 128), (16, 128), (5, 72)])
def test_weights_keep_their_bits(H, d, kind, behind):
    # Three keys with scores 0, -a and -a - 2^-12 and values 0, 1 and -1, behind others that are padding: O is the small difference of two weights, (w - w') /
    # (1 + w + w'), which shows what the weights lost on their way to the product with the values.  The scores are exact (a has 8 bits).  A weight: scale / ln 2
    # is the same for both (it cancels to first order), its product with the score, below 2, is rounded once (2^-24 of 1, 2^-24 ln 2 of the
    # weight), ex2 is good to 2^-22.  What is summed after the leading parts have cancelled is below 2^-8 (each sum 2^-23 of that, six of them).
    # Sum, division, joined with what attends nothing: 2^-22 of the result; its rounding to bf16: 2^-8 of it.  A weight is the sum of
    # two bf16, the second one of what the rounding of the first left, half a step, and rounded by half a step of that: 2^-8 2^-8 of it.
    import paper_2109_04312_b200 as m
    a = torch.arange(64, 64 + 256, dtype=torch.float64) / 256       # 0.25 to 1.25
    a = a[a.bfloat16().double() == a]
    S, n, delta = len(a), behind + 3, 2.0 ** -12
    assert S > 100
    c = m.Cache.empty(S * 7, 16, 1, d, S, 7, [0] * H)
    m.mate_cache_extend(c, None, torch.full((S,), n, dtype=torch.int32, device="cuda"))
    K, V = (torch.zeros(S, 1, n, d, dtype=torch.float64) for _ in range(2))
    K[:, 0, -2, 0], K[:, 0, -1, 0], K[:, 0, -1, 1] = -a, -a, -delta
    V[:, 0, -2], V[:, 0, -1] = 1.0, -1.0
    ids = torch.full((S, n), TEXT, dtype=torch.int32, device="cuda")
    # (every second one of those in front is padding, the others are attended with a weight of 0: all of them move the three to other places of a tile)
    ids[:, :behind:2] = -1
    K[:, 0, 1:behind:2, 0] = -1000.0
    m.mate_cache_append(c, K.bfloat16().cuda(), V.bfloat16().cuda(), row_ids=ids, col_ids=ids)
    B = 2 * S                                                       # every sequence twice
    Q = torch.zeros(B, H, d, device="cuda").bfloat16()
    Q[..., :2] = 1.0
    text, at = torch.full((B,), TEXT, dtype=torch.int32, device="cuda"), np.arange(B)
    groups = np.stack([at // 2 * 2, np.full(B, 2), np.full(B, n)]) if kind == "shared" else np.stack([at, np.ones(B), np.zeros(B)])
    O = m.mate_attn_decode_shared(c, Q, text, text, i32(groups), seqs=i32(at // 2), scale=1.0, always=True)[0].double().cpu()
    w, w2 = torch.exp(-a), torch.exp(-a - delta)
    want = ((w - w2) / (1 + w + w2)).repeat_interleave(2)[:, None, None]
    tol = (2 * w / (1 + 2 * w2)).repeat_interleave(2)[:, None, None] * (2.0 ** -22 + 2.0 ** -24 + 2.0 ** -16) + 6 * 2.0 ** -31 + (2.0 ** -22 + 2.0 ** -8) * want
    assert bool(((O - want).abs() <= tol).all()), ((O - want).abs() / tol).max()
    c.status()
