"""mate_attn_decode_shared where the scores of a row leave what its weights were made by: upwards, downwards, in tiles of one team and the other, with masks, and
with values that are not numbers in front of and behind such a step."""
import numpy as np
import pytest
import torch

from tests.cache_model import TEXT
from tests.test_decode import DT
from tests.test_decode_shared import Shared, i32, together

STEPS = {  # score of the tokens, 128 at a time (to the base e)
    "up by little": [0, 4, 8, 12, 16, 20],
    "up by much": [0, 60, 120, 180, 240, 300],
    "down": [300, 200, 100, 0, -100, -200],
    "far below 0": [-500, -490, -480, -490, -480, -470],
    "one team higher": [0, 40, 0, 40, 0, 40],
    "one tile": [0, 0, 0, 90, 0, 0],
    "just within, then just beyond": [5.5, -5.5, 5.5, 5.6, 11.1, 11.2],
    "at the end": [0, 0, 0, 0, 0, 88],
}


def stepped(m, name, d, dtype, seed=30):
    case = Shared(m, [(40, [100, 3, 0, 128])], 4, 2, d, 16, [0, 0, 1, 1], dtype, seed=seed, pad=0.0, rows=6, cols=5, prefix=0)
    c, g = case.c, torch.Generator().manual_seed(seed)
    for s in range(len(case.lens)):
        for j in range(case.lens[s]):
            at = c.k[0, case.table[s, j // 16], :, j % 16]          # the first elements make the step, the others some noise
            at[:, :8] = STEPS[name][j // 128] / 8
            if s == 0 or j >= 640:
                at[:, 8:] = (torch.randn(2, d - 8, generator=g) * 0.5).to(at)
    Q = torch.randn(len(case.lens), 4, d, generator=g) * 0.3
    Q[..., :8] = 1
    return case, Q.to(DT[dtype]).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["text", "cells"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", STEPS)
def test_steps(name, d, kind, dtype):
    import paper_2109_04312_b200 as m
    case, Q = stepped(m, name, d, dtype)
    B = len(case.lens)
    q_ids = np.full((2, B), TEXT, np.int32) if kind == "text" else np.array([[1, 2, 3, TEXT], [4, 2, 0, TEXT]], np.int32)
    for scale in (1.0, -1.0, 0.25):
        O, LSE = together(m)(case.c, Q, i32(q_ids[0]), i32(q_ids[1]), i32(case.groups), scale=scale)
        case.check(Q, list(range(B)), q_ids, O, LSE, scale)
    case.c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["up by much", "one team higher", "one tile", "down"])
@pytest.mark.parametrize("d", [64, 128])
def test_values_that_are_not_numbers_beside_a_step(d, name):
    import paper_2109_04312_b200 as m
    case, Q = stepped(m, name, d, "bf16")
    c, B = case.c, len(case.lens)
    q_ids = np.array([[1, 2, 3, TEXT], [4, 2, 0, TEXT]], np.int32)
    args = (Q, i32(q_ids[0]), i32(q_ids[1]), i32(case.groups))
    clean = together(m)(c, *args, scale=1.0)
    case.check(Q, list(range(B)), q_ids, *clean, 1.0)
    for j in (5, 130, 300, 500, 639):
        t = c.v[0, int(case.table[0, j // 16]), 1, j % 16]
        before = t.clone()
        t[3] = float("nan")
        O, LSE = together(m)(c, *args, scale=1.0)
        t.copy_(before)
        row, col = case.ids[0][:, j]
        for i in range(B):
            for h in range(4):
                hit = h >= 2 and (q_ids[0, i] == TEXT or col == q_ids[1, i] or row == TEXT)
                assert torch.equal(LSE[i, h], clean[1][i, h])
                if hit:
                    assert O[i, h, 3].isnan(), (j, i, h)
                    assert O[i, h][torch.arange(d, device="cuda") != 3].isfinite().all()
                else:
                    assert torch.equal(O[i, h], clean[0][i, h]), (j, i, h)


@pytest.mark.gpu
@pytest.mark.parametrize("magnitude", [3.0, 10.0])
@pytest.mark.parametrize("H,Hk,d", [(6, 2, 64), (64, 2, 128), (12, 12, 40)])
def test_large_scores_everywhere(H, Hk, d, magnitude):
    # the base of most rows moves, in some tile of one team or the other, in shared tokens and own ones
    import paper_2109_04312_b200 as m
    case = Shared(m, [(50, [300, 0, 20]), (20, [5] * 30), (0, [700])], H, Hk, d, 16, [h % 3 for h in range(H)], "bf16", seed=31, magnitude=magnitude,
                  rows=20, cols=9)
    B = len(case.lens)
    q_ids = case.new_ids(list(range(B)))
    q_ids[:, ::2] = TEXT
    Q = (torch.randn(B, H, d, generator=torch.Generator().manual_seed(7)) * magnitude).bfloat16().cuda()
    O, LSE = together(m)(case.c, Q, i32(q_ids[0]), i32(q_ids[1]), i32(case.groups))
    some = list(range(0, B, 3 if H > 12 else 1))
    case.check(Q[some], some, q_ids[:, some], O[some], LSE[some])
    for _ in range(3):
        o, l = together(m)(case.c, Q, i32(q_ids[0]), i32(q_ids[1]), i32(case.groups))
        assert torch.equal(o, O) and torch.equal(l, LSE)
    case.c.status()
