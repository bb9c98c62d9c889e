"""mate_attn_decode_shared where the scores of a row leave what its weights were made by: upwards, downwards, in every second tile, with masks, in long parts, and
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


def many_tables(d, L, tables=40, kv=8, heads=2, seed=0, step=0.0):
    """(cache, Q, groups): so many tables of L tokens, each with two questions, that a block has more than a kv head of one; every token is text.  step: how much
    the scores rise (or fall) every 512 tokens."""
    import paper_2109_04312_b200 as m
    ps, pages = 16, -(-L // 16)
    c = m.Cache.empty(tables * pages, ps, kv, d, 2 * tables, pages, [0] * (kv * heads))
    g = torch.Generator(device="cuda").manual_seed(seed)
    c.k[0].normal_(generator=g), c.v[0].normal_(generator=g)
    c.row_ids.fill_(TEXT), c.col_ids.fill_(TEXT), c.lens.fill_(L)
    c.table.copy_(torch.arange(tables * pages, device="cuda").view(tables, pages).repeat_interleave(2, 0))
    Q = torch.randn(2 * tables, kv * heads, d, device="cuda", generator=g)
    if step:
        at = torch.arange(pages, device="cuda").repeat(tables) * ps // 512
        c.k[0, :, :, :, 0] = (at * step)[:, None, None].to(c.k)
        Q[..., 0] = 8.0
    i = np.arange(2 * tables)
    return c, Q.bfloat16(), i32(np.stack([i // 2 * 2, np.full(2 * tables, 2), np.full(2 * tables, L // 16 * 16)])), pages


def exact(c, Q, L, pages, kv, heads, entry, scale):
    out = []
    for h in range(kv):
        k, v = (t[0, entry // 2 * pages:(entry // 2 + 1) * pages, h].reshape(-1, t.shape[-1])[:L].double() for t in (c.k, c.v))
        s = scale * (Q[entry, h * heads:(h + 1) * heads].double() @ k.T)
        out.append((torch.softmax(s, -1) @ v, torch.logsumexp(s, -1), s.max(-1).values - s.min(-1).values))
    return (torch.cat(x) for x in zip(*out))


@pytest.mark.gpu
@pytest.mark.parametrize("step", [0.0, 0.7, 3.0, -2.0])
@pytest.mark.parametrize("d,L", [(64, 700), (64, 5000), (128, 2100), (128, 6007), (40, 4100), (96, 3333)])
def test_long_parts(d, L, step):
    # a block takes tens of tiles of the same rows, and the base moves far behind the first one
    c, Q, groups, pages = many_tables(d, L, step=step)
    import paper_2109_04312_b200 as m
    text, scale = i32([TEXT] * len(Q)), d ** -0.5
    O, LSE = together(m)(c, Q, text, text, groups)
    for entry in (0, 1, 37, 78):
        want, lse, spread = exact(c, Q, L, pages, 8, 2, entry, scale)
        # weights: the exponent's rounding (2^-24 of the spread of the scores to the base 2) and ex2 (2^-22); scores: d products, 2^-23 of what they sum up (below
        # 40 times the scale each); sums: 16 products of up to 24 tiles of each team, cut off (2^-23), then a few hundred rounded; all of it on values of up to
        # 6; the two parts of a weight, 2^-16; and the result in bf16
        w = 2.0 ** -16 + 2.0 ** -22 + 2.0 ** -24 * 1.5 * (spread + 8) + (d + 4) * 2.0 ** -23 * scale * 40 * d ** 0.5
        o = 6 * (2 * w + 900 * 2.0 ** -23)[:, None] + 2.0 ** -8 * want.abs()
        assert bool(((O[entry].double() - want).abs() <= o).all()), ((O[entry].double() - want).abs() / o).max()
        assert bool(((LSE[entry].double() - lse).abs() <= 2 * w + 900 * 2.0 ** -23 + 2.0 ** -22 * lse.abs()).all())
    o, l = together(m)(c, Q, text, text, groups)
    assert torch.equal(o, O) and torch.equal(l, LSE)
    # a value that is not a number reaches the two entries of its table, wherever it lies
    for j in (3, L // 2, L - 17):
        page = c.v[0, 5 * pages + j // 16, 2, j % 16]
        before = page.clone()
        page[1] = float("nan")
        o, l = together(m)(c, Q, text, text, groups)
        page.copy_(before)
        hit = torch.zeros_like(O, dtype=torch.bool)
        hit[10:12, 4:6, 1] = True
        assert bool(o[hit].isnan().all()) and torch.equal(o[~hit], O[~hit]) and torch.equal(l, LSE)
    c.status()


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
