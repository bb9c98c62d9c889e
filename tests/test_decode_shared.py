"""mate_attn_decode_shared against masked softmax attention in 64 bits, sequence after sequence, and against mate_attn_decode."""
import ctypes
import functools

import numpy as np
import pytest
import torch

from tests.cache_model import TEXT, attention
from tests.test_cache_pages import struct
from tests.test_decode import DT, Case


def bounds(q, k, v, want, scale, dtype):
    """(O, LSE): how far fp32 arithmetic may be off.  q, k, v: what one head's new token and its keys are."""
    n, d = k.shape
    # a score: d products summed (each sum rounded, or cut off by the tensor cores: 2^-23), times the scale, times log2 e
    x = (d + 4) * 2.0 ** -23 * abs(scale) * (np.abs(k) @ np.abs(q)).max()
    s = scale * (k @ q)
    # its weight: the exponent's rounding (half an ulp of the distance to the base, which may lie 8 powers of two below the maximum) and ex2's 2 ulp
    w = np.expm1(x) + 2.0 ** -22 + 2.0 ** -23 * min(s.max() - s.min() + 8, 100.0)
    sums = (n + 400) * 2.0 ** -23  # sums over the keys (cut off by the tensor cores), joined over up to 300 parts, and one division
    top = np.abs(v).max()
    o = (2 * w + 2 * sums) * top
    if dtype == "bf16":            # weights as the sum of two bf16 (half a step of half a step, 2^-16), the result rounded to bf16
        o += 2.0 ** -16 * top + 2.0 ** -8 * np.abs(want[0])
    return o, w + sums + x + 2.0 ** -22 * (1 + abs(want[1]))


class Shared(Case):
    """Groups of sequences: (shared pages, the own tokens of each).  The members go through the first one's pages; each has a prefix of its
    own length, within which ids do not matter."""

    def __init__(self, m, groups, H, Hk, d, ps, views, dtype="bf16", **kw):
        lens = [f * ps + n for f, own in groups for n in own]
        super().__init__(m, lens, H, Hk, d, ps, views, dtype, **kw)
        table, self.groups, at = self.table, np.zeros((3, len(lens)), np.int32), 0
        for f, own in groups:
            for i in range(len(own)):
                table[at + i, :f] = table[at, :f]
                self.ids[at + i][:, :f * ps] = self.ids[at][:, :f * ps]
                self.groups[:, at + i] = (at, len(own), f * ps) if f and len(own) > 1 else (at + i, 1, 0)
            at += len(own)
        self.c.table.copy_(torch.from_numpy(table))

    def check(self, Q, seqs, q_ids, O, LSE, scale=None, layer=0, upto=1 << 30):
        scale = 1 / np.sqrt(self.d) if scale is None else scale
        Q, O, LSE = (t.double().cpu().numpy() for t in (Q, O, LSE))
        prefix = self.c.prefix.tolist()
        for i, s in enumerate(seqs):
            for h in range(self.H):
                k, v = self.rows_of(s, h // (self.H // self.Hk), layer, upto)
                ids = self.ids[s][:, :len(k)]
                keep = ids[0] >= 0
                k, v, ids, P = k[keep], v[keep], ids[:, keep], int(keep[:prefix[s]].sum())
                want = attention(Q[i, h], k, v, ids[0], ids[1], q_ids[0, i], q_ids[1, i], P, self.views[h], scale)
                if want[1] == -np.inf:
                    assert not O[i, h].any() and LSE[i, h] == -np.inf, (i, h)
                    continue
                bo, bl = bounds(Q[i, h], k, v, want, scale, self.dtype)
                assert np.all(np.abs(O[i, h] - want[0]) <= bo), (i, s, h, np.abs(O[i, h] - want[0]).max(), np.max(bo))
                assert abs(LSE[i, h] - want[1]) <= bl, (i, s, h, LSE[i, h], want[1], bl)


def together(m):
    """What shared tokens are read once by, however small the batch."""
    return functools.partial(m.mate_attn_decode_shared, always=True)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def run(m, case, seqs=None, groups=None, scale=None, seed=1, magnitude=1.0, layer=0, q_ids=None, **kw):
    seqs = list(range(len(case.lens))) if seqs is None else seqs
    groups = case.groups if groups is None else groups
    q_ids = case.new_ids(seqs) if q_ids is None else q_ids
    Q = (torch.randn(len(seqs), case.H, case.d, generator=torch.Generator().manual_seed(seed)) * magnitude).to(DT[case.dtype]).cuda()
    O, LSE = together(m)(case.c, Q, i32(q_ids[0]), i32(q_ids[1]), i32(groups), seqs=i32(seqs), scale=scale, layer=layer, **kw)
    case.check(Q, seqs, q_ids, O, LSE, scale, layer, kw.get("max_len", 1 << 30))
    return Q, q_ids, O, LSE


GROUPS = [(3, [5, 0, 17, 1]), (0, [9, 0]), (10, [200, 3, 40]), (1, [0]), (2, [1] * 9), (30, [0, 0, 0, 2, 7, 60])]
HEADS = [(2, 2, [0, 1]), (6, 2, [0, 0, 1, 1, 2, 0]), (8, 1, [0] * 4 + [1] * 4), (5, 5, [0, 0, 1, 1, 2]), (32, 2, [0] * 16 + [1] * 16),
         (17, 1, [0, 1, 2] * 5 + [1, 0])]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,views", HEADS)
@pytest.mark.parametrize("d,ps", [(64, 16), (128, 16), (8, 7), (48, 1), (96, 64), (120, 3)])
def test_shared(dtype, H, Hk, views, d, ps):
    import paper_2109_04312_b200 as m
    case = Shared(m, GROUPS, H, Hk, d, ps, views, dtype, slots_first=(d + H) % 3 == 0, seed=d + H)
    run(m, case)
    groups = m.mate_cache_groups(case.c)
    run(m, case, groups=groups.cpu().numpy(), seed=2)
    # nobody shares; the list in another order, with the groups that this leaves
    B = len(case.lens)
    run(m, case, groups=np.stack([np.arange(B), np.ones(B), np.zeros(B)]), seed=3)
    seqs = np.random.default_rng(0).permutation(B).tolist() + [0, 0, 1]
    run(m, case, seqs, m.mate_cache_groups(case.c, i32(seqs)).cpu().numpy(), seed=4)
    case.c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("groups", [[(300, [10, 20])], [(40, [3] * 70)], [(1, [0] * 300)], [(7, [i]) for i in range(40)], [(5, [300, 0, 40])] * 12,
                                    [(600, [700, 0, 0])], [(8, [0] * 3), (0, [0, 0]), (0, [1000])]])
@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 2, 128), (3, 1, 16)])
def test_lengths(dtype, groups, H, Hk, d):
    import paper_2109_04312_b200 as m
    case = Shared(m, groups, H, Hk, d, 16, [h % 3 for h in range(H)], dtype, seed=len(groups), rows=40, cols=7, prefix=60)
    run(m, case)
    run(m, case, max_len=max(max(case.lens), 1), seed=5)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["text", "cells", "padding", "strangers"])
@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 2, 128)])
def test_one_kind_of_token(dtype, kind, H, Hk, d):
    import paper_2109_04312_b200 as m
    case = Shared(m, [(20, [3, 9, 0, 30]), (50, [1] * 40)], H, Hk, d, 16, [0] * (H // 2) + [1] * (H // 2), dtype, seed=3, rows=30, cols=9, prefix=70)
    B = len(case.lens)
    q_ids = {"text": np.full((2, B), TEXT), "padding": np.full((2, B), -1), "strangers": np.full((2, B), 1000),
             "cells": np.stack([np.arange(B) % 30, np.arange(B) % 9])}[kind].astype(np.int32)
    case.c.prefix.mul_(torch.arange(B, device="cuda", dtype=torch.int32) % 3)    # of every length, none among them
    run(m, case, q_ids=q_ids)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale,magnitude", [(0.0, 1.0), (-0.3, 1.0), (1.0, 1.0), (0.125, 30.0), (-2.0, 4.0), (1e-30, 1.0)])
def test_scales_and_large_scores(dtype, scale, magnitude):
    import paper_2109_04312_b200 as m
    case = Shared(m, [(20, [3, 300, 0]), (0, [40, 2])], 4, 2, 64, 16, [0, 1, 2, 0], dtype, seed=5, magnitude=magnitude)
    run(m, case, scale=scale, magnitude=magnitude)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_that_grow_along_the_tokens(dtype):
    # the running maximum moves with every tile, in the shared part and in the own ones
    import paper_2109_04312_b200 as m
    case = Shared(m, [(60, [100, 3, 0, 700])], 4, 2, 64, 16, [0, 0, 1, 1], dtype, seed=6, pad=0.0)
    c, B = case.c, 4
    Q = torch.ones(B, 4, 64, device="cuda").to(DT[dtype])
    for s in range(B):
        for j in range(case.lens[s]):
            c.k[0, case.table[s, j // 16], :, j % 16] = 0.001 * j * 8 if (j // 128) % 2 == 0 else -1.0
    ids = np.full((2, B), TEXT, np.int32)
    O, LSE = together(m)(c, Q, i32(ids[0]), i32(ids[1]), i32(case.groups))
    case.check(Q, list(range(B)), ids, O, LSE)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_what_is_not_a_number_reaches_the_heads_that_attend_it(dtype, d):
    import paper_2109_04312_b200 as m
    case = Shared(m, [(20, [30, 9, 140])], 6, 2, d, 16, [0, 0, 1, 1, 2, 0], dtype, seed=8, rows=12, cols=5, pad=0.0, prefix=0)
    c, B = case.c, 3
    q_ids = np.array([[1, 2, TEXT], [1, 2, TEXT]], np.int32)
    Q = torch.randn(B, 6, d, device="cuda").to(DT[dtype])
    args = (Q, i32(q_ids[0]), i32(q_ids[1]), i32(case.groups))
    clean = together(m)(c, *args)
    for what, x in (("k", float("nan")), ("v", float("nan")), ("v", float("inf")), ("v", float("-inf"))):
        for s, j in ((0, 17), (0, 200), (1, 322), (2, 330), (2, 459)):
            page, slot, shared = int(case.table[s, j // 16]), j % 16, j < 320
            t = getattr(c, what)[0, page, 1, slot]
            before = t.clone()
            t[3] = x
            got = together(m)(c, *args)
            t.copy_(before)
            row, col = case.ids[s][:, j]
            for i in range(B):
                for h in range(6):
                    mine = (shared or i == s) and h >= 3
                    hit = mine and (q_ids[0, i] == TEXT or row == TEXT or case.views[h] != 1 and row == q_ids[0, i] or case.views[h] != 0 and col == q_ids[1, i])
                    where = (what, s, j, i, h)
                    if not hit:
                        # (the bits may differ by the order of nothing: tiles and shares are the same)
                        assert torch.equal(got[0][i, h], clean[0][i, h]) and torch.equal(got[1][i, h], clean[1][i, h]), where
                    elif what == "k":
                        assert got[0][i, h].isnan().all() and got[1][i, h].isnan(), where
                    else:
                        assert not got[0][i, h, 3].isfinite() and torch.equal(got[1][i, h], clean[1][i, h]), where
                        others = torch.arange(d, device="cuda") != 3
                        assert got[0][i, h][others].isfinite().all(), where


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layers_views_outputs_streams(dtype):
    import paper_2109_04312_b200 as m
    case = Shared(m, [(9, [30, 9, 140]), (0, [7])], 6, 2, 64, 16, [0, 0, 1, 1, 2, 0], dtype, seed=9, layers=3)
    run(m, case, layer=2)
    B = len(case.lens)
    q_ids = case.new_ids(list(range(B)))
    wide = torch.randn(B, 9, 64, device="cuda").to(DT[dtype])
    Q = wide[:, 2:8]
    args = (i32(q_ids[0]), i32(q_ids[1]), i32(case.groups))
    want = together(m)(case.c, Q, *args, layer=1)
    out, lse = torch.empty(B, 6, 64, device="cuda", dtype=DT[dtype]), torch.empty(B, 6, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r = together(m)(case.c, Q, *args, layer=1, out=out, lse=lse)
    side.synchronize()
    assert r[0] is out and r[1] is lse and torch.equal(out, want[0]) and torch.equal(lse, want[1])
    q = Q.contiguous()
    assert torch.equal(together(m)(case.c, q, *args, layer=1, out=q)[0], want[0])
    e = together(m)(case.c, Q[:0], args[0][:0], args[1][:0], args[2][:, :0].contiguous())
    assert e[0].shape == (0, 6, 64) and e[1].shape == (0, 6)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_graphs_and_calls_on_two_streams(dtype):
    import paper_2109_04312_b200 as m
    case = Shared(m, [(40, [30, 9, 140, 0] * 4), (3, [7, 90])], 6, 2, 64, 16, [0, 0, 1, 1, 2, 0], dtype, seed=10, layers=2)
    B = len(case.lens)
    q_ids = case.new_ids(list(range(B)))
    Q = torch.randn(B, 6, 64, device="cuda").to(DT[dtype])
    args = (i32(q_ids[0]), i32(q_ids[1]), i32(case.groups))
    want = [together(m)(case.c, Q, *args, layer=i) for i in range(2)]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[i]):
            outs.append(together(m)(case.c, Q, *args, layer=i))
        graphs.append(g)
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i][0], want[i][0]) and torch.equal(outs[i][1], want[i][1])
    for _ in range(5):  # the same bits on every launch
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                outs[i] = together(m)(case.c, Q, *args, layer=i)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i][0], want[i][0]) and torch.equal(outs[i][1], want[i][1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_groups_that_do_not_fit_together(dtype):
    # nothing is read or written out of place, status says so, and an entry that is left alone has its own result
    import paper_2109_04312_b200 as m
    case = Shared(m, [(9, [30, 9, 140]), (4, [7, 1])], 4, 2, 64, 16, [0, 0, 1, 1], dtype, seed=11)
    B = len(case.lens)
    q_ids = np.full((2, B), TEXT, np.int32)
    Q = torch.randn(B, 4, 64, device="cuda").to(DT[dtype])
    ids = (i32(q_ids[0]), i32(q_ids[1]))
    good = case.groups.copy()
    big = 2 ** 31 - 1
    for at, x, alone in (((0, 1), -5, [1]), ((0, 1), 2, [1]), ((0, 0), 1, [0, 1, 2]), ((1, 0), big, [0, 1, 2]), ((1, 3), 3, [3, 4]), ((2, 1), big, [1]),
                         ((2, 2), -1, [2]), ((2, 0), 16, [0, 1, 2]), ((1, 4), 0, [4]), ((0, 4), big, [4]), ((1, 2), -big, [2])):
        groups = good.copy()
        groups[at] = x
        O, LSE = together(m)(case.c, Q, *ids, i32(groups))
        case.check(Q[alone], alone, q_ids[:, alone], O[alone], LSE[alone])
        assert not O.isnan().any()
        if at != (1, 4) and at != (1, 2):          # (one alone is no error)
            with pytest.raises(m.MateError, match="invalid"):
                case.c.status()
        case.c.status()
    # more shared tokens than a sequence has, than there are pages for, a sequence that there is not, pages that there are not
    groups = good.copy()
    groups[2, :3] = 9 * 16 + 20
    O, LSE = together(m)(case.c, Q, *ids, i32(groups))
    case.check(Q[3:], [3, 4], q_ids[:, 3:], O[3:], LSE[3:])
    with pytest.raises(m.MateError, match="invalid"):
        case.c.status()
    seqs = i32([0, 1, 77, 3, -4])
    O, LSE = together(m)(case.c, Q, *ids, i32(good), seqs=seqs)
    case.check(Q[:2], [0, 1], q_ids[:, :2], O[:2], LSE[:2])
    assert not O[2].any() and not O[4].any() and (LSE[2] == -np.inf).all()
    with pytest.raises(m.MateError, match="invalid"):
        case.c.status()
    before = case.c.table.clone()
    case.c.table[0, 3], case.c.table[3, 1] = 10 ** 6, -1
    together(m)(case.c, Q, *ids, i32(good))
    with pytest.raises(m.MateError, match="invalid"):
        case.c.status()
    case.c.table.copy_(before)
    case.c.lens[2] = -5
    O, LSE = together(m)(case.c, Q, *ids, i32(good))
    case.check(Q[3:], [3, 4], q_ids[:, 3:], O[3:], LSE[3:])
    case.c.lens[2] = 10 ** 9
    together(m)(case.c, Q, *ids, i32(good))
    with pytest.raises(m.MateError, match="invalid"):
        case.c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk", [(1024, 1), (1024, 1024), (300, 2)])
def test_many_heads(dtype, H, Hk):
    # more heads of a group than a tile has rows, in groups whose tiles begin inside a sequence's heads
    import paper_2109_04312_b200 as m
    case = Shared(m, [(4, [3, 0, 20]), (2, [40])], H, Hk, 16, 8, [h % 3 for h in range(H)], dtype, seed=12)
    run(m, case)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_entries(dtype):
    import paper_2109_04312_b200 as m
    n = 4096
    case = Shared(m, [(3, [5, 0, 17, 1]), (2, [1, 2])], 4, 2, 16, 4, [0, 1, 2, 0], dtype, seed=13)
    seqs = ([0, 1, 2, 3] * (n // 8) + [4, 5] * (n // 4))
    sizes = [4] * (n // 8) + [2] * (n // 4)
    first = np.repeat(np.cumsum([0] + sizes[:-1]), sizes)
    groups = np.stack([first, np.repeat(sizes, sizes), np.repeat([12 if s == 4 else 8 for s in sizes], sizes)])
    q_ids = case.new_ids(seqs)
    Q = torch.randn(len(seqs), 4, 16, device="cuda").to(DT[dtype])
    O, LSE = together(m)(case.c, Q, i32(q_ids[0]), i32(q_ids[1]), i32(groups), seqs=i32(seqs))
    some = np.random.default_rng(0).permutation(len(seqs))[:300]
    case.check(Q[some.tolist()], [seqs[i] for i in some], q_ids[:, some], O[some.tolist()], LSE[some.tolist()])
    more = i32([0] * (n + 1))
    with pytest.raises(m.MateError, match="unsupported|not available"):
        together(m)(case.c, Q[:1].expand(n + 1, 4, 16).contiguous(), more, more, torch.zeros(3, n + 1, dtype=torch.int32, device="cuda"), seqs=more)


LAYOUTS = {  # of keys and values in memory that they share with one another, or with what is nobody's: [layers, pages, heads, slots, d]
    "keys and values slot by slot": lambda x, L, P, H, ps, d: [x(L, P, ps, 2, H, d)[:, :, :, i].transpose(2, 3) for i in range(2)],
    "keys and values of a head": lambda x, L, P, H, ps, d: [x(L, P, ps, H, 2, d)[..., i, :].transpose(2, 3) for i in range(2)],
    "keys and values page by page": lambda x, L, P, H, ps, d: [x(L, P, 2, H, ps, d)[:, :, i] for i in range(2)],
    "slots with room behind": lambda x, L, P, H, ps, d: [x(L, P, H, ps, d + 8)[..., :d] for i in range(2)],
    "pages with room behind": lambda x, L, P, H, ps, d: [x(L, P, H * ps * d + 24)[..., 16:-8].unflatten(2, (H, ps, d)) for i in range(2)],
}


@pytest.mark.gpu
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d,ps,dtype", [(64, 16, "bf16"), (128, 48, "bf16"), (128, 24, "bf16"), (96, 32, "bf16"), (40, 16, "bf16"), (64, 16, "f32")])
def test_layouts(layout, d, ps, dtype):
    # what lies between the rows is not a number
    import paper_2109_04312_b200 as m
    case = Shared(m, [(10, [200, 3, 150, 70]), (0, [300, 40])], 6, 2, d, ps, [0, 0, 1, 1, 2, 0], dtype, seed=14, layers=2, pad=0.02)
    c = case.c
    k, v = LAYOUTS[layout](lambda *shape: torch.full(shape, float("nan"), dtype=DT[dtype], device="cuda"), *c.k.shape)
    k.copy_(c.k), v.copy_(c.v)
    case.c = m.Cache(k, v, c.row_ids, c.col_ids, c.table, c.lens, c.prefix, c.refs, case.views)
    run(m, case, layer=1)
    case.c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_of_many_slots(dtype):
    import paper_2109_04312_b200 as m
    case = Shared(m, [(0, [70000]), (1, [5, 0])], 2, 1, 16, 1 << 16, [0, 2], dtype, seed=15, spare=0, rows=500, cols=40)
    run(m, case)
    case.c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_group(dtype):
    # one sequence as often as a list may have it, and rows of many entries in a tile
    import paper_2109_04312_b200 as m
    n = 4096
    case = Shared(m, [(3, [2, 9])], 2, 2, 16, 8, [0, 1], dtype, seed=16)
    seqs = [int(i % 7 == 3) for i in range(n)]
    groups = np.repeat([[0], [n], [24]], n, 1)
    assert (m.mate_cache_groups(case.c, i32(seqs)).cpu().numpy() == groups).all()
    q_ids = case.new_ids(seqs)
    Q = torch.randn(n, 2, 16, device="cuda").to(DT[dtype])
    O, LSE = together(m)(case.c, Q, i32(q_ids[0]), i32(q_ids[1]), i32(groups), seqs=i32(seqs))
    some = np.random.default_rng(1).permutation(n)[:300]
    case.check(Q[some.tolist()], [seqs[i] for i in some], q_ids[:, some], O[some.tolist()], LSE[some.tolist()])
    case.c.status()


@pytest.mark.gpu
def test_the_same_bits_from_call_to_call_and_from_cold_memory():
    # (a wait that runs out, or rows that are read before they are there, would show)
    import paper_2109_04312_b200 as m
    for groups, H, Hk, d, ps in (([(4, [3, 0, 20]), (2, [40])], 1024, 1, 16, 8), ([(60, [300, 9, 0])] * 20, 6, 2, 64, 16), ([(40, [90] * 60)], 8, 2, 128, 16)):
        case = Shared(m, groups, H, Hk, d, ps, [h % 3 for h in range(H)], seed=17, prefix=30)
        Q, q_ids, O, LSE = run(m, case)
        args, junk = (i32(q_ids[0]), i32(q_ids[1]), i32(case.groups)), torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
        for i in range(60):
            if i % 3 == 0:
                junk.fill_(i)
            o, l = together(m)(case.c, Q, *args)
            assert torch.equal(o, O) and torch.equal(l, LSE), i
        case.c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,d", [(6, 2, 64), (12, 12, 128)])
def test_small_batches_are_read_one_by_one(dtype, H, Hk, d):
    # the results of the call for one sequence after another, to the bit, and status tells what it tells where they are read together
    import paper_2109_04312_b200 as m
    case = Shared(m, [(9, [30, 9, 140]), (4, [7, 1]), (0, [300])], H, Hk, d, 16, [h % 3 for h in range(H)], dtype, seed=18)
    f, B = m.mate_attn_decode_shared, len(case.lens)
    seqs = [3, 4, 0, 1, 2, 5, 5]
    groups = m.mate_cache_groups(case.c, i32(seqs))
    q_ids = case.new_ids(seqs)
    Q = torch.randn(len(seqs), H, d, device="cuda").to(DT[dtype])
    a, b = i32(q_ids[0]), i32(q_ids[1])
    want = m.mate_attn_decode(case.c, Q, a, b, seqs=i32(seqs), max_len=200)
    got = f(case.c, Q, a, b, groups, seqs=i32(seqs), max_len=200)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(m.MateError, match="invalid"):      # (5 and 5 share more tokens than max_len)
        case.c.status()
    want, got = m.mate_attn_decode(case.c, Q, a, b, seqs=i32(seqs)), f(case.c, Q, a, b, groups, seqs=i32(seqs))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    case.c.status()
    good, big = case.groups.copy(), 2 ** 31 - 1
    for at, x in (((0, 1), -5), ((0, 1), 2), ((0, 0), 1), ((1, 0), big), ((1, 3), 3), ((2, 1), big), ((2, 2), -1), ((2, 0), 16), ((0, 4), big), ((2, 5), -7)):
        groups = good.copy()
        groups[at] = x
        for always in (False, True):
            f(case.c, Q[:B], a[:B], b[:B], i32(groups), always=always)
            with pytest.raises(m.MateError, match="invalid"):
                case.c.status()
        f(case.c, Q[:B], a[:B], b[:B], i32(good))
        case.c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_size_from_which_sequences_are_read_together(dtype):
    # by max_len: what a batch may read; at the limit itself one by one.  (The sums differ in their order, so some bits do.)
    import paper_2109_04312_b200 as m
    B, H, d = 32, 8, 128
    n = (1 << 30 if dtype == "f32" else 192 << 20) // (B * H * d * 2 * (4 if dtype == "f32" else 2))
    case = Shared(m, [(20, [3] * B)], H, H, d, 16, [0] * H, dtype, seed=19, prefix=300)
    c = case.c
    wide = torch.full((B, n // 16 + 2), -1, dtype=torch.int32, device="cuda")
    wide[:, :c.table.shape[1]] = c.table
    c = m.Cache(c.k, c.v, c.row_ids, c.col_ids, wide, c.lens, c.prefix, c.refs, case.views)
    Q = torch.randn(B, H, d, device="cuda").to(DT[dtype])
    text, g = torch.full((B,), TEXT, dtype=torch.int32, device="cuda"), i32(case.groups)
    alone, shared = m.mate_attn_decode(c, Q, text, text), together(m)(c, Q, text, text, g)
    assert not torch.equal(alone[1], shared[1])
    for max_len, want in ((n, alone), (n + 1, shared), (None, shared)):
        got = m.mate_attn_decode_shared(c, Q, text, text, g, max_len=max_len)
        assert torch.equal(got[1], want[1]) or max_len == n and torch.allclose(got[1], want[1], atol=2e-5)
        assert max_len == n or torch.equal(got[0], want[0])
        assert torch.equal(got[1], shared[1]) == (max_len != n)


@pytest.mark.gpu
def test_a_wait_that_ran_out_is_reported_once():
    import paper_2109_04312_b200 as m
    case = Shared(m, [(1, [1])], 1, 1, 16, 16, [0])
    case.c.status_word.fill_(4)
    with pytest.raises(m.MateError) as e:
        case.c.status()
    assert e.value.status == -5
    case.c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_beyond_32_bits(dtype):
    # pages at the far end of a cache of more than 4 GB
    import paper_2109_04312_b200 as m
    ps, Hk, d = 64, 8, 128
    pages = (5 << 30) // (ps * Hk * d * (2 if dtype == "bf16" else 4)) + 40
    c = m.Cache.empty(pages, ps, Hk, d, 3, 8, [0, 1] * 8, dtype=DT[dtype])
    far = list(range(pages - 20, pages))
    c.k[0, far] = torch.randn(20, Hk, ps, d, device="cuda").to(DT[dtype])
    c.v[0, far] = torch.randn(20, Hk, ps, d, device="cuda").to(DT[dtype])
    c.row_ids.fill_(TEXT), c.col_ids.fill_(TEXT)
    c.table[0, :6], c.table[1, :6], c.table[2, :6] = i32(far[:6]), i32(far[:4] + far[7:9]), i32(far[:4] + far[10:12])
    c.lens.copy_(i32([5 * ps + 3, 6 * ps, 4 * ps + 1]))
    Q, text = torch.randn(3, 16, d, device="cuda").to(DT[dtype]), i32([TEXT] * 3)
    groups = m.mate_cache_groups(c)
    assert groups.tolist() == [[0] * 3, [3] * 3, [4 * ps] * 3]
    O, LSE = together(m)(c, Q, text, text, groups)
    for i in range(3):
        pg, n = c.table[i, :6].long(), int(c.lens[i])
        k, v = (t[0, pg].transpose(0, 1).reshape(Hk, -1, d)[:, :n].double().cpu().numpy() for t in (c.k, c.v))
        for h in range(16):
            q = Q[i, h].double().cpu().numpy()
            z = np.zeros(n, np.int64)
            want = attention(q, k[h // 2], v[h // 2], z, z, TEXT, TEXT, 0, 0, 1 / np.sqrt(d))
            bo, bl = bounds(q, k[h // 2], v[h // 2], want, 1 / np.sqrt(d), dtype)
            assert np.all(np.abs(O[i, h].double().cpu().numpy() - want[0]) <= bo) and abs(LSE[i, h].item() - want[1]) <= bl


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_questions_about_one_table(dtype):
    """A table is cached, forked for its questions, and these are read and answered token by token: everything together, in a graph."""
    import paper_2109_04312_b200 as m
    H, Hk, d, ps, n, steps, A = 6, 2, 64, 16, 5, 20, 3
    f, axes = m.mate_rope_freqs(d), [i % A for i in range(d // 2)]
    c = m.Cache.empty(60, ps, Hk, d, n + 1, 10, [0, 0, 0, 1, 1, 1], dtype=DT[dtype], layers=2)
    g = torch.Generator(device="cuda").manual_seed(0)
    L = 70
    K, V = (torch.randn(1, Hk, L, d, device="cuda", generator=g).to(DT[dtype]) for _ in range(2))
    ids = torch.stack([torch.arange(L) // 7, torch.arange(L) % 7]).int().cuda()[:, None]
    pos = torch.stack([torch.arange(L), torch.arange(L) // 7, torch.arange(L) % 7]).int().cuda()[:, None].contiguous()
    m.mate_cache_extend(c, i32([n]), i32([L]))
    for layer in range(2):
        m.mate_cache_append_axes(c, K, V, f, pos, axes, seqs=i32([n]), row_ids=ids[0] if layer == 0 else None, col_ids=ids[1] if layer == 0 else None,
                                 layer=layer)
    m.mate_cache_fork(c, i32([n] * n), i32(range(n)))
    seqs, ones, text = i32(range(n)), i32([1] * n), i32([TEXT] * n)
    q, k, v = (torch.randn(n, h, 1, d, device="cuda", generator=g).to(DT[dtype]) for h in (H, Hk, Hk))
    where = i32([[[L], [L], [L], [L], [L]]] * A)
    groups = torch.zeros(3, n, dtype=torch.int32, device="cuda")
    outs = []

    def step():
        granted = m.mate_cache_extend(c, seqs, ones)
        m.mate_cache_groups(c, seqs, out=groups)
        outs.clear()
        for layer in range(2):
            turned = m.mate_cache_append_axes(c, k, v, f, where, axes, seqs=seqs, counts=granted, row_ids=text[:, None] if layer == 0 else None,
                                              col_ids=text[:, None] if layer == 0 else None, layer=layer, Q=q)
            outs.append((turned, together(m)(c, turned[:, :, 0], text, text, groups, seqs=seqs, layer=layer)))
        where.add_(1)

    step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for t in range(steps):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        graph.replay()
        assert groups.tolist() == [[0] * n, [n] * n, [64] * n]
        for layer, (turned, (O, LSE)) in enumerate(outs):
            o, l = m.mate_attn_decode(c, turned[:, :, 0], text, text, seqs=seqs, layer=layer)
            # (two results of the same sum in fp32, some hundred roundings each, and one rounding to the type: a step of the result)
            assert torch.allclose(O.float(), o.float(), atol=2e-4 if dtype == "bf16" else 2e-5, rtol=2 ** -7 if dtype == "bf16" else 2e-5)
            assert torch.allclose(LSE, l, atol=2e-5, rtol=1e-6)
    assert c.lens.tolist() == [L + steps + 1] * n + [L]
    c.status()


@pytest.mark.gpu
def test_refusals():
    import paper_2109_04312_b200 as m
    case = Shared(m, [(2, [10, 3])], 4, 2, 64, 16, [0, 1, 0, 1])
    c, Q, i, g = case.c, torch.zeros(2, 4, 64, device="cuda").bfloat16(), torch.zeros(2, dtype=torch.int32, device="cuda"), i32(case.groups)
    f = m.mate_attn_decode_shared
    for what, call in (("Q", lambda: f(c, Q.float(), i, i, g)), ("Q", lambda: f(c, Q[:, :3], i, i, g)), ("Q", lambda: f(c, Q.cpu(), i, i, g)),
                       ("row_ids", lambda: f(c, Q, i.long(), i, g)), ("col_ids", lambda: f(c, Q, i, i[:0], g)), ("groups", lambda: f(c, Q, i, i, g[:, :1])),
                       ("groups", lambda: f(c, Q, i, i, g[:2])), ("groups", lambda: f(c, Q, i, i, g.T.contiguous().T)), ("groups", lambda: f(c, Q, i, i, g.cpu())),
                       ("groups", lambda: f(c, Q, i, i, g.float())), ("seqs", lambda: f(c, Q, i, i, g, seqs=i.cpu())), ("max_len", lambda: f(c, Q, i, i, g, max_len=0)),
                       ("O", lambda: f(c, Q, i, i, g, out=Q.float())), ("LSE", lambda: f(c, Q, i, i, g, lse=Q)), ("layer", lambda: f(c, Q, i, i, g, layer=-1))):
        with pytest.raises(ValueError, match="^%s must be" % what):
            call()
    for call in (lambda: f(c, Q, i, i, g, layer=1), lambda: f(c, Q, i, i, g, scale=float("nan")),
                 lambda: f(c, Q.repeat(2, 1, 1), i.repeat(2), i.repeat(2), g.repeat(1, 2))):
        with pytest.raises(m.MateError, match="invalid argument"):
            call()
    with pytest.raises(m.MateError, match="aligned"):
        f(c, torch.zeros(4, 4, 65, device="cuda").bfloat16()[:2, :, 1:], i, i, g)


def test_the_c_entries_refuse_before_anything_is_launched():
    from paper_2109_04312_b200 import build
    lib = ctypes.CDLL(build.build())
    P, L, size = ctypes.c_void_p, ctypes.c_int64 * 3, ctypes.c_size_t()
    s, at = struct()
    z = L(0, 64, 64)

    def call(r=None, layer=0, q=at, qs=z, B=1, seqs=at, row=at, col=at, groups=at, scale=1.0, max_len=0, flags=0, o=at, l=at):
        p = lambda x: P(x) if x else None  # noqa: E731
        return lib.mate_attn_decode_shared(ctypes.byref(s) if r is None else r, layer, p(q), qs, B, p(seqs), p(row), p(col), p(groups), ctypes.c_float(scale),
                                           max_len, flags, p(o), p(l), P(at), ctypes.c_size_t(1 << 40), None)

    for kw in (dict(layer=1), dict(layer=-1), dict(q=0), dict(qs=None), dict(B=-1), dict(seqs=0, B=3), dict(row=0), dict(col=0), dict(groups=0), dict(max_len=-1),
               dict(o=0), dict(l=0), dict(flags=2), dict(flags=1 << 31), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert call(**kw) == -1, kw
    for kw in (dict(q=at + 2), dict(o=at + 8), dict(qs=L(4, 64, 0)), dict(qs=L(64, 4, 0))):
        assert call(**kw) == -3, kw
    assert call(scale=3e38) == -2
    for kw, want in ((dict(k=None), -1), (dict(heads=0), -1), (dict(d=4), -2), (dict(dtype=7), -2), (dict(page_stride=4), -3)):
        s2, _ = struct(**kw)
        assert call(r=ctypes.byref(s2)) == want, kw
        assert lib.mate_cache_shared_workspace_bytes(ctypes.byref(s2), 1, ctypes.byref(size)) == want, kw
    assert lib.mate_cache_shared_workspace_bytes(ctypes.byref(s), -1, ctypes.byref(size)) == -1
    assert lib.mate_cache_shared_workspace_bytes(ctypes.byref(s), 1, None) == -1
    assert lib.mate_cache_shared_workspace_bytes(ctypes.byref(s), 0, ctypes.byref(size)) == 0 and size.value == 0
