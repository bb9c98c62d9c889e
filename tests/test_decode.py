"""mate_attn_decode against masked softmax attention in 64 bits, token by token, and against the rows of mate_attn_fwd."""
import numpy as np
import pytest
import torch

from tests.cache_model import TEXT, attention
from tests import helpers as hp
from workloads import tables

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def bounds(q, k, v, want, scale, dtype):
    """(O, LSE): how far fp32 arithmetic may be off.  q, k, v: what one head's new token and its keys are."""
    n, d = k.shape
    if n == 0:
        return 0.0, 0.0
    # a score: d products summed (each sum rounded, or cut off by the tensor cores: 2^-23), times the scale, times log2 e
    x = (d + 4) * 2.0 ** -23 * abs(scale) * (np.abs(k) @ np.abs(q)).max()
    s = scale * (k @ q)
    # its weight: the exponent's rounding (half an ulp of the distance to the maximum) and ex2's 2 ulp
    w = np.expm1(x) + 2.0 ** -22 + 2.0 ** -23 * min(s.max() - s.min(), 100.0)
    sums = (n + 40) * 2.0 ** -24   # sums over the keys, joined over warps and blocks, and one division
    top = np.abs(v).max()
    o = (2 * w + 2 * sums) * top
    if dtype == "bf16":            # weights as the sum of two bf16 (half a step of half a step), the result rounded to bf16
        o += 2.0 ** -16 * top + 2.0 ** -8 * np.abs(want[0])
    return o, w + sums + x + 2.0 ** -22 * (1 + abs(want[1]))


class Case:
    """Sequences with prefix, table, text and padding (whose keys and values are not numbers) in pages that lie in no order."""

    def __init__(self, m, lens, H, Hk, d, ps, views, dtype="bf16", slots_first=False, layers=1, seed=0, magnitude=1.0, pad=0.1, prefix=5, spare=3,
                 rows=4, cols=3):
        rng = self.rng = np.random.default_rng(seed)
        self.lens, self.H, self.Hk, self.d, self.ps, self.views, self.dtype = lens, H, Hk, d, ps, views, dtype
        need = [-(-n // ps) for n in lens]
        pages, width, S = sum(need) + spare, max(max(need), 1) + 1, len(lens)
        shape = (layers, pages, ps, Hk, d) if slots_first else (layers, pages, Hk, ps, d)
        g = torch.Generator().manual_seed(seed)
        k, v = ((torch.randn(shape, generator=g) * magnitude).to(DT[dtype]).cuda() for _ in range(2))
        if slots_first:
            k, v = k.transpose(2, 3), v.transpose(2, 3)
        order, table = rng.permutation(pages), np.full((S, width), -1, np.int32)
        ids, used = np.full((2, pages, ps), 3, np.int32), np.zeros((pages, ps), bool)
        self.ids, self.prefix = [], np.minimum(rng.integers(0, prefix + 1, S), lens).astype(np.int32)
        at = 0
        for s, n in enumerate(lens):
            table[s, :need[s]] = order[at:at + need[s]]
            at += need[s]
            t = np.stack([np.sort(rng.integers(0, rows, n)), rng.integers(0, cols, n)]).astype(np.int32)
            t[:, :self.prefix[s]] = 0
            t[:, n - n // 8:] = TEXT
            t[:, rng.random(n) < pad] = -1
            self.ids.append(t)
            for j in range(n):
                page, slot = table[s, j // ps], j % ps
                ids[:, page, slot], used[page, slot] = t[:, j], t[0, j] >= 0
        nan = torch.from_numpy(~used).cuda()          # padding and slots of nobody
        for x in (k, v):
            x.masked_fill_(nan[None, :, None, :, None], float("nan"))
            x[:, order[at:]] = float("inf")
        i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()  # noqa: E731
        self.c = m.Cache(k, v, i32(ids[0]), i32(ids[1]), i32(table), i32(lens), i32(self.prefix), i32(np.zeros(pages)), views)
        self.table = table

    def new_ids(self, seqs):
        """Text, cells of the sequence, a row and a column that it has not, padding."""
        out = np.zeros((2, len(seqs)), np.int32)
        for i, s in enumerate(seqs):
            kind = self.rng.integers(0, 8)
            own = np.flatnonzero((self.ids[s][0] >= 0) & (self.ids[s][0] != TEXT))
            if kind < 3:
                out[:, i] = TEXT
            elif kind < 6 and len(own):
                out[:, i] = self.ids[s][:, self.rng.choice(own)]
            elif kind == 6:
                out[:, i] = 1000
            else:
                out[:, i] = -1
        return out

    def rows_of(self, s, head, layer, upto):
        n = min(self.lens[s], upto)
        pages = torch.from_numpy(self.table[s, :-(-n // self.ps)].astype(np.int64)).cuda()
        return [x[layer, pages, head].reshape(-1, self.d)[:n].double().cpu().numpy() for x in (self.c.k, self.c.v)]

    def check(self, Q, seqs, q_ids, O, LSE, scale=None, layer=0, upto=1 << 30):
        scale = 1 / np.sqrt(self.d) if scale is None else scale
        Q, O, LSE = (t.double().cpu().numpy() for t in (Q, O, LSE))
        for i, s in enumerate(seqs):
            for h in range(self.H):
                k, v = self.rows_of(s, h // (self.H // self.Hk), layer, upto)
                ids = self.ids[s][:, :len(k)]
                keep = ids[0] >= 0
                k, v, ids, prefix = k[keep], v[keep], ids[:, keep], int((keep[:self.prefix[s]]).sum())
                want = attention(Q[i, h], k, v, ids[0], ids[1], q_ids[0, i], q_ids[1, i], prefix, self.views[h], scale)
                if want[1] == -np.inf:
                    assert not O[i, h].any() and LSE[i, h] == -np.inf, (i, h)
                    continue
                bo, bl = bounds(Q[i, h], k, v, want, scale, self.dtype)
                assert np.all(np.abs(O[i, h] - want[0]) <= bo), (i, s, h, np.abs(O[i, h] - want[0]).max(), np.max(bo))
                assert abs(LSE[i, h] - want[1]) <= bl, (i, s, h, LSE[i, h], want[1], bl)


def run(m, case, seqs=None, scale=None, seed=1, magnitude=1.0, layer=0, **kw):
    seqs = list(range(len(case.lens))) if seqs is None else seqs
    q_ids = case.new_ids(seqs)
    Q = (torch.randn(len(seqs), case.H, case.d, generator=torch.Generator().manual_seed(seed)) * magnitude).to(DT[case.dtype]).cuda()
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    O, LSE = m.mate_attn_decode(case.c, Q, i32(q_ids[0]), i32(q_ids[1]), seqs=i32(seqs), scale=scale, layer=layer, **kw)
    case.check(Q, seqs, q_ids, O, LSE, scale, layer, kw.get("max_len", 1 << 30))
    return Q, q_ids, O, LSE


LENS = [0, 1, 15, 16, 17, 31, 33, 64, 65, 127, 128, 129, 255, 300, 511, 700]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,views", [(2, 2, [0, 1]), (6, 2, [0, 0, 1, 1, 2, 0]), (8, 1, [0] * 4 + [1] * 4), (5, 5, [0, 0, 1, 1, 2]),
                                        (32, 2, [0] * 16 + [1] * 16), (17, 1, [0, 1, 2] * 5 + [1, 0])])
@pytest.mark.parametrize("d,ps", [(64, 16), (128, 16), (8, 7), (48, 1), (96, 64), (120, 3)])
def test_decode(dtype, H, Hk, views, d, ps):
    import paper_2109_04312_b200 as m
    case = Case(m, LENS, H, Hk, d, ps, views, dtype, slots_first=(d + H) % 3 == 0, seed=d + H)
    for seed in range(2):
        run(m, case, np.random.default_rng(seed).permutation(len(LENS)).tolist(), seed=seed)
    case.c.status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[5000], [20000, 3, 700], [2500] * 9, list(range(0, 900, 13)), [0] * 5, [4097, 0, 0, 1]])
@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 2, 128), (3, 1, 16)])
def test_lengths(dtype, lens, H, Hk, d):
    import paper_2109_04312_b200 as m
    case = Case(m, lens, H, Hk, d, 16, [h % 3 for h in range(H)], dtype, seed=len(lens), rows=40, cols=7, prefix=60)
    run(m, case)
    run(m, case, max_len=max(max(lens), 1), seed=5)
    case.c.status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_padding_and_nothing_but_padding(dtype):
    import paper_2109_04312_b200 as m
    run(m, Case(m, [64, 700, 33], 4, 2, 64, 16, [0, 0, 1, 1], dtype, pad=0.0))
    run(m, Case(m, [64, 700, 33], 4, 2, 64, 16, [0, 0, 1, 1], dtype, pad=1.0))
    run(m, Case(m, [64, 700, 33, 1], 4, 2, 64, 16, [0, 1, 0, 1], dtype, pad=0.97))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale,magnitude", [(-0.3, 1.0), (0.0, 1.0), (0.125, 12.0), (0.125, 1e-3), (1.0, 4.0)])
def test_scales_and_large_scores(dtype, scale, magnitude):
    import paper_2109_04312_b200 as m
    case = Case(m, [1, 130, 900, 0], 6, 3, 64, 16, [0, 0, 1, 1, 2, 2], dtype, magnitude=magnitude)
    run(m, case, scale=scale, magnitude=magnitude)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_minus_infinity(dtype):
    # keys whose score is -inf have weight 0; a token all of whose scores are -inf gives O = 0, LSE = -inf
    import paper_2109_04312_b200 as m
    case = Case(m, [40, 40], 1, 1, 64, 16, [0], dtype, pad=0.0)
    case.c.k[..., 0].nan_to_num_(0.0).abs_().add_(1.0)
    Q = torch.zeros(2, 1, 64, device="cuda", dtype=DT[dtype])
    Q[:, :, 0] = 1.0
    pages = torch.from_numpy(case.table[0, :3].astype(np.int64)).cuda()
    case.c.k[0, pages, :, :, 0] = float("-inf")                     # all keys of sequence 0
    one = int(case.table[1, 1])
    case.c.k[0, one, 0, 3, 0] = float("-inf")                       # one key of sequence 1, whose value is then nobody's
    case.c.v[0, one, 0, 3] = 1e30
    t = torch.full((2,), TEXT, dtype=torch.int32, device="cuda")
    O, LSE = m.mate_attn_decode(case.c, Q, t, t)
    assert not O[0].any() and LSE[0, 0] == -float("inf")
    assert torch.isfinite(O[1]).all() and O[1].abs().max() < 10 and torch.isfinite(LSE[1]).all()


def test_layers_views_outputs_streams():
    import paper_2109_04312_b200 as m
    case = Case(m, [100, 5, 260], 4, 2, 64, 16, [0, 1, 1, 0], layers=3)
    for layer in range(3):
        run(m, case, [2, 0, 1], layer=layer)
    Q, q_ids, O, LSE = run(m, case)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    row, col = i32(q_ids[0]), i32(q_ids[1])
    # queries as a view of a wider tensor; outputs given; every sequence in order without a list
    wide = torch.zeros(3, 6, 4, 72, device="cuda").bfloat16()
    wide[:, 2, :, 8:] = Q
    o, l = torch.full_like(Q, 7), torch.full((3, 4), 7.0, device="cuda")
    r = m.mate_attn_decode(case.c, wide[:, 2, :, 8:], row, col, out=o, lse=l)
    assert r[0] is o and r[1] is l and torch.equal(o, O) and torch.equal(l, LSE)
    # the same sequence three times; rows of an outer tensor behind the batch stay
    big = torch.full((5, 4, 64), 9.0, device="cuda").bfloat16()
    two = m.mate_attn_decode(case.c, Q[[2, 2, 2]].contiguous(), row[[2, 2, 2]].contiguous(), col[[2, 2, 2]].contiguous(), seqs=i32([2, 2, 2]), out=big[:3])[0]
    assert all(torch.equal(two[i], O[2]) for i in range(3)) and bool((big[3:] == 9).all())
    assert m.mate_attn_decode(case.c, Q[:0], row[:0], col[:0])[0].shape == (0, 4, 64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = m.mate_attn_decode(case.c, Q, row, col)
    side.synchronize()
    assert torch.equal(again[0], O) and torch.equal(again[1], LSE)
    # the same bits from launch to launch, with others between
    for _ in range(5):
        m.mate_attn_decode(case.c, Q * 3, row, col)
        again = m.mate_attn_decode(case.c, Q, row, col)
        assert torch.equal(again[0], O) and torch.equal(again[1], LSE)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_graphs_and_calls_on_two_streams(dtype):
    # two captured calls on one cache, replayed at the same time, and with other lengths than they were captured with
    import paper_2109_04312_b200 as m
    case = Case(m, [6000, 7000], 4, 2, 64, 16, [0, 0, 1, 1], dtype, rows=50)
    Q = torch.randn(2, 2, 4, 64, device="cuda").to(DT[dtype])
    t = torch.full((2,), TEXT, dtype=torch.int32, device="cuda")
    streams, graphs, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    m.mate_attn_decode(case.c, Q[0], t, t)
    torch.cuda.synchronize()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[i]):
            outs.append(m.mate_attn_decode(case.c, Q[i], t, t))
        graphs.append(g)
    for lens in ([6000, 7000], [0, 123], [5999, 1]):
        case.c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        want = [m.mate_attn_decode(case.c, Q[i], t, t) for i in range(2)]
        torch.cuda.synchronize()
        for _ in range(20):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i][0], want[i][0]) and torch.equal(outs[i][1], want[i][1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_beyond_32_bits(dtype):
    import paper_2109_04312_b200 as m
    d, ps = 64, 16
    pages = 2 ** 32 // (ps * d * DT[dtype].itemsize) + 9          # 4 GB each, a little more
    k, v = (torch.empty(1, pages, 1, ps, d, dtype=DT[dtype], device="cuda") for _ in range(2))
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    c = m.Cache(k, v, z(pages, ps), z(pages, ps), z(1, 4) - 1, z(1), z(1), z(pages) + 1, [0])
    c.refs[-3:] = 0
    f = m.mate_rope_freqs(d)
    assert m.mate_cache_extend(c, None, z(1) + 40).tolist() == [40]
    assert c.table[0, :3].tolist() == [pages - 3, pages - 2, pages - 1]
    K, V = (torch.randn(1, 1, 40, d, device="cuda").to(DT[dtype]) for _ in range(2))
    m.mate_cache_append(c, K, V, row_ids=z(1, 40), col_ids=z(1, 40), freqs=f)
    Q = torch.randn(1, 1, d, device="cuda").to(DT[dtype])
    O, LSE = m.mate_attn_decode(c, Q, z(1), z(1))
    Kr = m.mate_rope(K, torch.arange(40, dtype=torch.int32, device="cuda"), f)
    q, kk, vv = (x.double().cpu().numpy() for x in (Q[0, 0], Kr[0, 0], V[0, 0]))
    want = attention(q, kk, vv, np.zeros(40), np.zeros(40), 0, 0, 0, 0, d ** -0.5)
    bo, bl = bounds(q, kk, vv, want, d ** -0.5, dtype)
    assert np.all(np.abs(O[0, 0].double().cpu().numpy() - want[0]) <= bo) and abs(float(LSE[0, 0]) - want[1]) <= bl
    c.refs[0] = 0
    assert int(m.mate_cache_compact(c)) == pages - 1 and c.table[0, :3].tolist() == [pages - 3, pages - 2, 0]
    assert torch.equal(k[0, 0, 0, :8], Kr[0, 0, 32:])
    c.status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_entries(dtype):
    # more entries than a block has threads, the same sequences over and over, split and whole, with and without tokens
    import paper_2109_04312_b200 as m
    case = Case(m, [0, 3, 700, 129, 64, 0, 2000, 31], 3, 1, 64, 16, [0, 1, 2], dtype, rows=20)
    rng = np.random.default_rng(0)
    seqs = rng.integers(0, 8, 700).tolist()
    q_ids = case.new_ids(seqs)
    Q = torch.randn(700, 3, 64, device="cuda").to(DT[dtype])
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    for kw in (dict(), dict(max_len=2000)):
        O, LSE = m.mate_attn_decode(case.c, Q, i32(q_ids[0]), i32(q_ids[1]), seqs=i32(seqs), **kw)
        some = rng.permutation(700)[:60].tolist()
        case.check(Q[some], [seqs[i] for i in some], q_ids[:, some], O[some], LSE[some])
    case.c.status()


def test_in_place_and_twice_in_a_row():
    # the result over the queries; calls back to back, with nothing between that waits
    import paper_2109_04312_b200 as m
    case = Case(m, [900, 64, 0, 5000], 4, 2, 64, 16, [0, 1, 0, 1], rows=30)
    t = torch.full((4,), TEXT, dtype=torch.int32, device="cuda")
    Q = torch.randn(4, 4, 64, device="cuda").bfloat16()
    want = [Q]
    for _ in range(3):
        want.append(m.mate_attn_decode(case.c, want[-1], t, t)[0])
        torch.cuda.synchronize()
    q = Q.clone()
    for _ in range(3):
        assert m.mate_attn_decode(case.c, q, t, t, out=q)[0] is q
    assert torch.equal(q, want[3])


def test_what_is_out_of_range_is_left_out():
    import paper_2109_04312_b200 as m
    case = Case(m, [100, 64, 40], 4, 2, 64, 16, [0, 1, 0, 1], pad=0.0)
    Q, q_ids, O, LSE = run(m, case)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    row, col = i32(q_ids[0]), i32(q_ids[1])
    case.c.status()
    for seqs in ([0, -1, 2], [0, 3, 2], [0, 2 ** 31 - 1, 2]):
        o, l = m.mate_attn_decode(case.c, Q, row, col, seqs=i32(seqs))
        assert torch.equal(o[::2], O[::2]) and not o[1].any() and bool((l[1] == -float("inf")).all())
        with pytest.raises(m.MateError, match="invalid argument"):
            case.c.status()
    # the last page of a sequence is none: its tokens do not count
    keep = int(case.c.table[0, 6])
    for page in (-1, case.c.k.shape[1], 2 ** 31 - 1):
        case.c.table[0, 6] = page
        t = torch.full((3,), TEXT, dtype=torch.int32, device="cuda")
        o, l = m.mate_attn_decode(case.c, Q, t, t)
        with pytest.raises(m.MateError, match="invalid argument"):
            case.c.status()
        case.c.lens[0] = 96
        want = m.mate_attn_decode(case.c, Q, t, t)
        case.c.lens[0] = 100
        assert torch.equal(o[1:], want[0][1:]) and torch.allclose(l, want[1], rtol=1e-6) and torch.allclose(o.float(), want[0].float(), atol=2e-2)
    case.c.table[0, 6] = keep
    case.c.status()
    # lengths beyond what the row of the table holds, below 0, and beyond max_len
    case.c.lens[0] = 10 ** 6
    with pytest.raises(m.MateError, match="invalid argument"):
        m.mate_attn_decode(case.c, Q, row, col)
        case.c.status()
    case.c.lens[0] = -5
    o, l = m.mate_attn_decode(case.c, Q, row, col)
    assert not o[0].any() and torch.equal(o[1:], O[1:])
    with pytest.raises(m.MateError, match="invalid argument"):
        case.c.status()
    case.c.lens[0] = 100
    t = torch.full((3,), TEXT, dtype=torch.int32, device="cuda")
    o, l = m.mate_attn_decode(case.c, Q, t, t, max_len=64)
    case.check(Q, [0, 1, 2], np.full((2, 3), TEXT), o, l, upto=64)
    with pytest.raises(m.MateError, match="invalid argument"):
        case.c.status()


def test_refusals():
    import paper_2109_04312_b200 as m
    case = Case(m, [10], 4, 2, 64, 16, [0, 1, 0, 1])
    c, Q, i = case.c, torch.zeros(1, 4, 64, device="cuda").bfloat16(), torch.zeros(1, dtype=torch.int32, device="cuda")
    K = torch.zeros(1, 2, 1, 64, device="cuda").bfloat16()
    f = m.mate_rope_freqs(64)
    for what, call in (("Q", lambda: m.mate_attn_decode(c, Q.float(), i, i)), ("Q", lambda: m.mate_attn_decode(c, Q[:, :3], i, i)),
                       ("Q", lambda: m.mate_attn_decode(c, Q.cpu(), i, i)), ("row_ids", lambda: m.mate_attn_decode(c, Q, i.long(), i)),
                       ("col_ids", lambda: m.mate_attn_decode(c, Q, i, i[:0])), ("seqs", lambda: m.mate_attn_decode(c, Q, i, i, seqs=i.cpu())),
                       ("max_len", lambda: m.mate_attn_decode(c, Q, i, i, max_len=0)), ("max_len", lambda: m.mate_attn_decode(c, Q, i, i, max_len=-1)),
                       ("O", lambda: m.mate_attn_decode(c, Q, i, i, out=Q.float())), ("LSE", lambda: m.mate_attn_decode(c, Q, i, i, lse=Q)),
                       ("layer", lambda: m.mate_attn_decode(c, Q, i, i, layer=-1)), ("K and V", lambda: m.mate_cache_append(c, K.float(), K.float())),
                       ("K and V", lambda: m.mate_cache_append(c, K, K[:, :1])), ("row_ids", lambda: m.mate_cache_append(c, K, K, row_ids=i, col_ids=i)),
                       ("freqs", lambda: m.mate_cache_append(c, K, K, freqs=m.mate_rope_freqs(66))), ("counts", lambda: m.mate_cache_extend(c, None, i.float())),
                       ("seqs", lambda: m.mate_cache_extend(c, i.long(), i)), ("granted", lambda: m.mate_cache_extend(c, i, i, i[:0])),
                       ("children", lambda: m.mate_cache_fork(c, i, i[:0])), ("parents", lambda: m.mate_cache_fork(c, i.cpu(), i)),
                       ("seqs", lambda: m.mate_cache_free(c, i.long())), ("n_live", lambda: m.mate_cache_compact(c, i)),
                       ("Q", lambda: m.mate_cache_append(c, K, K, freqs=f, Q=K))):
        with pytest.raises(ValueError, match="^%s must be" % what):
            call()
    for call in (lambda: m.mate_attn_decode(c, Q, i, i, layer=1), lambda: m.mate_cache_append(c, K, K, layer=1),
                 lambda: m.mate_cache_append(c, K, K, Q=Q[:, :, None]), lambda: m.mate_cache_append(c, K, K, row_ids=i[None]),
                 lambda: m.mate_attn_decode(c, Q.expand(2, 4, 64).contiguous(), i.repeat(2), i.repeat(2))):
        with pytest.raises(m.MateError, match="invalid argument"):
            call()
    # more units of work than 32 bits count
    wide = m.Cache(case.c.k, case.c.v, case.c.row_ids, case.c.col_ids, torch.zeros(1, 1 << 26, dtype=torch.int32, device="cuda"), case.c.lens,
                   case.c.prefix, case.c.refs, [0, 1, 0, 1])
    n = 200
    with pytest.raises(m.MateError, match="unsupported"):
        m.mate_attn_decode(wide, Q.expand(n, 4, 64).contiguous(), i.repeat(n), i.repeat(n), seqs=i.repeat(n))
    odd = torch.zeros(2, 4, 65, device="cuda").bfloat16()[:1, :, 1:]
    with pytest.raises(m.MateError, match="aligned"):
        m.mate_attn_decode(c, odd, i, i)


@pytest.mark.parametrize("name", ["bert", "medium"])
def test_a_table_read_token_by_token(name):
    # the calls as they are used together: a table rotated, attended by the forward and put into the cache; then the rows of the
    # forward, one token at a time, from the cache -- prefix tokens as text, table tokens with their cell's ids
    import paper_2109_04312_b200 as m
    cfg, rows, cols, info, vals = hp.make_case(name)
    B, H, N, d = 2, cfg.H, info["N"], cfg.d
    rows, cols = rows[:B], cols[:B]
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()  # noqa: E731
    Q, K, V = (hp.to_dev(vals[n][:B], cfg.dtype) for n in ("Q", "K", "V"))
    pos, f = torch.arange(N, dtype=torch.int32, device="cuda").repeat(B, 1), m.mate_rope_freqs(d)
    q, k = m.mate_rope(Q, pos, f, K=K)
    view = tables.head_view(cfg)
    plan = m.mate_plan(i32(rows), i32(cols), cfg.P, view)
    O, LSE = m.mate_attn_fwd(plan, q, k, V)
    c = m.Cache.empty(2 * B * (N // 16) + 3, 16, H, d, 2 * B, N // 16 + 1, view)
    seqs = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    c.prefix[seqs.long()] = cfg.P
    granted = m.mate_cache_extend(c, seqs, torch.full((B,), N, dtype=torch.int32, device="cuda"))
    qa = m.mate_cache_append(c, K, V, seqs, granted, i32(rows), i32(cols), freqs=f, positions=pos, Q=Q)
    assert torch.equal(qa, q)
    m.mate_cache_fork(c, seqs, torch.tensor([0, 2], dtype=torch.int32, device="cuda"))
    m.mate_cache_free(c, seqs)
    m.mate_cache_compact(c)
    seqs = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(0)
    for t in [0, cfg.P - 1, cfg.P, N - 1] + rng.integers(0, N, 20).tolist():
        ids = [np.where(t < cfg.P, TEXT, x[:, t]) for x in (rows, cols)]
        o, l = m.mate_attn_decode(c, q[:, :, t], i32(ids[0]), i32(ids[1]), seqs=seqs)
        # both round weights and result to bf16 once: 4 x 2^-8 of values of at most 2.5; sums of fp32
        assert (o.float() - O[:, :, t].float()).abs().max() < 4 * 2.0 ** -8 * V.abs().max()
        a, b = l.cpu().numpy(), LSE[:, :, t].cpu().numpy()
        ok = np.isfinite(a)
        assert np.array_equal(ok, np.isfinite(b)) and np.all(np.abs(a[ok] - b[ok]) < 1e-4)
    # an answer behind it: rows of a dense forward over everything
    steps = 5
    new = [(torch.randn(B, H, steps, d, device="cuda") * 0.5).bfloat16() for _ in range(3)]
    text = torch.full((B, 1), TEXT, dtype=torch.int32, device="cuda")
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    keys, values = [k], [V]
    for j in range(steps):
        granted = m.mate_cache_extend(c, seqs, one)
        qn = m.mate_cache_append(c, new[1][:, :, j:j + 1], new[2][:, :, j:j + 1], seqs, granted, text, text, freqs=f, Q=new[0][:, :, j:j + 1])
        o, l = m.mate_attn_decode(c, qn[:, :, 0], text[:, 0].contiguous(), text[:, 0].contiguous(), seqs=seqs)
        at = torch.full((B, 1), N + j, dtype=torch.int32, device="cuda")
        keys.append(m.mate_rope(new[1][:, :, j:j + 1], at, f))
        values.append(new[2][:, :, j:j + 1])
        kk, vv = torch.cat(keys, 2).double(), torch.cat(values, 2).double()
        x = (qn.double() @ kk.transpose(2, 3))[:, :, 0] * d ** -0.5
        valid = torch.cat([i32(rows) >= 0, torch.ones(B, j + 1, dtype=torch.bool, device="cuda")], 1)
        x = x.masked_fill(~valid[:, None], -float("inf"))
        want = (torch.softmax(x, -1)[:, :, None] @ vv)[:, :, 0]
        assert (o.double() - want).abs().max() < 2 * 2.0 ** -8 * vv.abs().max()
        assert (l.double() - torch.logsumexp(x, -1)).abs().max() < 1e-4
    c.status()
    plan.status()


@pytest.mark.parametrize("H,d", [(1, 64), (1, 128), (16, 64), (16, 128)])
def test_weights_keep_their_fp32_bits(H, d):
    # Three keys with scores 0, -a and -a - 2^-12 and values 0, 1 and -1: O is the small difference of two weights, (w - w') / (1 + w + w'), which shows
    # what the weights lost on their way to the product with the values.  The scores are exact (a has 8 bits).  A weight: scale / ln 2 is
    # the same for both (it cancels to first order), its product with the score, below 2, is rounded once (2^-24 of 1, 2^-24 ln 2 of the weight),
    # ex2 is good to 2^-22.  What is summed after the leading parts have cancelled is below 2^-8 (each sum 2^-23 of that, six of them).  Sum, division: 2^-22
    # of the result; its rounding to bf16: 2^-8 of it.
    import paper_2109_04312_b200 as m
    a = torch.arange(64, 64 + 256, dtype=torch.float64) / 256       # 0.25 to 1.25
    a = a[a.bfloat16().double() == a]
    S, delta = len(a), 2.0 ** -12
    assert S > 100
    c = m.Cache.empty(S, 16, 1, d, S, 1, [0] * H)
    m.mate_cache_extend(c, None, torch.full((S,), 3, dtype=torch.int32, device="cuda"))
    K, V = (torch.zeros(S, 1, 3, d, dtype=torch.float64) for _ in range(2))
    K[:, 0, 1, 0], K[:, 0, 2, 0], K[:, 0, 2, 1] = -a, -a, -delta
    V[:, 0, 1], V[:, 0, 2] = 1.0, -1.0
    ids = torch.full((S, 3), TEXT, dtype=torch.int32, device="cuda")
    m.mate_cache_append(c, K.bfloat16().cuda(), V.bfloat16().cuda(), row_ids=ids, col_ids=ids)
    Q = torch.zeros(S, H, d, device="cuda").bfloat16()
    Q[..., :2] = 1.0
    O = m.mate_attn_decode(c, Q, ids[:, 0].contiguous(), ids[:, 0].contiguous(), scale=1.0)[0].double().cpu()
    w, w2 = torch.exp(-a), torch.exp(-a - delta)
    want = ((w - w2) / (1 + w + w2))[:, None, None]
    tol = 2 * (w / (1 + 2 * w2))[:, None, None] * (2.0 ** -22 + 2.0 ** -24) + 6 * 2.0 ** -31 + (2.0 ** -22 + 2.0 ** -8) * want
    assert bool(((O - want).abs() <= tol).all()), ((O - want).abs() / tol).max()
    c.status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,views", [(3, 1, [0, 1, 2]), (8, 1, [0, 1] * 4), (8, 2, [0, 2, 0, 2, 1, 1, 2, 1]), (17, 1, [0, 1, 2] * 5 + [1, 0])])
@pytest.mark.parametrize("d", [64, 48, 128])
def test_what_is_not_a_number_reaches_the_heads_that_attend_it(H, Hk, views, d, dtype):
    # tokens of the new token's row, of its column and of neither get keys and values that are not numbers, each kind in turn: the heads that do
    # not attend them give the same bits as with zeros there
    import paper_2109_04312_b200 as m
    for lens in ([40, 7, 300, 130], [3000, 700], [0, 513] * 40):
        case = Case(m, lens, H, Hk, d, 16, views, dtype, pad=0.0, rows=6, cols=5, seed=H + d)
        S = len(lens)
        q_ids = np.full((2, S), 2, np.int32)
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
        Q = torch.randn(S, H, d, device="cuda").to(DT[dtype])
        clean = [x.clone() for x in (case.c.k, case.c.v)]
        call = lambda: m.mate_attn_decode(case.c, Q, i32(q_ids[0]), i32(q_ids[1]))  # noqa: E731
        case.check(Q[:3], list(range(min(S, 3))), q_ids, *[x[:3] for x in call()])
        for kind in ("row", "col", "both", "neither"):
            slots, reached = [], np.zeros((S, H), bool)
            for s, n in enumerate(lens):
                row, col = case.ids[s]
                always = (np.arange(n) < case.prefix[s]) | (row == TEXT)
                own = {"row": (row == 2) & (col != 2), "col": (row != 2) & (col == 2), "both": (row == 2) & (col == 2),
                       "neither": (row != 2) & (col != 2)}[kind] & ~always
                slots += [(case.table[s, j // 16], j % 16) for j in np.flatnonzero(own)]
                sees = {"row": (0, 2), "col": (1, 2), "both": (0, 1, 2), "neither": ()}[kind]
                reached[s] = own.any() & np.isin(views, sees)
            at = torch.tensor(slots, device="cuda").T
            results = []
            for value in (0.0, float("nan"), float("inf"), -float("inf")):
                for x, y in zip((case.c.k, case.c.v), clean):
                    x.copy_(y)
                    if len(slots):
                        x[0, at[0], :, at[1]] = value
                results.append(call())
            stays = torch.from_numpy(~reached).cuda()
            for i, (O, LSE) in enumerate(results[1:]):
                assert torch.equal(O[stays], results[0][0][stays]) and torch.equal(LSE[stays], results[0][1][stays]), (kind, i)
                assert i or (O[~stays].isnan().all() and LSE[~stays].isnan().all())   # (a NaN; infinite keys may also have weight 0)
    case.c.status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[5000], [20000, 3, 700], [2500] * 9, [0, 1, 1025, 0, 3000]])
@pytest.mark.parametrize("H,Hk,d", [(16, 1, 128), (17, 1, 64), (40, 2, 96), (50, 1, 128), (20, 2, 8)])
def test_large_groups_shared_out_and_joined(dtype, lens, H, Hk, d):
    # more than eight heads to a block, several blocks to a group (the last one with fewer heads), items that fall to several blocks
    import paper_2109_04312_b200 as m
    case = Case(m, lens, H, Hk, d, 16, [h % 3 if H < 20 else int(h >= 7) for h in range(H)], dtype, seed=len(lens) + H, rows=40, cols=7, prefix=60)
    run(m, case)
    run(m, case, max_len=max(lens), seed=5)
    case.c.status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,d", [(16, 1, 128), (32, 2, 64), (19, 1, 40)])
def test_large_groups_a_block_to_each_item(dtype, H, Hk, d):
    # more items than SMs, none of them long: four warps, an item to a block
    import paper_2109_04312_b200 as m
    rng = np.random.default_rng(H)
    lens = rng.integers(0, 500, 160).tolist()
    case = Case(m, lens, H, Hk, d, 16, [h % 2 for h in range(H)], dtype, seed=H, rows=9, cols=4)
    seqs = rng.permutation(160).tolist()
    q_ids = case.new_ids(seqs)
    Q = torch.randn(160, H, d, device="cuda").to(DT[dtype])
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    O, LSE = m.mate_attn_decode(case.c, Q, i32(q_ids[0]), i32(q_ids[1]), seqs=i32(seqs), max_len=512)
    some = rng.permutation(160)[:25].tolist()
    case.check(Q[some], [seqs[i] for i in some], q_ids[:, some], O[some], LSE[some])
    case.c.status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[700, 3], [3000]])
def test_the_most_heads(dtype, lens):
    import paper_2109_04312_b200 as m
    case = Case(m, lens, 1024, 1, 8, 16, [(h // 5) % 3 for h in range(1024)], dtype, seed=7, rows=9, cols=5)
    run(m, case)
    case.c.status()
    more = m.Cache(case.c.k, case.c.v, case.c.row_ids, case.c.col_ids, case.c.table, case.c.lens, case.c.prefix, case.c.refs, [0] * 1025)
    i = torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(m.MateError, match="unsupported"):
        m.mate_attn_decode(more, torch.zeros(1, 1025, 8, device="cuda").to(DT[dtype]), i, i)
