"""Pages of a cache (mate_cache_extend / append / fork / free / compact) against a restatement in plain Python: whole numbers and
copies, so everything is compared bit for bit."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from tests.cache_model import TEXT, CacheModel, turn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def make(m, pages=40, page_size=4, kv_heads=2, d=16, seqs=6, width=8, heads=4, layers=2, dtype=torch.bfloat16, slots_first=False):
    if slots_first:
        k, v = (torch.zeros(layers, pages, page_size, kv_heads, d, dtype=dtype, device="cuda").transpose(2, 3) for _ in range(2))
    else:
        k, v = (torch.zeros(layers, pages, kv_heads, page_size, d, dtype=dtype, device="cuda") for _ in range(2))
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    c = m.Cache(k, v, z(pages, page_size), z(pages, page_size), z(seqs, width) - 1, z(seqs), z(seqs), z(pages), [0, 1] * (heads // 2))
    return c, CacheModel(pages, page_size, seqs, width)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def value_of(marks, layers, kv_heads, d):
    """What stands in a slot with these marks: a number per layer, head and element, exact in bf16; zero for mark 0."""
    marks = np.asarray(marks)[..., None, None, None]
    x = (marks * 7 + np.arange(layers)[:, None, None] * 31 + np.arange(kv_heads)[:, None] * 11 + np.arange(d)) % 251 + 1
    return np.where(marks == 0, 0, x)  # [..., layers, kv_heads, d]


def same(c, model, where):
    for name in ("table", "lens", "prefix", "refs"):
        assert np.array_equal(getattr(c, name).cpu().numpy(), getattr(model, name)), (where, name)
    L, P, H, S, d = c.k.shape
    want = value_of(model.slots, L, H, d).transpose(2, 0, 3, 1, 4)  # [P, S, L, H, d] -> [L, P, H, S, d]
    assert np.array_equal(c.k.float().cpu().numpy(), want), where
    assert np.array_equal(c.v.float().cpu().numpy(), np.where(want == 0, 0, 252 - want)), where
    assert np.array_equal(c.row_ids.cpu().numpy(), model.slots % 1000) and np.array_equal(c.col_ids.cpu().numpy(), model.slots % 77), where


def append(m, c, model, seqs, counts, next_mark, ids=True):
    N = max(max(counts, default=0), 1)
    marks = np.zeros((len(seqs), N), np.int64)
    for i, n in enumerate(counts):
        marks[i, :n] = np.arange(next_mark, next_mark + n)
        next_mark += n
    L, _, H, _, d = c.k.shape
    for layer in range(L):
        x = value_of(marks, L, H, d)[:, :, layer].transpose(0, 2, 1, 3)  # [B, H, N, d]
        K = torch.from_numpy(np.ascontiguousarray(x).astype(np.float32)).cuda().to(c.k.dtype)
        V = torch.from_numpy(np.ascontiguousarray(252 - x).astype(np.float32)).cuda().to(c.k.dtype)
        ids = (ints(marks % 1000), ints(marks % 77)) if layer == 0 else (None, None)
        assert m.mate_cache_append(c, K, V, ints(seqs), ints(counts), *ids, layer=layer) is None
    model.append(seqs, counts, marks)
    return next_mark


@pytest.mark.gpu
@pytest.mark.parametrize("kw", [dict(), dict(slots_first=True, page_size=3, d=8, kv_heads=1), dict(dtype=torch.float32, page_size=1, width=20),
                                dict(page_size=5, kv_heads=3, heads=6, d=40, seqs=9, pages=23, width=5, layers=1),
                                dict(page_size=16, d=128, kv_heads=4, seqs=12, pages=260, width=40, slots_first=True, layers=3)])
@pytest.mark.parametrize("seed", range(3))
def test_a_history_of_calls(kw, seed):
    import paper_2109_04312_b200 as m
    c, model = make(m, **kw)
    rng, mark = np.random.default_rng(seed), 1
    S, most = len(model.lens), model.width * model.ps
    for step in range(40):
        what = rng.choice(["grow", "grow", "one", "fork", "free", "compact", "prefix"])
        if what in ("grow", "one"):
            seqs = rng.permutation(S)[:rng.integers(1, S + 1)].tolist()
            counts = [1] * len(seqs) if what == "one" else rng.integers(0, most // 2 + 2, len(seqs)).tolist()
            granted = m.mate_cache_extend(c, ints(seqs), ints(counts))
            assert granted.tolist() == model.extend(seqs, counts), step
            mark = append(m, c, model, seqs, granted.tolist(), mark)
        elif what == "fork":
            n = int(rng.integers(1, S + 1))
            parents, children = rng.integers(0, S, n).tolist(), rng.permutation(S)[:n].tolist()
            m.mate_cache_fork(c, ints(parents), ints(children))
            model.fork(parents, children)
        elif what == "free":
            seqs = rng.integers(0, S, rng.integers(1, S)).tolist()
            m.mate_cache_free(c, ints(seqs))
            model.free(seqs)
        elif what == "compact":
            assert int(m.mate_cache_compact(c)) == model.compact()
        else:
            s = int(rng.integers(S))
            model.prefix[s] = step
            c.prefix[s] = step
        same(c, model, (step, what))
        # shared pages are not appended to in part: a sequence's last, unfilled page is its own
        for s in range(S):
            if model.lens[s] % model.ps:
                assert model.refs[model.table[s, model.lens[s] // model.ps]] == 1


@pytest.mark.gpu
def test_the_same_index_twice_and_indexes_out_of_range():
    import paper_2109_04312_b200 as m
    c, model = make(m, width=8)
    with_status = lambda: pytest.raises(m.MateError, match="invalid argument")  # noqa: E731
    for seqs, counts in (([1, 2, 1, 1], [5, 6, 7, 8]), ([-1, 3, 6, 100], [4, 4, 4, 4]), ([4], [-3])):
        assert m.mate_cache_extend(c, ints(seqs), ints(counts)).tolist() == model.extend(seqs, counts)
        same(c, model, seqs)
        with with_status():
            c.status()
        c.status()  # said once
    for parents, children in (([1, 2, 3], [5, 5, 5]), ([1, -1, 6], [-1, 0, 0]), ([3], [2])):
        m.mate_cache_fork(c, ints(parents), ints(children))
        model.fork(parents, children)
        same(c, model, children)
        with with_status():
            c.status()
    m.mate_cache_free(c, ints([1, 1, 5, 1]))
    model.free([1])
    model.free([5])
    same(c, model, "free")
    c.status()
    m.mate_cache_free(c, ints([-1, 6, 3]))
    model.free([3])
    same(c, model, "free")
    with with_status():
        c.status()
    m.mate_cache_free(c)
    model.free(range(6))
    same(c, model, "all")
    assert not c.refs.any() and bool((c.table == -1).all())


@pytest.mark.gpu
def test_no_room():
    import paper_2109_04312_b200 as m
    c, model = make(m, pages=7, width=4)
    # the first needs 3 pages, the second 4, the third one more than there is: it and the fifth get nothing, the fourth needs none
    seqs, counts = [0, 1, 2, 4, 3], [12, 13, 1, 0, 5]
    assert m.mate_cache_extend(c, ints(seqs), ints(counts)).tolist() == [12, 13, 0, 0, 0] == model.extend(seqs, counts)
    same(c, model, "extend")
    with pytest.raises(m.MateError, match="out of memory"):
        c.status()
    # 3 more fit into a page that is there; 4 do not; more than a row of the table holds never do
    assert m.mate_cache_extend(c, ints([1]), ints([3])).tolist() == [3] == model.extend([1], [3])
    c.status()
    assert m.mate_cache_extend(c, ints([0]), ints([1])).tolist() == [0] == model.extend([0], [1])
    assert m.mate_cache_extend(c, ints([1]), ints([1])).tolist() == [0] == model.extend([1], [1])
    with pytest.raises(m.MateError, match="out of memory"):
        c.status()
    m.mate_cache_free(c, ints([0]))
    model.free([0])
    assert m.mate_cache_extend(c, ints([0]), ints([9])).tolist() == [9] == model.extend([0], [9])
    # copies of a last page: none is free
    m.mate_cache_fork(c, ints([0, 1]), ints([2, 3]))
    model.fork([0, 1], [2, 3])
    same(c, model, "fork")
    assert c.lens.tolist() == [9, 16, 0, 16, 0, 0]
    with pytest.raises(m.MateError, match="out of memory"):
        c.status()


@pytest.mark.gpu
def test_contents_that_make_no_sense_are_left_out():
    # a table, lengths and counts full of numbers out of range: nothing outside of the arrays is touched (guard values around
    # them stay), and the status says so
    import paper_2109_04312_b200 as m
    rng = np.random.default_rng(1)
    pages, ps, H, d, S, W = 16, 4, 2, 16, 5, 6

    def guarded(*shape, dtype=torch.int32):
        n = int(np.prod(shape))
        flat = torch.full((n + 512,), 77, dtype=dtype, device="cuda")
        return flat, flat[256:256 + n].view(shape)

    for trial in range(6):
        arrays = {n: guarded(*s, dtype=t) for n, s, t in (("k", (1, pages, H, ps, d), torch.bfloat16), ("v", (1, pages, H, ps, d), torch.bfloat16),
                  ("row", (pages, ps), torch.int32), ("col", (pages, ps), torch.int32), ("table", (S, W), torch.int32), ("lens", (S,), torch.int32),
                  ("prefix", (S,), torch.int32), ("refs", (pages,), torch.int32))}
        c = m.Cache(*(arrays[n][1] for n in arrays), [0, 1])
        wild = np.array([-2 ** 31, -1, 0, 1, 3, 15, 16, 17, 23, 24, 25, 2 ** 31 - 1])
        for n in ("table", "lens", "prefix", "refs", "row", "col"):
            a = arrays[n][1]
            a.copy_(torch.from_numpy(rng.choice(wild, tuple(a.shape)).astype(np.int32)))
        lists = [ints(rng.choice(wild, 7).astype(np.int32)) for _ in range(3)]
        x = torch.zeros(7, H, 5, d, dtype=torch.bfloat16, device="cuda")
        m.mate_cache_append(c, x, x, lists[0], lists[1], freqs=m.mate_rope_freqs(d))
        m.mate_attn_decode(c, x[:, :, 0], lists[1], lists[2], seqs=lists[0])
        m.mate_cache_fork(c, lists[0], lists[1])
        m.mate_cache_extend(c, lists[1], lists[2])
        m.mate_cache_compact(c)
        m.mate_cache_free(c, lists[2])
        with pytest.raises(m.MateError):
            c.status()
        for n, (flat, _) in arrays.items():
            assert bool((flat[:256] == 77).all()) and bool((flat[-256:] == 77).all()), n


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 16), (24, 20), (128, 128), (40, 24), (80, 40)])
def test_append_rotates(d, rot, interleaved, dtype):
    import paper_2109_04312_b200 as m
    T = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    B, N, H, Hk, ps = 3, 7, 6, 2, 4
    c = m.Cache.empty(30, ps, Hk, d, 5, 6, [0, 1] * 3, dtype=T)
    seqs, counts = ints([4, 0, 2]), ints([7, 0, 3])
    m.mate_cache_extend(c, ints([2]), ints([6]))
    m.mate_cache_extend(c, seqs, counts)
    qkv = torch.randn(B, N, H + 2 * Hk, d, device="cuda").to(T)
    Q, K, V = (t.transpose(1, 2) for t in qkv.split([H, Hk, Hk], 2))
    f, pos = m.mate_rope_freqs(rot), torch.randint(0, 5000, (B, N), dtype=torch.int32, device="cuda")
    for given in (pos, None):
        q = m.mate_cache_append(c, K, V, seqs, counts, freqs=f, positions=given, interleaved=interleaved, mscale=1.1, Q=Q)
        lens, table = c.lens.tolist(), c.table.tolist()
        if given is not None:   # the same arithmetic as mate_rope's, bit for bit
            want_q, want_k = m.mate_rope(Q, pos, f, K=K, interleaved=interleaved, mscale=1.1)
            assert torch.equal(q, want_q)
        else:
            own = torch.tensor([[lens[s] - n + j for j in range(N)] for s, n in zip(seqs.tolist(), counts.tolist())], dtype=torch.int32, device="cuda")
            want_k = m.mate_rope(K, own, f, interleaved=interleaved, mscale=1.1)
        for i, (s, n) in enumerate(zip(seqs.tolist(), counts.tolist())):
            for j in range(n):
                at = lens[s] - n + j
                page, slot = table[s][at // ps], at % ps
                assert torch.equal(c.k[0, page, :, slot], want_k[i, :, j]) and torch.equal(c.v[0, page, :, slot], V[i, :, j])
    c.status()
    assert not c.row_ids.any()


@pytest.mark.gpu
def test_one_tensor_as_keys_and_values():
    import paper_2109_04312_b200 as m
    c = m.Cache.empty(9, 4, 2, 16, 3, 3, [0, 1])
    n = ints([5, 0, 9])
    m.mate_cache_extend(c, None, n)
    x = torch.randn(3, 2, 9, 16, device="cuda").bfloat16()
    m.mate_cache_append(c, x, x, counts=n)
    assert torch.equal(c.k, c.v)
    for s, k in enumerate([5, 0, 9]):
        for j in range(k):
            assert torch.equal(c.k[0, c.table[s, j // 4], :, j % 4], x[s, :, j])
    c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("pages,S", [(70001, 4096), (70001, 5000), (9000, 4097), (31, 33)])
def test_long_lists_and_many_pages(pages, S):
    import paper_2109_04312_b200 as m
    c = m.Cache.empty(pages, 2, 1, 8, S, 20, [0])
    model = CacheModel(pages, 2, S, 20)
    rng = np.random.default_rng(3)
    seqs, counts = rng.permutation(S)[:4096].tolist(), rng.integers(0, 41, min(S, 4096)).tolist()
    seqs[5], seqs[-1] = seqs[3], seqs[0]   # (one entry more of two sequences)
    for _ in range(2):
        assert m.mate_cache_extend(c, ints(seqs), ints(counts)).tolist() == model.extend(seqs, counts)
        gone = rng.permutation(S)[:S // 2].tolist()
        m.mate_cache_free(c, ints(gone))
        model.free(gone)
    parents, children = rng.integers(0, S, S)[:4096].tolist(), rng.permutation(S)[:4096].tolist()
    children[1] = children[-1]
    m.mate_cache_fork(c, ints(parents), ints(children))
    model.fork(parents, children)
    assert int(m.mate_cache_compact(c)) == model.compact()
    for name in ("table", "lens", "refs"):
        assert np.array_equal(getattr(c, name).cpu().numpy(), getattr(model, name)), name
    with pytest.raises(m.MateError, match="unsupported"):
        m.mate_cache_extend(c, ints([0] * 4097), ints([0] * 4097))


@pytest.mark.gpu
def test_granted_over_its_own_inputs():
    import paper_2109_04312_b200 as m
    for which in range(2):
        c, model = make(m)
        args = [ints([4, 0, 3]), ints([9, 13, 1])]
        granted = m.mate_cache_extend(c, *args, granted=args[which])
        assert granted is args[which] and granted.tolist() == model.extend([4, 0, 3], [9, 13, 1])
        for name in ("table", "lens", "refs"):
            assert np.array_equal(getattr(c, name).cpu().numpy(), getattr(model, name)), name
        c.status()


@pytest.mark.gpu
def test_wishes_beyond_32_bits():
    # together the list wants 2^31 pages and more; whoever fits in front of it gets theirs, nobody behind it
    import paper_2109_04312_b200 as m
    S, W = 4096, 530000
    c = m.Cache.empty(70, 1, 1, 8, S, W, [0])
    counts = torch.full((S,), W, dtype=torch.int32, device="cuda")
    counts[0], counts[2], counts[-1] = 60, 0, 1
    granted = m.mate_cache_extend(c, None, counts)
    want = torch.zeros_like(granted)
    want[0] = 60
    assert torch.equal(granted, want) and torch.equal(c.lens, want)
    assert c.table[0, :60].tolist() == list(range(60)) and int((c.table >= 0).sum()) == 60 and int(c.refs.sum()) == 60
    with pytest.raises(m.MateError, match="out of memory"):
        c.status()


@pytest.mark.gpu
def test_more_tokens_than_a_launch_takes():
    import paper_2109_04312_b200 as m
    cache = m.Cache.empty(2, 4, 2, 128, 2, 1, [0, 1])
    for B, offset in ((2, 0), (1024, 0), (1024, 1)):      # (one element at a time where the address is odd: eight times as many threads)
        K = torch.ones(129, device="cuda", dtype=torch.bfloat16)[offset:offset + 128].expand(B, 2, 2 ** 31 - 1, 128)
        many = torch.zeros(B, dtype=torch.int32, device="cuda")
        if B == 2:
            K = K[:, :, :0]                               # none at all is fine
            m.mate_cache_append(cache, K, K, many, many)
            continue
        with pytest.raises(m.MateError, match="unsupported"):
            m.mate_cache_append(cache, K, K, many, many)
    cache.status()
    assert not cache.k.any() and not cache.lens.any()


@pytest.mark.gpu
def test_a_step_in_a_graph():
    # extend and append captured once, replayed for token after token; forks and frees between the replays
    import paper_2109_04312_b200 as m
    c, model = make(m, layers=1, pages=60)
    seqs, counts = ints([2, 0, 5]), ints([1, 1, 1])
    K = torch.zeros(3, 2, 1, 16, dtype=torch.bfloat16, device="cuda")
    marks = torch.zeros(3, 1, dtype=torch.int32, device="cuda")
    V, row, col, granted = K.clone(), marks.clone(), marks.clone(), counts.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.mate_cache_extend(c, seqs, counts, granted)
        m.mate_cache_append(c, K, V, seqs, granted, row, col)
    same(c, model, "captured only")
    mark = 1
    for step in range(9):
        new = np.arange(mark, mark + 3)[:, None]
        mark += 3
        x = value_of(new, 1, 2, 16)[:, :, 0].transpose(0, 2, 1, 3).astype(np.float32)
        K.copy_(torch.from_numpy(x))
        V.copy_(torch.from_numpy(252 - x))
        row.copy_(ints(new % 1000))
        col.copy_(ints(new % 77))
        g.replay()
        model.extend([2, 0, 5], [1, 1, 1])
        model.append([2, 0, 5], [1, 1, 1], new)
        if step == 5:
            m.mate_cache_fork(c, ints([2]), ints([1]))
            model.fork([2], [1])
            m.mate_cache_free(c, ints([0]))
            model.free([0])
        same(c, model, step)
    c.status()


# ---- without a GPU

class Struct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "row_ids", "col_ids", "table", "lens", "prefix", "refs", "status", "head_view")] + \
        [(n, ctypes.c_int64) for n in ("layer_stride", "page_stride", "head_stride", "slot_stride")] + \
        [(n, ctypes.c_int32) for n in ("layers", "pages", "page_size", "seqs", "width", "heads", "kv_heads", "d", "dtype", "device")]


def struct(**kw):
    buf = ctypes.create_string_buffer(8192)
    at = (ctypes.addressof(buf) + 255) & ~255
    view = (ctypes.c_uint8 * 8)(0, 1, 2, 0, 1, 2, 0, 1)
    s = Struct(*[at] * 9, ctypes.addressof(view), 1024, 512, 256, 64, 1, 4, 4, 2, 2, 4, 2, 64, 0, 0)
    s.keep = (buf, view)
    for k, x in kw.items():
        setattr(s, k, x)
    return s, at


def test_the_c_entries_refuse_before_anything_is_launched():
    from paper_2109_04312_b200 import build
    lib = ctypes.CDLL(build.build())
    P, L = ctypes.c_void_p, ctypes.c_int64 * 3
    size = ctypes.c_size_t()

    def every(s, at, n=1, ws=1 << 20, rows=P):
        z = L(0, 64, 64)
        r = ctypes.byref(s) if s is not None else None
        return [lib.mate_cache_extend(r, P(at), P(at), n, P(at), None),
                lib.mate_cache_fork(r, P(at), P(at), n, P(at), ctypes.c_size_t(ws), None),
                lib.mate_cache_free(r, P(at), n, None),
                lib.mate_cache_compact(r, P(at), P(at), ctypes.c_size_t(ws), None),
                lib.mate_cache_append(r, 0, P(at), P(at), z, z, n, 1, P(at), P(at), P(at), P(at), P(at), P(at), 64, ctypes.c_float(1), 0, None, None,
                                      None, None, None),
                lib.mate_attn_decode(r, 0, P(at), z, n, P(at), P(at), P(at), ctypes.c_float(1), 0, P(at), P(at), P(at), ctypes.c_size_t(ws), None),
                lib.mate_cache_workspace_bytes(r, n, ctypes.byref(size), None, None), lib.mate_cache_status(r, None)]

    assert every(None, 0)[:6] == [-1] * 6
    for bad in ("k", "v", "row_ids", "col_ids", "table", "lens", "prefix", "refs", "status", "head_view"):
        assert every(*struct(**{bad: None})) == [-1] * 8, bad
    for kw in (dict(layers=0), dict(pages=0), dict(page_size=0), dict(seqs=0), dict(width=-1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3)):
        assert every(*struct(**kw)) == [-1] * 8, kw
    for kw in (dict(d=0), dict(d=4), dict(d=136), dict(dtype=2), dict(pages=2 ** 29, page_size=16), dict(width=2 ** 29, page_size=16),
               dict(page_size=2 ** 30, kv_heads=2), dict(layers=40000)):
        assert every(*struct(**kw)) == [-2] * 8, kw
    s, at = struct()
    for kw in (dict(page_stride=4), dict(layer_stride=-8), dict(k=at + 2), dict(v=at + 8)):
        assert every(*struct(**kw)) == [-3] * 8, kw
    s, at = struct()
    s.keep[1][2] = 3   # no such view
    assert every(s, at) == [-1] * 8
    s, at = struct()
    r, z = ctypes.byref(s), L(0, 64, 64)
    one = ctypes.c_float(1)
    assert lib.mate_cache_extend(r, P(at), None, 1, P(at), None) == -1 and lib.mate_cache_extend(r, P(at), P(at), 1, None, None) == -1
    assert lib.mate_cache_extend(r, None, P(at), 3, P(at), None) == -1 and lib.mate_cache_extend(r, P(at), P(at), -1, P(at), None) == -1
    assert lib.mate_cache_extend(r, P(at), P(at), 4097, P(at), None) == -2
    assert lib.mate_cache_fork(r, None, P(at), 1, P(at), 4096, None) == -1 and lib.mate_cache_fork(r, P(at), None, 1, P(at), 4096, None) == -1
    assert lib.mate_cache_fork(r, P(at), P(at), 1, None, 4096, None) == -7 and lib.mate_cache_fork(r, P(at), P(at), 1, P(at), 1, None) == -7
    assert lib.mate_cache_fork(r, P(at), P(at), 1, P(at + 16), 4096, None) == -3 and lib.mate_cache_fork(r, P(at), P(at), 4097, P(at), 1 << 20, None) == -2
    assert lib.mate_cache_compact(r, None, P(at), 1 << 20, None) == -1 and lib.mate_cache_compact(r, P(at), P(at), 8, None) == -7
    assert lib.mate_cache_free(r, None, 3, None) == -1 and lib.mate_cache_free(r, P(at), -1, None) == -1

    def append(layer=0, k=at, v=at, ks=z, B=1, N=1, seqs=at, row=at, col=at, f=at, rot=64, flags=0, q=None, qs=None, qo=None):
        p = lambda x: P(x) if x else None  # noqa: E731
        return lib.mate_cache_append(r, layer, p(k), p(v), ks, z, B, N, p(seqs), None, p(row), p(col), None, p(f), rot, one, flags, p(q), qs, p(qo), qs, None)

    for kw in (dict(layer=1), dict(layer=-1), dict(k=0), dict(v=0), dict(ks=None), dict(B=-1), dict(N=-1), dict(seqs=0, B=3), dict(row=0), dict(col=0),
               dict(rot=66), dict(rot=3), dict(f=0), dict(flags=8), dict(q=at), dict(q=at, qs=z), dict(qo=at), dict(q=at, qs=z, qo=at, f=0, rot=0)):
        assert append(**kw) == -1, kw
    assert append(k=at + 1) == -3

    def decode(layer=0, q=at, qs=z, B=1, seqs=at, row=at, col=at, max_len=0, o=at, l=at):
        p = lambda x: P(x) if x else None  # noqa: E731
        return lib.mate_attn_decode(r, layer, p(q), qs, B, p(seqs), p(row), p(col), one, max_len, p(o), p(l), P(at), ctypes.c_size_t(1 << 30), None)

    for kw in (dict(layer=1), dict(layer=-1), dict(q=0), dict(qs=None), dict(B=-1), dict(seqs=0, B=3), dict(row=0), dict(col=0), dict(max_len=-1), dict(o=0),
               dict(l=0)):
        assert decode(**kw) == -1, kw
    for kw in (dict(q=at + 2), dict(o=at + 8), dict(qs=L(4, 64, 0)), dict(qs=L(64, 4, 0))):
        assert decode(**kw) == -3, kw


def test_refusals_of_the_binding():
    # host tensors: what is refused here is refused for its type, shape or layout; what passes stops at the next check, that
    # the tensors are on a GPU
    import paper_2109_04312_b200 as m
    z = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    k = torch.zeros(1, 4, 2, 4, 16)
    good = [k, k.clone(), z(4, 4), z(4, 4), z(2, 3), z(2), z(2), z(4)]

    def cache(**kw):
        a = list(good)
        for i, x in kw.items():
            a[int(i[1:])] = x
        return m.Cache(*a, [0, 1])

    for what, kw in (("k and v", dict(_0=k[0])), ("k and v", dict(_1=k[:, :3])), ("k and v", dict(_1=k.bfloat16())),
                     ("k and v", dict(_0=k.transpose(2, 3).contiguous().transpose(2, 3))), ("k must be contiguous", dict(_0=torch.zeros(1, 4, 2, 16, 4).transpose(3, 4))),
                     ("k and v", dict(_0=k[:, :1].expand(1, 4, 2, 4, 16), _1=k[:, :1].expand(1, 4, 2, 4, 16))), ("row_ids", dict(_2=z(4, 3))),
                     ("col_ids", dict(_3=z(4, 4).long())), ("table", dict(_4=z(6))), ("lens", dict(_5=z(3))), ("prefix", dict(_6=z(2, 1))), ("refs", dict(_7=z(5)))):
        with pytest.raises(ValueError, match="^" + what):
            cache(**kw)
    with pytest.raises(ValueError, match="CUDA"):
        cache()
    with pytest.raises(ValueError, match="^k and v"):
        cache(_1=k)
    with pytest.raises(TypeError):
        cache(_0=k.half(), _1=k.half())


@pytest.fixture(scope="module")
def arithmetic(tmp_path_factory):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    so = str(tmp_path_factory.mktemp("arith") / "arith.so")
    subprocess.run([nvcc, "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-cudart", "none", "-I", os.path.join(ROOT, "paper_2109_04312_b200", "csrc"), "-I",
                    os.path.join(ROOT, "include"), "-o", so, os.path.join(ROOT, "tests", "cache_arithmetic.cpp")], check=True)
    return ctypes.CDLL(so)


def test_index_arithmetic(arithmetic):
    a = arithmetic
    for x, n in ((-2 ** 31, 5), (-1, 5), (0, 5), (4, 5), (5, 5), (2 ** 31 - 1, 5), (0, 0)):
        assert a.in_range_(x, n) == (0 <= x < n)
    for n in (0, 1, 3, 4, 5, 2 ** 30, 2 ** 30 - 1):
        for ps in (1, 3, 4, 24, 2 ** 30):
            assert a.pages_of_(n, ps) == -(-n // ps)
    bad = ctypes.c_int()
    for n, most in ((-2 ** 31, 9), (-1, 9), (0, 9), (9, 9), (10, 9), (2 ** 31 - 1, 2 ** 30)):
        assert a.clip_len_(n, most, ctypes.byref(bad)) == min(max(n, 0), most) and bad.value == (not 0 <= n <= most)
    rng = np.random.default_rng(0)
    for _ in range(50):
        need = rng.integers(0, 4, rng.integers(1, 40))
        off = np.concatenate([[0], np.cumsum(need)]).astype(np.int32)
        owners = np.repeat(np.arange(len(need)), need)
        for r, want in enumerate(owners):
            assert a.owner_of_(off.ctypes.data_as(ctypes.c_void_p), len(need), r) == want
            long = np.concatenate([off[:-1], [2 ** 40]]).astype(np.int64)   # the last one wants more than there can be
            assert a.owner_of_64(long.ctypes.data_as(ctypes.c_void_p), len(need), r) == want


# ---- lists with an entry that is refused ahead of another one of the same sequence

@pytest.mark.gpu
@pytest.mark.parametrize("seqs", [6, 5000])   # (claims in shared memory, and in the lengths)
def test_a_refused_entry_is_its_sequences_first_all_the_same(seqs):
    import paper_2109_04312_b200 as m
    c = m.Cache.empty(40, 4, 1, 8, seqs, 3, [0])
    m.mate_cache_extend(c, ints([3]), ints([2]))
    # sequence 1: more than its row of the table holds, then what would fit; 2: a negative count, then one; 3: 2 + 11 tokens, then 4;
    # 4 stands once
    granted = m.mate_cache_extend(c, ints([1, 1, 2, 2, 3, 3, 4, 1]), ints([13, 5, -1, 1, 11, 4, 12, 1]))
    assert granted.tolist() == [0, 0, 0, 0, 0, 0, 12, 0]
    assert c.lens[:6].tolist() == [0, 0, 0, 2, 12, 0] and not c.lens[6:].any()
    assert int(c.refs.sum()) == 4 and c.table[4].tolist() == [1, 2, 3] and c.table[3].tolist() == [0, -1, -1]
    with pytest.raises(m.MateError):
        c.status()
    # lengths that are none stay as they are, and nobody gets anything on their account
    c.lens[0], c.lens[5] = -7, 13
    assert m.mate_cache_extend(c, ints([0, 5, 0, 5, 2]), ints([1, 1, 2, 2, 1])).tolist() == [0, 0, 0, 0, 1]
    assert c.lens[:6].tolist() == [-7, 0, 1, 2, 12, 13]
    with pytest.raises(m.MateError, match="invalid argument"):
        c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("seqs", [6, 5000])
def test_a_refused_entry_is_its_childs_first_all_the_same(seqs):
    import paper_2109_04312_b200 as m
    c = m.Cache.empty(40, 4, 1, 8, seqs, 3, [0])
    assert m.mate_cache_extend(c, ints([1, 4]), ints([6, 3])).tolist() == [6, 3]
    lens, table, refs = c.lens.clone(), c.table.clone(), c.refs.clone()
    # child 0: of no parent, then of 1; child 2: of a sequence that is out of range, then of 1; child 4: not empty, twice
    m.mate_cache_fork(c, ints([-1, 1, seqs, 1, 1, 1]), ints([0, 0, 2, 2, 4, 4]))
    assert torch.equal(c.lens, lens) and torch.equal(c.table, table) and torch.equal(c.refs, refs)
    with pytest.raises(m.MateError, match="invalid argument"):
        c.status()
    # a parent whose length is none; then the children are still to be had
    c.lens[3] = -5
    m.mate_cache_fork(c, ints([3, 1, 1]), ints([0, 0, 2]))
    assert c.lens[:6].tolist() == [0, 6, 6, -5, 3, 0] and c.table[2, 0] == c.table[1, 0] and c.refs[:4].tolist() == [2, 1, 1, 1]
    with pytest.raises(m.MateError, match="invalid argument"):
        c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_append_with_no_pairs_to_turn(dtype):
    # as mate_rope: every element is passed on, queries too
    import paper_2109_04312_b200 as m
    c = m.Cache.empty(9, 4, 2, 16, 3, 3, [0, 1, 1, 0], dtype=dtype)
    n = ints([5, 0, 3])
    m.mate_cache_extend(c, None, n)
    Q, K, V = (torch.randn(3, h, 5, 16, device="cuda").to(dtype) for h in (4, 2, 2))
    none = m.mate_rope_freqs(0)
    assert torch.equal(m.mate_rope(Q, ints([[7] * 5] * 3), none), Q)
    for positions in (None, ints([[7] * 5] * 3)):
        q = m.mate_cache_append(c, K, V, counts=n, freqs=none, positions=positions, mscale=3.0, Q=Q)
        assert torch.equal(q, Q) and q.data_ptr() != Q.data_ptr()
    for s, count in enumerate([5, 0, 3]):
        for j in range(count):
            assert torch.equal(c.k[0, c.table[s, j // 4], :, j % 4], K[s, :, j]) and torch.equal(c.v[0, c.table[s, j // 4], :, j % 4], V[s, :, j])
    c.status()


@pytest.mark.gpu
def test_append_refuses_an_output_without_queries():
    import paper_2109_04312_b200 as m
    c = m.Cache.empty(9, 4, 2, 16, 3, 3, [0, 1, 1, 0])
    K = torch.zeros(3, 2, 1, 16, device="cuda").bfloat16()
    with pytest.raises(ValueError, match="^out must be None"):
        m.mate_cache_append(c, K, K, freqs=m.mate_rope_freqs(16), out=torch.zeros(3, 4, 1, 16, device="cuda").bfloat16())


@pytest.mark.gpu
def test_the_memory_stays_while_the_cache_lives():
    # attributes set to other tensors: the calls go by the ones the cache was made of, whose memory nobody else gets meanwhile
    import gc

    import paper_2109_04312_b200 as m
    torch.cuda.synchronize()
    gc.collect()
    base = torch.cuda.memory_allocated()
    c = m.Cache.empty(64, 16, 4, 64, 8, 8, [0] * 4, layers=4)
    held = torch.cuda.memory_allocated() - base
    assert held > 2 * 64 * 16 * 4 * 64 * 2 * 4
    for name in ("k", "v", "row_ids", "col_ids", "table", "lens", "prefix", "refs", "status_word"):
        setattr(c, name, None)
    gc.collect()
    assert torch.cuda.memory_allocated() - base == held
    assert m.mate_cache_extend(c, ints([3]), ints([17])).tolist() == [17]
    assert m.mate_cache_compact(c) == 2
    c.status()
    c = m.Cache.empty(4, 4, 1, 8, 2, 2, [0])
    k = c.k.data_ptr()
    c.k.data = torch.zeros(1, 4, 1, 4, 8, device="cuda").bfloat16()      # the tensor itself gets other memory
    assert torch.zeros(1, 4, 1, 4, 8, device="cuda").bfloat16().data_ptr() != k
    del c
    gc.collect()
    assert torch.cuda.memory_allocated() == base


def test_scales_that_the_attention_of_one_token_refuses():
    from paper_2109_04312_b200 import build
    lib = ctypes.CDLL(build.build())
    s, at = struct()
    P, z = ctypes.c_void_p, (ctypes.c_int64 * 3)(0, 64, 64)

    def decode(scale, B=0):
        return lib.mate_attn_decode(ctypes.byref(s), 0, P(at), z, B, P(at), P(at), P(at), ctypes.c_float(scale), 0, P(at), P(at), P(at),
                                    ctypes.c_size_t(1 << 30), None)

    for scale, status in ((float("nan"), -1), (float("inf"), -1), (-float("inf"), -1), (3.4e38, -2), (-2.4e38, -2)):
        assert decode(scale) == status == decode(scale, 1), scale
    for scale in (2.3e38, -2.3e38, 0.0, 1e-45):    # these go on to the next check: here, for the device
        assert decode(scale) not in (-1, -2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_queries_turn_by_their_positions_in_their_sequences(interleaved, dtype):
    # no positions given: token j of the last n of a sequence of L stands at L - n + j, its query as its key; behind them there is no
    # token, and the queries are turned by position 0
    import paper_2109_04312_b200 as m
    B, N, H, Hk, d = 3, 5, 4, 2, 16
    c, f = m.Cache.empty(40, 4, Hk, d, 6, 9, [0, 1] * 2, dtype=dtype), m.mate_rope_freqs(d)
    seqs, counts = ints([4, 0, 2]), ints([5, 0, 3])
    m.mate_cache_extend(c, ints([2, 0]), ints([17, 9]))
    m.mate_cache_extend(c, seqs, counts)
    Q, K, V = (torch.randn(B, h, N, d, device="cuda").to(dtype) for h in (H, Hk, Hk))
    q = m.mate_cache_append(c, K, V, seqs, counts, freqs=f, interleaved=interleaved, mscale=0.9, Q=Q)
    own = ints([[0, 1, 2, 3, 4], [0, 0, 0, 0, 0], [17, 18, 19, 0, 0]])
    assert torch.equal(q, m.mate_rope(Q, own, f, interleaved=interleaved, mscale=0.9))
    want = turn(Q.double().cpu().numpy(), own.cpu().numpy()[:, None], f.cpu().numpy(), interleaved, 0.9)
    # sine, cosine and their products in fp32 (6e-7 of |a| + |b|), the result's rounding
    tol = 6e-7 * 2 * Q.abs().max().item() + (np.abs(want) * 2.0 ** -8 if dtype == torch.bfloat16 else 0)
    assert np.all(np.abs(q.double().cpu().numpy() - want) <= tol)
    c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("slots_first", [False, True])
def test_pages_of_the_largest_size(slots_first, dtype):
    # 2^20 rows of keys to a page: partly filled ones copied, whole ones moved
    import paper_2109_04312_b200 as m
    ps, pages, d = 1 << 19, 5, 8
    shape = (1, pages, ps, 2, d) if slots_first else (1, pages, 2, ps, d)
    k, v = (torch.zeros(shape, dtype=dtype, device="cuda") for _ in range(2))
    if slots_first:
        k, v = k.transpose(2, 3), v.transpose(2, 3)
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    c = m.Cache(k, v, z(pages, ps), z(pages, ps), z(4, 2) - 1, z(4), z(4), z(pages), [0, 1])
    n = ints([ps + 5, ps - 3])
    assert m.mate_cache_extend(c, None, n).tolist() == n.tolist() and c.table[:2].tolist() == [[0, 1], [2, -1]]
    K, V = (torch.randn(2, 2, ps + 5, d, device="cuda").to(dtype) for _ in range(2))
    ids = torch.arange(2 * (ps + 5), dtype=torch.int32, device="cuda").view(2, -1)
    m.mate_cache_append(c, K, V, counts=n, row_ids=ids, col_ids=ids + 1)
    m.mate_cache_fork(c, ints([1, 0]), ints([3, 2]))
    assert c.table[2:].tolist() == [[0, 4], [3, -1]] and c.lens.tolist() == [ps + 5, ps - 3] * 2
    m.mate_cache_free(c, ints([1]))
    assert int(m.mate_cache_compact(c)) == 4 and c.table.tolist() == [[0, 1], [-1, -1], [0, 2], [3, -1]]
    for s, of in ((0, 0), (2, 0), (3, 1)):
        for i, page in enumerate(p for p in c.table[s].tolist() if p >= 0):
            some = slice(i * ps, min((i + 1) * ps, int(n[of])))
            fill = some.stop - some.start
            assert torch.equal(c.k[0, page, :, :fill], K[of, :, some]) and torch.equal(c.v[0, page, :, :fill], V[of, :, some])
            assert torch.equal(c.row_ids[page, :fill], ids[of, some]) and torch.equal(c.col_ids[page, :fill], ids[of, some] + 1)
    c.status()


@pytest.mark.gpu
def test_beams_in_a_graph():
    # children dropped, made anew and moved together, captured once and replayed after the parents have grown; another graph shares no workspace
    import paper_2109_04312_b200 as m
    c, model = make(m, pages=70, seqs=8, width=6, page_size=4)
    parents, children = ints([0, 1, 0, 1]), ints([4, 5, 6, 7])
    mark = append(m, c, model, [0, 1], m.mate_cache_extend(c, ints([0, 1]), ints([3, 6])).tolist() and model.extend([0, 1], [3, 6]), 1)
    m.mate_cache_fork(c, parents, children)
    model.fork([0, 1, 0, 1], [4, 5, 6, 7])
    graphs, lives = [], []
    for _ in range(2):
        g, live = torch.cuda.CUDAGraph(), ints(0)
        with torch.cuda.graph(g):
            m.mate_cache_free(c, children)
            m.mate_cache_fork(c, parents, children)
            m.mate_cache_compact(c, live)
        graphs.append(g)
        lives.append(live)
    same(c, model, "captured only")
    for step in range(6):
        granted = m.mate_cache_extend(c, ints([0, 1]), ints([2, 1])).tolist()
        assert granted == model.extend([0, 1], [2, 1])
        mark = append(m, c, model, [0, 1], granted, mark)
        graphs[step % 2].replay()
        model.free([4, 5, 6, 7])
        model.fork([0, 1, 0, 1], [4, 5, 6, 7])
        assert int(lives[step % 2]) == model.compact()
        same(c, model, step)
    c.status()
