"""mate_cache_groups against its description, entry by entry."""
import ctypes

import numpy as np
import pytest
import torch

from tests.test_cache_pages import struct


def model(table, lens, ps, pages, seqs, min_len):
    least, n, width = max(1, -(-min_len // ps)), len(seqs), table.shape[1]

    def full(s):
        return min(max(lens[s], 0), width * ps) // ps if 0 <= s < len(lens) else 0

    def common(a, b):
        k = 0
        while k < min(full(a), full(b)) and table[a, k] == table[b, k] and 0 <= table[a, k] < pages:
            k += 1
        return k

    out, i = np.zeros((3, n), np.int32), 0
    while i < n:
        j = i + 1
        while j < n and common(seqs[j - 1], seqs[j]) >= least:
            j += 1
        out[0, i:j], out[1, i:j] = i, j - i
        # all of them against the first one, not each against the one before
        out[2, i:j] = ps * min(common(seqs[i], s) for s in seqs[i + 1:j]) if j - i > 1 else 0
        i = j
    return out


def cache(m, table, lens, ps, pages):
    c = m.Cache.empty(pages, ps, 1, 8, len(lens), table.shape[1], [0])
    c.table.copy_(torch.from_numpy(table))
    c.lens.copy_(torch.from_numpy(lens))
    return c


def family(rng, S, width, ps, pages):
    """Sequences that share pages with the one before, more or less of them, or none."""
    table, lens = np.full((S, width), -1, np.int32), np.zeros(S, np.int32)
    for s in range(S):
        table[s] = rng.integers(0, pages, width)
        if s and rng.random() < 0.8:
            k = int(rng.integers(0, width + 1))
            table[s, :k] = table[s - 1, :k]
        lens[s] = rng.integers(0, width * ps + 1) if rng.random() < 0.5 else width * ps
    return table, lens


@pytest.mark.gpu
@pytest.mark.parametrize("S,width,ps", [(1, 1, 1), (7, 3, 4), (40, 9, 16), (300, 130, 2), (130, 40, 1), (20, 5000, 1)])
@pytest.mark.parametrize("min_len", [0, 1, 17])
def test_groups(S, width, ps, min_len):
    import paper_2109_04312_b200 as m
    rng = np.random.default_rng(S + width)
    table, lens = family(rng, S, width, ps, 50)
    c = cache(m, table, lens, ps, 50)
    assert np.array_equal(m.mate_cache_groups(c, min_len=min_len).cpu().numpy(), model(table, lens, ps, 50, list(range(S)), min_len))
    # in another order, some of them twice
    seqs = np.concatenate([np.arange(S)[::-1], rng.integers(0, S, 5), [0, 0]]).tolist()
    out = torch.full((3, len(seqs)), 77, dtype=torch.int32, device="cuda")
    r = m.mate_cache_groups(c, torch.tensor(seqs, dtype=torch.int32, device="cuda"), min_len, out)
    assert r is out and np.array_equal(out.cpu().numpy(), model(table, lens, ps, 50, seqs, min_len))
    c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["one group", "pairs", "alone", "mixed"])
def test_the_longest_list(kind):
    import paper_2109_04312_b200 as m
    n, width, ps = 4096, 6, 4
    rng = np.random.default_rng(1)
    table = {"one group": np.zeros(n, int), "pairs": np.arange(n) // 2, "alone": np.arange(n), "mixed": np.sort(rng.integers(0, 90, n))}[kind]
    table = np.repeat(table[:, None], width, 1).astype(np.int32)
    table[:, 4:] = rng.integers(0, 4, (n, 2))
    lens = rng.integers(3 * ps, width * ps + 1, n).astype(np.int32)
    c = cache(m, table, lens, ps, n)
    assert np.array_equal(m.mate_cache_groups(c).cpu().numpy(), model(table, lens, ps, n, list(range(n)), 1))


@pytest.mark.gpu
def test_what_is_out_of_range_is_alone():
    import paper_2109_04312_b200 as m
    table = np.array([[0, 1, 2], [0, 1, 2], [0, 1, -1], [0, 1, -1], [9, 1, 1], [9, 1, 1], [0, 1, 2], [0, 1, 2]], np.int32)
    lens = np.array([12, 12, 12, 12, 12, 12, -3, 999], np.int32)
    for seqs in ([0, 1, 2, 3], [4, 5], [0, 8, 1], [0, -1, -1, 1], [0, 6, 1], [0, 7, 1]):
        c = cache(m, table, lens, 4, 5)
        got = m.mate_cache_groups(c, torch.tensor(seqs, dtype=torch.int32, device="cuda")).cpu().numpy()
        assert np.array_equal(got, model(table, lens, 4, 5, seqs, 1)), seqs
        if set(seqs) & {-1, 8, 6, 7}:
            with pytest.raises(m.MateError, match="invalid"):
                c.status()
        c.status()


@pytest.mark.gpu
def test_forks_in_a_graph():
    # beams as mate_cache_fork makes them; captured once, replayed with other lengths and on a stream of its own
    import paper_2109_04312_b200 as m
    c = m.Cache.empty(64, 4, 1, 8, 12, 8, [0])
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    m.mate_cache_extend(c, i32(0, 1, 2), i32(9, 16, 3))
    m.mate_cache_fork(c, i32(0, 0, 1, 1, 1, 2), i32(3, 4, 5, 6, 7, 8))
    seqs = i32(0, 3, 4, 1, 5, 6, 7, 2, 8)
    want = [[0] * 3 + [3] * 4 + [7, 8], [3] * 3 + [4] * 4 + [1, 1], [8] * 3 + [16] * 4 + [0, 0]]
    assert m.mate_cache_groups(c, seqs).tolist() == want
    side, graph, out = torch.cuda.Stream(), torch.cuda.CUDAGraph(), i32(*[0] * 27).view(3, 9)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        m.mate_cache_groups(c, seqs, out=out)
    m.mate_cache_free(c, i32(5))
    graph.replay()
    assert out.tolist() == [[0] * 3 + [3, 4, 5, 5, 7, 8], [3] * 3 + [1, 1, 2, 2, 1, 1], [8] * 3 + [0, 0, 16, 16, 0, 0]]
    assert m.mate_cache_groups(c, seqs[:0]).shape == (3, 0)


@pytest.mark.gpu
def test_refusals():
    import paper_2109_04312_b200 as m
    c, i = m.Cache.empty(4, 4, 1, 8, 2, 2, [0]), torch.zeros(12, dtype=torch.int32, device="cuda")
    for what, call in (("seqs", lambda: m.mate_cache_groups(c, i.long())), ("seqs", lambda: m.mate_cache_groups(c, i.cpu())),
                       ("out", lambda: m.mate_cache_groups(c, i[:2], out=i[:4].view(2, 2))), ("min_len", lambda: m.mate_cache_groups(c, min_len=-1)),
                       ("out", lambda: m.mate_cache_groups(c, i[:3], out=i[:9].view(3, 3)))):
        with pytest.raises(ValueError, match="^%s must be|^%s without" % (what, what)):
            call()
    with pytest.raises(m.MateError, match="unsupported|not available"):
        m.mate_cache_groups(c, torch.zeros(4097, dtype=torch.int32, device="cuda"))


def test_the_c_entry_refuses_before_anything_is_launched():
    from paper_2109_04312_b200 import build
    lib = ctypes.CDLL(build.build())
    P = ctypes.c_void_p
    assert lib.mate_cache_groups(None, None, 1, 1, None, None) == -1
    s, at = struct()
    r = ctypes.byref(s)
    assert lib.mate_cache_groups(r, P(at), 1, 1, None, None) == -1 and lib.mate_cache_groups(r, P(at), 1, -1, P(at), None) == -1
    assert lib.mate_cache_groups(r, P(at), -1, 1, P(at), None) == -1 and lib.mate_cache_groups(r, None, 3, 1, P(at), None) == -1
    assert lib.mate_cache_groups(r, P(at), 4097, 1, P(at), None) == -2
    s, at = struct(d=4)
    assert lib.mate_cache_groups(ctypes.byref(s), P(at), 1, 1, P(at), None) == -2
