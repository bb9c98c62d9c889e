"""Groups of mate_attn_decode_shared that have entries in common: the outer one is none, status says so, and every entry's result is its own."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from tests.cache_model import TEXT
from tests.conftest import ROOT
from tests.test_decode import DT
from tests.test_decode_shared import Shared, i32


@pytest.fixture(scope="module")
def fit(tmp_path_factory):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    so = str(tmp_path_factory.mktemp("fit") / "fit.so")
    subprocess.run([nvcc, "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-cudart", "none", "-I", os.path.join(ROOT, "paper_2109_04312_b200", "csrc"), "-I",
                    os.path.join(ROOT, "include"), "-o", so, os.path.join(ROOT, "tests", "groups_that_overlap.cpp")], check=True)
    return ctypes.CDLL(so)


def members(lib, groups, max_len=1 << 30):
    groups = np.ascontiguousarray(groups, np.int32)
    B = groups.shape[1]
    begins, member = np.zeros(128, np.uint32), np.zeros(B, np.int32)
    lib.members_(*(x.ctypes.data_as(ctypes.c_void_p) if isinstance(x, np.ndarray) else x for x in (groups, B, max_len, begins, member)))
    return member.astype(bool)


def model(groups, max_len=1 << 30):
    """The same, from the description: which entries claim a group that is in range, whose first entry says the same and in which no other one begins."""
    first, count, shared = groups.tolist()
    B = len(first)

    def in_range(b):
        return shared[b] > 0 and count[b] > 1 and 0 <= first[b] <= b < first[b] + count[b] <= B and shared[b] <= max_len

    leaders = [b for b in range(B) if in_range(b) and first[b] == b]
    out = []
    for b in range(B):
        f = first[b]
        same = in_range(b) and (first[f], count[f], shared[f]) == (f, count[b], shared[b])
        out.append(same and not any(f < x < f + count[b] for x in leaders))
    return np.array(out)


def test_a_group_that_begins_inside_another_one(fit):
    rng = np.random.default_rng(0)
    for B in (1, 5, 33, 64, 200, 4096):
        for _ in range(300 if B < 100 else 10):
            begins = (rng.random(B) < rng.choice([0.02, 0.3])).astype(np.uint8)
            bits = np.packbits(np.pad(begins, (0, 4096 - B)), bitorder="little").view(np.uint32)
            first = int(rng.integers(0, B))
            count = int(rng.integers(2, B - first + 1)) if B - first > 1 else 0
            if count:
                got = fit.begins_inside_(bits.ctypes.data_as(ctypes.c_void_p), first, count)
                assert bool(got) == bool(begins[first + 1:first + count].any()), (B, first, count)


def test_no_two_groups_have_an_entry_in_common(fit):
    rng = np.random.default_rng(1)
    seen = 0
    for _ in range(3000):
        B = int(rng.integers(1, 12))
        # most of them nearly right: groups one after another, in which numbers are put out of place
        groups, at = np.zeros((3, B), np.int32), 0
        while at < B:
            n = int(rng.integers(1, B - at + 1))
            groups[:, at:at + n] = np.array([[at], [n], [16 * n]])
            at += n
        good = groups.copy()
        for _ in range(int(rng.integers(0, 4))):
            groups[rng.integers(0, 3), rng.integers(0, B)] = rng.choice([-1, 0, 1, 2, 3, 4, 5, 16, 32, 48, 2 ** 31 - 1, -2 ** 31])
        is_in = members(fit, groups)
        assert np.array_equal(is_in, model(groups)), groups
        assert np.array_equal(members(fit, good), good[1] > 1)
        taken = np.zeros(B, int)
        for b in np.flatnonzero(is_in):
            f, n, _ = groups[:, b]
            assert is_in[f]
            if b == f:
                taken[f:f + n] += 1
        assert taken.max() <= 1, groups        # rows, and places of results, of one group only
        seen += len(np.flatnonzero(is_in)) < B
    assert seen > 1000


OVERLAPPING = {  # of three and two entries that share 9 and 4 pages: (first, count) where they differ
    "a group inside another one": {1: (1, 2)},
    "the members of one divided": {1: (1, 2), 2: (1, 2)},
    "one that calls itself first of what it was a member of": {1: (1, 3)},
    "one that reaches into the next one": {0: (0, 5)},
    "all of them reach into the next one": {0: (0, 5), 1: (0, 5), 2: (0, 5)},
    "one after another": {0: (0, 5), 1: (1, 4), 2: (2, 3), 3: (3, 2)},
    "the last one of a group leads the next one's": {2: (2, 3)},
}


@pytest.mark.gpu
@pytest.mark.parametrize("always", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,d", [(4, 2, 64), (300, 2, 16), (8, 1, 128)])
def test_every_entry_has_its_own_result(always, dtype, H, Hk, d):
    import paper_2109_04312_b200 as m
    case = Shared(m, [(9, [30, 9, 140]), (4, [7, 1])], H, Hk, d, 16, [h % 3 for h in range(H)], dtype, seed=H)
    B = len(case.lens)
    q_ids = case.new_ids(list(range(B)))
    q_ids[:, 1] = TEXT
    Q = torch.randn(B, H, d, generator=torch.Generator().manual_seed(d)).to(DT[dtype]).cuda()
    args = (case.c, Q, i32(q_ids[0]), i32(q_ids[1]))
    for what, differ in OVERLAPPING.items():
        groups = case.groups.copy()
        for b, (first, count) in differ.items():
            groups[0, b], groups[1, b] = first, count
            if first != 0 and b < 3:          # (an inner group of its own tokens)
                groups[2, b] = 5 * 16
        O, LSE = m.mate_attn_decode_shared(*args, i32(groups), always=always)
        with pytest.raises(m.MateError, match="invalid"):
            case.c.status()
        case.check(Q, list(range(B)), q_ids, O, LSE)
        for _ in range(5):
            o, l = m.mate_attn_decode_shared(*args, i32(groups), always=always)
            assert torch.equal(o, O) and torch.equal(l, LSE), what
        with pytest.raises(m.MateError, match="invalid"):
            case.c.status()
    # entries of none between the members are no error
    groups = case.groups.copy()
    groups[:, 1] = 1, 1, 0
    O, LSE = m.mate_attn_decode_shared(*args, i32(groups), always=always)
    case.c.status()
    case.check(Q, list(range(B)), q_ids, O, LSE)


@pytest.mark.gpu
@pytest.mark.parametrize("always", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [256, 4096])
def test_long_lists(always, dtype, n):
    # (what a block keeps of the first entries, and what it looks up again of those behind them)
    import paper_2109_04312_b200 as m
    case = Shared(m, [(3, [5, 2])], 2, 2, 16, 8, [0, 1], dtype, seed=20)
    seqs = [i % 2 for i in range(n)]
    q_ids = case.new_ids(seqs)
    Q = torch.randn(n, 2, 16, generator=torch.Generator().manual_seed(n)).to(DT[dtype]).cuda()
    some = list(range(20)) + list(range(n // 2 - 20, n // 2 + 20)) + list(range(n - 40, n))

    def check(groups, bad):
        O, LSE = m.mate_attn_decode_shared(case.c, Q, i32(q_ids[0]), i32(q_ids[1]), i32(groups), seqs=i32(seqs), always=always)
        if bad:
            with pytest.raises(m.MateError, match="invalid"):
                case.c.status()
        case.c.status()
        case.check(Q[some], [seqs[i] for i in some], q_ids[:, some], O[some], LSE[some])

    at = np.arange(n)
    good = np.stack([at // 4 * 4, np.full(n, 4), np.full(n, 24)])
    check(good, False)
    groups = good.copy()
    groups[1, n - 8:n - 4] = 8                     # reaches over the last group
    check(groups, True)
    groups = good.copy()
    groups[:2, n - 2:] = np.array([[n - 2], [2]])  # inside the last group
    check(groups, True)
    groups = good.copy()
    groups[1, 0] = n                               # the first entry's reaches over them all
    check(groups, True)
    # every entry the first of all behind it: all of them together would have n (n + 1) / 2 entries
    check(np.stack([at, n - at, np.full(n, 24)]), True)
