"""Groups of mate_attn_decode_shared that say more than there is, where nothing else is out of range: status tells of the groups alone."""
import numpy as np
import pytest
import torch

from tests.test_decode import DT
from tests.test_decode_shared import Shared, i32


@pytest.mark.gpu
@pytest.mark.parametrize("always", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_shared_tokens_than_max_len(always, dtype):
    # all lengths are below max_len, so mate_attn_decode finds nothing wrong
    import paper_2109_04312_b200 as m
    case = Shared(m, [(9, [30, 9, 40]), (4, [7, 1])], 6, 2, 64, 16, [0, 0, 1, 1, 2, 0], dtype, seed=21)
    B, max_len = len(case.lens), 200
    assert max(case.lens) < max_len
    q_ids = case.new_ids(list(range(B)))
    Q = torch.randn(B, 6, 64, generator=torch.Generator().manual_seed(3)).to(DT[dtype]).cuda()
    a, b = i32(q_ids[0]), i32(q_ids[1])
    alone = m.mate_attn_decode(case.c, Q, a, b, max_len=max_len)
    case.c.status()
    m.mate_attn_decode_shared(case.c, Q, a, b, i32(case.groups), max_len=max_len, always=always)
    case.c.status()
    for shared in (max_len + 1, 208, 2 ** 31 - 1):     # (one token more than max_len, whole pages, what no table holds)
        groups = case.groups.copy()
        groups[2, :3] = shared
        O, LSE = m.mate_attn_decode_shared(case.c, Q, a, b, i32(groups), max_len=max_len, always=always)
        with pytest.raises(m.MateError, match="invalid"):
            case.c.status()
        case.c.status()
        case.check(Q, list(range(B)), q_ids, O, LSE)   # every entry alone
        if not always:
            assert torch.equal(O, alone[0]) and torch.equal(LSE, alone[1])
    # as many as max_len, in a table that holds them, but more than the sequences have
    groups = case.groups.copy()
    groups[2, 3:] = max_len
    O, LSE = m.mate_attn_decode_shared(case.c, Q, a, b, i32(groups), max_len=max_len, always=always)
    with pytest.raises(m.MateError, match="invalid"):
        case.c.status()
    case.check(Q, list(range(B)), q_ids, O, LSE)       # (each is too short for its group, and alone)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,d", [(4, 2, 64), (140, 1, 128)])
def test_whatever_is_claimed(dtype, H, Hk, d):
    """All sequences have the same first pages, so that whatever claims come to a group, its entries share what they say: every result is the one of the sequence
    alone, and the same from call to call."""
    import paper_2109_04312_b200 as m
    rng = np.random.default_rng(H)
    case = Shared(m, [(12, rng.integers(0, 60, 24).tolist())], H, Hk, d, 16, [h % 3 for h in range(H)], dtype, seed=22)
    for turn in range(25):
        B = int(rng.integers(2, 60))
        seqs = rng.integers(0, 24, B)
        groups, at = np.zeros((3, B), np.int32), 0
        while at < B:
            n = int(rng.integers(1, min(B - at, 20) + 1))
            groups[:, at:at + n] = np.array([[at], [n], [16 * rng.integers(0, 13)]])
            at += n
        for _ in range(int(rng.integers(0, 8))):
            i = int(rng.integers(0, B))
            row = int(rng.integers(0, 3))
            groups[row, i] = (rng.integers(-1, B + 1), rng.integers(-1, B + 1), 16 * rng.integers(0, 13))[row]
        for _ in range(int(rng.integers(0, 3))):       # a group more, wherever it comes to lie
            f = int(rng.integers(0, B - 1))
            n = int(rng.integers(2, B - f + 1))
            groups[:, f:f + n:int(rng.integers(1, 3))] = np.array([[f], [n], [32]])
        q_ids = case.new_ids(seqs.tolist())
        Q = torch.randn(B, H, d, generator=torch.Generator().manual_seed(turn)).to(DT[dtype]).cuda()
        args, g = (case.c, Q, i32(q_ids[0]), i32(q_ids[1])), i32(groups)
        O, LSE = m.mate_attn_decode_shared(*args, g, seqs=i32(seqs), always=True)
        o, l = m.mate_attn_decode_shared(*args, g, seqs=i32(seqs), always=True)
        assert torch.equal(o, O) and torch.equal(l, LSE), turn
        some = rng.permutation(B)[:6 if H < 100 else 2]
        case.check(Q[some.tolist()], seqs[some].tolist(), q_ids[:, some], O[some.tolist()], LSE[some.tolist()])
        o, l = m.mate_attn_decode(*args, seqs=i32(seqs))
        # two results, each with weights that are off by some 2^-17 (products of 64 or 128 terms summed up in fp32, their exponents) times values of up to 5, in
        # bf16 by 2^-17 more (weights of 16 bits) and rounded to the type, by 2^-8 of the result at most
        assert torch.allclose(O.float(), o.float(), atol=4e-4 if dtype == "bf16" else 1e-4, rtol=2 ** -7 if dtype == "bf16" else 1e-5), turn
        assert torch.equal(LSE.isinf(), l.isinf()) and torch.allclose(LSE.nan_to_num(), l.nan_to_num(), atol=1e-4, rtol=1e-5), turn
        try:
            case.c.status()
        except m.MateError as e:
            assert "invalid" in str(e)
