"""mate_rope_axes and mate_cache_append_axes against the formula in 64 bits, against mate_rope, their backward against differences."""
import ctypes

import numpy as np
import pytest
import torch

from tests.cache_model import turn
from tests.test_rope import DT, bound


def turn_axes(x, pos, axes, freqs, interleaved, mscale=1.0, backward=False):
    """Pair by pair in 64 bits: x [..., N, d], pos [A, ..., N]."""
    y, half = np.array(x, np.float64), len(freqs)
    for i, (f, a) in enumerate(zip(freqs, axes)):
        at = [2 * i, 2 * i + 1] if interleaved else [i, i + half]
        y[..., at] = turn(y[..., at], pos[a], [f], False, mscale, backward)
    return y


def check(got, x, pos, axes, freqs, dtype, interleaved=False, mscale=1.0, backward=False):
    x64, p = x.detach().double().cpu().numpy(), pos.cpu().numpy()
    want = turn_axes(x64, p if p.ndim == 2 or x.dim() == 3 else p[:, :, None], axes, freqs.cpu().numpy(), interleaved, mscale, backward)
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.all(err <= bound(x64, want, dtype, mscale)), err.max()


def some_axes(kind, pairs, A):
    return {"sections": [i * A // max(pairs, 1) for i in range(pairs)], "mixed": [i % A for i in range(pairs)],
            "any": np.random.default_rng(pairs).integers(0, A, pairs).tolist(), "last": [A - 1] * pairs}[kind]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("A,kind", [(1, "sections"), (2, "any"), (3, "sections"), (3, "mixed"), (4, "mixed"), (4, "last")])
@pytest.mark.parametrize("B,H,Hk,N,d,rot", [(1, 1, 1, 1, 2, 2), (2, 3, 1, 17, 64, 32), (3, 5, 2, 33, 40, 20), (1, 2, 2, 5, 33, 6), (1, 32, 8, 47, 128, 128),
                                            (1, 2, 1, 3, 1023, 1022), (1, 1, 2, 9, 1024, 1024), (2, 7, 1, 16, 128, 0), (2, 3, 2, 19, 80, 40)])
def test_rope_axes(B, H, Hk, N, d, rot, A, kind, interleaved, dtype):
    import paper_2109_04312_b200 as m
    g = torch.Generator().manual_seed(B * 1000 + d)
    Q, K = (torch.randn(B, h, N, d, generator=g).to(DT[dtype]).cuda() for h in (H, Hk))
    pos = torch.randint(-50, 100000, (A, B, N), generator=g, dtype=torch.int32).cuda()
    f, axes = m.mate_rope_freqs(rot), some_axes(kind, rot // 2, A)
    for backward in (False, True):
        q, k = m.mate_rope_axes(Q, pos, f, axes, K=K, interleaved=interleaved, backward=backward, mscale=1.25)
        for got, x in ((q, Q), (k, K)):
            assert got.is_contiguous()
            check(got, x, pos, axes, f, dtype, interleaved, 1.25, backward)
    # alone, one row of positions an axis for all examples, packed
    row = pos[:, 0].contiguous()
    check(m.mate_rope_axes(Q, row, f, axes, interleaved=interleaved), Q, row, axes, f, dtype, interleaved)
    check(m.mate_rope_axes(Q[0], row, f, bytes(axes), interleaved=interleaved), Q[0], row, axes, f, dtype, interleaved)
    # all axes alike: mate_rope bit for bit
    same = pos[:1].expand(A, B, N).contiguous()
    for x, y in zip(m.mate_rope_axes(Q, same, f, axes, K=K, interleaved=interleaved), m.mate_rope(Q, pos[0], f, K=K, interleaved=interleaved)):
        assert torch.equal(x, y)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_streams_and_graphs(dtype):
    import paper_2109_04312_b200 as m
    B, N, H, Hk, d, A = 2, 37, 6, 2, 64, 3
    qkv = torch.randn(B, N, H + 2 * Hk, d, device="cuda").to(DT[dtype])
    Q, K = qkv[:, :, :H].transpose(1, 2), qkv[:, :, H:H + Hk].transpose(1, 2)
    pos, f = torch.randint(0, 5000, (A, B, N), dtype=torch.int32, device="cuda"), m.mate_rope_freqs(d)
    axes = np.array(some_axes("mixed", d // 2, A))
    q, k = m.mate_rope_axes(Q, pos, f, axes, K=K)
    check(q, Q, pos, axes, f, dtype)
    check(k, K, pos, axes, f, dtype)
    # a stream of the caller's, and a graph: new positions in the old place
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        q2 = m.mate_rope_axes(Q, pos, f, axes)
    side.synchronize()
    assert torch.equal(q, q2)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.graph(graph):
        m.mate_rope_axes(Q, pos, f, axes, out=out)
    pos += 7
    graph.replay()
    assert torch.equal(out, m.mate_rope_axes(Q, pos, f, axes))
    # in place through the views, what is not theirs stays; the gradient turns back
    other, before = qkv[:, :, H + Hk:].clone(), qkv.clone()
    m.mate_rope_axes(Q, pos, f, axes, K=K, out=(Q, K))
    assert torch.equal(qkv[:, :, H + Hk:], other)
    m.mate_rope_axes(Q, pos, f, axes, K=K, out=(Q, K), backward=True)
    # (two roundings to the type, each half a step of values of up to 6, and the two turns' own)
    assert (qkv - before).abs().max().item() <= 2 * (6 * 2.0 ** -8 if dtype == "bf16" else 0) + 4 * 6e-7 * 2 * before.abs().max().item()
    assert m.mate_rope_axes(Q[:, :, :0], pos[:, :, :0].contiguous(), f, axes).shape == (B, H, 0, d)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_backward_against_differences(interleaved):
    # the operator is linear: <dy, rope(x + e) - rope(x)> = <rope^T dy, e> up to rounding, for every single element
    import paper_2109_04312_b200 as m
    N, d, A = 3, 16, 3
    g = torch.Generator().manual_seed(0)
    x, dy = (torch.randn(1, 1, N, d, generator=g).cuda() for _ in range(2))
    pos, f, axes = torch.randint(0, 300, (A, N), generator=g, dtype=torch.int32).cuda(), m.mate_rope_freqs(12), some_axes("mixed", 6, A)
    dx = m.mate_rope_axes(dy, pos, f, axes, interleaved=interleaved, backward=True)
    y0 = m.mate_rope_axes(x, pos, f, axes, interleaved=interleaved).double()
    for i in range(N * d):
        e = torch.zeros_like(x)
        e.view(-1)[i] = 1.0
        diff = m.mate_rope_axes(x + e, pos, f, axes, interleaved=interleaved).double() - y0
        # (each y is off by up to 6e-7 of 2 max |x + e|, x + e by 2^-24 of itself: 16 elements, of which two differ, times |dy|)
        assert abs((dy.double() * diff).sum().item() - dx.view(-1)[i].item()) <= 2 * 4 * 7e-7 * 2 * 5 * dy.abs().max().item()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,rot,N", [(64, 64, 1), (128, 64, 1), (48, 16, 5), (40, 20, 3)])
def test_append_axes(d, rot, N, dtype):
    # what mate_rope_axes and mate_cache_append do one after the other, bit for bit
    import paper_2109_04312_b200 as m
    B, H, Hk, ps, A = 3, 4, 2, 4, 3
    f, axes = m.mate_rope_freqs(rot), some_axes("any", rot // 2, A)
    caches = [m.Cache.empty(12, ps, Hk, d, 4, 4, [0, 1] * 2, dtype=DT[dtype], layers=2) for _ in range(2)]
    seqs = torch.tensor([2, 0, 3], dtype=torch.int32, device="cuda")
    counts = torch.tensor([N, max(N - 1, 0), N], dtype=torch.int32, device="cuda")
    Q, K, V = (torch.randn(B, N, h, d, device="cuda").to(DT[dtype]).transpose(1, 2) for h in (H, Hk, Hk))
    pos = torch.randint(0, 3000, (A, B, N), dtype=torch.int32, device="cuda")
    ids = torch.randint(0, 9, (2, B, N), dtype=torch.int32, device="cuda")
    for c in caches:
        m.mate_cache_extend(c, seqs, counts + 5)
    q = m.mate_cache_append_axes(caches[0], K, V, f, pos, axes, seqs=seqs, counts=counts, row_ids=ids[0], col_ids=ids[1], layer=1, Q=Q)
    q2, k2 = m.mate_rope_axes(Q, pos, f, axes, K=K)
    m.mate_cache_append(caches[1], k2, V, seqs, counts, ids[0], ids[1], layer=1)
    assert torch.equal(q, q2)
    for a, b in zip((caches[0].k, caches[0].v, caches[0].row_ids, caches[0].col_ids), (caches[1].k, caches[1].v, caches[1].row_ids, caches[1].col_ids)):
        assert torch.equal(a, b)
    assert m.mate_cache_append_axes(caches[0], K, V, f, pos, axes, seqs=seqs, counts=counts) is None
    assert torch.equal(caches[0].k[0], caches[1].k[1])
    for c in caches:
        c.status()


@pytest.mark.gpu
def test_refusals():
    import paper_2109_04312_b200 as m
    Q, f = torch.zeros(1, 2, 3, 16, device="cuda"), m.mate_rope_freqs(16)
    pos, axes = torch.zeros(2, 1, 3, dtype=torch.int32, device="cuda"), [0, 1] * 4
    for what, call in (("positions", lambda: m.mate_rope_axes(Q, pos[0, 0], f, axes)), ("positions", lambda: m.mate_rope_axes(Q, pos.long(), f, axes)),
                       ("positions", lambda: m.mate_rope_axes(Q, pos[:, :, :2].contiguous(), f, axes)),
                       ("positions", lambda: m.mate_rope_axes(Q, pos.cpu(), f, axes)), ("positions", lambda: m.mate_rope_axes(Q, None, f, axes)),
                       ("axes", lambda: m.mate_rope_axes(Q, pos, f, axes[:7])), ("axes", lambda: m.mate_rope_axes(Q, pos, f, [0.5] * 8)),
                       ("axes", lambda: m.mate_rope_axes(Q, pos, f, [-1] * 8)), ("axes", lambda: m.mate_rope_axes(Q, pos, f, [256] * 8)),
                       ("out", lambda: m.mate_rope_axes(Q, pos, f, axes, K=Q, out=Q))):
        with pytest.raises(ValueError, match="^%s must be" % what):
            call()
    with pytest.raises(m.MateError, match="invalid argument"):
        m.mate_rope_axes(Q, pos, f, [0, 2] * 4)                       # no such axis
    with pytest.raises(m.MateError, match="unsupported|not available"):
        m.mate_rope_axes(Q, pos.repeat(3, 1, 1), f, axes)             # six axes
    c = m.Cache.empty(4, 4, 2, 16, 2, 2, [0, 1], dtype=torch.float32)
    K = torch.zeros(1, 2, 3, 16, device="cuda")
    for what, call in (("positions", lambda: m.mate_cache_append_axes(c, K, K, f, pos[0], axes)), ("axes", lambda: m.mate_cache_append_axes(c, K, K, f, pos, [0])),
                       ("freqs", lambda: m.mate_cache_append_axes(c, K, K, None, pos, axes))):
        with pytest.raises(ValueError, match="^%s must be" % what):
            call()
    with pytest.raises(m.MateError, match="invalid argument"):
        m.mate_cache_append_axes(c, K, K, f, pos, [3] * 8)


def test_refusals_without_a_gpu():
    import paper_2109_04312_b200 as m
    Q, pos, f = torch.zeros(1, 2, 3, 16), torch.zeros(2, 1, 3, dtype=torch.int32), m.mate_rope_freqs(16, device="cpu")
    for what, axes in (("axes", ["0"] * 8), ("axes", [[0, 1]] * 4), ("axes", [300] * 8), ("Q", [0, 1] * 4)):
        with pytest.raises(ValueError, match="^%s must be" % what):
            m.mate_rope_axes(Q, pos, f, axes)


def test_the_c_entry_refuses_before_anything_is_launched():
    from paper_2109_04312_b200 import build
    lib = ctypes.CDLL(build.build())
    P = ctypes.c_void_p
    buf = ctypes.create_string_buffer(4096)
    at = ctypes.addressof(buf) + 15 & ~15

    class Tensor(ctypes.Structure):
        _fields_ = [("x", P), ("y", P), ("xs", ctypes.c_int64 * 3), ("ys", ctypes.c_int64 * 3), ("heads", ctypes.c_int32)]

    def call(x=at, n=1, B=1, N=1, d=16, dtype=1, pos=at, axes=bytes([0, 1] * 4), n_axes=2, freqs=at, rot=16, flags=0):
        t = Tensor(x, at, (0, 16, 16), (0, 16, 16), 1)
        return lib.mate_rope_axes(ctypes.byref(t), n, B, N, d, dtype, P(pos), ctypes.c_int64(1), ctypes.c_int64(1), axes, n_axes, P(freqs), rot,
                                  ctypes.c_float(1), flags, None)

    for kw in (dict(x=None), dict(n=3), dict(B=-1), dict(N=-1), dict(d=0), dict(pos=None), dict(axes=None), dict(axes=bytes([0, 2] * 4)), dict(n_axes=0),
               dict(n_axes=1), dict(freqs=None), dict(rot=18), dict(rot=3), dict(flags=4)):
        assert call(**kw) == -1, kw
    for kw in (dict(n_axes=5), dict(dtype=2), dict(d=1026)):
        assert call(**kw) == -2, kw
    assert call(x=at + 2) == -3
