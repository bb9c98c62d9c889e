"""mate_rope against the formula in 64 bits, its backward against the formula's transpose and against differences."""
import ctypes

import numpy as np
import pytest
import torch

from tests.cache_model import turn

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def bound(x, want, dtype, mscale=1.0):
    # Angle: the fraction of a turn is rounded to fp32 once (2^-25 of at most half a turn, 1e-7 rad); sine and cosine are good to
    # an ulp (1.2e-7), times mscale (2^-24); two products and a sum (3 x 2^-24).  Together below 6e-7 of |a| + |b|, which is at most
    # 2 max |x| here.  Stored in bf16: half a step of the value.
    err = 6e-7 * abs(mscale) * 2 * np.abs(x).max()
    return err + (np.abs(want) * 2.0 ** -8 if dtype == "bf16" else 0)


def check(got, x, pos, freqs, dtype, **kw):
    x64 = x.detach().double().cpu().numpy()
    p = pos.cpu().numpy()
    want = turn(x64, p if p.ndim == 1 or x.dim() == 3 else p[:, None], freqs.cpu().numpy(), kw.get("interleaved", False),
                kw.get("mscale", 1.0), kw.get("backward", False))
    got = got.double().cpu().numpy()
    assert got.shape == want.shape
    err = np.abs(got - want)
    assert np.all(err <= bound(x64, want, dtype, kw.get("mscale", 1.0))), err.max()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,H,Hk,N,d,rot", [(1, 1, 1, 1, 2, 2), (1, 4, 4, 1, 64, 64), (2, 3, 1, 17, 64, 32), (3, 5, 2, 33, 40, 20), (1, 2, 2, 5, 33, 6),
                                            (2, 12, 12, 130, 64, 64), (1, 32, 8, 47, 128, 128), (1, 1, 3, 19, 1024, 512),
                                            (1, 2, 1, 3, 1023, 1022), (2, 7, 1, 16, 128, 0), (1, 3, 2, 9, 48, 16), (2, 3, 2, 19, 80, 40),
                                            (1, 2, 3, 21, 24, 8), (3, 1, 1, 5, 128, 72)])
def test_rope(B, H, Hk, N, d, rot, interleaved, dtype):
    import paper_2109_04312_b200 as m
    g = torch.Generator().manual_seed(B * 1000 + d)
    Q, K = (torch.randn(B, h, N, d, generator=g).to(DT[dtype]).cuda() for h in (H, Hk))
    pos = torch.randint(-50, 100000, (B, N), generator=g, dtype=torch.int32).cuda()
    f = m.mate_rope_freqs(rot)
    for backward in (False, True):
        q, k = m.mate_rope(Q, pos, f, K=K, interleaved=interleaved, backward=backward, mscale=1.25)
        for got, x in ((q, Q), (k, K)):
            assert got.is_contiguous()
            check(got, x, pos, f, dtype, interleaved=interleaved, backward=backward, mscale=1.25)
    # alone, one row of positions for all examples
    check(m.mate_rope(Q, pos[0], f, interleaved=interleaved), Q, pos[0], f, dtype, interleaved=interleaved)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_in_and_out(dtype):
    import paper_2109_04312_b200 as m
    B, N, H, Hk, d = 2, 37, 6, 2, 64
    qkv = torch.randn(B, N, H + 2 * Hk, d, device="cuda").to(DT[dtype])
    Q, K = qkv[:, :, :H].transpose(1, 2), qkv[:, :, H:H + Hk].transpose(1, 2)
    pos, f = torch.arange(N, dtype=torch.int32, device="cuda"), m.mate_rope_freqs(d)
    q, k = m.mate_rope(Q, pos, f, K=K)
    check(q, Q, pos, f, dtype)
    check(k, K, pos, f, dtype)
    # in place, through the views; what is not theirs stays
    other, before = qkv[:, :, H + Hk:].clone(), qkv.clone()
    r = m.mate_rope(Q, pos, f, K=K, out=(Q, K))
    assert r[0] is Q and r[1] is K
    assert torch.equal(Q, q) and torch.equal(K, k) and torch.equal(qkv[:, :, H + Hk:], other)
    # rows at an odd distance: elements one by one, with the same results
    wide = torch.zeros(B, H, N, d + 1, device="cuda").to(DT[dtype])
    odd = wide[..., 1:]
    odd.copy_(before[:, :, :H].transpose(1, 2))
    out = torch.full((B, H, N, d + 3), float("nan"), device="cuda").to(DT[dtype])
    m.mate_rope(odd, pos, f, out=out[..., 2:2 + d])
    assert torch.equal(out[..., 2:2 + d], q) and out[..., :2].isnan().all() and out[..., 2 + d:].isnan().all()
    # one head for all (a stride of zero), packed
    one = torch.randn(1, N, d, device="cuda").to(DT[dtype])
    check(m.mate_rope(one.expand(5, N, d), pos, f), one.expand(5, N, d), pos, f, dtype)
    # nothing to do
    assert m.mate_rope(Q[:, :, :0], pos[:0], f).shape == (B, H, 0, d)
    e, k2 = m.mate_rope(Q[:, :0], pos, f, K=K.contiguous())
    assert e.shape == (B, 0, N, d) and k2.shape == K.shape


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_and_scaled_frequencies(interleaved):
    import paper_2109_04312_b200 as m
    d = 64
    f = m.mate_rope_freqs(d, factor=8.0, original_len=8192)
    plain = 10000.0 ** (-np.arange(0, d, 2) / d)
    got = f.cpu().numpy()
    turns = 8192 * plain / (2 * np.pi)
    assert np.allclose(got[turns >= 4], plain[turns >= 4], rtol=1e-14) and np.allclose(got[turns <= 1], plain[turns <= 1] / 8, rtol=1e-14)
    assert np.all(np.diff(got) < 0)
    pos = torch.tensor([0, 1, 131071, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    x = torch.randn(1, 2, len(pos), d, device="cuda")
    # (64-bit angles of 2^31 rad and their cosines in 64 bits are good to 2^31 x 2^-52 = 5e-7 on either side)
    want = turn(x.double().cpu().numpy(), pos.cpu().numpy(), got, interleaved)
    err = np.abs(m.mate_rope(x, pos, f, interleaved=interleaved).double().cpu().numpy() - want)
    assert err.max() <= bound(x.cpu().numpy(), want, "f32").max() + 2e-6 * x.abs().max().item()


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_backward_against_differences(interleaved):
    # the operator is linear: <dy, rope(x + e) - rope(x)> = <rope^T dy, e> up to rounding, for every single element
    import paper_2109_04312_b200 as m
    N, d = 3, 16
    f, pos = m.mate_rope_freqs(12), torch.tensor([1, 7, 1000], dtype=torch.int32, device="cuda")
    x, dy = torch.randn(1, 1, N, d, device="cuda"), torch.randn(1, 1, N, d, device="cuda")
    dx = m.mate_rope(dy, pos, f, interleaved=interleaved, mscale=0.7, backward=True).double()
    num = torch.zeros(N * d, dtype=torch.float64)
    for i in range(N * d):
        e = torch.zeros(N * d, device="cuda")
        e[i] = 0.5
        up, down = (m.mate_rope(x + s * e.view_as(x), pos, f, interleaved=interleaved, mscale=0.7).double() for s in (1, -1))
        num[i] = float(((up - down) * dy.double()).sum())
    # values up to about 4, each rounded (6e-7 of it) twice, two elements of them times |dy| <= 4
    assert (num - dx.view(-1).cpu()).abs().max() < 4 * 4 * 2 * 2 * 6e-7


@pytest.mark.gpu
def test_stream_and_graph():
    import paper_2109_04312_b200 as m
    Q = torch.randn(2, 4, 50, 64, device="cuda").bfloat16()
    pos, f = torch.arange(50, dtype=torch.int32, device="cuda"), m.mate_rope_freqs(64)
    want = m.mate_rope(Q, pos, f)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = m.mate_rope(Q, pos, f)
    side.synchronize()
    assert torch.equal(got, want)
    g, out = torch.cuda.CUDAGraph(), torch.empty_like(Q)
    with torch.cuda.graph(g):
        m.mate_rope(Q, pos, f, out=out)
    Q.mul_(2)
    pos.add_(3)
    g.replay()
    assert torch.equal(out, m.mate_rope(Q, pos, f))


def test_refusals_of_the_binding():
    import paper_2109_04312_b200 as m
    x, pos = torch.zeros(1, 2, 3, 8), torch.zeros(1, 3, dtype=torch.int32)
    f = torch.zeros(4, dtype=torch.float64)
    for bad in (x, x[0, 0], None):
        with pytest.raises(ValueError, match="^Q must be"):
            m.mate_rope(bad, pos, f)
    with pytest.raises(ValueError):
        m.mate_rope_freqs(3, device="cpu")
    with pytest.raises(ValueError):
        m.mate_rope_freqs(4, factor=0, device="cpu")


@pytest.mark.gpu
def test_refusals():
    import paper_2109_04312_b200 as m
    x, pos = torch.zeros(1, 2, 3, 8, device="cuda"), torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    f = m.mate_rope_freqs(8)
    for what, call in (("freqs", lambda: m.mate_rope(x, pos, f.float())), ("freqs", lambda: m.mate_rope(x, pos, m.mate_rope_freqs(10))),
                       ("freqs", lambda: m.mate_rope(x, pos, f.cpu())),
                       ("positions", lambda: m.mate_rope(x, pos.long(), f)), ("positions", lambda: m.mate_rope(x, pos[:, :2], f)),
                       ("positions", lambda: m.mate_rope(x, pos.cpu(), f)), ("K", lambda: m.mate_rope(x, pos, f, K=x[..., :4])),
                       ("K", lambda: m.mate_rope(x, pos, f, K=x.bfloat16())), ("out", lambda: m.mate_rope(x, pos, f, out=x[:, :1])),
                       ("out", lambda: m.mate_rope(x, pos, f, out=x[:, :1].expand(1, 2, 3, 8))), ("Q", lambda: m.mate_rope(x.transpose(2, 3), pos, f))):
        with pytest.raises(ValueError, match="^%s must be" % what):
            call()
    with pytest.raises(TypeError):
        m.mate_rope(x.half(), pos, f)
    with pytest.raises(ValueError, match="pair"):
        m.mate_rope(x, pos, f, K=x, out=torch.zeros(2, 1, 2, 3, 8, device="cuda"))
    with pytest.raises(m.MateError):
        m.mate_rope(torch.zeros(1, 1, 3, 1026, device="cuda"), pos, f)


def test_the_c_entry_refuses_before_anything_is_launched():
    from paper_2109_04312_b200 import build

    class Tensor(ctypes.Structure):
        _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("xs", ctypes.c_int64 * 3), ("ys", ctypes.c_int64 * 3), ("heads", ctypes.c_int32)]

    lib = ctypes.CDLL(build.build())
    buf = (ctypes.c_char * 4096)()
    at = (ctypes.addressof(buf) + 15) & ~15

    def call(x=at, y=at, heads=2, n=1, B=1, N=3, d=8, dtype=1, pos=at, f=at, rot=8, flags=0, tensors=True):
        t = (Tensor * 2)(*[Tensor(x, y, (ctypes.c_int64 * 3)(0, 24, 8), (ctypes.c_int64 * 3)(0, 24, 8), heads) for _ in range(2)])
        return lib.mate_rope(t if tensors else None, n, B, N, d, dtype, ctypes.c_void_p(pos), ctypes.c_int64(0), ctypes.c_void_p(f), rot,
                             ctypes.c_float(1), flags, None)

    for kw in (dict(tensors=False), dict(x=0), dict(y=0), dict(heads=-1), dict(n=0), dict(n=3), dict(B=-1), dict(N=-1), dict(d=0), dict(rot=3),
               dict(rot=10), dict(rot=-2), dict(pos=0), dict(f=0), dict(flags=4)):
        assert call(**kw) == -1, kw
    for kw in (dict(dtype=2), dict(d=1025)):
        assert call(**kw) == -2, kw
    for kw in (dict(x=at + 2), dict(y=at + 1)):
        assert call(**kw) == -3, kw
    for kw in (dict(B=0), dict(N=0), dict(heads=0)):
        assert call(**kw) == 0, kw


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,N", [(65535, 2, 1), (65536, 1, 1), (70000, 66000, 1), (140001, 3, 2)])
def test_more_heads_than_a_launch_has_rows_of_blocks(H, Hk, N, dtype):
    # examples folded into the heads
    import paper_2109_04312_b200 as m
    g = torch.Generator().manual_seed(H)
    Q, K = (torch.randn(h, N, 8, generator=g).to(DT[dtype]).cuda() for h in (H, Hk))
    pos, f = torch.arange(N, dtype=torch.int32, device="cuda") + 5, m.mate_rope_freqs(8)
    q, k = m.mate_rope(Q, pos, f, K=K)
    check(q, Q, pos, f, dtype)
    check(k, K, pos, f, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("backward", [False, True])
def test_the_angle_keeps_more_bits_than_fp32(interleaved, backward):
    # rows of (1, 0) and (0, 1): what comes out is the cosine and the sine themselves.  sincospif is good to an ulp, 2^-24 for values below
    # 1; what is added to it is rounded with it once, 2^-25; the 32-bit fraction of a turn is cut off by at most pi 2^-31 = 1.5e-9 rad, and the
    # 64-bit angle on either side (1e5 x 2^-52 rad) does not count.  The angle rounded to fp32 would be off by up to pi 2^-25 = 9.4e-8 rad more.
    import paper_2109_04312_b200 as m
    N, d = 20000, 64
    pos = torch.randint(0, 100000, (N,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    f = m.mate_rope_freqs(d)
    x = torch.zeros(1, 2, N, d, device="cuda")
    first = torch.arange(d, device="cuda") % 2 == 0 if interleaved else torch.arange(d, device="cuda") < d // 2
    x[:, 0, :, first], x[:, 1, :, ~first] = 1.0, 1.0
    got = m.mate_rope(x, pos, f, interleaved=interleaved, backward=backward).double().cpu().numpy()
    want = turn(x.double().cpu().numpy(), pos.cpu().numpy(), f.cpu().numpy(), interleaved, backward=backward)
    assert np.abs(got - want).max() <= 2.0 ** -24 + 2.0 ** -25 + 2e-9
