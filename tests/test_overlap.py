"""Outputs that share memory with inputs or with one another: the check itself against bytes counted one by one, and the calls that
refuse such outputs."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def overlap(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("overlap") / "overlap.so")
    subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2109_04312_b200", "csrc"),
                    "-o", so, os.path.join(ROOT, "tests", "overlap.cpp")], check=True)
    lib = ctypes.CDLL(so)

    def call(a, b):
        args = [(ctypes.c_int64 * (3 + 2 * len(dims)))(at, size, len(dims), *[x for d in dims for x in d]) for at, size, dims in (a, b)]
        return bool(lib.overlap_(*args))
    return call


def bytes_of(view):
    at, size, dims = view
    starts = np.array([at])
    for stride, n in dims:
        starts = (starts[:, None] + stride * np.arange(n)).reshape(-1)
    return {int(s) + i for s in starts for i in range(size)}


def test_against_bytes_counted_one_by_one(overlap):
    rng = np.random.default_rng(0)
    found = [0, 0]
    for trial in range(6000):
        views = []
        for _ in range(2):
            size = int(rng.choice([2, 4]))
            dims = [(int(rng.choice([0, 1, 2, 3, 5, 6, 8, 12, 24, 40])) * size, int(rng.integers(0, 5) if trial % 50 == 0 else rng.integers(1, 5)))
                    for _ in range(rng.integers(0, 5))]
            views.append((int(rng.integers(0, 300)) * 2, size, dims))
        want = bool(bytes_of(views[0]) & bytes_of(views[1]))
        found[want] += 1
        assert overlap(*views) == want == overlap(views[1], views[0]), views
    assert min(found) > 500   # (both answers are met)


def test_views_of_large_tensors(overlap):
    # parts of a fused projection [B, N, H + 2 Hk, d] in bf16, as [B, h, N, d]
    B, N, H, Hk, d = 64, 32768, 32, 8, 128
    row = (H + 2 * Hk) * d

    def part(first, heads, tokens=N, shift=0):
        return (2 * (first * d + shift), 2, [(2 * N * row, B), (2 * d, heads), (2 * row, tokens), (2, d)])
    assert not overlap(part(0, H), part(H, Hk)) and not overlap(part(H, Hk), part(H + Hk, Hk))
    assert overlap(part(0, H + 1), part(H, Hk)) and overlap(part(0, H), part(0, H)) and overlap(part(0, H, shift=1), part(H, Hk))
    # the same memory in another order, and next to it
    there = (0, 2, [(2 * N * H * d, B), (2 * d, H), (2 * H * d, N), (2, d)])
    assert overlap(there, (0, 2, [(2 * N * H * d, B), (2 * N * d, H), (2 * d, N), (2, d)]))
    assert not overlap(there, (2 * B * N * H * d, 2, [(2 * N * H * d, B), (2 * N * d, H), (2 * d, N), (2, d)]))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rope_refuses_outputs_that_overlap(dtype):
    import paper_2109_04312_b200 as m
    B, N, H, d = 2, 40, 3, 16
    pos, f = torch.arange(N, dtype=torch.int32, device="cuda"), m.mate_rope_freqs(d)
    flat = torch.randn(4 * B * H * N * d, device="cuda").to(dtype)
    at = lambda first: flat[first:first + B * H * N * d].view(B, H, N, d)  # noqa: E731
    Q, K, other = at(0), at(B * H * N * d), at(2 * B * H * N * d)
    before = flat.clone()
    for call in (lambda: m.mate_rope(Q, pos, f, out=at(d)), lambda: m.mate_rope(at(d), pos, f, out=Q),                  # shifted by a token
                 lambda: m.mate_rope(Q, pos, f, out=flat[:B * H * N * d].view(B, N, H, d).transpose(1, 2)),           # in another order
                 lambda: m.mate_rope(Q, pos, f, K=K, out=(other, other)), lambda: m.mate_rope(Q, pos, f, K=K, out=(K, Q)),
                 lambda: m.mate_rope(Q, pos, f, K=K, out=(K, other)), lambda: m.mate_rope(Q, pos, f, K=Q, out=(Q, other)),
                 lambda: m.mate_rope(Q, pos, f, K=K, out=(other, at(2 * B * H * N * d - d))), lambda: m.mate_rope(Q, pos, f, K=K, out=(None, Q))):
        with pytest.raises(ValueError, match="^out must be the inputs themselves"):
            call()
    torch.cuda.synchronize()
    assert torch.equal(flat, before)
    q, k = m.mate_rope(Q, pos, f, K=K)
    # what does not overlap goes through: Q and K in place, one of them only, next to one another, interleaved row by row
    two = torch.zeros(B, H, 2 * N, d, device="cuda").to(dtype)
    r = m.mate_rope(Q, pos, f, K=K, out=(two[:, :, 0::2], two[:, :, 1::2]))
    assert torch.equal(r[0], q) and torch.equal(r[1], k)
    assert torch.equal(m.mate_rope(Q, pos, f, K=K, out=(other, None))[0], q)
    assert torch.equal(m.mate_rope(Q, pos, f, K=Q, out=(other, at(3 * B * H * N * d)))[1], q)
    m.mate_rope(Q, pos, f, K=K, out=(Q, K))
    assert torch.equal(Q, q) and torch.equal(K, k)


@pytest.mark.gpu
def test_append_refuses_an_output_that_overlaps():
    import paper_2109_04312_b200 as m
    B, N, H, Hk, d = 3, 4, 4, 2, 16
    c, f = m.Cache.empty(9, 4, Hk, d, B, 2, [0, 1] * 2), m.mate_rope_freqs(d)
    m.mate_cache_extend(c, None, torch.full((B,), N, dtype=torch.int32, device="cuda"))
    flat = torch.randn(B, N, H + 2 * Hk + H, d, device="cuda").bfloat16()
    Q, K, V, other = (t.transpose(1, 2) for t in flat.split([H, Hk, Hk, H], 2))
    want = m.mate_cache_append(c, K, V, freqs=f, Q=Q).clone()
    before = flat.clone()
    for out in (flat[:, :, 1:H + 1].transpose(1, 2), flat[:, :, H:2 * H].transpose(1, 2), flat[:, :, H + 1:2 * H + 1].transpose(1, 2),
                flat[:, :, H + 2:2 * H + 2].transpose(1, 2)):
        with pytest.raises(ValueError, match="^out must be Q itself"):
            m.mate_cache_append(c, K, V, freqs=f, Q=Q, out=out)
    torch.cuda.synchronize()
    assert torch.equal(flat, before)
    for out in (other, Q):
        assert m.mate_cache_append(c, K, V, freqs=f, Q=Q, out=out) is out and torch.equal(out, want)
    assert torch.equal(flat[:, :, H:H + 2 * Hk], before[:, :, H:H + 2 * Hk])
    c.status()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_decode_refuses_outputs_that_overlap(dtype):
    import paper_2109_04312_b200 as m
    B, H, d = 5, 4, 16
    c = m.Cache.empty(9, 4, 2, d, B, 1, [0, 1] * 2, dtype=dtype)
    m.mate_cache_extend(c, None, torch.full((B,), 1, dtype=torch.int32, device="cuda"))
    c.v.normal_()
    text = torch.full((B,), m.ID_TEXT, dtype=torch.int32, device="cuda")
    flat = torch.randn(2 * B + 2, H, d, device="cuda").to(dtype)
    Q = flat[:B]
    want, lse = m.mate_attn_decode(c, Q, text, text)
    before = flat.clone()
    words = flat.view(-1).view(torch.float32)
    for out in (flat[1:B + 1], flat[B - 1:2 * B - 1]):
        with pytest.raises(ValueError, match="^O must be Q itself"):
            m.mate_attn_decode(c, Q, text, text, out=out)
    with pytest.raises(ValueError, match="^O must be Q itself"):                       # the same beginning, other strides
        m.mate_attn_decode(c, flat[:2 * B:2], text, text, out=flat[:B])
    with pytest.raises(ValueError, match="^LSE must be"):
        m.mate_attn_decode(c, Q, text, text, lse=words[7:7 + B * H].view(B, H))
    with pytest.raises(ValueError, match="^LSE must be"):
        m.mate_attn_decode(c, Q, text, text, out=flat[B:2 * B], lse=words[flat[:B + 1].numel() * flat.element_size() // 4:][:B * H].view(B, H))
    torch.cuda.synchronize()
    assert torch.equal(flat, before)
    # every other row is a query, the rows between are not touched
    o, l = m.mate_attn_decode(c, flat[:2 * B:2], text, text, out=torch.empty_like(want), lse=torch.empty_like(lse))
    assert torch.equal(flat, before)
    # next to one another, and in place
    o, l = m.mate_attn_decode(c, Q, text, text, out=flat[B:2 * B], lse=words[-B * H:].view(B, H))
    assert torch.equal(o, want) and torch.equal(l, lse)
    assert torch.equal(m.mate_attn_decode(c, Q, text, text, out=Q)[0], want)
    c.status()


def test_a_cache_refuses_keys_and_values_that_overlap():
    # (host tensors: what passes stops at the next check)
    import paper_2109_04312_b200 as m
    z = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    rest = [z(4, 4), z(4, 4), z(2, 3), z(2), z(2), z(4)]
    n = 4 * 2 * 4 * 16
    flat, both = torch.zeros(2 * n), torch.zeros(4, 2, 2, 4, 16)
    at = lambda first: flat[first:first + n].view(1, 4, 2, 4, 16)  # noqa: E731
    for k, v in ((at(0), at(0)), (at(0), at(16)), (at(n - 4), at(0)), (at(0), at(n - 128))):
        with pytest.raises(ValueError, match="^k and v must be laid out alike"):
            m.Cache(k, v, *rest, [0, 1])
    for k, v in ((at(0), at(n)), (at(n), at(0)), (both[None, :, 0], both[None, :, 1])):   # keys and values side by side in every page
        with pytest.raises(ValueError, match="CUDA"):
            m.Cache(k, v, *rest, [0, 1])
