"""The axis of every pair, as mate_rope_axes and mate_cache_append_axes take it: a sequence of whole numbers and nothing else."""
import numpy as np
import pytest
import torch

N = 8
NO_SEQUENCE = [N, 0, True, np.int64(N), np.array(N), torch.tensor(N), {0: 1}, {0, 1}, None, "0" * N, 1.5, object()]
NO_WHOLE_NUMBERS = [[0.0] * N, np.zeros(N), ["0"] * N, [None] * N, [[0]] * N, np.zeros((N, 1), int), np.zeros((1, N), int), [-1] + [0] * (N - 1), [256] * N]


@pytest.mark.parametrize("axes", NO_SEQUENCE + NO_WHOLE_NUMBERS, ids=repr)
def test_what_is_refused(axes):
    # (ahead of everything else: the tensors are not looked at)
    import paper_2109_04312_b200 as m

    class Cached:
        class _native:
            cache_append_axes = None
        _info = None

    f = np.ones(N)
    with pytest.raises(ValueError, match="^axes must be whole numbers, one for each frequency"):
        m.mate_rope_axes(None, None, f, axes)
    with pytest.raises(ValueError, match="^axes must be whole numbers, one for each frequency"):
        m.mate_cache_append_axes(Cached, None, None, f, None, axes)


@pytest.mark.parametrize("kind", [list, tuple, bytes, np.array, torch.tensor, lambda x: np.array(x, np.uint8), bytearray, lambda x: [np.int64(i) for i in x]])
def test_what_is_taken(kind):
    from paper_2109_04312_b200 import api
    x = [i % 3 for i in range(N)]
    assert api._axes(kind(x)) == bytes(x)
    assert api._axes(range(4)) == bytes(range(4)) and api._axes([]) == b""


@pytest.mark.gpu
def test_a_number_of_pairs_is_not_their_axes():
    import paper_2109_04312_b200 as m
    Q, pos = torch.randn(1, 1, 5, 2 * N, device="cuda"), torch.arange(10, dtype=torch.int32, device="cuda").view(2, 1, 5)
    f = m.mate_rope_freqs(2 * N)
    for axes in (N, np.int64(N), np.array(N)):
        with pytest.raises(ValueError, match="^axes must be whole numbers"):
            m.mate_rope_axes(Q, pos, f, axes)
    assert m.mate_rope_axes(Q, pos, f, [0] * N).shape == Q.shape
