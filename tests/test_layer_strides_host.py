"""CPU tests of what the calls around the attention refuse in a tensor's strides before anything is launched."""
import pytest

from tests.test_layer_host import SHAPE, _norm, _rope, _window, _window_bwd


@pytest.mark.parametrize("n", [1 << 62, 1 << 61, (1 << 60) + (1 << 56), 1 << 32, 1 << 31])
def test_distances_of_rows_that_would_wrap(n):
    """Bytes of a head that are within 2^32 only as what is left of them in 64 bits."""
    assert _window("fwd", sq=(0, 0, n), B=1, Hq=2) == SHAPE
    assert _window("fwd", skv=(0, 0, n)) == SHAPE
    assert _window("fwd", so=(1 << 20, 1 << 14, n)) == SHAPE
    for name in ("dout", "q", "kv", "out", "dq", "dkv"):
        assert _window_bwd(s=((name, (1 << 20, 1 << 14, n)),)) == SHAPE


# b, h, n distances of [2, 3, 40, 64]: rows that meet, each distance by itself a row or more
MEETING = [(1 << 20, 64, 64), (64, 1 << 14, 64), (64, 64, 64), (64 * 40, 64 * 40, 64), (1 << 20, 128, 64), (1 << 20, 64 * 39, 64),
           (1 << 20, 64 * 12, 64 * 3), (1 << 20, 72, 128), (64 * 100, 64 * 40, 64), (1 << 20, 96, 64), (64 * 39, 64 * 82, 64)]


@pytest.mark.parametrize("s", MEETING)
def test_outputs_whose_rows_meet(s):
    import numpy as np

    start = np.sort((np.arange(2)[:, None, None] * s[0] + np.arange(3)[:, None] * s[1] + np.arange(40) * s[2]).ravel())
    assert np.diff(start).min() < 64  # it is so
    assert _window("fwd", B=2, Hq=3, Hkv=3, Nq=40, so=s) == SHAPE
    for name in ("dq", "dkv"):
        assert _window_bwd(B=2, Hq=3, Hkv=3, Nq=40, Nk=40, s=((name, s),)) == SHAPE
    assert _rope(B=2, Hq=3, k=None, ko=None, N=40, grid=(2, 4, 4), so=s) == SHAPE
    assert _norm("fwd", n=(2, 3, 40), sy=s) == SHAPE and _norm("bwd", n=(2, 3, 40), sy=s) == SHAPE


def test_layouts_that_would_take_long_to_look_through():
    """Three long axes of which no one holds the next."""
    assert _norm("fwd", n=(500, 500, 500), sy=(64 * 499, 64 * 501, 64 * 503)) == SHAPE
