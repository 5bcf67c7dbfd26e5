"""CPU tests of what the calls around the attention refuse in a tensor's strides before anything is launched."""
import pytest

from tests.test_layer_host import SHAPE, _window, _window_bwd


@pytest.mark.parametrize("n", [1 << 62, 1 << 61, (1 << 60) + (1 << 56), 1 << 32, 1 << 31])
def test_distances_of_rows_that_would_wrap(n):
    """Bytes of a head that are within 2^32 only as what is left of them in 64 bits."""
    assert _window("fwd", sq=(0, 0, n), B=1, Hq=2) == SHAPE
    assert _window("fwd", skv=(0, 0, n)) == SHAPE
    assert _window("fwd", so=(1 << 20, 1 << 14, n)) == SHAPE
    for name in ("dout", "q", "kv", "out", "dq", "dkv"):
        assert _window_bwd(s=((name, (1 << 20, 1 << 14, n)),)) == SHAPE
