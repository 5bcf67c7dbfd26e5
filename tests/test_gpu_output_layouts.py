"""GPU tests of outputs in unusual layouts: rows that interleave without meeting get the bits of packed outputs, rows that meet
are refused and left as they were."""
import math

import numpy as np
import pytest

from tests.test_gpu_window import make

pytestmark = pytest.mark.gpu

B, H, N, D = 2, 3, 40, 64
# b, h, n distances
APART = [(64 * 120, 64 * 40, 64), (64, 64 * 80, 128), (64 * 3, 64, 64 * 6), (64 * 300, 64 * 41, 64 * 2), (64 * 41, 64 * 82, 64 * 2),
         (64 * 7, 64 * 2, 64 * 14)]
MEETING = [(1 << 14, 64, 64), (64, 1 << 12, 64), (64 * 100, 64 * 40, 64), (1 << 14, 96, 64)]


def rows_at(s):
    return (np.arange(B)[:, None, None] * s[0] + np.arange(H)[:, None] * s[1] + np.arange(N) * s[2]).ravel()


def output(like, s):
    import torch

    buf = torch.full((int(rows_at(s).max()) + D,), 7.0, dtype=like.dtype, device="cuda")
    return buf, buf.as_strided((B, H, N, D), (*s, 1))


@pytest.mark.parametrize("s", APART)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_rows_that_interleave(lib, s, dtype):
    import torch

    assert np.diff(np.sort(rows_at(s))).min() >= D  # so they do
    rng = np.random.default_rng(1)
    q, k, v, dout = (make(rng, (B, H, N, D), dtype) for _ in range(4))
    rope = lib.RotaryAxes((24, 20, 20), (2, 4, 5))
    window, scale, lse = lib.Window(9, 2, 3), 1 / math.sqrt(D), torch.empty((B, H, N), device="cuda")
    out = torch.empty_like(q)
    lib.window_attn_fwd(q, k, v, out, window, scale, lse=lse)
    grads = lib.window_attn_bwd(dout, q, k, v, out, lse, window, scale)
    calls = [(lambda y: lib.layer_norm_fwd(q, out=y), lib.layer_norm_fwd(q)),
             (lambda y: lib.layer_norm_bwd(dout, q, dx=y), lib.layer_norm_bwd(dout, q)[0]),
             (lambda y: lib.rope_axes(q, None, rope, grid=(2, 4, 5), q_out=y), lib.rope_axes(q, None, rope, grid=(2, 4, 5))[0]),
             (lambda y: lib.window_attn_fwd(q, k, v, y, window, scale), out),
             (lambda y: lib.window_attn_bwd(dout, q, k, v, out, lse, window, scale, dq=y), grads[0]),
             (lambda y: lib.window_attn_bwd(dout, q, k, v, out, lse, window, scale, dk=y, dv=output(y, s)[1]), grads[1])]
    between = np.ones(int(rows_at(s).max()) + D, bool)
    between[(rows_at(s)[:, None] + np.arange(D)).ravel()] = False
    for call, want in calls:
        buf, y = output(q, s)
        call(y)
        assert torch.equal(y, want)
        assert (buf[torch.from_numpy(between).cuda()] == 7.0).all()


@pytest.mark.parametrize("s", MEETING)
def test_rows_that_meet(lib, s):
    import torch

    assert np.diff(np.sort(rows_at(s))).min() < D
    x = torch.ones((B, H, N, D), dtype=torch.bfloat16, device="cuda")
    k, lse, window = x.clone(), torch.zeros((B, H, N), device="cuda"), lib.Window(9)
    out = torch.ones_like(x)
    rope = lib.RotaryAxes((24, 20, 20), (2, 4, 5))
    for call in (lambda y: lib.layer_norm_fwd(x, out=y), lambda y: lib.layer_norm_bwd(x, x, dx=y),
                 lambda y: lib.rope_axes(x, None, rope, grid=(2, 4, 5), q_out=y), lambda y: lib.window_attn_fwd(x, k, k, y, window, 1.0),
                 lambda y: lib.window_attn_bwd(x, x, k, k, out, lse, window, 1.0, dq=y),
                 lambda y: lib.window_attn_bwd(x, x, k, k, out, lse, window, 1.0, dk=y, dv=output(y, s)[1])):
        buf, y = output(x, s)
        with pytest.raises(lib.CalibattError):
            call(y)
        torch.cuda.synchronize()
        assert (buf == 7.0).all()
    # as inputs such rows are fine
    buf, y = output(x, s)
    assert torch.equal(lib.layer_norm_fwd(y, out=torch.empty_like(x)), lib.layer_norm_fwd(y.contiguous()))
