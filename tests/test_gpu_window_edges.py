"""GPU tests of attention in a window and its gradients at the edges of what a call may be: every key a sink, frames longer
than all there is, empty batches, one key, gradients of broadcast inputs."""
import math

import numpy as np
import pytest

from tests.test_gpu_window import check_forward, check_grads, make, visible

pytestmark = pytest.mark.gpu

EDGES = [
    # B, Hq, Hkv, Nq, Nk, D, window, start, q_len, k_len
    (1, 4, 2, 300, 300, 128, dict(left=5, right=0, sinks=2 ** 31 - 1, frame=1), [0], [300], [300]),      # every key is a sink
    (2, 2, 2, 290, 513, 64, dict(left=0, right=0, sinks=513, frame=7), [223, 0], [290, 290], [513, 200]),
    (1, 2, 1, 150, 400, 64, dict(left=0, right=0, sinks=0, frame=2 ** 31 - 1), [250], [150], [400]),     # one frame holds all
    (1, 2, 1, 150, 400, 128, dict(left=2 ** 31 - 1, right=2 ** 31 - 1, sinks=9, frame=2 ** 31 - 1), [-20], [150], [390]),
    (3, 4, 1, 70, 90, 128, dict(left=-1, right=0, sinks=3, frame=1), [20, 20, 20], [0, 0, 0], [90, 90, 90]),  # nothing to ask
    (3, 4, 1, 70, 90, 64, dict(left=-1, right=0, sinks=3, frame=1), [20, 20, 20], [70, 70, 70], [0, 0, 0]),   # nothing to see
    (2, 3, 3, 1, 1, 128, dict(left=0, right=0, sinks=0, frame=1), [0, 1], [1, 1], [1, 1]),
    (1, 33, 1, 1, 700, 128, dict(left=-1, right=0, sinks=0, frame=1), [699], [1], [700]),                # a row more than shared ones
    (2, 16, 1, 5, 1100, 64, dict(left=300, right=0, sinks=5, frame=1), [1095, 500], [5, 2], [1100, 502]),
]


@pytest.mark.parametrize("B,Hq,Hkv,Nq,Nk,D,c,start,q_len,k_len", EDGES)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_edges(lib, B, Hq, Hkv, Nq, Nk, D, c, start, q_len, k_len, dtype):
    import torch

    print(f"edge {B} {Hq} {Hkv} {Nq} {Nk} {D} {c} {start} {q_len} {k_len} {dtype}", flush=True)
    rng = np.random.default_rng(Nq + Nk + D)
    q, k, v, dout = (make(rng, s, dtype) for s in ((B, Hq, Nq, D), (B, Hkv, Nk, D), (B, Hkv, Nk, D), (B, Hq, Nq, D)))
    see, scale, w = visible(c, B, Nq, Nk, start, q_len, k_len), 1 / math.sqrt(D), lib.Window(**c)
    at = dict(zip(("q_start", "q_len", "k_len"), (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (start, q_len, k_len))))
    out, lse = torch.full_like(q, 7.0), torch.full((B, Hq, Nq), 7.0, device="cuda")
    lib.window_attn_fwd(q, k, v, out, w, scale, lse=lse, **at)
    check_forward(out, lse, q, k, v, see, scale, dtype)
    check_grads(lib.window_attn_bwd(dout, q, k, v, out, lse, w, scale, **at), dout, q, k, v, see, scale, dtype)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_broadcast_inputs(lib, dtype):
    """q, k, v and dout that are the same for all heads or batch entries, as views: the bits of their copies."""
    import torch

    rng = np.random.default_rng(3)
    one = lambda h, n: make(rng, (1, h, n, 64), dtype)  # noqa: E731
    q, k, v, dout = one(4, 200).expand(3, 4, 200, 64), one(1, 260).expand(3, 2, 260, 64), one(1, 260).expand(3, 2, 260, 64), one(1, 200).expand(3, 4, 200, 64)
    w, lse = lib.Window(50, 3, 7, offset=60), torch.empty((3, 4, 200), device="cuda")
    out = torch.empty((3, 4, 200, 64), dtype=q.dtype, device="cuda")
    lib.window_attn_fwd(q, k, v, out, w, 0.125, lse=lse)
    copies = [t.contiguous() for t in (q, k, v, dout)]
    again, lse2 = torch.empty_like(out), torch.empty_like(lse)
    lib.window_attn_fwd(*copies[:3], again, w, 0.125, lse=lse2)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    grads = lib.window_attn_bwd(dout, q, k, v, out, lse, w, 0.125)
    want = lib.window_attn_bwd(copies[3], *copies[:3], out, lse, w, 0.125)
    assert all(torch.equal(a, b) for a, b in zip(grads, want))
    see = visible(dict(left=50, right=3, sinks=7, frame=1, offset=60), 3, 200, 260)
    check_grads(grads, copies[3], *copies[:3], see, 0.125, dtype)
