"""GPU tests of fp16 gradients of attention in a window over the type's range: dO of a scaled loss, tiny ones, rows of very
different size, large and small V, against the fp64 oracle.

Tolerances: half a step (2^-11) of P, of dS, of the rounded out in delta, and of the results, and 2^-14 of what the fp32 sums
are sums of, as in test_gpu_window.grad_bounds.  What is small besides: fp16 values below its normal range are off by up to
2^-25, which is a result's last error, that of out in delta (2^-25 sum |dO|), that of P as it is kept, times 2^15 (2^-40), and
that of dS as it is kept, times a power of two F with |dS| F >= 2^14 where |dS| is as large as its bound 2 |dO| |V| (norms of
rows, the largest that meet anything): 2^-39 of the bound, of every visible pair."""
import math

import numpy as np
import pytest

from oracle import layer
from tests.test_gpu_window import f64, grad_bounds, make, visible

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -11 * 1.01


def small_bounds(dout, q, k, v, see, scale):
    """What is off because of values below the normal range, see above."""
    G = q.shape[1] // k.shape[1]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    norm = lambda x, some: np.sqrt((np.where(some[:, None], x, 0.0) ** 2).sum(-1))  # noqa: E731
    for b in range(q.shape[0]):
        some, keys, s = see[b].any(-1), see[b].any(0), see[b].astype(np.float64)
        for h in range(q.shape[1]):
            group = range(h // G * G, h // G * G + G)
            v_max, do_max = norm(v[b, h // G], keys).max(), max(norm(dout[b, g], some).max() for g in group)
            of_out = 2.0 ** -25 * np.abs(dout[b, h]).sum(-1)
            pairs_q = (2.0 ** -39 * 2 * norm(dout[b, h], some) * v_max + of_out)[:, None] * s
            pairs_k = (2.0 ** -39 * 2 * do_max * v_max + of_out)[:, None] * s
            dq[b, h] = abs(scale) * pairs_q @ np.abs(k[b, h // G])
            dk[b, h // G] += abs(scale) * pairs_k.T @ np.abs(q[b, h])
            dv[b, h // G] += 2.0 ** -40 * s.T @ np.abs(dout[b, h])
    return [x + 2.0 ** -25 for x in (dq, dk, dv)]


def check(got, dout, q, k, v, see, scale):
    args = [f64(t) for t in (dout, q, k, v)]
    want = layer.window_attention_grads(*args, see, scale)
    for name, g, w, bound, small in zip(("dq", "dk", "dv"), got, want, grad_bounds(*args, see, scale, HALF), small_bounds(*args, see, scale)):
        allowed, g = HALF * np.abs(w) + bound + small, f64(g)
        inside = np.abs(w) + allowed < 65504.0  # what fp16 can say
        assert inside.mean() > 0.99, name
        off = np.where(inside, np.abs(g - w) / allowed, 0.0)
        assert np.isfinite(g[inside]).all() and off.max() <= 1.0, f"{name}: worst {off.max():.2f} of what is allowed"


CASES = [
    # B, Hq, Hkv, Nq, Nk, D, window
    (2, 4, 2, 200, 200, 128, dict(left=-1, right=0, sinks=0, frame=1)),
    (1, 2, 2, 330, 330, 64, dict(left=60, right=5, sinks=9, frame=1)),
    (1, 4, 1, 2, 900, 128, dict(left=-1, right=0, sinks=0, frame=1, offset=898)),
    (1, 2, 1, 2100, 2100, 64, dict(left=300, right=0, sinks=4, frame=1)),   # sums of parts
    (1, 1, 1, 5, 2, 128, dict(left=1, right=0, sinks=0, frame=1)),          # two keys: dS as large as it gets
]


@pytest.mark.parametrize("B,Hq,Hkv,Nq,Nk,D,c", CASES)
@pytest.mark.parametrize("do_gain,v_gain,uneven", [
    (2.0 ** 11, 1.0, False), (2.0 ** 8, 1.0, False), (2.0 ** 8, 2.0 ** 5, False), (2.0 ** -8, 1.0, False), (2.0 ** -14, 1.0, False),
    (2.0 ** -4, 2.0 ** -6, False), (1.0, 1.0, True), (2.0 ** 3, 2.0 ** -3, True)])
def test_f16_gradients_over_the_range(lib, B, Hq, Hkv, Nq, Nk, D, c, do_gain, v_gain, uneven):
    import torch

    print(f"fp16 range {B} {Hq} {Hkv} {Nq} {Nk} {D} {c} {do_gain} {v_gain} {uneven}", flush=True)
    rng = np.random.default_rng(Nq + D)
    q, k = make(rng, (B, Hq, Nq, D), "float16"), make(rng, (B, Hkv, Nk, D), "float16")
    v, dout = make(rng, (B, Hkv, Nk, D), "float16", v_gain), make(rng, (B, Hq, Nq, D), "float32", do_gain)
    if uneven:  # one row in seven 2^8 times the others
        dout[:, :, ::7] *= 2.0 ** 8
    dout = dout.half()
    scale, w = 1 / math.sqrt(D), lib.Window(**c)
    out, lse = torch.empty_like(q), torch.empty((B, Hq, Nq), device="cuda")
    lib.window_attn_fwd(q, k, v, out, w, scale, lse=lse)
    check(lib.window_attn_bwd(dout, q, k, v, out, lse, w, scale), dout, q, k, v, visible(c, B, Nq, Nk), scale)


@pytest.mark.parametrize("D", [64, 128])
def test_rows_that_meet_nothing_have_no_say(lib, D):
    """Huge, infinite and NaN rows of V and dO that meet nothing leave every bit as it is; an infinite row of dO
    that meets keys spoils their gradients and its own, and no other query's and no other key head's."""
    import torch

    rng = np.random.default_rng(D)
    B, Hq, Hkv, N = 2, 4, 2, 300
    q, k, v, dout = (make(rng, (B, h, N, D), "float16") for h in (Hq, Hkv, Hkv, Hq))
    start, q_len, k_len = [-20, 100], [300, 180], [280, 290]
    c = dict(left=16, right=2, sinks=0, frame=4)
    see = visible(c, B, N, N, start, q_len, k_len)
    at = dict(zip(("q_start", "q_len", "k_len"), (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (start, q_len, k_len))))
    w, scale = lib.Window(**c), 1 / math.sqrt(D)
    out, lse = torch.empty_like(q), torch.empty((B, Hq, N), device="cuda")
    lib.window_attn_fwd(q, k, v, out, w, scale, lse=lse, **at)
    want = lib.window_attn_bwd(dout, q, k, v, out, lse, w, scale, **at)
    check(want, dout, q, k, v, see, scale)
    for value in (65504.0, float("inf"), float("nan")):
        vn, dn = v.clone(), dout.clone()
        for b in range(B):
            vn[b, :, torch.from_numpy(~see[b].any(0)).cuda()] = value
            dn[b, :, torch.from_numpy(~see[b].any(1)).cuda()] = value
        assert all(torch.equal(a, g) for a, g in zip(lib.window_attn_bwd(dn, q, k, vn, out, lse, w, scale, **at), want)), value
    dn = dout.clone()
    dn[0, 0, 40] = float("inf")  # of key head 0
    got = lib.window_attn_bwd(dn, q, k, v, out, lse, w, scale, **at)
    assert all(torch.equal(a[1], g[1]) for a, g in zip(got, want))
    assert torch.equal(got[0][0, 1:], want[0][0, 1:]) and all(torch.equal(got[i][0, 1:], want[i][0, 1:]) for i in (1, 2))
    rows = torch.arange(N, device="cuda") != 40
    assert torch.equal(got[0][0, 0, rows], want[0][0, 0, rows])


def test_f16_gradients_in_a_graph_follow_their_inputs(lib):
    """A captured pass whose dO grows from replay to replay: the factors are those of the replay."""
    import torch

    rng = np.random.default_rng(7)
    q, k, v, dout = (make(rng, (1, 2, 260, 64), "float16") for _ in range(4))
    c, scale = dict(left=50, right=0, sinks=3), 0.125
    w, out, lse = lib.Window(**c), torch.empty_like(q), torch.empty((1, 2, 260), device="cuda")
    lib.window_attn_fwd(q, k, v, out, w, scale, lse=lse)
    lib.window_attn_bwd(dout, q, k, v, out, lse, w, scale)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = lib.window_attn_bwd(dout, q, k, v, out, lse, w, scale)
    base = dout.clone()
    for gain in (2.0 ** -6, 2.0 ** 10, 1.0):
        dout.copy_(base * gain)
        graph.replay()
        eager = lib.window_attn_bwd(dout, q, k, v, out, lse, w, scale)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager)), gain
        check(held, dout, q, k, v, visible(dict(c, frame=1), 1, 260, 260), scale)
