"""GPU tests of attention in a window with first tokens that stay visible, against the fp64 oracle.

Tolerances of the forward: the probabilities and the result are each rounded to the element type, half a step at most,
relative to the probability and to the value.  An output off by both is within half a step of sum_j p_j |v_j| and half a
step of itself; fp32 sums and exponentials add 2^-24 times the number of keys' logits, which is far below (counted as
2^-14 of sum_j p_j |v_j|: logits of up to 2^6 with 2^-24 each, 2^8 roundings in a row).  The log-sum-exp is fp32: logits
of up to 2^6 in log2 units, and sums of positive numbers, 2^-24 * (2^8 + |lse| 2^2)."""
import math

import numpy as np
import pytest

from oracle import layer

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _torch():
    import torch

    return torch


def make(rng, shape, dtype, gain=1.0):
    torch = _torch()
    return torch.from_numpy((gain * rng.standard_normal(shape)).astype(np.float32)).cuda().to(getattr(torch, dtype))


def laid_out(x, layout):
    """The same values in another memory layout, between rows of NaN."""
    torch = _torch()
    B, H, N, D = x.shape
    if layout == "packed":
        return x.clone()
    if layout == "bnhd":
        buf = torch.full((B, N + 3, H, D), float("nan"), dtype=x.dtype, device=x.device)
        view = buf[:, 1:N + 1].transpose(1, 2)
    else:  # one of three neighbours in a fused projection
        buf = torch.full((B, N + 2, 3, H, D), float("nan"), dtype=x.dtype, device=x.device)
        view = buf[:, 1:N + 1, 1].transpose(1, 2)
    view.copy_(x)
    return view


def f64(t):
    return t.double().cpu().numpy()


def visible(c, B, Nq, Nk, start=None, q_len=None, k_len=None):
    return np.stack([layer.window_visible(Nq, Nk, c["left"], c["right"], c["sinks"], c["frame"],
                                          c.get("offset", 0) if start is None else start[b],
                                          None if q_len is None else q_len[b], None if k_len is None else k_len[b])
                     for b in range(B)])


def check_forward(out, lse, q, k, v, see, scale, dtype):
    torch = _torch()
    half = 0.5 * torch.finfo(getattr(torch, dtype)).eps
    qs, ks, vs = f64(q), f64(k), f64(v)
    want, want_lse = layer.window_attention(qs, ks, vs, see, scale)
    size, _ = layer.window_attention(qs, ks, np.abs(vs), see, scale)
    got = f64(out)
    allowed = half * 1.01 * (np.abs(want) + size) + 2.0 ** -14 * size + 1e-7
    off = np.abs(got - want) / allowed
    assert np.isfinite(got).all() and off.max() <= 1.0, f"out: worst {off.max():.2f} of what is allowed"
    empty = ~np.isfinite(want_lse)
    assert (got[empty] == 0).all()
    if lse is not None:
        z = f64(lse)
        assert np.array_equal(np.isneginf(z), empty)
        off = np.abs(z - want_lse)[~empty] / (U * (2 ** 8 + 4 * np.abs(want_lse[~empty])))
        assert off.size == 0 or off.max() <= 1.0, f"lse: worst {off.max():.2f} of what is allowed"


# B, Hq, Hkv, Nq, Nk, D, window
CASES = [
    (1, 2, 2, 1, 1, 64, dict(left=0, right=0, sinks=0, frame=1)),
    (2, 4, 2, 130, 130, 128, dict(left=-1, right=0, sinks=0, frame=1)),
    (1, 3, 3, 300, 300, 128, dict(left=40, right=0, sinks=4, frame=1)),
    (1, 2, 1, 517, 517, 64, dict(left=60, right=13, sinks=70, frame=1)),
    (1, 2, 2, 6 * 77, 6 * 77, 128, dict(left=1, right=0, sinks=77, frame=77)),
    (2, 2, 2, 5 * 150, 5 * 150, 64, dict(left=1, right=1, sinks=33, frame=150)),
    (1, 1, 1, 1000, 1000, 128, dict(left=0, right=0, sinks=200, frame=1)),
    (1, 2, 2, 700, 700, 128, dict(left=-1, right=-1, sinks=0, frame=1)),
    (1, 2, 2, 260, 900, 128, dict(left=100, right=0, sinks=10, frame=1, offset=640)),
    (1, 2, 2, 260, 900, 64, dict(left=2, right=-1, sinks=0, frame=64, offset=300)),
    (1, 2, 2, 400, 200, 128, dict(left=30, right=0, sinks=0, frame=1, offset=-100)),  # queries before and behind all keys
    (1, 2, 2, 400, 200, 64, dict(left=3, right=1, sinks=6, frame=16, offset=-150)),
    (1, 40, 40, 129, 65, 128, dict(left=-1, right=-1, sinks=0, frame=1)),
    # few rows of queries: single tokens, shared key heads
    (3, 8, 2, 1, 700, 64, dict(left=256, right=0, sinks=4, frame=1, offset=699)),
    (2, 16, 2, 1, 5000, 128, dict(left=-1, right=0, sinks=0, frame=1, offset=4999)),
    (1, 4, 4, 1, 33, 128, dict(left=10, right=0, sinks=3, frame=1, offset=32)),
    (2, 8, 1, 4, 3001, 128, dict(left=1000, right=0, sinks=70, frame=1, offset=2997)),
    (1, 2, 2, 32, 2100, 64, dict(left=500, right=0, sinks=0, frame=7, offset=2068)),
    (1, 4, 2, 3, 900, 64, dict(left=5, right=0, sinks=0, frame=100, offset=-2)),
]


@pytest.mark.parametrize("B,Hq,Hkv,Nq,Nk,D,c", CASES)
@pytest.mark.parametrize("dtype,layout", [("bfloat16", "packed"), ("float16", "bnhd"), ("bfloat16", "fused")])
def test_window_forward(lib, B, Hq, Hkv, Nq, Nk, D, c, dtype, layout):
    torch = _torch()
    print(f"window {B} {Hq} {Hkv} {Nq} {Nk} {D} {c} {dtype} {layout}", flush=True)
    rng = np.random.default_rng(Nq + Nk)
    q, k, v = make(rng, (B, Hq, Nq, D), dtype, 1.5), make(rng, (B, Hkv, Nk, D), dtype, 1.5), make(rng, (B, Hkv, Nk, D), dtype)
    scale = 1 / math.sqrt(D)
    out, lse = laid_out(torch.full_like(q, 7.0), layout), torch.full((B, Hq, Nq), 7.0, device="cuda")
    w = lib.Window(**c)
    args = [laid_out(t, layout) for t in (q, k, v)]
    assert lib.window_attn_fwd(*args, out, w, scale, lse=lse) is out
    check_forward(out, lse, q, k, v, visible(c, B, Nq, Nk), scale, dtype)
    again = torch.empty_like(q)
    lib.window_attn_fwd(q, k, v, again, w, scale)
    assert torch.equal(again, out)  # the same bits whatever the layout, with and without lse


LENGTHS = [
    # B, Hq, Hkv, Nq, Nk, D, window, start, q_len, k_len
    (4, 2, 2, 300, 300, 128, dict(left=64, right=0, sinks=5, frame=1), [0, 0, 0, 0], [300, 0, 131, 1], [300, 0, 131, 1]),
    (3, 4, 2, 200, 640, 64, dict(left=2, right=1, sinks=40, frame=50), [440, 17, 0], [200, 128, 129], [640, 145, 3]),
    (3, 2, 1, 150, 400, 128, dict(left=-1, right=-1, sinks=0, frame=1), [0, 5, 9], [150, 150, 7], [0, 400, 399]),
    (5, 8, 2, 1, 4096, 128, dict(left=1023, right=0, sinks=16, frame=1), [4095, -1, 0, 999, 2500], [1, 0, 1, 1, 1], [4096, 0, 1, 1000, 2501]),
    (3, 4, 4, 3, 777, 64, dict(left=-1, right=0, sinks=0, frame=1), [774, 100, -5], [3, 2, 3], [777, 102, 777]),
    # lengths that are not lengths, positions beyond all measure
    (4, 2, 2, 130, 200, 64, dict(left=20, right=0, sinks=3, frame=1), [70, 2 ** 31 - 1, -(2 ** 31), 0], [1000, 130, 130, -7], [2 ** 31 - 1, 200, 200, 200]),
]


@pytest.mark.parametrize("B,Hq,Hkv,Nq,Nk,D,c,start,q_len,k_len", LENGTHS)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_window_forward_with_lengths(lib, B, Hq, Hkv, Nq, Nk, D, c, start, q_len, k_len, dtype):
    """Padded batches; behind a sequence's end, and where no query sees, there is NaN."""
    torch = _torch()
    print(f"lengths {B} {Nq} {Nk} {D} {c} {start} {q_len} {k_len} {dtype}", flush=True)
    rng = np.random.default_rng(B + Nk)
    q, k, v = make(rng, (B, Hq, Nq, D), dtype), make(rng, (B, Hkv, Nk, D), dtype), make(rng, (B, Hkv, Nk, D), dtype)
    see = visible(c, B, Nq, Nk, np.clip(start, -(2 ** 30), 2 ** 30), q_len, k_len)
    scale, nan = 0.11, float("nan")
    qn, kn, vn = q.clone(), k.clone(), v.clone()
    for b in range(B):
        qn[b, :, max(0, q_len[b]):] = nan
        unseen = torch.from_numpy(~see[b].any(0)).cuda()
        kn[b, :, unseen] = nan
        vn[b, :, unseen] = float("inf")
    at = [torch.tensor(np.array(x, dtype=np.int64).astype(np.int32), device="cuda") for x in (start, q_len, k_len)]
    out, lse = torch.full_like(q, 7.0), torch.full((B, Hq, Nq), 7.0, device="cuda")
    lib.window_attn_fwd(qn, kn, vn, out, lib.Window(**c), scale, lse=lse, q_start=at[0], q_len=at[1], k_len=at[2])
    check_forward(out, lse, q, k, v, see, scale, dtype)


# few blocks over many keys: cut along the keys
@pytest.mark.parametrize("B,Hq,Hkv,Nq,Nk,D,c,start,q_len,k_len", [
    (1, 2, 2, 100, 1700, 128, dict(left=-1, right=-1, sinks=0, frame=1), [0], [100], [1700]),
    (2, 2, 1, 33, 4099, 64, dict(left=3000, right=0, sinks=50, frame=1), [4066, 1500], [33, 32], [4099, 1532]),
    (1, 2, 2, 300, 2600, 128, dict(left=20, right=0, sinks=20, frame=100), [2300], [259], [2559]),
    (3, 1, 1, 64, 3500, 64, dict(left=-1, right=0, sinks=0, frame=1), [3436, 0, -7], [64, 0, 64], [3500, 3500, 1])])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_window_forward_of_few_blocks_over_many_keys(lib, B, Hq, Hkv, Nq, Nk, D, c, start, q_len, k_len, dtype):
    assert lib.Window(**c).workspace_bytes(B, Hq, Hkv, Nq, Nk, D)[0] > 0
    test_window_forward_with_lengths(lib, B, Hq, Hkv, Nq, Nk, D, c, start, q_len, k_len, dtype)


@pytest.mark.parametrize("case", [i for i, x in enumerate(CASES) if x[3] > 32] + [-1 - i for i, x in enumerate(LENGTHS) if x[3] > 32])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_window_forward_of_many_blocks(lib, case, dtype):
    """The same calls among so many copies of themselves that they fill the GPU: the oracle's values for the first, its bits
    for all others."""
    torch = _torch()
    B, Hq, Hkv, Nq, Nk, D, c = (CASES[case] if case >= 0 else LENGTHS[-1 - case])[:7]
    start, q_len, k_len = (None,) * 3 if case >= 0 else LENGTHS[-1 - case][7:]
    times = -(-600 // (B * Hq * -(-Nq // 32)))
    print(f"many blocks {times} x {B} {Hq} {Hkv} {Nq} {Nk} {D} {c} {start} {q_len} {k_len} {dtype}", flush=True)
    rng = np.random.default_rng(Nq + Nk + D)
    q, k, v = make(rng, (B, Hq, Nq, D), dtype, 1.5), make(rng, (B, Hkv, Nk, D), dtype, 1.5), make(rng, (B, Hkv, Nk, D), dtype)
    many = lambda t: t.repeat(times, *(1,) * (t.dim() - 1))  # noqa: E731
    lengths = {}
    if start is not None:
        for name, x in (("q_start", start), ("q_len", q_len), ("k_len", k_len)):
            lengths[name] = many(torch.tensor(np.array(x, dtype=np.int64).astype(np.int32), device="cuda"))
        start = np.clip(start, -(2 ** 30), 2 ** 30)
    out, lse = torch.full_like(many(q), 7.0), torch.full((B * times, Hq, Nq), 7.0, device="cuda")
    lib.window_attn_fwd(many(q), many(k), many(v), out, lib.Window(**c), 0.11, lse=lse, **lengths)
    check_forward(out[:B], lse[:B], q, k, v, visible(c, B, Nq, Nk, start, q_len, k_len), 0.11, dtype)
    assert torch.equal(out, many(out[:B])) and torch.equal(lse, many(lse[:B]))


@pytest.mark.parametrize("Nq", [1, 200])
@pytest.mark.parametrize("gain", [1.0, 30.0])
def test_window_large_logits_and_any_scale(lib, Nq, gain):
    """Rows that one key takes, negative and zero scales."""
    torch = _torch()
    rng = np.random.default_rng(3)
    q, k, v = (make(rng, (1, 2, n, 128), "bfloat16", g) for n, g in ((Nq, gain), (500, 1.0), (500, 1.0)))
    c = dict(left=300, right=0, sinks=9, frame=1, offset=500 - Nq)
    for scale in (1 / math.sqrt(128), -1 / math.sqrt(128), 0.0):
        out = torch.empty_like(q)
        lib.window_attn_fwd(q, k, v, out, lib.Window(**c), scale)
        half = 2.0 ** -8
        want, _ = layer.window_attention(f64(q), f64(k), f64(v), visible(c, 1, Nq, 500), scale)
        size, _ = layer.window_attention(f64(q), f64(k), np.abs(f64(v)), visible(c, 1, Nq, 500), scale)
        # logits of up to 30 * 128 / sqrt(128) * 4 = 2^10.4 in fp32: exponents off by 2^-24 * 2^11 * 2^2 from 128 products
        assert (np.abs(f64(out) - want) <= half * 1.01 * (np.abs(want) + size) + 2.0 ** -10 * size + 1e-7).all()


# ---- gradients ----------------------------------------------------------------------------------------------
def grad_bounds(dout, q, k, v, see, scale, half):
    """How far the gradients may be off.  P and dS are rounded to the element type (half a step of each, in every product),
    delta is taken from the rounded output (half a step of sum |dO| |O|, times P), the results are rounded, and fp32 sums and
    exponentials add 2^-14 of what they are sums of (2^8 roundings of 2^-24, logits of up to 2^6)."""
    G = q.shape[1] // k.shape[1]
    out, lse = layer.window_attention(q, k, v, see, scale)
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b in range(q.shape[0]):
        some = see[b].any(-1)
        for h in range(q.shape[1]):
            kk, vv = np.where(see[b].any(0)[:, None], k[b, h // G], 0.0), np.where(see[b].any(0)[:, None], v[b, h // G], 0.0)
            qq, do = np.where(some[:, None], q[b, h], 0.0), np.where(some[:, None], dout[b, h], 0.0)
            p = np.where(see[b], np.exp(np.where(see[b], qq @ kk.T * scale, 0.0) - np.where(some, lse[b, h], 0.0)[:, None]), 0.0)
            delta = (do * out[b, h]).sum(-1, keepdims=True)
            adelta = (np.abs(do) * np.abs(out[b, h])).sum(-1, keepdims=True)
            ds = p * (half * np.abs(do @ vv.T - delta) + half * adelta + 2.0 ** -14 * (np.abs(do) @ np.abs(vv).T + adelta))
            dq[b, h] = abs(scale) * ds @ np.abs(kk)
            dk[b, h // G] += abs(scale) * ds.T @ np.abs(qq)
            dv[b, h // G] += (half + 2.0 ** -14) * p.T @ np.abs(do)
    return dq, dk, dv


def check_grads(got, dout, q, k, v, see, scale, dtype):
    torch = _torch()
    half = 0.5 * torch.finfo(getattr(torch, dtype)).eps * 1.01
    args = [f64(t) for t in (dout, q, k, v)]
    want, bounds = layer.window_attention_grads(*args, see, scale), grad_bounds(*args, see, scale, half)
    for name, g, w, bound in zip(("dq", "dk", "dv"), got, want, bounds):
        g = f64(g)
        assert np.isfinite(g).all(), name
        off = np.abs(g - w) / (half * np.abs(w) + bound + 1e-7)
        assert off.max() <= 1.0, f"{name}: worst {off.max():.2f} of what is allowed"
        assert (g[bound == 0] == 0).all(), name  # nothing seen: exactly zero


GRAD_CASES = CASES + [
    # enough heads, or keys, for the wide blocks of either kernel
    (1, 64, 64, 1030, 1030, 64, dict(left=100, right=0, sinks=5, frame=1)),
    (1, 40, 40, 1801, 1801, 128, dict(left=1, right=0, sinks=300, frame=225)),
    (2, 64, 32, 300, 530, 128, dict(left=-1, right=0, sinks=0, frame=1, offset=230)),
    # a few sinks and many queries: their block's queries are cut
    (1, 2, 1, 6000, 6000, 64, dict(left=64, right=0, sinks=4, frame=1)),
]


@pytest.mark.parametrize("B,Hq,Hkv,Nq,Nk,D,c", GRAD_CASES)
@pytest.mark.parametrize("dtype,layout", [("bfloat16", "bnhd"), ("float16", "packed")])
def test_window_gradients(lib, B, Hq, Hkv, Nq, Nk, D, c, dtype, layout):
    torch = _torch()
    print(f"grads {B} {Hq} {Hkv} {Nq} {Nk} {D} {c} {dtype} {layout}", flush=True)
    rng = np.random.default_rng(Nq + 2 * Nk)
    q, k, v, dout = (make(rng, s, dtype) for s in ((B, Hq, Nq, D), (B, Hkv, Nk, D), (B, Hkv, Nk, D), (B, Hq, Nq, D)))
    scale, w = 1 / math.sqrt(D), lib.Window(**c)
    qv, kv, vv, dv_ = (laid_out(t, layout) for t in (q, k, v, dout))
    out, lse = laid_out(torch.empty_like(q), layout), torch.empty((B, Hq, Nq), device="cuda")
    lib.window_attn_fwd(qv, kv, vv, out, w, scale, lse=lse)
    got = lib.window_attn_bwd(dv_, qv, kv, vv, out, lse, w, scale)
    if Hq * Nq * Nk < 3e7 or Hq == 2:
        check_grads(got, dout, q, k, v, visible(c, B, Nq, Nk), scale, dtype)
    else:  # the oracle on some of the heads
        at = [0, Hq // 2, Hq - 1]
        G = Hq // Hkv
        for h in at:
            hk = h // G
            heads = slice(hk * G, hk * G + G)
            check_grads((got[0][:, heads], got[1][:, hk:hk + 1], got[2][:, hk:hk + 1]), dout[:, heads], q[:, heads],
                        k[:, hk:hk + 1], v[:, hk:hk + 1], visible(c, B, Nq, Nk), scale, dtype)
    # given tensors of another layout, rows around them untouched; the same bits again
    dq = laid_out(torch.full_like(q, 7.0), layout)
    whole = torch.full((2, B, Nk + 2, Hkv, D), float("nan"), dtype=q.dtype, device="cuda")
    dk, dv = (x[:, 1:Nk + 1].transpose(1, 2) for x in whole)
    again = lib.window_attn_bwd(dout, q, k, v, out.contiguous(), lse, w, scale, dq=dq, dk=dk, dv=dv)
    assert again[0] is dq and all(torch.equal(a, g) for a, g in zip(again, got))
    assert torch.isnan(whole[:, :, 0]).all() and torch.isnan(whole[:, :, -1]).all()


@pytest.mark.parametrize("B,Hq,Hkv,Nq,Nk,D,c,start,q_len,k_len", LENGTHS)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_window_gradients_with_lengths(lib, B, Hq, Hkv, Nq, Nk, D, c, start, q_len, k_len, dtype):
    """Padded batches: NaN in all rows that are not there or meet nothing, dout's among them."""
    torch = _torch()
    print(f"grads, lengths {B} {Nq} {Nk} {D} {c} {start} {q_len} {k_len} {dtype}", flush=True)
    rng = np.random.default_rng(B + 3 * Nk)
    q, k, v, dout = (make(rng, s, dtype) for s in ((B, Hq, Nq, D), (B, Hkv, Nk, D), (B, Hkv, Nk, D), (B, Hq, Nq, D)))
    see = visible(c, B, Nq, Nk, np.clip(start, -(2 ** 30), 2 ** 30), q_len, k_len)
    qn, kn, vn, dn = q.clone(), k.clone(), v.clone(), dout.clone()
    for b in range(B):
        qn[b, :, max(0, q_len[b]):] = float("nan")
        dn[b, :, max(0, q_len[b]):] = float("nan")
        unseen = torch.from_numpy(~see[b].any(0)).cuda()
        past = torch.arange(Nk, device="cuda") >= k_len[b]
        kn[b, :, unseen & past], vn[b, :, unseen & past] = float("nan"), float("nan")
    at = dict(zip(("q_start", "q_len", "k_len"), (torch.tensor(np.array(x, dtype=np.int64).astype(np.int32), device="cuda") for x in (start, q_len, k_len))))
    out, lse, w = torch.empty_like(q), torch.empty((B, Hq, Nq), device="cuda"), lib.Window(**c)
    lib.window_attn_fwd(qn, kn, vn, out, w, 0.11, lse=lse, **at)
    got = lib.window_attn_bwd(dn, qn, kn, vn, out, lse, w, 0.11, **at)
    check_grads(got, dout, q, k, v, see, 0.11, dtype)


def test_window_gradient_against_differences(lib):
    """Directional differences of the fp64 forward at the library's inputs; and the oracle's gradients against them."""
    rng = np.random.default_rng(9)
    c, scale = dict(left=20, right=3, sinks=4, frame=1), 0.2
    q, k, v, dout = (make(rng, s, "float16", 0.7) for s in ((1, 4, 90, 64), (1, 2, 90, 64), (1, 2, 90, 64), (1, 4, 90, 64)))
    torch = _torch()
    out, lse, w = torch.empty_like(q), torch.empty((1, 4, 90), device="cuda"), lib.Window(**c)
    lib.window_attn_fwd(q, k, v, out, w, scale, lse=lse)
    grads = lib.window_attn_bwd(dout, q, k, v, out, lse, w, scale)
    see, args = visible(c, 1, 90, 90), [f64(t) for t in (q, k, v)]
    exact = layer.window_attention_grads(f64(dout), *args, see, scale)
    f = lambda a: (layer.window_attention(*a, see, scale)[0] * f64(dout)).sum()  # noqa: E731
    for i in range(3):
        u, step = rng.standard_normal(args[i].shape), 1e-5
        up, dn = list(args), list(args)
        up[i], dn[i] = up[i] + step * u, dn[i] - step * u
        slope = (f(up) - f(dn)) / (2 * step)
        assert abs(slope - (exact[i] * u).sum()) <= 1e-5 * max(1.0, abs(slope))
        # 2^-11 of every term, as in grad_bounds, three roundings deep, over independent terms
        assert abs(slope - (f64(grads[i]) * u).sum()) <= 4 * 2.0 ** -11 * np.sqrt((exact[i] ** 2 * u ** 2).sum()) * 8 + 1e-3


def test_window_gradient_refusals(lib):
    torch = _torch()
    q, k = torch.zeros((1, 2, 64, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 2, 96, 64), dtype=torch.bfloat16, device="cuda")
    v, dout, out, lse, w = torch.zeros_like(k), torch.zeros_like(q), torch.zeros_like(q), torch.zeros((1, 2, 64), device="cuda"), lib.Window(4)
    f = lib.window_attn_bwd
    for call in (lambda: f(dout.half(), q, k, v, out, lse, w, 1.0), lambda: f(dout, q, k, v, out, lse.half(), w, 1.0),
                 lambda: f(dout, q, k, v, out[:, :1], lse, w, 1.0), lambda: f(dout, q, k, v, out, lse, w, 1.0, dk=torch.zeros_like(k)),
                 lambda: f(dout, q, k, v, out, lse, w, 1.0, dk=torch.zeros_like(q), dv=torch.zeros_like(q)),
                 lambda: f(dout, q, k, v, out, lse, w, 1.0, dq=torch.zeros_like(k))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: f(dout, q, k, v, out, lse, w, 1.0, dq=q), lambda: f(dout, q, k, v, out, lse, w, 1.0, dk=k, dv=torch.zeros_like(k)),
                 lambda: f(dout, q, k, v, out, lse, w, math.nan), lambda: f(dout, q, k, v, out, lse, lib.Window(-5), 1.0)):
        with pytest.raises(lib.CalibattError):
            call()
    dk = torch.zeros_like(k)
    with pytest.raises(lib.CalibattError):
        f(dout, q, k, v, out, lse, w, 1.0, dk=dk, dv=dk)
    torch.cuda.synchronize()


def test_window_refusals(lib):
    torch = _torch()
    q = torch.zeros((2, 4, 64, 64), dtype=torch.bfloat16, device="cuda")
    k, out, w = torch.zeros((2, 2, 96, 64), dtype=torch.bfloat16, device="cuda"), torch.empty_like(q), lib.Window(4)
    one = torch.zeros(2, dtype=torch.int32, device="cuda")
    f = lib.window_attn_fwd
    for call in (lambda: f(q.float(), k, k, out, w, 1.0), lambda: f(q, k.half(), k, out, w, 1.0), lambda: f(q, k, k[:, :, :64], out, w, 1.0),
                 lambda: f(q, k, k.transpose(1, 2).contiguous().transpose(1, 2), out, w, 1.0), lambda: f(q[:, :3], k, k, out[:, :3], w, 1.0),
                 lambda: f(q, k[:1], k[:1], out, w, 1.0), lambda: f(q, k, k, out[:, :, :32], w, 1.0), lambda: f(q, k, k, out.half(), w, 1.0),
                 lambda: f(q, k, k, out, w, 1.0, lse=torch.zeros((2, 4, 64), device="cuda").half()),
                 lambda: f(q, k, k, out, w, 1.0, lse=torch.zeros((2, 64, 4), device="cuda").transpose(1, 2)),
                 lambda: f(q, k, k, out, w, 1.0, q_len=one.long()), lambda: f(q, k, k, out, w, 1.0, k_len=one[:1]),
                 lambda: f(q, k, k, out, w, 1.0, q_start=one.cpu()), lambda: f(q[0], k, k, out, w, 1.0), lambda: f(q.cpu(), k, k, out, w, 1.0)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: f(q, k, k, out, lib.Window(-2), 1.0), lambda: f(q, k, k, out, lib.Window(1, -2), 1.0),
                 lambda: f(q, k, k, out, lib.Window(1, sinks=-1), 1.0), lambda: f(q, k, k, out, lib.Window(1, frame=0), 1.0),
                 lambda: f(q, k, k, q, w, 1.0), lambda: f(q, k, k, out, w, math.inf), lambda: f(q, k, k, out, w, math.nan),
                 lambda: f(q[..., :32], k[..., :32], k[..., :32], out[..., :32], w, 1.0), lambda: f(q, k, k, out, lib.Window(1, offset=2 ** 30 + 1), 1.0),
                 lambda: f(q.expand(2, 4, 64, 64)[:, :, :1].expand(2, 4, 64, 64), k, k, out, w, 1.0)):
        with pytest.raises(lib.CalibattError):
            call()
    with pytest.raises(ValueError):
        lib.Window(2 ** 31)
    torch.cuda.synchronize()
