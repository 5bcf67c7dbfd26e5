"""GPU tests of rotary positions with several axes and of layer norm with its gradients, against the fp64 oracle.

Tolerances: half a step of the output's type relative to the value, plus what fp32 arithmetic may lose before that
(counted in roundings of 2^-24 where it is used)."""
import numpy as np
import pytest

from oracle import layer

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _torch():
    import torch

    return torch


def make(rng, shape, dtype, gain=1.0, shift=0.0):
    torch = _torch()
    return torch.from_numpy((gain * rng.standard_normal(shape) + shift).astype(np.float32)).cuda().to(getattr(torch, dtype))


def laid_out(x, layout, spare=0):
    """x [B, H, N, D] in another memory layout, with `spare` more rows of NaN behind the tokens."""
    torch = _torch()
    B, H, N, D = x.shape
    if layout == "packed":
        buf = torch.full((B, H, N + spare, D), float("nan"), dtype=x.dtype, device=x.device)
        view = buf[:, :, :N]
    elif layout == "bnhd":
        buf = torch.full((B, N + spare, H, D), float("nan"), dtype=x.dtype, device=x.device)
        view = buf[:, :N].transpose(1, 2)
    else:
        buf = torch.full((B, N + spare, 3, H, D), float("nan"), dtype=x.dtype, device=x.device)
        view = buf[:, :N, 1].transpose(1, 2)
    view.copy_(x)
    return view, buf


def f64(t):
    return t.double().cpu().numpy()


def assert_near(got, want, dtype, slack, what):
    """|got - want| <= half a step of dtype at want + slack, NaN where want has it."""
    torch = _torch()
    got = f64(got)
    info = torch.finfo(getattr(torch, dtype))
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), what
    allowed = 0.5 * info.eps * np.abs(want) * 1.001 + 0.5 * info.tiny * info.eps + slack
    bad = ~(np.abs(got - want) <= allowed) & ~nan
    worst = np.max(np.where(nan, 0, np.abs(got - want) / allowed)) if want.size else 0.0
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {worst:.2f} of what is allowed"


ROPE_CASES = [
    # B, Hq, Hk, N, D, dims, grid, interleaved, layout
    (1, 2, 2, 1, 64, (32, 16, 16), (1, 1, 1), True, "packed"),
    (2, 3, 1, 3 * 5 * 7 + 4, 64, (24, 20, 20), (3, 5, 7), True, "bnhd"),
    (1, 5, 5, 4 * 6 * 9, 128, (44, 42, 42), (4, 6, 9), True, "fused"),
    (2, 4, 2, 2 * 9 * 11 + 13, 128, (44, 42, 42), (2, 9, 11), False, "bnhd"),
    (1, 1, 3, 257, 64, (32,), (250,), False, "packed"),
    (1, 7, 2, 120, 96, (16, 16), (10, 12), True, "packed"),       # the last 64 channels are copied
    (1, 2, 2, 90, 96, (16, 16), (9, 10), False, "fused"),
    (2, 2, 2, 2 * 3 * 4 * 5, 40, (8, 0, 16, 8), (2, 3, 4, 5), True, "bnhd"),
    (1, 33, 9, 40, 1024, (512, 512), (5, 8), False, "packed"),
]


@pytest.mark.parametrize("B,Hq,Hk,N,D,dims,grid,interleaved,layout", ROPE_CASES)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_grid(lib, B, Hq, Hk, N, D, dims, grid, interleaved, layout, dtype, inverse):
    torch = _torch()
    print(f"rope grid {B} {Hq} {Hk} {N} {D} {dims} {grid} {interleaved} {layout} {dtype} {inverse}", flush=True)
    rng = np.random.default_rng(N + D)
    start = tuple(range(len(grid)))
    lengths = tuple(g + s + 2 for g, s in zip(grid, start))
    rope = lib.RotaryAxes(dims, lengths, theta=500.0, scale=[1.0 + 0.25 * a for a in range(len(dims))], interleaved=interleaved)
    q, k = make(rng, (B, Hq, N, D), dtype), make(rng, (B, Hk, N, D), dtype)
    (qv, _), (kv, _) = laid_out(q, layout), laid_out(k, layout)
    q0, k0 = laid_out(torch.full_like(q, -5.0), layout, spare=2)
    q1, kb = laid_out(torch.full_like(k, -5.0), layout, spare=2)
    got = lib.rope_axes(qv, kv, rope, grid=grid, start=start, q_out=q0, k_out=q1, inverse=inverse)
    assert got[0] is q0 and got[1] is q1
    pos = layer.grid_positions(N, grid, start)
    for x, y in ((q, q0), (k, q1)):
        want = layer.rope(f64(x), pos, dims, lengths, 500.0, rope_scale(dims), interleaved, inverse)
        # the table's rounding and three roundings of products and their sum, of values up to |x| + |y|
        assert_near(y, want, dtype, 4 * U * 2 * np.abs(f64(x)).max(), "rope")
    assert torch.isnan(k0[:, :, N:] if layout == "packed" else k0[:, N:]).all()  # rows behind the tokens are not touched
    # the same bits into new tensors, for q alone, and in place
    new_q, new_k = lib.rope_axes(qv, kv, rope, grid=grid, start=start, inverse=inverse)
    alone, none = lib.rope_axes(qv, None, rope, grid=grid, start=start, inverse=inverse)
    assert none is None and torch.equal(new_q, q0) and torch.equal(new_k, q1) and torch.equal(alone, q0)
    lib.rope_axes(qv, kv, rope, grid=grid, start=start, q_out=qv, k_out=kv, inverse=inverse)
    assert torch.equal(qv, q0) and torch.equal(kv, q1)


def rope_scale(dims):
    return [1.0 + 0.25 * a for a in range(len(dims))]


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("per_batch", [True, False])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_rope_positions(lib, interleaved, per_batch, dtype):
    """Listed positions: any order, negative ones (not turned), ones behind the table (NaN), far ones."""
    torch = _torch()
    rng = np.random.default_rng(5)
    B, H, N, D, dims, lengths = 3, 2, 77, 64, (32, 16, 16), (100000, 9, 12)
    rope = lib.RotaryAxes(dims, lengths, interleaved=interleaved)
    pos = np.stack([rng.integers(-2, m, (B, N)) for m in lengths], -1)
    pos[0, 3, 1] = 9
    pos[1, 0, 0] = 100000
    pos[2, 5, 2] = 2 ** 31 - 1
    pos[2, 6, 0] = -(2 ** 31)
    if not per_batch:
        pos = pos[2]
    x = make(rng, (B, H, N, D), dtype)
    at = torch.from_numpy(pos.astype(np.int32)).cuda()
    got, _ = lib.rope_axes(x, None, rope, positions=at)
    assert_near(got, layer.rope(f64(x), pos, dims, lengths, interleaved=interleaved), dtype, 4 * U * 2 * np.abs(f64(x)).max(), "rope")
    # positions of every second batch entry of a larger tensor
    if per_batch:
        apart = torch.full((2 * B, N, 3), 12345678, dtype=torch.int32, device="cuda")
        apart[::2] = at
        again, _ = lib.rope_axes(x, None, rope, positions=apart[::2])
        assert torch.equal(again.view(torch.int16), got.view(torch.int16))


def test_rope_is_undone_and_is_the_gradients_transpose(lib):
    torch = _torch()
    rng = np.random.default_rng(6)
    rope = lib.RotaryAxes((24, 20, 20), (4, 6, 8))
    x, dy = make(rng, (1, 2, 192, 64), "float32"), make(rng, (1, 2, 192, 64), "float32")
    y, _ = lib.rope_axes(x, None, rope, grid=(4, 6, 8))
    back, dx = lib.rope_axes(y, dy, rope, grid=(4, 6, 8), inverse=True)
    assert (back - x).abs().max() <= 16 * U * x.abs().max()
    a, b = (y.double() * dy.double()).sum().item(), (x.double() * dx.double()).sum().item()
    assert abs(a - b) <= 8 * U * (x.double().abs() * dy.double().abs()).sum().item()


def test_rope_refusals(lib):
    torch = _torch()
    rope = lib.RotaryAxes((32, 16, 16), (4, 4, 4))
    q = torch.zeros((1, 2, 64, 64), dtype=torch.bfloat16, device="cuda")
    bad = [dict(k=q.float()), dict(k=q[:, :, :32]), dict(grid=None), dict(positions=torch.zeros((64, 3), dtype=torch.int32, device="cuda")),
           dict(grid=None, positions=torch.zeros((64, 3), device="cuda")), dict(grid=None, positions=torch.zeros((64, 2), dtype=torch.int32, device="cuda")),
           dict(grid=None, positions=torch.zeros((64, 3), dtype=torch.int32)), dict(q=q.double()), dict(q=q[..., ::2]), dict(q=q[0]),
           dict(q=q.cpu()), dict(q_out=q.float()), dict(k_out=q), dict(grid=(4, 16))]
    for kw in bad:
        args = dict(q=q, k=None, rope=rope, grid=(4, 4, 4))
        args.update(kw)
        with pytest.raises(ValueError):
            lib.rope_axes(**args)
    for kw in (dict(grid=(4, 4, 5)), dict(grid=(4, 4, 4), start=(1, 0, 0)), dict(grid=(2, 4, 4), q=q[:, :, :31])):
        args = dict(q=q, k=None, rope=rope)
        args.update(kw)
        with pytest.raises(lib.CalibattError):
            lib.rope_axes(**args)
    with pytest.raises(lib.CalibattError):
        lib.RotaryAxes((7,), (4,))
    with pytest.raises(ValueError):
        lib.RotaryAxes((8, 8), (4,))
    torch.cuda.synchronize()


# ---- layer norm ---------------------------------------------------------------------------------------------
def norm_slack(x, w, b, h, r):
    """Roundings of the statistics: up to 32 elements in a lane and 8 joins for the mean, as many again for the deviation,
    a square root, a quotient and four products, each 2^-24 of what it is of."""
    return 64 * U * (np.abs(h) + r * np.abs(x).mean(-1, keepdims=True)) * np.abs(w) + 2 * U * np.abs(b)


NORM_SHAPES = [(1, 1), (3, 5), (7, 64), (130, 64), (33, 128), (2, 3, 4, 96), (5, 200), (65, 512), (9, 1000), (3, 1001), (40, 1280),
               (2, 2048), (6, 2056), (3, 4104), (700, 5120), (2, 6152), (2, 7, 8192), (1, 8191)]


@pytest.mark.parametrize("shape", NORM_SHAPES)
@pytest.mark.parametrize("dtype,wtype", [("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float16", "float16"),
                                         ("float16", None), ("float32", "float32"), ("float32", None)])
@pytest.mark.parametrize("center", [True, False])
def test_norm_and_gradients(lib, shape, dtype, wtype, center):
    torch = _torch()
    print(f"norm {shape} {dtype} {wtype} {center}", flush=True)
    rng = np.random.default_rng(shape[-1])
    C, eps = shape[-1], 1e-5
    x, dy = make(rng, shape, dtype, 1.5, 0.7), make(rng, shape, dtype)
    w = None if wtype is None else make(rng, (C,), wtype, 0.3, 1.0)
    b = None if wtype is None else make(rng, (C,), wtype)
    y = lib.layer_norm_fwd(x, w, b, eps=eps, center=center)
    xs, ws, bs = f64(x), 1.0 if w is None else f64(w), 0.0 if b is None else f64(b)
    d = xs - xs.mean(-1, keepdims=True) if center else xs
    r = 1 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    h = d * r
    assert_near(y, layer.layer_norm(xs, ws, bs, eps, center), dtype, norm_slack(xs, ws, bs, h, r), "y")
    dx, dw, db = lib.layer_norm_bwd(dy, x, w, b, eps=eps, center=center)
    want = layer.layer_norm_grads(f64(dy), xs, ws, eps, center)
    g = f64(dy) * ws
    # as many roundings for the two sums of g, of what they are sums of, beside those of h and r
    size = np.abs(g) + np.abs(g).mean(-1, keepdims=True) + (np.abs(h) + r * np.abs(xs).mean(-1, keepdims=True)) * (
        np.abs(g) * (1 + np.abs(h))).mean(-1, keepdims=True)
    assert_near(dx, want[0], dtype, 160 * U * r * (1 + r * np.abs(xs).mean(-1, keepdims=True)) * size, "dx")
    if w is None:
        assert dw is None and db is None
        return
    assert dw.dtype == w.dtype and db.dtype == w.dtype
    rows = tuple(range(len(shape) - 1))
    # a chain of at most 2 rows in a lane, 32 groups, 1024 / 8 shares and 32 slices, and the error of h
    err = 64 * U * (np.abs(f64(dy)) * (np.abs(h) + r * np.abs(xs).mean(-1, keepdims=True))).sum(rows)
    assert_near(dw, want[1], wtype, err + 200 * U * np.abs(f64(dy) * h).sum(rows), "dweight")
    assert_near(db, want[2], wtype, 200 * U * np.abs(f64(dy)).sum(rows), "dbias")
    # without a bias, and in place, the same bits
    dx2, dw2, db2 = lib.layer_norm_bwd(dy.clone(), x, w, None, eps=eps, center=center)
    assert db2 is None and torch.equal(dx2, dx) and torch.equal(dw2, dw)
    into = dy.clone()
    assert lib.layer_norm_bwd(into, x, w, b, eps=eps, center=center, dx=into)[0] is into and torch.equal(into, dx)
    z = x.clone()
    assert lib.layer_norm_fwd(z, w, b, eps=eps, center=center, out=z) is z and torch.equal(z, y)


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("rows,C,dtype", [(6000, 2056, "bfloat16"), (6000, 301, "float32"), (4100, 5120, "float16")])
def test_norm_of_many_long_rows(lib, rows, C, dtype, center):
    """More rows of a workgroup each than workgroups: the sums of one row do not meet those of the next.  Rows of very
    different size, so that a sum of the wrong row would show."""
    torch = _torch()
    rng = np.random.default_rng(rows)
    gain = torch.from_numpy((2.0 ** rng.integers(-6, 7, (rows, 1))).astype(np.float32)).cuda()
    x = (make(rng, (rows, C), "float32") * gain).to(getattr(torch, dtype))
    y = lib.layer_norm_fwd(x, eps=1e-6, center=center)
    xs = f64(x)
    d = xs - xs.mean(-1, keepdims=True) if center else xs
    r = 1 / np.sqrt((d * d).mean(-1, keepdims=True) + 1e-6)
    assert_near(y, d * r, dtype, norm_slack(xs, 1.0, 0.0, d * r, r), "y")
    for _ in range(3):
        assert torch.equal(lib.layer_norm_fwd(x, eps=1e-6, center=center), y)


@pytest.mark.parametrize("layout", ["bnhd", "fused"])
@pytest.mark.parametrize("D", [64, 128, 40])
def test_norm_of_heads_in_other_layouts(lib, layout, D):
    """Rows of strided [B, H, N, D] views: the bits of packed copies (their parameters' sums in another order)."""
    torch = _torch()
    rng = np.random.default_rng(D)
    x, dy = make(rng, (2, 5, 67, D), "bfloat16"), make(rng, (2, 5, 67, D), "bfloat16")
    w, b = make(rng, (D,), "float32"), make(rng, (D,), "float32")
    (xv, _), (dv, _) = laid_out(x, layout, spare=3), laid_out(dy, "bnhd")
    y, buf = laid_out(torch.zeros_like(x), layout, spare=3)
    lib.layer_norm_fwd(xv, w, b, out=y)
    assert torch.equal(y, lib.layer_norm_fwd(x, w, b))
    assert torch.isnan(buf[:, 67:]).all()
    dx, dw, db = lib.layer_norm_bwd(dv, xv, w, b)
    dx0, dw0, db0 = lib.layer_norm_bwd(dy, x, w, b)
    assert torch.equal(dx, dx0)
    size = dy.double().abs().sum((0, 1, 2)).cpu().numpy()
    for a, c, bound in ((dw, dw0, (dy.double().abs() * x.double().abs()).sum((0, 1, 2)).cpu().numpy() * 4 + size), (db, db0, size)):
        assert (np.abs(f64(a) - f64(c)) <= 400 * U * bound).all()
    # [N, H * D] as a view of every second row of [2 N, H * D]
    rows = make(rng, (46, 5 * D), "float16")
    assert torch.equal(lib.layer_norm_fwd(rows[::2]), lib.layer_norm_fwd(rows[::2].contiguous()))
    # a row that is the same for all (a broadcast input)
    one = make(rng, (1, D), "float16")
    assert torch.equal(lib.layer_norm_fwd(one.expand(9, D), out=torch.empty((9, D), dtype=torch.float16, device="cuda")),
                       lib.layer_norm_fwd(one.expand(9, D).contiguous()))


def test_norm_gradient_against_differences(lib):
    """Directional differences of the library's own forward in fp32."""
    torch = _torch()
    rng = np.random.default_rng(8)
    x, w, b, dy = (make(rng, s, "float32") for s in ((6, 48), (48,), (48,), (6, 48)))
    grads = lib.layer_norm_bwd(dy, x, w, b, eps=1e-3)
    step = 2.0 ** -8
    for i in range(3):
        u = make(rng, (x, w, b)[i].shape, "float32")
        up, dn = [x, w, b], [x, w, b]
        up[i], dn[i] = up[i] + step * u, dn[i] - step * u
        f = lambda a: (lib.layer_norm_fwd(*a, eps=1e-3).double() * dy.double()).sum().item()  # noqa: E731
        want = (grads[i].double() * u.double()).sum().item()
        # 2^-16 of third derivatives, and fp32 rounding of the forwards (2^-24 * 300 values) over the step
        assert abs((f(up) - f(dn)) / (2 * step) - want) <= 2e-3 * max(1.0, abs(want))


def test_norm_special_rows(lib):
    """Constant rows (no deviation), huge and tiny ones, rows with an infinity or a NaN: no other row is touched."""
    torch = _torch()
    x = torch.zeros((6, 128), device="cuda")
    x[0] = 3.25
    x[1, ::2], x[1, 1::2] = 2.0 ** 60, -(2.0 ** 60)
    x[2, ::2], x[2, 1::2] = 2.0 ** -60, -(2.0 ** -60)
    x[3, 5] = float("inf")
    x[4, 7] = float("nan")
    x[5] = torch.arange(128, device="cuda")
    y = lib.layer_norm_fwd(x, eps=1e-6)
    assert (y[0] == 0).all()
    assert (y[1].abs() - 1).abs().max() <= 8 * U
    assert y[2].abs().max() < 1e-12
    assert torch.isnan(y[3]).all() and torch.isnan(y[4]).all()
    assert torch.equal(y[5:], lib.layer_norm_fwd(x[5:].contiguous(), eps=1e-6))
    dx, _, _ = lib.layer_norm_bwd(torch.ones_like(x), x, eps=1e-6)
    assert torch.isfinite(dx[[0, 1, 2, 5]]).all()


def test_norm_refusals(lib):
    torch = _torch()
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    w, wide = torch.ones(64, dtype=torch.bfloat16, device="cuda"), torch.ones(64, device="cuda")
    for call in (lambda: lib.layer_norm_fwd(x.double()), lambda: lib.layer_norm_fwd(x.cpu()), lambda: lib.layer_norm_fwd(x, None, w),
                 lambda: lib.layer_norm_fwd(x, w, wide), lambda: lib.layer_norm_fwd(x, w[:32]), lambda: lib.layer_norm_fwd(x, w.half()),
                 lambda: lib.layer_norm_fwd(x, out=x.float()), lambda: lib.layer_norm_fwd(x.t()), lambda: lib.layer_norm_fwd(x, w.cpu()),
                 lambda: lib.layer_norm_bwd(x[:2], x), lambda: lib.layer_norm_bwd(x.float(), x), lambda: lib.layer_norm_bwd(x, x, w, dx=x.float())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(lib.CalibattError):
        lib.layer_norm_fwd(torch.zeros((2, 8200), device="cuda"))
    with pytest.raises(lib.CalibattError):
        lib.layer_norm_fwd(x, eps=-1.0)
    torch.cuda.synchronize()


def test_rows_on_another_stream_and_in_a_graph(lib):
    torch = _torch()
    rng = np.random.default_rng(11)
    x, dy = make(rng, (2, 4, 60, 64), "bfloat16"), make(rng, (2, 4, 60, 64), "bfloat16")
    w, b = make(rng, (64,), "float32"), make(rng, (64,), "float32")
    rope = lib.RotaryAxes((32, 16, 16), (3, 4, 5))

    def step(stream=None):
        y = lib.layer_norm_fwd(x, w, b, stream=stream)
        q, _ = lib.rope_axes(y, None, rope, grid=(3, 4, 5), stream=stream)
        g, _ = lib.rope_axes(dy, None, rope, grid=(3, 4, 5), inverse=True, stream=stream)
        return (q,) + lib.layer_norm_bwd(g, x, w, b, stream=stream)

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    for a, c in zip(got, want):
        assert torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        x.copy_(make(rng, x.shape, "bfloat16"))
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        for a, c in zip(held, eager):
            assert torch.equal(a, c), i
