"""CPU tests of the calls around the attention: tables of rotary positions, refusals that the host makes before anything
is launched, and the oracle's gradients against differences."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2603_05503_amd as pkg
from oracle import layer
from paper_2603_05503_amd.layer_ops import _CRope, _CRopePlace

SHAPE, NULL, UNSUPPORTED, TOO_SMALL = -2, -1, -3, -7
P = 4096  # stands for a device pointer: aligned, never read by the host


def i32(*x):
    return (C.c_int32 * len(x))(*x)


@pytest.mark.parametrize("dims,lengths,scale", [((8,), (5,), None), ((44, 42, 42), (21, 30, 52), (1.0, 0.5, 2.25)),
                                                ((2, 0, 4, 10), (1, 3, 70000, 9), None)])
def test_rope_table(dims, lengths, scale):
    lib = pkg.load_library()
    n = len(dims)
    sc = None if scale is None else (C.c_double * n)(*scale)
    entries = C.c_int64(-1)
    assert lib.calibatt_rope_table(n, i32(*dims), i32(*lengths), sc, 10000.0, None, 0, C.byref(entries)) == 0
    assert entries.value == sum(d // 2 * m for d, m in zip(dims, lengths))
    got = np.full((entries.value, 2), 7.0, np.float32)
    ptr = got.ctypes.data_as(C.POINTER(C.c_float))
    assert lib.calibatt_rope_table(n, i32(*dims), i32(*lengths), sc, 10000.0, ptr, entries.value - 1, C.byref(entries)) == TOO_SMALL
    assert lib.calibatt_rope_table(n, i32(*dims), i32(*lengths), sc, 10000.0, ptr, entries.value, C.byref(entries)) == 0
    want = []
    for a, (d, m) in enumerate(zip(dims, lengths)):
        f = np.array([10000.0 ** (-2.0 * i / d) for i in range(d // 2)])
        ang = (np.arange(m) * (1.0 if scale is None else scale[a]))[:, None] * f
        want.append(np.stack([np.cos(ang), np.sin(ang)], -1).reshape(-1, 2))
    # half a step of fp32, and the angles' own rounding in 64 bits (70 000 positions: 2^-53 * 7e4)
    assert np.abs(got - np.concatenate(want)).max() <= 2.0 ** -24 + 1e-10


@pytest.mark.parametrize("n,dims,lengths,theta,status", [
    (0, (8,), (4,), 1e4, UNSUPPORTED), (5, (2,) * 5, (1,) * 5, 1e4, UNSUPPORTED), (1, (7,), (4,), 1e4, SHAPE),
    (1, (-2,), (4,), 1e4, SHAPE), (2, (0, 0), (4, 4), 1e4, SHAPE), (1, (8,), (0,), 1e4, SHAPE), (1, (1026,), (4,), 1e4, SHAPE),
    (1, (8,), (4,), 0.0, SHAPE), (1, (8,), (4,), math.nan, SHAPE), (1, (1024,), (1 << 30,), 1e4, SHAPE)])
def test_rope_table_refusals(n, dims, lengths, theta, status):
    entries = C.c_int64(0)
    lib = pkg.load_library()
    assert lib.calibatt_rope_table(n, i32(*dims), i32(*lengths), None, theta, None, 0, C.byref(entries)) == status
    assert lib.calibatt_rope_table(1, None, i32(4), None, 1e4, None, 0, C.byref(entries)) == NULL


def _rope(q=P, qo=P, k=P, ko=P, B=1, Hq=2, Hk=2, N=64, D=64, dims=(32, 16, 16), length=(4, 4, 4), grid=(4, 4, 4), start=(0, 0, 0),
          interleaved=1, positions=None, positions_b=0, sq=None, so=None, dtype=0, table=P):
    pad = lambda x: (C.c_int32 * 4)(*x)  # noqa: E731
    r = _CRope(len(dims), interleaved, pad(dims), pad(length), table)
    place = _CRopePlace(pad(grid), pad(start), positions, positions_b)
    s, o = (None if x is None else (C.c_int64 * 3)(*x) for x in (sq, so))
    return pkg.load_library().calibatt_rope_axes(q, qo, k, ko, B, Hq, Hk, N, D, C.addressof(r), C.addressof(place),
                                                 None if s is None else C.addressof(s), None if o is None else C.addressof(o),
                                                 None, None, dtype, 0, None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), NULL), (dict(qo=None), NULL), (dict(ko=None), NULL), (dict(table=None), NULL),
    (dict(B=0), SHAPE), (dict(N=0), SHAPE), (dict(Hk=0), SHAPE), (dict(B=70000), SHAPE), (dict(Hq=70000), SHAPE),
    (dict(D=60), UNSUPPORTED), (dict(D=2048), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(dims=(32, 30, 16)), SHAPE),
    (dict(dims=(30, 16, 16)), UNSUPPORTED), (dict(dims=(24, 16, 16), interleaved=0), UNSUPPORTED),
    (dict(grid=(5, 4, 4)), SHAPE), (dict(grid=(4, 4, 0)), SHAPE), (dict(start=(1, 0, 0)), SHAPE), (dict(start=(-1, 0, 0)), SHAPE),
    (dict(N=63), SHAPE), (dict(q=P + 8), SHAPE), (dict(ko=P + 2), SHAPE), (dict(table=P + 4), SHAPE),
    (dict(positions=P + 2), SHAPE), (dict(positions=P, positions_b=-3), SHAPE),
    (dict(sq=(8192, 4096, 60)), SHAPE), (dict(sq=(8192, 4096, 56)), SHAPE), (dict(sq=(8192, -4096, 64)), SHAPE),
    (dict(so=(8192, 0, 64)), SHAPE), (dict(B=2, so=(56, 4096, 64)), SHAPE), (dict(N=(1 << 30) + 1), SHAPE), (dict(N=1 << 30, D=1024), SHAPE)])
def test_rope_refusals(kw, status):
    assert _rope(**kw) == status


def _norm(fn, n=(2, 3, 4), C_=64, sy=None, x=P, y=P, dy=P, w=P, b=P, eps=1e-6, dtype=0, wtype=0, dw=P, db=P, ws=P, nbytes=1 << 40):
    lib = pkg.load_library()
    sy = None if sy is None else (C.c_int64 * 3)(*sy)
    if fn == "fwd":
        return lib.calibatt_layer_norm_fwd(x, w, b, y, *n, C_, None, sy, eps, 1, dtype, wtype, None)
    return lib.calibatt_layer_norm_bwd(dy, x, w, y, dw, db, *n, C_, None, None, sy, eps, 1, dtype, wtype, ws, nbytes, None)


@pytest.mark.parametrize("fn", ["fwd", "bwd"])
@pytest.mark.parametrize("kw,status", [
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(n=(0, 3, 4)), SHAPE), (dict(n=(2, 3, -1)), SHAPE), (dict(C_=0), SHAPE),
    (dict(n=(1 << 20, 1 << 20, 1)), SHAPE), (dict(C_=8193), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(wtype=1), UNSUPPORTED),
    (dict(eps=-1.0), SHAPE), (dict(eps=math.nan), SHAPE), (dict(x=P + 1), SHAPE), (dict(w=P + 1), SHAPE), (dict(wtype=2, w=P + 2), SHAPE),
    (dict(sy=(768, 256, 0)), SHAPE), (dict(sy=(768, 63, 256)), SHAPE), (dict(sy=(-1, 256, 64)), SHAPE)])
def test_norm_refusals(fn, kw, status):
    assert _norm(fn, **kw) == status


def test_norm_parameter_refusals():
    assert _norm("fwd", w=None) == NULL                    # a bias without a weight
    assert _norm("bwd", dy=None) == NULL
    assert _norm("bwd", w=None, db=None) == NULL           # dweight without a weight
    assert _norm("bwd", ws=None) == NULL
    n = C.c_int64(0)
    assert pkg.load_library().calibatt_layer_norm_bwd_workspace_bytes(0, C.byref(n)) == SHAPE
    assert pkg.load_library().calibatt_layer_norm_bwd_workspace_bytes(8193, C.byref(n)) == UNSUPPORTED
    assert pkg.load_library().calibatt_layer_norm_bwd_workspace_bytes(8, None) == NULL


@pytest.mark.parametrize("center", [True, False])
def test_oracle_norm_gradient_against_differences(center):
    rng = np.random.default_rng(1)
    x, w, b, dy = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((3, 7))
    f = lambda x, w, b: (layer.layer_norm(x, w, b, 1e-3, center) * dy).sum()  # noqa: E731
    dx, dw, db = layer.layer_norm_grads(dy, x, w, 1e-3, center)
    h = 1e-6
    for got, arg in ((dx, 0), (dw, 1), (db, 2)):
        for i in np.ndindex(got.shape):
            args = [x.copy(), w.copy(), b.copy()]
            args[arg][i] += h
            up = f(*args)
            args[arg][i] -= 2 * h
            assert abs((up - f(*args)) / (2 * h) - got[i]) < 1e-7


def test_oracle_rope_gradient_is_the_inverse():
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((2, 2, 6, 16)), rng.standard_normal((2, 2, 6, 16))
    pos = rng.integers(-1, 9, (2, 6, 3))
    for interleaved in (True, False):
        args = pos, (8, 4, 4), (9, 9, 9), 100.0, (1.0, 0.5, 3.0), interleaved
        y = layer.rope(x, *args)
        assert np.allclose(layer.rope(y, *args, inverse=True), x, atol=1e-13)
        assert abs((y * dy).sum() - (x * layer.rope(dy, *args, inverse=True)).sum()) < 1e-12


# ---- attention in a window: refusals, and sizes of workspaces ------------------------------------------------
def _window(fn="bytes", B=2, Hq=4, Hkv=2, Nq=300, Nk=300, D=64, left=10, right=0, sinks=0, frame=1, offset=0, q_start=None, q=P, k=P,
            v=P, out=2 * P, lse=P, scale=1.0, dtype=0, sq=None, skv=None, so=None, ws=None, nbytes=0):
    from paper_2603_05503_amd.layer_ops import _CWindow

    w = _CWindow(left, right, sinks, frame, offset, q_start, None, None)
    lib = pkg.load_library()
    if fn == "bytes":
        n, back = C.c_int64(-1), C.c_int64(-1)
        st = lib.calibatt_window_attn_workspace_bytes(B, Hq, Hkv, Nq, Nk, D, C.addressof(w), C.byref(n), C.byref(back))
        return st if st else n.value
    arrays = [None if s is None else (C.c_int64 * 3)(*s) for s in (sq, skv, so)]
    return lib.calibatt_window_attn_fwd(q, k, v, out, lse, B, Hq, Hkv, Nq, Nk, D, C.addressof(w), scale,
                                        *(None if a is None else C.addressof(a) for a in arrays), dtype, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), SHAPE), (dict(Hq=3), SHAPE), (dict(Hkv=0), SHAPE), (dict(Nq=0), SHAPE), (dict(Nk=-1), SHAPE), (dict(D=96), UNSUPPORTED),
    (dict(left=-2), SHAPE), (dict(right=-2), SHAPE), (dict(sinks=-1), SHAPE), (dict(frame=0), SHAPE), (dict(offset=-(1 << 30) - 1), SHAPE),
    (dict(q_start=P + 2), SHAPE), (dict(B=1 << 12, Nq=1 << 20), SHAPE), (dict(B=1 << 12, Nk=1 << 19), SHAPE)])
def test_window_size_refusals(kw, status):
    assert _window(**kw) == status
    assert _window("fwd", **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(out=None), NULL), (dict(out=P), SHAPE),
    (dict(scale=math.inf), SHAPE), (dict(scale=math.nan), SHAPE), (dict(dtype=2), UNSUPPORTED), (dict(q=P + 8), SHAPE),
    (dict(lse=P + 2), SHAPE), (dict(sq=(1 << 20, 1 << 14, 60)), SHAPE), (dict(skv=(1 << 20, 1 << 14, 68)), SHAPE),
    (dict(so=(-8, 1 << 14, 64)), SHAPE), (dict(so=(1 << 20, 0, 64)), SHAPE), (dict(so=(0, 1 << 14, 64)), SHAPE),
    (dict(skv=(0, 0, 0xffffffff // 2 // 300 & ~7)), SHAPE), (dict(skv=(0, 0, 1 << 24)), SHAPE), (dict(ws=P, nbytes=0, Nk=4096, left=-1), TOO_SMALL)])
def test_window_forward_refusals(kw, status):
    assert _window("fwd", **kw) == status


def _window_bwd(B=2, Hq=4, Hkv=2, Nq=300, Nk=300, D=64, left=10, frame=1, dout=P, q=2 * P, k=3 * P, v=4 * P, out=5 * P, lse=6 * P,
                dq=7 * P, dk=8 * P, dv=9 * P, scale=1.0, dtype=0, s=(), ws=10 * P, nbytes=1 << 40):
    from paper_2603_05503_amd.layer_ops import _CWindow

    w = _CWindow(left, 0, 0, frame, 0, None, None, None)
    names = ("dout", "q", "kv", "out", "dq", "dkv")
    arrays = {n: (C.c_int64 * 3)(*x) for n, x in dict(s).items()}
    return pkg.load_library().calibatt_window_attn_bwd(
        dout, q, k, v, out, lse, dq, dk, dv, B, Hq, Hkv, Nq, Nk, D, C.addressof(w), scale,
        *(C.addressof(arrays[n]) if n in arrays else None for n in names), dtype, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [({name: None}, NULL) for name in ("dout", "q", "k", "v", "out", "lse", "dq", "dk", "dv", "ws")] + [
    (dict(Hq=3), SHAPE), (dict(Nk=0), SHAPE), (dict(D=96), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(frame=0), SHAPE),
    (dict(scale=math.inf), SHAPE), (dict(dk=9 * P), SHAPE), (dict(dq=8 * P), SHAPE), (dict(dq=2 * P), SHAPE), (dict(dv=4 * P), SHAPE),
    (dict(dk=P), SHAPE), (dict(ws=5 * P), SHAPE), (dict(lse=6 * P + 2), SHAPE), (dict(dv=9 * P + 8), SHAPE), (dict(ws=10 * P + 4), SHAPE),
    (dict(s=(("q", (1 << 20, 1 << 14, 60)),)), SHAPE), (dict(s=(("dout", (1 << 20, 1 << 14, 68)),)), SHAPE),
    (dict(s=(("dq", (1 << 20, 0, 64)),)), SHAPE), (dict(s=(("dkv", (0, 1 << 15, 64)),)), SHAPE),
    (dict(s=(("kv", (0, 0, 0xffffffff // 2 // 300 & ~7)),)), SHAPE), (dict(nbytes=2 * 4 * 300 * 8 - 1), TOO_SMALL)])
def test_window_gradient_refusals(kw, status):
    assert _window_bwd(**kw) == status


def test_a_window_does_not_change():
    w = pkg.Window(3, 1, 2, 5, -7)
    assert (w.left, w.right, w.sinks, w.frame, w.offset) == (3, 1, 2, 5, -7)
    with pytest.raises(AttributeError):
        w.left = 4


def test_window_workspace_follows_the_work():
    assert _window(Nq=32760, Nk=32760, Hq=40, Hkv=40) == 0                       # fills the GPU by itself
    few = _window(B=1, Hq=1, Hkv=1, Nq=128, Nk=32760, left=-1)
    assert few > 0 and few % ((64 + 2) * 4 * 128) == 0 and few // ((64 + 2) * 4 * 128) <= 64
    assert _window(B=1, Hq=8, Hkv=2, Nq=1, Nk=100, left=-1) == 0                 # one short stream: one launch
    assert _window(B=1, Hq=8, Hkv=2, Nq=1, Nk=1 << 20, left=-1) > 0
    assert _window(B=1, Hq=8, Hkv=2, Nq=1, Nk=1 << 20, left=300) == 0            # by what is seen, not by the cache
