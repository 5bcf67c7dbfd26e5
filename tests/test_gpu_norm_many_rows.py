"""GPU tests of layer norm and its gradients where every workgroup takes several rounds of rows: long rows, one to a workgroup,
and short ones, several to a wave.  Rows of very different size, so that a sum of the wrong row would show.

Roundings are counted as in test_gpu_rows.  dweight and dbias: a lane adds up its rows one after the other, at most
ceil(rows / (512 workgroups x groups)) of them, then up to 32 groups of a workgroup, then 16 shares in each of 32 slices and the
32 slices, or up to 64 and 8 (layer_norm_params_kernel)."""
import numpy as np
import pytest

from oracle import layer
from tests.test_gpu_rows import U, assert_near, f64, make, norm_slack

pytestmark = pytest.mark.gpu

SHAPES = [
    # rows, C, type: whole 16-byte pieces in long rows, single elements, short rows of 8, 16 and 64 lanes
    (3000, 2056, "bfloat16"), (2100, 5120, "float16"), (1800, 8192, "float32"), (2500, 301, "float32"), (1500, 1001, "bfloat16"),
    (70000, 64, "bfloat16"), (40000, 128, "bfloat16"), (70000, 40, "float16"), (9000, 512, "bfloat16"), (66000, 33, "bfloat16")]


def uneven(rng, rows, C, dtype):
    torch = __import__("torch")
    gain = torch.from_numpy((2.0 ** rng.integers(-6, 7, (rows, 1))).astype(np.float32)).cuda()
    return (make(rng, (rows, C), "float32") * gain).to(getattr(torch, dtype))


@pytest.mark.parametrize("rows,C,dtype", SHAPES)
@pytest.mark.parametrize("center", [True, False])
def test_forward_and_gradients_of_many_rows(lib, rows, C, dtype, center):
    import torch

    print(f"many rows {rows} {C} {dtype} {center}", flush=True)
    rng = np.random.default_rng(rows + C)
    x, dy = uneven(rng, rows, C, dtype), uneven(rng, rows, C, dtype)
    w, b = make(rng, (C,), "float32", 0.3, 1.0), make(rng, (C,), "float32")
    eps = 1e-6
    xs, gs, ws, bs = f64(x), f64(dy), f64(w), f64(b)
    mean = xs.mean(-1, keepdims=True) if center else 0.0
    r = 1 / np.sqrt(((xs - mean) ** 2).mean(-1, keepdims=True) + eps)
    h, of_x = (xs - mean) * r, r * np.abs(xs).mean(-1, keepdims=True)
    y = lib.layer_norm_fwd(x, w, b, eps=eps, center=center)
    assert_near(y, layer.layer_norm(xs, ws, bs, eps, center), dtype, norm_slack(xs, ws, bs, h, r), "y")
    got = lib.layer_norm_bwd(dy, x, w, b, eps=eps, center=center)
    dx, dw, db = layer.layer_norm_grads(gs, xs, ws, eps, center)
    g = gs * ws
    size = np.abs(g) + np.abs(g).mean(-1, keepdims=True) + (np.abs(h) + of_x) * (np.abs(g) * (1 + np.abs(h))).mean(-1, keepdims=True)
    assert_near(got[0], dx, dtype, 160 * U * r * (1 + of_x) * size, "dx")
    # a lane's rows: without the groups of a workgroup at most rows / 512 + 1, and 32 + 64 + 32 joins
    chain = rows // 512 + 1 + 128
    err = 64 * U * (np.abs(gs) * (np.abs(h) + of_x)).sum(0)
    assert_near(got[1], dw, "float32", err + chain * U * np.abs(gs * h).sum(0), "dweight")
    assert_near(got[2], db, "float32", chain * U * np.abs(gs).sum(0), "dbias")
    for _ in range(3):  # the same bits every time
        assert torch.equal(lib.layer_norm_fwd(x, w, b, eps=eps, center=center), y)
        assert all(torch.equal(a, c) for a, c in zip(lib.layer_norm_bwd(dy, x, w, b, eps=eps, center=center), got))
    # without parameters, and in place of dy
    alone, none, _ = lib.layer_norm_bwd(dy, x, eps=eps, center=center)
    dx1 = layer.layer_norm_grads(gs, xs, 1.0, eps, center)[0]
    size = np.abs(gs) + np.abs(gs).mean(-1, keepdims=True) + (np.abs(h) + of_x) * (np.abs(gs) * (1 + np.abs(h))).mean(-1, keepdims=True)
    assert none is None
    assert_near(alone, dx1, dtype, 160 * U * r * (1 + of_x) * size, "dx without parameters")
    lib.layer_norm_bwd(dy, x, w, b, eps=eps, center=center, dx=dy)
    assert torch.equal(dy, got[0])
