"""GPU tests of small probabilities in fp16, forward: a key that takes the row but has no value, and thousands that share what
is left, each below 2^-14 of it.

Tolerance: half a step (2^-11) of every probability and of the result, and 2^-14 of sum p |v| in fp32, as in test_gpu_window.
Probabilities are kept times 2^7 at least of what they are of the row's largest, so one below 2^-21 of it is off by up to 2^-25
in those units: 2^-32 of sum |v|."""
import numpy as np
import pytest

from oracle import layer
from tests.test_gpu_window import f64, visible

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form,B,Hq,Hkv,Nq,Nk,D", [
    ("WINDOW_SHARED_ROWS", 1, 4, 2, 1, 4096, 64), ("WINDOW_SHARED_ROWS", 2, 8, 1, 3, 9000, 128),
    ("WINDOW_BLOCKS_32", 1, 2, 1, 100, 4096, 64), ("WINDOW_BLOCKS_32", 1, 2, 2, 130, 3000, 128),
    ("WINDOW_BLOCKS_128", 2, 9, 3, 1000, 4096, 64), ("WINDOW_BLOCKS_128", 1, 10, 10, 900, 5000, 128)])
@pytest.mark.parametrize("gap", [12.0, 16.0, 20.0])
def test_many_small_probabilities(lib, form, B, Hq, Hkv, Nq, Nk, D, gap):
    import torch

    print(f"small probabilities {form} {B} {Hq} {Hkv} {Nq} {Nk} {D} {gap}", flush=True)
    w = lib.Window(-1, -1)
    assert w.form(B, Hq, Hkv, Nq, Nk, D)["forward"] == getattr(lib, form)
    rng = np.random.default_rng(Nk)
    scale = 8.0 / D  # logits are 8 times what a key holds in every channel
    x = rng.uniform(-0.05, 0.05, (B, Hkv, Nk, 1))
    x[:, :, 17] = gap / 8.0
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().half()  # noqa: E731
    q, k = to(np.ones((B, Hq, Nq, D))), to(np.broadcast_to(x, (B, Hkv, Nk, D)))
    v = to(1.0 + 0.25 * rng.standard_normal((B, Hkv, Nk, D)))
    v[:, :, 17] = 0.0
    out, lse = torch.empty_like(q), torch.empty((B, Hq, Nq), device="cuda")
    lib.window_attn_fwd(q, k, v, out, w, scale, lse=lse)
    heads = slice(0, Hq // Hkv) if Nq > 200 else slice(0, Hq)  # of many blocks the oracle on one key head
    keys = slice(0, 1) if Nq > 200 else slice(0, Hkv)
    see = visible(dict(left=-1, right=-1, sinks=0, frame=1), B, 1, Nk)
    args = f64(q[:, heads, :1]), f64(k[:, keys]), f64(v[:, keys])  # every query is the same
    want, want_lse = layer.window_attention(*args, see, scale)
    size, _ = layer.window_attention(*args[:2], np.abs(args[2]), see, scale)
    sums = np.repeat(np.abs(args[2]).sum(2, keepdims=True), Hq // Hkv, axis=1)
    allowed = 2.0 ** -11 * 1.01 * (np.abs(want) + size) + 2.0 ** -14 * size + 2.0 ** -32 * sums + 2.0 ** -25
    off = np.abs(f64(out[:, heads]) - want) / allowed
    assert off.max() <= 1.0, f"worst {off.max():.2f} of what is allowed"
    assert np.abs(f64(lse[:, heads]) - want_lse).max() <= 2.0 ** -24 * (2 ** 8 + 4 * gap)
