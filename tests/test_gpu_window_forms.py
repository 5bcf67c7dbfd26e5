"""GPU tests of the forms that calls of attention in a window take, each asked for by name so that a change of the choice
cannot drop one: blocks of 128 queries cut along the keys and whole, blocks of 32, shared rows; joins of few and of many rows;
gradients whose queries and keys are cut.  Bounds as in test_gpu_window."""
import ctypes as C
import math

import numpy as np
import pytest

from tests.test_gpu_window import check_forward, check_grads, make, visible

pytestmark = pytest.mark.gpu

FORMS = ("WINDOW_BLOCKS_128", "WINDOW_BLOCKS_32", "WINDOW_SHARED_ROWS")
ALL = None

# form, cut, B, Hq, Hkv, Nq, Nk, D, window, start, q_len, k_len
CUT = [
    (0, True, 1, 4, 4, 3000, 3000, 128, dict(left=-1, right=0, sinks=0, frame=1), ALL, ALL, ALL),
    (0, True, 1, 16, 8, 1024, 8192, 64, dict(left=-1, right=0, sinks=5, frame=1, offset=7168), ALL, ALL, ALL),
    # padded batches: an empty one, rows that see nothing, parts without a visible key
    (0, True, 3, 4, 2, 700, 4000, 128, dict(left=1500, right=0, sinks=40, frame=1), [3300, 100, -300], [700, 513, 650], [4000, 613, 250]),
    (0, True, 4, 4, 2, 1100, 3000, 64, dict(left=-1, right=1, sinks=0, frame=130), [1900, 0, 700, -600], [1100, 0, 1001, 1100], [3000, 0, 1701, 333]),
    (0, True, 1, 9, 3, 1027, 1027, 128, dict(left=-1, right=-1, sinks=3, frame=1), ALL, ALL, ALL),
    (1, True, 1, 4, 2, 300, 2000, 128, dict(left=-1, right=0, sinks=0, frame=1, offset=1700), ALL, ALL, ALL),
    (1, True, 2, 4, 4, 280, 1900, 64, dict(left=1200, right=0, sinks=9, frame=1), [1620, 300], [280, 117], [1900, 417]),
    (2, True, 70, 8, 1, 1, 3000, 64, dict(left=-1, right=0, sinks=0, frame=1), "last", ALL, "uneven"),  # 560 rows to join
    (2, True, 2, 8, 1, 4, 3001, 128, dict(left=1000, right=0, sinks=700, frame=1, offset=2997), ALL, ALL, ALL),
]
WHOLE = [
    (0, False, 2, 20, 10, 700, 500, 128, dict(left=60, right=9, sinks=3, frame=1), [0, -150], ALL, [500, 377]),
    (0, False, 1, 40, 40, 600, 600, 64, dict(left=1, right=0, sinks=50, frame=50), ALL, ALL, ALL),
    (1, False, 1, 4, 2, 200, 500, 128, dict(left=300, right=0, sinks=0, frame=1, offset=300), ALL, ALL, ALL),
    (2, False, 3, 8, 2, 3, 400, 64, dict(left=100, right=0, sinks=8, frame=1), [397, 20, 0], [3, 1, 0], [400, 21, 0]),
]


def lengths_of(B, Nq, Nk, start, q_len, k_len, c):
    if k_len == "uneven":
        k_len = [Nk - 41 * b for b in range(B)]
    if start == "last":
        start = [n - 1 for n in k_len]
    given = {"q_start": start, "q_len": q_len, "k_len": k_len}
    see = visible(c, B, Nq, Nk, start, q_len, k_len)
    return {name: x for name, x in given.items() if x is not None}, see


@pytest.mark.parametrize("form,cut,B,Hq,Hkv,Nq,Nk,D,c,start,q_len,k_len", CUT + WHOLE)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("workspace", [True, False])
def test_forms_of_the_forward(lib, form, cut, B, Hq, Hkv, Nq, Nk, D, c, start, q_len, k_len, dtype, workspace):
    """With a workspace, and without one, where nothing is cut."""
    import torch

    print(f"form {form} {cut} {B} {Hq} {Hkv} {Nq} {Nk} {D} {c} {dtype} {workspace}", flush=True)
    w = lib.Window(**c)
    f = w.form(B, Hq, Hkv, Nq, Nk, D)
    assert f["forward"] == getattr(lib, FORMS[form]) and (f["forward_parts"] > 1) == cut
    nbytes = w.workspace_bytes(B, Hq, Hkv, Nq, Nk, D)[0]
    assert nbytes == (f["forward_parts"] * B * Hq * Nq * (D + 2) * 4 if cut else 0)
    rng = np.random.default_rng(Nq + Nk + D)
    q, k, v = make(rng, (B, Hq, Nq, D), dtype, 1.5), make(rng, (B, Hkv, Nk, D), dtype, 1.2), make(rng, (B, Hkv, Nk, D), dtype)
    k[:, :, 77::191] *= 3.0  # keys that move a row's reference on the way, and leave parts with different ones
    given, see = lengths_of(B, Nq, Nk, start, q_len, k_len, c)
    at = {name: torch.tensor(x, dtype=torch.int32, device="cuda") for name, x in given.items()}
    scale, out, lse = 1 / math.sqrt(D), torch.full_like(q, 7.0), torch.full((B, Hq, Nq), 7.0, device="cuda")
    if workspace:
        lib.window_attn_fwd(q, k, v, out, w, scale, lse=lse, **at)
    else:
        cw = w._c(*(at.get(n) for n in ("q_start", "q_len", "k_len")), B, q.device)
        st = lib.load_library().calibatt_window_attn_fwd(
            *(t.data_ptr() for t in (q, k, v, out, lse)), B, Hq, Hkv, Nq, Nk, D, C.addressof(cw), scale, None, None, None,
            0 if dtype == "bfloat16" else 1, None, 0, torch.cuda.current_stream().cuda_stream)
        assert st == 0
    if B == 70:  # the oracle on some entries
        some = [0, 1, 33, 69]
        check_forward(out[some], lse[some], q[some], k[some], v[some], see[some], scale, dtype)
    else:
        check_forward(out, lse, q, k, v, see, scale, dtype)


# B, Hq, Hkv, Nq, Nk, D, window, start, q_len, k_len
GRADS = [
    (1, 4, 2, 3000, 3000, 128, dict(left=600, right=0, sinks=20, frame=1), ALL, ALL, ALL),
    (2, 4, 2, 1300, 1500, 128, dict(left=400, right=100, sinks=300, frame=1), [200, 900], [1300, 520], [1500, 1420]),
    (2, 4, 2, 1300, 1500, 64, dict(left=4, right=1, sinks=90, frame=90), [200, -400], [1300, 1111], [1500, 700]),
]


@pytest.mark.parametrize("B,Hq,Hkv,Nq,Nk,D,c,start,q_len,k_len", GRADS)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_forms_of_the_gradients(lib, B, Hq, Hkv, Nq, Nk, D, c, start, q_len, k_len, dtype):
    """Blocks of keys with sinks and without, both cut, beside blocks of queries that are cut."""
    import torch

    print(f"gradients {B} {Hq} {Hkv} {Nq} {Nk} {D} {c} {start} {q_len} {k_len} {dtype}", flush=True)
    w = lib.Window(**c)
    f = w.form(B, Hq, Hkv, Nq, Nk, D)
    assert f["dq_parts"] > 1 and f["dkv_parts"] > 1 and f["sink_parts"] > f["dkv_parts"] and 0 < f["sink_blocks"] < -(-Nk // 256)
    rng = np.random.default_rng(Nq + Nk + D)
    q, k, v, dout = (make(rng, s, dtype) for s in ((B, Hq, Nq, D), (B, Hkv, Nk, D), (B, Hkv, Nk, D), (B, Hq, Nq, D)))
    given, see = lengths_of(B, Nq, Nk, start, q_len, k_len, c)
    at = {name: torch.tensor(x, dtype=torch.int32, device="cuda") for name, x in given.items()}
    out, lse, scale = torch.empty_like(q), torch.empty((B, Hq, Nq), device="cuda"), 1 / math.sqrt(D)
    lib.window_attn_fwd(q, k, v, out, w, scale, lse=lse, **at)
    got = lib.window_attn_bwd(dout, q, k, v, out, lse, w, scale, **at)
    check_grads(got, dout, q, k, v, see, scale, dtype)
    again = lib.window_attn_bwd(dout, q, k, v, out, lse, w, scale, **at)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
