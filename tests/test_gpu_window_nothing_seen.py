"""GPU tests of the gradients of attention in a window at keys that no query sees and queries that see no key: their rows
hold NaN or infinities, get zeros, and change no other row."""
import math

import numpy as np
import pytest

from tests.test_gpu_window import LENGTHS, check_forward, check_grads, make, visible

pytestmark = pytest.mark.gpu

EVERY = None  # every query and key is there
CASES = [x for x in LENGTHS] + [
    # B, Hq, Hkv, Nq, Nk, D, window, start, q_len, k_len
    (1, 4, 2, 90, 700, 128, dict(left=40, right=0, sinks=3, frame=1), [610], EVERY, EVERY),      # evicted keys behind sinks
    (2, 2, 2, 70, 600, 64, dict(left=1, right=0, sinks=0, frame=32), [0, 500], EVERY, EVERY),    # keys ahead, evicted ones
    (1, 2, 1, 400, 200, 128, dict(left=30, right=0, sinks=0, frame=1), [-100], EVERY, EVERY),    # queries before and behind all keys
    (1, 2, 2, 400, 200, 64, dict(left=3, right=1, sinks=6, frame=16), [-150], EVERY, EVERY),
    (1, 2, 2, 3000, 2900, 128, dict(left=20, right=0, sinks=0, frame=1), [1500], EVERY, EVERY),  # whole blocks of either kind
]


@pytest.mark.parametrize("B,Hq,Hkv,Nq,Nk,D,c,start,q_len,k_len", CASES)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("filling", ["nan", "inf"])
def test_rows_that_meet_nothing(lib, B, Hq, Hkv, Nq, Nk, D, c, start, q_len, k_len, dtype, filling):
    import torch

    print(f"nothing seen {B} {Hq} {Hkv} {Nq} {Nk} {D} {c} {start} {q_len} {k_len} {dtype} {filling}", flush=True)
    rng = np.random.default_rng(B + Nk + D)
    scale, value = 1 / math.sqrt(D), float(filling)
    q, k, v, dout = (make(rng, s, dtype) for s in ((B, Hq, Nq, D), (B, Hkv, Nk, D), (B, Hkv, Nk, D), (B, Hq, Nq, D)))
    q_len, k_len = q_len or [Nq] * B, k_len or [Nk] * B
    see = visible(c, B, Nq, Nk, np.clip(start, -(2 ** 30), 2 ** 30), q_len, k_len)
    qn, kn, vn, dn = q.clone(), k.clone(), v.clone(), dout.clone()
    for b in range(B):
        keys, queries = torch.from_numpy(~see[b].any(0)).cuda(), torch.from_numpy(~see[b].any(1)).cuda()
        kn[b, :, keys], vn[b, :, keys] = value, value
        qn[b, :, queries], dn[b, :, queries] = value, value
    assert not all(see[b].any(0).all() and see[b].any(1).all() for b in range(B))
    at = dict(zip(("q_start", "q_len", "k_len"), (torch.tensor(np.array(x, dtype=np.int64).astype(np.int32), device="cuda")
                                                  for x in (start, q_len, k_len))))
    out, lse, w = torch.empty_like(q), torch.empty((B, Hq, Nq), device="cuda"), lib.Window(**c)
    lib.window_attn_fwd(qn, kn, vn, out, w, scale, lse=lse, **at)
    check_forward(out, lse, q, k, v, see, scale, dtype)
    got = lib.window_attn_bwd(dn, qn, kn, vn, out, lse, w, scale, **at)
    check_grads(got, dout, q, k, v, see, scale, dtype)
    for b in range(B):
        keys, queries = torch.from_numpy(~see[b].any(0)).cuda(), torch.from_numpy(~see[b].any(1)).cuda()
        assert not got[0][b, :, queries].any() and not got[1][b, :, keys].any() and not got[2][b, :, keys].any()
